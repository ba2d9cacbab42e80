"""A batch's pages and slots (gsrq_paged_plan) and the verification of drafts
(gsrq_verify_drafts): whole numbers, equal to those of plain loops; and a serving
loop of all of the paged cache's operators over 8-bit pages."""
import random

import pytest

from tests import cache8_ref as C
from tests import paged_ref as R
from tests.gpu_util import say

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from paper_2607_01065_amd import gsrq as B  # noqa: E402


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    B.load_library()


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


# ---------------------------------------------------------------- planning

class Batch:
    """A batch's state on the GPU and, as lists, on the host."""

    def __init__(self, Bn, per, page, F, lens=None, free=None, seed=0):
        self.page, self.rng = page, random.Random(seed)
        pool = list(range(F))
        self.rng.shuffle(pool)
        lens = lens or [0] * Bn
        self.table = [[-1] * per for _ in range(Bn)]
        for b, n in enumerate(lens):
            for i in range(-(-n // page)):
                self.table[b][i] = pool.pop()
        self.count = len(pool) if free is None else free
        self.free = pool + [-1] * (F - len(pool))
        self.lens = list(lens)
        self.dev = [_i32(self.table), _i32(self.free), _i32([self.count]), _i32(self.lens)]

    def step(self, change, rows, **kw):
        self.table, self.free, self.count, self.lens, *out = C.plan(self.table, self.free, self.count, self.lens, change, self.page, rows)
        got = B.paged_plan(*self.dev, _i32(change), page_size=self.page, rows=rows, **kw)
        torch.cuda.synchronize()
        for name, x, ref in zip(("q_start", "slots", "positions"), got, out):
            assert x.tolist() == ref, name
        self.same()
        return got

    def same(self):
        for name, x, ref in zip(("table", "free", "n_free", "seq_len"), self.dev, (self.table, self.free, [self.count], self.lens)):
            assert x.tolist() == ref, name


def test_one_sequence_token_by_token():
    b = Batch(1, 5, 8, 7)
    for _ in range(42):                                    # (past the table's 40 tokens: not served)
        b.step([1], 1)
    b.step([-13], 3)
    b.step([-100], 0)
    assert b.lens == [0] and b.count == 7
    b.step([0], 5)


def test_grow_and_shrink_restores_the_state():
    b = Batch(6, 9, 16, 40, [3, 0, 16, 17, 100, 31])
    before = [x.clone() for x in b.dev]
    b.step([5, 40, 1, 0, 44, 2], 100)
    b.step([-5, -40, -1, 0, -44, -2], 100)
    for x, y in zip(before, b.dev):
        assert torch.equal(x, y)


def test_pages_rows_and_table_rows_that_do_not_suffice():
    """Sequences are served in order as far as the pages and rows go; one that its table row cannot hold asks for nothing."""
    b = Batch(5, 4, 8, 20, [8, 8, 8, 8, 8], free=3)
    b.step([9, 100, 9, 9, 0], 100)                         # two pages, too long, one left: not served
    assert b.lens == [17, 8, 8, 8, 8] and b.count == 1
    b.step([1, 8, 1, 0, 1], 100)                           # no page, one page, none left
    b.step([2, -8, 2, 3, -3], 4)                           # 4 rows: the third is served, the fourth is not
    b.step([2 ** 31 - 1, -(2 ** 31), 2 ** 31 - 1, -1, 1], 50)
    b.step([0, 0, 0, 0, 0], 1)


def test_lists_shorter_than_what_comes_back_and_absent_entries():
    b = Batch(2, 6, 8, 12, [48, 40])
    b.table[0][2] = b.table[1][4] = -1
    b.dev[0] = _i32(b.table)
    b.step([-30, -33], 8)
    b = Batch(2, 6, 8, 12, [48, 40])
    b.free, b.dev[1] = b.free[:4], _i32(b.free[:4])
    b.step([-48, -40], 8)                                  # eleven pages on a list of four
    assert b.count == 4
    for count in (-5, 99):
        b = Batch(1, 3, 8, 6, [0], free=count)
        b.step([20], 20)


@pytest.mark.parametrize("Bn,page,rows", [(1, 8, 40), (3, 16, 300), (64, 8, 5000), (1025, 16, 3000), (8192, 8, 9000)])
def test_random_batches(Bn, page, rows):
    """Growing, shrinking, ending and idle sequences, step after step; more sequences than threads."""
    rng = random.Random(Bn)
    per, F = 12, max(4, Bn * 3)
    lens = [rng.randint(0, 2 * page) for _ in range(Bn)]
    b = Batch(Bn, per, page, F + 2 * Bn, lens, seed=Bn)
    for step in range(6 if Bn < 8000 else 3):
        say("plan", Bn, page, step)
        top = max(2, 2 * rows // Bn)
        b.step([rng.choice([0, 1, 1, rng.randint(1, top), -rng.randint(1, 40), -1000]) for _ in range(Bn)], rows)


def test_large_step_and_given_tensors():
    """100000 rows, a table inside a wider one, results into given tensors, on another stream."""
    b = Batch(100, 130, 8, 13100)
    wide = torch.full((100, 200), 77, dtype=torch.int32, device="cuda")
    wide[:, :130] = b.dev[0]
    b.dev[0] = wide[:, :130]
    out = dict(q_start=torch.empty(101, dtype=torch.int32, device="cuda"), slots=torch.empty(100001, dtype=torch.int64, device="cuda"),
               positions=torch.empty(100001, dtype=torch.int32, device="cuda"))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = b.step([1000] * 100, 100001, stream=side, **out)
    assert all(x is y for x, y in zip(got, out.values())) and torch.all(wide[:, 130:] == 77)


# ------------------------------------------------------------- verification

def _probabilities(T, V, dtype, seed, near=0.5):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((T, V), generator=g) * 2
    p = torch.softmax(x, -1).to(dtype)
    return p, torch.softmax(x + near * torch.randn((T, V), generator=g), -1).to(dtype), g


def _verify(tokens, p, q, u, d, start):
    ref = C.verify(tokens, p, q, u, d, start)
    got = B.verify_drafts(tokens.cuda(), p.cuda(), None if q is None else q.cuda(), u.cuda(), d.cuda(), start.cuda())
    torch.cuda.synchronize()
    assert got[0].tolist() == ref[0].tolist(), "accepted"
    assert got[1].tolist() == ref[1].tolist(), "next"
    return ref


@pytest.mark.parametrize("counts,V,dtype,draft", [
    ([1], 1, "f32", True), ([2], 7, "f32", True), ([5], 1000, "f16", True), ([5, 0, 1, 8], 4097, "bf16", True),
    ([3] * 20, 8191, "f32", True), ([4, 9, 2], 32000, "f16", False), ([4, 9, 2], 4090, "f32", True), ([3, 5], 4096, "bf16", True), ([3, 5], 4097, "f16", True),
    ([6] * 5, 100003, "f32", False), ([7, 3], 300001, "bf16", True),
    ([150, 70], 513, "f32", True), ([1] * 300, 100, "f16", True)])
def test_verify(counts, V, dtype, draft):
    """Ragged drafts; most of what the draft proposes is its own draw, some tokens are unlikely or not in the vocabulary."""
    say("verify", counts[:6], V, dtype, draft)
    start, T = R.new_rows(counts, 2)
    near = 0.02 if max(counts) > 100 else 0.5
    p, q, g = _probabilities(T, V, R.TYPES[dtype], V, near)
    drawn = torch.multinomial((q if draft else p).float(), 1, generator=g)[:, 0]
    tokens = torch.cat([torch.tensor([V + 5]), drawn[:-1]]).to(torch.int32)
    u, d = torch.rand(T, generator=g), torch.rand(len(counts), generator=g)
    if not draft:
        u *= p.float().gather(1, drawn[:, None])[:, 0] * 1.5
    for seed in range(3):
        _verify(tokens, p, q if draft else None, u, d, start)
        u, d = torch.rand(T, generator=g) * (1 if draft else 0.01), torch.rand(len(counts), generator=g)
        tokens[T // 2] = (V, -1, 2 ** 31 - 1)[seed]


def test_draws_at_the_borders_between_tokens():
    """Sixteenths, whose sums are exact: a draw on a border belongs to the token behind it, at 0 to the first of any weight,
    just below 1 and beyond to the last of any weight."""
    short = torch.tensor([[0, 4, 0, 8, 0, 4, 0, 0]]) / 16.0
    want = {0.0: 1, 0.25: 3, 0.25 - 2 ** -20: 1, 0.75: 5, 0.75 - 2 ** -20: 3, 1 - 2 ** -24: 5, 1.0: 5, 7.0: 5, -1.0: 1}
    for spread in (1, 9000):                               # (both ways to sum)
        p = torch.zeros((1, 8 * spread))
        p[0, ::spread] = short[0]
        for draw, token in want.items():
            got = B.verify_drafts(_i32([3]), p.cuda(), None, torch.zeros(1, device="cuda"), torch.tensor([draw], device="cuda"), _i32([0, 1]))
            assert (int(got[0]), int(got[1])) == (0, token * spread), draw


@pytest.mark.parametrize("V", [8, 4096, 4097, 8193, 70000])
def test_acceptance_at_its_border(V):
    """u q = p is a rejection, u q just below p none; q = 0 with p above zero stands, p = 0 never; the rest of a rejection
    where p <= q everywhere is p."""
    p, q = torch.zeros((2, V)), torch.zeros((2, V))
    p[:, 1], p[:, V - 1] = 0.25, 0.75
    q[:, 1], q[:, 5] = 0.5, 0.5
    rows = torch.tensor([0, 2], dtype=torch.int32)
    half = torch.tensor([0.5])
    for token, u, accepted in ((1, 0.5, 0), (1, 0.5 - 2.0 ** -25, 1), (V - 1, 0.999, 1), (5, 0.0, 0), (2, 0.0, 0), (V, 0.0, 0), (-1, 0.0, 0)):
        ref = _verify(torch.tensor([0, token], dtype=torch.int32), p, q, torch.tensor([u, 0.9]), half, rows)
        assert int(ref[0]) == accepted
        _verify(torch.tensor([0, token], dtype=torch.int32), p, None, torch.tensor([u, 0.9]), half, rows)
    ref = _verify(torch.tensor([0, 1], dtype=torch.int32), p, torch.maximum(p, torch.tensor(0.3)), torch.tensor([0.99, 0.0]), half, rows)
    assert int(ref[0]) == 0 and int(ref[1]) == V - 1


@pytest.mark.parametrize("V", [3001, 50001])
def test_weights_of_nothing_nan_and_strided_rows(V):
    p, q, g = _probabilities(6, V, torch.float32, 3)
    p[0], p[1, 7], p[2] = 0.0, float("nan"), float("nan")
    p[3] = -p[3]
    start = torch.tensor([0, 1, 2, 3, 4, 6], dtype=torch.int32)
    tokens, u = torch.zeros(6, dtype=torch.int32), torch.rand(6, generator=g)
    ref = _verify(tokens, p, q, u, torch.rand(5, generator=g), start)
    assert ref[1].tolist()[0] == ref[1].tolist()[2] == ref[1].tolist()[3] == -1
    wide = torch.zeros((6, 2 * V + 3), device="cuda", dtype=torch.float16)
    wide[:, 1:V + 1], wide[:, V + 1:2 * V + 1] = p.half().cuda(), q.half().cuda()       # odd starts and strides
    d = torch.rand(5, generator=g)
    got = B.verify_drafts(tokens.cuda(), wide[:, 1:V + 1], wide[:, V + 1:2 * V + 1], u.cuda(), d.cuda(), start.cuda())
    ref = C.verify(tokens, p.half(), q.half(), u, d, start)
    assert got[0].tolist() == ref[0].tolist() and got[1].tolist() == ref[1].tolist()


def test_rows_more_than_2_31_elements_apart():
    big = torch.zeros((1 << 31) + 2000, dtype=torch.float16, device="cuda")
    p, q, g = _probabilities(3, 700, torch.float16, 5)
    far = [big[i:].as_strided((3, 700), (1 << 30, 1)) for i in (0, 1001)]
    far[0].copy_(p)
    far[1].copy_(q)
    tokens, u, d = torch.tensor([0, 9, 600], dtype=torch.int32), torch.tensor([0.1, 0.9, 0.5]), torch.tensor([0.3, 0.7])
    for start in ([0, 3, 3], [0, 1, 3]):
        start = torch.tensor(start, dtype=torch.int32)
        ref = C.verify(tokens, p, q, u, d, start)
        got = B.verify_drafts(tokens.cuda(), far[0], far[1], u.cuda(), d.cuda(), start.cuda())
        assert got[0].tolist() == ref[0].tolist() and got[1].tolist() == ref[1].tolist()


@pytest.mark.parametrize("V", [4000, 70001])
def test_verify_graph_workspace_and_stream(V):
    start, T = R.new_rows([4, 4, 2])
    p, q, g = _probabilities(T, V, torch.float32, 1)
    tokens = torch.randint(0, V, (T,), generator=g).to(torch.int32)
    dev = [x.cuda() for x in (tokens, p, q, torch.rand(T, generator=g), torch.rand(3, generator=g), start)]
    ws = torch.empty(B.verify_drafts_workspace_bytes(T, V, 3), dtype=torch.uint8, device="cuda")
    assert (ws.numel() > 0) == (V > 4096)
    if ws.numel():
        with pytest.raises(ValueError):
            B.verify_drafts(*dev, workspace=ws[:64])
    out = [torch.empty(3, dtype=torch.int32, device="cuda") for _ in range(2)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.verify_drafts(*dev, accepted=out[0], next_token=out[1], workspace=ws)
    side = torch.cuda.Stream()
    for _ in range(4):
        dev[3].copy_(torch.rand(T, generator=g))
        dev[4].copy_(torch.rand(3, generator=g))
        graph.replay()
        torch.cuda.synchronize()
        ref = C.verify(tokens, p, q, dev[3].cpu(), dev[4].cpu(), start)
        side.wait_stream(torch.cuda.current_stream())
        again = B.verify_drafts(*dev, stream=side)
        torch.cuda.current_stream().wait_stream(side)
        for x, y, z in zip(out, again, ref):
            assert x.tolist() == y.tolist() == z.tolist()


# ---------------------------------------------------------------- together

def test_serving_loop_over_8_bit_pages():
    """Prompts, then steps of drafts: plan, append, attention, verification, and the rejected drafts taken back; every
    step's attention against 64 bits over the pages as they are, every row's numbers in its slot."""
    Hq, Hkv, hd, page, V, drafts = 4, 2, 64, 8, 500, 3
    prompts = [37, 8, 150]
    n = len(prompts)
    b = Batch(n, 30, page, 90)
    kp, vp = (torch.full((90, page, Hkv, hd), 0x7f, dtype=torch.uint8, device="cuda").view(C.E4M3) for _ in range(2))
    ke, ve = (torch.full((90, Hkv), 99, dtype=torch.int8, device="cuda") for _ in range(2))
    theta = 10000.0 ** (torch.arange(hd // 2, dtype=torch.float64, device="cuda") * (-2.0 / hd))
    g = torch.Generator().manual_seed(4)
    change, rows = prompts, sum(prompts)
    for step in range(7):
        say("serving step", step, change)
        start, slots, positions = b.step(change, rows)
        k, v = (torch.randn((rows, Hkv, hd), generator=g).half().cuda() for _ in range(2))
        q = torch.randn((rows, Hq, hd), generator=g).half().cuda()
        tab, lens = b.dev[0], b.dev[3]
        qt = B.paged_append(k, v, kp, vp, tab, start, lens, q=q, theta=theta, k_exp=ke, v_exp=ve)
        stored = C.numbers(vp.cpu(), ve.cpu()).view(-1, Hkv, hd)[slots.cpu()]
        scale = (2.0 ** ve.cpu().double())[slots.cpu() // page][..., None]
        ref = v.cpu().double()
        assert torch.all((stored - ref).abs() <= 2.0 ** -4 * ref.abs() + 2.0 ** -10 * scale)
        out, lse = B.attn_paged(qt, kp, vp, tab, start, lens, lse=True, k_exp=ke, v_exp=ve)
        o, z, t_out, t_lse = C.attention(qt.cpu(), kp.cpu(), vp.cpu(), ke.cpu(), ve.cpu(), tab.cpu(), start.cpu(), lens.cpu(), hd ** -0.5)
        assert torch.all((out.double().cpu() - o).abs() <= t_out) and torch.all((lse.double().cpu() - z).abs() <= t_lse)
        if step:
            p, qp, _ = _probabilities(rows, V, torch.float32, 50 + step)
            tokens = torch.multinomial(qp, 1, generator=g)[:, 0].roll(1).to(torch.int32)
            u, d = torch.rand(rows, generator=g), torch.rand(n, generator=g)
            accepted, token = B.verify_drafts(tokens.cuda(), p.cuda(), qp.cuda(), u.cuda(), d.cuda(), start)
            ref = C.verify(tokens, p, qp, u, d, start.cpu())
            assert accepted.tolist() == ref[0].tolist() and token.tolist() == ref[1].tolist()
            before = list(b.lens)
            b.step((accepted - drafts).tolist(), 0)
            assert b.lens == [x - drafts + a for x, a in zip(before, accepted.tolist())]
        change, rows = [1 + drafts] * n, n * (1 + drafts)


def test_captured_step_is_the_eager_one():
    """A whole step of drafts in one graph, replayed on changing inputs, against eager calls on a copy of the state."""
    Hq, Hkv, hd, page, V, drafts, n = 8, 2, 128, 16, 3001, 2, 4
    rows, F = n * (1 + drafts), 80
    g = torch.Generator().manual_seed(8)

    def state():
        b = Batch(n, 12, page, F, [30, 5, 100, 64])
        (kp, ke), (vp, ve) = C.pool(F, page, Hkv, hd, "token", 1, (-3, -3)), C.pool(F, page, Hkv, hd, "token", 2, (-3, -3))
        return b.dev + [x.cuda() for x in (kp, vp, ke, ve)]

    inputs = dict(k=torch.zeros((rows, Hkv, hd), dtype=torch.float16), v=torch.zeros((rows, Hkv, hd), dtype=torch.float16),
                  q=torch.zeros((rows, Hq, hd), dtype=torch.float16), p=torch.zeros((rows, V)), qp=torch.zeros((rows, V)),
                  u=torch.zeros(rows), d=torch.zeros(n), tokens=torch.zeros(rows, dtype=torch.int32))
    inputs = {name: x.cuda() for name, x in inputs.items()}
    theta = 10000.0 ** (torch.arange(hd // 2, dtype=torch.float64, device="cuda") * (-2.0 / hd))
    grow = _i32([1 + drafts] * n)

    def step(s):
        tab, free, count, lens, kp, vp, ke, ve = s
        start, slots, positions = B.paged_plan(tab, free, count, lens, grow, page_size=page, rows=rows)
        qt = B.paged_append(inputs["k"], inputs["v"], kp, vp, tab, start, lens, q=inputs["q"], theta=theta, k_exp=ke, v_exp=ve)
        out = B.attn_paged(qt, kp, vp, tab, start, lens, k_exp=ke, v_exp=ve)
        accepted, token = B.verify_drafts(inputs["tokens"], inputs["p"], inputs["qp"], inputs["u"], inputs["d"], start)
        back = B.paged_plan(tab, free, count, lens, accepted - drafts, page_size=page, rows=0)
        return [start, slots, positions, qt, out, accepted, token, back[0]]

    def refill():
        for name in ("k", "v", "q"):
            inputs[name].copy_(torch.randn(inputs[name].shape, generator=g).half() * 2)
        x = torch.randn((rows, V), generator=g)
        inputs["p"].copy_(torch.softmax(x, -1))
        inputs["qp"].copy_(torch.softmax(x + 0.3 * torch.randn((rows, V), generator=g), -1))
        inputs["tokens"].copy_(torch.multinomial(inputs["qp"].cpu(), 1, generator=g)[:, 0].roll(1))
        inputs["u"].copy_(torch.rand(rows, generator=g))
        inputs["d"].copy_(torch.rand(n, generator=g))

    eager, held = state(), state()
    refill()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):                          # (warm, on a state that is thrown away)
        step(state())
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = step(held)
    for _ in range(5):
        refill()
        want = step(eager)
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip(captured, want):
            assert torch.equal(x, y)
        for x, y in zip(held, eager):
            assert torch.equal(x.view(torch.uint8) if x.dtype is C.E4M3 else x, y.view(torch.uint8) if y.dtype is C.E4M3 else y)


def test_readme_example_of_8_bit_pages():
    """The block of the README that plans, appends, attends and verifies over 8-bit pages, as it stands there."""
    import os
    import re
    text = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "README.md")).read()
    block = next(b for b in re.findall(r"```python\n(.*?)```", text, re.S) if "verify_drafts" in b)
    n, Hkv, V, counts = 3, 2, 300, [4, 1, 20]
    T = sum(counts)
    g = torch.Generator(device="cuda").manual_seed(7)
    k, v, q = (torch.randn((T, h, 128), generator=g, device="cuda").half() for h in (Hkv, Hkv, 4))
    target, draft = (torch.rand((T, V), generator=g, device="cuda") for _ in range(2))
    names = dict(torch=torch, B=B, n=n, per=4, pages=12, Hkv=Hkv, T=T, new=_i32(counts), k=k, v=v, q=q, target=target, draft=draft,
                 theta=10000.0 ** (torch.arange(64, dtype=torch.float64, device="cuda") * (-2.0 / 128)),
                 tokens=torch.randint(0, V, (T,), generator=g, device="cuda").int(), uniform=torch.rand(T, generator=g, device="cuda"),
                 draw=torch.rand(n, generator=g, device="cuda"))
    exec(block, names)
    torch.cuda.synchronize()
    assert names["out"].shape == (T, 4, 128) and torch.all(torch.isfinite(names["out"]))
    ref = C.verify(names["tokens"].cpu(), target.cpu(), draft.cpu(), names["uniform"].cpu(), names["draw"].cpu(), names["q_start"].cpu())
    assert names["accepted"].tolist() == ref[0].tolist() and names["next_token"].tolist() == ref[1].tolist()
    assert names["seq_len"].tolist() == [1 + a for a in names["accepted"].tolist()]
    assert int(names["n_free"]) == 12 - sum(-(-(1 + a) // 16) for a in names["accepted"].tolist())


def test_readme_step_leaves_sequences_that_were_not_served():
    """The README's step once more, for a sequence that grows, one that asks for more pages than are free and one that brings
    nothing: the lengths, pages and the list of those that got no rows stay as they are."""
    import os
    import re
    text = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "README.md")).read()
    block = next(b for b in re.findall(r"```python\n(.*?)```", text, re.S) if "verify_drafts" in b)
    at = block.index("# `new` [n]")
    n, Hkv, V = 3, 2, 300
    g = torch.Generator(device="cuda").manual_seed(11)
    names = dict(torch=torch, B=B, n=n, per=4, pages=5, Hkv=Hkv, theta=10000.0 ** (torch.arange(64, dtype=torch.float64, device="cuda") * (-2.0 / 128)))
    exec(block[:at], names)

    def step(new):
        T = sum(new)
        k, v, q = (torch.randn((T, h, 128), generator=g, device="cuda").half() for h in (Hkv, Hkv, 4))
        target, draft = (torch.rand((T, V), generator=g, device="cuda") for _ in range(2))
        names.update(T=T, new=_i32(new), k=k, v=v, q=q, target=target, draft=draft, tokens=torch.randint(0, V, (T,), generator=g, device="cuda").int(),
                     uniform=torch.zeros(T, device="cuda"), draw=torch.rand(n, generator=g, device="cuda"))
        exec(block[at:], names)
        return names["accepted"].tolist()

    assert step([4, 18, 9]) == [3, 17, 8]                      # (every draft stands)
    state = [names[x] for x in ("table", "free", "n_free", "seq_len")]
    assert state[3].tolist() == [4, 18, 9] and int(state[2]) == 1
    table = state[0].tolist()
    assert step([3, 40, 0]) == [2, 0, 0]
    assert names["q_start"].tolist() == [0, 3, 3, 3] and names["next_token"].tolist()[1:] == [-1, -1]
    assert state[3].tolist() == [7, 18, 9] and state[0].tolist() == table and int(state[2]) == 1
    assert step([1, 14, 0])[1] == 13 and state[3].tolist() == [8, 32, 9]    # (and it goes on from there)


def test_captured_step_whose_pages_run_short():
    """A step in a graph, replayed until the list is empty, against eager calls on a copy of the state and lists on the host:
    a sequence that was not served keeps its length and pages."""
    n, drafts, V, page, F, per = 4, 3, 500, 8, 14, 12
    rows = n * (1 + drafts)
    g = torch.Generator().manual_seed(2)
    lens = [8, 15, 1, 16]                                  # (6 of 14 pages)
    host, eager = (Batch(n, per, page, F, lens, seed=5) for _ in range(2))
    held = [x.clone() for x in eager.dev]
    p, q = (torch.rand((rows, V), generator=g).cuda() for _ in range(2))
    u, d, grow = torch.zeros(rows, device="cuda"), torch.zeros(n, device="cuda"), _i32([1 + drafts] * n)
    tokens = torch.randint(0, V, (rows,), generator=g).int().cuda()

    def step(s):
        start, slots, positions = B.paged_plan(*s, grow, page_size=page, rows=rows)
        accepted, token = B.verify_drafts(tokens, p, q, u, d, start)
        got = start[1:] - start[:-1]
        B.paged_plan(*s, torch.where(got > 0, accepted - (got - 1), 0), page_size=page, rows=0)
        return [start, slots, positions, accepted, token]

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step([x.clone() for x in held])
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = step(held)
    short = 0
    for _ in range(12):
        u.copy_(torch.rand(rows, generator=g))
        d.copy_(torch.rand(n, generator=g))
        before = list(host.lens)
        want = step(eager.dev)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(captured + held, want + eager.dev))
        host.step([1 + drafts] * n, rows)
        new = [x - y for x, y in zip(host.lens, before)]
        ref = C.verify(tokens.cpu(), p.cpu(), q.cpu(), u.cpu(), d.cpu(), want[0].cpu())
        assert want[3].tolist() == ref[0].tolist() and want[4].tolist() == ref[1].tolist()
        host.step([a - (m - 1) if m else 0 for a, m in zip(ref[0].tolist(), new)], 0)
        assert held[3].tolist() == host.lens and held[0].tolist() == host.table
        short += new.count(0)
    assert short                                           # (the list did run short)
