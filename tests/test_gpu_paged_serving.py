"""The paged cache's operators together, as a serving loop uses them: prompts in
chunks, drafts and single tokens over one cache; a coded session restored and
carried on, beside the decode attention over its codes; captured steps; pools
past 2^31 elements."""
import numpy as np
import pytest

from tests import paged_ref as R
from tests.gpu_util import say

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from paper_2607_01065_amd import gsrq as B  # noqa: E402

BASE = 500000.0


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    B.load_library()


def _theta(hd):
    return BASE ** (torch.arange(hd // 2, dtype=torch.float64) * (-2.0 / hd))


def _share(got, ref, tol):
    got = got.double().cpu()
    assert not torch.isnan(got).any()
    return float(((got - ref).abs() / tol.clamp(min=1e-300)).max())


@pytest.mark.parametrize("dtype,Hq,Hkv,hd,page", [("f16", 8, 2, 128, 16), ("bf16", 4, 4, 64, 8), ("bf16", 6, 2, 256, 32)])
def test_chunks_drafts_and_tokens(dtype, Hq, Hkv, hd, page):
    """Three sequences grow together: prompts in chunks of unequal size, then drafts, then single tokens.  After every
    call the new rows' attention is compared, in 64 bits, over the pages as the calls have left them, and at the end
    the pages with the turned keys."""
    dt = R.TYPES[dtype]
    g = torch.Generator().manual_seed(1)
    steps = [[70, 0, 200], [130, 33, 1], [5, 1, 3], [1, 1, 1], [1, 1, 0]]
    total = [sum(s[b] for s in steps) for b in range(3)]
    per = -(-max(total) // page)
    tab = R.table(3, per, 3 * per + 2)
    kp = torch.full((3 * per + 2, page, Hkv, hd), float("nan"), dtype=dt).cuda()      # nobody may look at these
    vp = torch.full_like(kp, float("inf"))
    theta = _theta(hd)
    w = [1 + 0.2 * torch.randn(hd, generator=g) for _ in range(2)]
    dev = dict(theta=theta.cuda(), k_norm=w[0].cuda(), q_norm=w[1].cuda())
    have = [0, 0, 0]
    for counts in steps:
        start, T = R.new_rows(counts)
        x = torch.randn((T, Hq + 2 * Hkv, hd), generator=g).to(dt)
        q, k, v = x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]
        have = [a + n for a, n in zip(have, counts)]
        lens = torch.tensor(have, dtype=torch.int32)
        before = kp.cpu(), vp.cpu()
        qd, kd, vd, qm, km, vm = R.append(k, v, *before, tab, start, lens, q, theta, *w)
        xd = x.cuda()
        place = (kp, vp, tab.cuda(), start.cuda(), lens.cuda())
        turned = B.paged_append(xd[:, Hq:Hq + Hkv], xd[:, Hq + Hkv:], *place, q=xd[:, :Hq], **dev)
        out, lse = B.attn_paged(turned, *place, lse=True)
        torch.cuda.synchronize()
        rel, sub = R.half_step(dt)
        for name, got, ref, scale in (("q", turned, qd, qm), ("k", kp, kd, km), ("v", vp, vd, vm)):
            got, fine = got.double().cpu(), torch.isfinite(ref)
            off = (got - ref).abs()[fine]
            assert torch.all(off <= (rel * ref.abs() + 2.0 ** -19 * scale + sub)[fine]), name
            assert torch.equal(torch.isfinite(got), fine), name
        ref, z, t_out, t_lse = R.attention(turned.cpu(), kp.cpu(), vp.cpu(), tab, start, lens, hd ** -0.5)
        shares = _share(out, ref, t_out), _share(lse, z, t_lse)
        say(counts, "shares of the tolerance", shares)
        assert max(shares) <= 1.0


def _book(M, G, d, rng):
    gain = np.abs(rng.standard_normal((M, G, 256))).astype(np.float32) * 0.7 ** np.arange(M, dtype=np.float32)[:, None, None]
    shape = rng.standard_normal((M, G, 256, d))
    return gain, (shape / np.linalg.norm(shape, axis=-1, keepdims=True)).astype(np.float32)


@pytest.mark.parametrize("d,M,GQ", [(8, 1, 4), (128, 12, 2)])
def test_coded_session_comes_back(d, M, GQ):
    """A session kept as codes is restored into pages, keys turned; attending to it with one token gives what the decode
    attention over the codes gives, within both calls' own tolerances; then the session goes on with a chunk."""
    import synth
    from tests import attn_bound as AB
    from tests import attn_rq_bound as AQ
    Hkv, hd, lens, cap, page = 2, 128, [900, 333, 1], 900, 16
    if d == 8:
        case = synth.attn_case(3, cap, lens, Hkv, GQ, seed=5, q_dtype="float16")
        bound = AB.reference
    else:
        case = synth.attn_case_rq(3, cap, lens, Hkv, GQ, M, seed=5, q_dtype="float16")
        bound = AQ.reference
    t = {k: torch.from_numpy(np.ascontiguousarray(case[k])).cuda() for k in
         ("k_codes", "v_codes", "lens", "k_gain", "k_shape", "v_gain", "v_shape", "q")}
    Hq = Hkv * GQ
    coded = B.attn_decode(t["k_codes"], t["v_codes"], t["lens"], t["k_gain"], t["k_shape"], t["v_gain"], t["v_shape"], t["q"])
    per = cap // page + 20
    tab = R.table(3, per, 3 * per + 1)
    kp = torch.zeros((3 * per + 1, page, Hkv, hd), dtype=torch.float16, device="cuda")
    vp = torch.zeros_like(kp)
    theta = _theta(hd)
    place = (kp, vp, tab.cuda())
    B.paged_restore(t["k_codes"], t["v_codes"], t["lens"], t["k_gain"], t["k_shape"], t["v_gain"], t["v_shape"], *place,
                    theta=theta.cuda())
    # the decode attention takes the newest token's query before its rotation
    q = case["q"].astype(np.float64)
    turned = torch.stack([R.rope(torch.from_numpy(q[b]), L - 1, theta) for b, L in enumerate(lens)]).half()
    start = torch.arange(4, dtype=torch.int32)
    out = B.attn_paged(turned.cuda(), *place, start.cuda(), t["lens"])
    torch.cuda.synchronize()
    ref, z, t_out, t_lse = R.attention(turned, kp.cpu(), vp.cpu(), tab, start, torch.tensor(lens), hd ** -0.5)
    assert _share(out, ref, t_out) <= 1.0
    # both sides are near the session's attention in 64 bits; the pages' keys and the turned queries are rounded to
    # float16 (2^-11 of each side of every score), the values and the result too
    for b in range(3):
        want, tol = bound(case, b)
        want, tol = torch.from_numpy(want), torch.from_numpy(tol)
        assert torch.all((coded[b].double().cpu() - want).abs() <= tol)
        x, L = turned[b].double(), lens[b]
        at = torch.tensor([R.page_of(tab, kp.shape[0], page, b, i) for i in range(L)])
        i = torch.arange(L)
        K, V = kp.cpu()[at, i % page].double(), vp.cpu()[at, i % page].double()
        for h in range(Hq):
            s = (K[:, h // GQ] @ x[h]) * hd ** -0.5
            p = torch.softmax(s, 0)
            A = p @ V[:, h // GQ].abs()
            e = 2 * 2.0 ** -11 * float((K[:, h // GQ].abs() @ x[h].abs()).max()) * hd ** -0.5
            room = tol[h] + t_out[b, h] + 2 * (np.exp(2 * e) - 1) * A + 2.0 ** -11 * A + 2.0 ** -25
            assert torch.all((out[b, h].double().cpu() - want[h]).abs() <= room)
    # the session goes on
    counts = [40, 3, 150]
    start, T = R.new_rows(counts)
    g = torch.Generator().manual_seed(2)
    x = torch.randn((T, Hq + 2 * Hkv, hd), generator=g).half().cuda()
    longer = torch.tensor([a + n for a, n in zip(lens, counts)], dtype=torch.int32)
    qt = B.paged_append(x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:], *place, start.cuda(), longer.cuda(), q=x[:, :Hq], theta=theta.cuda())
    out = B.attn_paged(qt, *place, start.cuda(), longer.cuda())
    ref, z, t_out, t_lse = R.attention(qt.cpu(), kp.cpu(), vp.cpu(), tab, start, longer, hd ** -0.5)
    assert _share(out, ref, t_out) <= 1.0


def test_captured_steps_share_a_workspace():
    """Two captured steps (append and attention) with one workspace, replayed in turn among eager work."""
    Hq, Hkv, hd, page, Bn = 8, 2, 128, 16, 3
    per = 40
    tab = R.table(Bn, per, Bn * per).cuda()
    theta = _theta(hd).cuda()
    g = torch.Generator().manual_seed(3)

    def state(counts):
        start, T = R.new_rows(counts)
        return dict(kp=torch.randn((Bn * per, page, Hkv, hd), generator=g).half().cuda(),
                    vp=torch.randn((Bn * per, page, Hkv, hd), generator=g).half().cuda(), start=start.cuda(),
                    lens=torch.tensor([600, 333, 40], dtype=torch.int32).cuda(),
                    x=torch.randn((T, Hq + 2 * Hkv, hd), generator=g).half().cuda(),
                    out=torch.empty((T, Hq, hd), dtype=torch.float16, device="cuda"), T=T)

    def step(s, ws, out):
        x = s["x"]
        q = B.paged_append(x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:], s["kp"], s["vp"], tab, s["start"], s["lens"], q=x[:, :Hq],
                           theta=theta)
        return B.attn_paged(q, s["kp"], s["vp"], tab, s["start"], s["lens"], out=out, workspace=ws)

    states = [state([1, 1, 1]), state([50, 1, 40])]
    need = max(B.attn_paged_workspace_bytes(s["T"], Hq, s["kp"], s["vp"], tab) for s in states)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    graphs = []
    for s in states:
        step(s, ws, s["out"])
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step(s, ws, s["out"])
        graphs.append(graph)
    for i in range(4):
        for s in states:
            s["x"].copy_(torch.randn(s["x"].shape, generator=g).half())
            s["lens"].add_(1 if i % 2 else -1)
        for s, graph in zip(states, graphs):
            graph.replay()
        torch.cuda.synchronize()
        for s in states:
            again = step(s, None, torch.empty_like(s["out"]))
            torch.cuda.synchronize()
            assert torch.equal(again, s["out"])


def test_pools_past_32_bit_offsets():
    """Pages at both ends of pools of 2.3e9 elements."""
    Hq, Hkv, hd, page, pages = 8, 8, 256, 16, 70000
    free = torch.cuda.mem_get_info()[0]
    if free < 24 << 30:
        pytest.skip("less than 24 GiB free")
    kp = torch.zeros((pages, page, Hkv, hd), dtype=torch.bfloat16, device="cuda")
    vp = torch.zeros_like(kp)
    used = torch.tensor([[69999, 3, 69001, 65537], [32768, 69998, 0, 65536]], dtype=torch.int32)
    small_tab = torch.arange(8, dtype=torch.int32).view(2, 4)
    g = torch.Generator().manual_seed(4)
    counts, lens = [50, 1], torch.tensor([61, 64], dtype=torch.int32)
    start, T = R.new_rows(counts)
    theta = _theta(hd)
    pools = []
    for pool in (kp, vp):
        x = torch.randn((8, page, Hkv, hd), generator=g).bfloat16()
        pool[used.view(-1).long().cuda()] = x.cuda()
        pools.append(x)
    x = torch.randn((T, Hq + 2 * Hkv, hd), generator=g).bfloat16()
    q, k, v = x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]
    xd = x.cuda()
    place = (kp, vp, used.cuda(), start.cuda(), lens.cuda())
    turned = B.paged_append(xd[:, Hq:Hq + Hkv], xd[:, Hq + Hkv:], *place, q=xd[:, :Hq], theta=theta.cuda())
    out, lse = B.attn_paged(turned, *place, lse=True)
    held = [pool[used.view(-1).long().cuda()].cpu() for pool in (kp, vp)]
    qd, kd, vd, qm, km, vm = R.append(k, v, *pools, small_tab, start, lens, q, theta)
    rel, sub = R.half_step(torch.bfloat16)
    for got, ref, scale in ((held[0], kd, km), (held[1], vd, vm)):
        assert torch.all((got.double() - ref).abs() <= rel * ref.abs() + 2.0 ** -19 * scale + sub)
    ref, z, t_out, t_lse = R.attention(turned.cpu(), *held, small_tab, start, lens, hd ** -0.5)
    assert _share(out, ref, t_out) <= 1.0 and _share(lse, z, t_lse) <= 1.0
    # restoring there: 1-bit codes of zero gain but one codeword
    G = Hkv * hd // 8
    gain = torch.ones((1, G, 256), device="cuda")
    shape = torch.zeros((1, G, 256, 8), device="cuda")
    shape[0, :, 7] = torch.arange(8, device="cuda", dtype=torch.float32)
    codes = torch.full((2, 64, G // 4), 0x07070707, dtype=torch.int32, device="cuda")
    B.paged_restore(codes, codes, lens.cuda(), gain, shape, gain, shape, kp, vp, used.cuda())
    for pool in (kp, vp):
        rows = pool[used.view(-1).long().cuda()].view(2, 64, Hkv, hd // 8, 8)
        for b in range(2):
            assert torch.all(rows[b, : int(lens[b])] == torch.arange(8, device="cuda").bfloat16())
        assert not torch.all(rows[0, 61:] == torch.arange(8, device="cuda").bfloat16())


def test_no_rows_and_odd_starts():
    """No rows: nothing runs.  Starts outside [0, T] or out of order name rows that are not there: they are held inside
    the call's rows, and a proper sequence among them keeps its result."""
    Hq, Hkv, hd, page = 4, 2, 64, 16
    kp = torch.randn((8, page, Hkv, hd)).half().cuda()
    vp = torch.randn((8, page, Hkv, hd)).half().cuda()
    tab = torch.arange(8, dtype=torch.int32).view(2, 4).cuda()
    lens = torch.tensor([60, 50], dtype=torch.int32).cuda()
    none = torch.empty((0, Hq, hd), dtype=torch.float16, device="cuda")
    kv = torch.empty((0, Hkv, hd), dtype=torch.float16, device="cuda")
    start = torch.zeros(3, dtype=torch.int32, device="cuda")
    out, lse = B.attn_paged(none, kp, vp, tab, start, lens, lse=True)
    assert out.shape == (0, Hq, hd) and lse.shape == (0, Hq)
    assert B.paged_append(kv, kv, kp, vp, tab, start, lens, q=none).shape == (0, Hq, hd)
    assert B.paged_append(kv, kv, kp, vp, tab, start, lens) is None
    q = torch.randn((5, Hq, hd)).half().cuda()
    good = B.attn_paged(q, kp, vp, tab, torch.tensor([0, 2, 5], dtype=torch.int32).cuda(), lens)
    odd = B.attn_paged(q, kp, vp, tab, torch.tensor([-3, 2, 9], dtype=torch.int32).cuda(), lens)
    torch.cuda.synchronize()
    assert torch.equal(good, odd)
    B.attn_paged(q, kp, vp, tab, torch.tensor([4, 1, 2], dtype=torch.int32).cuda(), lens)
    kpc = kp.clone()
    B.paged_append(q[:, :Hkv].contiguous(), q[:, :Hkv].contiguous(), kp, vp, tab,
                   torch.tensor([4, 1, 2], dtype=torch.int32).cuda(), lens)
    torch.cuda.synchronize()
    changed = (kp != kpc).flatten(1).any(1)
    assert int(changed.sum()) <= 4


def test_launches_are_timed():
    Hq, Hkv, hd = 4, 2, 64
    kp = torch.randn((8, 16, Hkv, hd)).half().cuda()
    vp = torch.randn((8, 16, Hkv, hd)).half().cuda()
    tab = torch.arange(8, dtype=torch.int32).view(2, 4).cuda()
    lens, start = torch.tensor([60, 50], dtype=torch.int32).cuda(), torch.tensor([0, 1, 2], dtype=torch.int32).cuda()
    x = torch.randn((2, Hkv, hd)).half().cuda()
    q = torch.randn((2, Hq, hd)).half().cuda()
    B.timing_enable(kinds=["append", "attention"])
    B.paged_append(x, x, kp, vp, tab, start, lens)
    B.attn_paged(q, kp, vp, tab, start, lens)
    B.timing_enable(False)
    t = B.timing_read()
    assert t["append"][1] == 1 and t["attention"][1] == 1 and t["append"][0] > 0
