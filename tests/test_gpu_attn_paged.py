"""Attention of new tokens over a paged cache (gsrq_attn_paged) against plain
loops in 64 bits; the tolerances are those derived in paged_ref.attention."""
import pytest

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


def _case(counts, lens, Hq, Hkv, hd, page, dtype="f16", gap=0, order="token", spread=1.0, seed=0, per=None):
    dt = R.TYPES[dtype]
    start, T = R.new_rows(counts, gap)
    per = per or max(1, -(-max(max(lens), 1) // page))
    pages = len(counts) * per + 1
    g = torch.Generator().manual_seed(seed)
    return dict(q=(torch.randn((T, Hq, hd), generator=g) * spread).to(dt), kp=R.pool(pages, page, Hkv, hd, dt, order, seed + 1),
                vp=R.pool(pages, page, Hkv, hd, dt, order, seed + 2), tab=R.table(len(counts), per, pages, seed),
                start=start, lens=torch.tensor(lens, dtype=torch.int32))


ORDER = ("q", "kp", "vp", "tab", "start", "lens")


def _dev(c):
    return [c[n].cuda() for n in ORDER]


def _same(got, ref, tol, what):
    """`got` within `tol` of `ref`; infinities and NaN in the same places."""
    got = got.double().cpu()
    fine = torch.isfinite(ref)
    held = ~torch.isnan(ref)
    assert torch.equal(torch.isnan(got), torch.isnan(ref)), f"{what}: NaN in other places"
    assert torch.equal(got[~fine & held], ref[~fine & held]), f"{what}: infinities differ"
    off = (got - ref).abs()[fine]
    if not off.numel():
        return 0.0
    share = float((off / tol[fine].clamp(min=1e-300)).max())
    assert share <= 1.0, f"{what}: {share:.3g} of the tolerance"
    return share


def _check(c, window=0, scale=None, **kw):
    scale = scale if scale is not None else c["q"].shape[2] ** -0.5
    ref, z, t_out, t_lse = R.attention(*(c[n] for n in ORDER), scale, window)
    T, behind = c["q"].shape[0], int(c["start"][-1])
    out = torch.full(c["q"].shape, 5.0, dtype=c["q"].dtype, device="cuda")
    got, lse = B.attn_paged(*_dev(c), scale=scale, window=window, lse=True, out=out, **kw)
    torch.cuda.synchronize()
    assert got is out and torch.all(out[behind:] == 5.0)
    share = (_same(got[:behind], ref[:behind], t_out[:behind], "out"), _same(lse[:behind], z[:behind], t_lse[:behind], "lse"))
    say("shares of the tolerance", *(f"{x:.3g}" for x in share))
    return got, lse


@pytest.mark.parametrize("counts,lens,Hq,Hkv,hd,page,dtype,window,gap,order", [
    ([1], [1], 1, 1, 64, 8, "f16", 0, 0, "token"),
    ([1], [1], 4, 1, 128, 16, "bf16", 0, 2, "token"),
    ([1], [63], 4, 1, 128, 16, "f16", 0, 0, "token"),
    ([1], [701], 32, 8, 128, 16, "f16", 0, 0, "token"),
    ([1, 1, 0, 1, 1], [64, 65, 7, 200, 1], 8, 2, 128, 16, "f16", 0, 0, "head"),
    ([1, 1], [3000, 17], 16, 1, 64, 32, "bf16", 0, 0, "token"),
    ([1, 1], [900, 333], 14, 2, 256, 8, "f16", 0, 0, "token"),
    ([5, 3, 9], [400, 3, 10], 6, 2, 128, 8, "bf16", 0, 1, "token"),            # drafts
    ([40], [40], 4, 4, 64, 64, "f16", 0, 0, "head"),                           # a prompt
    ([200, 129], [200, 1029], 8, 2, 128, 16, "f16", 0, 0, "token"),
    ([130], [600], 3, 1, 256, 128, "bf16", 0, 0, "token"),
    ([1, 150, 1, 7], [500, 400, 1, 7], 7, 1, 64, 16, "f16", 0, 0, "token"),    # a chunk among single tokens
    ([70, 1], [300, 500], 6, 2, 128, 16, "f16", 33, 0, "token"),               # sliding windows
    ([3, 1], [300, 500], 6, 2, 128, 16, "bf16", 1, 0, "token"),
    ([300], [300], 2, 1, 64, 16, "f16", 100, 0, "head"),
    ([2, 1], [90, 700], 4, 2, 256, 16, "f16", 200, 0, "token"),
])
def test_attention(counts, lens, Hq, Hkv, hd, page, dtype, window, gap, order):
    say("attn_paged", counts, lens, Hq, Hkv, hd, page, dtype, window)
    _check(_case(counts, lens, Hq, Hkv, hd, page, dtype, gap, order), window)


@pytest.mark.parametrize("hd", [64, 128, 256])
def test_peaked_and_rising_scores(hd):
    """Queries x 6, and keys that grow along the sequence, so that the maximum in use is raised again and again."""
    c = _case([9, 1], [700, 1500], 4, 2, hd, 16, spread=6.0)
    c["kp"] *= torch.linspace(0.2, 2.0, c["kp"].shape[0], dtype=torch.float16)[:, None, None, None]
    _check(c)


def test_rows_that_see_nothing():
    """More new tokens than the sequence has, a length of zero, and a sequence whose pages are all absent."""
    c = _case([6, 4, 3], [2, 0, 40], 4, 2, 128, 8)
    c["tab"][2] = torch.tensor([-1, 1000, -5, 99, -1], dtype=torch.int32)
    got, lse = _check(c)
    assert torch.all(got[:4] == 0) and torch.all(lse[:4] == -float("inf"))
    assert torch.all(got[6:] == 0) and torch.all(lse[6:] == -float("inf"))


@pytest.mark.parametrize("hd", [64, 128, 256])
def test_prompts_that_see_nothing(hd):
    """More rows than one workgroup's queries, all or some of them before the first token, and lengths of zero."""
    c = _case([200, 150, 90], [40, 0, 130], 4, 2, hd, 16)
    got, lse = _check(c)
    assert torch.all(got[:160] == 0) and torch.all(lse[:160] == -float("inf"))
    assert torch.all(got[200:350] == 0) and torch.all(lse[200:350] == -float("inf"))


def test_lengths_below_zero():
    """They count as zero, down to the type's lowest, for few rows and for many."""
    c = _case([2, 3, 70, 80, 40], [9, 9, 9, 9, 64], 4, 2, 64, 16)
    ref = _dev(c)
    c["lens"][:4] = torch.tensor([-(2 ** 31), -1, -(2 ** 31), -5], dtype=torch.int32)
    got, lse = B.attn_paged(*_dev(c), lse=True)
    assert torch.all(got[:155] == 0) and torch.all(lse[:155] == -float("inf"))
    want, z = B.attn_paged(*ref, lse=True)
    assert torch.equal(got[155:], want[155:]) and torch.equal(lse[155:], z[155:])


def test_absent_pages_and_stale_places():
    """Holes in the table, and NaN and infinities in every place that no row sees: pages of nobody, places behind
    a sequence's end in its last page."""
    c = _case([1, 5, 140], [130, 77, 333], 8, 2, 128, 16, "bf16")
    c["tab"][0, 3], c["tab"][1, 0], c["tab"][2, 7] = -1, 10 ** 6, -7
    _stale(c)
    _check(c)


@pytest.mark.parametrize("window", [0, 40])
@pytest.mark.parametrize("counts,lens,hd,dtype", [([3, 1], [50, 40], 128, "f16"), ([170, 5], [300, 70], 128, "bf16"),
                                                  ([100], [100], 64, "f16"), ([90, 2], [200, 99], 256, "bf16")])
def test_infinities_reach_only_the_rows_that_see_them(counts, lens, hd, dtype, window):
    """Infinities and NaN in values and keys of tokens in the middle of a chunk: rows before them (and, with a window,
    rows far behind) stay what they were, rows that see them get what the definition gives."""
    c = _case(counts, lens, 4, 2, hd, 16, dtype)
    page = 16
    bad = [float("nan"), float("inf"), -float("inf")]
    for b, L in enumerate(lens):
        for i, t in enumerate((L - 1, L - 2, L - counts[b] // 2 - 1, L // 3)):
            at = int(c["tab"][b, t // page])
            c["vp"][at, t % page, i % 2, (7 * i + b) % hd] = bad[i % 3]
            if i == 1:
                c["kp"][at, t % page, 1, 3] = bad[0]
    _check(c, window)


def _stale(c):
    """NaN and infinities wherever no sequence has a token."""
    pages, page = c["kp"].shape[:2]
    used = torch.zeros((pages, page), dtype=torch.bool)
    for b in range(len(c["lens"])):
        for t in range(int(c["lens"][b])):
            at = R.page_of(c["tab"], pages, page, b, t)
            if at is not None:
                used[at, t % page] = True
    for i, name in enumerate(("kp", "vp")):
        bad = torch.tensor([float("nan"), float("inf"), -float("inf")], dtype=c[name].dtype)
        n = int((~used).sum())
        c[name][~used] = bad[(torch.arange(n) + i) % 3][:, None, None].expand(n, *c[name].shape[2:])


def test_length_past_the_table():
    """A sequence longer than its row of the table: rows sit at their positions and see what is there."""
    _check(_case([3], [70], 4, 2, 64, 16, per=3))


def test_strided_queries_shared_pages_and_scale():
    """q a slice of a projection's rows, two sequences with the same first pages, another scale."""
    c = _case([3, 2], [40, 50], 4, 2, 128, 16)
    c["tab"][1, :2] = c["tab"][0, :2]
    wide = torch.randn((5, 8, 128), generator=torch.Generator().manual_seed(3)).half()
    c["q"] = wide[:, 2:6]
    ref, z, t_out, t_lse = R.attention(*(c[n] for n in ORDER), 0.2)
    got, lse = B.attn_paged(wide.cuda()[:, 2:6], *_dev(c)[1:], scale=0.2, lse=True)
    _same(got, ref, t_out, "out")
    _same(lse, z, t_lse, "lse")


def test_long_context_one_token():
    """One token over 20000, cut into pieces; uniform weights (keys of zeros) give the plain mean of the values."""
    c = _case([1, 1], [20000, 15001], 8, 2, 128, 64, "bf16")
    _check(c)
    c["kp"].zero_()
    _check(c)


@pytest.mark.parametrize("counts,lens,Hq,Hkv,hd", [([1], [9000], 4, 1, 128), ([40], [20000], 2, 1, 64), ([2, 0, 30], [6000, 5, 7000], 3, 1, 256),
                                                   ([1, 90], [5000, 4500], 2, 1, 128)])
def test_many_pieces(counts, lens, Hq, Hkv, hd):
    """So few heads that the keys are cut into more than 32 pieces, for rows of both kinds."""
    _check(_case(counts, lens, Hq, Hkv, hd, 16))


def test_repeatable():
    c = _dev(_case([1, 60, 1], [3000, 2000, 900], 8, 2, 128, 16))
    first = B.attn_paged(*c, lse=True)
    for _ in range(3):
        again = B.attn_paged(*c, lse=True)
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


def test_workspace_other_stream_and_graph():
    """A given workspace, another stream, and a captured call replayed on changed inputs."""
    c = _case([1, 4], [2500, 700], 8, 2, 128, 16)
    args = _dev(c)
    ref = B.attn_paged(*args)
    n = B.attn_paged_workspace_bytes(5, 8, *args[1:4])
    ws = torch.empty(max(n, 1), dtype=torch.uint8, device="cuda")
    assert torch.equal(B.attn_paged(*args, workspace=ws), ref)
    with pytest.raises(ValueError):
        B.attn_paged(*args, workspace=ws[: n // 2])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = B.attn_paged(*args, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, ref)
    out = torch.empty_like(ref)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.attn_paged(*args, out=out, workspace=ws)
    for seed in range(3):
        args[0].copy_(torch.randn(args[0].shape, generator=torch.Generator().manual_seed(seed)).half())
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, B.attn_paged(*args))
