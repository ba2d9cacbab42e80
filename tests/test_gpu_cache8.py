"""Appending to 8-bit pages (gsrq_paged_append8) and attention over them
(gsrq_attn_paged8) against plain loops in 64 bits.

Appending.  Exponents are those of 64 bits, and codes in front of the new ones
are the old ones rounded again, both exactly.  A new code's number is within
half a step of e4m3 (2^-4 of itself, below the normal codes 2^-10 of the scale)
of the 64-bit one, and of the float32 work before the rounding 2^-19 of
|x| + |y|, as in 16-bit pages.  Attention: tolerances derived in
paged_ref.attention and cache8_ref.attention."""
import math

import pytest

from tests import cache8_ref as C
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


def _raw(x):
    return x.cpu().view(torch.uint8)


# ---------------------------------------------------------------- appending

def _stored(x, pos, theta, norm, eps=1e-6):
    """Rows as they are stored, in 64 bits, and the size that float32 roundings go by."""
    y = R.rms(x.double(), norm, eps)
    mag = y.abs() + y.abs().roll(y.shape[-1] // 2, -1) if norm is not None or theta is not None else torch.zeros_like(y)
    if theta is not None:
        y = torch.stack([R.rope(y[r], int(p), theta) for r, p in enumerate(pos)]) if len(pos) else y
    return y, mag


def _check_append(k, v, q, kp, vp, ke, ve, tab, start, lens, theta=None, kn=None, qn=None, out=None, eps=1e-6):
    """One call on copies of the pages; returns them."""
    pos = torch.zeros(k.shape[0], dtype=torch.long)
    for b in range(len(lens)):
        lo, hi = int(start[b]), int(start[b + 1])
        pos[lo:hi] = int(lens[b]) - (hi - lo) + torch.arange(hi - lo)
    dev = [None if t is None else t.cuda() for t in (k, v, kp, vp, tab, start, lens, q, theta, kn, qn)]
    dke, dve = ke.cuda(), ve.cuda()
    got = B.paged_append(*dev[:7], q=dev[7], theta=dev[8], k_norm=dev[9], q_norm=dev[10], q_out=out, k_exp=dke, v_exp=dve, eps=eps)
    torch.cuda.synchronize()
    worst = 0.0
    for name, rows, norm, turn, before, exp, after, exp_after in (("k", k, kn, theta, kp, ke, dev[2], dke), ("v", v, None, None, vp, ve, dev[3], dve)):
        y, mag = _stored(rows, pos, turn, norm, eps)
        codes, e, want, size, new = C.append(y, mag, before, exp, tab, start, lens)
        assert torch.equal(exp_after.cpu(), e), f"{name}: exponents differ"
        assert torch.equal(_raw(after)[~new], _raw(codes)[~new]), f"{name}: codes of other places differ"
        num = C.numbers(after.cpu(), e)[new]
        scale = (2.0 ** e.double())[:, None, :, None].expand(before.shape)[new]
        ref, top = want[new], 448 * scale
        ref = torch.where(torch.isfinite(ref), torch.maximum(torch.minimum(ref, top), -top), math.nan)
        assert torch.equal(torch.isnan(num), torch.isnan(ref)), f"{name}: NaN in other places"
        tol = 2.0 ** -4 * ref.abs() + 2.0 ** -10 * scale + 2.0 ** -19 * size[new]
        share = ((num - ref).abs() / tol).nan_to_num(0)
        assert not share.numel() or float(share.max()) <= 1.0, f"{name}: {float(share.max()):.3g} of the tolerance"
        worst = max(worst, float(share.max()) if share.numel() else 0.0)
        if norm is None and turn is None:                    # nothing before the rounding: bit for bit
            eb = e.double()[:, None, :, None].expand(before.shape)[new]
            exact = torch.where(torch.isfinite(want[new]), want[new] * 2.0 ** -eb, math.nan).clamp(-448, 448).float().to(C.E4M3)
            x, y8 = exact.view(torch.uint8), _raw(after)[new]
            assert torch.equal(x & 0x7f, y8 & 0x7f) and torch.equal(x[~torch.isnan(ref)], y8[~torch.isnan(ref)])
    if q is not None:
        y, mag = _stored(q, pos, theta, qn, eps)
        behind = int(start[-1])
        rel, sub = R.half_step(got.dtype)
        tol = rel * y.abs() + 2.0 ** -19 * (mag + y.abs()) + sub
        assert torch.all((got.double().cpu() - y).abs()[:behind] <= tol[:behind])
    say("worst share of the tolerance", f"{worst:.3g}")
    return dev[2], dev[3], dke, dve, got


def _rows(counts, Hq, Hkv, hd, dtype, gap=0, seed=0, spread=3.0):
    start, T = R.new_rows(counts, gap)
    g = torch.Generator().manual_seed(seed)
    k, v = ((torch.randn((T, Hkv, hd), generator=g) * spread * torch.exp2(torch.randint(-6, 7, (T, Hkv, 1), generator=g).float())).to(dtype)
            for _ in range(2))
    q = torch.randn((T, Hq, hd), generator=g).to(dtype)
    w = [1 + 0.3 * torch.randn(hd, generator=g) for _ in range(2)]
    return start, k, v, q, w


def _pools(pages, page, Hkv, hd, order):
    (kp, ke), (vp, ve) = C.pool(pages, page, Hkv, hd, order, 1), C.pool(pages, page, Hkv, hd, order, 2)
    return kp, vp, ke, ve


@pytest.mark.parametrize("src,out,counts,lens,Hq,Hkv,hd,page,order,rope,norm,gap", [
    ("f16", "f16", [1], [1], 1, 1, 64, 8, "token", True, False, 0),                    # one token
    ("f16", "f16", [1] * 9, [1, 2, 15, 16, 17, 31, 100, 64, 65], 32, 8, 128, 16, "token", True, False, 0),
    ("bf16", "bf16", [5, 0, 33, 1], [70, 9, 33, 128], 12, 4, 128, 32, "head", True, True, 3),   # rows behind the last
    ("f32", "f16", [7, 40], [7, 41], 16, 16, 64, 8, "token", False, False, 0),
    ("f32", "bf16", [11, 2], [50, 2], 6, 2, 256, 64, "head", True, True, 1),
    ("bf16", "f16", [3, 3], [200, 3], 3, 1, 128, 16, "token", False, True, 0),
    ("f16", "bf16", [130], [130], 7, 1, 64, 128, "token", True, True, 0),
    ("f16", "f16", [150, 33], [333, 40], 3, 3, 128, 128, "token", True, False, 0),     # pages longer than one table of turns
    ("f32", "f16", [70], [100], 2, 2, 256, 256, "head", True, False, 0),
    ("f16", "f16", [1, 2, 3], [40, 41, 42], 40, 40, 64, 16, "token", False, False, 0),
])
def test_append(src, out, counts, lens, Hq, Hkv, hd, page, order, rope, norm, gap):
    say("append8", src, out, counts, lens, Hq, Hkv, hd, page, order)
    per = -(-max(lens) // page)
    pages = len(counts) * per + 2
    start, k, v, q, w = _rows(counts, Hq, Hkv, hd, R.TYPES[src], gap)
    tab, lens = R.table(len(counts), per, pages), torch.tensor(lens, dtype=torch.int32)
    q_out = torch.full(q.shape, 7.0, dtype=R.TYPES[out], device="cuda")
    got = _check_append(k, v, q, *_pools(pages, page, Hkv, hd, order), tab, start, lens, _theta(hd) if rope else None,
                        *(w if norm else (None, None)), out=q_out)[4]
    assert got is q_out and torch.all(q_out[int(start[-1]):] == 7.0)


@pytest.mark.parametrize("dtype,made", [("f16", "f16"), ("bf16", "bf16"), ("f32", "bf16")])
def test_query_types(dtype, made):
    start, k, v, q, _ = _rows([3], 4, 2, 64, R.TYPES[dtype])
    got = _check_append(k, v, q, *_pools(3, 8, 2, 64, "token"), R.table(1, 2, 3), start, torch.tensor([9], dtype=torch.int32))[4]
    assert got.dtype is R.TYPES[made]


def test_a_page_fills_token_by_token():
    """Exponents rise with the tokens, never fall inside a page, and start anew with the next one; every code of the
    page is within what its roundings allow: half a step for each exponent that it has lived through."""
    hd, page, T = 64, 16, 40
    g = torch.Generator().manual_seed(5)
    x = torch.randn((T, 1, hd), generator=g) * torch.exp2((torch.arange(T) % 16 - 8).float())[:, None, None]
    x[20:24] *= 2.0 ** -12                                    # (far below the page's largest)
    kp, vp, ke, ve = (t.cuda() for t in _pools(5, page, 1, hd, "token"))
    tab = torch.tensor([[3, 0, 4]], dtype=torch.int32)
    host = [t.cpu() for t in (kp, vp, ke, ve)]
    for t in range(T):
        host = [y.cpu() for y in _check_append(x[t:t + 1], x[t:t + 1], None, *host, tab, torch.tensor([0, 1], dtype=torch.int32),
                                               torch.tensor([t + 1], dtype=torch.int32))[:4]]
    num = C.numbers(host[0], host[2])
    for t in range(T):
        at = int(tab[0, t // page])
        scale = 2.0 ** float(host[2][at, 0])
        tol = 2.0 ** -4 * x[t, 0].double().abs() + page * 2.0 ** -10 * scale
        assert torch.all((num[at, t % page, 0] - x[t, 0].double()).abs() <= tol), t


def test_infinities_nan_zeros_and_the_ends_of_the_range():
    """Not finite: NaN, and no part of the exponent; zeros: the lowest exponent; sizes below and beyond the range."""
    hd, page = 64, 8
    start, lens = torch.tensor([0, 5], dtype=torch.int32), torch.tensor([5], dtype=torch.int32)
    k, v = (torch.randn((5, 4, hd), generator=torch.Generator().manual_seed(s)) for s in (1, 2))
    k[1, 0, 3], k[2, 0, 40], k[3, 0, 5] = math.inf, -math.inf, math.nan
    k[:, 1] = 0.0
    v[:, 1] = math.nan
    v[:, 2] *= 1e-20
    v[:, 3] *= 1e30
    _check_append(k, v, None, *_pools(3, page, 4, hd, "token"), R.table(1, 2, 3), start, lens)
    _check_append(k, v, None, *_pools(3, page, 4, hd, "head"), R.table(1, 2, 3), start, lens, _theta(hd))


def test_exponents_at_their_borders():
    """Largest sizes of exactly 448 * 2^e and a float32 step to either side, rotated by nothing (position 0), normed to a
    weight, and turned at far positions: the exponent of 64 bits."""
    hd = 64
    one = torch.tensor([0, 1], dtype=torch.int32)
    for top in (448.0, 448.0 * (1 + 2.0 ** -22), 448.0 * (1 - 2.0 ** -23), 448.0 * (1 + 2.0 ** -17)):
        x = torch.full((1, 2, hd), top)
        x[0, 0] *= 2.0 ** -9
        for theta in (None, _theta(hd)):
            _check_append(x, x, None, *_pools(2, 8, 2, hd, "token"), R.table(1, 1, 2), one, torch.tensor([1], dtype=torch.int32), theta)
        _check_append(torch.ones((1, 2, hd)), x, None, *_pools(2, 8, 2, hd, "token"), R.table(1, 1, 2), one, torch.tensor([1], dtype=torch.int32),
                      None, torch.full((hd,), top), eps=0.0)
    # turned pairs whose larger element is 448 to within float32
    theta = _theta(hd)
    for n, pos in enumerate((1, 77, 4001)):
        a = pos * theta
        want = torch.full((hd // 2,), 448.0, dtype=torch.float64)
        k = torch.cat([want * torch.cos(a), -want * torch.sin(a)]).float().view(1, 1, hd)
        per = pos // 8 + 1
        _check_append(k, k, None, *_pools(per, 8, 1, hd, "token"), R.table(1, per, per), one, torch.tensor([pos + 1], dtype=torch.int32), theta)


SIZES = (1.0, 2.0 ** 62, 2.0 ** 64, 2.0 ** 100, 2.0 ** 124, 2.0 ** -48, 2.0 ** -52, 2.0 ** -64, 2.0 ** -80, 2.0 ** -110, 2.0 ** -130)


@pytest.mark.parametrize("eps", [0.0, 1e-6, 2.0 ** -104, 2.0 ** 110])
@pytest.mark.parametrize("src,tokens,Hkv,hd,page,rope", [("f32", 33, 3, 64, 64, True), ("bf16", 33, 2, 128, 16, True), ("bf16", 11, 1, 256, 8, False),
                                                         ("f32", 77, 1, 256, 128, True)])
def test_norms_of_rows_whose_squares_leave_float32(src, tokens, Hkv, hd, page, rope, eps):
    """Rows of 2^-130 to 2^124 next to each other, whose sums of squares float32 does not hold: normed like any others."""
    start, k, v, q, w = _rows([tokens], 2 * Hkv, Hkv, hd, torch.float32, spread=1.0)
    size = torch.tensor(SIZES)[torch.arange(tokens) % len(SIZES)][:, None, None]
    k, q = (torch.randn(x.shape, generator=torch.Generator().manual_seed(i)) * size for i, x in enumerate((k, q)))
    per = -(-(tokens + 5) // page)
    _check_append(k.to(R.TYPES[src]), v.to(R.TYPES[src]), q.to(R.TYPES[src]), *_pools(per + 1, page, Hkv, hd, "token"), R.table(1, per, per + 1), start,
                  torch.tensor([tokens + 5], dtype=torch.int32), _theta(hd) if rope else None, *w, eps=eps)


@pytest.mark.parametrize("src,out,counts,lens,Hq,Hkv,hd,page,order", [
    ("bf16", "bf16", [100, 130], [100, 200], 4, 2, 256, 128, "token"),
    ("f16", "f16", [200], [237], 2, 1, 128, 256, "head"),
    ("f32", "f16", [300], [300], 3, 3, 64, 512, "token"),
])
def test_norms_and_turns_in_pages_longer_than_what_is_kept(src, out, counts, lens, Hq, Hkv, hd, page, order):
    """More new tokens in a page than stay in registers, normed and turned; from the page's first token on and from inside it."""
    per = -(-max(lens) // page)
    pages = len(counts) * per + 1
    start, k, v, q, w = _rows(counts, Hq, Hkv, hd, R.TYPES[src])
    q_out = torch.empty(q.shape, dtype=R.TYPES[out], device="cuda")
    _check_append(k, v, q, *_pools(pages, page, Hkv, hd, order), R.table(len(counts), per, pages), start,
                  torch.tensor(lens, dtype=torch.int32), _theta(hd), *w, out=q_out)


def test_exponents_at_their_borders_after_norm_and_turn():
    """Pairs in directions that the turn takes onto an axis: normed
    and turned, the largest is 448 to within float32, or a little to either side."""
    hd = 64
    theta, one = _theta(hd), torch.tensor([0, 1], dtype=torch.int32)
    for pos in (0, 8, 80, 4000):                               # (pages that start anew)
        a = pos * theta
        k = torch.cat([torch.cos(a), -torch.sin(a)]).float().view(1, 1, hd)
        per = pos // 8 + 1
        for step in (0.0, 2.0 ** -23, -(2.0 ** -22), 2.0 ** -18):
            w = torch.full((hd,), 448.0 / math.sqrt(2) * (1 + step))
            got = _check_append(k * 3, k, None, *_pools(per, 8, 1, hd, "token"), R.table(1, per, per), one, torch.tensor([pos + 1], dtype=torch.int32),
                                theta, w, eps=0.0)[2]
            assert int(got[int(R.table(1, per, per)[0, pos // 8]), 0]) in (0, 1)


def test_a_coded_session_into_8_bit_pages():
    """decode() and paged_append(): what a 1-bit cache holds, turned and in 8-bit pages."""
    T, Hkv, hd, page = 300, 2, 128, 16
    g = torch.Generator().manual_seed(3)
    rows = []
    for i in range(2):
        x = torch.randn((T, Hkv * hd), generator=g).half().cuda()
        seeds = torch.stack([torch.randperm(T, generator=g)[:256] for _ in range(Hkv * hd // 8)]).int().numpy()
        r = B.train_stage(x, d=8, K=256, T=3, seed_rows=seeds)
        codes, _ = B.encode(x, r.gain[None], r.shape[None])
        rows.append(B.decode(codes, r.gain[None], r.shape[None], Hkv * hd).view(T, Hkv, hd).cpu())
    assert float(rows[0].abs().max()) > 0
    per = -(-T // page)
    _check_append(*rows, None, *_pools(per + 1, page, Hkv, hd, "token"), R.table(1, per, per + 1), torch.tensor([0, T], dtype=torch.int32),
                  torch.tensor([T], dtype=torch.int32), _theta(hd))


def test_far_positions_strided_rows_and_strided_exponents():
    """Positions near 2^30, k, v, q as slices of one projection's rows, exponents of keys and values side by side."""
    hd, page, Hkv = 64, 1 << 14, 2
    L = (1 << 30) - 3
    per = 1 << 16
    tab = torch.full((1, per), -1, dtype=torch.int32)
    tab[0, (L - 1) // page] = 1
    start, lens = torch.tensor([0, 4], dtype=torch.int32), torch.tensor([L], dtype=torch.int32)
    wide = torch.randn((4, 12, hd), generator=torch.Generator().manual_seed(9))
    k, v, q = wide[:, :2], wide[:, 2:4], wide[:, 4:10]
    kp, vp, ke, ve = _pools(2, page, Hkv, hd, "token")
    both = torch.stack([ke, ve], -1).cuda()
    d = [t.cuda() for t in (kp, vp)]
    w = wide.cuda()
    got = B.paged_append(w[:, :2], w[:, 2:4], *d, tab.cuda(), start.cuda(), lens.cuda(), q=w[:, 4:10], theta=_theta(hd).cuda(),
                         k_exp=both[..., 0], v_exp=both[..., 1])
    ref = _check_append(k, v, q, kp, vp, ke, ve, tab, start, lens, _theta(hd))
    assert torch.equal(_raw(d[0]), _raw(ref[0])) and torch.equal(_raw(d[1]), _raw(ref[1])) and torch.equal(got, ref[4])
    assert torch.equal(both[..., 0], ref[2]) and torch.equal(both[..., 1], ref[3])


def test_positions_that_the_table_does_not_hold():
    """More new tokens than the sequence has, a row past the table's end, absent pages, a sequence of none: what is held
    is written, nothing else."""
    start, k, v, q, _ = _rows([6, 9, 5, 0], 4, 2, 64, torch.float16)
    tab = torch.tensor([[0, 1], [2, 3], [-1, 99], [4, 5]], dtype=torch.int32)
    lens = torch.tensor([2, 20, 12, 9], dtype=torch.int32)
    _check_append(k, v, q, *_pools(6, 8, 2, 64, "token"), tab, start, lens, _theta(64))
    lens = torch.tensor([-3, 2 ** 31 - 1, 0, 0], dtype=torch.int32)
    _check_append(k, v, None, *_pools(6, 8, 2, 64, "token"), tab, start, lens)


def test_queries_in_place_and_another_stream():
    """q_out is q itself, on a stream that is not the current one."""
    start, k, v, q, w = _rows([5, 70], 40, 2, 128, torch.bfloat16)
    tab, lens = R.table(2, 6, 14), torch.tensor([9, 90], dtype=torch.int32)
    pools = _pools(14, 16, 2, 128, "token")
    ref = _check_append(k, v, q, *pools, tab, start, lens, _theta(128), *w)
    dev = [t.cuda() for t in (k, v, pools[0], pools[1], tab, start, lens, q, pools[2], pools[3])]
    theta, kn, qn = _theta(128).cuda(), w[0].cuda(), w[1].cuda()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = B.paged_append(*dev[:7], q=dev[7], q_out=dev[7], theta=theta, k_norm=kn, q_norm=qn, k_exp=dev[8], v_exp=dev[9], stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert got is dev[7] and torch.equal(got, ref[4])
    assert torch.equal(_raw(dev[2]), _raw(ref[0])) and torch.equal(_raw(dev[3]), _raw(ref[1]))


# ---------------------------------------------------------------- attention

ORDER = ("q", "kp", "vp", "ke", "ve", "tab", "start", "lens")


def _case(counts, lens, Hq, Hkv, hd, page, dtype="f16", gap=0, order="token", spread=1.0, seed=0, per=None, exps=(-7, -3)):
    dt = R.TYPES[dtype]
    start, T = R.new_rows(counts, gap)
    per = per or max(1, -(-max(max(lens), 1) // page))
    pages = len(counts) * per + 1
    g = torch.Generator().manual_seed(seed)
    (kp, ke), (vp, ve) = (C.pool(pages, page, Hkv, hd, order, seed + s, exps) for s in (1, 2))
    ve += 3
    return dict(q=(torch.randn((T, Hq, hd), generator=g) * spread).to(dt), kp=kp, vp=vp, ke=ke, ve=ve,
                tab=R.table(len(counts), per, pages, seed), start=start, lens=torch.tensor(lens, dtype=torch.int32))


def _call(c, **kw):
    d = {n: c[n].cuda() for n in ORDER}
    return B.attn_paged(d["q"], d["kp"], d["vp"], d["tab"], d["start"], d["lens"], k_exp=d["ke"], v_exp=d["ve"], lse=True, **kw)


def _same(got, ref, tol, what):
    """`got` within `tol` of `ref`; infinities and NaN in the same places."""
    got = got.double().cpu()
    fine, held = torch.isfinite(ref), ~torch.isnan(ref)
    assert torch.equal(torch.isnan(got), torch.isnan(ref)), f"{what}: NaN in other places"
    assert torch.equal(got[~fine & held], ref[~fine & held]), f"{what}: infinities differ"
    off = (got - ref).abs()[fine]
    share = float((off / tol[fine].clamp(min=1e-300)).max()) if off.numel() else 0.0
    assert share <= 1.0, f"{what}: {share:.3g} of the tolerance"
    return share


def _check(c, window=0, scale=None, **kw):
    scale = scale if scale is not None else c["q"].shape[2] ** -0.5
    ref, z, t_out, t_lse = C.attention(*(c[n] for n in ORDER), scale, window)
    behind = int(c["start"][-1])
    out = torch.full(c["q"].shape, 5.0, dtype=c["q"].dtype, device="cuda")
    got, lse = _call(c, scale=scale, window=window, out=out, **kw)
    torch.cuda.synchronize()
    assert got is out and torch.all(out[behind:] == 5.0)
    say("shares of the tolerance", f"{_same(got[:behind], ref[:behind], t_out[:behind], 'out'):.3g}",
        f"{_same(lse[:behind], z[:behind], t_lse[:behind], 'lse'):.3g}")
    return got, lse


@pytest.mark.parametrize("counts,lens,Hq,Hkv,hd,page,dtype,window,gap,order", [
    ([1], [1], 1, 1, 64, 8, "f16", 0, 0, "token"),
    ([1], [1], 4, 1, 128, 16, "bf16", 0, 2, "token"),
    ([1], [63], 4, 1, 128, 16, "f16", 0, 0, "token"),
    ([1], [701], 32, 8, 128, 16, "f16", 0, 0, "token"),
    ([1, 1, 0, 1, 1], [64, 65, 7, 200, 1], 8, 2, 128, 16, "f16", 0, 0, "head"),
    ([1, 1], [3000, 17], 16, 1, 64, 32, "bf16", 0, 0, "token"),
    ([1, 1], [900, 333], 14, 2, 256, 8, "f16", 0, 0, "token"),
    ([1, 1, 2], [555, 1300, 9], 4, 1, 64, 8, "bf16", 0, 0, "head"),            # pages of half a load of rows of 64
    ([5, 3, 9], [400, 3, 10], 6, 2, 128, 8, "bf16", 0, 1, "token"),            # drafts
    ([40], [40], 4, 4, 64, 64, "f16", 0, 0, "head"),                           # a prompt
    ([200, 129], [200, 1029], 8, 2, 128, 16, "f16", 0, 0, "token"),
    ([150], [420], 4, 2, 64, 8, "f16", 0, 0, "head"),
    ([130], [600], 3, 1, 256, 128, "bf16", 0, 0, "token"),
    ([1, 150, 1, 7], [500, 400, 1, 7], 7, 1, 64, 16, "f16", 0, 0, "token"),    # a chunk among single tokens
    ([70, 1], [300, 500], 6, 2, 128, 16, "f16", 33, 0, "token"),               # sliding windows
    ([3, 1], [300, 500], 6, 2, 128, 16, "bf16", 1, 0, "token"),
    ([300], [300], 2, 1, 64, 16, "f16", 100, 0, "head"),
    ([2, 1], [90, 700], 4, 2, 256, 16, "f16", 200, 0, "token"),
])
def test_attention(counts, lens, Hq, Hkv, hd, page, dtype, window, gap, order):
    say("attn_paged8", counts, lens, Hq, Hkv, hd, page, dtype, window)
    _check(_case(counts, lens, Hq, Hkv, hd, page, dtype, gap, order), window)


@pytest.mark.parametrize("counts,lens,hd,dtype", [([9, 1], [700, 1500], 64, "f16"), ([140], [900], 128, "bf16"), ([1], [2500], 256, "f16")])
def test_scales_of_neighbouring_pages_far_apart(counts, lens, hd, dtype):
    """Value exponents from -12 to 12 from page to page, at the ends of their range and beyond: those count as the ends."""
    c = _case(counts, lens, 4, 2, hd, 8, dtype)
    g = torch.Generator().manual_seed(7)
    c["ve"] = torch.randint(-12, 13, c["ve"].shape, generator=g).to(torch.int8)
    c["vp"] = c["vp"].float().clamp(-4, 4).to(C.E4M3)         # (within float16)
    _check(c)
    c["ve"] = torch.where(torch.rand(c["ve"].shape, generator=g) < 0.5, -128, -41).to(torch.int8)
    c["q"] = c["q"].bfloat16()                                # (2^-40 is zero in float16)
    _check(c)
    c["ve"] = torch.where(torch.rand(c["ve"].shape, generator=g) < 0.5, 127, 40).to(torch.int8)
    _check(c)


@pytest.mark.parametrize("hd", [64, 128, 256])
def test_peaked_and_rising_scores(hd):
    """Queries x 6, and key scales that grow along the sequence, so that the maximum in use is raised again and again."""
    c = _case([9, 1], [700, 1500], 4, 2, hd, 16, spread=6.0)
    c["ke"] = torch.linspace(-9, -5, c["ke"].shape[0]).round().to(torch.int8)[:, None].repeat(1, 2)
    _check(c)


def test_rows_that_see_nothing():
    """More new tokens than the sequence has, lengths of zero and below, absent pages; few rows and many."""
    c = _case([6, 4, 3], [2, 0, 40], 4, 2, 128, 8)
    c["tab"][2] = torch.tensor([-1, 1000, -5, 99, -1], dtype=torch.int32)
    got, lse = _check(c)
    assert torch.all(got[:4] == 0) and torch.all(lse[:4] == -math.inf) and torch.all(got[6:] == 0)
    c = _case([200, 150, 90, 3], [40, 0, 130, 9], 4, 2, 64, 16)
    c["lens"][3] = -(2 ** 31)
    c["start"] = c["start"].clone()
    got, lse = _call(c)
    assert torch.all(got[:160] == 0) and torch.all(lse[:160] == -math.inf)
    assert torch.all(got[200:350] == 0) and torch.all(got[440:] == 0) and torch.all(lse[440:] == -math.inf)


def _stale(c):
    """NaN wherever no sequence has a token, and any exponent in pages of nobody."""
    pages, page = c["kp"].shape[:2]
    used = torch.zeros((pages, page), dtype=torch.bool)
    for b in range(len(c["lens"])):
        for t in range(int(c["lens"][b])):
            at = R.page_of(c["tab"], pages, page, b, t)
            if at is not None:
                used[at, t % page] = True
    for i, (name, exp) in enumerate((("kp", "ke"), ("vp", "ve"))):
        raw = c[name].view(torch.uint8)
        raw[~used] = torch.tensor([0x7f, 0xff], dtype=torch.uint8)[(torch.arange(int((~used).sum())) + i) % 2][:, None, None]
        c[exp][~used.any(1)] = 127


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_absent_pages_and_stale_places(dtype):
    """Holes in the table, and NaN in every place that no row sees."""
    c = _case([1, 5, 140], [130, 77, 333], 8, 2, 128, 16, dtype)
    c["tab"][0, 3], c["tab"][1, 0], c["tab"][2, 7] = -1, 10 ** 6, -7
    _stale(c)
    _check(c)
    c = _case([2, 70], [60, 111], 4, 2, 64, 8, dtype)
    _stale(c)
    _check(c, 20)


@pytest.mark.parametrize("window", [0, 40])
@pytest.mark.parametrize("counts,lens,hd,dtype", [([3, 1], [50, 40], 128, "f16"), ([170, 5], [300, 70], 128, "bf16"),
                                                  ([100], [100], 64, "f16"), ([90, 2], [200, 99], 256, "bf16")])
def test_nan_reaches_only_the_rows_that_see_it(counts, lens, hd, dtype, window):
    c = _case(counts, lens, 4, 2, hd, 16, dtype)
    kr, vr = c["kp"].view(torch.uint8), c["vp"].view(torch.uint8)
    for b, L in enumerate(lens):
        for i, t in enumerate((L - 1, L - 2, L - counts[b] // 2 - 1, L // 3)):
            at = int(c["tab"][b, t // 16])
            vr[at, t % 16, i % 2, (7 * i + b) % hd] = (0x7f, 0xff)[i % 2]
            if i == 1:
                kr[at, t % 16, 1, 3] = 0x7f
    _check(c, window)


def test_nan_reaches_a_row_however_small_its_weight():
    """A NaN among values whose weight comes to zero, for few rows and many, in one piece and in several."""
    for counts, lens in (([1], [300]), ([1], [6000]), ([140], [800])):
        c = _case(counts, lens, 4, 1, 64, 16, spread=0.0)
        c["q"][:, :, 0] = 8.0
        kr = c["kp"].view(torch.uint8)
        kr[..., 0] = 0
        t = lens[0] - counts[0] - 1
        at = int(c["tab"][0, t // 16])
        kr[int(c["tab"][0, 0]), 0, 0, 0] = 0x7e                # one token takes all weight
        c["ke"][:] = 0
        c["vp"].view(torch.uint8)[at, t % 16, 0, 7] = 0x7f
        got, _ = _call(c)
        assert torch.all(torch.isnan(got[..., 7])) and torch.all(torch.isfinite(got[..., 8:]))


def test_what_a_row_does_not_see_changes_no_bit():
    """Other codes behind a chunk's rows (not the exponents of their pages): the same bits."""
    c = _case([100], [230], 4, 2, 128, 16)
    a, za = _call(c)
    d = dict(c, kp=c["kp"].clone(), vp=c["vp"].clone())
    for t in range(180, 230):
        at = int(c["tab"][0, t // 16])
        d["kp"].view(torch.uint8)[at, t % 16] ^= 0x2a
        d["vp"].view(torch.uint8)[at, t % 16] = 0x7f
    b, zb = _call(d)
    assert torch.equal(a[:50], b[:50]) and torch.equal(za[:50], zb[:50])


def test_length_past_the_table_scale_and_strides():
    _check(_case([3], [70], 4, 2, 64, 16, per=3))
    c = _case([3, 2], [40, 50], 4, 2, 128, 16)
    c["tab"][1, :2] = c["tab"][0, :2]                          # a shared prompt
    ref, z, t_out, t_lse = C.attention(*(c[n] for n in ORDER), 0.2)
    wide = torch.zeros((5, 8, 128), dtype=torch.float16, device="cuda")
    wide[:, 2:6] = c["q"].cuda()
    both = torch.stack([c["ke"], c["ve"]]).cuda()
    tables = torch.full((2, c["tab"].shape[1] + 5), -9, dtype=torch.int32, device="cuda")
    tables[:, :c["tab"].shape[1]] = c["tab"].cuda()
    got, lse = B.attn_paged(wide[:, 2:6], c["kp"].cuda(), c["vp"].cuda(), tables[:, :c["tab"].shape[1]], c["start"].cuda(), c["lens"].cuda(),
                            scale=0.2, lse=True, k_exp=both[0], v_exp=both[1])
    _same(got, ref, t_out, "out")
    _same(lse, z, t_lse, "lse")


@pytest.mark.parametrize("counts,lens,Hq,Hkv,hd", [([1, 1], [20000, 15001], 8, 2, 128), ([1], [9000], 4, 1, 128), ([40], [20000], 2, 1, 64),
                                                   ([2, 0, 30], [6000, 5, 7000], 3, 1, 256), ([1, 90], [5000, 4500], 2, 1, 128)])
def test_long_contexts_in_many_pieces(counts, lens, Hq, Hkv, hd):
    c = _case(counts, lens, Hq, Hkv, hd, 16)
    _check(c)
    if len(counts) == 2 and counts[0] == 1 and hd == 128 and lens[0] > 10000:
        c["kp"].view(torch.uint8).zero_()                      # uniform weights
        _check(c)


def test_every_head_of_wide_groups():
    """33 and 64 query heads to a key head: more queries of one token than the few rows' kind takes."""
    for Hq in (33, 64):
        _check(_case([1, 2], [300, 77], Hq, 1, 64, 16))


def test_repeatable_other_stream_workspace_and_graph():
    c = _case([1, 60, 1], [3000, 2000, 900], 8, 2, 128, 16)
    d = {n: c[n].cuda() for n in ORDER}
    args = [d[n] for n in ("q", "kp", "vp", "tab", "start", "lens")]
    exps = dict(k_exp=d["ke"], v_exp=d["ve"])
    ref = B.attn_paged(*args, **exps)
    n = B.attn_paged_workspace_bytes(62, 8, *args[1:4])
    ws = torch.empty(max(n, 1), dtype=torch.uint8, device="cuda")
    assert torch.equal(B.attn_paged(*args, workspace=ws, **exps), ref)
    with pytest.raises(ValueError):
        B.attn_paged(*args, workspace=ws[: n // 2], **exps)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = B.attn_paged(*args, stream=side, **exps)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, ref)
    out = torch.empty_like(ref)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.attn_paged(*args, out=out, workspace=ws, **exps)
    for seed in range(3):
        args[0].copy_(torch.randn(args[0].shape, generator=torch.Generator().manual_seed(seed)).half())
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, B.attn_paged(*args, **exps))


def test_large_pools():
    """Pages whose offsets pass 32 bits."""
    hd, page, Hkv = 128, 64, 8
    pages = (1 << 32) // (page * Hkv * hd) + 40
    kp = torch.zeros((pages, page, Hkv, hd), dtype=torch.uint8, device="cuda").view(C.E4M3)
    vp = torch.zeros((pages, page, Hkv, hd), dtype=torch.uint8, device="cuda").view(C.E4M3)
    ke, ve = (torch.zeros((pages, Hkv), dtype=torch.int8, device="cuda") for _ in range(2))
    tab = torch.arange(pages - 5, pages, dtype=torch.int32).view(1, 5)
    small = torch.arange(5, dtype=torch.int32).view(1, 5)
    start, k, v, q, _ = _rows([300], 16, Hkv, hd, torch.float16)
    lens = torch.tensor([300], dtype=torch.int32)
    outs = []
    for t in (tab, small):
        dev = [x.cuda() for x in (k, v)], [x.cuda() for x in (t, start, lens)]
        qo = B.paged_append(*dev[0], kp, vp, *dev[1], q=q.cuda(), theta=_theta(hd).cuda(), k_exp=ke, v_exp=ve)
        outs.append(B.attn_paged(qo, kp, vp, *dev[1], k_exp=ke, v_exp=ve))
    assert torch.equal(outs[0], outs[1]) and torch.equal(ke[-5:], ke[:5]) and torch.equal(_raw(kp[-5:]), _raw(kp[:5]))
    assert torch.all(torch.isfinite(outs[0])) and float(outs[0].abs().max()) > 0
