"""Appending to a paged cache (gsrq_paged_append) and restoring codes into one
(gsrq_paged_restore) against plain loops in 64 bits.

Tolerance of an element that comes out as z = x c - y s (or x alone): half a
step of the pages' type on z, and the float32 work before it.  The norm's
factor: 16 squares in a lane's chain, four additions across lanes, the mean,
eps, the root (which halves the error) and the division: (16 + 4 + 2) / 2 + 2
roundings; two products with it: 2; cosine and sine: at most 4 roundings of
their largest value each with the angle's own (2 pi 2^-26 of a turn rounded to
float32), 6 in all; the rotation: 3.  Together under 32 roundings of 2^-24 of
|x| + |y|: 2^-19.  A plain copy has the half step alone."""
import numpy as np
import pytest

from oracle import gsrq_oracle as O
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


def _close(got, ref, scale, what):
    rel, sub = R.half_step(got.dtype)
    got = got.double().cpu()
    tol = rel * ref.abs() + 2.0 ** -19 * scale + sub
    held = ~torch.isnan(ref)
    off = (got - ref).abs()[held]
    assert torch.all(off <= tol[held]), f"{what}: {float((off / tol[held]).max()):.3g} of the tolerance"
    return float((off / tol[held].clamp(min=1e-300)).max()) if off.numel() else 0.0


def _inputs(counts, Hq, Hkv, hd, dtype, gap=0, seed=0):
    start, T = R.new_rows(counts, gap)
    g = torch.Generator().manual_seed(seed)
    k, v = (torch.randn((T, Hkv, hd), generator=g).mul(3).to(dtype) for _ in range(2))
    q = torch.randn((T, Hq, hd), generator=g).to(dtype)
    w = [1 + 0.3 * torch.randn(hd, generator=g) for _ in range(2)]
    return start, k, v, q, w


@pytest.mark.parametrize("src,held,counts,lens,Hq,Hkv,hd,page,order,rope,norm,gap", [
    ("f16", "f16", [1], [1], 1, 1, 64, 8, "token", True, False, 0),                    # one token
    ("f16", "f16", [1] * 9, [1, 2, 15, 16, 17, 31, 100, 64, 65], 32, 8, 128, 16, "token", True, False, 0),
    ("bf16", "bf16", [5, 0, 33, 1], [70, 9, 33, 128], 12, 4, 128, 32, "head", True, True, 3),   # rows behind the last
    ("f32", "f16", [7, 40], [7, 41], 16, 16, 64, 8, "token", False, False, 0),
    ("f32", "bf16", [11, 2], [50, 2], 6, 2, 256, 64, "head", True, True, 1),
    ("bf16", "f16", [3, 3], [200, 3], 3, 1, 128, 16, "token", False, True, 0),
    ("f16", "bf16", [130], [130], 7, 1, 64, 128, "token", True, True, 0),
])
def test_append(src, held, counts, lens, Hq, Hkv, hd, page, order, rope, norm, gap):
    say("append", src, held, counts, lens, Hq, Hkv, hd, page, order)
    per = -(-max(lens) // page)
    pages = len(counts) * per + 2
    start, k, v, q, w = _inputs(counts, Hq, Hkv, hd, R.TYPES[src], gap)
    kp, vp = (R.pool(pages, page, Hkv, hd, R.TYPES[held], order, s) for s in (1, 2))
    tab, lens = R.table(len(counts), per, pages), torch.tensor(lens, dtype=torch.int32)
    theta = _theta(hd) if rope else None
    kn, qn = w if norm else (None, None)
    qd, kd, vd, qm, km, vm = R.append(k, v, kp, vp, tab, start, lens, q, theta, kn, qn)
    dev = [None if t is None else t.cuda() for t in (k, v, kp, vp, tab, start, lens, q, theta, kn, qn)]
    out = torch.full(q.shape, 7.0, dtype=R.TYPES[held], device="cuda")
    got = B.paged_append(*dev[:7], q=dev[7], theta=dev[8], k_norm=dev[9], q_norm=dev[10], q_out=out)
    assert got is out
    behind = int(start[-1])
    assert torch.all(out[behind:] == 7.0)              # rows of no sequence stay
    touched = km.abs().sum((-1, -2)) > 0
    for x, y in ((dev[2], kp), (dev[3], vp)):          # other places of the pool stay, bit for bit
        assert torch.equal(x.cpu()[~touched], y[~touched])
    say("worst share of the tolerance", _close(got, qd, qm, "q"), _close(dev[2], kd, km, "k"),
        _close(dev[3], vd, vm, "v"))


@pytest.mark.parametrize("eps", [0.0, 1e-6, 2.0 ** -104, 2.0 ** 110])
@pytest.mark.parametrize("src,held,hd,rope", [("f32", "bf16", 64, True), ("bf16", "bf16", 128, True), ("f32", "f16", 256, False)])
def test_append_norms_of_rows_whose_squares_leave_float32(src, held, hd, rope, eps):
    """Rows of 2^-130 to 2^124 next to each other, whose sums of squares float32 does not hold: normed like any others."""
    sizes = torch.tensor((1.0, 2.0 ** 62, 2.0 ** 64, 2.0 ** 100, 2.0 ** 124, 2.0 ** -48, 2.0 ** -52, 2.0 ** -64, 2.0 ** -80, 2.0 ** -110, 2.0 ** -130))
    T, Hkv, Hq, page = 33, 2, 3, 16
    start, k, v, q, w = _inputs([T], Hq, Hkv, hd, torch.float32)
    k, q = ((torch.randn(x.shape, generator=torch.Generator().manual_seed(i)) * sizes[torch.arange(T) % 11][:, None, None]).to(R.TYPES[src])
            for i, x in enumerate((k, q)))
    v = v.to(R.TYPES[src])
    kp, vp = (R.pool(4, page, Hkv, hd, R.TYPES[held], "token", s) for s in (1, 2))
    tab, lens, theta = R.table(1, 3, 4), torch.tensor([T + 5], dtype=torch.int32), _theta(hd) if rope else None
    qd, kd, vd, qm, km, vm = R.append(k, v, kp, vp, tab, start, lens, q, theta, *w, eps=eps)
    dev = [t.cuda() for t in (k, v, kp, vp, tab, start, lens)]
    got = B.paged_append(*dev, q=q.cuda(), theta=None if theta is None else theta.cuda(), k_norm=w[0].cuda(), q_norm=w[1].cuda(), eps=eps)
    say("worst share of the tolerance", _close(got, qd, qm, "q"), _close(dev[2], kd, km, "k"), _close(dev[3], vd, vm, "v"))


def test_append_far_positions_and_strided_rows():
    """Positions near 2^30, and k, v, q as slices of one projection's rows."""
    Hq, Hkv, hd, page, per = 4, 2, 128, 1 << 14, 1 << 16
    start, T = R.new_rows([3])
    g = torch.Generator().manual_seed(5)
    x = torch.randn((T, Hq + 2 * Hkv, hd), generator=g).to(torch.float16)
    q, k, v = x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]
    last = per * page
    lens = torch.tensor([last - 5], dtype=torch.int32)
    tab = torch.full((1, per), -1, dtype=torch.int32)
    tab[0, -1] = 1
    kp, vp = (R.pool(2, page, Hkv, hd, torch.float16, "token", s) for s in (1, 2))
    theta = _theta(hd)
    qd, kd, vd, qm, km, vm = R.append(k, v, kp, vp, tab, start, lens, q, theta)
    xd = x.cuda()
    kc, vc = kp.cuda(), vp.cuda()
    got = B.paged_append(xd[:, Hq:Hq + Hkv], xd[:, Hq + Hkv:], kc, vc, tab.cuda(), start.cuda(), lens.cuda(),
                         q=xd[:, :Hq], theta=theta.cuda())
    _close(got, qd, qm, "q")
    _close(kc, kd, km, "k")
    _close(vc, vd, vm, "v")


def test_append_leaves_out_what_has_no_place():
    """Absent pages, positions before the first and behind the last: nothing is written for them, the queries
    are turned all the same."""
    Hq, Hkv, hd, page = 2, 2, 64, 8
    counts, lens = [6, 6, 12], [3, 36, 24]              # before the first; behind the table's 32; a hole
    start, k, v, q, _ = _inputs(counts, Hq, Hkv, hd, torch.float16)
    tab = torch.tensor([[0, 1, 2, 3], [4, 5, 6, 7], [8, -1, 99, 10]], dtype=torch.int32)
    kp, vp = (R.pool(12, page, Hkv, hd, torch.float16, "token", s) for s in (1, 2))
    lens = torch.tensor(lens, dtype=torch.int32)
    theta = _theta(hd)
    qd, kd, vd, qm, km, vm = R.append(k, v, kp, vp, tab, start, lens, q, theta)
    kc, vc = kp.cuda(), vp.cuda()
    got = B.paged_append(k.cuda(), v.cuda(), kc, vc, tab.cuda(), start.cuda(), lens.cuda(), q=q.cuda(),
                         theta=theta.cuda())
    _close(got, qd, qm, "q")
    touched = km.abs().sum((-1, -2)) > 0
    assert int(touched.sum()) == 3 + 2                  # of 24 tokens
    assert torch.equal(kc.cpu()[~touched], kp[~touched]) and torch.equal(vc.cpu()[~touched], vp[~touched])
    _close(kc, kd, km, "k")
    _close(vc, vd, vm, "v")


def test_append_in_place_queries_and_many_sequences():
    """q_out = q; 130 sequences, every third without a new token (the search for a row's sequence passes 64)."""
    counts = [0 if b % 3 == 2 else 1 + b % 2 for b in range(130)]
    lens = [max(1, n) + 7 * b for b, n in enumerate(counts)]
    Hq, Hkv, hd, page = 5, 1, 128, 16
    start, k, v, q, w = _inputs(counts, Hq, Hkv, hd, torch.bfloat16)
    per = -(-max(lens) // page)
    kp, vp = (R.pool(130 * per, page, Hkv, hd, torch.bfloat16, "token", s, fill=0) for s in (1, 2))
    tab, lens = R.table(130, per, 130 * per), torch.tensor(lens, dtype=torch.int32)
    theta = _theta(hd)
    qd, kd, vd, qm, km, vm = R.append(k, v, kp, vp, tab, start, lens, q, theta, w[0], w[1])
    kc, vc, qc = kp.cuda(), vp.cuda(), q.cuda()
    got = B.paged_append(k.cuda(), v.cuda(), kc, vc, tab.cuda(), start.cuda(), lens.cuda(), q=qc, theta=theta.cuda(),
                         k_norm=w[0].cuda(), q_norm=w[1].cuda(), q_out=qc)
    assert got is qc
    _close(got, qd, qm, "q")
    _close(kc, kd, km, "k")
    _close(vc, vd, vm, "v")


def _books(M, G, K, d, seed):
    rng = np.random.default_rng(seed)
    gain = np.abs(rng.standard_normal((M, G, K))).astype(np.float32) * 2
    shape = rng.standard_normal((M, G, K, d))
    shape = (shape / np.linalg.norm(shape, axis=-1, keepdims=True)).astype(np.float32)
    return gain, shape


@pytest.mark.parametrize("lens,cap,Hkv,hd,d,K,M,page,held,rope", [
    ([1], 1, 1, 64, 8, 256, 1, 8, "f16", True),
    ([77, 0, 130], 130, 8, 128, 8, 256, 1, 16, "f16", True),        # the 1-bit layout, one sequence empty
    ([40, 100], 90, 2, 128, 128, 256, 12, 8, "bf16", True),         # 0.75 bit; a length past the codes
    ([33], 40, 3, 128, 16, 256, 4, 64, "f16", False),
    ([50, 51], 60, 2, 64, 64, 64, 3, 16, "bf16", True),             # 6-bit codes, across words
    ([20], 20, 4, 128, 256, 4096, 2, 32, "f16", True),              # a codeword over two heads, 12-bit codes
    ([70, 65], 70, 2, 256, 8, 256, 2, 16, "bf16", True),
    ([25], 30, 2, 256, 32, 2, 5, 8, "f16", True),
    ([1500, 3, 900], 1500, 2, 64, 8, 256, 1, 16, "f16", True),      # several chunks, ranges over sequences
    ([700], 700, 1, 128, 16, 256, 4, 16, "f16", True),              # more stages than LDS holds, codes of their own
    ([800, 10], 801, 8, 128, 128, 256, 20, 32, "bf16", True),       # past 16 stages
    ([1300, 641, 2600], 2600, 8, 128, 128, 256, 3, 32, "f16", True),  # chunks of 640 tokens
    ([130], 130, 1, 256, 64, 16, 40, 8, "f16", True),               # 4-bit codes, 40 stages
    ([60], 60, 2, 64, 32, 512, 1, 8, "bf16", True),                 # 9-bit codes
])
def test_restore(lens, cap, Hkv, hd, d, K, M, page, held, rope):
    """Codes of both sides into pages.  Tolerance: half a step of the type; a rotation's, whose cosine and sine may come
    from two rotations joined (6 roundings each and 3 of the product) and which adds 3: 18 under 2^-19; and M
    roundings of a codeword and of the float32 sum: 2 M 2^-24 of the codewords' magnitudes."""
    say("restore", lens, cap, Hkv, hd, d, K, M, page, held)
    Bn, G = len(lens), Hkv * hd // d
    rng = np.random.default_rng(3)
    book = [_books(M, G, K, d, s) for s in (1, 2)]
    k = [rng.integers(0, K, (Bn * cap, M, G)) for _ in range(2)]
    codes = [O.pack_codes(x, K) for x in k]
    per = -(-cap // page)
    pages = Bn * per + 1
    kp, vp = (R.pool(pages, page, Hkv, hd, R.TYPES[held], "token", s) for s in (1, 2))
    tab = R.table(Bn, per, pages)
    if per > 2:
        tab[0, 1] = -1                                   # a page that is not there
    theta = _theta(hd)
    dev = [torch.from_numpy(np.ascontiguousarray(c).view(np.int32)).cuda().view(Bn, cap, -1) for c in codes]
    kc, vc = kp.cuda(), vp.cuda()
    B.paged_restore(*dev, torch.tensor(lens, dtype=torch.int32, device="cuda"),
                    *(torch.from_numpy(x).cuda() for pair in book for x in pair), kc, vc, tab.cuda(),
                    theta=theta.cuda() if rope else None)
    for side, (pool, got) in enumerate(((kp, kc), (vp, vc))):
        gain, shape = (x.astype(np.float64) for x in book[side])
        ref, scale = pool.double().clone(), torch.zeros(pool.shape, dtype=torch.float64)
        held_at = torch.zeros(pool.shape[:2], dtype=torch.bool)
        for b, n in enumerate(lens):
            for t in range(min(n, cap)):
                at = R.page_of(tab, pages, page, b, t)
                if at is None:
                    continue
                c = k[side][b * cap + t]
                parts = np.stack([gain[m][np.arange(G), c[m]][:, None] * shape[m][np.arange(G), c[m]] for m in range(M)])
                x = torch.from_numpy(parts.sum(0)).reshape(Hkv, hd)
                mag = torch.from_numpy(np.abs(parts).sum(0)).reshape(Hkv, hd)
                turned = side == 0 and rope
                ref[at, t % page] = R.rope(x, t, theta) if turned else x
                whole = mag + mag.roll(hd // 2, -1) if turned else mag
                scale[at, t % page] = whole * (2.0 ** -19 * turned + 2 * M * 2.0 ** -24) / 2.0 ** -19
                held_at[at, t % page] = True
        assert torch.equal(got.cpu()[~held_at], pool[~held_at])
        _close(got, ref, scale, "kv"[side])
