"""What the 8-bit pages' entry points, paged_plan and verify_drafts refuse, on
the CPU: the C ABI checks its arguments before any HIP call (dummy pointers
stand for device memory), and the binding checks tensors before it calls."""
import ctypes
import os

import pytest
import torch

from paper_2607_01065_amd import gsrq as B
from tests.test_paged_args import PTR, _pages

pytestmark = pytest.mark.skipif(not os.path.exists(B.LIB_PATH), reason="libgsrq.so not built")

E4M3 = torch.float8_e4m3fn


def _p(**kw):
    return _pages(**{**dict(dtype=B.GSRQ_E4M3), **kw})


def _exps(k=PTR, v=PTR, ks=(8, 1), vs=(8, 1)):
    S2 = ctypes.c_int64 * 2
    return B.PageExps(k, v, S2(*ks), S2(*vs))


BAD_PAGES = [(dict(k=None), 1), (dict(v=PTR + 8), 1), (dict(dtype=B.GSRQ_F16), 1), (dict(dtype=B.GSRQ_F32), 1),
             (dict(page_size=24), 2), (dict(head_dim=96), 2), (dict(ks=(16 * 8 * 128, 8 * 128 + 8, 128)), 1),
             (dict(vs=(0, 8 * 128, 128)), 1), (dict(ks=(1 << 30, 1 << 26, 128)), 2), (dict(per=1 << 20, page_size=1 << 12, ldt=1 << 20), 1)]
BAD_EXPS = [dict(k=None), dict(v=None), dict(ks=(0, 1)), dict(vs=(8, 0)), dict(ks=(-8, 1))]


def _append(pages=None, exps=None, T=5, q_start=PTR, seq_len=PTR, k=PTR, v=PTR, q=PTR, stride=1024, Hq=32, dtype=B.GSRQ_F16,
            theta=None, k_norm=None, q_norm=None, eps=1e-6, q_out=PTR, q_dtype=B.GSRQ_F16):
    lib = B.load_library()
    heads = [None if x is None else ctypes.byref(B.Heads(x, stride, 128)) for x in (k, v, q)]
    return lib.gsrq_paged_append8(ctypes.byref(pages or _p()), ctypes.byref(exps or _exps()), T, q_start, seq_len, *heads, Hq,
                                  dtype, theta, k_norm, q_norm, eps, q_out, q_dtype, None)


def _attn(pages=None, exps=None, T=5, Hq=32, window=0, scale=0.1, flags=0, q_start=PTR, seq_len=PTR, q=PTR, q_dtype=B.GSRQ_F16,
          stride=4096, out=PTR, ws=PTR, nbytes=1 << 40):
    lib = B.load_library()
    s = B.PagedAttn(T, Hq, window, scale, flags)
    qh = None if q is None else ctypes.byref(B.Heads(q, stride, 128))
    return lib.gsrq_attn_paged8(ctypes.byref(s), ctypes.byref(pages or _p()), ctypes.byref(exps or _exps()), q_start, seq_len, qh,
                                q_dtype, out, None, ws, nbytes, None)


@pytest.mark.parametrize("kw,status", BAD_PAGES)
def test_pages_refused(kw, status):
    assert _append(_p(**kw)) == status and _attn(_p(**kw)) == status


@pytest.mark.parametrize("kw", BAD_EXPS)
def test_exponents_refused(kw):
    assert _append(exps=_exps(**kw)) == 1 and _attn(exps=_exps(**kw)) == 1


def test_sixteen_bit_calls_refuse_eight_bit_pages():
    lib = B.load_library()
    h = ctypes.byref(B.Heads(PTR, 1024, 128))
    assert lib.gsrq_paged_append(ctypes.byref(_p()), 5, PTR, PTR, h, h, None, 0, B.GSRQ_F16, None, None, None, 1e-6, None, None) == 1
    n, s = ctypes.c_size_t(), B.PagedAttn(5, 32, 0, 0.1, 0)
    assert lib.gsrq_attn_paged_workspace_bytes(ctypes.byref(s), ctypes.byref(_p()), ctypes.byref(n)) == 1
    assert lib.gsrq_attn_paged8_workspace_bytes(ctypes.byref(s), ctypes.byref(_p()), ctypes.byref(n)) == 0
    assert lib.gsrq_attn_paged8_workspace_bytes(ctypes.byref(s), ctypes.byref(_pages()), ctypes.byref(n)) == 1
    assert lib.gsrq_attn_paged8_workspace_bytes(ctypes.byref(s), ctypes.byref(_p()), None) == 1


@pytest.mark.parametrize("kw,status", [
    (dict(T=0), 1), (dict(T=1 << 24), 2), (dict(q_start=None), 1), (dict(seq_len=None), 1), (dict(k=None), 1),
    (dict(v=PTR + 2), 1), (dict(stride=1028), 1), (dict(Hq=0), 1), (dict(dtype=3), 1), (dict(eps=-1.0), 1),
    (dict(eps=float("nan")), 1), (dict(q_out=None), 1), (dict(q=None), 1), (dict(q=None, q_out=None, q_norm=PTR), 1),
    (dict(theta=PTR + 4), 1), (dict(Hq=1 << 17), 2), (dict(q_dtype=B.GSRQ_F32), 1), (dict(q_dtype=B.GSRQ_E4M3), 1),
    (dict(pages=_p(B=(1 << 20) + 1)), 2)])
def test_append_refuses(kw, status):
    assert _append(**kw) == status


LONG = dict(per=1 << 14, ldt=1 << 14)


@pytest.mark.parametrize("kw,status", [
    (dict(T=0), 1), (dict(Hq=12), 1), (dict(window=-1), 1), (dict(scale=0.0), 1), (dict(scale=float("nan")), 1), (dict(flags=1), 1),
    (dict(q_start=None), 1), (dict(seq_len=None), 1), (dict(q=None), 1), (dict(q=PTR + 2), 1), (dict(stride=4100), 1),
    (dict(out=None), 1), (dict(out=PTR + 8), 1), (dict(q_dtype=B.GSRQ_F32), 1), (dict(q_dtype=7), 1),
    (dict(pages=_p(**LONG), ws=None), 1), (dict(pages=_p(**LONG), nbytes=0), 3), (dict(T=1 << 30), 2)])
def test_attention_refuses(kw, status):
    assert _attn(**kw) == status


def _plan(T=100, ldt=16, Bn=4, per=16, page=16, F=64, table=PTR, free=PTR, n_free=PTR, seq_len=PTR, change=PTR, q_start=PTR,
          slots=PTR, positions=PTR):
    s = B.PagedBatch(T, ldt, Bn, per, page, F)
    return B.load_library().gsrq_paged_plan(ctypes.byref(s), table, free, n_free, seq_len, change, q_start, slots, positions, None)


@pytest.mark.parametrize("kw,status", [
    (dict(T=-1), 1), (dict(ldt=15), 1), (dict(Bn=0), 1), (dict(per=0), 1), (dict(page=0), 1), (dict(F=0), 1), (dict(table=None), 1),
    (dict(free=None), 1), (dict(n_free=None), 1), (dict(seq_len=None), 1), (dict(change=None), 1), (dict(q_start=None), 1),
    (dict(slots=None), 1), (dict(positions=None), 1), (dict(page=24), 2), (dict(page=4), 2), (dict(Bn=8193), 2),
    (dict(T=1 << 31), 2), (dict(per=1 << 20, ldt=1 << 20, page=1 << 12), 1), (dict(Bn=8192, per=1 << 19, ldt=1 << 19, page=8), 2)])
def test_plan_refuses(kw, status):
    assert _plan(**kw) == status


LARGE = dict(V=50000, ldp=50000, ldq=50000)          # (fewer tokens need no workspace)


def _verify(T=10, V=100, Bn=2, tokens=PTR, target=PTR, ldp=100, draft=PTR, ldq=100, dtype=B.GSRQ_F32, uniform=PTR, draw=PTR,
            q_start=PTR, accepted=PTR, nxt=PTR, ws=PTR, nbytes=1 << 30):
    return B.load_library().gsrq_verify_drafts(T, V, Bn, tokens, target, ldp, draft, ldq, dtype, uniform, draw, q_start, accepted,
                                               nxt, ws, nbytes, None)


@pytest.mark.parametrize("kw,status", [
    (dict(T=-1), 1), (dict(V=0), 1), (dict(Bn=0), 1), (dict(Bn=(1 << 16) + 1), 2), (dict(V=1 << 31), 2), (dict(T=1 << 31), 2),
    (dict(tokens=None), 1), (dict(target=None), 1), (dict(uniform=None), 1), (dict(draw=None), 1), (dict(q_start=None), 1),
    (dict(accepted=None), 1), (dict(nxt=None), 1), (dict(ldp=99), 1), (dict(ldq=99), 1), (dict(dtype=3), 1), (dict(target=PTR + 2), 1),
    (dict(draft=PTR + 1, dtype=B.GSRQ_F16), 1), (dict(ws=None, **LARGE), 1), (dict(ws=PTR + 16, **LARGE), 1), (dict(nbytes=0, **LARGE), 3)])
def test_verify_refuses(kw, status):
    assert _verify(**kw) == status


def test_packed_structures_are_the_abi_s():
    k = torch.zeros((4, 3, 2), dtype=torch.int8)
    kp = torch.zeros((4, 8, 3, 64), dtype=torch.uint8).view(E4M3)
    x = B.PageExps.from_buffer_copy(B._exps(k[..., 0], k[..., 1], kp))
    assert (x.k, x.v) == (k.data_ptr(), k.data_ptr() + 1)
    assert (list(x.k_stride), list(x.v_stride)) == ([6, 2], [6, 2])
    p = B.Pages.from_buffer_copy(B._pages(kp, kp, torch.zeros((2, 2), dtype=torch.int32), True))
    assert (p.pages, p.page_size, p.Hkv, p.head_dim, p.dtype) == (4, 8, 3, 64, B.GSRQ_E4M3)
    s = B.PagedBatch.from_buffer_copy(B._PAGED_BATCH.pack(7, 6, 5, 4, 16, 3))
    assert (s.T, s.ldt, s.B, s.per, s.page_size, s.F) == (7, 6, 5, 4, 16, 3)


def _cache(**kw):
    t = dict(kp=torch.zeros((4, 8, 2, 64), dtype=torch.uint8).view(E4M3), vp=torch.zeros((4, 8, 2, 64), dtype=torch.uint8).view(E4M3),
             ke=torch.zeros((4, 2), dtype=torch.int8), ve=torch.zeros((4, 2), dtype=torch.int8))
    t.update(kw)
    return t


@pytest.mark.parametrize("kw,error", [
    (dict(ke=None), ValueError), (dict(ve=None), ValueError), (dict(ke=torch.zeros((4, 2))), TypeError),
    (dict(ve=torch.zeros((4, 1), dtype=torch.int8)), ValueError), (dict(ke=torch.zeros(8, dtype=torch.int8)), ValueError),
    (dict(kp=torch.zeros((4, 8, 2, 64), dtype=torch.float16), vp=torch.zeros((4, 8, 2, 64), dtype=torch.float16)), TypeError),
    (dict(vp=torch.zeros((4, 8, 2, 64), dtype=torch.uint8)), TypeError), (dict(ke=None, ve=None), TypeError),
    (dict(), ValueError),                                # no GPU tensors
])
def test_binding_refuses_pages(kw, error):
    c = _cache(**kw)
    tab, start, lens = torch.zeros((2, 2), dtype=torch.int32), torch.zeros(3, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    k, q = torch.zeros((3, 2, 64), dtype=torch.float16), torch.zeros((3, 4, 64), dtype=torch.float16)
    with pytest.raises(error):
        B.paged_append(k, k, c["kp"], c["vp"], tab, start, lens, k_exp=c["ke"], v_exp=c["ve"])
    with pytest.raises(error):
        B.attn_paged(q, c["kp"], c["vp"], tab, start, lens, k_exp=c["ke"], v_exp=c["ve"])


def test_binding_refuses_query_types():
    c = _cache()
    tab, start, lens = torch.zeros((2, 2), dtype=torch.int32), torch.zeros(3, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    k, q = torch.zeros((3, 2, 64)), torch.zeros((3, 4, 64))
    with pytest.raises(TypeError):
        B.attn_paged(q, c["kp"], c["vp"], tab, start, lens, k_exp=c["ke"], v_exp=c["ve"])
    with pytest.raises(TypeError):
        B.paged_append(k, k, c["kp"], c["vp"], tab, start, lens, q=q, q_out=q, k_exp=c["ke"], v_exp=c["ve"])
    with pytest.raises(TypeError):                       # codes go back into 16-bit pages
        codes, gain, shape = torch.zeros((2, 5, 4), dtype=torch.int32), torch.zeros((1, 16, 256)), torch.zeros((1, 16, 256, 8))
        B.paged_restore(codes, codes, lens, gain, shape, gain, shape, c["kp"], c["vp"], tab)


def test_binding_plan_refuses():
    i32 = dict(dtype=torch.int32)
    good = dict(table=torch.zeros((2, 4), **i32), free_pages=torch.zeros(9, **i32), n_free=torch.zeros(1, **i32),
                seq_len=torch.zeros(2, **i32), change=torch.zeros(2, **i32), page_size=16, rows=5)
    for kw, error in ((dict(table=torch.zeros((2, 4))), TypeError), (dict(table=torch.zeros((2, 8), **i32)[:, ::2]), ValueError),
                      (dict(free_pages=torch.zeros(9)), TypeError), (dict(n_free=torch.zeros(2, **i32)), ValueError),
                      (dict(seq_len=torch.zeros(3, **i32)), ValueError), (dict(change=torch.zeros(2)), TypeError),
                      (dict(rows=-1), ValueError), (dict(page_size=1 << 40), ValueError), (dict(page_size=None), ValueError),
                      (dict(q_start=torch.zeros(2, **i32)), ValueError), (dict(slots=torch.zeros(5, **i32)), TypeError),
                      (dict(positions=torch.zeros(4, **i32)), ValueError), (dict(), ValueError)):
        with pytest.raises(error):
            B.paged_plan(**{**good, **kw})


def test_binding_verify_refuses():
    i32 = dict(dtype=torch.int32)
    p = torch.zeros((5, 7))
    good = dict(tokens=torch.zeros(5, **i32), target=p, draft=p, uniform=torch.zeros(5), draw=torch.zeros(2), q_start=torch.zeros(3, **i32))
    for kw, error in ((dict(tokens=torch.zeros(4, **i32)), ValueError), (dict(tokens=torch.zeros(5)), TypeError), (dict(target=p[0]), ValueError),
                      (dict(target=p.double()), TypeError), (dict(draft=p.half()), ValueError), (dict(draft=p[:4]), ValueError),
                      (dict(target=p.T.contiguous().T), ValueError), (dict(uniform=torch.zeros(2)), ValueError), (dict(draw=torch.zeros(5)), ValueError),
                      (dict(draft=p[:1].expand(5, 7)), ValueError), (dict(q_start=torch.zeros(1, **i32)), ValueError),
                      (dict(accepted=torch.zeros(3, **i32)), ValueError), (dict(next_token=torch.zeros(2)), TypeError), (dict(), ValueError)):
        with pytest.raises(error):
            B.verify_drafts(**{**good, **kw})


@pytest.mark.parametrize("Bn,per", [(8191, 262176), (1023, 2099202), (17, 126322567)])
def test_plan_refuses_tables_whose_entries_cannot_be_counted_in_rounds(Bn, per):
    """Just below 2^31 entries: the counter of a round of 4096 moves would wrap and never end."""
    assert (1 << 31) - 4096 <= Bn * per < 1 << 31
    assert _plan(Bn=Bn, per=per, ldt=per, page=8) == 2


@pytest.mark.parametrize("kw", [dict(page_size=1 << 25), dict(page_size=1 << 24, head_dim=256), dict(page_size=1 << 26, head_dim=64),
                                dict(page_size=1 << 30, Hkv=4, head_dim=64)])
def test_append_refuses_pages_whose_codes_cannot_be_counted(kw):
    """Pages of 2^31 pieces of 16 bytes and more: the counter of the codes that are rounded again would wrap."""
    assert _append(_p(per=1, ldt=1, pages=1, **kw)) == 2
