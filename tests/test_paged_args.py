"""What the paged cache's entry points refuse, on the CPU: the C ABI checks its
arguments before any HIP call (dummy pointers stand for device memory), and
the binding checks tensors before it calls."""
import ctypes
import os

import pytest
import torch

from paper_2607_01065_amd import gsrq as B

pytestmark = pytest.mark.skipif(not os.path.exists(B.LIB_PATH), reason="libgsrq.so not built")

PTR = 1 << 20


def _pages(**kw):
    base = dict(k=PTR, v=PTR, ks=(16 * 8 * 128, 8 * 128, 128), vs=(16 * 8 * 128, 8 * 128, 128), table=PTR, ldt=4,
                pages=10, page_size=16, per=4, B=2, Hkv=8, head_dim=128, dtype=B.GSRQ_F16)
    base.update(kw)
    S3 = ctypes.c_int64 * 3
    return B.Pages(base["k"], base["v"], S3(*base["ks"]), S3(*base["vs"]), base["table"], base["ldt"], base["pages"],
                   base["page_size"], base["per"], base["B"], base["Hkv"], base["head_dim"], base["dtype"])


BAD_PAGES = [(dict(k=None), 1), (dict(v=PTR + 8), 1), (dict(table=None), 1), (dict(pages=0), 1), (dict(per=0), 1),
             (dict(B=0), 1), (dict(Hkv=0), 1), (dict(ldt=3), 1), (dict(dtype=B.GSRQ_F32), 2), (dict(dtype=9), 1),
             (dict(page_size=24), 2), (dict(page_size=4), 2), (dict(ks=(1 << 30, 1 << 26, 128)), 2), (dict(vs=(1 << 31, 8 * 128, 128)), 2), (dict(page_size=0), 1), (dict(head_dim=96), 2), (dict(head_dim=0), 1),
             (dict(ks=(16 * 8 * 128, 8 * 128 + 4, 128)), 1), (dict(vs=(0, 8 * 128, 128)), 1),
             (dict(per=1 << 20, page_size=1 << 12, ldt=1 << 20), 1)]


def _append(pages=None, T=5, q_start=PTR, seq_len=PTR, k=PTR, v=PTR, q=PTR, stride=1024, Hq=32, dtype=B.GSRQ_F16,
            theta=None, k_norm=None, q_norm=None, eps=1e-6, q_out=PTR):
    lib = B.load_library()
    heads = [None if x is None else ctypes.byref(B.Heads(x, stride, 128)) for x in (k, v, q)]
    return lib.gsrq_paged_append(ctypes.byref(pages or _pages()), T, q_start, seq_len, *heads, Hq, dtype, theta, k_norm,
                                 q_norm, eps, q_out, None)


@pytest.mark.parametrize("kw,status", BAD_PAGES)
def test_append_refuses_pages(kw, status):
    assert _append(_pages(**kw)) == status


@pytest.mark.parametrize("kw,status", [
    (dict(T=0), 1), (dict(T=1 << 24), 2), (dict(q_start=None), 1), (dict(seq_len=None), 1), (dict(k=None), 1),
    (dict(v=PTR + 2), 1), (dict(stride=1028), 1), (dict(Hq=0), 1), (dict(dtype=3), 1), (dict(eps=-1.0), 1),
    (dict(eps=float("nan")), 1), (dict(q_out=None), 1), (dict(q=None), 1), (dict(q=None, q_out=None, q_norm=PTR), 1),
    (dict(theta=PTR + 4), 1), (dict(Hq=1 << 17), 2)])
def test_append_refuses_arguments(kw, status):
    assert _append(**kw) == status


def _restore(pages=None, N=200, D=1024, d=8, K=256, M=1, cap=100, codes=PTR, shape=PTR, seq_len=PTR):
    lib = B.load_library()
    sh = B.make_shape(N, D, d, K, M)
    return lib.gsrq_paged_restore(ctypes.byref(pages or _pages()), ctypes.byref(sh), cap, codes, codes, seq_len, PTR, shape,
                                  PTR, shape, None, None)


@pytest.mark.parametrize("kw,status", BAD_PAGES)
def test_restore_refuses_pages(kw, status):
    assert _restore(_pages(**kw)) == status


@pytest.mark.parametrize("kw,status", [
    (dict(cap=0), 1), (dict(N=199), 1), (dict(D=512), 1), (dict(d=0), 1), (dict(d=4), 2), (dict(d=512), 2), (dict(K=200), 1),
    (dict(M=0), 1), (dict(codes=None), 1), (dict(shape=PTR + 4), 1), (dict(seq_len=None), 1), (dict(K=1 << 17), 1),
    (dict(cap=2 ** 31 - 1, N=2 ** 40), 2)])
def test_restore_refuses_arguments(kw, status):
    assert _restore(**kw) == status


def test_packed_structures_are_the_abi_s():
    """The binding packs what the ctypes structures describe."""
    kp = torch.zeros((4, 8, 3, 64), dtype=torch.bfloat16).transpose(1, 2).contiguous().transpose(1, 2)
    vp, tab = torch.zeros((4, 8, 3, 64), dtype=torch.bfloat16), torch.zeros((5, 9), dtype=torch.int32)[:, :2]
    p = B.Pages.from_buffer_copy(B._pages(kp, vp, tab))
    assert (p.k, p.v, p.table) == (kp.data_ptr(), vp.data_ptr(), tab.data_ptr())
    assert (list(p.k_stride), list(p.v_stride)) == ([1536, 64, 512], [1536, 192, 64])
    assert (p.ldt, p.pages, p.page_size, p.per, p.B, p.Hkv, p.head_dim, p.dtype) == (9, 4, 8, 2, 5, 3, 64, B.GSRQ_BF16)
    h = B.Heads.from_buffer_copy(B._heads(vp[0], "x", 3, 64, 8, torch.bfloat16, vp))
    assert (h.data, h.token_stride, h.head_stride) == (vp.data_ptr(), 192, 64)
    a = B.PagedAttn.from_buffer_copy(B._PAGED_ATTN.pack(7, 6, 5, 0.5, 0))
    assert (a.T, a.Hq, a.window, a.scale, a.flags) == (7, 6, 5, 0.5, 0)


def _tensors(**kw):
    t = dict(k=torch.zeros((3, 2, 64), dtype=torch.float16), v=torch.zeros((3, 2, 64), dtype=torch.float16),
             kp=torch.zeros((4, 8, 2, 64), dtype=torch.float16), vp=torch.zeros((4, 8, 2, 64), dtype=torch.float16),
             table=torch.zeros((2, 2), dtype=torch.int32), q_start=torch.zeros(3, dtype=torch.int32),
             seq_len=torch.zeros(2, dtype=torch.int32))
    t.update(kw)
    return [t[n] for n in ("k", "v", "kp", "vp", "table", "q_start", "seq_len")]


@pytest.mark.parametrize("kw,error", [
    (dict(kp=torch.zeros((4, 8, 64), dtype=torch.float16)), ValueError),
    (dict(vp=torch.zeros((4, 8, 2, 64), dtype=torch.bfloat16)), TypeError),
    (dict(kp=torch.zeros((4, 8, 2, 64)), vp=torch.zeros((4, 8, 2, 64))), TypeError),
    (dict(table=torch.zeros((2, 2), dtype=torch.int64)), TypeError),
    (dict(table=torch.zeros((2, 4), dtype=torch.int32)[:, ::2]), ValueError),
    (dict(k=torch.zeros((3, 1, 64), dtype=torch.float16)), ValueError),
    (dict(v=torch.zeros((2, 2, 64), dtype=torch.float16)), ValueError),
    (dict(v=torch.zeros((3, 2, 64))), TypeError),
    (dict(k=torch.zeros((3, 2, 64), dtype=torch.float64)), TypeError),
    (dict(k=torch.zeros((3, 2, 128), dtype=torch.float16)[..., ::2]), ValueError),
    (dict(q_start=torch.zeros(2, dtype=torch.int32)), ValueError),
    (dict(q_start=torch.zeros(3)), TypeError),
    (dict(seq_len=torch.zeros(3, dtype=torch.int32)), ValueError),
    (dict(), ValueError),                                # no GPU tensors
])
def test_binding_append_refuses(kw, error):
    with pytest.raises(error):
        B.paged_append(*_tensors(**kw))


def test_binding_append_refuses_options():
    t = _tensors()
    for kw, error in ((dict(theta=torch.zeros(32)), TypeError), (dict(theta=torch.zeros(31, dtype=torch.float64)), ValueError),
                      (dict(q_norm=torch.zeros(64)), ValueError), (dict(k_norm=torch.zeros(32)), ValueError),
                      (dict(q=torch.zeros((2, 4, 64), dtype=torch.float16)), ValueError),
                      (dict(q_out=torch.zeros((3, 4, 64), dtype=torch.float16)), ValueError)):
        with pytest.raises(error):
            B.paged_append(*t, **kw)


def test_binding_restore_refuses():
    kp = torch.zeros((4, 8, 2, 64), dtype=torch.float16)
    tab, lens = torch.zeros((2, 2), dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    codes = torch.zeros((2, 5, 4), dtype=torch.int32)
    gain, shape = torch.zeros((1, 16, 256)), torch.zeros((1, 16, 256, 8))
    good = dict(k_codes=codes, v_codes=codes, seq_len=lens, k_gain=gain, k_shape=shape, v_gain=gain, v_shape=shape,
                k_pages=kp, v_pages=kp, table=tab)
    for kw, error in ((dict(k_codes=codes[:1]), ValueError), (dict(k_codes=codes[..., :3].contiguous()), ValueError),
                      (dict(v_codes=codes[:, :4]), ValueError), (dict(v_gain=gain[..., :128]), ValueError),
                      (dict(k_shape=shape[0]), ValueError), (dict(seq_len=lens.long()), TypeError), (dict(), ValueError)):
        with pytest.raises(error):
            B.paged_restore(**{**good, **kw})


def _attn(pages=None, T=5, Hq=32, window=0, scale=0.1, flags=0, q_start=PTR, seq_len=PTR, q=PTR, stride=4096, out=PTR,
          ws=PTR, nbytes=1 << 40):
    lib = B.load_library()
    s = B.PagedAttn(T, Hq, window, scale, flags)
    qh = None if q is None else ctypes.byref(B.Heads(q, stride, 128))
    return lib.gsrq_attn_paged(ctypes.byref(s), ctypes.byref(pages or _pages()), q_start, seq_len, qh, out, None, ws, nbytes,
                               None)


@pytest.mark.parametrize("kw,status", BAD_PAGES)
def test_attention_refuses_pages(kw, status):
    assert _attn(_pages(**kw)) == status


LONG = dict(per=1 << 14, ldt=1 << 14)


@pytest.mark.parametrize("kw,status", [
    (dict(T=0), 1), (dict(Hq=0), 1), (dict(Hq=12), 1), (dict(window=-1), 1), (dict(scale=0.0), 1), (dict(scale=-1.0), 1),
    (dict(scale=float("inf")), 1), (dict(scale=float("nan")), 1), (dict(flags=1), 1), (dict(q_start=None), 1),
    (dict(seq_len=None), 1), (dict(q=None), 1), (dict(q=PTR + 2), 1), (dict(stride=4100), 1), (dict(out=None), 1),
    (dict(out=PTR + 8), 1), (dict(pages=_pages(**LONG), ws=None), 1), (dict(pages=_pages(**LONG), ws=PTR + 16), 1),
    (dict(pages=_pages(**LONG), nbytes=0), 3), (dict(T=1 << 30), 2)])
def test_attention_refuses_arguments(kw, status):
    assert _attn(**kw) == status


def test_binding_attention_refuses():
    kp = torch.zeros((4, 8, 2, 64), dtype=torch.float16)
    tab, lens, start = torch.zeros((2, 2), dtype=torch.int32), torch.zeros(2, dtype=torch.int32), torch.zeros(3, dtype=torch.int32)
    q = torch.zeros((3, 4, 64), dtype=torch.float16)
    good = dict(q=q, k_pages=kp, v_pages=kp, table=tab, q_start=start, seq_len=lens)
    for kw, error in ((dict(q=q.bfloat16()), TypeError), (dict(q=q[0]), ValueError), (dict(q=q[..., :32]), ValueError),
                      (dict(q_start=start[:2]), ValueError), (dict(seq_len=lens.long()), TypeError),
                      (dict(out=torch.zeros(3, 4, 64)), TypeError), (dict(window=1 << 31), ValueError), (dict(scale="1"), ValueError), (dict(out=q[:2]), ValueError),
                      (dict(workspace=torch.zeros(8, dtype=torch.uint8)[::2]), ValueError), (dict(), ValueError)):
        with pytest.raises(error):
            B.attn_paged(**{**good, **kw})


def test_streams_and_devices():
    """A stream of another device is refused; tensors of another device than the current one make theirs current."""
    import types
    cuda0, cuda1 = torch.device("cuda", 0), torch.device("cuda", 1)
    with pytest.raises(ValueError):
        B._paged_device(cuda0, types.SimpleNamespace(device=cuda1))
    with pytest.raises(ValueError):
        B._paged_device(torch.device("cpu"), None)


@pytest.mark.parametrize("current,index,made", [(0, 0, None), (0, 1, 1), (1, 0, 0)])
def test_another_device_becomes_current(monkeypatch, current, index, made):
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: current, raising=False)
    monkeypatch.setattr(torch.cuda, "device", lambda d: ("device", d.index))
    got = B._paged_device(torch.device("cuda", index), None)
    assert got == (None if made is None else ("device", made))
