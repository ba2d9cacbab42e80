"""The paged cache's operators in 64 bits, token by token on the CPU, and the
inputs of their tests.  Plain loops over sequences and tokens; nothing of the
library is used."""
import math

import torch

TYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}


def half_step(dtype):
    """A rounding's largest share of the value, and the absolute half step of its subnormals."""
    f = torch.finfo(dtype)
    return f.eps / 2, f.tiny * f.eps / 2


def pool(pages, page, Hkv, hd, dtype, order="token", seed=0, fill=None):
    """A pool [pages, page, Hkv, hd], its tokens or its heads outermost in a page."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((pages, page, Hkv, hd), generator=g).to(dtype)
    if fill is not None:
        x.fill_(fill)
    return x if order == "token" else x.transpose(1, 2).contiguous().transpose(1, 2)


def table(B, per, pages, seed=0):
    g = torch.Generator().manual_seed(seed)
    return torch.randperm(pages, generator=g)[: B * per].view(B, per).to(torch.int32)


def page_of(tab, pages, page, b, pos):
    """The page of a position, or None."""
    if pos < 0 or pos // page >= tab.shape[1]:
        return None
    at = int(tab[b, pos // page])
    return at if 0 <= at < pages else None


def rope(x, pos, theta):
    """x [..., hd] in 64 bits, turned by pos * theta."""
    h = x.shape[-1] // 2
    a = pos * theta
    c, s = torch.cos(a), torch.sin(a)
    lo, hi = x[..., :h], x[..., h:]
    return torch.cat([lo * c - hi * s, hi * c + lo * s], -1)


def rms(x, w, eps):
    return x if w is None else x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * w.double()


def append(k, v, kp, vp, tab, q_start, seq_len, q=None, theta=None, k_norm=None, q_norm=None, eps=1e-6):
    """(q, k pages, v pages) in 64 bits, and the magnitudes |x| + |y| that a rotation's rounding goes by, laid
    out the same.  Rows of no sequence in q are NaN."""
    pages, page = kp.shape[:2]
    kd, vd = kp.double().clone(), vp.double().clone()
    km, vm = torch.zeros_like(kd), torch.zeros_like(vd)
    qd = None if q is None else torch.full(q.shape, math.nan, dtype=torch.float64)
    qm = None if q is None else torch.zeros(q.shape, dtype=torch.float64)
    for b in range(len(seq_len)):
        lo, hi = int(q_start[b]), int(q_start[b + 1])
        for r in range(lo, hi):
            pos = int(seq_len[b]) - (hi - lo) + r - lo
            turn = (lambda x: x) if theta is None else (lambda x, p=pos: rope(x, p, theta))
            if q is not None:
                x = rms(q[r].double(), q_norm, eps)
                qd[r] = turn(x)
                qm[r] = x.abs() + x.abs().roll(x.shape[-1] // 2, -1)
            at = page_of(tab, pages, page, b, pos)
            if at is None:
                continue
            x = rms(k[r].double(), k_norm, eps)
            kd[at, pos % page] = turn(x)
            km[at, pos % page] = x.abs() + x.abs().roll(x.shape[-1] // 2, -1)
            vd[at, pos % page] = v[r].double()
            vm[at, pos % page] = 0
    return qd, kd, vd, qm, km, vm


def new_rows(counts, gap=0):
    """q_start of sequences that bring `counts` tokens, and the rows of a call that holds `gap` more behind them."""
    start = [0]
    for n in counts:
        start.append(start[-1] + n)
    return torch.tensor(start, dtype=torch.int32), start[-1] + gap
