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


def attention(q, kp, vp, tab, q_start, seq_len, scale, window=0):
    """(out, lse, tol_out, tol_lse) of attention over pages in 64 bits, [T, Hq, hd] and [T, Hq]; rows of no sequence
    are NaN, rows that see nothing zero and -inf.

    The tolerances follow a library that multiplies in the pages' type (products exact, float32 sums), rounds the
    weights to that type and the result once.  With u = 2^-24:
      a score is off by e_s = scale sum_i |q_i k_i| (hd + 4) u + |s| 4 u (its sum; the scale, its factor log2 e and the
        subtraction of a maximum that is itself at most 2^8 below the largest), an exponential by 2^-22 more, so a
        weight by e = e_s + (|s| + |max s| + 16) 4 u + 2^-22 of itself;
      the product adds half a step of the weight's type, the sum over n tokens n u, and both sum and product carry e:
        2 e + half step + n u, of A = sum_j p_j |v_j| / sum_j p_j;
      float16 weights below 2^-14 are held to 2^-25, where the largest is at least 2^6: 2^-31 sum_j |v_j|;
      the result is rounded: half a step of itself.
    lse: e + n u and a logarithm, 8 u of its own size."""
    T, Hq, hd = q.shape
    pages, page, Hkv = kp.shape[:3]
    u = 2.0 ** -24
    rel, sub = half_step(q.dtype)
    out = torch.full((T, Hq, hd), math.nan, dtype=torch.float64)
    lse = torch.full((T, Hq), math.nan, dtype=torch.float64)
    t_out, t_lse = torch.zeros_like(out), torch.zeros_like(lse)
    for b in range(len(seq_len)):
        lo, hi = int(q_start[b]), int(q_start[b + 1])
        L = int(seq_len[b])
        n = hi - lo
        if n == 0:
            continue
        tokens = [t for t in range(min(max(L, 0), tab.shape[1] * page)) if page_of(tab, pages, page, b, t) is not None]
        at = torch.tensor([page_of(tab, pages, page, b, t) for t in tokens], dtype=torch.long)
        t = torch.tensor(tokens, dtype=torch.long)
        K, V = kp[at, t % page].double(), vp[at, t % page].double()
        pos = L - n + torch.arange(n)
        seen = t[None] <= pos[:, None]
        if window:
            seen &= t[None] > pos[:, None] - window
        for h in range(Hq):
            k, v = K[:, h // (Hq // Hkv)], V[:, h // (Hq // Hkv)]
            x = q[lo:hi, h].double()
            # a token that a row does not see takes no part, whatever it holds
            ks, vs = torch.nan_to_num(k, 0, 0, 0), torch.nan_to_num(v, 0, 0, 0)
            s = torch.where(seen, (x @ ks.T) * scale, -math.inf)
            z = torch.logsumexp(s, 1) if t.numel() else torch.full((n,), -math.inf, dtype=torch.float64)
            empty = ~seen.any(1)
            p = torch.where(seen, torch.exp(s - torch.where(empty, 0.0, z)[:, None]), 0.0)
            o = p @ vs
            for i in range(n):                      # infinities and NaN that a row does see
                if seen[i].any() and not torch.isfinite(torch.cat([k[seen[i]], v[seen[i]]])).all():
                    si = (k[seen[i]] @ x[i]) * scale
                    o[i], z[i] = torch.softmax(si, 0) @ v[seen[i]], torch.logsumexp(si, 0)
            out[lo:hi, h] = torch.where(empty[:, None], 0.0, o)
            lse[lo:hi, h] = z
            mag = torch.where(seen, (x.abs() @ ks.abs().T) * scale, 0.0)
            big = torch.where(seen, s.abs(), 0.0).amax(1) if t.numel() else torch.zeros(n, dtype=torch.float64)
            e = (mag.amax(1) if t.numel() else 0.0) * (hd + 4) * u + (2 * big + 16) * 4 * u + 2.0 ** -22
            few = len(tokens) * u
            A = p @ vs.abs()
            t_out[lo:hi, h] = (rel * out[lo:hi, h].abs().nan_to_num(0, 0, 0) + (2 * e + rel + few)[:, None] * A + sub
                               + 2.0 ** -31 * (seen.double() @ vs.abs()))
            t_lse[lo:hi, h] = e + few + 8 * u * z.abs().nan_to_num(0, 0, 0)
    return out, lse, t_out, t_lse
