"""The 8-bit paged cache in 64 bits on the CPU, page by page, and the inputs of
its tests.  Nothing of the library is used."""
import math

import torch

from tests import paged_ref as R

E4M3 = torch.float8_e4m3fn
LOW, HIGH = -40, 40


def exponent(a):
    """The smallest e of the range with a <= 448 * 2^e."""
    e = LOW
    while e < HIGH and a > 448.0 * 2.0 ** e:
        e += 1
    return e


def held(exp):
    return exp.clamp(LOW, HIGH)


def numbers(pages, exp):
    """What codes [pages, page, Hkv, hd] and exponents [pages, Hkv] stand for, in 64 bits."""
    return pages.double() * (2.0 ** held(exp).double())[:, None, :, None]


def pool(pages, page, Hkv, hd, order="token", seed=0, exps=(-6, 3)):
    """Codes of about 100 and exponents drawn from a range; tokens or heads outermost in a page."""
    g = torch.Generator().manual_seed(seed)
    x = (torch.randn((pages, page, Hkv, hd), generator=g) * 60).clamp(-448, 448).to(E4M3)
    e = torch.randint(exps[0], exps[1] + 1, (pages, Hkv), generator=g).to(torch.int8)
    return (x if order == "token" else reordered(x)), e


def reordered(x):
    return x.view(torch.uint8).transpose(1, 2).contiguous().transpose(1, 2).view(E4M3)


def coded(x, e):
    """x * 2^-e as codes: to the nearest, ties to even, beyond 448 held there, not finite: NaN."""
    y = (x * 2.0 ** -e)
    y = torch.where(torch.isfinite(y), y.clamp(-448, 448), math.nan)
    return y.float().to(E4M3)


def append(rows, mags, pages, exp, tab, q_start, seq_len):
    """Rows [T, Hkv, hd] in 64 bits, as they are stored, into a copy of a pool: (codes bit for bit, exponents, the
    numbers that new codes come from and their magnitudes, which places are new).  `mags`: the size that float32
    roundings of a row's elements go by."""
    codes, e = pages.clone(), exp.clone()
    n_pages, page = pages.shape[:2]
    want = torch.zeros(pages.shape, dtype=torch.float64)
    size = torch.zeros(pages.shape, dtype=torch.float64)
    new = torch.zeros(pages.shape[:2], dtype=torch.bool)
    for b in range(len(seq_len)):
        lo, hi = int(q_start[b]), int(q_start[b + 1])
        pos0 = int(seq_len[b]) - (hi - lo)
        touched = {}
        for r in range(lo, hi):
            pos = pos0 + r - lo
            at = R.page_of(tab, n_pages, page, b, pos)
            if at is not None:
                touched.setdefault(at, []).append((pos % page, r))
        for at, places in touched.items():
            slots, rs = [p for p, _ in places], [r for _, r in places]
            for h in range(pages.shape[2]):
                x = rows[rs, h]
                fine = x[torch.isfinite(x)].abs()
                now = exponent(float(fine.max()) if fine.numel() else 0.0)
                if slots[0]:
                    before = int(held(exp[at, h]))
                    now = max(now, before)
                    if now > before:
                        codes[at, :slots[0], h] = coded(pages[at, :slots[0], h].double(), now - before)
                e[at, h] = now
                want[at, slots, h], size[at, slots, h] = x, mags[rs, h]
            new[at, slots] = True
    return codes, e, want, size, new


def attention(q, kp, vp, ke, ve, tab, q_start, seq_len, scale, window=0):
    """paged_ref.attention over what the pages stand for.  To its tolerances come, with codes d_j and exponents e_j of
    the values and E the largest exponent:
      the exponent is added to a score and taken off again: 4 * 80 u of a weight, twice in the result;
      float16 products of weight and scale are held to 2^-25 where the largest is at least 2^6, so what is missing is
        2^-31 sum_j |d_j| 2^E / (the sum of weights, at least 1) where the plain one has 2^-31 sum_j |v_j|."""
    out, lse, t_out, t_lse = R.attention(q, numbers(kp, ke), numbers(vp, ve), tab, q_start, seq_len, scale, window)
    u = 2.0 ** -24
    pages, page, Hkv = kp.shape[:3]
    group = q.shape[1] // Hkv
    for b in range(len(seq_len)):
        lo, hi = int(q_start[b]), int(q_start[b + 1])
        L = int(seq_len[b])
        tokens = [t for t in range(min(max(L, 0), tab.shape[1] * page)) if R.page_of(tab, pages, page, b, t) is not None]
        if not tokens or hi == lo:
            continue
        at = torch.tensor([R.page_of(tab, pages, page, b, t) for t in tokens], dtype=torch.long)
        t = torch.tensor(tokens, dtype=torch.long)
        pos = L - (hi - lo) + torch.arange(hi - lo)
        seen = t[None] <= pos[:, None]
        if window:
            seen &= t[None] > pos[:, None] - window
        for h in range(q.shape[1]):
            g = h // group
            d = vp[at, t % page, g].double().nan_to_num(0).abs()
            e = held(ve[at, g]).double()
            top = torch.where(seen, e, -math.inf).amax(1)
            big = torch.where(seen[..., None], (d * (2.0 ** e)[:, None])[None], 0.0).amax(1) if t.numel() * (hi - lo) * d.shape[1] < 2 ** 24 else (d * (2.0 ** e)[:, None]).amax(0)[None]
            t_out[lo:hi, h] += 2 * 4 * 80 * u * big + 2.0 ** -31 * (2.0 ** top)[:, None].nan_to_num(0, 0, 0) * (seen.double() @ d)
    return out, lse, t_out, t_lse + 4 * 80 * u


def plan(table, free, n_free, seq_len, change, page, rows):
    """paged_plan on lists: (table, free list, count, lengths, q_start, slots, positions)."""
    table, free = [list(r) for r in table], list(free)
    B, per, F = len(table), len(table[0]), len(free)
    count = min(max(n_free, 0), F)
    cap = per * page
    lens = [min(max(x, 0), cap) for x in seq_len]
    want = [lens[b] + change[b] for b in range(B)]
    back = []
    for b in range(B):
        if want[b] <= cap:
            want[b] = max(want[b], 0)
            for i in range(-(-want[b] // page), -(-lens[b] // page)):
                back.append(table[b][i])
                table[b][i] = -1
    for entry in reversed(back):
        if entry >= 0:
            if count < F:
                free[count] = entry
                count += 1
    start, slots, positions = [0], [], []
    pages_asked = rows_asked = 0
    held_count, taken = count, 0
    for b in range(B):
        more, need = 0, 0
        if want[b] <= cap:
            more = max(want[b] - lens[b], 0)
            need = max(-(-want[b] // page) - -(-lens[b] // page), 0)
            pages_asked += need
            rows_asked += more
            if more and (pages_asked > held_count or rows_asked > rows):
                more = need = 0
                want[b] = lens[b]
        else:
            want[b] = lens[b]
        first = -(-lens[b] // page)
        for i in range(need):
            at = held_count - 1 - taken
            table[b][first + i] = free[at]
            free[at] = -1
            taken += 1
        for p in range(lens[b], lens[b] + more):
            entry = table[b][p // page]
            slots.append(entry * page + p % page if entry >= 0 else -1)
            positions.append(p)
        start.append(start[-1] + more)
        lens[b] = want[b]
    count -= taken
    rest = rows - len(slots)
    return table, free, count, lens, start, slots + [-1] * rest, positions + [-1] * rest


def verify(tokens, target, draft, uniform, draw, q_start):
    """verify_drafts in 64 bits, one sequence after another."""
    accepted, after = [], []
    V = target.shape[1]
    clean = lambda x: torch.where(x > 0, x, torch.zeros_like(x))  # noqa: E731  (NaN and below zero: zero)
    for b in range(len(q_start) - 1):
        r, end = int(q_start[b]), int(q_start[b + 1]) - 1
        first = r
        if end < r:
            accepted.append(0)
            after.append(-1)
            continue
        while r < end:
            t = int(tokens[r + 1])
            inside = 0 <= t < V
            p = float(target[r, t]) if inside else 0.0
            q = (1.0 if draft is None else float(draft[r, t])) if inside else 0.0
            if not float(uniform[r]) * q < p:
                break
            r += 1
        p = target[r].double()
        w = clean(p)
        if r < end:
            if draft is None:
                rest = w.clone()
                if 0 <= int(tokens[r + 1]) < V:
                    rest[int(tokens[r + 1])] = 0
            else:
                rest = clean(p - draft[r].double())
            if float(rest.sum()) > 0:
                w = rest
        c = w.cumsum(0)
        hit = torch.nonzero((c > float(draw[b]) * float(c[-1])) & (w > 0))
        some = torch.nonzero(w)
        after.append(int(hit[0]) if len(hit) else int(some[-1]) if len(some) else -1)
        accepted.append(r - first)
    return torch.tensor(accepted, dtype=torch.int32), torch.tensor(after, dtype=torch.int32)
