"""Timed cases of a serving step over a paged cache held in 8 bits: the operators around and on such pages.

Kinds of case, each one pass through the Python entry points:

  plan       paged_plan: the tokens that a batch of requests brings get their pages, rows and slots, and are taken back
             again (drafts that were rejected, sequences that have ended)
  append     paged_append with exponents: keys and values of new tokens into 8-bit pages, with head norms and rotation
  attention  attn_paged with exponents: the new tokens of every sequence attend to 8-bit pages
  verify     verify_drafts: drafted tokens against the target's probabilities, and the token after the accepted ones

8-bit pages hold e4m3 codes (3 bits of mantissa, at most 448) and, for every page and key/value head, the exponent of a
scale: a code c of page g and head h stands for c * 2^exp[g, h].  An exponent is the smallest e >= -40 with which the
largest value written to the page and head is at most 448 * 2^e; it never falls while the page fills, and where it rises
the codes before are rounded again to the new scale.  A pool of pages is [pages, page size, key/value heads, head dim]; row b
of the table [sequences, pages a sequence] names the pages of sequence b in order.  q_start [sequences + 1] says where each
sequence's new tokens start among the rows of a call, and seq_len [sequences] how many tokens it has with them.
"""
import math

import torch

own = False

DEV = "cuda"
TYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
E4M3 = torch.float8_e4m3fn
BASE = 500000.0
LOWEST, HIGHEST = -40, 40           # exponents of a page's scales


def listed():
    return [
        # One decoding step of a batch of 32: a token each, a page more for some; the smallest call.
        dict(name="plan_step", kind="plan", B=32, new=1, most=1, cap=4096, page=16),
        # 128 prompts of up to 2048 tokens come and, later, end.
        dict(name="plan_prompts", kind="plan", B=128, new=100, most=2048, cap=2048, page=16, whole=True),
        # One decoding step of a batch of 8, queries turned with the keys.
        dict(name="append_step", kind="append", B=8, new=1, most=1, cap=4096, page=16, Hq=32, Hkv=8, hd=128, dtype="f16",
             rope=True, norm=False, queries=True),
        # Prefill of four ragged prompts of a model with norms on its query and key heads.
        dict(name="append_prompts_norm", kind="append", B=4, new=2900, most=7777, cap=8192, page=64, Hq=32, Hkv=8, hd=128,
             dtype="bf16", rope=True, norm=True, queries=True),
        # float32 rows of three chunks that begin inside a page, heads of 64, no queries.
        dict(name="append_chunks_f32", kind="append", B=3, new=777, most=2050, cap=4401, page=32, Hq=16, Hkv=16, hd=64,
             dtype="f32", rope=True, norm=False, queries=False),
        # The smallest attention: one sequence, one token, a short context.
        dict(name="attn_one", kind="attention", B=1, new=1, most=1, least=701, cap=701, page=16, Hq=32, Hkv=8, hd=128,
             window=0, dtype="f16"),
        # One decoding step of a batch of eight long sequences.
        dict(name="attn_step", kind="attention", B=8, new=1, most=1, least=20000, cap=32768, page=16, Hq=32, Hkv=8, hd=128,
             window=0, dtype="bf16"),
        # Checking five drafted tokens in each of sixteen sequences, with a sliding window.
        dict(name="attn_draft_window", kind="attention", B=16, new=5, most=5, least=3000, cap=9000, page=32, Hq=12, Hkv=4,
             hd=128, window=4096, dtype="f16"),
        # A chunk of a long prompt over the pages filled before it.
        dict(name="attn_chunk", kind="attention", B=1, new=1024, most=1024, least=40000, cap=40000, page=64, Hq=32, Hkv=8,
             hd=128, window=0, dtype="bf16"),
        # Two whole prompts: every token attends to those before it.
        dict(name="attn_prompts", kind="attention", B=2, new=3500, most=4096, least=0, cap=4096, page=16, Hq=32, Hkv=8,
             hd=128, window=0, dtype="f16"),
        # Four drafts of one sequence against a small vocabulary, float16 probabilities.
        dict(name="verify_one", kind="verify", B=1, drafts=4, most=4, V=32000, dtype="f16", draft=True),
        # Three to seven drafts in each of 64 sequences against a large vocabulary of odd size.
        dict(name="verify_batch", kind="verify", B=64, drafts=3, most=7, V=131071, dtype="f32", draft=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["plan", "append", "append", "attention", "attention", "attention", "verify"])
    page = rng.choice([8, 16, 16, 32, 64, 128])
    if kind == "plan":
        B = _log_int(rng, 1, 600)
        most = rng.choice([1, _log_int(rng, 1, 100000 // B)])
        whole = rng.random() < 0.3
        return dict(kind=kind, B=B, new=max(1, most // 3), most=most, cap=most if whole else most + _log_int(rng, 1, 4000),
                    page=page, whole=whole)
    if kind == "verify":
        B = _log_int(rng, 1, 64)
        drafts = rng.randint(0, 4)
        return dict(kind=kind, B=B, drafts=drafts, most=rng.randint(drafts, 7), V=_log_int(rng, 100, 131071),
                    dtype=rng.choice(["f16", "bf16", "f32"]), draft=rng.random() < 0.7)
    Hkv, group = rng.choice([(8, 4), (8, 4), (8, 1), (4, 8), (6, 3), (2, 7), (1, 16)])
    hd = rng.choice([64, 128, 128, 128, 256])
    if kind == "append":
        B = _log_int(rng, 1, 32)
        most = _log_int(rng, 1, 16384 // B)
        norm = rng.random() < 0.5
        return dict(kind=kind, B=B, new=rng.choice([1, most]), most=most, cap=most + _log_int(rng, 1, 2000), page=page,
                    Hq=Hkv * group, Hkv=Hkv, hd=hd, dtype=rng.choice(["f16", "bf16", "f32"]), rope=rng.random() < 0.8,
                    norm=norm, queries=norm or rng.random() < 0.7)
    shape = rng.choice(["step", "step", "draft", "chunk", "mixed", "prompts"])
    case = dict(kind=kind, page=page, Hq=Hkv * group, Hkv=Hkv, hd=hd, dtype=rng.choice(["f16", "bf16"]),
                window=rng.choice([0, 0, 0, _log_int(rng, 16, 8192)]))
    if shape in ("step", "draft"):
        B = _log_int(rng, 1, 32)
        new = 1 if shape == "step" else rng.randint(2, 9)
        cap = new + _log_int(rng, 16, min(100000, 200000 // B))
        return dict(case, B=B, new=new, most=new, least=new + (cap - new) // 3, cap=cap)
    if shape == "chunk":
        new = _log_int(rng, 16, 1024)
        cap = new + _log_int(rng, 100, 30000)
        return dict(case, B=1, new=new, most=new, least=cap, cap=cap)
    if shape == "mixed":
        most = _log_int(rng, 16, 600)
        return dict(case, B=rng.randint(2, 8), new=1, most=most, least=most, cap=most + _log_int(rng, 100, 4000))
    B = rng.randint(1, 3)
    most = _log_int(rng, 10, 3000)
    return dict(case, B=B, new=max(1, most // 2), most=most, least=0, cap=most)


# ---------------------------------------------------------------- inputs

def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    return g


def _spread(B, lo, hi):
    """`hi` in the last of B sequences; in the others `lo` or, where that is above one, spread between the two."""
    spread = hi - lo if lo > 1 else 0
    return [hi if b == B - 1 else lo + int(spread * (0.618 * (b + 1) % 1)) for b in range(B)]


def _lengths(case, g):
    """New tokens and lengths of every sequence; one is as long as the cache holds."""
    B, n = case["B"], torch.tensor(_spread(case["B"], case["new"], case["most"]))
    least, cap = case.get("least", 0), case["cap"]
    L = (least + (cap - least) * torch.rand(B, generator=g, device=DEV).cpu()).long()
    if case.get("whole") or case["kind"] == "attention" and least == 0:      # whole prompts
        return n, n.clone()
    L[0] = cap
    return n, torch.maximum(L, n).clamp(min=1)


def _channels(n, g, outliers):
    scale = (torch.randn(n, generator=g, device=DEV) * (0.6 if outliers else 0.25)).exp()
    if outliers:
        scale[torch.randperm(n, generator=g, device=DEV)[: max(1, round(0.01 * n))]] *= 5
    return scale


def _rows(n, heads, hd, g, dtype, outliers=False):
    x = torch.randn((n, heads, hd), generator=g, device=DEV) * _channels(heads * hd, g, outliers).view(heads, hd)
    return x.to(dtype)


def _held(pages, page, Hkv, hd, g, outliers):
    """A filled 8-bit pool and its exponents."""
    x = _rows(pages * page, Hkv, hd, g, torch.float32, outliers).view(pages, page, Hkv, hd)
    e = _exponent(x.abs().amax((1, 3)).double())
    return (x * torch.ldexp(torch.ones_like(x[:, :1, :, :1]), -e[:, None, :, None])).to(E4M3), e.to(torch.int8)


def prepare(case, seed):
    g = _gen(seed)
    kind, B = case["kind"], case["B"]
    if kind == "verify":
        return _prepare_verify(case, g)
    page, cap = case["page"], case["cap"]
    n, L = _lengths(case, g)
    per = -(-cap // page)
    pages = B * per + 3
    order = torch.randperm(pages, generator=g, device=DEV).to(torch.int32)
    T = int(n.sum())
    state = dict(case=case, rows=T, longest=int(L.max()), most=int(n.max()))
    if kind == "plan":
        had = (L - n).to(DEV)
        table = order[: B * per].view(B, per).clone()
        gone = torch.arange(per, device=DEV) >= (-(-had // page))[:, None]
        free = torch.cat([table[gone], order[B * per:]])
        n_free = torch.tensor([free.numel()], device=DEV, dtype=torch.int32)
        table[gone] = -1
        return dict(state, table=table, free=torch.cat([free, torch.full((pages - free.numel(),), -1, device=DEV,
                                                                         dtype=torch.int32)]),
                    n_free=n_free, seq_len=had.to(torch.int32), new=n.to(DEV, torch.int32), back=-n.to(DEV, torch.int32))
    Hkv, hd = case["Hkv"], case["hd"]
    state["table"] = order[: B * per].view(B, per)
    state["seq_len"] = L.to(DEV, torch.int32)
    state["q_start"] = torch.cat([torch.zeros(1, dtype=torch.int64), n.cumsum(0)]).to(DEV, torch.int32)
    state["theta"] = BASE ** (torch.arange(hd // 2, device=DEV, dtype=torch.float64) * (-2.0 / hd))
    state["k_pages"], state["k_exp"] = _held(pages, page, Hkv, hd, g, True)
    state["v_pages"], state["v_exp"] = _held(pages, page, Hkv, hd, g, False)
    src = TYPES[case["dtype"]]
    if kind == "attention":
        state["q"] = _rows(T, case["Hq"], hd, g, src)
        return state
    state["k"], state["v"] = _rows(T, Hkv, hd, g, src, True), _rows(T, Hkv, hd, g, src)
    state["q"] = _rows(T, case["Hq"], hd, g, src) if case["queries"] else None
    weight = [1 + 0.2 * torch.randn(hd, generator=g, device=DEV) for _ in range(2)]
    state["k_norm"] = weight[0] if case["norm"] else None
    state["q_norm"] = weight[1] if case["norm"] and case["queries"] else None
    return state


def _prepare_verify(case, g):
    """Rows of a target and a draft model that agree in the main; drafts drawn from the draft's probabilities."""
    n = torch.tensor(_spread(case["B"], case["drafts"], case["most"])) + 1
    T, V, dtype = int(n.sum()), case["V"], TYPES[case["dtype"]]
    x = 2.5 * torch.randn((T, V), generator=g, device=DEV)
    target = torch.softmax(x, -1).to(dtype)
    x += 0.5 * torch.randn((T, V), generator=g, device=DEV)
    draft = torch.softmax(x, -1)
    at = torch.rand((T, 1), generator=g, device=DEV, dtype=torch.float64)
    drawn = torch.searchsorted(draft.double().cumsum(-1), at).clamp(max=V - 1)[:, 0]
    tokens = torch.cat([torch.zeros(1, device=DEV, dtype=torch.int64), drawn[:-1]]).to(torch.int32)
    return dict(case=case, tokens=tokens, target=target, draft=draft.to(dtype) if case["draft"] else None,
                uniform=torch.rand(T, generator=g, device=DEV), draw=torch.rand(case["B"], generator=g, device=DEV),
                q_start=torch.cat([torch.zeros(1, dtype=torch.int64), n.cumsum(0)]).to(DEV, torch.int32))


# ---------------------------------------------------------------- the plain forms

def _move(s, change):
    """One change of the requests' lengths: tables, free list and lengths in place; first rows, slots, positions."""
    page, table, free, T = s["case"]["page"], s["table"], s["free"], s["rows"]
    B, per = table.shape
    had, count = s["seq_len"].long(), s["n_free"].long()
    new = (had + change).clamp(min=0)
    old_pages, new_pages = -(-had // page), -(-new // page)
    i = torch.arange(per, device=DEV)
    spare = torch.arange(free.numel(), device=DEV)
    # the pages given back go on the list so that taking as many again brings them in the same order
    out = (i >= new_pages[:, None]) & (i < old_pages[:, None]) & (table >= 0)
    total = out.sum()
    rank = out.flatten().cumsum(0).view(B, per) - 1
    given = torch.where(out, count + total - 1 - rank, free.numel())
    free_more = torch.cat([free, free[:1]]).scatter(0, given.flatten(), table.flatten())[:-1]
    free.copy_(free_more)
    table.masked_fill_((i >= new_pages[:, None]) & (i < old_pages[:, None]), -1)
    count = count + total
    # who fits, in order
    fits = new <= per * page
    need = (new_pages - old_pages).clamp(min=0) * fits
    rows = (new - had).clamp(min=0) * fits
    served = (new <= had) | (fits & (need.cumsum(0) <= count) & (rows.cumsum(0) <= T))
    need, rows = need * served, rows * served
    first = need.cumsum(0) - need
    got = (i >= old_pages[:, None]) & (i < (old_pages + need)[:, None])
    at = (count - 1 - (first[:, None] + i - old_pages[:, None])).clamp(min=0, max=free.numel() - 1)
    table.copy_(torch.where(got, free[at], table))
    count = count - need.sum()
    free.masked_fill_(spare >= count, -1)
    s["n_free"].copy_(count)
    s["seq_len"].copy_(torch.where(served, new, had))
    q_start = torch.cat([torch.zeros_like(rows[:1]), rows.cumsum(0)])
    r = torch.arange(T, device=DEV)
    b = torch.searchsorted(q_start[1:], r, right=True)
    real = b < B
    b = b.clamp(max=B - 1)
    pos = s["seq_len"].long()[b] - q_start[b + 1] + r
    entry = table.long()[b, (pos // page).clamp(0, per - 1)]
    slots = torch.where(real & (entry >= 0), entry * page + pos % page, -1)
    return q_start.to(torch.int32), slots, torch.where(real, pos, -1).to(torch.int32)


def _plan(s):
    rows = _move(s, s["new"])
    _move(s, s["back"])
    return rows, s["table"], s["free"], s["n_free"], s["seq_len"]


def _places(s):
    """Sequence, position, page and slot of every new token."""
    n = (s["q_start"][1:] - s["q_start"][:-1]).long()
    rows, page = s["k"].shape[0], s["case"]["page"]
    b = torch.repeat_interleave(torch.arange(n.numel(), device=DEV), n, output_size=rows)
    pos = torch.arange(rows, device=DEV) - s["q_start"].long()[b] + (s["seq_len"].long() - n)[b]
    return pos, s["table"].long()[b, pos // page], pos % page


def _norm(x, w):
    return x if w is None else x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6) * w


def _turn(x, pos, theta):
    """x [rows, heads, hd] turned at its rows' positions."""
    a = pos[:, None].double() * theta
    c, s = a.cos().to(x.dtype)[:, None], a.sin().to(x.dtype)[:, None]
    lo, hi = x.chunk(2, -1)
    return torch.cat([lo * c - hi * s, hi * c + lo * s], -1)


def _exponent(a):
    """The smallest e with a <= 448 * 2^e, inside the range of exponents."""
    m, e = torch.frexp(a)
    return torch.where(a > 0, e - 9 + (m > 0.875), LOWEST).clamp(LOWEST, HIGHEST)


def _codes(x, e):
    """x * 2^-e in 8 bits, [..., hd] with exponents [...]."""
    return (x * torch.ldexp(torch.ones_like(x[..., :1]), -e[..., None])).clamp(-448, 448).float().to(E4M3).view(torch.uint8)


def _put(s, x, pages, exp, g, slot):
    """New rows x (64 bits, next to the borders between codes and exponents) to their places."""
    page, raw = s["case"]["page"], pages.view(torch.uint8)
    n = (s["q_start"][1:] - s["q_start"][:-1]).long()
    at0 = s["seq_len"].long() - n                                # where every sequence's new tokens begin
    edge = s["table"].long().gather(1, (at0 // page).clamp(max=s["table"].shape[1] - 1)[:, None])[:, 0]
    kept = (at0 % page > 0) & (n > 0)
    peak = torch.zeros(exp.shape, device=DEV, dtype=torch.float64)
    peak.scatter_reduce_(0, g[:, None].expand(-1, exp.shape[1]), x.abs().amax(-1), "amax")
    old = exp[edge].clamp(LOWEST, HIGHEST).int()
    after = _exponent(peak)
    after[edge] = torch.where(kept[:, None], torch.maximum(after[edge], old), after[edge])
    # codes in front of the new ones, again under the new scale
    front = raw[edge].view(E4M3).float()                         # [B, page, Hkv, hd]
    moved = _codes(front, (after[edge] - old)[:, None].expand(-1, page, -1))
    mine = (kept[:, None] & (torch.arange(page, device=DEV) < (at0 % page)[:, None]))[..., None, None]
    raw[edge] = torch.where(mine, moved, raw[edge])
    raw[g, slot] = _codes(x, after[g])
    exp[g] = after[g].to(torch.int8)


def _append(s):
    pos, g, slot = _places(s)
    theta = s["theta"] if s["case"]["rope"] else None
    k = _norm(s["k"].double(), s["k_norm"])
    _put(s, k if theta is None else _turn(k, pos, theta), s["k_pages"], s["k_exp"], g, slot)
    _put(s, s["v"].double(), s["v_pages"], s["v_exp"], g, slot)
    q = None
    if s["q"] is not None:
        q = _norm(s["q"].float(), s["q_norm"])
        q = (q if theta is None else _turn(q, pos, theta)).to(_query_type(s))
    return q, s["k_pages"], s["v_pages"], s["k_exp"], s["v_exp"]


def _query_type(s):
    return torch.bfloat16 if s["q"].dtype is torch.float32 else s["q"].dtype


def _cache(s, pages, exp):
    """The pages of every sequence in order: [sequences, heads, tokens, head dim] in 32 bits."""
    per = -(-s["longest"] // s["case"]["page"])
    at = s["table"][:, :per].long()
    x = pages.view(torch.uint8)[at].view(E4M3).float()
    x = torch.ldexp(x, exp[at].int()[:, :, None, :, None])
    return x.flatten(1, 2)[:, : s["longest"]].transpose(1, 2)


def _attention(s):
    case = s["case"]
    B, Hq, Hkv, hd = case["B"], case["Hq"], case["Hkv"], case["hd"]
    start, L, T = s["q_start"].long(), s["seq_len"].long(), s["q"].shape[0]
    n = start[1:] - start[:-1]
    i = torch.arange(s["most"], device=DEV)
    at = start[:-1, None] + i                                    # [B, most]
    held = i < n[:, None]
    pos = (L - n)[:, None] + i
    j = torch.arange(s["longest"], device=DEV)
    seen = held[..., None] & (j <= pos[..., None])               # [B, most, tokens]
    if case["window"]:
        seen &= j > pos[..., None] - case["window"]
    q = s["q"][at.clamp(max=T - 1)].float().view(B, s["most"], Hkv, Hq // Hkv, hd).permute(0, 2, 3, 1, 4)
    k, v = _cache(s, s["k_pages"], s["k_exp"]), _cache(s, s["v_pages"], s["v_exp"])
    x = torch.matmul(q.reshape(B, Hkv, -1, hd), k.transpose(2, 3).contiguous()).view(B, Hkv, Hq // Hkv, s["most"], -1)
    x = (x * hd ** -0.5).masked_fill_(~seen[:, None, None], -math.inf)
    m = x.amax(-1, keepdim=True).clamp(min=torch.finfo(torch.float32).min)
    x = x.sub_(m).exp_()
    l = x.sum(-1, keepdim=True)
    o = torch.matmul(x.flatten(2, 3), v.contiguous()).view(B, Hkv, Hq // Hkv, s["most"], hd) / l
    o = o.permute(0, 3, 1, 2, 4).reshape(B, s["most"], Hq, hd)
    lse = (m + l.log())[..., 0].permute(0, 3, 1, 2).reshape(B, s["most"], Hq)
    out = torch.zeros((T, Hq, hd), device=DEV, dtype=s["q"].dtype)
    total = torch.zeros((T, Hq), device=DEV)
    out[at[held]], total[at[held]] = o[held].to(out.dtype), lse[held]
    return out, total


def _verify(s):
    """64 bits: sums over a vocabulary, and draws next to the borders between tokens."""
    start, tokens, target, draft = s["q_start"].long(), s["tokens"].long(), s["target"], s["draft"]
    T, V = target.shape
    B = start.numel() - 1
    n = start[1:] - start[:-1]
    b = torch.repeat_interleave(torch.arange(B, device=DEV), n, output_size=T)
    last = torch.arange(T, device=DEV) == start[b + 1] - 1
    t = tokens.roll(-1)[:, None]                                 # the draft that a row's probabilities are for
    p = target.gather(1, t)[:, 0].double()
    q = torch.ones_like(p) if draft is None else draft.gather(1, t)[:, 0].double()
    stops = last | ~(s["uniform"].double() * q < p)
    row = torch.arange(T, device=DEV)
    stop = torch.full((B,), T, device=DEV).scatter_reduce_(0, b, torch.where(stops, row, T), "amin")
    w = target[stop].double()
    if draft is None:
        less = torch.zeros_like(w).scatter_(1, t[stop], torch.finfo(torch.float64).max)
    else:
        less = draft[stop].double()
    rest = (w - less).clamp(min=0)
    plain = last[stop] | (rest.sum(-1) == 0)
    w = torch.where(plain[:, None], w, rest)
    c = w.cumsum(-1)
    token = torch.searchsorted(c, s["draw"].double()[:, None] * c[:, -1:], right=True)[:, 0]
    top = torch.where(w > 0, torch.arange(V, device=DEV), -1).amax(-1)
    return (stop - start[:-1]).to(torch.int32), torch.minimum(token, top).to(torch.int32)


# ---------------------------------------------------------------- one pass

def run(state):
    kind = state["case"]["kind"]
    if not own:
        return {"plan": _plan, "append": _append, "attention": _attention, "verify": _verify}[kind](state)
    from paper_2607_01065_amd import gsrq
    s = state
    if kind == "plan":
        rows = gsrq.paged_plan(s["table"], s["free"], s["n_free"], s["seq_len"], s["new"], page_size=s["case"]["page"],
                               rows=s["rows"])
        gsrq.paged_plan(s["table"], s["free"], s["n_free"], s["seq_len"], s["back"], page_size=s["case"]["page"],
                        rows=s["rows"])
        return rows, s["table"], s["free"], s["n_free"], s["seq_len"]
    if kind == "append":
        q = gsrq.paged_append(s["k"], s["v"], s["k_pages"], s["v_pages"], s["table"], s["q_start"], s["seq_len"], q=s["q"],
                              theta=s["theta"] if s["case"]["rope"] else None, k_norm=s["k_norm"], q_norm=s["q_norm"],
                              eps=1e-6, k_exp=s["k_exp"], v_exp=s["v_exp"])
        return q, s["k_pages"], s["v_pages"], s["k_exp"], s["v_exp"]
    if kind == "attention":
        return gsrq.attn_paged(s["q"], s["k_pages"], s["v_pages"], s["table"], s["q_start"], s["seq_len"],
                               window=s["case"]["window"], lse=True, k_exp=s["k_exp"], v_exp=s["v_exp"])
    return gsrq.verify_drafts(s["tokens"], s["target"], s["draft"], s["uniform"], s["draw"], s["q_start"])


# ---------------------------------------------------------------- what a pass cannot do without

def work(case):
    """Lengths that prepare() draws count with their mean."""
    B = case["B"]
    size = {"f16": 2, "bf16": 2, "f32": 4}
    if case["kind"] == "verify":
        T = sum(_spread(B, case["drafts"], case["most"])) + B
        rows = B * (2 if case["draft"] else 1)                  # one row of each model, and the drafts' own entries
        return {"bytes": int(rows * case["V"] * size[case["dtype"]] + T * 16), "flops": int(3 * B * case["V"])}
    new = _spread(B, case["new"], case["most"])
    T = sum(new)
    if case["kind"] == "plan":
        entries = sum(-(-n // case["page"]) for n in new)
        return {"bytes": int(2 * (8 * entries + 12 * T + 20 * B)), "flops": int(2 * (4 * T + 8 * B))}
    hd, Hkv = case["hd"], case["Hkv"]
    if case["kind"] == "append":
        held = T * 2 * Hkv * hd
        queries = T * case["Hq"] * hd if case["queries"] else 0
        s = size[case["dtype"]]
        return {"bytes": int(held * (s + 1) + queries * (s + 2)), "flops": int((held + queries) * (5 + 4 * case["norm"]))}
    seen, read = 0.0, 0.0
    for b, n in enumerate(new):
        has = n
        if case["least"]:
            has = max(n, case["cap"] if b == 0 else (case["least"] + case["cap"]) / 2)
        w = case["window"] or has
        # a token at position p sees min(w, p + 1): the last `full` of the n new ones see w, those before them p + 1
        full = max(0.0, min(n, has - w))
        seen += full * w + (n - full) * (2 * has - n - full + 1) / 2
        read += min(has, w + n - 1)
    return {"bytes": int(2 * read * Hkv * (hd + 1 / case["page"]) + 2 * T * case["Hq"] * hd * 2 + T * case["Hq"] * 4),
            "flops": int(4 * seen * case["Hq"] * hd)}


# ---------------------------------------------------------------- 64 bits

def _rope64(x, p, theta):
    h = x.shape[-1] // 2
    z = torch.complex(x[..., :h].contiguous(), x[..., h:].contiguous())
    turn = torch.polar(torch.ones_like(theta), torch.remainder(p.double().unsqueeze(-1) * theta, 2 * math.pi))
    z = z * turn.unsqueeze(-2)
    return torch.cat([z.real, z.imag], dim=-1)


def _rms64(x, w):
    return x if w is None else x / (x.pow(2).sum(-1, keepdim=True) / x.shape[-1] + 1e-6).sqrt() * w.double()


def _exact_plan(s):
    """On lists; the batch grows and shrinks back to what it was."""
    page, T = s["case"]["page"], s["rows"]
    table, free = s["table"].tolist(), s["free"].tolist()
    free = free[: int(s["n_free"])]
    lens, new = s["seq_len"].tolist(), s["new"].tolist()
    start, slots, positions = [0], [], []
    for b, n in enumerate(new):
        for p in range(lens[b], lens[b] + n):
            if p % page == 0:
                table[b][p // page] = free.pop()
            slots.append(table[b][p // page] * page + p % page)
            positions.append(p)
        start.append(start[-1] + n)
    rest = T - len(slots)
    i32 = dict(device=DEV, dtype=torch.int32)
    rows = (torch.tensor(start, **i32), torch.tensor(slots + [-1] * rest, device=DEV), torch.tensor(positions + [-1] * rest, **i32))
    return rows, s["table"], s["free"], s["n_free"], s["seq_len"]


def _exact_append(s, case):
    page, start, lens = case["page"], s["q_start"].tolist(), s["seq_len"].tolist()
    table = s["table"].tolist()
    q = None if s["q"] is None else _rms64(s["q"].double(), s["q_norm"])
    done = []
    for rows, pages, exp, keys in ((s["k"], s["k_pages"], s["k_exp"], True), (s["v"], s["v_pages"], s["v_exp"], False)):
        rows = _rms64(rows.double(), s["k_norm"] if keys else None)
        codes, e = pages.double(), exp.long()
        for b, n in enumerate(lens):
            lo, hi = start[b], start[b + 1]
            t = torch.arange(n - (hi - lo), n, device=DEV)
            x = _rope64(rows[lo:hi], t, s["theta"]) if keys and case["rope"] else rows[lo:hi]
            if keys and q is not None and case["rope"]:
                q[lo:hi] = _rope64(q[lo:hi], t, s["theta"])
            for i in range((n - (hi - lo)) // page, -(-n // page)):
                g, first = table[b][i], max(0, n - (hi - lo) - i * page)
                y = x[max(0, i * page - (n - (hi - lo))): (i + 1) * page - (n - (hi - lo))]
                top = y.abs().amax((0, 2))
                # powers of two around the quotient's logarithm, each tried
                want = torch.floor(torch.log2(top.clamp(min=1e-30) / 448)).long().clamp(LOWEST, HIGHEST)
                want = torch.where(top > 448 * 2.0 ** want, want + 1, want)
                want = torch.where(top > 448 * 2.0 ** want, want + 1, want).clamp(LOWEST, HIGHEST)
                if first:
                    want = torch.maximum(want, e[g])
                    codes[g, :first] *= (2.0 ** (e[g] - want))[None, :, None]
                codes[g, first: first + len(y)] = y / (2.0 ** want)[None, :, None]
                e[g] = want
        done.append((codes, e.to(torch.int8)))
    return q, done[0][0], done[1][0], done[0][1], done[1][1]


def _exact_attention(s, case):
    page, hd, Hkv = case["page"], case["hd"], case["Hkv"]
    lens, start, table = s["seq_len"].tolist(), s["q_start"].tolist(), s["table"].long()
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    lse = torch.zeros(s["q"].shape[:2], dtype=torch.float64, device=DEV)
    group = case["Hq"] // Hkv
    for b, n in enumerate(lens):
        first = start[b]
        new = start[b + 1] - first
        t = torch.arange(n, device=DEV)
        g, o = table[b][t // page], t % page
        K, V = (p.view(torch.uint8)[g, o].view(E4M3).double() * (2.0 ** e[g].double())[..., None]
                for p, e in ((s["k_pages"], s["k_exp"]), (s["v_pages"], s["v_exp"])))
        for lo in range(0, new, 256):
            hi = min(new, lo + 256)
            at = n - new + torch.arange(lo, hi, device=DEV)
            hide = t[None] > at[:, None]
            if case["window"]:
                hide |= t[None] <= at[:, None] - case["window"]
            for h in range(case["Hq"]):
                z = s["q"][first + lo: first + hi, h].double() @ K[:, h // group].T.contiguous() / math.sqrt(hd)
                z[hide] = -math.inf
                total = torch.logsumexp(z, dim=1)
                lse[first + lo: first + hi, h] = total
                out[first + lo: first + hi, h] = torch.exp(z - total[:, None]) @ V[:, h // group].contiguous()
    return out, lse


def _exact_verify(s):
    start = s["q_start"].tolist()
    tokens, u, draw = s["tokens"].tolist(), s["uniform"].tolist(), s["draw"].tolist()
    accepted, after = [], []
    for b in range(len(start) - 1):
        r, end = start[b], start[b + 1] - 1
        while r < end:
            t = tokens[r + 1]
            p, q = float(s["target"][r, t]), 1.0 if s["draft"] is None else float(s["draft"][r, t])
            if not u[r] * q < p:
                break
            r += 1
        w = s["target"][r].double()
        if r < end:
            rest = w.clone()
            if s["draft"] is None:
                rest[tokens[r + 1]] = 0
            else:
                rest -= s["draft"][r].double()
            rest[rest < 0] = 0
            w = rest if bool(rest.any()) else w
        c = torch.cumsum(w.cpu(), 0)
        beyond = torch.nonzero(c > draw[b] * float(c[-1]))
        after.append(int(beyond[0]) if len(beyond) else int(torch.nonzero(w.cpu())[-1]))
        accepted.append(r - start[b])
    return torch.tensor(accepted, device=DEV, dtype=torch.int32), torch.tensor(after, device=DEV, dtype=torch.int32)


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "plan":
        return _exact_plan(s)
    if case["kind"] == "append":
        return _exact_append(s, case)
    if case["kind"] == "attention":
        return _exact_attention(s, case)
    return _exact_verify(s)
