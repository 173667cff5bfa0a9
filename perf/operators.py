"""Cases of the 8-bit paged K/V cache and of the batch planning in front of it.

Kinds (the "kind" of a case):
  plan    page tables, slots and per-token lists of a batch, built from the requests' lengths
  append  K/V rows of a batch's new tokens quantised into the cache, and the pages that they
          touched read back as bf16
  attend  attention of a batch's new tokens over the cache: one token a row (a decode step), a
          few (drafts to be checked), or a prompt's chunk; all in one batch where they are mixed

The cache of one layer: codes uint8 [pages][Hkv][K|V][16 hd] hold e4m3 values, scales uint8
[pages][Hkv][K|V] the exponent of a power of two, 2^(scale - 127), for the 16 positions of a page.
  K: position t, feature d = 64 h + 16 g + j at byte ((h * 4 + g) * 16 + t) * 16 + j
  V: position t = 4 g + i, feature d = 64 h + 16 c + m at byte ((h * 4 + g) * 16 + m) * 16 + 4 c + i

Heads and lengths are those of the repository's model shapes and workloads (32 query heads over 8
KV heads, 40 over 8, 28 over 4, all of 128 features; the tiny model's 64).  K has channels of
different size, as keys after a projection and rotary positions do; V and the queries are N(0, 1).
"""
import math

import numpy as np
import torch

own = False

PAGE = 16
SPARE = 4  # pages of a table row past the longest request, as a serving program keeps


def listed():
    return [
        # the plan of a decode step of the benchmark's batch: latency alone
        {"name": "plan_step_64", "kind": "plan", "rows": 64, "lo": 512, "hi": 768, "new_lo": 1, "new_hi": 1},
        # 256 prompts admitted at once, the most rows that a step takes
        {"name": "plan_prompts_256", "kind": "plan", "rows": 256, "lo": 0, "hi": 0, "new_lo": 16, "new_hi": 2048},
        # a decode step's append: one token a row, each on a page that holds others already
        {"name": "append_step_64", "kind": "append", "hq": 32, "hkv": 8, "hd": 128, "rows": 64, "lo": 512, "hi": 768,
         "new_lo": 1, "new_hi": 1},
        # the append of 40 ragged prompt chunks, which begin and end inside pages
        {"name": "append_prompts_40", "kind": "append", "hq": 28, "hkv": 4, "hd": 128, "rows": 40, "lo": 0, "hi": 200,
         "new_lo": 100, "new_hi": 500},
        # one request decoded alone: the call's latency
        {"name": "attn_step_1", "kind": "attend", "hq": 32, "hkv": 8, "hd": 128, "rows": 1, "lo": 511, "hi": 511,
         "new_lo": 1, "new_hi": 1, "window": 0, "softcap": 0.0},
        # the benchmark's batch of 64 at contexts of 512 and up
        {"name": "attn_step_64", "kind": "attend", "hq": 32, "hkv": 8, "hd": 128, "rows": 64, "lo": 512, "hi": 768,
         "new_lo": 1, "new_hi": 1, "window": 0, "softcap": 0.0},
        # 128 ragged contexts, 5 query heads a KV head
        {"name": "attn_step_128_ragged", "kind": "attend", "hq": 40, "hkv": 8, "hd": 128, "rows": 128, "lo": 127,
         "hi": 2047, "new_lo": 1, "new_hi": 1, "window": 0, "softcap": 0.0},
        # the long-context workload's 32 rows: the cache is all that is read
        {"name": "attn_step_32_long", "kind": "attend", "hq": 32, "hkv": 8, "hd": 128, "rows": 32, "lo": 4095,
         "hi": 16383, "new_lo": 1, "new_hi": 1, "window": 0, "softcap": 0.0},
        # four drafted tokens a row checked at once, 7 query heads a KV head
        {"name": "attn_drafts_23", "kind": "attend", "hq": 28, "hkv": 4, "hd": 128, "rows": 23, "lo": 300, "hi": 5000,
         "new_lo": 4, "new_hi": 4, "window": 0, "softcap": 0.0},
        # one prompt from its start, of an odd length
        {"name": "attn_prompt_1", "kind": "attend", "hq": 28, "hkv": 4, "hd": 128, "rows": 1, "lo": 0, "hi": 0,
         "new_lo": 2001, "new_hi": 2001, "window": 0, "softcap": 0.0},
        # chunks of 2048 tokens of four long prompts: the most work of a call
        {"name": "attn_chunks_4", "kind": "attend", "hq": 32, "hkv": 8, "hd": 128, "rows": 4, "lo": 0, "hi": 6144,
         "new_lo": 2048, "new_hi": 2048, "window": 0, "softcap": 0.0},
        # a mixed batch: 20 decoding rows beside 4 chunks, heads of 64, sliding window, capped scores
        {"name": "attn_mixed_24", "kind": "attend", "hq": 16, "hkv": 2, "hd": 64, "rows": 24, "lo": 40, "hi": 4000,
         "new_lo": 300, "new_hi": 600, "single": 20, "window": 1024, "softcap": 30.0},
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _span(rng, lo, hi):
    a, b = _log_int(rng, lo, hi), _log_int(rng, lo, hi)
    return min(a, b), max(a, b)


def draw(rng):
    kind = rng.choices(["plan", "append", "step", "drafts", "prompt", "mixed"], [2, 2, 4, 1, 2, 1])[0]
    if kind == "plan":
        lo, hi = _span(rng, 1, 4000)
        a, b = (1, 1) if rng.random() < 0.4 else _span(rng, 1, 2000)
        return {"kind": kind, "rows": _log_int(rng, 1, 256), "lo": lo, "hi": hi, "new_lo": a, "new_hi": b}
    hq, hkv, hd = rng.choice([(32, 8, 128), (40, 8, 128), (28, 4, 128), (4, 2, 64), (16, 2, 64), (12, 12, 64)])
    c = {"kind": "append" if kind == "append" else "attend", "hq": hq, "hkv": hkv, "hd": hd}
    if kind == "append":
        rows = _log_int(rng, 1, 256)
        lo, hi = _span(rng, 1, 1000)
        a, b = (1, 1) if rng.random() < 0.4 else _span(rng, 1, max(2, 12000 // rows))
        return dict(c, rows=rows, lo=lo, hi=hi, new_lo=a, new_hi=b)
    if kind in ("step", "drafts"):
        rows = _log_int(rng, 1, 256 if kind == "step" else 40)
        lo, hi = _span(rng, 16, min(16383, 300000 // rows))
        new = 1 if kind == "step" else rng.randint(2, 6)
        c.update(rows=rows, lo=lo, hi=hi, new_lo=new, new_hi=new)
    elif kind == "prompt":
        rows = _log_int(rng, 1, 6)
        a, b = _span(rng, 32, 4096 // rows)
        lo, hi = (0, 0) if rng.random() < 0.4 else _span(rng, 1, 4000)
        c.update(rows=rows, lo=lo, hi=hi, new_lo=a, new_hi=b)
    else:
        rows = _log_int(rng, 4, 40)
        lo, hi = _span(rng, 16, 4000)
        a, b = _span(rng, 32, 500)
        c.update(rows=rows, lo=lo, hi=hi, new_lo=a, new_hi=b, single=rng.randint(1, rows - 1))
    c["window"] = rng.choice([0, 0, 0, _log_int(rng, 20, 2000)])
    c["softcap"] = rng.choice([0.0, 0.0, 0.0, 20.0, 50.0])
    return c


# ---------------------------------------------------------------- inputs


def _lengths(case):
    """Positions in the cache before the call and new tokens, row by row (in no seed's order)."""
    n, one = case["rows"], case.get("single", 0)
    ctx = np.linspace(case["lo"], case["hi"], n).astype(np.int64)
    new = np.ones(n, np.int64)
    new[one:] = np.linspace(case["new_lo"], case["new_hi"], n - one)[::-1].astype(np.int64)
    if one:  # the chunks are spread over the contexts
        new = new[np.argsort((np.arange(n) * 7919) % 10007, kind="stable")]
    return ctx, new


def _layout(case, seed):
    """Lengths in the seed's order, a page table of the rows' pages before the call (in a random
    order of the pool) and the free pages; every page of the pool is one or the other."""
    rng = np.random.RandomState(seed % (1 << 32))
    ctx, new = _lengths(case)
    order = rng.permutation(len(ctx))
    ctx, new = ctx[order], new[order]
    held = (ctx + PAGE - 1) // PAGE
    most = int((ctx + new + PAGE - 1).max()) // PAGE + SPARE
    n_free = int(((ctx + new + PAGE - 1) // PAGE - held).sum()) + 7
    pool = rng.permutation(int(held.sum()) + n_free).astype(np.int32)
    table = np.full((len(ctx), most), -1, np.int32)
    o = 0
    for r, k in enumerate(held):
        table[r, :k] = pool[o:o + k]
        o += k
    return ctx, new, table, pool[o:]


def _planned(ctx, new, table, free):
    """The page table with the new tokens' pages, taken from the end of the free pages."""
    table, o = table.copy(), len(free)
    for r in range(len(ctx)):
        a, b = -(-int(ctx[r]) // PAGE), -(-int(ctx[r] + new[r]) // PAGE)
        table[r, a:b] = free[o - (b - a):o][::-1]
        o -= b - a
    return table


def _i32(a):
    return torch.as_tensor(np.ascontiguousarray(a, np.int32)).cuda()


def _exponent(amax):
    """The scale byte of the largest magnitude of a page: the least power of two times 448 above it."""
    bits = amax.contiguous().view(torch.int32)
    return ((bits >> 23) - 8 + ((bits & 0x7fffff) > 0x600000).to(torch.int32)).clamp(16, 254)


def _pow2(byte):
    return (byte.to(torch.int32) << 23).view(torch.float32)


def _k_store(x):  # [..., 16, hd] -> [..., 16 hd] in the cache's order
    s = x.shape[:-2]
    return x.reshape(*s, 16, -1, 4, 16).movedim(-4, -2).reshape(*s, -1)


def _v_store(x):
    s = x.shape[:-2]
    n = len(s)
    y = x.reshape(*s, 4, 4, -1, 4, 16)  # g, i, h, c, m
    return y.permute(*range(n), n + 2, n, n + 4, n + 3, n + 1).reshape(*s, -1)


def _k_load(x):  # [..., 16 hd] -> [..., 16, hd]
    s = x.shape[:-1]
    return x.reshape(*s, -1, 4, 16, 16).movedim(-2, -4).reshape(*s, 16, -1)


def _v_load(x):
    s = x.shape[:-1]
    n = len(s)
    y = x.reshape(*s, -1, 4, 16, 4, 4)  # h, g, m, c, i
    return y.permute(*range(n), n + 1, n + 4, n, n + 3, n + 2).reshape(*s, 16, -1)


def _filled(n_pages, hkv, hd, g):
    """Codes and scales of a pool whose pages all hold 16 positions."""
    ch = torch.exp(0.5 * torch.randn((hkv, 1, hd), generator=g, device="cuda"))
    codes = torch.empty((n_pages, hkv, 2, 16 * hd), dtype=torch.uint8, device="cuda")
    scales = torch.empty((n_pages, hkv, 2), dtype=torch.uint8, device="cuda")
    for side, store in ((0, _k_store), (1, _v_store)):
        x = torch.randn((n_pages, hkv, 16, hd), generator=g, device="cuda")
        x = (x * ch if side == 0 else x).bfloat16().float()
        b = _exponent(x.abs().amax((2, 3)))
        x = (x * _pow2(254 - b)[:, :, None, None]).to(torch.float8_e4m3fn)
        codes[:, :, side] = store(x.view(torch.uint8))
        scales[:, :, side] = b.to(torch.uint8)
        del x
    return codes, scales, ch


def prepare(case, seed):
    ctx, new, table, free = _layout(case, seed)
    if case["kind"] == "plan":
        return {"case": case, "ctx": _i32(ctx), "new": _i32(new), "free": _i32(free), "n_free": _i32([len(free)]),
                "table": _i32(table), "max_tokens": int(new.sum()) + 5}
    hq, hkv, hd = case["hq"], case["hkv"], case["hd"]
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    n_pages = int((table >= 0).sum()) + len(free)
    codes, scales, ch = _filled(n_pages, hkv, hd, g)
    table = _planned(ctx, new, table, free)
    st = {"case": case, "codes": codes, "scales": scales}
    T = int(new.sum())
    if case["kind"] == "append":
        # k and v are the last columns of a QKV projection's rows
        qkv = torch.randn((T, hq + 2 * hkv, hd), generator=g, device="cuda")
        qkv[:, hq:hq + hkv] *= ch[:, 0]
        qkv = qkv.bfloat16()
        at = [(r, p) for r in range(len(ctx)) for p in range(ctx[r], ctx[r] + new[r])]
        back = [(r, p) for r in range(len(ctx)) for p in range(ctx[r] // PAGE * PAGE, ctx[r] + new[r])]
        slot = [np.array([table[r, p // PAGE] * PAGE + p % PAGE for r, p in x], np.int32) for x in (at, back)]
        st.update(k=qkv[:, hq:hq + hkv], v=qkv[:, hq + hkv:], slots=_i32(slot[0]), read=_i32(slot[1]))
        return st
    st.update(q=torch.randn((T, hq, hd), generator=g, device="cuda").bfloat16(), table=_i32(table),
              lens=_i32(ctx + new), cu=_i32(np.concatenate([[0], np.cumsum(new)])), max_new=int(new.max()),
              max_len=int((ctx + new).max()))
    return st


# ---------------------------------------------------------------- the passes


def run(st):
    kind = st["case"]["kind"]
    if own:
        from paper_2605_30218_amd import mg
        if kind == "plan":
            p = mg.batch_plan(st["ctx"], st["new"], st["free"], st["n_free"], st["table"], st["max_tokens"])
            return {"table": st["table"], "cu": p.cu_new, "lens": p.lens, "admitted": p.admitted,
                    "positions": p.positions, "rows": p.rows, "slots": p.slots, "n_left": p.n_left}
        if kind == "append":
            mg.kv8_append(st["codes"], st["scales"], st["k"], st["v"], st["slots"])
            k, v = mg.kv8_read(st["codes"], st["scales"], st["read"])
            return {"k": k, "v": v}
        return mg.kv8_attention(st["codes"], st["scales"], st["q"], st["table"], st["lens"], cu_new=st["cu"],
                                max_new=st["max_new"], max_len=st["max_len"], window=st["case"]["window"],
                                softcap=st["case"]["softcap"])
    return {"plan": _plan, "append": _append, "attend": _attend}[kind](st)


def _plan(st):
    ctx, new, table = st["ctx"].long(), st["new"].long(), st["table"]
    B, cap = table.shape
    dev = ctx.device
    valid = (ctx >= 0) & (new >= 0) & (ctx + new <= cap * PAGE)
    have = (ctx + PAGE - 1) // PAGE
    tok = torch.where(valid, new, 0)
    pages = torch.where(valid, (ctx + new + PAGE - 1) // PAGE - have, 0)
    ct, cp = tok.cumsum(0), pages.cumsum(0)
    ok = valid & (cp <= st["n_free"]) & (ct <= st["max_tokens"])
    tok, pages = tok * ok, pages * ok
    cu = torch.cat([torch.zeros(1, dtype=torch.long, device=dev), tok.cumsum(0)])
    pu = torch.cat([torch.zeros(1, dtype=torch.long, device=dev), pages.cumsum(0)])
    # the pages: entry (row, have + i) is the (pu[row] + i)-th from the end of the free list
    i = torch.arange(cap, device=dev)[None, :] - have[:, None]
    at = st["n_free"] - 1 - (pu[:-1, None] + i)
    table.copy_(torch.where((i >= 0) & (i < pages[:, None]), st["free"][at.clamp(0, len(st["free"]) - 1)], table))
    # the tokens
    t = torch.arange(st["max_tokens"], device=dev)
    live = t < cu[-1]
    row = torch.searchsorted(cu, t, right=True).clamp(max=B) - 1
    pos = ctx[row] + t - cu[row]
    slot = table[row, (pos // PAGE).clamp(0, cap - 1)] * PAGE + pos % PAGE
    put = lambda x: torch.where(live, x, -1).int()  # noqa: E731
    return {"table": table, "cu": cu.int(), "lens": (ctx.clamp(min=0) + tok).int(), "admitted": ok.int(),
            "positions": put(pos), "rows": put(row), "slots": put(slot), "n_left": (st["n_free"] - pu[-1]).int()}


def _append(st):
    codes, scales, slots, back = st["codes"], st["scales"], st["slots"].long(), st["read"].long()
    page, off = slots // PAGE, slots % PAGE
    out = {}
    old = scales.int()
    base = old.clone()
    base[page[off == 0]] = 0  # a token at a page's first position starts the page anew
    new = base.clone()
    for side, name, x in ((0, "k", st["k"].float()), (1, "v", st["v"].float())):
        fine = torch.where(torch.isfinite(x), x.abs(), 0.0)
        need = _exponent(fine.amax(-1))
        idx = page[:, None].expand(-1, need.shape[1])
        new[:, :, side].scatter_reduce_(0, idx, need, "amax")
        load, store = (_k_load, _v_load)[side], (_k_store, _v_store)[side]
        held = load(codes[page, :, side]).view(torch.float8_e4m3fn).float()
        held = held * _pow2((127 + base - new).clamp(min=0)[page, :, side])[..., None, None]
        held = torch.where((base == new)[page, :, side][..., None, None], load(codes[page, :, side]),
                           held.to(torch.float8_e4m3fn).view(torch.uint8))
        held = torch.where((base == 0)[page, :, side][..., None, None], 0, held)
        mine = x * _pow2(254 - new[page, :, side])[..., None]
        mine = torch.where(torch.isfinite(x), mine, math.nan).to(torch.float8_e4m3fn).view(torch.uint8)
        body = torch.empty((codes.shape[0],) + held.shape[1:], dtype=torch.uint8, device=codes.device)
        body[page] = held
        body[page, :, off] = mine
        codes[page, :, side] = store(body[page])
        now = load(codes[back // PAGE, :, side]).view(torch.float8_e4m3fn).float()
        now = now[torch.arange(len(back), device=codes.device), :, back % PAGE]
        out[name] = (now * _pow2(new[back // PAGE, :, side])[..., None]).bfloat16()
    scales.copy_(new.to(torch.uint8))
    return out


def _attend(st):
    case, q, table, lens, cu = st["case"], st["q"], st["table"].long(), st["lens"].long(), st["cu"].long()
    codes, scales = st["codes"], st["scales"]
    dev = q.device
    T, hq, hd = q.shape
    hkv, B, M = codes.shape[1], len(lens), st["max_new"]
    used = (st["max_len"] + PAGE - 1) // PAGE
    pages = table[:, :used].clamp(min=0)
    kv = codes[pages]  # [B][used][Hkv][2][16 hd]
    sc = _pow2(scales[pages])[..., None, None]
    k = (_k_load(kv[:, :, :, 0]).view(torch.float8_e4m3fn).float() * sc[:, :, :, 0]).transpose(1, 2).reshape(B, hkv, -1, hd)
    v = (_v_load(kv[:, :, :, 1]).view(torch.float8_e4m3fn).float() * sc[:, :, :, 1]).transpose(1, 2).reshape(B, hkv, -1, hd)
    new = cu[1:] - cu[:-1]
    i = torch.arange(M, device=dev)
    tok = (cu[:-1, None] + i).clamp(max=T - 1)
    x = q[tok].float().reshape(B, M, hkv, hq // hkv, hd).permute(0, 2, 1, 3, 4).reshape(B, hkv, -1, hd)
    s = torch.matmul(x, k.transpose(2, 3)).reshape(B, hkv, M, hq // hkv, -1) * (1.0 / math.sqrt(hd))
    if case["softcap"]:
        s = torch.tanh(s / case["softcap"]) * case["softcap"]
    p = ((lens - new)[:, None] + i)[:, :, None]  # [B][M][1]
    j = torch.arange(used * PAGE, device=dev)
    see = (j <= p) & (j < lens[:, None, None])
    if case["window"]:
        see &= j > p - case["window"]
    see = see[:, None, :, None, :]
    s = s.masked_fill(~see, -math.inf)
    e = torch.exp(s - s.amax(-1, keepdim=True).clamp(min=-3e38))
    total = e.sum(-1, keepdim=True)
    o = torch.matmul(e.reshape(B, hkv, -1, e.shape[-1]), v).reshape(B, hkv, M, hq // hkv, hd)
    o = torch.where(total > 0, o / total, 0.0).permute(0, 2, 1, 3, 4).reshape(B, M, hq, hd)
    t = torch.arange(T, device=dev)
    row = torch.searchsorted(cu, t, right=True) - 1
    return o[row, t - cu[row]].bfloat16()


# ---------------------------------------------------------------- work


def work(case):
    ctx, new = _lengths(case)
    end = ctx + new
    T = float(new.sum())
    if case["kind"] == "plan":
        pages = float(((end + PAGE - 1) // PAGE - (ctx + PAGE - 1) // PAGE).sum())
        return {"bytes": 12.0 * (T + 5) + 8.0 * pages + 20.0 * len(ctx), "flops": 0.0}
    hq, hkv, hd = case["hq"], case["hkv"], case["hd"]
    if case["kind"] == "append":
        touched = float((-(-end // PAGE) - ctx // PAGE).sum())
        back = float((end - ctx // PAGE * PAGE).sum())
        # new rows read and coded; the touched pages' positions read and written as bf16
        return {"bytes": 2.0 * hkv * hd * (2 * T + T + back + 2 * back) + 4.0 * hkv * touched + 4.0 * (T + back),
                "flops": 0.0}
    w = case["window"] or 1 << 40
    seen = float((end - np.maximum(0, ctx - w + 1)).sum())
    pairs = 0.0
    for c, n in zip(ctx.tolist(), new.tolist()):
        p = np.arange(c, c + n)
        pairs += float(np.minimum(p + 1, w).sum())
    return {"bytes": 2.0 * hkv * hd * seen + (2.0 * hkv + 4.0) * seen / PAGE + 4.0 * T * hq * hd,
            "flops": 4.0 * hq * hd * pairs}


# ---------------------------------------------------------------- the same in 64 bits


def _e4m3(x):
    """The nearest e4m3 value of each float64, ties to even."""
    step = torch.exp2(torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(x / step) * step


def _values(codes, scales, page, head, side):
    """One page's positions of one head as float64 [16][hd], byte by byte as the layout says."""
    hd = codes.shape[-1] // 16
    t, d = torch.meshgrid(torch.arange(16), torch.arange(hd), indexing="ij")
    if side == 0:
        at = ((d // 16) * 16 + t) * 16 + d % 16
    else:
        at = ((d // 64 * 4 + t // 4) * 16 + d % 16) * 16 + d % 64 // 16 * 4 + t % 4
    c = codes[page, head, side][..., at.to(codes.device)].long()
    mant, ex = c & 7, (c >> 3) & 15
    mag = torch.where(ex == 0, mant.double() * 2.0 ** -9, (8 + mant).double() * torch.exp2(ex.double() - 10))
    mag = torch.where((c & 127) == 127, math.nan, mag)
    return torch.where(c >= 128, -mag, mag) * torch.exp2(scales[page, head, side].double() - 127)[..., None, None]


def exact(case, seed):
    st = prepare(case, seed)
    if case["kind"] == "plan":
        return None
    codes, scales, hkv = st["codes"], st["scales"], case["hkv"]
    if case["kind"] == "append":
        slots = st["slots"].cpu().numpy()
        back = st["read"].cpu().numpy()
        if len(slots) > 20000:
            return None
        page = torch.as_tensor(np.unique(slots // PAGE)).cuda()
        where = torch.full((codes.shape[0],), -1, dtype=torch.long, device="cuda")
        where[page] = torch.arange(len(page), device="cuda")
        out = {}
        s = torch.as_tensor(slots).long().cuda()
        for side, name in ((0, "k"), (1, "v")):
            x = st[name].double()
            rows = []
            for h in range(hkv):
                held = _values(codes, scales, page, h, side)
                wrote = torch.zeros(held.shape[:2], dtype=torch.bool, device="cuda")
                wrote[where[s // PAGE], s % PAGE] = True
                first = wrote[:, 0]
                fresh = torch.zeros_like(held)
                fresh[where[s // PAGE], s % PAGE] = x[:, h]
                top = fresh.abs().amax((1, 2))
                ex = torch.ceil(torch.log2((top / 448).clamp(min=2.0 ** -111))).clamp(min=-111)
                before = torch.where(first, -127.0, scales[page, h, side].double() - 127)
                ex = torch.maximum(ex, before)
                unit = torch.exp2(ex)[:, None, None]
                val = torch.where(wrote[..., None], fresh, held)
                grown = (ex > before)[:, None, None] | wrote[..., None]
                val = torch.where(grown, _e4m3(val / unit) * unit, val)
                b = torch.as_tensor(back).long().cuda()
                rows.append(val[where[b // PAGE], b % PAGE])
            out[name] = torch.stack(rows, 1)
        return out
    q, table = st["q"], st["table"].cpu().numpy()
    ctx, new, _, _ = _layout(case, seed)
    T, hq, hd = q.shape
    o = torch.zeros((T, hq, hd), dtype=torch.float64, device="cuda")
    t0 = 0
    G = hq // hkv
    for r in range(len(ctx)):
        c, n = int(ctx[r]), int(new[r])
        pg = torch.as_tensor(table[r, :-(-(c + n) // PAGE)]).long().cuda()
        seen = torch.arange(c + n, device="cuda")[None, :] - torch.arange(c, c + n, device="cuda")[:, None]
        seen = (seen <= 0) & (seen > -(case["window"] or 1 << 40))
        for h in range(hkv):
            k = _values(codes, scales, pg, h, 0).reshape(-1, hd)[:c + n]
            v = _values(codes, scales, pg, h, 1).reshape(-1, hd)[:c + n]
            x = q[t0:t0 + n, h * G:(h + 1) * G].double()
            s = (x.reshape(-1, hd) @ k.T.contiguous()).reshape(n, G, -1) / math.sqrt(hd)
            if case["softcap"]:
                s = case["softcap"] * torch.tanh(s / case["softcap"])
            w = torch.softmax(s.masked_fill(~seen[:, None, :], -math.inf), -1)
            o[t0:t0 + n, h * G:(h + 1) * G] = (w.reshape(n * G, -1) @ v).reshape(n, G, hd)
        t0 += n
    return o
