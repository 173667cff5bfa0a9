"""Cases of the 4-bit paged K/V cache (rotation and append, attention) and of token log probabilities.

Kinds (the "kind" of a case):
  append  q and k rows of a batch's new tokens rotated by their positions, k and v quantised into the
          cache; the pages that they touched are read back as bf16
  attend  attention of a batch's new tokens over the cache: one token a row (a decode step), a few
          (drafts to be checked), or a prompt's chunk; all in one batch where they are mixed
  logp    log probabilities of given tokens from rows of logits, the rows' entropies and their top
          alternatives

The cache of one layer: codes uint8 [pages][Hkv][K|V][8 hd] hold e2m1 values (0, 1/2, 1, 3/2, 2, 3, 4, 6 and a sign),
two a byte, the low nibble first; scales uint8 [pages][Hkv][hd / 2 + 16] the exponent of a power of two,
2^(scale - 127).
  K: position t, feature d = 32 g + j at byte (g * 16 + t) * 16 + j / 2, nibble j % 2; its scale at byte g * 16 + t
  V: position t = 4 g + i, feature d = 16 c + m at byte (g * 16 + m) * hd / 8 + 2 c + i / 2, nibble i % 2; its scale
     at byte hd / 2 + t
So a scale serves 32 features of a position's key, or a position's whole value; it is the least power of two, from
2^-111, whose sevenfold holds the largest magnitude (6.. 7 become 6), and 255 where something is not finite.

Rotation: the pair (i, i + hd / 2) of a head at position p becomes (a c - b s, b c + a s) with c, s = table[p][2 i], [2 i + 1],
products and sums each rounded to 32 bits, and the result to bf16.

Heads and lengths are those of the repository's model shapes and workloads (32 query heads over 8
KV heads, 40 over 8, 28 over 4, all of 128 features; the tiny model's 64), vocabularies theirs and generic ones.
K has channels of different size, as keys after a projection do; V and the queries are N(0, 1).
"""
import math

import numpy as np
import torch

own = False

PAGE = 16
SPARE = 4  # pages of a table row past the longest request, as a serving program keeps


def listed():
    return [
        # a decode step's rotation and append: one token a row, each on a page that holds others already
        {"name": "append_step_64", "kind": "append", "hq": 32, "hkv": 8, "hd": 128, "rows": 64, "lo": 512, "hi": 768,
         "new_lo": 1, "new_hi": 1},
        # 40 ragged prompt chunks, which begin and end inside pages
        {"name": "append_prompts_40", "kind": "append", "hq": 28, "hkv": 4, "hd": 128, "rows": 40, "lo": 0, "hi": 200,
         "new_lo": 100, "new_hi": 500},
        # drafts of a few tokens, heads of 64
        {"name": "append_drafts_9", "kind": "append", "hq": 16, "hkv": 2, "hd": 64, "rows": 9, "lo": 3, "hi": 1000,
         "new_lo": 3, "new_hi": 7},
        # one request decoded alone: the call's latency
        {"name": "attn_step_1", "kind": "attend", "hq": 32, "hkv": 8, "hd": 128, "rows": 1, "lo": 511, "hi": 511,
         "new_lo": 1, "new_hi": 1, "window": 0, "softcap": 0.0},
        # the benchmark's batch of 64 at contexts of 512 and up
        {"name": "attn_step_64", "kind": "attend", "hq": 32, "hkv": 8, "hd": 128, "rows": 64, "lo": 512, "hi": 768,
         "new_lo": 1, "new_hi": 1, "window": 0, "softcap": 0.0},
        # 32 rows of long, ragged contexts: the cache is all that is read
        {"name": "attn_step_32_long", "kind": "attend", "hq": 40, "hkv": 8, "hd": 128, "rows": 32, "lo": 4095,
         "hi": 16383, "new_lo": 1, "new_hi": 1, "window": 0, "softcap": 0.0},
        # four drafted tokens a row checked at once, 7 query heads a KV head
        {"name": "attn_drafts_23", "kind": "attend", "hq": 28, "hkv": 4, "hd": 128, "rows": 23, "lo": 300, "hi": 5000,
         "new_lo": 4, "new_hi": 4, "window": 0, "softcap": 0.0},
        # chunks of 2048 tokens of four long prompts: the most work of a call
        {"name": "attn_chunks_4", "kind": "attend", "hq": 32, "hkv": 8, "hd": 128, "rows": 4, "lo": 0, "hi": 6144,
         "new_lo": 2048, "new_hi": 2048, "window": 0, "softcap": 0.0},
        # a mixed batch: 20 decoding rows beside 4 chunks, heads of 64, sliding window, capped scores
        {"name": "attn_mixed_24", "kind": "attend", "hq": 16, "hkv": 2, "hd": 64, "rows": 24, "lo": 40, "hi": 4000,
         "new_lo": 300, "new_hi": 600, "single": 20, "window": 1024, "softcap": 30.0},
        # one answer's token with five alternatives: latency
        {"name": "logp_step_1", "kind": "logp", "rows": 1, "vocab": 128256, "pad": 0, "bf16": False, "top": 5, "masked": 0.0},
        # the benchmark's batch, a step's answers with 20 alternatives; a tenth of the vocabulary is masked
        {"name": "logp_step_64", "kind": "logp", "rows": 64, "vocab": 128256, "pad": 0, "bf16": False, "top": 20, "masked": 0.1},
        # a prompt of 2001 tokens scored from 16-bit logits
        {"name": "logp_prompt_2001", "kind": "logp", "rows": 2001, "vocab": 152064, "pad": 0, "bf16": True, "top": 8,
         "masked": 0.0},
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _span(rng, lo, hi):
    a, b = _log_int(rng, lo, hi), _log_int(rng, lo, hi)
    return min(a, b), max(a, b)


def draw(rng):
    kind = rng.choices(["append", "step", "drafts", "prompt", "mixed", "logp"], [3, 3, 1, 2, 1, 3])[0]
    if kind == "logp":
        rows = _log_int(rng, 1, 2001)
        vocab = _log_int(rng, 500, 152064)
        return {"kind": kind, "rows": rows, "vocab": vocab, "pad": rng.choice([0, 0, 1, 5, 64]),
                "bf16": rng.random() < 0.5, "top": rng.choice([0, 1, 5, 8, 20, 20]), "masked": rng.choice([0.0, 0.0, 0.3, 0.999])}
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
    """Lengths in the seed's order and a page table of the rows' pages, in a random order of the pool."""
    rng = np.random.RandomState(seed % (1 << 32))
    ctx, new = _lengths(case)
    order = rng.permutation(len(ctx))
    ctx, new = ctx[order], new[order]
    held = (ctx + new + PAGE - 1) // PAGE
    pool = rng.permutation(int(held.sum()) + 7).astype(np.int32)
    table = np.full((len(ctx), int(held.max()) + SPARE), -1, np.int32)
    o = 0
    for r, k in enumerate(held):
        table[r, :k] = pool[o:o + k]
        o += k
    return ctx, new, table, len(pool)


def _i32(a):
    return torch.as_tensor(np.ascontiguousarray(a, np.int32)).cuda()


def _rope(n, hd):
    """cos and sin of position times frequency, interleaved, [n][hd], from angles in 64 bits."""
    ang = np.arange(n)[:, None] * 500000.0 ** (-2.0 * np.arange(hd // 2) / hd)
    return torch.as_tensor(np.stack([np.cos(ang), np.sin(ang)], -1).reshape(n, hd).astype(np.float32)).cuda()


def _scale_byte(amax):
    """The scale byte of the largest magnitude of a block (NaN or infinity: 255)."""
    bits = amax.contiguous().view(torch.int32)
    b = ((bits >> 23) - 2 + ((bits & 0x7fffff) > 0x600000).to(torch.int32)).clamp(16, 254)
    return torch.where(torch.isfinite(amax), b, 255)


def _pow2(byte):
    return (byte.to(torch.int32) << 23).view(torch.float32)


def _code(y):
    """The nearest e2m1 value of each number as its four bits, ties to the even code."""
    a = y.abs()
    c = ((a > 0.25).int() + (a >= 0.75).int() + (a > 1.25).int() + (a >= 1.75).int() + (a > 2.5).int() + (a >= 3.5).int() +
         (a > 5.0).int())
    return (c + 8 * torch.signbit(y).int()).to(torch.uint8)


def _quantise(x, block):
    """Codes [..., hd] and scale bytes [..., hd / block] of rows of float32."""
    y = x.unflatten(-1, (-1, block))
    top = torch.where(torch.isfinite(y), y.abs(), math.inf).amax(-1)
    b = _scale_byte(top)
    unit = _pow2(254 - b.clamp(max=253))[..., None]
    return _code(torch.where((b == 255)[..., None], 0.0, y * unit)).flatten(-2), b.to(torch.uint8)


def _value(code):
    """The e2m1 value of four bits."""
    c = code.long()
    v = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device=code.device)[c & 7]
    return torch.where(c >= 8, -v, v)


def _unit(byte):
    """What a scale byte stands for; 255 is NaN, and nothing stored counts as the least."""
    return torch.where(byte == 255, math.nan, _pow2(byte.int().clamp(1, 254)))


def _k_codes(codes, hd):  # a view: [pages][Hkv][g][t][16 bytes]
    return codes[:, :, 0].view(*codes.shape[:2], hd // 32, 16, 16)


def _v_codes(codes, hd):  # a view: [pages][Hkv][g][m][c][2 bytes]
    return codes[:, :, 1].view(*codes.shape[:2], 4, 16, hd // 16, 2)


def _k_page(codes, scales):
    """Keys of pages: codes [..., 8 hd] and scales [..., hd / 2 + 16] -> float32 [..., 16, hd]."""
    hd = codes.shape[-1] // 8
    b = codes.unflatten(-1, (hd // 32, 16, 16)).transpose(-3, -2)  # [..., t, g, 16]
    x = _value(torch.stack([b & 15, b >> 4], -1)).flatten(-2)
    s = _unit(scales[..., :hd // 2].unflatten(-1, (hd // 32, 16)).transpose(-1, -2))
    return (x * s[..., None]).flatten(-2)


def _v_page(codes, scales):
    hd = codes.shape[-1] // 8
    b = codes.unflatten(-1, (4, 16, hd // 16, 2))  # g, m, c, byte
    x = _value(torch.stack([b & 15, b >> 4], -1)).flatten(-2)  # g, m, c, i
    n = x.dim() - 4
    x = x.permute(*range(n), n, n + 3, n + 2, n + 1).flatten(-2).flatten(-3, -2)  # [..., 16, hd]
    return x * _unit(scales[..., hd // 2:])[..., None]


def _put(codes, scales, page, t, k, v):
    """Rows of float32 [n, Hkv, hd] quantised into the cache at positions t of pages page."""
    hd = k.shape[-1]
    c, b = _quantise(k, 32)
    c = c.unflatten(-1, (hd // 32, 16, 2))
    _k_codes(codes, hd)[page, :, :, t] = c[..., 0] | c[..., 1] << 4
    scales[:, :, :hd // 2].unflatten(-1, (hd // 32, 16))[page, :, :, t] = b
    c, b = _quantise(v, hd)
    scales[:, :, hd // 2:][page, :, t] = b[..., 0]
    c = c.unflatten(-1, (hd // 16, 16)).transpose(-1, -2)  # [n, Hkv, m, c]
    # two positions share a byte: what a nibble changes by is added to it
    dev = codes.device
    at = (page[:, None, None, None], torch.arange(codes.shape[1], device=dev)[:, None, None], (t // 4)[:, None, None, None],
          torch.arange(16, device=dev)[:, None], torch.arange(hd // 16, device=dev), (t % 4 // 2)[:, None, None, None])
    up = (4 * (t % 2))[:, None, None, None]
    view = _v_codes(codes, hd)
    old = view[at].int() >> up & 15
    view.index_put_(at, (c.int() - old << up).to(torch.uint8), accumulate=True)


def _filled(n_pages, hkv, hd, g):
    """Codes and scales of a pool whose pages all hold 16 positions, and the sizes of K's channels."""
    ch = torch.exp(0.5 * torch.randn((hkv, 1, hd), generator=g, device="cuda"))
    codes = torch.empty((n_pages, hkv, 2, 8 * hd), dtype=torch.uint8, device="cuda")
    scales = torch.empty((n_pages, hkv, hd // 2 + 16), dtype=torch.uint8, device="cuda")
    x = (torch.randn((n_pages, hkv, 16, hd), generator=g, device="cuda") * ch).bfloat16().float()
    c, b = _quantise(x, 32)
    c = c.unflatten(-1, (hd // 32, 16, 2))
    codes[:, :, 0] = (c[..., 0] | c[..., 1] << 4).transpose(2, 3).flatten(2)
    scales[:, :, :hd // 2] = b.transpose(2, 3).flatten(2)
    x = torch.randn((n_pages, hkv, 16, hd), generator=g, device="cuda").bfloat16().float()
    c, b = _quantise(x, hd)
    scales[:, :, hd // 2:] = b[..., 0]
    c = c.unflatten(-1, (hd // 16, 16)).unflatten(2, (4, 2, 2))  # g, i / 2, i % 2, c, m
    codes[:, :, 1] = (c[:, :, :, :, 0] | c[:, :, :, :, 1] << 4).permute(0, 1, 2, 5, 4, 3).flatten(2)
    return codes, scales, ch


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    if case["kind"] == "logp":
        n, V = case["rows"], case["vocab"]
        x = torch.empty((n, V + case["pad"]), dtype=torch.bfloat16 if case["bf16"] else torch.float32, device="cuda")[:, :V]
        hot = torch.randint(0, V, (n, 40), generator=g, device="cuda")
        for a in range(0, n, 256):  # a few likely tokens above the rest
            y = 2.0 * torch.randn((len(x[a:a + 256]), V), generator=g, device="cuda")
            if case["masked"]:
                off = torch.rand((len(y), V), generator=g, device="cuda") < case["masked"]
                y.masked_fill_(off, -math.inf)
            y.scatter_reduce_(1, hot[a:a + 256], 14.0 * torch.rand((len(y), 40), generator=g, device="cuda"), "amax")
            x[a:a + 256] = y
        pick = torch.randint(0, 40, (n, 1), generator=g, device="cuda")
        return {"case": case, "logits": x, "tokens": hot.gather(1, pick)[:, 0].int()}
    ctx, new, table, n_pages = _layout(case, seed)
    hq, hkv, hd = case["hq"], case["hkv"], case["hd"]
    codes, scales, ch = _filled(n_pages, hkv, hd, g)
    st = {"case": case, "codes": codes, "scales": scales}
    T = int(new.sum())
    if case["kind"] == "append":
        # q, k and v are the columns of a QKV projection's rows
        qkv = torch.randn((T, hq + 2 * hkv, hd), generator=g, device="cuda")
        qkv[:, hq:hq + hkv] *= ch[:, 0]
        qkv = qkv.bfloat16()
        at = [(r, p) for r in range(len(ctx)) for p in range(ctx[r], ctx[r] + new[r])]
        back = [(r, p) for r in range(len(ctx)) for p in range(ctx[r] // PAGE * PAGE, ctx[r] + new[r])]
        slot = [np.array([table[r, p // PAGE] * PAGE + p % PAGE for r, p in x], np.int32) for x in (at, back)]
        st.update(q=qkv[:, :hq], k=qkv[:, hq:hq + hkv], v=qkv[:, hq + hkv:], slots=_i32(slot[0]), read=_i32(slot[1]),
                  positions=_i32([p for _, p in at]), rope=_rope(int((ctx + new).max()), hd))
        return st
    st.update(q=torch.randn((T, hq, hd), generator=g, device="cuda").bfloat16(), table=_i32(table),
              lens=_i32(ctx + new), cu=_i32(np.concatenate([[0], np.cumsum(new)])), max_new=int(new.max()),
              max_len=int((ctx + new).max()))
    return st


# ---------------------------------------------------------------- the passes


def run(st):
    case = st["case"]
    if own:
        from paper_2605_30218_amd import mg
        if case["kind"] == "logp":
            return mg.token_logprobs(st["logits"], st["tokens"], top=case["top"])._asdict()
        if case["kind"] == "append":
            q = mg.kv4_append(st["codes"], st["scales"], st["k"], st["v"], st["slots"], positions=st["positions"],
                              rope=st["rope"], q=st["q"])
            k, v = mg.kv4_read(st["codes"], st["scales"], st["read"])
            return {"q": q, "k": k, "v": v}
        return mg.kv4_attention(st["codes"], st["scales"], st["q"], st["table"], st["lens"], cu_new=st["cu"],
                                max_new=st["max_new"], max_len=st["max_len"], window=case["window"],
                                softcap=case["softcap"])
    return {"append": _append, "attend": _attend, "logp": _logp}[case["kind"]](st)


def _rotate(x, cs):
    h = x.shape[-1] // 2
    c, s = cs[:, None, 0::2], cs[:, None, 1::2]
    a, b = x[..., :h].float(), x[..., h:].float()
    return torch.cat([a * c - b * s, b * c + a * s], -1).bfloat16()


def _append(st):
    codes, scales, slots, back = st["codes"], st["scales"], st["slots"].long(), st["read"].long()
    cs = st["rope"][st["positions"].long()]
    q, k = _rotate(st["q"], cs), _rotate(st["k"], cs)
    _put(codes, scales, slots // PAGE, slots % PAGE, k.float(), st["v"].float())
    pg, t = back // PAGE, back % PAGE
    i = torch.arange(len(back), device=codes.device)
    out = {"q": q}
    for name, side, load in (("k", 0, _k_page), ("v", 1, _v_page)):
        out[name] = load(codes[pg, :, side], scales[pg])[i, :, t].bfloat16()
    return out


def _attend(st):
    case, q, table, lens, cu = st["case"], st["q"], st["table"].long(), st["lens"].long(), st["cu"].long()
    codes, scales = st["codes"], st["scales"]
    dev = q.device
    T, hq, hd = q.shape
    hkv, B, M = codes.shape[1], len(lens), st["max_new"]
    used = (st["max_len"] + PAGE - 1) // PAGE
    pages = table[:, :used].clamp(min=0)
    sc = scales[pages]
    k = _k_page(codes[pages, :, 0], sc).transpose(1, 2).reshape(B, hkv, -1, hd)  # [B][Hkv][positions][hd]
    v = _v_page(codes[pages, :, 1], sc).transpose(1, 2).reshape(B, hkv, -1, hd)
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


def _logp(st):
    logits, tokens, k = st["logits"], st["tokens"].long(), st["case"]["top"]
    out = {"logprob": [], "entropy": [], "top_tokens": [], "top_logprobs": []}
    for a in range(0, len(logits), 128):
        x, tok = logits[a:a + 128].float(), tokens[a:a + 128, None]
        m = x.amax(-1, keepdim=True)
        m = torch.where(m == -math.inf, 0.0, m)  # (a row that is masked whole: log probabilities of -inf, an entropy of 0)
        y = x - m
        e = torch.exp(y)
        s = e.sum(-1, keepdim=True, dtype=torch.float64)
        u = (e * y.clamp(min=-200.0)).sum(-1, keepdim=True, dtype=torch.float64)
        u = torch.where(s == 0, 0.0, u / s)
        ln = torch.where(s == 0, 0.0, torch.log(s))
        out["logprob"].append((y.gather(1, tok).double() - ln)[:, 0].float())
        out["entropy"].append((ln - u)[:, 0].float())
        val, idx = torch.sort(x, dim=-1, descending=True, stable=True)
        val, idx = val[:, :k], idx[:, :k]
        out["top_tokens"].append(torch.where(val == -math.inf, -1, idx).int())
        out["top_logprobs"].append(((val - m).double() - ln).float())
    return {n: torch.cat(x) for n, x in out.items()}


# ---------------------------------------------------------------- work


def work(case):
    if case["kind"] == "logp":
        n, V = case["rows"], case["vocab"]
        return {"bytes": n * ((2.0 if case["bf16"] else 4.0) * V + 12.0 + 8.0 * case["top"]), "flops": 6.0 * n * V}
    ctx, new = _lengths(case)
    end = ctx + new
    T = float(new.sum())
    hq, hkv, hd = case["hq"], case["hkv"], case["hd"]
    per = hkv * (hd + hd // 32 + 1.0)  # bytes of a position in the cache
    if case["kind"] == "append":
        back = float((end - ctx // PAGE * PAGE).sum())
        # rows and angles read, rotated q and codes written; the touched pages' positions read and written as bf16
        return {"bytes": T * (2.0 * (2 * hq + 2 * hkv) * hd + per + 8.0) + 4.0 * hd * float(end.max()) +
                back * (per + 4.0 * hkv * hd + 4.0), "flops": 3.0 * T * (hq + hkv) * hd}
    w = case["window"] or 1 << 40
    seen = float((end - np.maximum(0, ctx - w + 1)).sum())
    pairs = 0.0
    for c, n in zip(ctx.tolist(), new.tolist()):
        p = np.arange(c, c + n)
        pairs += float(np.minimum(p + 1, w).sum())
    return {"bytes": per * seen + 4.0 * seen / PAGE + 4.0 * T * hq * hd, "flops": 4.0 * hq * hd * pairs}


# ---------------------------------------------------------------- the same in 64 bits


def _e2m1(x):
    """The nearest e2m1 value of each float64, ties to even, 6 above."""
    step = torch.exp2(torch.floor(torch.log2(x.abs().clamp(min=1.0))) - 1)
    return (torch.round(x / step) * step).clamp(-6, 6)


def _held(codes, scales, page, head, side):
    """One page's positions of one head as float64 [16][hd], nibble by nibble as the layout says."""
    hd = codes.shape[-1] // 8
    t, d = torch.meshgrid(torch.arange(16), torch.arange(hd), indexing="ij")
    if side == 0:
        at, nib, sc = (d // 32 * 16 + t) * 16 + d % 32 // 2, d % 2, d // 32 * 16 + t
    else:
        at, nib, sc = (t // 4 * 16 + d % 16) * (hd // 8) + d // 16 * 2 + t % 4 // 2, t % 2, hd // 2 + t
    dev = codes.device
    c = codes[page, head, side][..., at.to(dev)].long() >> (4 * nib.to(dev)) & 15
    ex, m = c >> 1 & 3, c & 1
    mag = torch.where(ex == 0, 0.5 * m.double(), (2 + m).double() * torch.exp2(ex.double() - 2))
    b = scales[page, head][..., sc.to(dev)].double()
    return torch.where(c >= 8, -mag, mag) * torch.where(b == 255, math.nan, torch.exp2(b - 127))


def _stored(x, block):
    """What rows of float64 become in the cache."""
    y = x.reshape(*x.shape[:-1], -1, block)
    ex = torch.ceil(torch.log2(y.abs().amax(-1, keepdim=True).clamp(min=2.0 ** -130) / 7)).clamp(min=-111)
    return (_e2m1(y / torch.exp2(ex)) * torch.exp2(ex)).reshape(x.shape)


def exact(case, seed):
    if case["kind"] == "logp" and case["rows"] * case["vocab"] > 4e8:
        return None
    st = prepare(case, seed)
    if case["kind"] == "logp":
        out = {"logprob": [], "entropy": [], "top_tokens": [], "top_logprobs": []}
        for r in range(case["rows"]):
            x = st["logits"][r].double()
            live = torch.nonzero(x > -math.inf)[:, 0]
            p = torch.log_softmax(x[live], 0)
            mine = x[st["tokens"][r].long()]
            out["logprob"].append(mine - torch.logsumexp(x, 0) if len(live) else mine)
            out["entropy"].append(-(p.exp() * p).sum())
            order = torch.argsort(x[live], descending=True, stable=True)[:case["top"]]
            ids = torch.full((case["top"],), -1, dtype=torch.long, device=x.device)
            lp = torch.full((case["top"],), -math.inf, dtype=torch.float64, device=x.device)
            ids[:len(order)], lp[:len(order)] = live[order], p[order]
            out["top_tokens"].append(ids)
            out["top_logprobs"].append(lp)
        return {n: torch.stack(v).int() if n == "top_tokens" else torch.stack(v) for n, v in out.items()}
    codes, scales, hkv, hd = st["codes"], st["scales"], case["hkv"], case["hd"]
    if case["kind"] == "append":
        r32 = lambda z: z.float().double()  # noqa: E731 (a rounding that the definition names)
        ang = st["rope"].double()[st["positions"].long()].reshape(-1, 1, hd // 2, 2)
        turned = {}
        for name in ("q", "k"):
            a, b = st[name].double()[..., :hd // 2], st[name].double()[..., hd // 2:]
            lo = r32(r32(a * ang[..., 0]) - r32(b * ang[..., 1]))
            hi = r32(r32(b * ang[..., 0]) + r32(a * ang[..., 1]))
            turned[name] = torch.cat([lo, hi], -1).bfloat16().double()
        out = {"q": turned["q"]}
        slots, back = st["slots"].long(), st["read"].long()
        place = torch.full((codes.shape[0] * PAGE,), -1, dtype=torch.long, device="cuda")
        place[slots] = torch.arange(len(slots), device="cuda")
        src = place[back]
        pages, inv = torch.unique(back // PAGE, return_inverse=True)
        for side, name, block in ((0, "k", 32), (1, "v", hd)):
            fresh = _stored(turned["k"] if side == 0 else st["v"].double(), block)
            rows = []
            for h in range(hkv):
                old = _held(codes, scales, pages, h, side)[inv, back % PAGE]
                rows.append(torch.where(src[:, None] >= 0, fresh[src.clamp(min=0), h], old))
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
            k = _held(codes, scales, pg, h, 0).reshape(-1, hd)[:c + n]
            v = _held(codes, scales, pg, h, 1).reshape(-1, hd)[:c + n]
            x = q[t0:t0 + n, h * G:(h + 1) * G].double()
            s = (x.reshape(-1, hd) @ k.T.contiguous()).reshape(n, G, -1) / math.sqrt(hd)
            if case["softcap"]:
                s = case["softcap"] * torch.tanh(s / case["softcap"])
            w = torch.softmax(s.masked_fill(~seen[:, None, :], -math.inf), -1)
            o[t0:t0 + n, h * G:(h + 1) * G] = (w.reshape(n * G, -1) @ v).reshape(n, G, hd)
        t0 += n
    return o
