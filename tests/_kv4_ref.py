"""The 4-bit paged K/V cache, its rotation and its attention in float64, from their definitions (include/mg.h), for the tests of the HIP
kernels.  Nothing here is shared with the library."""
import numpy as np
from scipy.ndimage import maximum_filter1d

PAGE = 16
E2M1 = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])


def f32(x):
    with np.errstate(over="ignore", invalid="ignore"):
        return np.asarray(x, np.float64).astype(np.float32).astype(np.float64)


def to_bf16(x):
    """float64 -> the nearest bf16 value, ties to even, by way of no other format (infinity past the largest)."""
    x = np.asarray(x, np.float64)
    with np.errstate(invalid="ignore", over="ignore"):
        _, e = np.frexp(np.where(np.isfinite(x), x, 0.0))
        step = np.exp2(np.maximum(e - 1, -126) - 7.0)
        y = np.rint(x / step) * step
        return np.where(np.isfinite(x), np.where(np.abs(y) >= 2.0 ** 128, np.sign(y) * np.inf, y), x)


def rotate(x, table, pos):
    """Heads x [n][H][hd] (bf16 values) turned by positions pos: products and sums rounded to fp32, the result to bf16."""
    h = x.shape[-1] // 2
    out = np.full(x.shape, np.nan)
    ok = pos < len(table)
    cs = table[np.where(ok, pos, 0)].astype(np.float64)
    c, s = cs[:, None, 0::2], cs[:, None, 1::2]
    a, b = x[..., :h], x[..., h:]
    with np.errstate(invalid="ignore", over="ignore"):
        out[..., :h] = to_bf16(f32(f32(a * c) - f32(b * s)))
        out[..., h:] = to_bf16(f32(f32(b * c) + f32(a * s)))
    out[~ok] = np.nan
    return out


def round_e2m1(x):
    """The nearest of E2M1 with a sign, ties to the even code."""
    a = np.minimum(np.abs(x), 6.0)
    up = np.searchsorted(E2M1, a, side="left")
    lo = np.maximum(up - 1, 0)
    d_lo, d_up = a - E2M1[lo], E2M1[up] - a
    pick = np.where((d_up < d_lo) | ((d_up == d_lo) & (up % 2 == 0)), up, lo)
    return np.copysign(E2M1[pick], x)


def scale_byte(top):
    """The least byte in 16 .. 254 with top <= 7 * 2^(b - 127); 255 where top is not finite."""
    top = np.asarray(top, np.float64)
    fine = np.isfinite(top)
    m, e = np.frexp(np.where(fine, top, 0.0) / 7.0)  # m in [1/2, 1)
    b = np.where(m == 0.5, e - 1, e) + 127
    b = np.where(top == 0, 16, b)
    return np.where(fine, np.clip(b, 16, 254), 255)


def stored(x, block):
    """(values, scale bytes) that rows x [..., hd] have in the cache."""
    y = x.reshape(*x.shape[:-1], x.shape[-1] // block, block)
    b = scale_byte(np.where(np.isfinite(y), np.abs(y), np.inf).max(-1))
    unit = np.exp2(np.where(b == 255, 127, b) - 127.0)[..., None]
    v = np.where((b == 255)[..., None], np.nan, round_e2m1(np.where(np.isfinite(y), y, 0.0) / unit) * unit)
    return v.reshape(x.shape), b


def unpack(codes, scales):
    """(values [n_pages][Hkv][2][16][hd], K's scale bytes [n_pages][Hkv][16][hd / 32], V's [n_pages][Hkv][16])."""
    c, s = codes.cpu().numpy(), scales.cpu().numpy().astype(np.int64)
    n, hkv, _, w = c.shape
    hd = w // 8
    t, d = np.meshgrid(np.arange(PAGE), np.arange(hd), indexing="ij")
    at = [((d // 32 * 16 + t) * 16 + d % 32 // 2, d % 2), ((t // 4 * 16 + d % 16) * (hd // 8) + d // 16 * 2 + t % 4 // 2, t % 2)]
    kb = s[:, :, :hd // 2].reshape(n, hkv, hd // 32, PAGE).transpose(0, 1, 3, 2)
    vb = s[:, :, hd // 2:]
    val = np.zeros((n, hkv, 2, PAGE, hd))
    for side, (byte, nib) in enumerate(at):
        x = (c[:, :, side][:, :, byte] >> (4 * nib)) & 15
        val[:, :, side] = np.where(x >= 8, -1.0, 1.0) * E2M1[x & 7]
    per = np.stack([np.repeat(kb, 32, axis=3), np.repeat(vb[..., None], hd, axis=3)], 2)
    return val * np.where(per == 255, np.nan, np.exp2(np.where(per == 255, 127, per) - 127.0)), kb, vb


class RefCache:
    """val [n_pages][Hkv][2][16][hd]; unit [n_pages][Hkv][16]: what a code of V is a multiple of."""

    def __init__(self, n_pages, hkv, hd):
        self.val = np.zeros((n_pages, hkv, 2, PAGE, hd))
        self.unit = np.zeros((n_pages, hkv, PAGE))

    @staticmethod
    def of(codes, scales):
        r = RefCache(codes.shape[0], codes.shape[1], codes.shape[3] // 8)
        r.val, _, vb = unpack(codes, scales)
        r.unit = np.exp2(np.where(vb == 255, 0, vb) - 127.0)
        return r

    def append(self, k, v, slots):
        hd = k.shape[-1]
        for side, x, block in ((0, k, 32), (1, v, hd)):
            val, b = stored(x, block)
            for i, s in enumerate(slots):
                if 0 <= s < len(self.val) * PAGE:
                    self.val[s // PAGE, :, side, s % PAGE] = val[i]
                    if side:
                        self.unit[s // PAGE, :, s % PAGE] = np.exp2(np.where(b[i, :, 0] == 255, 0, b[i, :, 0]) - 127.0)


def attention(cache, q, table, lens, cu, scale, window=0, softcap=0.0):
    """(out, bound) in float64: the definition's result for q [T][Hq][hd], and how far a bf16 result may be from it.  With w the
    softmax weights and A = sum_j w_j |v_j| the bound adds
      the output's rounding, half a step of bf16: 2^-8 |out|;
      a query value's three 6-bit terms under S, S / 32, S / 1024 with the block's largest in [S, 2 S): their steps are an eighth of these, so a
        value from S / 64 up, a multiple of S / 8192 in bf16, is exact, and one below is off by half a step, S / 16384, at most: a
        score by 2^-14 * scale * sum (largest of the block) |k|;
      fp32 scores: hd + 16 roundings of 2^-24 relative to scale * sum |q k| (a capped score: 2^-20 of the largest score more), and exp's argument,
        rounded once relative to the largest score; each weight moves by at most 2 (E + 2^-23 max|s|) of itself, twice for the quotient;
      a probability times its value's scale as two 6-bit terms, for each code, under s and s / 32 with the largest of its 32 positions from
        3.75 s to 7.5 s: the first leaves s / 4 of a number x from 4 s up, s / 8 from 2 s, s / 16 below; the second's steps, under s / 32,
        are 1/2, 1/4, 1/8 of that with nothing above 7.5, so it leaves s (1/4 - 7.5/32) = s / 64, s / 256, s / 512: 2^-8 x from 4 s up,
        2^-9 x from 2 s, below them s / 512 <= largest / 1920;
        these 32 positions lie within 127 of each other;
      fp32 sums over n positions and exp itself: (n + 32) 2^-23 A."""
    T, Hq, hd = q.shape
    hkv = cache.val.shape[1]
    G = Hq // hkv
    out, bound = np.zeros(q.shape), np.zeros(q.shape)
    for r in range(len(lens)):
        t0, t1 = int(cu[r]), int(cu[r + 1])
        n, L = t1 - t0, int(min(max(lens[r], 0), table.shape[1] * PAGE))
        if n <= 0 or L == 0:
            continue
        pg = table[r, :-(-L // PAGE)]
        here = (pg >= 0) & (pg < len(cache.val))
        kv = cache.val[np.where(here, pg, 0)]
        unit = cache.unit[np.where(here, pg, 0)]
        j = np.arange(L)
        p = int(lens[r]) - n + np.arange(n)[:, None]
        see = (j <= p) & np.repeat(here, PAGE)[:L]
        if window:
            see &= j > p - window
        see = np.repeat(see, G, 0)
        some = see.any(1)
        for h in range(hkv):
            k, v = (kv[:, h, side].reshape(-1, hd)[:L] for side in (0, 1))
            u = unit[:, h].reshape(-1)[:L]
            bad = np.isnan(k).any(1) | np.isnan(v).any(1)
            k, v = np.nan_to_num(k), np.nan_to_num(v)
            x = q[t0:t1, h * G:(h + 1) * G].reshape(-1, hd)
            odd = ~np.isfinite(x).all(1)
            x = np.where(odd[:, None], 0.0, x)
            s = x @ k.T * scale
            E = (hd + 16) * 2.0 ** -24 * scale * np.where(see, np.abs(x) @ np.abs(k).T, 0.0).max(1)
            xb = np.repeat(np.abs(x).reshape(len(x), -1, 32).max(2), 32, 1)
            E += 2.0 ** -14 * scale * np.where(see, xb @ np.abs(k).T, 0.0).max(1)
            if softcap:
                s = softcap * np.tanh(s / softcap)
                E = E + 2.0 ** -20 * np.where(see, np.abs(s), 0.0).max(1)
            s = np.where(see, s, -np.inf)
            with np.errstate(invalid="ignore"):
                w = np.exp(s - s.max(1, keepdims=True))
                w = np.where(some[:, None], w / w.sum(1, keepdims=True), 0.0)
            o, A = w @ v, w @ np.abs(v)
            top = np.where(see, np.abs(s), 0.0).max(1)
            rel = 4 * (E + 2.0 ** -23 * top) + (L + 32) * 2.0 ** -23
            big = maximum_filter1d(w * u, 255, axis=1, mode="constant")
            code = np.abs(v) / np.where(u > 0, u, 1.0)[:, None]
            P = np.maximum(2.0 ** -8 * w * u, big / 1920) @ code
            o[(see & bad).any(1) | (odd & some)] = np.nan
            out[t0:t1, h * G:(h + 1) * G] = o.reshape(n, G, hd)
            b = 2.0 ** -8 * np.abs(o) + (1 + 2.0 ** -8) * (rel[:, None] * A + P) + 1e-38
            bound[t0:t1, h * G:(h + 1) * G] = b.reshape(n, G, hd)
    return out, bound


def logprobs(x, tokens, top):
    """(logprob, entropy, ids, values) of rows of float64 logits."""
    lp, ent, ids, vals = [], [], [], []
    for row, t in zip(x, tokens):
        live = np.nonzero(row > -np.inf)[0]
        bad = np.isnan(row).any() or np.isinf(row[live]).any()
        if bad:
            p = np.full(len(row), np.nan)
        elif len(live):
            m = row.max()
            p = (row - m) - np.log(np.exp(row[live] - m).sum())  # (m + ln S would lose ln S beside a large m)
        else:
            p = row
        lp.append(p[t] if 0 <= t < len(row) else np.nan)
        q = p[live]
        ent.append(np.nan if bad else -(np.exp(q) * q).sum() if len(live) else 0.0)
        order = live[np.lexsort((live, -row[live]))][:top]
        ids.append(np.concatenate([order, np.full(top - len(order), -1)]))
        vals.append(np.concatenate([p[order], np.full(top - len(order), -np.inf)]))
    return np.array(lp), np.array(ent), np.array(ids, np.int64).reshape(len(x), top), np.array(vals).reshape(len(x), top)
