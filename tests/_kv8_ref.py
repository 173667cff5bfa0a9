"""The 8-bit paged K/V cache and the batch plan in float64 and Python integers, from their definitions
(include/mg.h), for the tests of the HIP kernels.  Nothing here is shared with the library."""
import numpy as np
import torch

PAGE = 16


def bf16(a):
    """float64 values of a bf16 tensor."""
    return a.detach().cpu().view(torch.int16).numpy().view(np.uint16).astype(np.uint32).__lshift__(16).view(
        np.float32).astype(np.float64)


def byte_index(hd, side):
    """[16][hd] byte of a page at which position t's feature d stands."""
    t, d = np.meshgrid(np.arange(PAGE), np.arange(hd), indexing="ij")
    h, r = d // 64, d % 64
    if side == 0:
        return ((h * 4 + r // 16) * 16 + t) * 16 + r % 16
    return ((h * 4 + t // 4) * 16 + r % 16) * 16 + 4 * (r // 16) + t % 4


def code_values(c):
    """float64 values of e4m3 codes."""
    c = np.asarray(c).astype(np.int64)
    e, m = (c >> 3) & 15, c & 7
    v = np.where(e == 0, m * 2.0 ** -9, (8 + m) * np.exp2(e - 10.0))
    v = np.where((c & 127) == 127, np.nan, v)
    return np.where(c >= 128, -v, v)


def round_e4m3(x):
    """The nearest e4m3 value, ties to even (|x| <= 448)."""
    with np.errstate(invalid="ignore"):
        _, e = np.frexp(np.where(np.isfinite(x), x, 0.0))
        step = np.exp2(np.maximum(e - 1, -6) - 3.0)
        return np.rint(x / step) * step


def need_byte(top):
    """The least byte b in [16, 254] with top <= 448 * 2^(b - 127)."""
    b = 16
    while top > 448.0 * 2.0 ** (b - 127):
        b += 1
    return b


class RefCache:
    """values [n_pages][Hkv][2][16][hd] in float64 and their scale bytes."""

    def __init__(self, n_pages, hkv, hd):
        self.val = np.zeros((n_pages, hkv, 2, PAGE, hd))
        self.byte = np.zeros((n_pages, hkv, 2), np.int64)

    @staticmethod
    def of(codes, scales):
        c, s = codes.cpu().numpy(), scales.cpu().numpy()
        n, hkv, _, w = c.shape
        r = RefCache(n, hkv, w // PAGE)
        r.byte[:] = s
        for side in (0, 1):
            r.val[:, :, side] = code_values(c[:, :, side][:, :, byte_index(w // PAGE, side)]) * np.exp2(
                s[:, :, side] - 127.0)[..., None, None]
        return r

    def append(self, k, v, slots):
        """k, v float64 [n][Hkv][hd]; one page's run of tokens after the other."""
        i, n = 0, len(slots)
        while i < n:
            s = int(slots[i])
            if s < 0 or s >= len(self.val) * PAGE:
                i += 1
                continue
            j = i + 1
            while j < n and slots[j] == slots[j - 1] + 1 and slots[j] // PAGE == s // PAGE:
                j += 1
            pg, o = s // PAGE, s % PAGE
            for side, x in ((0, k), (1, v)):
                for h in range(x.shape[1]):
                    new = x[i:j, h]
                    fin = np.abs(new[np.isfinite(new)])
                    old = 0 if o == 0 else self.byte[pg, h, side]
                    b = max(old, need_byte(fin.max() if fin.size else 0.0))
                    page = self.val[pg, h, side]
                    if old == 0:
                        page[:] = 0.0
                    elif b > old:
                        page[:] = round_e4m3(page / 2.0 ** (b - 127)) * 2.0 ** (b - 127)
                    q = np.where(np.isfinite(new), new, np.nan)
                    page[o:o + j - i] = round_e4m3(q / 2.0 ** (b - 127)) * 2.0 ** (b - 127)
                    self.byte[pg, h, side] = b
            i = j

    def read(self, slots):
        s = np.asarray(slots)
        x = self.val[s // PAGE, :, :, s % PAGE]
        return x[:, :, 0], x[:, :, 1]


def attention(cache, q, table, lens, cu, scale, window=0, softcap=0.0, p_bits=8):
    """(out, bound) in float64: the definition's result for q [T][Hq][hd], and how far a bf16 result may be
    from it.  With A = sum_j w_j |v_j| (w the softmax weights), the bound adds
      the output's rounding, half a step of bf16: 2^-8 |out|;
      a probability's rounding to p_bits bits: 2^-p_bits A;
      fp32 scores: hd + 16 roundings (the products' sum, scale, cap) of 2^-24 relative to scale * sum |q k|, E
        at most (a capped score: 2^-20 of the largest score more, for tanh with an error of 2^-22
        of itself below 1/2 and 2^-23 above), and exp's argument, rounded once relative to the largest score: each weight moves by at most
        2 (E + 2^-23 max|s|) of itself, twice for the quotient;
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
        kv = cache.val[np.where(here, pg, 0)]  # [pages][Hkv][2][16][hd]
        j = np.arange(L)
        p = int(lens[r]) - n + np.arange(n)[:, None]
        see = (j <= p) & np.repeat(here, PAGE)[:L]
        if window:
            see &= j > p - window
        see = np.repeat(see, G, 0)  # [n G][L]
        some = see.any(1)
        for h in range(hkv):
            k, v = (kv[:, h, side].reshape(-1, hd)[:L] for side in (0, 1))
            bad_k, bad_v = np.isnan(k).any(1), np.isnan(v)
            k, v = np.nan_to_num(k), np.nan_to_num(v)
            x = q[t0:t1, h * G:(h + 1) * G].reshape(-1, hd)
            s = x @ k.T * scale
            E = (hd + 16) * 2.0 ** -24 * scale * np.where(see, np.abs(x) @ np.abs(k).T, 0.0).max(1)
            if softcap:
                s = softcap * np.tanh(s / softcap)
                top = np.where(see, np.abs(s), 0.0).max(1)
                E = E + 2.0 ** -20 * top
            s = np.where(see, s, -np.inf)
            with np.errstate(invalid="ignore"):
                w = np.exp(s - s.max(1, keepdims=True))
                w = np.where(some[:, None], w / w.sum(1, keepdims=True), 0.0)
            o, A = w @ v, w @ np.abs(v)
            top = np.where(see, np.abs(s), 0.0).max(1)
            rel = 4 * (E + 2.0 ** -23 * top) + (L + 32) * 2.0 ** -23 + 2.0 ** -p_bits
            o[(see & bad_k).any(1)] = np.nan
            o[(see.astype(np.float64) @ bad_v) > 0] = np.nan
            out[t0:t1, h * G:(h + 1) * G] = o.reshape(n, G, hd)
            bound[t0:t1, h * G:(h + 1) * G] = (2.0 ** -8 * np.abs(o) + (1 + 2.0 ** -8) * rel[:, None] * A + 1e-38).reshape(n, G, hd)
    return out, bound


def plan(ctx, new, free, n_free, table, max_tokens):
    """The batch plan, row by row: a dict of the outputs."""
    table = np.array(table)
    B, maxp = table.shape
    pos, rows, slots, cu, lens, adm = [], [], [], [0], [], []
    need_t = need_p = 0
    left, stopped = max(n_free, 0), False
    for b in range(B):
        c, n = int(ctx[b]), int(new[b])
        ok = c >= 0 and n >= 0 and c + n <= PAGE * maxp
        if ok:
            need_t += n
            need_p += -(-(c + n) // PAGE) - -(-c // PAGE)
            if need_t > max_tokens or need_p > max(n_free, 0):
                stopped = True
            ok = not stopped
        if ok:
            for i in range(-(-c // PAGE), -(-(c + n) // PAGE)):
                left -= 1
                table[b, i] = free[left]
            for p in range(c, c + n):
                pos.append(p)
                rows.append(b)
                slots.append(table[b, p // PAGE] * PAGE + p % PAGE)
        adm.append(int(ok))
        lens.append(max(c, 0) + (n if ok else 0))
        cu.append(len(pos))
    pad = [-1] * (max_tokens - len(pos))
    return {"table": table, "cu_new": cu, "lens": lens, "admitted": adm, "positions": pos + pad, "rows": rows + pad,
            "slots": slots + pad, "n_left": [left]}
