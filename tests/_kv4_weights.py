"""Attention over the 4-bit cache in float64 where the scores themselves are exact in fp32 (whole numbers), with the bound that is then left."""
import numpy as np
from scipy.ndimage import maximum_filter1d

PAGE = 16


def attention(cache, q, table, lens, cu, scale, window=0):
    """(out, bound) for q [T][Hq][hd], whose products with the keys (RefCache `cache`) are exact in fp32.  With w the weights, d a position's
    distance from its row's largest score, u V's scale of a position, A = sum_j w_j |v_j|, the bound adds
      the output's rounding, half a step of bf16: 2^-8 |out|;
      the exponent d log2 e scale: the factor is rounded twice and the exponent once, 2^-22 d together, of which up to 110 matters (behind it a
        weight is below fp32's numbers beside the largest); a reference up to 4096 (in powers of two) is rounded by 2^-13 at most, which is an
        error where splits with different references join; twice for the quotient;
      fp32 sums over n positions and exp2: (n + 32) 2^-23 A;
      a weight in 6-bit terms, as many as V's scales ask for: 2^-8 of itself or 1/480 of the largest of 32 positions, whatever the scales; these 32
        positions lie within 127 of each other.
    A value of V that is not finite makes NaN what sees it."""
    T, Hq, hd = q.shape
    hkv = cache.val.shape[1]
    G = Hq // hkv
    out, bound = np.zeros(q.shape), np.zeros(q.shape)
    for r in range(len(lens)):
        t0, t1 = int(cu[r]), int(cu[r + 1])
        n, L = t1 - t0, int(lens[r])
        pg = table[r, :-(-L // PAGE)]
        kv = cache.val[pg]
        j = np.arange(L)
        p = L - n + np.arange(n)[:, None]
        see = j <= p
        if window:
            see &= j > p - window
        see = np.repeat(see, G, 0)
        for h in range(hkv):
            k, v = (kv[:, h, side].reshape(-1, hd)[:L] for side in (0, 1))
            bad = np.isnan(v).any(1)
            v = np.nan_to_num(v)
            x = q[t0:t1, h * G:(h + 1) * G].reshape(-1, hd) @ k.T
            assert (x == x.astype(np.float32)).all()
            x = np.where(see, x, -np.inf)
            d = (x - x.max(1, keepdims=True)) * scale
            w = np.exp(d)
            w /= w.sum(1, keepdims=True)
            o, A = w @ v, w @ np.abs(v)
            rel = 2 * (2.0 ** -22 * 110 + 2.0 ** -13) + (L + 32) * 2.0 ** -23
            big = maximum_filter1d(w, 255, axis=1, mode="constant")
            P = np.maximum(2.0 ** -8 * w, big / 480) @ np.abs(v)
            o[(see & bad).any(1)] = np.nan
            out[t0:t1, h * G:(h + 1) * G] = o.reshape(n, G, hd)
            b = 2.0 ** -8 * np.abs(o) + (1 + 2.0 ** -8) * (rel * A + P) + 1e-38
            bound[t0:t1, h * G:(h + 1) * G] = b.reshape(n, G, hd)
    return out, bound
