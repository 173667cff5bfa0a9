"""The 8-bit cache's attention (GPU) over scores up to 2^23, the most that its contract takes: keys and queries are small whole numbers, so that products
are exact in fp32 and only the softmax's own arithmetic is at work."""
import numpy as np
import pytest
import torch

import _kv4_weights as exact
import _kv8_ref as ref
from _gpu_common import dev_i32
from paper_2605_30218_amd import mg
from test_gpu_kv8 import Batch

pytestmark = pytest.mark.gpu

# rows of single tokens, of a few, and chunks, over contexts that are split and that are not
KINDS = [[1, 1, 1], [4, 2, 3], [90, 1, 40]]
CTX = [30, 1300, 500]
LARGEST = 2.0 ** 23
WHOLE = np.array([0, 1, 2, 3, 4, 6, -1, -2, -3, -4, -6.0])


def batch(new, hd, kind, seed, ctx=CTX):
    b = Batch(np.add(ctx, new), new, 8, 2, hd, seed=seed)
    rng = np.random.RandomState(seed)
    b.q = torch.as_tensor(rng.randint(-8, 9, tuple(b.q.shape)).astype(np.float32)).to(torch.bfloat16)
    for r, n in enumerate(b.lens):
        j = np.arange(n)
        k = rng.choice(WHOLE, (n, 2, hd))
        if kind == "negative":  # every score far below zero
            k = np.abs(k) + (k == 0)
        else:  # sizes along the positions; the first third of "rise" and the last of "fall" have scores of zero
            step = {"flat": np.ones(n), "rise": 2.0 ** (j * 8 // n), "fall": 2.0 ** ((n - 1 - j) * 8 // n)}[kind]
            at = {"flat": j >= 0, "rise": j > n // 3, "fall": j < n - n // 3}[kind]
            k = k * (step * at)[:, None, None]
        slots = dev_i32(b.table[r, j // 16] * 16 + j % 16)
        v = torch.as_tensor(rng.randn(n, 2, hd).astype(np.float32)).to(torch.bfloat16)
        mg.kv8_append(b.codes, b.scales, torch.as_tensor(k.astype(np.float32)).to(torch.bfloat16).cuda(), v.cuda(), slots)
        np.testing.assert_array_equal(ref.bf16(mg.kv8_read(b.codes, b.scales, slots)[0]), k)
    if kind == "negative":
        b.q = -b.q.abs() - 1
    return b


def largest(b):
    """The largest |q . k| of a batch, seen or not."""
    k = ref.RefCache.of(b.codes, b.scales).val[:, :, 0]
    q = ref.bf16(b.q).reshape(len(b.q), k.shape[1], -1, b.hd)
    pages = np.unique(b.table[b.table >= 0])
    return max(np.abs(q[:, h].reshape(-1, b.hd) @ k[pages, h].reshape(-1, b.hd).T).max() for h in range(k.shape[1]))


def check(b, scale, got=None, **kw):
    got = ref.bf16(b.run(scale=scale, **kw)) if got is None else got
    assert largest(b) * scale <= 1.01 * LARGEST
    out, bound = exact.attention(ref.RefCache.of(b.codes, b.scales), ref.bf16(b.q), b.table, b.lens, b.cu, float(np.float32(scale)), **kw)
    assert np.isfinite(got).all()
    worst = (np.abs(got - out) / bound).max()
    assert worst <= 1.0, f"{worst} of the bound"


@pytest.mark.parametrize("size", [1.0, LARGEST])
@pytest.mark.parametrize("kind", ["flat", "rise", "fall", "negative"])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("new", KINDS)
def test_scores_up_to_the_largest(new, hd, kind, size):
    b = batch(new, hd, kind, seed=hd + len(kind))
    check(b, size if size < 2 else size / largest(b))


@pytest.mark.parametrize("new", KINDS)
def test_large_scores_behind_a_window(new):
    """Tokens that see nothing of a wave's first positions, and later much."""
    b = batch(new, 128, "rise", seed=5)
    check(b, LARGEST / largest(b), window=100)


@pytest.mark.parametrize("ctx,new", [([9000, 20], [1, 1]), ([5000, 100, 20], [4] * 3), ([20, 1500], [600, 300])])
def test_large_scores_of_long_rows(ctx, new):
    """Splits, rows of unequal length, and two groups of waves a block."""
    b = batch(new, 128, "flat", seed=9, ctx=ctx)
    check(b, LARGEST / largest(b))
