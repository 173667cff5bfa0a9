"""The 4-bit cache's attention (GPU) over scores of any size: keys and queries are small whole numbers, so that products are exact in fp32 and only
the softmax's own arithmetic is at work."""
import numpy as np
import pytest
import torch

import _kv4_ref as ref
import _kv4_weights as exact
from _gpu_common import dev_i32
from _kv8_ref import bf16
from paper_2605_30218_amd import mg
from test_gpu_kv4 import Batch

pytestmark = pytest.mark.gpu

# rows of single tokens, of a few, and chunks, over contexts that are split and that are not
KINDS = [[1, 1, 1], [4, 2, 3], [90, 1, 40]]
CTX = [30, 1300, 500]
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
        slots = b.table[r, j // 16] * 16 + j % 16
        v = torch.as_tensor(rng.randn(n, 2, hd).astype(np.float32)).to(torch.bfloat16)
        mg.kv4_append(b.codes, b.scales, torch.as_tensor(k.astype(np.float32)).to(torch.bfloat16).cuda(), v.cuda(), dev_i32(slots))
        back, _ = mg.kv4_read(b.codes, b.scales, dev_i32(slots))
        np.testing.assert_array_equal(bf16(back), k)
    if kind == "negative":
        b.q = -b.q.abs() - 1
    return b


def check(b, scale, got=None, **kw):
    got = bf16(b.run(scale=scale, **kw)) if got is None else got
    out, bound = exact.attention(ref.RefCache.of(b.codes, b.scales), bf16(b.q), b.table, b.lens, b.cu, float(np.float32(scale)), **kw)
    assert np.isfinite(got).all()
    worst = (np.abs(got - out) / bound).max()
    assert worst <= 1.0, f"{worst} of the bound"


@pytest.mark.parametrize("scale", [1e-3, 7.0, 1e9, 1e15])
@pytest.mark.parametrize("kind", ["flat", "rise", "fall", "negative"])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("new", KINDS)
def test_scores_of_any_size(new, hd, kind, scale):
    check(batch(new, hd, kind, seed=hd + len(kind)), scale)


@pytest.mark.parametrize("scale", [7.0, 1e9])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("new", KINDS)
def test_scores_of_any_size_behind_a_window(new, hd, scale):
    """Tokens that see nothing of a wave's first positions, and later much."""
    check(batch(new, hd, "rise", seed=5), scale, window=100)


@pytest.mark.parametrize("ctx,new", [([9000, 20], [1, 1]), ([5000, 100, 20], [4] * 3), ([20, 1500], [600, 300])])
def test_large_scores_of_long_rows(ctx, new):
    """Splits, rows of unequal length, and two groups of waves a block."""
    check(batch(new, 128, "flat", seed=9, ctx=ctx), 1e9)


@pytest.mark.parametrize("new", KINDS)
def test_large_caps(new):
    """A cap that is far above the scores leaves them as they are, whatever its size; one far below makes their signs the scores."""
    b = batch(new, 128, "flat", seed=11)
    check(b, 1.0, bf16(b.run(scale=1.0, softcap=1e15)))
    got = bf16(b.run(scale=1e15, softcap=1e15))  # scores of 1e15 times the tanh of whole numbers: the largest alone
    assert np.isfinite(got).all() and (np.abs(got).reshape(len(got), -1).max(1) > 0).all()
