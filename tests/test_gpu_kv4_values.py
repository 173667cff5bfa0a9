"""The 4-bit cache's attention (GPU) over values of unequal size: a position's weight keeps its accuracy beside neighbours whose scales are many times its
own.  Keys and queries are whole numbers, so that products are exact in fp32."""
import numpy as np
import pytest
import torch

import _kv4_ref as ref
import _kv4_weights as exact
from _gpu_common import dev_i32
from _kv8_ref import bf16
from paper_2605_30218_amd import mg
from test_gpu_kv4_scores import CTX, KINDS, batch

pytestmark = pytest.mark.gpu


def put_values(b, make, seed=0):
    """V of every row's positions anew: make(rng, v [n][2][hd]) changes N(0, 1) values."""
    rng = np.random.RandomState(seed)
    for r, n in enumerate(b.lens):
        j = np.arange(n)
        slots = dev_i32(b.table[r, j // 16] * 16 + j % 16)
        k, _ = mg.kv4_read(b.codes, b.scales, slots)
        v = make(rng, rng.randn(n, 2, b.hd))
        mg.kv4_append(b.codes, b.scales, k, torch.as_tensor(v.astype(np.float32)).to(torch.bfloat16).cuda(), slots)


def check(b, scale=0.01, **kw):
    got = bf16(b.run(scale=scale, **kw))
    out, bound = exact.attention(ref.RefCache.of(b.codes, b.scales), bf16(b.q), b.table, b.lens, b.cu, float(np.float32(scale)), **kw)
    np.testing.assert_array_equal(np.isnan(got), np.isnan(out))
    worst = np.nanmax(np.abs(got - out) / bound)
    assert worst <= 1.0, f"{worst} of the bound"


@pytest.mark.parametrize("to", [3, 9, 14, 60])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("new", KINDS)
def test_one_large_feature_of_one_position_in_32(new, hd, to):
    """That position's other features are zeros in the cache, and theirs come from its neighbours alone."""
    b = batch(new, hd, "flat", seed=to)

    def make(rng, v):
        v[5::32, :, 7] = 2.0 ** to
        return v

    put_values(b, make)
    check(b)


@pytest.mark.parametrize("spread", [1, 6, 40])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("new", KINDS)
def test_sizes_of_every_kind(new, hd, spread):
    """Each position's and head's values of a size of their own."""
    b = batch(new, hd, "flat", seed=spread)
    put_values(b, lambda rng, v: v * 2.0 ** rng.uniform(-spread, spread, v.shape[:2])[..., None])
    check(b)


@pytest.mark.parametrize("window", [0, 70])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("new", KINDS)
def test_positions_that_hold_little_or_nothing(new, hd, window):
    """Values of zero, tiny ones, ones that are not finite and large ones beside ordinary ones."""
    b = batch(new, hd, "flat", seed=7)

    def make(rng, v):
        v[0] = v[0] * 2.0 ** -20
        v[9::40] = 0.0
        v[11::40] *= 2.0 ** -10
        v[12::40] *= 2.0 ** -90
        v[17::100] *= 2.0 ** 6
        v[20, 1, 3] = np.inf
        return v

    put_values(b, make)
    check(b, window=window)


@pytest.mark.parametrize("ctx,new", [([9000, 20], [1, 1]), ([5000, 100, 20], [4] * 3), ([20, 1500], [600, 300])])
def test_unequal_values_of_long_rows(ctx, new):
    """Splits, rows of unequal length, and two groups of waves a block."""
    b = batch(new, 128, "flat", seed=9, ctx=ctx)

    def make(rng, v):
        v[3::50, :, 7] = 2.0 ** 10
        return v

    put_values(b, make)
    check(b)


def test_ordinary_steps_beside_others():
    """A far page of unequal values changes nothing for rows that do not see it."""
    b = batch(KINDS[2], 128, "flat", seed=3, ctx=CTX)
    clean = bf16(b.run())
    row = int(b.cu[1])
    slots = dev_i32(b.table[1, 40] * 16 + np.arange(16))
    k, v = mg.kv4_read(b.codes, b.scales, slots)
    v[::5] *= 2.0 ** 12
    mg.kv4_append(b.codes, b.scales, k, v, slots)
    got = bf16(b.run())
    keep = np.ones(len(got), bool)
    keep[row:int(b.cu[2])] = False
    np.testing.assert_array_equal(got[keep], clean[keep])
    assert (got[~keep] != clean[~keep]).any()


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("window", [0, 70])
@pytest.mark.parametrize("new", KINDS)
def test_what_no_token_sees_changes_no_bit(new, hd, window):
    """Positions behind the lengths, before the window, on unmapped pages and in the pages that holes stand for: scales and codes of any kind."""
    b = batch(new, hd, "flat", seed=13)
    put_values(b, lambda rng, v: v * 2.0 ** rng.uniform(-2, 2, v.shape[:2])[..., None], seed=4)
    b.table[1, 20:23] = -1
    seen = np.zeros((len(b.codes), 16), bool)
    for r, n in enumerate(b.lens):
        j = np.arange(max(0, n - b.new[r] - window + 1) if window else 0, n)
        j = j[b.table[r, j // 16] >= 0]
        seen[b.table[r, j // 16], j % 16] = True
    clean = bf16(b.run(window=window))
    assert np.isfinite(clean).all()
    rng = np.random.RandomState(17)
    for kind in range(3):
        sc = b.scales.cpu().numpy()
        s = sc[:, :, hd // 2:].transpose(0, 2, 1)
        s[~seen] = [rng.randint(0, 256, s[~seen].shape), 255, rng.choice([17, 250], s[~seen].shape)][kind]
        b.scales.copy_(torch.as_tensor(sc))
        np.testing.assert_array_equal(bf16(b.run(window=window)), clean)


@pytest.mark.parametrize("cap", [0.0, 20.0])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("new", [[4, 2, 3], [40, 30, 60]])
def test_a_value_that_is_not_finite_is_no_large_one(new, hd, cap):
    """A row's last position holds infinity: the row's last token is NaN, and the others, which do not see it, keep every bit."""
    b = batch(new, hd, "flat", seed=23)
    clean = bf16(b.run(softcap=cap))
    for r, n in enumerate(b.lens):
        slot = dev_i32([b.table[r, (n - 1) // 16] * 16 + (n - 1) % 16])
        k, v = mg.kv4_read(b.codes, b.scales, slot)
        v[:, :, 5] = np.inf
        mg.kv4_append(b.codes, b.scales, k, v, slot)
    got = bf16(b.run(softcap=cap))
    last = np.zeros(len(got), bool)
    last[b.cu[1:] - 1] = True
    assert np.isnan(got[last]).all()
    np.testing.assert_array_equal(got[~last], clean[~last])
