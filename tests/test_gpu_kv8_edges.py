"""The batch plan and the 8-bit paged K/V cache (GPU) at the edges of their contract, against the
definitions in float64 and Python integers (_kv8_ref.py), each row of an attention call within the bound of
its own probabilities."""
import numpy as np
import pytest

import _kv8_ref as ref
from test_gpu_kv8 import Batch

pytestmark = pytest.mark.gpu


def probability_bits(new, G):
    """Per row: 16 bits where the call's rows have at most 32 query rows, or the row itself at most 16; else 8."""
    return [16 if max(new) * G <= 32 or n * G <= 16 else 8 for n in new]


def compare(b, got, cache=None, **kw):
    """got against the definition, row by row within the bound of the row's probabilities."""
    kw["scale"] = kw.get("scale") or 1 / np.sqrt(b.hd)
    cache = ref.RefCache.of(b.codes, b.scales) if cache is None else cache
    got, bits = ref.bf16(got), probability_bits(b.new, b.G)
    for p_bits in sorted(set(bits)):
        out, bound = ref.attention(cache, ref.bf16(b.q), b.table, b.lens, b.cu, p_bits=p_bits, **kw)
        for r in range(len(b.new)):
            if bits[r] != p_bits:
                continue
            t = slice(int(b.cu[r]), int(b.cu[r + 1]))
            np.testing.assert_array_equal(np.isnan(got[t]), np.isnan(out[t]), err_msg=f"row {r}")
            off = np.abs(got[t] - out[t]) > bound[t]
            assert not off.any(), f"row {r}: {off.sum()} of {off.size} past the bound, by up to " \
                                  f"{np.nanmax(np.abs(got[t] - out[t]) / np.where(bound[t] > 0, bound[t], 1e-38))}"
    return got


def run_and_compare(b, max_len=0, **kw):
    return compare(b, b.run(max_len=max_len, **kw), **kw)


# ---------------------------------------------------------------- windows

PAST = 2 ** 31 - 1


@pytest.mark.parametrize("new", [[1, 1, 1, 1], [3, 1, 2, 4], [60, 1, 40, 20]])
@pytest.mark.parametrize("window", [63, 64, 65, 900, 936, 937, 990, 999, 1000, 1001, PAST - 70, PAST - 1, PAST])
def test_window_of_rows_longer_than_their_page_table(window, new):
    """A row's positions past its table are not there, but its tokens stand behind them: the window counts from
    where they stand.  Tables of 64 positions."""
    b = Batch([64, 64, 64, 64], new, 8, 2, 64, seed=1, spare=0)
    b.lens = np.array([1000, 1000, PAST, min(3, new[3] - 1)])
    run_and_compare(b, window=window)
