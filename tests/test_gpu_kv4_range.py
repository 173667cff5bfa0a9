"""The 4-bit cache's attention (GPU) at the ends of what it takes: queries of any finite size, against the definition in
float64 and the bounds that its roundings give."""
import numpy as np
import pytest
import torch

from _kv8_ref import bf16
from test_gpu_kv4 import Batch

pytestmark = pytest.mark.gpu

# rows of single tokens, of a few, and chunks
KINDS = [[1, 1, 1], [4, 2, 3], [90, 1, 40]]


# ---------------------------------------------------------------- queries


@pytest.mark.parametrize("e", [100, 107, 108, 115, 124])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("new", KINDS)
def test_finite_queries_of_any_size(new, hd, e):
    """Queries around 2^e over keys so small that the scores are ordinary numbers: every term of a query value counts."""
    b = Batch(np.add([30, 300, 700], new), new, 8, 2, hd, seed=e, std=2.0 ** (46 - e))
    b.q = (b.q.double() * 2.0 ** e).to(torch.bfloat16)
    assert torch.isfinite(b.q).all() and float(b.q.float().abs().max()) > 2.0 ** e
    b.check(scale=2.0 ** -49)


def test_large_and_small_queries_of_one_call_keep_their_bits():
    """A block's size has no part in another row's outputs: rows of ordinary queries beside one of large ones, bit for bit."""
    new = [3, 1, 60]
    b = Batch(np.add([30, 300, 700], new), new, 8, 2, 128, seed=3)
    clean = bf16(b.run())
    b.q[1] = (b.q[1].double() * 2.0 ** 120).to(torch.bfloat16)
    got = bf16(b.run())
    keep = np.arange(len(got)) != 1
    np.testing.assert_array_equal(got[keep], clean[keep])
