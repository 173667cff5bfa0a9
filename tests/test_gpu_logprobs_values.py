"""Token log probabilities (GPU) of logits far from zero and far from each other, against their definition in float64."""
import numpy as np
import pytest
import torch

from _gpu_common import dev_i32
from paper_2605_30218_amd import mg
from test_gpu_logprobs import check, logits

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("add", [-1e4, 3e3, 1e6, -1e30, 1e38])
@pytest.mark.parametrize("V", [100, 9000])
def test_logits_far_from_zero(V, add, dtype):
    """Differences of such logits are exact, or the logits are equal: results are as near as those of small ones."""
    x = (logits(5, V, seed=V).double() + add).to(dtype)
    check(x, [0, 1, V // 2, V - 2, V - 1], 20)


@pytest.mark.parametrize("size", [100.0, 1e4, 1e20, 1e38])
def test_logits_far_from_each_other(size):
    """A few logits have all the weight; log probabilities of the others are nearly their distances."""
    x = logits(4, 5000, seed=3) / 16 * size
    x[1, 4000] = x[1].max()
    got = check(x, [7, 4000, 0, 4999], 8)
    assert torch.isfinite(got.entropy).all()


def test_the_largest_magnitude_that_a_row_has():
    """The first alternative's logit is the row's largest, whatever its size, and its log probability at most 0."""
    for size in (1e-30, 1.0, 1e30):
        x = logits(3, 3000, seed=9) * size
        got = mg.token_logprobs(x, dev_i32([0, 1, 2]), top=1)
        far = x.abs().amax(1)
        first = x.gather(1, got.top_tokens.long())[:, 0]
        assert torch.equal(first, x.amax(1)) and (first <= far).all()
        assert (got.top_logprobs <= 0).all() and np.isfinite(got.top_logprobs.cpu().numpy()).all()
