"""Token log probabilities (GPU) of the most rows that a call takes."""
import numpy as np
import pytest
import torch

from paper_2605_30218_amd import mg

pytestmark = pytest.mark.gpu


def test_the_most_rows_of_a_call():
    """2^24 - 1 rows of three logits, against the same formula in float64."""
    n, V = (1 << 24) - 1, 3
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    x = torch.randn((n, V), generator=g, device="cuda")
    tok = torch.randint(0, V, (n,), generator=g, device="cuda", dtype=torch.int32)
    got = mg.token_logprobs(x, tok, top=2)
    for a in (0, n // 2, n - 1000):
        y = torch.log_softmax(x[a:a + 1000].double(), -1)
        want = y.gather(1, tok[a:a + 1000, None].long())[:, 0]
        # differences of logits, a sum of three exponentials and a logarithm, each within some steps of fp32 of numbers below 16
        np.testing.assert_allclose(got.logprob[a:a + 1000].cpu().numpy(), want.cpu().numpy(), rtol=2.0 ** -21, atol=2.0 ** -20)
        assert torch.equal(got.top_tokens[a:a + 1000].long(), x[a:a + 1000].topk(2).indices)
