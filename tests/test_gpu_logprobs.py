"""Token log probabilities (GPU) against their definition in float64: the tokens exactly, the numbers within what fp32 sums give."""
import numpy as np
import pytest
import torch

import _kv4_ref as ref
from _gpu_common import dev_i32
from paper_2605_30218_amd import mg

pytestmark = pytest.mark.gpu


def check(x, tokens, top, got=None, **kw):
    """x: a tensor of logits on the GPU.  An exponent's argument y (at most 200 where its term matters) is off by 2^-24 |y| for the difference and
    2^-23 |y| for the product with log2 e, exp2 by 2^-22 of itself; a lane adds up to V / 64 + 64 terms and the joins some 30 more, each
    2^-24 of the sum; the logarithm and the differences after it round three times."""
    got = mg.token_logprobs(x, dev_i32(tokens), top=top, **kw) if got is None else got
    h = x.double().cpu().numpy()
    lp, ent, ids, vals = ref.logprobs(h, tokens, top)
    n, V = h.shape
    np.testing.assert_array_equal(got.top_tokens.cpu().numpy(), ids)
    with np.errstate(invalid="ignore"):
        live = np.where(np.isfinite(h), h, np.nan)
        far = np.where(np.isfinite(h).any(1), np.fmax.reduce(np.where(np.isfinite(live), np.abs(live), 0), 1), 0.0)
    # mean distance from the top under the weights, of which each term's relative error is a multiple: at most ln V + 1
    rel = (np.log(V) + 2) * 2.0 ** -22 + 2.0 ** -22 + (V / 64 + 100) * 2.0 ** -24
    tol = rel + 3 * 2.0 ** -24 * (np.log(V) + 2)
    # differences of logits are rounded once, and their sum with ln S: half a step of the result
    for g, w in ((got.logprob, lp), (got.top_logprobs, vals)):
        g, w = g.double().cpu().numpy(), np.asarray(w)
        np.testing.assert_array_equal(np.isnan(g), np.isnan(w))
        np.testing.assert_array_equal(np.isneginf(g), np.isneginf(w))
        fin = np.isfinite(w)
        d = np.abs(g[fin] - w[fin])
        assert (d <= (tol + 2.0 ** -23 * np.abs(w))[fin]).all(), d.max()
    g = got.entropy.double().cpu().numpy()
    np.testing.assert_array_equal(np.isnan(g), np.isnan(ent))
    ok = ~np.isnan(ent)
    # T / S is a mean of y with the same relative errors, and y's own rounding
    assert (np.abs(g - ent)[ok] <= (2 * tol * (np.log(V) + 2))).all(), np.abs(g - ent)[ok].max()
    assert far.shape == (n,)
    return got


def logits(n, V, seed=0, dtype=torch.float32, pad=0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    x = torch.empty((n, V + pad), dtype=dtype, device="cuda")[:, :V]
    x.copy_(3.0 * torch.randn((n, V), generator=g, device="cuda"))
    return x


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,V,top", [(1, 1, 1), (3, 5, 5), (2, 63, 0), (1, 2048, 32), (4, 2049, 20), (7, 4095, 1), (65, 8193, 20), (1, 128256, 20),
                                     (5, 152064, 32), (300, 9999, 8), (1100, 500, 3)])
def test_rows_of_many_sizes(n, V, top, dtype):
    x = logits(n, V, seed=n, dtype=dtype, pad=V % 3)
    check(x, np.random.RandomState(n).randint(0, V, n), top)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("kind", ["equal", "two_values", "rising", "falling", "steps", "one_lane"])
def test_orders_and_ties(kind, dtype):
    """Equal logits go by their index, wherever in the row they are; orders that take the list apart again and again."""
    V, n = 20000, 2
    j = torch.arange(V, device="cuda", dtype=torch.float32)
    x = {"equal": torch.zeros(V, device="cuda") + 1.5, "two_values": (j * 7919 % 97 < 3).float(), "rising": j / 256, "falling": -j / 256,
         "steps": (j / 1000).floor(), "one_lane": torch.where(j % 256 < 8, j / 100, -j)}[kind]
    x = torch.stack([x, x.flip(0)]).to(dtype).contiguous()
    for top in (1, 20, 32):
        check(x, [3, V - 1], top)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_masked_rows(dtype):
    """Rows with a few logits, one, none; the type's lowest value and infinities."""
    low = torch.finfo(dtype).min
    x = logits(9, 6000, seed=1, dtype=dtype)
    x[0, 7:] = -np.inf
    x[1, :5999] = -np.inf
    x[2] = -np.inf
    x[3] = low
    x[4, 10:] = low
    x[5, 100] = np.nan
    x[6, 5000] = np.inf
    x[7] = -np.inf
    x[7, 4321] = np.nan
    x[8, 4000:] = -np.inf
    x[8, 3000] = -x[8, 3000].abs() - 60000.0
    got = check(x, [2, 3, 4, 5, 20, 6, 5000, 0, 3000], 20)
    assert got.top_tokens[1].tolist() == [5999] + [-1] * 19 and got.top_tokens[2].tolist() == [-1] * 20
    assert float(got.entropy[2]) == 0.0 and float(got.entropy[1]) == 0.0 and float(got.logprob[2]) == -np.inf


def test_tokens_outside_the_vocabulary():
    x = logits(4, 700)
    got = check(x, [-1, 700, 2 ** 31 - 1, 699], 2)
    assert got.logprob[:3].isnan().all()


def test_unaligned_rows_and_outputs_that_are_not_wanted():
    """Rows that begin at any value's address; fields of None are not computed."""
    for dtype in (torch.float32, torch.bfloat16):
        for off in (1, 3):
            wide = logits(3, 5011, seed=off, dtype=dtype)
            check(wide[:, off:], [0, 5, 9], 6)
    x = logits(3, 5011)
    want = mg.token_logprobs(x, dev_i32([1, 2, 3]), top=4)
    ids = torch.full((3, 4), -7, dtype=torch.int32, device="cuda")
    got = mg.token_logprobs(x, None, top=4, out=mg.TokenLogprobs(None, None, ids, None))
    assert got.logprob is None and torch.equal(ids, want.top_tokens)
    lp = torch.zeros(3, device="cuda")
    mg.token_logprobs(x, dev_i32([1, 2, 3]), out=mg.TokenLogprobs(lp, None, None, None))
    assert torch.equal(lp, want.logprob)
    assert mg.token_logprobs(x[:0], dev_i32([]), top=3).top_tokens.shape == (0, 3)


def test_agrees_with_the_margin_gate():
    """Top 1 and the difference to the second are the gate's top1 and margin, bit for bit."""
    x = logits(64, 128256, seed=5)
    x[3, 77] = x[3].max()
    got = mg.token_logprobs(x, dev_i32([0] * 64), top=2)
    i32 = dict(dtype=torch.int32, device="cuda")
    top1, rows_, n = torch.zeros(64, **i32), torch.zeros(64, **i32), torch.zeros(1, **i32)
    margin, gate = torch.zeros(64, device="cuda"), torch.zeros(64, dtype=torch.uint8, device="cuda")
    mg.margin_gate_noalloc(64, 128256, x, None, 0.1, top1, margin, gate, rows_, n)
    assert torch.equal(got.top_tokens[:, 0], top1)
    v = x.gather(1, got.top_tokens.long())
    assert torch.equal(v[:, 0] - v[:, 1], margin)


def test_captured_and_on_two_streams():
    """A graph of the call follows its buffers; calls on two streams with workspaces of their own."""
    n, V = 3, 128256
    x = logits(n, V)
    tok = dev_i32([5, 6, 7])
    out = mg.token_logprobs(x, tok, top=5)
    ws = torch.empty(mg.token_logprobs_workspace_bytes(n, V, 5), dtype=torch.uint8, device="cuda")
    assert ws.numel() > 0
    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        mg.token_logprobs(x, tok, top=5, out=out, workspace=ws)
    for seed in (1, 2, 3):
        x.copy_(logits(n, V, seed))
        tok.fill_(seed)
        g.replay()
        torch.cuda.synchronize()
        for a, b in zip(out, mg.token_logprobs(x, tok, top=5)):
            assert torch.equal(a, b)
    xs = [logits(n, V, s) for s in (8, 9)]
    want = [mg.token_logprobs(y, tok, top=5) for y in xs]
    torch.cuda.synchronize()
    st = [torch.cuda.Stream() for _ in xs]
    got = []
    for _ in range(10):
        got = [mg.token_logprobs(y, tok, top=5, stream=s) for y, s in zip(xs, st)]
    torch.cuda.synchronize()
    for w, o in zip(want, got):
        for a, b in zip(w, o):
            assert torch.equal(a, b)
