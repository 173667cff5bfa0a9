"""The host side of the 4-bit K/V cache and of token log probabilities (CPU): sizes, and what is refused before any work is enqueued.
The pointers of the refused calls are never followed."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

import _kv4_ref as ref
from paper_2605_30218_amd import mg

ARG, SHAPE, WORKSPACE = -1, -2, -3
P = 1 << 20  # an aligned address that no refused call reads


def cache(codes=P, scales=P, n_pages=8, hkv=2, hd=64):
    return mg.MgKv4Cache(codes, scales, n_pages, hkv, hd)


def fill(a, d):
    for k, v in d.items():
        setattr(a, k, v)
    return a


def attn(**kw):
    return fill(mg.MgKv8AttnArgs(), dict(n_rows=3, n_tokens=5, n_q_heads=4, max_new=2, max_len=0, max_pages_per_row=4, window=0, scale=0.0,
                                         softcap=0.0, q=P, q_stride=256, out=4 * P, out_stride=256, page_table=P, lens=P, cu_new=P) | kw)


def app(**kw):
    return fill(mg.MgKv4AppendArgs(), dict(n_tokens=1, n_q_heads=4, q=P, q_stride=256, q_out=8 * P, q_out_stride=256, k=2 * P, k_stride=128, v=3 * P,
                                           v_stride=128, slots=P, positions=P, rope=P, n_positions=100) | kw)


def test_sizes():
    lib = mg.load()
    assert lib.mg_kv4_code_bytes(10, 8, 128) == 10 * 8 * 2 * 8 * 128
    assert lib.mg_kv4_scale_bytes(10, 8, 128) == 10 * 8 * 80
    for bad in ((0, 8, 128), (10, 0, 128), (10, 8, 96), (1 << 27, 8, 128), (-1, 8, 64)):
        assert lib.mg_kv4_code_bytes(*bad) == 0 and lib.mg_kv4_scale_bytes(*bad) == 0
    assert lib.mg_token_logprobs_workspace_bytes(1, 128256, 5) > 0
    for bad in ((0, 100, 5), (-1, 100, 5), (1, 0, 0), (1, 100, 33), (1, 4, 5), (1 << 25, 100, 1), (1, (1 << 30) + 1, 1)):
        assert lib.mg_token_logprobs_workspace_bytes(*bad) == 0


@pytest.mark.parametrize("kw,rc", [(dict(codes=None), ARG), (dict(scales=None), ARG), (dict(codes=P + 8), ARG), (dict(scales=P + 2), ARG),
                                   (dict(n_pages=0), SHAPE), (dict(n_pages=1 << 27), SHAPE), (dict(hkv=0), SHAPE),
                                   (dict(n_pages=(1 << 27) - 1, hkv=1024), SHAPE), (dict(hd=96), SHAPE), (dict(hd=256), SHAPE)])
def test_caches_that_are_refused(kw, rc):
    lib, c = mg.load(), cache(**kw)
    assert lib.mg_kv4_append(C.byref(c), C.byref(app()), None) == rc
    assert lib.mg_kv4_read(C.byref(c), 1, P, P, 128, P, 128, None) == rc
    assert lib.mg_kv4_attention(C.byref(c), C.byref(attn()), P, 1 << 30, None) == rc
    assert lib.mg_kv4_attention_workspace_bytes(C.byref(c), C.byref(attn())) == 0


@pytest.mark.parametrize("kw,rc", [
    (dict(n_tokens=-1), ARG), (dict(n_tokens=1 << 25), ARG), (dict(n_q_heads=-1), SHAPE), (dict(n_q_heads=4097), SHAPE), (dict(q=None), ARG),
    (dict(q=P + 2), ARG), (dict(q_stride=248), ARG), (dict(q_stride=260), ARG), (dict(q_out=None), ARG), (dict(q_out=P + 8), ARG),
    (dict(q_out_stride=0), ARG), (dict(k=None), ARG), (dict(k=P + 2), ARG), (dict(k_stride=120), ARG), (dict(k_stride=-128), ARG),
    (dict(v=None), ARG), (dict(v_stride=132), ARG), (dict(slots=None), ARG), (dict(rope=None), ARG), (dict(rope=P + 4), ARG),
    (dict(n_positions=0), ARG)])
def test_appends_that_are_refused(kw, rc):
    assert mg.load().mg_kv4_append(C.byref(cache()), C.byref(app(**kw)), None) == rc


@pytest.mark.parametrize("kw", [
    dict(q_out=P + 16), dict(q_out=P, q_out_stride=264), dict(q_out=2 * P), dict(q_out=3 * P + 128), dict(q_out=P - 16),
    # columns of one buffer of 512 values a row: q at 0, k at 256, v at 384
    dict(q_stride=512, k=P + 512, k_stride=512, v=P + 768, v_stride=512, q_out=P + 512, q_out_stride=512),
    dict(q_stride=512, k=P + 512, k_stride=512, v=P + 768, v_stride=512, q_out=P + 16, q_out_stride=512)])
def test_queries_on_other_rows_are_refused(kw):
    assert mg.load().mg_kv4_append(C.byref(cache()), C.byref(app(n_tokens=9, **kw)), None) == ARG


def test_appends_of_nothing():
    lib, c = mg.load(), cache()
    assert lib.mg_kv4_append(C.byref(c), C.byref(app(n_tokens=0, q=None, k=None, v=None, slots=None)), None) == 0
    assert lib.mg_kv4_append(None, C.byref(app()), None) == ARG and lib.mg_kv4_append(C.byref(c), None, None) == ARG
    assert lib.mg_kv4_read(C.byref(c), 0, None, None, 0, None, 0, None) == 0
    assert lib.mg_kv4_read(C.byref(c), 4, P, None, 0, None, 0, None) == 0
    ok = [1, P, P, 128, P, 128, None]
    for i, bad in ((0, -1), (0, 1 << 26), (1, None), (2, P + 4), (3, 64), (4, P + 2), (5, 130)):
        assert lib.mg_kv4_read(C.byref(c), *[bad if k == i else x for k, x in enumerate(ok)]) == ARG, (i, bad)


@pytest.mark.parametrize("kw,rc", [
    (dict(n_rows=-1), ARG), (dict(n_q_heads=5), SHAPE), (dict(n_q_heads=34, q_stride=34 * 64, out_stride=34 * 64), SHAPE), (dict(max_new=0), ARG),
    (dict(max_len=-1), ARG), (dict(max_pages_per_row=0), ARG), (dict(window=-1), ARG), (dict(scale=math.nan), ARG), (dict(softcap=-2.0), ARG),
    (dict(q=None), ARG), (dict(q_stride=255), ARG), (dict(out=P + 8), ARG), (dict(page_table=None), ARG), (dict(lens=None), ARG),
    (dict(cu_new=None), ARG), (dict(n_rows=1 << 30, n_tokens=1 << 30), ARG)])
def test_attention_arguments_that_are_refused(kw, rc):
    lib, c, a = mg.load(), cache(), attn(**kw)
    assert lib.mg_kv4_attention(C.byref(c), C.byref(a), P, 1 << 40, None) == rc
    assert lib.mg_kv4_attention_workspace_bytes(C.byref(c), C.byref(a)) == 0


def test_attention_refuses_a_short_workspace_and_work_in_place():
    lib, c = mg.load(), cache(n_pages=1 << 20, hkv=8, hd=128)
    a = attn(n_rows=1, n_tokens=1, n_q_heads=32, max_new=1, max_pages_per_row=1024, q_stride=4096, out_stride=4096)
    need = lib.mg_kv4_attention_workspace_bytes(C.byref(c), C.byref(a))
    assert 0 < need < 64 << 20
    for ws, n in ((None, need), (P, need - 1), (P, 0)):
        assert lib.mg_kv4_attention(C.byref(c), C.byref(a), ws, n, None) == WORKSPACE
    assert lib.mg_kv4_attention(C.byref(c), C.byref(a), P + 4, need, None) == ARG
    a.out = a.q
    assert lib.mg_kv4_attention(C.byref(c), C.byref(a), P, need, None) == ARG
    for kw in (dict(n_rows=0), dict(n_tokens=0)):
        assert lib.mg_kv4_attention(C.byref(cache()), C.byref(attn(q=None, out=None, page_table=None, lens=None, **kw)), None, 0, None) == 0


def test_logprob_arguments_that_are_refused():
    lib = mg.load()
    ok = [3, 100, P, 0, 100, P, 5, 2 * P, 3 * P, 4 * P, 5 * P, 6 * P, 1 << 30, None]
    for i, bad in ((0, -1), (0, (1 << 24) + 1), (1, 0), (1, (1 << 30) + 1), (2, None), (2, P + 2), (3, 2), (4, 99), (4, -100), (5, None), (6, -1),
                   (6, 33), (6, 101)):
        assert lib.mg_token_logprobs(*[bad if k == i else x for k, x in enumerate(ok)]) == ARG, (i, bad)
    big = [1, 128256, P, 0, 128256, P, 5, 2 * P, 3 * P, 4 * P, 5 * P, 6 * P, 0, None]
    need = lib.mg_token_logprobs_workspace_bytes(1, 128256, 5)
    assert lib.mg_token_logprobs(*big) == WORKSPACE
    big[12] = need - 1
    assert lib.mg_token_logprobs(*big) == WORKSPACE
    big[11], big[12] = 6 * P + 4, need
    assert lib.mg_token_logprobs(*big) == ARG
    assert lib.mg_token_logprobs(0, 100, None, 0, 100, None, 0, None, None, None, None, None, 0, None) == 0
    assert lib.mg_token_logprobs(3, 100, P, 0, 100, None, 5, None, None, None, None, None, 0, None) == 0  # nothing is wanted


def test_the_binding_checks_tensors():
    codes, scales = torch.zeros((4, 2, 2, 512), dtype=torch.uint8), torch.zeros((4, 2, 48), dtype=torch.uint8)
    k, q = torch.zeros((3, 2, 64), dtype=torch.bfloat16), torch.zeros((3, 4, 64), dtype=torch.bfloat16)
    s, rope = torch.zeros(3, dtype=torch.int32), torch.zeros((10, 64))
    with pytest.raises(ValueError, match="on the GPU"):
        mg.kv4_append(codes, scales, k, k, s, positions=s, rope=rope, q=q)
    for args, kw in (((codes, scales, k.float(), k, s), {}), ((codes, scales, k[:2], k, s), {}), ((codes, scales, k, k, s.long()), {}),
                     ((codes, scales, k, k.transpose(1, 2), s), {}), ((codes.int(), scales, k, k, s), {}), ((codes[:, :1], scales, k, k, s), {}),
                     ((codes, scales[..., :40], k, k, s), {}), ((codes, scales, k, k, s), dict(positions=s)),
                     ((codes, scales, k, k, s), dict(rope=rope)), ((codes, scales, k, k, s), dict(positions=s[:2], rope=rope)),
                     ((codes, scales, k, k, s), dict(positions=s, rope=rope.double())), ((codes, scales, k, k, s), dict(positions=s, rope=rope[:, :32])),
                     ((codes, scales, k, k, s), dict(positions=s, rope=rope[:0])), ((codes, scales, k, k, s), dict(q=q[..., :32])),
                     ((codes, scales, k, k, s), dict(q=q[0])), ((codes, scales, k, k, s), dict(q_out=q)), ((codes, scales, k, k, s), dict(q=q, q_out=k))):
        with pytest.raises(ValueError):
            mg.kv4_append(*args, **kw)
    with pytest.raises(ValueError):
        mg.kv4_read(codes, scales, s, k_out=k[:, :1])
    t = torch.zeros((3, 4), dtype=torch.int32)
    for call in (mg.kv4_attention, mg.kv4_attention_workspace_bytes):
        for a, kw in (((q[..., :32], t, s), {}), ((q, t, s[:2]), {}), ((q, t.t(), s), {}), ((q, t, s), dict(cu_new=s)), ((q, t, s), dict(window=2 ** 31)),
                      ((q, t, s), dict(max_len=2 ** 40))):
            with pytest.raises(ValueError):
                call(codes, scales, *a, **kw)
    with pytest.raises(mg.MgError):
        mg.kv4_empty(4, 2, 96, device="cpu")
    x = torch.zeros((3, 50))
    with pytest.raises(ValueError, match="on the GPU"):
        mg.token_logprobs(x, s, top=2)
    for a, kw in (((x.double(), s), {}), ((x[0], s), {}), ((x.t()[:3], s), {}), ((x, s.long()), {}), ((x, s[:2]), {}), ((x, s), dict(top=33)),
                  ((x, s), dict(top=-1)), ((x, s), dict(out=mg.TokenLogprobs(s, None, None, None))),
                  ((x, s), dict(top=2, out=mg.TokenLogprobs(None, None, t, None)))):
        with pytest.raises(ValueError):
            mg.token_logprobs(*a, **kw)


def test_the_rotation_s_table():
    t = mg.rope_table(40, 64, 1e4, device="cpu")
    assert t.shape == (40, 64) and t.dtype == torch.float32
    ang = np.arange(40)[:, None] / 1e4 ** (np.arange(32) / 32)
    np.testing.assert_allclose(t[:, 0::2].numpy(), np.cos(ang), rtol=0, atol=2.0 ** -24)
    np.testing.assert_allclose(t[:, 1::2].numpy(), np.sin(ang), rtol=0, atol=2.0 ** -24)


def test_the_reference_rounds_as_defined():
    """The test's own oracle: every e2m1 value keeps itself, halfway goes to the even code, and a scale byte is the least that holds."""
    np.testing.assert_array_equal(ref.round_e2m1(np.concatenate([ref.E2M1, -ref.E2M1])), np.concatenate([ref.E2M1, -ref.E2M1]))
    np.testing.assert_array_equal(ref.round_e2m1(np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.0])), [0, 1, 1, 2, 2, 4, 4, 6])
    for top in (7.0, 7.0000001, 3.5, 1.0, 2.0 ** 127, 3.0e38, 1e-30, 2.0 ** -120):
        b = int(ref.scale_byte(top))
        assert top <= 7 * 2.0 ** (b - 127) and (b == 16 or top > 7 * 2.0 ** (b - 128))
    assert ref.scale_byte(np.inf) == 255 and ref.scale_byte(0.0) == 16
