"""The host side of the batch plan and of the 8-bit K/V cache (CPU): sizes, and what is refused before
any work is enqueued.  The pointers of the refused calls are never followed."""
import ctypes as C
import math

import pytest
import torch

from paper_2605_30218_amd import mg

ARG, SHAPE, WORKSPACE = -1, -2, -3
P = 1 << 20  # an aligned address that no refused call reads


def cache(codes=P, scales=P, n_pages=8, hkv=2, hd=64):
    return mg.MgKv8Cache(codes, scales, n_pages, hkv, hd)


def attn(**kw):
    d = dict(n_rows=3, n_tokens=5, n_q_heads=4, max_new=2, max_len=0, max_pages_per_row=4, window=0, scale=0.0,
             softcap=0.0, q=P, q_stride=256, out=4 * P, out_stride=256, page_table=P, lens=P, cu_new=P) | kw
    a = mg.MgKv8AttnArgs()
    for k, v in d.items():
        setattr(a, k, v)
    return a


def test_sizes():
    lib = mg.load()
    assert lib.mg_kv8_code_bytes(10, 8, 128) == 10 * 8 * 2 * 16 * 128
    assert lib.mg_kv8_scale_bytes(10, 8, 128) == 10 * 8 * 2
    for bad in ((0, 8, 128), (10, 0, 128), (10, 8, 96), (1 << 27, 8, 128), (-1, 8, 64)):
        assert lib.mg_kv8_code_bytes(*bad) == 0 and lib.mg_kv8_scale_bytes(*bad) == 0


@pytest.mark.parametrize("kw,rc", [(dict(codes=None), ARG), (dict(scales=None), ARG), (dict(codes=P + 8), ARG),
                                   (dict(scales=P + 1), ARG),
                                   (dict(n_pages=0), SHAPE), (dict(n_pages=1 << 27), SHAPE), (dict(hkv=0), SHAPE),
                                   (dict(hd=96), SHAPE), (dict(hd=256), SHAPE)])
def test_caches_that_are_refused(kw, rc):
    lib, c, a = mg.load(), cache(**kw), attn()
    assert lib.mg_kv8_append(C.byref(c), 1, P, 128, P, 128, P, None) == rc
    assert lib.mg_kv8_read(C.byref(c), 1, P, P, 128, P, 128, None) == rc
    assert lib.mg_kv8_attention(C.byref(c), C.byref(a), P, 1 << 30, None) == rc
    assert lib.mg_kv8_attention_workspace_bytes(C.byref(c), C.byref(a)) == 0


def test_rows_that_are_refused():
    lib, c = mg.load(), cache()
    ok = [1, P, 128, P, 128, P, None]
    for i, bad in ((0, -1), (0, (1 << 25) + 1), (1, None), (1, P + 2), (2, 120), (2, 132), (2, -128), (3, None), (3, P + 8), (4, 0), (5, None)):
        assert lib.mg_kv8_append(C.byref(c), *[bad if k == i else x for k, x in enumerate(ok)]) == ARG, (i, bad)
    ok = [1, P, P, 128, P, 128, None]
    for i, bad in ((0, -1), (1, None), (2, P + 4), (3, 64), (4, P + 2), (5, 130)):
        assert lib.mg_kv8_read(C.byref(c), *[bad if k == i else x for k, x in enumerate(ok)]) == ARG, (i, bad)
    assert lib.mg_kv8_append(None, *[1, P, 128, P, 128, P, None]) == ARG
    # nothing to do
    assert lib.mg_kv8_append(C.byref(c), 0, None, 0, None, 0, None, None) == 0
    assert lib.mg_kv8_read(C.byref(c), 0, None, None, 0, None, 0, None) == 0
    assert lib.mg_kv8_read(C.byref(c), 4, P, None, 0, None, 0, None) == 0


@pytest.mark.parametrize("kw,rc", [
    (dict(n_rows=-1), ARG), (dict(n_tokens=-1), ARG), (dict(n_q_heads=5), SHAPE), (dict(n_q_heads=0), SHAPE),
    (dict(n_q_heads=34, q_stride=34 * 64, out_stride=34 * 64), SHAPE), (dict(max_new=0), ARG), (dict(max_len=-1), ARG),
    (dict(max_pages_per_row=0), ARG), (dict(max_pages_per_row=1 << 27), ARG), (dict(window=-1), ARG),
    (dict(scale=-1.0), ARG), (dict(scale=1e-38), ARG), (dict(scale=1e16), ARG), (dict(softcap=1e16), ARG),
    (dict(max_pages_per_row=(1 << 26) + 1), ARG), (dict(n_rows=1 << 30, n_tokens=1 << 30), ARG),
    (dict(n_tokens=1 << 30, max_new=1 << 30), ARG), (dict(scale=math.nan), ARG), (dict(scale=math.inf), ARG), (dict(softcap=-2.0), ARG),
    (dict(softcap=math.nan), ARG), (dict(softcap=math.inf), ARG), (dict(softcap=1e-40), ARG), (dict(q=None), ARG),
    (dict(q=P + 2), ARG), (dict(q_stride=255), ARG), (dict(q_stride=248), ARG), (dict(out=None), ARG),
    (dict(out=P + 8), ARG), (dict(out_stride=260), ARG), (dict(page_table=None), ARG), (dict(lens=None), ARG),
    (dict(cu_new=None), ARG), (dict(cu_new=None, n_tokens=3), ARG)])
def test_attention_arguments_that_are_refused(kw, rc):
    lib, c, a = mg.load(), cache(), attn(**kw)
    assert lib.mg_kv8_attention(C.byref(c), C.byref(a), P, 1 << 40, None) == rc
    assert lib.mg_kv8_attention_workspace_bytes(C.byref(c), C.byref(a)) == 0


def test_workspace_follows_the_host_bounds():
    """Splits are taken where rows are few and long, and a bound on the lengths saves them."""
    lib = mg.load()
    c = cache(n_pages=1 << 20, hkv=8, hd=128)

    def need(**kw):
        d = dict(n_rows=1, n_tokens=1, n_q_heads=32, max_new=1, max_pages_per_row=1024, q_stride=4096, out_stride=4096) | kw
        return lib.mg_kv8_attention_workspace_bytes(C.byref(c), C.byref(attn(**d)))

    assert need(max_len=512) == 0
    one = need()
    assert 0 < one < 64 << 20 and need(max_len=4096) <= one
    assert need(window=256) == 0
    assert need(n_rows=256, n_tokens=256, max_len=1024) == 0
    assert 0 < need(n_tokens=64, max_new=64) < 256 << 20
    assert need(n_tokens=8192, max_new=8192, max_len=2048) == 0


def test_attention_refuses_a_short_workspace_and_work_in_place():
    lib, c = mg.load(), cache(n_pages=1 << 20, hkv=8, hd=128)
    a = attn(n_rows=1, n_tokens=1, n_q_heads=32, max_new=1, max_pages_per_row=1024, q_stride=4096, out_stride=4096)
    need = lib.mg_kv8_attention_workspace_bytes(C.byref(c), C.byref(a))
    assert need > 0
    for ws, n in ((None, need), (P, need - 1), (P, 0)):
        assert lib.mg_kv8_attention(C.byref(c), C.byref(a), ws, n, None) == WORKSPACE
    assert lib.mg_kv8_attention(C.byref(c), C.byref(a), P + 4, need, None) == ARG
    a.out = a.q
    assert lib.mg_kv8_attention(C.byref(c), C.byref(a), P, need, None) == ARG


def test_attention_of_nothing():
    lib, c = mg.load(), cache()
    for kw in (dict(n_rows=0), dict(n_tokens=0)):
        a = attn(q=None, out=None, page_table=None, lens=None, **kw)
        assert lib.mg_kv8_attention(C.byref(c), C.byref(a), None, 0, None) == 0


def test_plan_arguments_that_are_refused():
    lib = mg.load()
    ok = [4, 8, P, 2 * P, P, P, 10, P, P, P, P, P, P, P, 2 * P, None]
    bad = [(0, 0), (0, 1025), (1, 0), (1, 1 << 27), (6, -1), (6, (1 << 30) + 1), (14, P), (9, P)]
    ok[9] = 3 * P  # lens: another buffer than ctx_len
    for i, x in bad + [(i, None) for i in (2, 3, 4, 5, 7, 8, 9, 10, 11, 12, 13, 14)]:
        assert lib.mg_batch_plan(*[x if k == i else y for k, y in enumerate(ok)]) == ARG, (i, x)


def test_the_binding_checks_tensors():
    codes, scales = (torch.zeros(s, dtype=torch.uint8) for s in ((4, 2, 2, 1024), (4, 2, 2)))
    k = torch.zeros((3, 2, 64), dtype=torch.bfloat16)
    s = torch.zeros(3, dtype=torch.int32)
    with pytest.raises(ValueError, match="on the GPU"):
        mg.kv8_append(codes, scales, k, k, s)
    for args in ((codes, scales, k.float(), k, s), (codes, scales, k[:2], k, s), (codes, scales, k, k, s.long()),
                 (codes, scales, k, k.transpose(1, 2), s), (codes.int(), scales, k, k, s),
                 (codes[:, :1], scales, k, k, s), (codes, scales[:3], k, k, s)):
        with pytest.raises(ValueError):
            mg.kv8_append(*args)
    with pytest.raises(ValueError):
        mg.kv8_read(codes, scales, s, k_out=k[:, :1])
    q, t = torch.zeros((3, 4, 64), dtype=torch.bfloat16), torch.zeros((3, 4), dtype=torch.int32)
    for kw in (dict(q=q[..., :32]), dict(lens=s[:2]), dict(cu_new=s), dict(page_table=t.t()), dict(page_table=t[0])):
        a = dict(q=q, page_table=t, lens=s) | kw
        with pytest.raises(ValueError):
            mg.kv8_attention(codes, scales, a.pop("q"), a.pop("page_table"), a.pop("lens"), **a)
    with pytest.raises(ValueError):
        mg.batch_plan(s, s, s, s[:1], t, -1)
    with pytest.raises(ValueError):
        mg.batch_plan(s, s[:2], s, s[:1], t, 4)
    with pytest.raises(mg.MgError):
        mg.kv8_empty(4, 2, 96, device="cpu")
