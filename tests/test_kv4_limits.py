"""The largest calls of the 4-bit K/V cache and of token log probabilities (CPU): what a launch cannot take is refused before any work is enqueued.  The
pointers of the refused calls are never followed."""
import ctypes as C

import pytest

from paper_2605_30218_amd import mg

ARG, SHAPE = -1, -2
P = 1 << 20  # an aligned address that no refused call reads


def test_log_probabilities_of_more_rows_than_a_launch_takes():
    """A row has a block of 256 threads, and 2^24 of these are the 2^32 threads that no launch has."""
    lib = mg.load()
    call = lambda n: lib.mg_token_logprobs(n, 2, P, 0, 2, P, 1, 2 * P, 3 * P, 4 * P, 5 * P, 6 * P, 1 << 40, None)  # noqa: E731
    assert call(1 << 24) == ARG and call((1 << 24) + 1) == ARG
    assert lib.mg_token_logprobs_workspace_bytes(1 << 24, 128256, 5) == 0


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("n", [(1 << 25) + 1, 59700000, 63200000, 1 << 26])
def test_appends_of_more_tokens_than_a_launch_takes(n, hd):
    """A token's values take 64 threads whatever its heads, so pairs alone do not bound a call of one KV head and no queries."""
    c = mg.MgKv4Cache(P, P, 8, 1, hd)
    a = mg.MgKv4AppendArgs(n, 0, None, 0, None, 0, 2 * P, hd, 3 * P, hd, P, None, None, 0)
    assert mg.load().mg_kv4_append(C.byref(c), C.byref(a), None) == ARG


@pytest.mark.parametrize("n_pages,hkv", [((1 << 27) - 1, 1024), (1 << 21, 1024), (1 << 26, 32)])
def test_sizes_of_caches_that_the_calls_refuse_are_zero(n_pages, hkv):
    """A page of a head has a number of 31 bits."""
    lib = mg.load()
    for hd in (64, 128):
        c = mg.MgKv4Cache(P, P, n_pages, hkv, hd)
        assert lib.mg_kv4_read(C.byref(c), 1, P, P, hkv * hd, P, hkv * hd, None) == SHAPE
        assert lib.mg_kv4_code_bytes(n_pages, hkv, hd) == 0 and lib.mg_kv4_scale_bytes(n_pages, hkv, hd) == 0
        assert lib.mg_kv4_code_bytes((1 << 31) // hkv - 1, hkv, hd) == ((1 << 31) // hkv - 1) * hkv * 16 * hd
    with pytest.raises(mg.MgError):
        mg.kv4_empty(n_pages, hkv, 128, device="cpu")
