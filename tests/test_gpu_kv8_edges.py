"""The batch plan and the 8-bit paged K/V cache (GPU) at the edges of their contract, against the
definitions in float64 and Python integers (_kv8_ref.py), each row of an attention call within the bound of
its own probabilities."""
import numpy as np
import pytest
import torch

import _kv8_ref as ref
from _gpu_common import dev_i32
from paper_2605_30218_amd import mg
from test_gpu_kv8 import Batch, check_append, check_plan, noisy_cache, rows_bf16, tables

pytestmark = pytest.mark.gpu


def probability_bits(new, G):
    """Per row: 16 bits where the call's rows have at most 32 query rows, or the row itself at most 16; else 8."""
    return [16 if max(new) * G <= 32 or n * G <= 16 else 8 for n in new]


def compare(b, got, cache=None, bits=None, **kw):
    """got against the definition, row by row within the bound of the row's probabilities (bits: the same for all)."""
    kw["scale"] = kw.get("scale") or 1 / np.sqrt(b.hd)
    cache = ref.RefCache.of(b.codes, b.scales) if cache is None else cache
    got, bits = ref.bf16(got), [bits] * len(b.new) if bits else probability_bits(b.new, b.G)
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


# ---------------------------------------------------------------- bounds that a caller need not give


@pytest.mark.parametrize("new", [[1, 1, 1], [3, 1, 2], [4, 0, 9], [70, 1, 20], [0, 0, 0]])
def test_rows_of_several_tokens_without_a_bound_on_them(new):
    """Token offsets alone say how many tokens a row has: without max_new every one of them is answered."""
    b = Batch(np.add([300, 5, 900], new), new, 8, 2, 64, seed=3)
    args = b.codes, b.scales, b.q.cuda(), dev_i32(b.table), dev_i32(b.lens), dev_i32(b.cu)
    n = mg.kv8_attention_workspace_bytes(*args)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    outs = []
    for workspace in (None, ws):
        out = torch.full(b.q.shape, 9.0, dtype=torch.bfloat16, device="cuda")
        outs.append(mg.kv8_attention(*args, out=out, workspace=workspace))
        compare(b, outs[-1], bits=8)
    assert torch.equal(*outs)


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


# ---------------------------------------------------------------- values that are not finite in bf16


def store_one(b, row, pos, head, side, d, x, others=0.0):
    """The page of the row's position anew: x at (pos, head, side, d), `others` elsewhere in that head and side."""
    hkv = b.codes.shape[1]
    page = int(b.table[row, pos // 16])
    old_k, old_v = mg.kv8_read(b.codes, b.scales, dev_i32(16 * page + np.arange(16)))
    kv = [old_k, old_v]
    kv[side][:, head] = others
    kv[side][pos % 16, head, d] = x
    mg.kv8_append(b.codes, b.scales, *kv, dev_i32(16 * page + np.arange(16)))


def not_finite_as_nan(b):
    """The cache with NaN for the values of V that bf16 does not hold."""
    c = ref.RefCache.of(b.codes, b.scales)
    v = c.val[:, :, 1]
    v[np.abs(v) >= 2.0 ** 128] = np.nan
    return c


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("new", [[1, 1, 1], [4, 2, 3], [12, 16, 9], [100, 1, 65]])
@pytest.mark.parametrize("window", [0, 40])
@pytest.mark.parametrize("x", [3.38e38, -3.38e38])
def test_a_value_that_reads_as_infinity_reaches_only_who_sees_it(hd, new, window, x):
    """V above 1.9375 * 2^127 at the last position, behind the length and before the window."""
    b = Batch(np.add([50, 77, 200], new), new, 4, 2, hd, seed=7)
    L = b.lens
    store_one(b, 0, int(L[0]) - 1, 0, 1, 3, x)
    store_one(b, 0, 2, 1, 1, 5, x)
    if L[1] % 16:
        store_one(b, 1, int(L[1]), 1, 1, 9, x)
    store_one(b, 2, int(L[2]) - new[2] // 2 - 1, 1, 1, 40, x)
    cache = not_finite_as_nan(b)
    assert np.isnan(cache.val).any()
    got = b.run(window=window)
    got = compare(b, torch.where(got.isinf(), torch.nan, got), cache=cache, window=window)  # (who sees it: infinity or NaN)
    assert np.isnan(got).any() and not np.isnan(got).all()


@pytest.mark.parametrize("byte", [246, 247, 248, 251, 254])
@pytest.mark.parametrize("new", [[1, 1], [5, 8], [70, 40]])
@pytest.mark.parametrize("hd", [64, 128])
def test_every_code_under_a_large_scale_has_no_effect_where_it_is_not_seen(byte, new, hd):
    """The last page of a row: zeros up to the row's end, V's other positions hold every code under a scale whose larger
    codes stand for infinity."""
    b = Batch(np.add([36, 104], new) // 16 * 16 + 4, new, 4, 2, hd, seed=8)
    idx = ref.byte_index(hd, 1)
    for r in range(2):
        page = int(b.table[r, (b.lens[r] - 1) // 16])
        codes = np.zeros((2, 16 * hd), np.uint8)
        codes[:, idx[4:].ravel()] = np.resize(np.arange(256), 12 * hd)
        b.codes[page, :, 1] = torch.as_tensor(codes).cuda()
        b.scales[page, :, 1] = byte
    got = run_and_compare(b)
    assert np.isfinite(got).all()


# ---------------------------------------------------------------- scale bytes


@pytest.mark.parametrize("byte", [16, 230, 247, 253, 254])
@pytest.mark.parametrize("hkv,hd", [(1, 64), (4, 128)])
@pytest.mark.parametrize("start,n", [(3, 1), (3, 7), (20, 12)])
def test_append_to_a_page_of_any_scale(byte, hkv, hd, start, n):
    """Pages of another program under scales up to the largest: codes stay where the scale does, the new values are rounded
    to it."""
    rng = np.random.RandomState(byte)
    codes, scales = noisy_cache(rng, 2, hkv, hd)
    scales.fill_(byte)
    k, v = (rows_bf16(rng, (n, hkv, hd)) * torch.tensor(2.0 ** (byte - 127)).to(torch.bfloat16) for _ in range(2))
    check_append(codes, scales, k, v, np.arange(start, start + n, dtype=np.int32), ref.RefCache.of(codes, scales))


# ---------------------------------------------------------------- every refill of the page ids, every variant


def with_holes(b, seed):
    rng = np.random.RandomState(seed)
    for r in range(len(b.lens)):
        n = -(-int(b.lens[r]) // 16)
        if n < 24:
            continue
        at = np.concatenate([rng.randint(0, n, n // 12), [x for x in (31, 32, 33, 63, 64, 65, 127, 128, 180, 212) if x < n - 8]])
        b.table[r, at.astype(np.int64)] = rng.choice([-1, -9, 10 ** 6], len(at))
    return b


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("holes,window", [(False, 0), (True, 0), (True, 3100)])
def test_chunks_whose_groups_pass_many_pages(hd, holes, window):
    """Tiles that one block takes whole: up to 150 pages a group of waves, so their ids are fetched three times."""
    b = Batch(np.add([4500, 10, 0, 2100], 130), [130] * 4, 32, 8, hd, seed=31)
    run_and_compare(with_holes(b, 1) if holes else b, window=window)


@pytest.mark.parametrize("holes", [False, True])
@pytest.mark.parametrize("ctx,new", [([4000], [200]), ([9000, 3], [64, 33])])
def test_split_chunks_of_long_contexts(holes, ctx, new):
    b = Batch(np.add(ctx, new), new, 16, 4, 64, seed=32)
    run_and_compare(with_holes(b, 2) if holes else b)


@pytest.mark.parametrize("hq,hkv,rows", [(8, 2, 3), (32, 8, 7)])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("holes,window,cap", [(False, 0, 0.0), (True, 0, 0.0), (True, 4700, 20.0)])
def test_long_short_rows_beside_a_chunk(hq, hkv, rows, hd, holes, window, cap):
    """Rows of few tokens that are split and joined in the launch of the chunks: at 128 pages a split where these rows'
    blocks are few, at 256 where they are not."""
    new = [1, 60, 4] + [1] * (rows - 3)
    ctx = [6000, 90, 5200] + [20 + 700 * i for i in range(rows - 3)]
    b = Batch(np.add(ctx, new), new, hq, hkv, hd, seed=33)
    run_and_compare(with_holes(b, 3) if holes else b, window=window, softcap=cap)


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("new", [1, 3])
def test_splits_of_many_pages(hd, new):
    """65 rows, so that the blocks do not share the lengths: splits of up to 128 pages, whose ids are fetched twice."""
    lens = [9, 3100, 40, 2900] + [20 + i for i in range(61)]
    run_and_compare(with_holes(Batch(lens, [new] * 65, 16, 8, hd, seed=34), 4))


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("holes,window,cap", [(True, 0, 0.0), (False, 900, 0.0), (False, 0, 20.0), (True, 2500, 50.0)])
@pytest.mark.parametrize("hq,new", [(8, 1), (32, 1), (28, 4), (32, 5)])
def test_even_splits_with_holes_windows_and_caps(hq, new, hd, holes, window, cap):
    """One long row among many: splits that follow all rows' lengths, of one tile of query rows and of two."""
    hkv = 4 if hq == 28 else 8
    lens = [7000, 0, 40, 3000] + [5 * i + 6 for i in range(44)]
    b = Batch(lens, [min(new, n) if i % 7 else 1 for i, n in enumerate(lens)], hq, hkv, hd, seed=35)
    run_and_compare(with_holes(b, 5) if holes else b, window=window, softcap=cap)


@pytest.mark.parametrize("hq,hkv,hd", [(32, 8, 128), (28, 4, 128), (4, 2, 64)])
@pytest.mark.parametrize("new", [[1, 1, 1], [4, 2, 4], [10, 16, 12], [80, 1, 3]])
@pytest.mark.parametrize("cap,window", [(0.5, 0), (30.0, 0), (30.0, 90), (1e5, 0)])
def test_caps_on_every_kind_of_block(hq, hkv, hd, new, cap, window):
    run_and_compare(Batch(np.add([300, 5, 1300], new), new, hq, hkv, hd, seed=36), softcap=cap, window=window)


@pytest.mark.parametrize("hq,hkv,hd", [(28, 4, 128), (32, 8, 128), (4, 2, 64)])
@pytest.mark.parametrize("new", [[4, 3, 4], [8, 1, 5], [60, 2, 1, 4]])
def test_probabilities_keep_their_bits(hq, hkv, hd, new):
    """16 bits for rows of up to 32 query rows among their kind, and for rows of up to 16 beside longer ones."""
    b = Batch(np.add([400, 90, 1500, 33][:len(new)], new), new, hq, hkv, hd, seed=37)
    run_and_compare(b)


@pytest.mark.parametrize("x", [np.inf, -np.inf])
@pytest.mark.parametrize("new", [[1, 1, 1], [6, 2, 4], [40, 1, 30]])
def test_an_infinite_query_stays_in_its_row(x, new):
    b = Batch(np.add([50, 77, 200], new), new, 4, 2, 64, seed=8)
    b.q[b.cu[1] - 1, 2, 7] = float(x)
    got = ref.bf16(b.run())
    clean = b.q.clone()
    clean[b.cu[1] - 1, 2, 7] = 0.0
    out, bound = ref.attention(ref.RefCache.of(b.codes, b.scales), ref.bf16(clean), b.table, b.lens, b.cu, 1 / 8,
                               p_bits=8 if max(new) > 16 else 16)
    ok = np.abs(got - out) <= bound
    ok[b.cu[1] - 1, 2] = True
    assert ok.all()


# ---------------------------------------------------------------- the plan


@pytest.mark.parametrize("n_free,most,admitted", [(100, 100, [1, 1, 1, 1, 1]), (4, 100, [1, 1, 1, 0, 0]), (3, 100, [1, 1, 0, 0, 0]),
                                                  (100, 39, [1, 1, 0, 0, 0]), (100, 20, [1, 1, 0, 0, 0]), (0, 100, [0, 0, 0, 0, 0]),
                                                  (100, 0, [0, 0, 0, 0, 0])])
def test_plan_admits_these_rows(n_free, most, admitted):
    """Rows of 20, 0, 20, 1 and 0 new tokens, of 2, 0, 2, 1 and 0 new pages."""
    ctx, new = np.array([0, 7, 16, 32, 5]), np.array([20, 0, 20, 1, 0])
    table, free = tables(np.random.RandomState(0), ctx, 4, 100)
    got = check_plan(ctx, new, free, n_free, table, most)
    assert got["admitted"].tolist() == admitted


def test_plan_gives_no_slot_on_a_page_that_is_not_there():
    """A row whose table lacks the page of its next position: no slot of another page stands for it."""
    missing = [-1, -2 ** 27, -2 ** 31, 2 ** 27, 2 ** 31 - 1, -2 ** 28 + 3]
    table = np.full((len(missing), 3), -1, np.int32)
    table[:, 0] = missing
    p = mg.batch_plan(dev_i32([5] * 6), dev_i32([13] * 6), dev_i32(np.arange(40)), dev_i32([40]), dev_i32(table), 100)
    slots, at = p.slots.cpu().numpy()[:78].reshape(6, 13), 39 - np.arange(6)
    assert (slots[:, :11] == -1).all()
    np.testing.assert_array_equal(slots[:, 11:], 16 * at[:, None] + [0, 1])


@pytest.mark.parametrize("new,admitted", [([1, 3, 0], [1, 1, 1]), ([0, 0, 0], [1, 1, 1]), ([1, 9, 2], [1, 0, 0])])
def test_plan_without_a_free_page(new, admitted):
    """An empty list of free pages: what fits the rows' own pages is admitted."""
    ctx, table = np.array([5, 8, 30]), np.array([[3, -1], [0, -1], [2, 1]], np.int32)
    got = check_plan(ctx, np.array(new), np.array([], np.int32), 0, table, 20)
    assert got["admitted"].tolist() == admitted
