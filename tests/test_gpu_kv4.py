"""The 4-bit paged K/V cache (GPU) against its definitions in float64 (_kv4_ref.py): rotation, append and read bit for bit, attention
within the bound that its roundings give."""
import numpy as np
import pytest
import torch

import _kv4_ref as ref
from _gpu_common import dev_i32
from _kv8_ref import bf16
from paper_2605_30218_amd import mg

pytestmark = pytest.mark.gpu

THETA = 5e5


def rows(rng, shape, std=1.0):
    return torch.as_tensor((std * rng.randn(*shape)).astype(np.float32)).to(torch.bfloat16)


def same_bits(got, want):
    """bf16 tensor against float64 values, NaN against NaN, the signs of zeros too."""
    np.testing.assert_array_equal(bf16(got), want)
    zero = want == 0
    np.testing.assert_array_equal(np.signbit(bf16(got))[zero], np.signbit(want)[zero])


# ---------------------------------------------------------------- rotation, append, read


def check_append(cache, want, k, v, slots, pos=None, q=None, table=None, **kw):
    """One append, against the definition; want: the RefCache that stands for `cache` before it."""
    args = dict(positions=dev_i32(pos), rope=torch.as_tensor(table).cuda()) if pos is not None else {}
    out = mg.kv4_append(*cache, k.cuda(), v.cuda(), dev_i32(slots), q=None if q is None else q.cuda(), **args, **kw)
    kk, vv, slots = bf16(k), bf16(v), np.array(slots)
    if pos is not None:
        pos = np.array(pos)
        slots[pos < 0] = -1
        kk = ref.rotate(kk, table, np.maximum(pos, 0))
    want.append(kk, vv, slots)
    got, _, _ = ref.unpack(*cache)
    np.testing.assert_array_equal(got, want.val)
    if q is not None:
        live = np.ones(len(slots), bool) if pos is None else pos >= 0
        qq = bf16(q) if pos is None else ref.rotate(bf16(q), table, np.maximum(pos, 0))
        same_bits(out[torch.as_tensor(live).cuda()], qq[live])
    return out


def table_of(n, hd):
    t = mg.rope_table(n, hd, THETA, device="cpu").numpy()
    ang = np.arange(n)[:, None] * THETA ** (-2.0 * np.arange(hd // 2) / hd)
    np.testing.assert_array_equal(t, np.stack([np.cos(ang), np.sin(ang)], -1).reshape(n, hd).astype(np.float32))
    return t


@pytest.mark.parametrize("hq,hkv,hd", [(4, 2, 64), (32, 8, 128), (7, 1, 128), (28, 4, 128), (3, 3, 64), (65, 5, 64)])
@pytest.mark.parametrize("piece", [1, 3, 4, 37])
def test_append_in_pieces(hq, hkv, hd, piece):
    """A request's positions on scattered pages, `piece` at a time, rotated with their queries."""
    rng = np.random.RandomState(hq + piece)
    n, pages = 37 if piece < 37 else 74, rng.permutation(7)[:5]
    cache, want = mg.kv4_empty(7, hkv, hd), ref.RefCache(7, hkv, hd)
    t = table_of(80, hd)
    for a in range(0, n, piece):
        p = np.arange(a, min(a + piece, n))
        m = len(p)
        check_append(cache, want, rows(rng, (m, hkv, hd), 2.0), rows(rng, (m, hkv, hd)), pages[p // 16] * 16 + p % 16, p, rows(rng, (m, hq, hd)), t)


def test_append_of_many_requests_with_padding():
    """Ragged rows, each from anywhere in a page, tokens without a slot and tokens left out between them."""
    rng = np.random.RandomState(3)
    hq, hkv, hd = 8, 2, 128
    slots, pos = [], []
    pages = iter(rng.permutation(200))
    for _ in range(40):
        a, n = rng.randint(0, 60), rng.randint(0, 40)
        own = [next(pages) for _ in range((a + n + 15) // 16 - a // 16)]
        slots += [own[p // 16 - a // 16] * 16 + p % 16 for p in range(a, a + n)]
        pos += list(range(a, a + n))
    slots, pos = np.array(slots), np.array(pos)
    drop = rng.rand(len(pos)) < 0.1
    slots[rng.rand(len(pos)) < 0.1] = -1
    slots[5], slots[9] = 200 * 16, 2 ** 31 - 1  # behind the cache
    pos[drop] = -1 - rng.randint(0, 5, drop.sum())
    pos[11], pos[12] = 100, 2 ** 31 - 1       # behind the table
    n = len(pos)
    cache, want = mg.kv4_empty(200, hkv, hd), ref.RefCache(200, hkv, hd)
    q = rows(rng, (n, hq, hd))
    out = torch.full((n, hq, hd), 7.0, dtype=torch.bfloat16, device="cuda")
    check_append(cache, want, rows(rng, (n, hkv, hd)), rows(rng, (n, hkv, hd)), slots, pos, q, table_of(100, hd), q_out=out)
    assert (out[torch.as_tensor(pos < 0).cuda()] == 7.0).all()
    assert np.isnan(want.val).any() == bool(slots[11] >= 0 or slots[12] >= 0)


def test_append_without_rotation_and_without_queries():
    rng = np.random.RandomState(4)
    cache, want = mg.kv4_empty(3, 2, 64), ref.RefCache(3, 2, 64)
    k, v, q = rows(rng, (5, 2, 64)), rows(rng, (5, 2, 64)), rows(rng, (5, 4, 64))
    assert check_append(cache, want, k, v, [30, 31, 32, 33, 34]) is None
    check_append(cache, want, k, v, [1, 2, 3, 4, 5], q=q)
    check_append(cache, want, k[:0], v[:0], [])


def test_append_in_place_of_a_projection_s_rows():
    """q, k and v as the columns of one buffer, the rotated queries in place; the rest of the buffer stays."""
    rng = np.random.RandomState(5)
    hq, hkv, hd, n = 8, 2, 128, 21
    buf = rows(rng, (n, hq + 2 * hkv + 1, hd)).cuda()
    before = buf.clone()
    t = table_of(64, hd)
    cache, want = mg.kv4_empty(4, hkv, hd), ref.RefCache(4, hkv, hd)
    q = buf[:, :hq]
    pos = np.arange(10, 10 + n)
    out = mg.kv4_append(*cache, buf[:, hq:hq + hkv], buf[:, hq + hkv:hq + 2 * hkv], dev_i32(pos), positions=dev_i32(pos),
                        rope=torch.as_tensor(t).cuda(), q=q, q_out=q)
    assert out is q
    same_bits(buf[:, :hq], ref.rotate(bf16(before[:, :hq]), t, pos))
    assert torch.equal(buf[:, hq:], before[:, hq:])
    want.append(ref.rotate(bf16(before[:, hq:hq + hkv]), t, pos), bf16(before[:, hq + hkv:hq + 2 * hkv]), pos)
    np.testing.assert_array_equal(ref.unpack(*cache)[0], want.val)


@pytest.mark.parametrize("hd", [64, 128])
def test_every_bf16_value_is_coded_as_defined(hd):
    """All 2^16 bit patterns as values of V and K, each block's values near each other and far apart."""
    x = torch.arange(-32768, 32768, dtype=torch.int32).to(torch.int16).view(torch.bfloat16)
    for y in (x, x.view(256, 256).t().contiguous().view(-1)):
        y = y.view(-1, 1, hd)
        cache, want = mg.kv4_empty(len(y) // 16, 1, hd), ref.RefCache(len(y) // 16, 1, hd)
        check_append(cache, want, y, y, np.arange(len(y)))
        s = dev_i32(np.arange(len(y)))
        k, v = mg.kv4_read(*cache, s)
        for got, side in ((k, 0), (v, 1)):
            w = ref.to_bf16(want.val[:, 0, side].reshape(-1, 1, hd))
            np.testing.assert_array_equal(bf16(got), w)


@pytest.mark.parametrize("scale", [1e-38, 1e-30, 1.0, 3e38])
def test_appended_values_of_any_size(scale):
    rng = np.random.RandomState(6)
    cache, want = mg.kv4_empty(4, 3, 64), ref.RefCache(4, 3, 64)
    check_append(cache, want, rows(rng, (40, 3, 64), scale), rows(rng, (40, 3, 64), scale), np.arange(3, 43), np.arange(40),
                 rows(rng, (40, 3, 64), scale), table_of(40, 64))


@pytest.mark.parametrize("hkv,hd,n", [(1, 64, 1), (8, 128, 77), (3, 64, 200)])
def test_read_gives_every_slot_and_leaves_rows_outside(hkv, hd, n):
    rng = np.random.RandomState(n)
    cache, want = mg.kv4_empty(9, hkv, hd), ref.RefCache(9, hkv, hd)
    check_append(cache, want, rows(rng, (144, hkv, hd)), rows(rng, (144, hkv, hd)), np.arange(144))
    s = rng.randint(0, 144, n)
    s[rng.rand(n) < 0.2] = rng.choice([-1, 144, 2 ** 31 - 1, -2 ** 31])
    out = torch.full((n, 2 * hkv, hd), 5.0, dtype=torch.bfloat16, device="cuda")
    k, v = mg.kv4_read(*cache, dev_i32(s), k_out=out[:, :hkv], v_out=out[:, hkv:])
    live = (s >= 0) & (s < 144)
    for x, side in ((k, 0), (v, 1)):
        x = bf16(x)
        np.testing.assert_array_equal(x[live], want.val[s[live] // 16, :, side, s[live] % 16])
        assert (x[~live] == 5.0).all()


# ---------------------------------------------------------------- attention


def tables(rng, lens, maxp, spare):
    held = [max(0, min(maxp, -(-int(c) // 16))) for c in lens]
    pool = rng.permutation(sum(held) + spare).astype(np.int32)
    t = np.full((len(lens), maxp), -1, np.int32)
    o = 0
    for b, k in enumerate(held):
        t[b, :k] = pool[o:o + k]
        o += k
    return t, len(pool)


class Batch:
    """Rows of lengths lens with new tokens each, over a filled cache."""

    def __init__(self, lens, new, hq, hkv, hd, seed=0, spare=1, std=1.0):
        rng = np.random.RandomState(seed)
        self.lens, self.new = np.asarray(lens), np.asarray(new)
        self.table, n = tables(rng, self.lens, max(1, -(-int(max(self.lens.max(), 1)) // 16)) + spare, 3)
        k = rows(rng, (16 * n, hkv, hd), std) * torch.as_tensor(np.exp(0.4 * rng.randn(hkv, hd))).to(torch.bfloat16)
        v = rows(rng, (16 * n, hkv, hd)) * torch.as_tensor(np.exp(rng.randn(16 * n, 1, 1))).to(torch.bfloat16)
        self.codes, self.scales = mg.kv4_empty(n, hkv, hd)
        mg.kv4_append(self.codes, self.scales, k.cuda(), v.cuda(), dev_i32(np.arange(16 * n)))
        self.cu = np.concatenate([[0], np.cumsum(self.new)])
        self.q = rows(rng, (int(self.cu[-1]), hq, hd))
        self.hd, self.G = hd, hq // hkv

    def run(self, **kw):
        return mg.kv4_attention(self.codes, self.scales, self.q.cuda(), dev_i32(self.table), dev_i32(self.lens),
                                cu_new=dev_i32(self.cu), max_new=max(1, int(self.new.max())), **kw)

    def check(self, got=None, **kw):
        got = self.run(**kw) if got is None else got
        kw.pop("max_len", None)
        kw["scale"] = kw.get("scale") or 1 / np.sqrt(self.hd)
        most = int(self.new.max()) * self.G
        args = (ref.RefCache.of(self.codes, self.scales), bf16(self.q), self.table, self.lens, self.cu)
        out, bound = ref.attention(*args, **kw)
        got = bf16(got)
        np.testing.assert_array_equal(np.isnan(got), np.isnan(out))
        worst = np.nanmax(np.abs(got - out) / np.where(bound > 0, bound, 1e-38)) if out.size else 0.0
        assert worst <= 1.0, f"{worst} of the bound"
        return got


HEADS = [(32, 8, 128), (40, 8, 128), (28, 4, 128), (4, 2, 64), (8, 8, 64), (16, 1, 128), (3, 1, 64)]


@pytest.mark.parametrize("hq,hkv,hd", HEADS)
def test_single_tokens(hq, hkv, hd):
    Batch([1, 2, 15, 16, 17, 31, 33, 100, 127, 128, 129, 257, 600], [1] * 13, hq, hkv, hd).check()


@pytest.mark.parametrize("hq,hkv,hd", [(4, 2, 64), (28, 4, 128)])
@pytest.mark.parametrize("lens", [[5000], [1], [2049, 64, 3], [700] * 40, [16] * 100, [1023, 1024, 1025]])
def test_single_tokens_of_other_batches(hq, hkv, hd, lens):
    Batch(lens, [1] * len(lens), hq, hkv, hd, seed=len(lens)).check()


@pytest.mark.parametrize("hq,hkv,hd", HEADS)
@pytest.mark.parametrize("n", [2, 4, 7])
def test_few_tokens(hq, hkv, hd, n):
    Batch([n, n + 1, 40, 333, 1100], [n] * 5, hq, hkv, hd, seed=n).check()


@pytest.mark.parametrize("hq,hkv,hd", HEADS)
@pytest.mark.parametrize("ctx,new", [([0, 0], [33, 130]), ([17, 500], [200, 64]), ([3000], [70])])
def test_chunks(hq, hkv, hd, ctx, new):
    Batch(np.add(ctx, new), new, hq, hkv, hd, seed=sum(new)).check()


@pytest.mark.parametrize("hq,hkv,hd", [(32, 8, 128), (4, 2, 64)])
def test_mixed_batches_with_empty_rows(hq, hkv, hd):
    new = [1, 70, 0, 1, 5, 1, 0, 300, 2, 1]
    ctx = [40, 0, 50, 0, 900, 333, 0, 200, 15, 1000]
    Batch(np.add(ctx, new), new, hq, hkv, hd).check()


@pytest.mark.parametrize("window", [1, 16, 100, 2000, 2 ** 31 - 1])
@pytest.mark.parametrize("new", [[1, 1, 1, 1], [3, 1, 2, 4], [150, 1, 90, 20]])
def test_window(window, new):
    Batch(np.add([0, 40, 333, 1300], new), new, 8, 2, 128, seed=3).check(window=window)


@pytest.mark.parametrize("cap", [0.5, 20.0, 1e5])
@pytest.mark.parametrize("hq,hkv,hd,new", [(28, 4, 64, [1, 1, 1]), (28, 4, 128, [4, 1, 3]), (8, 2, 128, [80, 1, 3])])
def test_softcap_and_scale(cap, hq, hkv, hd, new):
    Batch(np.add([33, 200, 700], new), new, hq, hkv, hd, seed=4).check(softcap=cap, scale=0.3, window=150 if cap == 20 else 0)


@pytest.mark.parametrize("new", [[1, 1], [5, 1], [100, 40]])
def test_large_scores(new):
    """Scores of some hundreds: one position has all the weight."""
    Batch(np.add([300, 70], new), new, 8, 2, 64, seed=15, std=40.0).check()


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("window", [0, 300])
@pytest.mark.parametrize("new", [[1, 1], [90, 40]])
@pytest.mark.parametrize("to", [0.02, 30.0])
def test_scores_that_rise_and_fall_over_the_positions(hd, window, new, to):
    """Keys that grow (or shrink) by a power over the positions, so that the reference moves in some steps and for some rows only."""
    b = Batch(np.add([1500, 700], new), new, 8, 2, hd, seed=29)
    rng = np.random.RandomState(31)
    for r, n in enumerate(b.lens):
        j = np.arange(n)
        slots = b.table[r, j // 16] * 16 + j % 16
        k = rows(rng, (n, 2, hd)) * torch.as_tensor(to ** (j / n)[:, None, None]).to(torch.bfloat16)
        mg.kv4_append(b.codes, b.scales, k.cuda(), rows(rng, (n, 2, hd)).cuda(), dev_i32(slots))
    b.check(window=window)


@pytest.mark.parametrize("new", [[1, 1, 1, 1], [20, 2, 33, 4]])
def test_rows_that_see_nothing(new):
    """No positions, fewer positions than tokens, all pages unmapped, lengths past the table."""
    b = Batch([200, 64, 50, 130], new, 4, 2, 64, seed=5, spare=0)
    b.lens = np.array([0, min(1, new[1] - 1), 50, 10 ** 6])
    b.table[2] = -1
    got = b.check()
    assert (got[:b.cu[1]] == 0).all() and (got[b.cu[2]:b.cu[3]] == 0).all()


@pytest.mark.parametrize("new", [[1, 1, 1], [6, 1, 2], [120, 1, 3]])
@pytest.mark.parametrize("window", [0, 90])
def test_holes_in_the_page_table(new, window):
    b = Batch(np.add([333, 500, 20], new), new, 8, 2, 128, seed=6)
    b.table[0, 3:6] = -1
    b.table[0, 9] = 10 ** 6
    b.table[1, 0::2] = -7
    b.table[1, 31:] = -1
    b.check(window=window)


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("new", [[1, 1, 1], [4, 2, 3], [100, 1, 65]])
@pytest.mark.parametrize("window", [0, 40])
def test_nan_reaches_only_who_sees_it(hd, new, window):
    """Blocks of K and V that are not finite, at single positions: behind the length, outside the window, later than a token."""
    b = Batch(np.add([50, 77, 200], new), new, 4, 2, hd, seed=7)
    L = b.lens

    def poison(row, pos, head, at):
        b.scales[int(b.table[row, pos // 16]), head, at + pos % 16] = 255

    poison(0, int(L[0]) - 1, 0, hd // 2)        # the last position's value, seen by the last token alone
    poison(0, 2, 1, hd // 2)
    if L[1] % 16:                               # behind the length, on a mapped page
        poison(1, int(L[1]), 1, hd // 2)
        poison(1, int(L[1]), 1, 16)
    poison(2, 150, 0, 16)                       # features 32 .. 63 of a key
    poison(2, int(L[2]) - new[2] // 2 - 1, 1, hd // 2)
    got = b.check(window=window)
    assert np.isnan(got).any() and not np.isnan(got).all()


@pytest.mark.parametrize("x", [np.nan, np.inf, -np.inf])
@pytest.mark.parametrize("new", [[1, 1, 1], [6, 2, 4], [40, 1, 30]])
def test_what_is_not_finite_in_a_query_stays_in_its_row(x, new):
    b = Batch(np.add([50, 77, 200], new), new, 4, 2, 64, seed=8)
    clean = bf16(b.run())
    b.q[b.cu[1] - 1, 2, 7] = float(x)
    got = bf16(b.run())
    assert np.isnan(got[b.cu[1] - 1, 2]).all()
    got[b.cu[1] - 1, 2] = clean[b.cu[1] - 1, 2]
    np.testing.assert_array_equal(got, clean)


@pytest.mark.parametrize("new", [[1, 1], [40, 3]])
def test_queries_and_values_of_very_unequal_size(new):
    """Queries, keys and values over many powers of two, within a block and from block to block."""
    rng = np.random.RandomState(16)
    b = Batch(np.add([300, 130], new), new, 8, 2, 128, seed=17)
    b.q = (b.q.float() * torch.as_tensor(np.exp2(rng.randint(-12, 2, b.q.shape)).astype(np.float32))).to(torch.bfloat16)
    b.scales[:, :, 64:] = torch.as_tensor(rng.randint(60, 190, tuple(b.scales[:, :, 64:].shape)), dtype=torch.uint8).cuda()
    b.check()


def test_strided_rows_and_rows_behind_the_last_token():
    new = [1, 20, 1]
    b = Batch(np.add([50, 77, 200], new), new, 4, 2, 64, seed=9)
    T = int(b.cu[-1])
    wide = torch.zeros((T + 3, 8, 64), dtype=torch.bfloat16, device="cuda")
    wide[:T, :4] = b.q.cuda()
    out = torch.full((T + 3, 6, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    mg.kv4_attention(b.codes, b.scales, wide[:, :4], dev_i32(b.table), dev_i32(b.lens), cu_new=dev_i32(b.cu),
                     max_new=20, out=out[:, :4])
    b.check(out[:T, :4])
    assert (out[T:] == 7.0).all() and (out[:, 4:] == 7.0).all()


@pytest.mark.parametrize("max_len", [1, 64, 5000])
def test_max_len_shapes_the_launch_only(max_len):
    for new in ([1, 1], [40, 1]):
        Batch(np.add([700, 130], new), new, 8, 2, 128, seed=11).check(max_len=max_len)


def test_without_token_offsets_every_row_has_one():
    b = Batch([3, 70, 200], [1, 1, 1], 8, 2, 128, seed=10)
    b.check(mg.kv4_attention(b.codes, b.scales, b.q.cuda(), dev_i32(b.table), dev_i32(b.lens)))


@pytest.mark.parametrize("max_len", [0, 700])
@pytest.mark.parametrize("hq,hkv,hd,new", [(8, 2, 128, 1), (28, 4, 64, 4), (32, 8, 64, 3)])
def test_rows_of_very_unequal_length(hq, hkv, hd, new, max_len):
    """One long row among short, empty and absent ones, within the host's bound and past it."""
    rng = np.random.RandomState(hq + new)
    for lens in ([6000, 0, 40, 17, 3000, 5], list(rng.randint(0, 5000, 24)), [7000] + [90] * 63):
        n = [0 if i % 5 == 4 else min(new, l) if l else 1 for i, l in enumerate(lens)]
        Batch(lens, n, hq, hkv, hd, seed=len(lens)).check(max_len=max_len)


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("holes,window,cap,long", [(False, 0, 0.0, 5000), (True, 4700, 20.0, 5000), (False, 0, 0.0, 9000), (True, 8700, 20.0, 12000)])
def test_long_short_rows_beside_a_chunk(hd, holes, window, cap, long):
    new = [1, 1, 90, 1]
    b = Batch(np.add([long, 9, 4000, 2500], new), new, 32, 8, hd, seed=18)
    if holes:
        b.table[np.random.RandomState(1).rand(*b.table.shape) < 0.1] = -1
    b.check(window=window, softcap=cap)


@pytest.mark.parametrize("new", [1, 40])
def test_offsets_past_32_bits(new):
    """Pages behind 4 GiB of codes."""
    hkv, hd, n_pages = 16, 128, 140000
    codes, scales = mg.kv4_empty(n_pages, hkv, hd)
    assert codes.numel() > 1 << 32
    rng = np.random.RandomState(12)
    L = 100 + new
    table = np.array([n_pages - 1 - np.arange(10)], np.int32)
    slots = np.array([table[0, p // 16] * 16 + p % 16 for p in range(L)], np.int32)
    k, v, q = (rows(rng, (n, h, hd)) for n, h in ((L, hkv), (L, hkv), (new, 32)))
    mg.kv4_append(codes, scales, k.cuda(), v.cuda(), dev_i32(slots))
    got = mg.kv4_attention(codes, scales, q.cuda(), dev_i32(table), dev_i32([L]), cu_new=dev_i32([0, new]), max_new=new)
    back = mg.kv4_read(codes, scales, dev_i32(slots))
    small = ref.RefCache(10, hkv, hd)
    t2, s2 = np.arange(10, dtype=np.int32)[None], np.arange(L)
    small.append(bf16(k), bf16(v), s2)
    for side, x in enumerate(back):
        np.testing.assert_array_equal(bf16(x), small.val[s2 // 16, :, side, s2 % 16])
    out, bound = ref.attention(small, bf16(q), t2, [L], [0, new], 1 / np.sqrt(hd))
    assert (np.abs(bf16(got) - out) <= bound).all()


def test_same_call_gives_the_same_bits():
    """Many times over: grids of several blocks a compute unit, every kind of block."""
    for new, ctx in (([1, 300, 4, 1], [900, 20, 700, 5000]), ([1] * 48, list(range(2000, 6800, 100))), ([4] * 20, list(range(500, 4500, 200)))):
        b = Batch(np.add(ctx, new), new, 28, 4, 128, seed=13)
        args = (b.codes, b.scales, b.q.cuda(), dev_i32(b.table), dev_i32(b.lens))
        one = mg.kv4_attention(*args, cu_new=dev_i32(b.cu), max_new=max(new))
        for _ in range(10):
            assert torch.equal(one, mg.kv4_attention(*args, cu_new=dev_i32(b.cu), max_new=max(new)))


# ---------------------------------------------------------------- together


class Loop:
    """A serving loop's state: requests whose tokens arrive chunk by chunk, on one set of buffers; a step plans, rotates and appends,
    attends, and takes log probabilities of a head's logits."""

    def __init__(self, B, hq, hkv, hd, maxp, n_pages, most, vocab=999):
        self.codes, self.scales = mg.kv4_empty(n_pages, hkv, hd)
        z = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")  # noqa: E731
        self.most, self.hq, self.hd = most, hq, hd
        self.ctx, self.new, self.table, self.n_free = z(B), z(B), z(B, maxp) - 1, z(1) + n_pages
        self.free = dev_i32(np.random.RandomState(0).permutation(n_pages))
        self.plan = mg.BatchPlan(z(B + 1), z(B), z(B), z(most), z(most), z(most), z(1))
        self.qkv = torch.zeros((most, hq + 2 * hkv, hd), dtype=torch.bfloat16, device="cuda")
        self.qr = torch.zeros((most, hq, hd), dtype=torch.bfloat16, device="cuda")
        self.out = torch.zeros_like(self.qr)
        self.rope = mg.rope_table(16 * maxp, hd, THETA)
        self.ws = torch.empty(max(1, mg.kv4_attention_workspace_bytes(
            self.codes, self.scales, self.qr, self.table, self.plan.lens, cu_new=self.plan.cu_new, max_new=most)),
            dtype=torch.uint8, device="cuda")
        self.head = torch.as_tensor(np.random.RandomState(9).randn(hq * hd, vocab).astype(np.float32)).cuda()
        self.logits = torch.zeros((most, vocab), device="cuda")
        self.tokens = z(most) + 5
        f = lambda *s: torch.zeros(s, device="cuda")  # noqa: E731
        self.lp = mg.TokenLogprobs(f(most), f(most), z(most, 4), f(most, 4))
        self.lws = torch.empty(max(1, mg.token_logprobs_workspace_bytes(most, vocab, 4)), dtype=torch.uint8, device="cuda")

    def step(self):
        hq, hkv = self.hq, self.codes.shape[1]
        mg.batch_plan(self.ctx, self.new, self.free, self.n_free, self.table, self.most, out=self.plan)
        mg.kv4_append(self.codes, self.scales, self.qkv[:, hq:hq + hkv], self.qkv[:, hq + hkv:], self.plan.slots,
                      positions=self.plan.positions, rope=self.rope, q=self.qkv[:, :hq], q_out=self.qr)
        mg.kv4_attention(self.codes, self.scales, self.qr, self.table, self.plan.lens, cu_new=self.plan.cu_new,
                         max_new=self.most, out=self.out, workspace=self.ws)
        torch.mm(self.out.view(self.most, -1).float(), self.head, out=self.logits)
        mg.token_logprobs(self.logits, self.tokens, top=4, out=self.lp, workspace=self.lws)
        self.ctx.copy_(self.plan.lens)
        self.n_free.copy_(self.plan.n_left)


STEPS = [[20, 0, 33], [1, 16, 1], [1, 1, 1], [1, 40, 0], [1, 1, 1], [2, 1, 30]]


def drive(loop, step):
    """The steps of STEPS through `step`, each checked against the definitions."""
    rng = np.random.RandomState(1)
    hkv, hd, hq = loop.codes.shape[1], loop.hd, loop.hq
    want = ref.RefCache(loop.codes.shape[0], hkv, hd)
    table, outs = loop.rope.cpu().numpy(), []
    for new in STEPS:
        n = sum(new)
        loop.qkv.copy_(rows(rng, tuple(loop.qkv.shape)))
        loop.new.copy_(torch.as_tensor(new, dtype=torch.int32))
        step()
        torch.cuda.synchronize()
        slots, pos = (getattr(loop.plan, k).cpu().numpy()[:n] for k in ("slots", "positions"))
        x = bf16(loop.qkv)[:n]
        want.append(ref.rotate(x[:, hq:hq + hkv], table, pos), x[:, hq + hkv:], slots)
        np.testing.assert_array_equal(ref.unpack(loop.codes, loop.scales)[0], want.val)
        cu = np.concatenate([[0], np.cumsum(new)])
        out, bound = ref.attention(want, ref.rotate(x[:, :hq], table, pos), loop.table.cpu().numpy(), loop.ctx.cpu().numpy(), cu,
                                   1 / np.sqrt(hd))
        assert (np.abs(bf16(loop.out)[:n] - out) <= bound).all()
        lp = ref.logprobs(loop.logits[:n].double().cpu().numpy(), [5] * n, 4)
        np.testing.assert_array_equal(loop.lp.top_tokens[:n].cpu().numpy(), lp[2])
        np.testing.assert_allclose(loop.lp.logprob[:n].cpu().numpy(), lp[0], rtol=2.0 ** -20, atol=2.0 ** -18)
        outs += [loop.out[:n].clone(), loop.lp.logprob[:n].clone(), loop.lp.top_logprobs[:n].clone()]
    return outs


def test_plan_append_attend_and_score_over_a_request_s_life():
    loop = Loop(3, 8, 2, 128, 8, 24, 60)
    drive(loop, loop.step)


def test_a_captured_step_follows_its_buffers():
    """One capture replayed over prompts and single tokens, on another stream than the buffers' own."""
    eager = drive(*(lambda l: (l, l.step))(Loop(3, 8, 2, 128, 8, 24, 60)))
    loop = Loop(3, 8, 2, 128, 8, 24, 60)
    loop.step()  # nothing new: warms the library up and changes nothing
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        loop.step()
    for a, b in zip(eager, drive(loop, g.replay)):
        assert torch.equal(a, b)


def test_two_streams_at_once():
    """Two batches on streams of their own, interleaved, with a workspace each."""
    bs = [Batch(np.add([2900, 130, 1700], [1, 1, 1]), [1, 1, 1], 8, 2, 128, seed=s) for s in (20, 21)]
    alone = [b.run() for b in bs]
    args = [(b.q.cuda(), dev_i32(b.table), dev_i32(b.lens)) for b in bs]
    outs = [torch.zeros_like(a) for a in alone]
    ws = [torch.empty(mg.kv4_attention_workspace_bytes(b.codes, b.scales, *a), dtype=torch.uint8, device="cuda")
          for b, a in zip(bs, args)]
    assert ws[0].numel() > 0
    torch.cuda.synchronize()
    st = [torch.cuda.Stream() for _ in bs]
    for _ in range(20):
        for b, (q, t, l), o, w, s in zip(bs, args, outs, ws, st):
            mg.kv4_attention(b.codes, b.scales, q, t, l, out=o, workspace=w, stream=s)
    torch.cuda.synchronize()
    for a, o in zip(alone, outs):
        assert torch.equal(a, o)
