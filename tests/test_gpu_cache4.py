"""GPU parity of the 4-bit cache (writing, reading back, attention of decode steps
and of chunks over it) against the float64 oracle.

Tolerances, before any run.  u = 2^-24 (float32 half step), bf16 half step 2^-8.
  write, read  equal: scaling by a power of two is exact, and so are codes times
               scales in bf16
  attention    a score is a sum of up to 384 exact products in float32 and a
               scaling: off by 390 u S, S = the row's largest sum of |q_e k_e| /
               sqrt(d); exponent and its argument 4 u more, and what three terms
               of a float32 query leave 2^-25; softmax turns a score error e into
               2 e of sum p |v|; a sum over N keys in three terms rounds 3 N times
               at most and the weights' sum N times; weights are split into terms
               that leave 2^-17 (decode, bf16 outputs), 2^-25 (float32), or are
               rounded to bf16 (chunks in bf16); then the output's rounding
"""
import numpy as np
import pytest

import oracle as O
from tests.test_gpu_streams import check_pools, made, zeros  # noqa: F401  (made: a fixture)

torch = pytest.importorskip("torch")
S = pytest.importorskip("paper_2608_03228_amd.saki")

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def dev(a, dtype=torch.float32):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEV, dtype)


def ints(a):
    return dev(np.asarray(a, np.int32), torch.int32)


def host(t):
    return t.double().cpu().numpy() if t.is_floating_point() else t.cpu().numpy()


def rounded(a, dt):
    """float64 values that the type holds."""
    return torch.from_numpy(np.asarray(a)).to(DT[dt]).double().numpy()


def random_cache(n_blocks, H, rng):
    """Any codes under scales of 2^-4 .. 2^-1, as host arrays."""
    codes = rng.integers(0, 256, (2, n_blocks, H, 64, 64)).astype(np.uint8)
    return codes[0], codes[1], rng.integers(123, 127, (n_blocks, H, 2, 64, 4)).astype(np.uint8)


def on_gpu(cache):
    return tuple(dev(c, torch.uint8) for c in cache)


def values(cache):
    return [O.cache4_values(cache[w], cache[2], w) for w in range(2)]


# ---------------------------------------------------------------- writing

@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("slots,H", [
    ([0], 1), ([63, 5], 3), (list(range(64)), 2), ([200, -1, 64 * 5 + 63, 7, 1 << 30, 6], 5),
    ([b * 64 + 7 * b % 64 for b in range(37)], 4), ([-1, -5], 1), (list(range(130, 3, -1)), 1),
])
def test_write(slots, H, dt):
    rng = np.random.default_rng(len(slots) + H)
    cache = random_cache(1 + max([s // 64 for s in slots if s < 1 << 20] + [0]), H, rng)
    T = len(slots)
    size = np.exp(3 * rng.standard_normal((T, H, 1)))
    size[rng.random((T, H, 1)) < 0.1] = 0
    x = [rounded(size * rng.standard_normal((T, H, 128)), dt) for _ in range(2)]
    got = on_gpu(cache)
    assert S.saki_cache4_write(dev(x[0], DT[dt]), dev(x[1], DT[dt]), ints(slots), *got)[0] is got[0]
    want_s = cache[2]
    for w in range(2):
        want, want_s = O.cache4_write(x[w], slots, cache[w], want_s, w)
        np.testing.assert_array_equal(host(got[w]), want)
    np.testing.assert_array_equal(host(got[2]), want_s)


def test_write_every_code_tie_and_edge_of_the_scale():
    e = O.E2M1
    vals = np.concatenate([e, (e[1:] + e[:-1]) / 2, e * (1 + 2.0 ** -20), (e[1:] + e[:-1]) / 2 * (1 + 2.0 ** -20),
                           (e[1:] + e[:-1]) / 2 * (1 - 2.0 ** -20), [6.5, 7.0, 0.0]])
    vals = np.concatenate([vals, -vals])
    x = np.zeros((6, 1, 128))
    x[0, 0] = np.resize(vals, 128)
    x[0, 0, ::32] = 7.0  # the scale is one
    x[1, 0] = np.resize(np.roll(vals, 11), 128)
    x[1, 0, 1::32] = -6.0
    x[2] = x[0] * 2.0 ** 119
    x[3] = x[0] * 2.0 ** -99
    x[4, 0] = np.resize([np.nextafter(np.float32(7), np.float32(8)), 1.0, -0.0, 0.0], 128)
    x[5, 0, :32] = 2.0 ** 127           # past the largest scale: saturates
    x[5, 0, 32:64] = 2.0 ** -140        # below the least one
    x[5, 0, 64] = 2.0 ** -100
    cache = random_cache(1, 1, np.random.default_rng(0))
    got = on_gpu(cache)
    S.saki_cache4_write(dev(x), dev(-x), ints(range(6)), *got)
    scales = cache[2]
    for w in range(2):
        want, scales = O.cache4_write(x * (1 - 2 * w), range(6), cache[w], scales, w)
        np.testing.assert_array_equal(host(got[w]), want)
    np.testing.assert_array_equal(host(got[2]), scales)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_write_of_what_is_not_finite_is_nan_in_its_group_alone(dt):
    rng = np.random.default_rng(3)
    x = rounded(rng.standard_normal((5, 2, 128)), dt)
    clean = O.cache4_round(x)
    x[1, 0, 33], x[2, 1, 5], x[3, 0, 127] = np.inf, np.nan, -np.inf
    got = on_gpu(random_cache(1, 2, rng))
    S.saki_cache4_write(dev(x, DT[dt]), dev(x, DT[dt]), ints(range(5)), *got)
    out = torch.empty(5, 2, 128, device=DEV)
    for back in S.saki_cache4_read(*got, ints([[0]]), ints([0, 5]), out, torch.empty_like(out)):
        want = np.where(clean[0] >= 8, -1, 1) * O.E2M1[clean[0] & 7] * np.repeat(2.0 ** (clean[1] - 127.0), 32, -1)
        want[1, 0, 32:64] = want[2, 1, :32] = want[3, 0, 96:] = np.nan
        np.testing.assert_array_equal(host(back), want)


def test_write_out_of_a_fused_projection():
    rng = np.random.default_rng(4)
    H, T = 3, 70
    x = rounded(rng.standard_normal((T, 3 * H, 128)), "bf16")
    t = dev(x, torch.bfloat16)
    cache = random_cache(2, H, rng)
    got, dense = on_gpu(cache), on_gpu(cache)
    slots = ints(rng.permutation(128)[:T])
    S.saki_cache4_write(t[:, H:2 * H], t[:, 2 * H:], slots, *got)
    S.saki_cache4_write(t[:, H:2 * H].contiguous(), t[:, 2 * H:].contiguous(), slots, *dense)
    assert all(torch.equal(a, b) for a, b in zip(got, dense))
    np.testing.assert_array_equal(host(t), x)


# ---------------------------------------------------------------- reading back

@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("cu,starts,H", [
    ([0, 1], [0], 1), ([0, 64, 64, 130], [3, 0, 62], 2), ([2, 5, 5, 21, 40], [200, 7, 0, 190], 3),
    ([0, 0, 0], [0, 0], 1), ([0, 300], None, 5), ([0, 17], [-3], 2), (list(range(0, 202, 2)), [1] * 100, 1),
    ([0] * 70 + [1] + [1] * 70 + [33], [0] * 141, 2),
    (list(range(3, 68)), list(range(64)), 1), (list(range(0, 130, 2)), None, 2), (list(range(66)), [5] * 65, 1),
    ([0] * 63 + [4, 40], [9] * 64, 2),
])
def test_read(cu, starts, H, dt):
    rng = np.random.default_rng(len(cu) + H)
    B = len(cu) - 1
    cache = random_cache(7, H, rng)
    tab = rng.integers(0, 7, (B, 4))
    tab[rng.random((B, 4)) < 0.15] = -1
    tab[0, -1] = 7   # behind the last block
    T = cu[-1] + 5
    k, v = torch.full((2, T, H, 128), -77.0, device=DEV, dtype=DT[dt])
    got = S.saki_cache4_read(*on_gpu(cache), ints(tab), ints(cu), k, v, starts=None if starts is None else ints(starts))
    assert got[0] is k and got[1] is v
    for w in range(2):
        want, mine = O.cache4_rows(values(cache)[w], tab, cu, starts or [0] * B, T)
        want[~mine] = -77
        np.testing.assert_array_equal(host(got[w]), want)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_read_of_more_than_the_caches_hold(dt):
    rng = np.random.default_rng(5)
    H, blocks = 4, 600
    cache = random_cache(blocks, H, rng)
    tab = rng.permutation(blocks).reshape(3, 200)
    cu, starts = np.array([0, 12800, 12800, 12800 + 12000]), [0, 5, 777]
    k, v = torch.zeros((2, cu[-1] + 3, H, 128), device=DEV, dtype=DT[dt])
    assert 2 * k.numel() * k.element_size() >= 32 << 20
    S.saki_cache4_read(*on_gpu(cache), ints(tab), ints(cu), k, v, starts=ints(starts))
    for got, x in zip((k, v), values(cache)):
        want = np.zeros(got.shape)
        want[:12800] = x[tab[0]].transpose(0, 2, 1, 3).reshape(-1, H, 128)
        want[12800:24800] = x[tab[2]].transpose(0, 2, 1, 3).reshape(-1, H, 128)[777:12777]
        np.testing.assert_array_equal(host(got), want)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_read_of_one_side_and_into_a_wider_row(dt):
    rng = np.random.default_rng(1)
    H, T = 2, 100
    cache = random_cache(4, H, rng)
    tab, cu, starts = [[3, 1, 0]], [0, T], [20]
    x = torch.full((T, 2 * H + 1, 128), 5.0, device=DEV, dtype=DT[dt])
    gpu = on_gpu(cache)
    want = [O.cache4_rows(v, tab, cu, starts, T)[0] for v in values(cache)]
    k, v = S.saki_cache4_read(*gpu, ints(tab), ints(cu), x[:, :H], None, starts=ints(starts))
    assert v is None
    np.testing.assert_array_equal(host(x[:, :H]), want[0])
    assert (x[:, H:] == 5).all()
    k, v = S.saki_cache4_read(*gpu, ints(tab), ints(cu), None, x[:, H:2 * H], starts=ints(starts))
    assert k is None
    np.testing.assert_array_equal(host(x[:, H:2 * H]), want[1])
    assert (x[:, 2 * H:] == 5).all()


def test_read_of_a_scale_byte_that_no_write_gives():
    """A cache that others filled: every byte is 2^(e - 127), where float32 holds the product."""
    cache = random_cache(1, 1, np.random.default_rng(2))
    cache[2][0, 0] = np.resize(np.arange(3, 252), (2, 64, 4))
    out = torch.empty(64, 1, 128, device=DEV)
    got = S.saki_cache4_read(*on_gpu(cache), ints([[0]]), ints([0, 64]), out, torch.empty_like(out))
    for w in range(2):
        np.testing.assert_array_equal(host(got[w])[:, 0], values(cache)[w][0, 0])


# ---------------------------------------------------------------- attention of decode steps

def held_tables(lens, rows, n_blocks, rng):
    """Tables of distinct blocks; behind a request's end an entry that names none."""
    ids = rng.permutation(n_blocks)
    tab = np.full((len(lens), rows), n_blocks + 7)
    at = 0
    for b, n in enumerate(lens):
        h = min(-(-max(n, 0) // 64), rows)
        tab[b, :h] = ids[at:at + h]
        at += h
    return tab


def attend_case(lens, H_q, H_kv, Q, dt, rows=None, seed=0, stale=True):
    rng = np.random.default_rng(seed + 17)
    held = [-(-max(n, 0) // 64) for n in lens]
    rows = max(1, max(held)) if rows is None else rows
    n_blocks = sum(held) + 2
    cache = random_cache(n_blocks, H_kv, rng)
    tab = held_tables(lens, rows, n_blocks, rng)
    if stale:  # slots behind a request's last key were never written
        for b, n in enumerate(lens):
            if n > 0 and n % 64 and n // 64 < rows:
                cache[2][tab[b, n // 64], :, :, n % 64:] = rng.choice([255, 254, 0], (H_kv, 2, 64 - n % 64, 4))
    q = rounded(1.5 * rng.standard_normal((len(lens), H_q, Q, 128)), dt)
    return q, cache, tab


def attention_bound(want, mass, size, N, dt, weights):
    score = (390 * U * size + 5 * U)[..., None]
    return (2 * score + (4 * N + 128) * U + (weights if dt == "bf16" else 0)) * mass \
        + (2.0 ** -8 if dt == "bf16" else U) * np.abs(want) + 1e-30


def close(got, want, bound):
    nan = np.isnan(want)
    np.testing.assert_array_equal(np.isnan(got), nan)
    err = np.where(nan, 0, np.abs(got - want) / np.where(nan, 1, bound))
    assert np.all(err <= 1), (np.max(err), np.unravel_index(np.argmax(err), err.shape))


def check_attend(case, lens, dt, top_idx=None, **kw):
    q, cache, tab = case
    out = S.saki_cache4_attend(dev(q, DT[dt]), *on_gpu(cache), ints(tab), ints(lens),
                               top_idx=None if top_idx is None else ints(top_idx), **kw)
    k, v = values(cache)
    want, mass, size = O.cache_attend(q, k, v, np.ones((*k.shape[:2], 2)), tab, lens, top_idx)
    close(host(out), want, attention_bound(want, mass, size, max(max(lens), 64), dt, 2.0 ** -17))
    return out, want


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("lens,H_q,H_kv,Q", [
    ([1], 1, 1, 1), ([63], 4, 1, 1), ([64], 8, 2, 1), ([65], 28, 4, 1), ([0, 5, 0], 4, 2, 1),
    ([0], 2, 1, 3), ([1000], 32, 8, 1), ([300, 1, 640, 129], 12, 1, 4), ([3, 200], 5, 5, 16),
    ([2], 4, 2, 16), ([700, 699], 17, 1, 1), ([-4, 70], 2, 1, 2), ([1500, 300], 4, 1, 1),
])
@pytest.mark.parametrize("rows", [None, 70])  # narrow tables: a work-group per pair; wide ones: shares, joined
def test_attend(rows, lens, H_q, H_kv, Q, dt):
    check_attend(attend_case(lens, H_q, H_kv, Q, dt, rows), lens, dt)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("rows", [15, 70, 130])
def test_attend_many_requests(rows, dt):
    rng = np.random.default_rng(0)
    lens = rng.integers(0, 70, 530).tolist()
    lens[400] = 900
    check_attend(attend_case(lens, 2, 2, 1, dt, rows), lens, dt)


def test_attend_table_entries_out_of_range():
    lens = [500, 300, 400]
    q, cache, tab = attend_case(lens, 4, 2, 1, "f32", stale=False)
    tab[0, 3], tab[0, 7], tab[1, :] = -1, 1 << 30, -5
    check_attend((q, cache, tab), lens, "f32")
    check_attend((q, cache, tab[:, :2].copy()), [1 << 30, 2147483647, 128], "f32")
    idx = np.tile(np.array([0, 200, 450, 2147483647, 499, -3]), (3, 4, 1, 1))
    check_attend((q, cache, tab), lens, "f32", top_idx=idx)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("lens,H_q,H_kv,Q", [
    ([1200, 700, 64], 8, 8, 1), ([500] * 20, 8, 4, 2), ([1100, 3] * 70, 4, 2, 1), ([9000], 3, 1, 1), ([20000, 5], 4, 2, 4),
])
def test_attend_more_shapes(lens, H_q, H_kv, Q, dt):
    """Eight waves to a pair and four, one head's keys in many parts, many pairs joined."""
    check_attend(attend_case(lens, H_q, H_kv, Q, dt), lens, dt)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("rows", [None, 70])
@pytest.mark.parametrize("H_q", [3, 8, 13])   # of one KV head: four, two and one term side by side
def test_attend_queries_that_are_not_finite(H_q, rows, dt):
    """Such a query's row is NaN and the others are what they were."""
    case = attend_case([300, 70], H_q, 1, 1, dt, rows)
    q, cache, tab = case
    clean = host(S.saki_cache4_attend(dev(q, DT[dt]), *on_gpu(cache), ints(tab), ints([300, 70])))
    q = q.copy()
    q[0, 1, 0, 7], q[1, 0, 0, 100], q[1, 2, 0, 31] = np.nan, np.inf, -np.inf
    got = host(S.saki_cache4_attend(dev(q, DT[dt]), *on_gpu(cache), ints(tab), ints([300, 70])))
    for b, h in ((0, 1), (1, 0), (1, 2)):
        assert np.isnan(got[b, h]).all()
        got[b, h] = clean[b, h]
    np.testing.assert_array_equal(got, clean)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("how", ["all", "lists", "chunk"])
def test_attention_over_scales_far_apart(how, dt):
    """Values of 2^90 in one head and 2^-90 in the other, groups of a token 2^30 apart,
    and keys of 2^-90 under queries of 2^88."""
    lens = [150, 40]
    q, cache, tab = attend_case(lens, 4, 2, 1, dt, stale=False)
    rng = np.random.default_rng(1)
    cache[2][:, 0, 1] = 127 + 90 - rng.choice([0, 30], cache[2][:, 0, 1].shape)
    cache[2][:, 1, 1] = 127 - 60 - rng.choice([0, 30], cache[2][:, 1, 1].shape)
    cache[2][:, 1, 0] = 127 - 90
    q[:, 2:] *= 2.0 ** 88
    q = rounded(q, dt)
    idx = np.stack([rng.integers(0, n, (4, 1, 33)) for n in lens]) if how == "lists" else None
    if how != "chunk":
        check_attend((q, cache, tab), lens, dt, top_idx=idx)
    else:
        check_chunk((q[:, :, 0], cache, tab, lens, np.array([0, 1, 2])), dt)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("k", [1, 15, 16, 17, 64])
@pytest.mark.parametrize("H_q,H_kv,Q", [(4, 2, 1), (28, 4, 1), (5, 5, 3), (12, 1, 16)])
def test_attend_lists(H_q, H_kv, Q, k, dt):
    rng = np.random.default_rng(k)
    lens = [500, 3, 0, 129]
    idx = np.stack([rng.integers(-3, max(n, 1) + 20, (H_q, Q, k)) for n in lens])  # some unseen, some twice
    idx[3, 0] = -1
    check_attend(attend_case(lens, H_q, H_kv, Q, dt), lens, dt, top_idx=idx)


@pytest.mark.parametrize("k", [0, 5])
def test_attend_lists_of_no_entry(k):
    case = attend_case([100], 4, 2, 1, "f32")
    out, _ = check_attend(case, [100], "f32", top_idx=np.full((1, 4, 1, k), -1))
    assert (out == 0).all()


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("rows", [None, 70])
@pytest.mark.parametrize("listed", [False, True])
def test_attend_nan_groups_reach_the_rows_that_see_them(listed, rows, dt):
    """A group that is NaN: a key's makes the rows that see it NaN, a value's their
    dims of the group; rows of earlier positions stay as they are."""
    lens, Q = [200, 130, 90], 6
    q, cache, tab = attend_case(lens, 4, 2, Q, dt, rows)
    cache[2][tab[0, 197 // 64], 0, 1, 197 % 64, 2] = 255   # a value that rows 3.. of 6 see
    cache[2][tab[0, 199 // 64], 1, 1, 199 % 64, 0] = 255
    cache[2][tab[1, 128 // 64], 1, 0, 128 % 64, 1] = 255   # a key
    cache[2][tab[2, 0], 0, 1, 10, 3] = 255                 # one that all rows see
    idx = None
    if listed:
        idx = np.tile(np.array([197, 3, 199, 10, 128, 50]), (3, 4, Q, 1))
    _, want = check_attend((q, cache, tab), lens, dt, top_idx=idx)
    assert np.isnan(want).any() and not np.isnan(want[0, 0, :3]).any()


# ---------------------------------------------------------------- attention of chunks

def chunk_case(ctx, new, H_q, H_kv, dt, rows=None, seed=0):
    lens = [a + b for a, b in zip(ctx, new)]
    _, cache, tab = attend_case(lens, H_q, H_kv, 1, dt, rows, seed)
    T = sum(new)
    cu = np.concatenate([[0], np.cumsum(new)])
    q = rounded(1.5 * np.random.default_rng(seed).standard_normal((T, H_q, 128)), dt)
    return q, cache, tab, lens, cu


def check_chunk(case, dt, before=0, after=0, **kw):
    """`before` and `after`: tokens of no request at the ends, whose rows stay as they were."""
    q, cache, tab, lens, cu = case
    full = np.concatenate([np.full((before, *q.shape[1:]), np.nan), q, np.full((after, *q.shape[1:]), np.nan)])
    out = torch.full(full.shape, -77.0, device=DEV, dtype=DT[dt])
    got = S.saki_cache4_prompt(dev(full, DT[dt]), *on_gpu(cache), ints(tab), ints(lens), ints(cu + before), out=out, **kw)
    assert got is out
    got = host(got)
    assert (got[:before] == -77).all() and (got[before + len(q):] == -77).all()
    k, v = values(cache)
    want, mass, size = O.cache4_prompt(q, k, v, tab, lens, cu)
    close(got[before:before + len(q)], want, attention_bound(want, mass, size, max(max(lens), 64), dt, 2.0 ** -8))
    return want


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("ctx,new,H_q,H_kv", [
    ([0], [1], 1, 1), ([0], [65], 4, 1), ([63], [2], 8, 2), ([100, 0, 7], [30, 64, 1], 28, 4), ([5, 5], [0, 40], 4, 2),
    ([300, 1000, 40], [129, 1, 33], 12, 1), ([0], [200], 5, 5), ([500], [70], 17, 1), ([64, 128], [64, 64], 2, 2),
])
@pytest.mark.parametrize("rows", [None, 400])  # wide tables: the keys of a row block are shared
def test_prompt(rows, ctx, new, H_q, H_kv, dt):
    check_chunk(chunk_case(ctx, new, H_q, H_kv, dt, rows), dt)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("rows", [None, 400])
def test_prompt_tokens_of_no_request_and_missing_blocks(rows, dt):
    q, cache, tab, lens, cu = chunk_case([300, 70, 0], [20, 100, 9], 4, 2, dt, rows)
    check_chunk((q, cache, tab, lens, cu), dt, before=3, after=50)
    tab[0, 2], tab[0, 4], tab[1, :2] = -1, 1 << 30, -5
    check_chunk((q, cache, tab, lens, cu), dt)
    # lengths below the chunk's: the first tokens stand before the request's start and see nothing
    want = check_chunk((q, cache, tab, [10, 170, -4], cu), dt)
    assert (want[:10] == 0).all() and (want[120:] == 0).all()
    # past the table's room
    check_chunk((q, cache, tab[:, :2].copy(), [1000, 170, 9], cu), dt)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("ctx,new,H_q,H_kv", [
    ([100] * 4, [4000, 3999, 4001, 3500], 4, 1), ([0], [2100], 8, 8), ([1000, 30], [700, 650], 32, 8),
])
def test_prompt_of_many_rows(ctx, new, H_q, H_kv, dt):
    """Whole blocks of 128 rows, shared and not; every 89th token and the requests' ends against the oracle."""
    q, cache, tab, lens, cu = chunk_case(ctx, new, H_q, H_kv, dt)
    got = host(S.saki_cache4_prompt(dev(q, DT[dt]), *on_gpu(cache), ints(tab), ints(lens), ints(cu)))
    assert np.isfinite(got).all()
    k, v = values(cache)
    for b, n in enumerate(new):
        for i in sorted({*range(b, n, 89), 0, 31, 32, 127, 128, n - 1}):
            t = cu[b] + i
            want, mass, size = O.cache4_prompt(q[t:t + 1], k, v, tab[b:b + 1], [lens[b] - n + i + 1], [0, 1])
            close(got[t:t + 1], want, attention_bound(want, mass, size, lens[b], dt, 2.0 ** -8))


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("rows", [None, 400])
def test_prompt_queries_that_are_not_finite(rows, dt):
    q, cache, tab, lens, cu = chunk_case([200], [50], 4, 2, dt, rows)
    args = *on_gpu(cache), ints(tab), ints(lens), ints(cu)
    clean = host(S.saki_cache4_prompt(dev(q, DT[dt]), *args))
    q = q.copy()
    q[3, 1, 7], q[20, 0, 100], q[49, 3, 64] = np.nan, np.inf, -np.inf
    got = host(S.saki_cache4_prompt(dev(q, DT[dt]), *args))
    for t, h in ((3, 1), (20, 0), (49, 3)):
        assert np.isnan(got[t, h]).all()
        got[t, h] = clean[t, h]
    np.testing.assert_array_equal(got, clean)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_prompt_many_requests(dt):
    rng = np.random.default_rng(1)
    new = rng.integers(0, 6, 300).tolist()
    check_chunk(chunk_case(rng.integers(0, 60, 300).tolist(), new, 4, 2, dt), dt)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("rows", [None, 400])
def test_prompt_nan_groups_reach_the_rows_that_see_them(rows, dt):
    q, cache, tab, lens, cu = chunk_case([100, 10], [90, 80], 4, 2, dt, rows)
    cache[2][tab[0, 150 // 64], 0, 1, 150 % 64, 2] = 255   # values of new tokens
    cache[2][tab[0, 189 // 64], 1, 1, 189 % 64, 0] = 255
    cache[2][tab[1, 60 // 64], 1, 0, 60 % 64, 1] = 255     # a key
    cache[2][tab[1, 0], 0, 1, 5, 3] = 255                  # a value that all rows see
    want = check_chunk((q, cache, tab, lens, cu), dt)
    assert np.isnan(want).any() and not np.isnan(want[:50, :2]).any()


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_prompt_of_scores_that_grow_along_the_row(dt):
    """The running maximum moves in every block, and far below it keys still count as zero or little."""
    q, cache, tab, lens, cu = chunk_case([400], [40], 2, 1, dt)
    cache[2][tab[0, :], :, 0] = 118 + np.arange(tab.shape[1])[:, None, None, None]
    check_chunk((q, cache, tab, lens, cu), dt)
    cache[2][tab[0, :], :, 0] = 126 - np.arange(tab.shape[1])[:, None, None, None]
    check_chunk((q, cache, tab, lens, cu), dt)


def test_prompt_of_one_token_each_is_a_decode_step():
    lens = [700, 64, 129]
    q, cache, tab = attend_case(lens, 8, 2, 1, "f32")
    gpu = on_gpu(cache)
    a = S.saki_cache4_attend(dev(q), *gpu, ints(tab), ints(lens))
    b = S.saki_cache4_prompt(dev(q[:, :, 0]), *gpu, ints(tab), ints(lens), ints([0, 1, 2, 3]))
    k, v = values(cache)
    want, mass, size = O.cache_attend(q, k, v, np.ones((*k.shape[:2], 2)), tab, lens)
    bound = attention_bound(want, mass, size, 700, "f32", 0)
    assert np.all(np.abs(host(a)[:, :, 0] - host(b)) <= 2 * bound[:, :, 0])


def test_prompt_queries_out_of_a_fused_projection():
    q, cache, tab, lens, cu = chunk_case([90], [50], 4, 2, "bf16")
    x = torch.zeros(50, 8, 128, device=DEV, dtype=torch.bfloat16)
    x[:, 2:6] = dev(q, torch.bfloat16)
    gpu = on_gpu(cache)
    a = S.saki_cache4_prompt(x[:, 2:6], *gpu, ints(tab), ints(lens), ints(cu))
    assert torch.equal(a, S.saki_cache4_prompt(dev(q, torch.bfloat16), *gpu, ints(tab), ints(lens), ints(cu)))


# ---------------------------------------------------------------- together

@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_a_conversation(dt):
    """Two prompts, a follow-up chunk, a decode step over every key and over lists:
    tables, rotation, write, attention and reading back, as a server calls them."""
    rng = np.random.default_rng(8)
    H_q, H_kv, B, n_blocks, rows = 8, 2, 2, 12, 6
    cache = on_gpu(random_cache(n_blocks, H_kv, rng))
    cache[2].fill_(255)  # memory as it comes
    free, tab = ints(rng.permutation(n_blocks)), ints(np.full((B, rows), -1))
    ctx, taken = np.zeros(B, np.int64), 0
    have = [[np.zeros((0, H_kv, 128))] * 2 for _ in range(B)]
    for new in ([100, 33], [7, 60], [1, 1]):
        T = sum(new)
        slots, pos = ints([0] * T), ints([0] * T)
        _, _, _, cu, lens, counts = S.saki_block_tables(ints(ctx), ints(new), free[taken:], tab, slots, pos)
        taken += int(counts[0])
        x = dev(rounded(rng.standard_normal((T, H_q + 2 * H_kv, 128)), dt), DT[dt])
        q, k = S.saki_rope(x[:, :H_q], x[:, H_q:H_q + H_kv], pos)
        v = x[:, H_q + H_kv:]
        S.saki_cache4_write(k, v, slots, *cache)
        back = torch.empty(2, T, H_kv, 128, device=DEV, dtype=torch.bfloat16)
        S.saki_cache4_read(*cache, tab, cu, back[0], back[1], starts=ints(ctx))
        for got, given in zip(host(back), (k, v)):
            codes, e = O.cache4_round(host(given))
            want = np.where(codes >= 8, -1, 1) * O.E2M1[codes & 7] * np.repeat(2.0 ** (e - 127.0), 32, -1)
            np.testing.assert_array_equal(got, want)
        at = host(cu)
        for b in range(B):
            have[b] = [np.concatenate([h, host(n)[at[b]:at[b + 1]]]) for h, n in zip(have[b], back)]
        ctx = ctx + np.array(new)
        out = host(S.saki_cache4_prompt(q, *cache, tab, lens, cu))
        for b in range(B):
            n = int(ctx[b])
            full = np.zeros((n, H_q, 128))
            full[n - new[b]:] = host(q)[at[b]:at[b + 1]]
            want, mass, size = (o[n - new[b]:] for o in O.prompt_attend(full, *have[b], [0, n]))
            close(out[at[b]:at[b + 1]], want, attention_bound(want, mass, size, 200, dt, 2.0 ** -8))
        if new == [1, 1]:
            q1 = q.view(B, H_q, 1, 128)
            idx = np.stack([rng.permutation(int(n))[:16] for n in ctx])[:, None, None].repeat(H_q, 1)
            for lists in (None, idx):
                got = host(S.saki_cache4_attend(q1, *cache, tab, lens, top_idx=None if lists is None else ints(lists)))
                blocks = np.zeros((2, B * rows, H_kv, 64, 128))
                for b in range(B):
                    for w in range(2):
                        for j, r in enumerate(have[b][w]):
                            blocks[w, b * rows + j // 64, :, j % 64] = r
                want, mass, size = O.cache_attend(host(q1), *blocks, np.ones((B * rows, H_kv, 2)),
                                                  np.arange(B * rows).reshape(B, rows), ctx, lists)
                close(got, want, attention_bound(want, mass, size, 200, dt, 2.0 ** -17))


def test_index_over_what_the_cache_holds():
    """Contexts read back, indexed and searched; the lists name the exact search's
    best keys of the 4-bit values, and the attention over them is the oracle's."""
    rng = np.random.default_rng(9)
    H_q, H_kv, N, r = 4, 2, 400, 32
    cache = random_cache(7, H_kv, rng)
    tab = rng.permutation(7)[None]
    gpu = on_gpu(cache)
    k = torch.empty(N, H_kv, 128, device=DEV)
    S.saki_cache4_read(*gpu, ints(tab), ints([0, N]), k, None)
    keys = k.transpose(0, 1).contiguous()[None]
    q = dev(rng.standard_normal((1, H_q, 1, 128)))
    cal = S.saki_calibrate(rng.standard_normal((H_q, 256, 128)), host(k)[:256].transpose(1, 0, 2), r)
    B_q, B_k, mu = (dev(cal[n]) for n in ("B_q", "B_k", "mu"))
    index = S.saki_build_index(keys, B_k, mu, r, "f32", H_q)
    idx, _ = S.saki_score_topk(index, "f32", q, B_q, mu, H_kv, N, N, r)
    out = S.saki_cache4_attend(q, *gpu, ints(tab), ints([N]), top_idx=idx)
    kv = values(cache)
    want, mass, size = O.cache_attend(host(q), *kv, np.ones((7, H_kv, 2)), tab, [N], host(idx))
    close(host(out), want, attention_bound(want, mass, size, 64, "f32", 0))


def test_captured_steps_replay():
    """A step captured in a graph and replayed over new inputs, eager work between."""
    rng = np.random.default_rng(10)
    B, H_q, H_kv, rows = 3, 8, 2, 40
    n_blocks = B * rows
    cache = on_gpu(random_cache(n_blocks, H_kv, rng))
    other = tuple(c.clone() for c in cache)
    tab = ints(rng.permutation(n_blocks).reshape(B, rows))
    lens, cu = ints([1500, 64, 2560]), ints([0, 1, 2, 3])
    at = lens.long() - 1
    slots = (tab[torch.arange(B, device=DEV), at // 64] * 64 + at % 64).to(torch.int32)
    x = dev(rng.standard_normal((B, H_q + 2 * H_kv, 128)), torch.bfloat16)

    def step(c):
        S.saki_cache4_write(x[:, H_q:H_q + H_kv], x[:, H_q + H_kv:], slots, *c)
        a = S.saki_cache4_attend(x[:, :H_q, None].contiguous(), *c, tab, lens)
        b = S.saki_cache4_prompt(x[:, :H_q], *c, tab, lens, cu)
        out = torch.empty(B, H_kv, 128, device=DEV, dtype=torch.bfloat16)
        k, v = S.saki_cache4_read(*c, tab, cu, out, torch.empty_like(out), starts=lens - 1)
        return a, b, k, v

    step(cache)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(cache)
    for i in range(4):
        x.copy_(dev(rng.standard_normal(x.shape), torch.bfloat16))
        graph.replay()
        torch.cuda.synchronize()
        for g, w in zip(got, step(other)):
            assert torch.equal(g, w)
        torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(cache, other))


def test_calls_on_a_stream_of_the_callers():
    case = attend_case([3000, 70], 8, 2, 1, "bf16", 50)
    q, cache, tab = case
    gpu, lens = on_gpu(cache), ints([3000, 70])
    args = dev(q, torch.bfloat16), *gpu, ints(tab), lens
    chunk = args[0][:, :, 0].contiguous(), *gpu, args[4], lens, ints([0, 1, 2])
    want = S.saki_cache4_attend(*args), S.saki_cache4_prompt(*chunk)
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    got = S.saki_cache4_attend(*args, stream=stream), S.saki_cache4_prompt(*chunk, stream=stream)
    torch.cuda.synchronize()
    assert all(torch.equal(g, w) for g, w in zip(got, want))


@pytest.mark.parametrize("name", ["attend", "prompt"])
def test_new_tensors_come_from_the_streams_memory(made, name):
    """An output and a workspace (wide tables)."""
    u8, i32 = dict(dtype=torch.uint8), dict(dtype=torch.int32)
    cache = zeros(2, 2, 64, 64, **u8), zeros(2, 2, 64, 64, **u8), zeros(2, 2, 2, 64, 4, **u8)
    tab, lens, cu = zeros(1, 100, **i32), zeros(1, **i32) + 70, torch.tensor([0, 9], device=DEV, **i32)
    if name == "attend":
        check_pools(made, lambda s: S.saki_cache4_attend(zeros(1, 4, 1, 128), *cache, tab, lens, stream=s), 2)
    else:
        check_pools(made, lambda s: S.saki_cache4_prompt(zeros(9, 4, 128), *cache, tab, lens, cu, stream=s), 2)


def test_a_cache_of_no_block():
    u8 = dict(dtype=torch.uint8, device=DEV)
    cache = torch.empty(0, 2, 64, 64, **u8), torch.empty(0, 2, 64, 64, **u8), torch.empty(0, 2, 2, 64, 4, **u8)
    x, tab, lens, cu = torch.ones(3, 2, 128, device=DEV), ints([[0, 5]]), ints([100]), ints([0, 3])
    S.saki_cache4_write(x, x, ints([0, 1, 2]), *cache)
    k, v = S.saki_cache4_read(*cache, tab, cu, x.clone(), x.clone())
    assert (k == 0).all() and (v == 0).all()
    q = torch.ones(1, 4, 1, 128, device=DEV)
    assert (S.saki_cache4_attend(q, *cache, tab, lens) == 0).all()
    assert (S.saki_cache4_attend(q, *cache, tab, lens, top_idx=ints(np.zeros((1, 4, 1, 2)))) == 0).all()
    assert (S.saki_cache4_attend(q, *cache, ints(np.zeros((1, 100))), lens) == 0).all()
    for t in (tab, ints(np.zeros((1, 400)))):
        assert (S.saki_cache4_prompt(torch.ones(3, 4, 128, device=DEV), *cache, t, lens, cu) == 0).all()


def test_offsets_past_32_bits():
    """Blocks beyond 2^32 bytes of codes, and beyond 2^31 of scales."""
    H, n_blocks = 8, 530000   # 17.4 GB a side and 2.2 GB of scales
    k, v = (torch.empty(n_blocks, H, 64, 64, dtype=torch.uint8, device=DEV) for _ in range(2))
    s = torch.empty(n_blocks, H, 2, 64, 4, dtype=torch.uint8, device=DEV)
    rng = np.random.default_rng(11)
    x = rounded(rng.standard_normal((2, 130, H, 128)), "bf16")
    ids = [n_blocks - 1, 131073, n_blocks - 7]
    assert ids[2] * H * 512 > 1 << 31
    slots = [64 * ids[t // 64] + t % 64 for t in range(130)]
    S.saki_cache4_write(dev(x[0], torch.bfloat16), dev(x[1], torch.bfloat16), ints(slots), k, v, s)
    out = torch.empty(2, 130, H, 128, device=DEV)
    S.saki_cache4_read(k, v, s, ints([ids]), ints([0, 130]), out[0], out[1])
    codes, e = O.cache4_round(x)
    vals = np.where(codes >= 8, -1, 1) * O.E2M1[codes & 7] * np.repeat(2.0 ** (e - 127.0), 32, -1)
    np.testing.assert_array_equal(host(out), vals)
    blocks = np.zeros((2, 3, H, 64, 128))
    for t in range(130):
        blocks[:, t // 64, :, t % 64] = vals[:, t]
    q = rounded(rng.standard_normal((1, H, 1, 128)), "f32")
    want, mass, size = O.cache_attend(q, *blocks, np.ones((3, H, 2)), [[0, 1, 2]], [130])
    bound = attention_bound(want, mass, size, 130, "f32", 0)
    tab, lens = ints([ids]), ints([130])
    lists = ints(np.arange(130)[None, None, None].repeat(H, 1)[..., :64])
    close(host(S.saki_cache4_attend(dev(q), k, v, s, tab, lens)), want, bound)
    close(host(S.saki_cache4_prompt(dev(q[:, :, 0]), k, v, s, tab, lens, ints([0, 1]))), want[:, :, 0], bound[:, :, 0])
    want, mass, size = O.cache_attend(q, *blocks, np.ones((3, H, 2)), [[0, 1, 2]], [130], host(lists))
    close(host(S.saki_cache4_attend(dev(q), k, v, s, tab, lens, top_idx=lists)), want,
          attention_bound(want, mass, size, 64, "f32", 0))


def test_refusals_of_tensors():
    q, cache, tab = attend_case([70], 4, 2, 1, "f32")
    gpu = on_gpu(cache)
    tab, lens, cu, q = ints(tab), ints([70]), ints([0, 1]), dev(q)
    x = torch.zeros(3, 2, 128, device=DEV)
    with pytest.raises(ValueError, match="scales must have shape"):
        S.saki_cache4_attend(q, gpu[0], gpu[1], gpu[2][:, :, :1], tab, lens)
    with pytest.raises(ValueError, match="v_cache must have shape"):
        S.saki_cache4_write(x, x, ints([0, 1, 2]), gpu[0], gpu[1][:1], gpu[2])
    with pytest.raises(ValueError, match="k_cache has dtype"):
        S.saki_cache4_write(x, x, ints([0, 1, 2]), gpu[0].to(torch.int8), gpu[1], gpu[2])
    with pytest.raises(ValueError, match="k_cache must be"):
        S.saki_cache4_write(x, x, ints([0, 1, 2]), gpu[0][:, :, :32], gpu[1], gpu[2])
    with pytest.raises(ValueError, match="slots has dtype"):
        S.saki_cache4_write(x, x, torch.zeros(3, dtype=torch.int64, device=DEV), *gpu)
    with pytest.raises(ValueError, match="v must have shape"):
        S.saki_cache4_write(x, x[:2], ints([0, 1, 2]), *gpu)
    with pytest.raises(ValueError, match="k_out must be contiguous"):
        S.saki_cache4_read(*gpu, tab, cu, x.transpose(0, 1).contiguous().transpose(0, 1), None)
    with pytest.raises(ValueError, match="k_out must have shape"):
        S.saki_cache4_read(*gpu, tab, cu, torch.zeros(3, 4, 128, device=DEV), None)
    with pytest.raises(ValueError, match="float32 or bfloat16"):
        S.saki_cache4_read(*gpu, tab, cu, x.half(), None)
    with pytest.raises(ValueError, match="starts must have shape"):
        S.saki_cache4_read(*gpu, tab, cu, x, x.clone(), starts=ints([0, 0]))
    with pytest.raises(ValueError, match="tables must have shape"):
        S.saki_cache4_prompt(q[:, :, 0], *gpu, torch.cat([tab, tab]), lens, cu)
    with pytest.raises(ValueError, match="out has dtype"):
        S.saki_cache4_prompt(q[:, :, 0], *gpu, tab, lens, cu, out=q[:, :, 0].bfloat16())
    with pytest.raises(S.SakiError, match="status -3"):
        S.saki_cache4_attend(q, *gpu, torch.zeros(1, 100, dtype=torch.int32, device=DEV), lens,
                             ws=torch.zeros(64, dtype=torch.uint8, device=DEV))
