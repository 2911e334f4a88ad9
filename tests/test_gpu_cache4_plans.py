"""Attention over the 4-bit cache: what is special about single rows (missing
blocks, tokens of no request, lengths below the chunk's, NaN, scores and scales far
apart), in every way that a call's rows and keys are divided.  Bounds of
test_gpu_cache4.py, single rows of a chunk against the oracle."""
import numpy as np
import pytest

pytest.importorskip("paper_2608_03228_amd.saki")

from tests.cache4_rows import check_rows, chunk_case, picked, run, shared  # noqa: E402
from tests.test_gpu_cache4 import attend_case, check_attend, rounded  # noqa: E402

pytestmark = pytest.mark.gpu

# contexts, new tokens, H_q, H_kv, the tables' width; rows of a work-group and shares of their keys
PLANS = [
    ([600], [40], 4, 2, 12, 64, 6),
    ([500, 450], [180, 120], 64, 1, 400, 128, 3),
    ([1100, 1000], [605, 605], 14, 2, 1155, 128, 7),
    ([0, 100, 30], [100, 100, 50], 256, 2, 12, 128, 1),
]


@pytest.fixture(params=[(p, dt) for p in PLANS for dt in ("f32", "bf16")], ids=lambda p: f"{p[0][5]}-{p[0][6]}-{p[1]}")
def chunk(request):
    (ctx, new, H_q, H_kv, width, rows, shares), dt = request.param
    case = chunk_case(ctx, new, H_q, H_kv, dt, width)
    assert shared(case, dt, rows, shares)
    return case, dt, picked(new, H_q // H_kv, H_q, np.random.default_rng(3), 20)


def held(tab, n_blocks):
    return [[j for j in range(len(r)) if 0 <= r[j] < n_blocks] for r in tab]


def test_finite(chunk):
    case, dt, rows = chunk
    got = run(case, dt)
    assert np.isfinite(got).all()
    check_rows(case, dt, got, rows)


def test_missing_blocks_and_tokens_of_no_request(chunk):
    (q, cache, tab, lens, cu), dt, rows = chunk
    for j, what in zip((1, 3, 4), (-1, 1 << 30, -7)):
        tab[0, j] = what
    tab[-1, :2] = -1
    case = q, cache, tab, lens, cu
    check_rows(case, dt, run(case, dt, before=3, after=70), rows)


def test_lengths_below_the_chunks(chunk):
    (q, cache, tab, lens, cu), dt, rows = chunk
    lens = [n // 3 if b == 0 else n for b, n in enumerate(lens)]
    lens[0] = min(lens[0], int(cu[1]) - 5)
    if len(lens) > 1:
        lens[-1] = -3
    got = run((q, cache, tab, lens, cu), dt)
    check_rows((q, cache, tab, lens, cu), dt, got, rows)
    assert (got[:cu[1] - lens[0]] == 0).all() and (len(lens) == 1 or (got[cu[-2]:] == 0).all())


def test_lengths_past_the_tables_room(chunk):
    """The width stays, so that the call is divided as it was."""
    (q, cache, tab, lens, cu), dt, rows = chunk
    width = tab.shape[1]
    case = q, cache, tab, [width * 64 + 700] + lens[1:], cu
    check_rows(case, dt, run(case, dt), rows)


def test_nan_groups(chunk):
    (q, cache, tab, lens, cu), dt, rows = chunk
    new, last = np.diff(cu), len(lens) - 1
    for b, H, back, dims in ((0, 0, new[0] // 2, 2), (0, cache[0].shape[1] - 1, 1, 0), (last, 0, 3, 3)):
        at = lens[b] - int(back) - 1   # a new token's value
        cache[2][tab[b, at // 64], H, 1, at % 64, dims] = 255
    if last > 0:   # a key that all rows of the request see, but the very first ones
        cache[2][tab[1, 0], 0, 0, 5, 1] = 255
    cache[2][tab[0, 0], 0, 1, 40, 1] = 255
    got = run((q, cache, tab, lens, cu), dt)
    want = check_rows((q, cache, tab, lens, cu), dt, got, rows)
    assert np.isnan(want).any()


def test_queries_that_are_not_finite(chunk):
    (q, cache, tab, lens, cu), dt, rows = chunk
    bad = [(0, 1, 7, np.nan), (len(q) // 3, 0, 100, np.inf), (len(q) - 1, q.shape[1] - 1, 64, -np.inf)]
    for t, h, d, x in bad:
        q[t, h, d] = x
    case = q, cache, tab, lens, cu
    got = run(case, dt)
    nan = np.zeros(got.shape[:2], bool)
    for t, h, _, _ in bad:
        nan[t, h] = True
    assert np.isnan(got[nan]).all() and np.isfinite(got[~nan]).all()
    check_rows(case, dt, got, [r for r in rows if not nan[cu[r[0]] + r[1], r[2]]])


@pytest.mark.parametrize("down", [False, True])
def test_scores_that_grow_or_shrink_along_the_row(chunk, down):
    (q, cache, tab, lens, cu), dt, rows = chunk
    for r, js in zip(tab, held(tab, len(cache[0]))):
        for j in js:
            cache[2][r[j], :, 0] = 118 + (len(js) - 1 - j if down else j) * 10 // len(js)
    case = q, cache, tab, lens, cu
    got = run(case, dt)
    assert np.isfinite(got).all()
    check_rows(case, dt, got, rows)


def test_scales_far_apart(chunk):
    """Values of 2^90 and 2^60 in a token, keys of 2^-90 under queries of 2^88."""
    (q, cache, tab, lens, cu), dt, rows = chunk
    cache[2][:, :, 1] = 127 + 90 - np.random.default_rng(1).choice([0, 30], cache[2][:, :, 1].shape)
    cache[2][:, :, 0] = 127 - 90
    case = rounded(q * 2.0 ** 88, dt), cache, tab, lens, cu
    check_rows(case, dt, run(case, dt), rows)


# ---------------------------------------------------------------- decode steps

@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("lens,H_q,H_kv,Q", [
    ([700, 3, 1500, 64, 0, 129] * 2, 16, 8, 1), ([900, 65, 2000, 4] * 4, 28, 4, 2), ([1300, 200] * 4, 16, 8, 9),   # 18 rows
    ([640, 3000] * 16, 8, 8, 1),
])
def test_decode_of_some_pairs_in_wide_tables(lens, H_q, H_kv, Q, dt):
    """64 to 256 pairs of a request and a KV head (16 rows at most), joined by four waves a pair."""
    pairs = len(lens) * H_kv * -(-(H_q // H_kv * Q) // 16)
    assert 64 <= pairs <= 256
    q, cache, tab = attend_case(lens, H_q, H_kv, Q, dt, 100)
    cache[2][tab[2, 0], 0, 1, 9, 2] = 255   # a value that all of the third request's rows see
    check_attend((q, cache, tab), lens, dt)
