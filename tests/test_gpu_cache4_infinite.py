"""Attention over the 4-bit cache with queries that are infinite, over keys whose
elements there have one sign: by the formula the row is NaN (all its scores are
the same infinity), not a row without a key.  The others keep the bounds of
test_gpu_cache4.py."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
S = pytest.importorskip("paper_2608_03228_amd.saki")

import oracle as O  # noqa: E402
from tests.cache4_rows import check_rows, chunk_case, picked, run  # noqa: E402
from tests.test_gpu_cache4 import (  # noqa: E402
    DT, attend_case, attention_bound, close, dev, host, ints, on_gpu, values)

pytestmark = pytest.mark.gpu


def of_one_sign(cache):
    """Dim 7 of every key is its scale."""
    cache[0][..., 3] = cache[0][..., 3] & 15 | 0x20
    return cache


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("listed", [False, True])
@pytest.mark.parametrize("width", [None, 70])
@pytest.mark.parametrize("H_q", [3, 8, 13])
def test_attend(H_q, width, listed, sign, dt):
    lens = [300, 1, 0]
    q, cache, tab = attend_case(lens, H_q, 1, 1, dt, width)
    args = *on_gpu(of_one_sign(cache)), ints(tab), ints(lens)
    idx = np.broadcast_to(np.array([0, 5, 299]), (3, H_q, 1, 3)) if listed else None
    k, v = values(cache)
    want, mass, size = O.cache_attend(q, k, v, np.ones((*k.shape[:2], 2)), tab, lens, idx)
    q[0, 1, 0, 7] = q[1, 2, 0, 7] = q[2, 0, 0, 7] = sign * np.inf
    got = host(S.saki_cache4_attend(dev(q, DT[dt]), *args, top_idx=ints(idx) if listed else None))
    assert (got[2] == 0).all()   # no key
    for b, h in ((0, 1), (1, 2)):
        assert np.isnan(got[b, h]).all()
        got[b, h] = want[b, h]
    close(got, want, attention_bound(want, mass, size, 300, dt, 2.0 ** -17))


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("ctx,new,H_q,H_kv,width", [
    ([200, 0], [50, 1], 4, 2, None), ([200, 0], [50, 1], 4, 2, 400),                   # 64 rows a work-group
    ([0, 100, 30], [100, 100, 50], 256, 2, 12), ([500, 0], [180, 120], 64, 1, 400),    # 128
])
def test_prompt(ctx, new, H_q, H_kv, width, sign, dt):
    case = chunk_case(ctx, new, H_q, H_kv, dt, width)
    of_one_sign(case[1])
    bad = [(0, 0), (0, H_q - 1), (new[0] - 1, 1), (new[0], 2), (len(case[0]) - 1, H_q // 2)]
    for i, (t, h) in enumerate(bad):
        case[0][t, h, 7] = sign * np.inf if i % 2 == 0 else -np.inf
    got = run(case, dt)
    for t, h in set(bad):
        assert np.isnan(got[t, h]).all()
        got[t, h] = 0
    assert np.isfinite(got).all()
    rows = [r for r in picked(new, H_q // H_kv, H_q, np.random.default_rng(0)) if (case[4][r[0]] + r[1], r[2]) not in bad]
    check_rows(case, dt, got, rows)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_prompt_rows_without_a_key(dt):
    case = chunk_case([0], [9], 4, 2, dt)
    case[0][:4, 1, 7] = -np.inf
    assert (run((*case[:3], [5], case[4]), dt)[:4] == 0).all()
