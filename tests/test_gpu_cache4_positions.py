"""Chunks over the 4-bit cache: where their tokens stand, for lengths at the ends
of their range.  Bounds of test_gpu_cache4.py."""
import numpy as np
import pytest

pytest.importorskip("paper_2608_03228_amd.saki")

from tests.cache4_rows import check_rows, chunk_case, picked, run  # noqa: E402
from tests.test_gpu_cache4 import attend_case, check_attend  # noqa: E402

pytestmark = pytest.mark.gpu
LEAST = -(1 << 31)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("width", [None, 400])
def test_lengths_near_the_lowest_int(width, dt):
    """As every other length below zero: no key, rows of zeros."""
    q, cache, tab, lens, cu = chunk_case([100, 30, 200], [40, 70, 5], 4, 2, dt, width)
    case = (q, cache, tab, [LEAST, 100, LEAST + 3], cu)
    got = run(case, dt)
    assert (got[:40] == 0).all() and (got[110:] == 0).all()
    check_rows(case, dt, got, picked([40, 70, 5], 2, 4, np.random.default_rng(0)))


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("width", [None, 400])
def test_lengths_near_the_highest_int(width, dt):
    q, cache, tab, lens, cu = chunk_case([100, 30], [40, 70], 4, 2, dt, width)
    case = (q, cache, tab[:, :1].copy() if width is None else tab, [(1 << 31) - 1, 100], cu)
    check_rows(case, dt, run(case, dt), picked([40, 70], 2, 4, np.random.default_rng(0)))


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("width", [None, 70])
@pytest.mark.parametrize("listed", [False, True])
def test_decode_steps_of_such_lengths(listed, width, dt):
    lens, Q = [LEAST, 70, LEAST + 20, (1 << 31) - 1], 16
    q, cache, tab = attend_case([64, 70, 64, 128], 4, 2, Q, dt, width, stale=False)
    idx = np.broadcast_to(np.array([3, 60, 69, 100]), (4, 4, Q, 4)) if listed else None
    got, _ = check_attend((q, cache, tab), lens, dt, top_idx=idx)
    assert (got[0] == 0).all() and (got[2] == 0).all()
