"""saki_attend_prompt where tokens hold NaN or infinities: a row is what its own
and the earlier tokens make it.  Rows that see none keep the bound of
test_gpu_prompt.py; of the others, elements that the formula leaves finite do, and
the rest are not finite."""
import numpy as np
import pytest

import oracle as O
from tests.test_gpu_prompt import make
from tests.test_gpu_serve import DT, U, dev, host, ints

torch = pytest.importorskip("torch")
S = pytest.importorskip("paper_2608_03228_amd.saki")

pytestmark = pytest.mark.gpu


def check(q, k, v, cu, dt, heads=1, beyond=()):
    """`heads` copies of the heads say how the rows are divided; rows `beyond`
    float32 (their scores are finite in the oracle alone) are left out."""
    H_q, H_kv = q.shape[1], k.shape[1]
    out = S.saki_attend_prompt(*(dev(np.tile(x, (1, heads, 1)), DT[dt]) for x in (q, k, v)), ints(cu))
    with np.errstate(invalid="ignore", over="ignore"):
        want, mass, size = O.prompt_attend(q, k, v, cu)
    fine = np.isfinite(want)
    here = np.ones(len(q), bool)
    here[list(beyond)] = False
    n = np.diff(cu).max()
    score = (140 * U * size + 4 * U)[..., None]
    b = 2.0 ** -8 if dt == "bf16" else 0
    for h in range(0, heads, max(1, heads - 1)):
        got = host(out[:, h * H_q:(h + 1) * H_q])
        assert not np.isfinite(got[here][~fine[here]]).any()
        with np.errstate(invalid="ignore"):
            bound = (2 * score + (max(n, 64) / 32 + 64) * U + b) * mass + (b + U) * np.abs(want)
            bad = fine & ~(np.abs(got - want) <= bound) & here[:, None, None]
            assert not bad.any(), np.argwhere(bad)[:5]
    return fine


CASES = [(1, 1, 1), (4, 1, 1), (2, 2, 32), (4, 1, 40)]  # H_q, H_kv, copies: halved work-groups, whole ones


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("H_q,H_kv,heads", CASES)
@pytest.mark.parametrize("bad", [np.nan, np.inf, -np.inf])
def test_values(bad, H_q, H_kv, heads, dt):
    """Single elements of values, at and between the borders of tiles."""
    T, cu = 300, np.array([0, 230, 231, 300])
    q, k, v = make(T, H_q, H_kv, dt, 1)
    rng = np.random.default_rng(2)
    for t in (70, 127, 128, 200, 231 + 40, 299):
        v[t, rng.integers(H_kv), rng.integers(128, size=3)] = bad
    fine = check(q, k, v, cu, dt, heads)
    assert fine[:70].all() and fine[70:].any() and not fine[70:].all()


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("H_q,H_kv,heads", CASES)
def test_values_of_both_signs_meet(H_q, H_kv, heads, dt):
    T, cu = 100, np.array([0, 100])
    q, k, v = make(T, H_q, H_kv, dt, 3)
    v[50, 0, 7], v[60, 0, 7], v[60, 0, 8], v[61, 0, 9] = np.inf, -np.inf, np.inf, np.nan
    check(q, k, v, cu, dt, heads)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("H_q,H_kv,heads", CASES)
def test_keys(H_q, H_kv, heads, dt):
    """A key of NaN makes every row that sees it NaN, and no other."""
    T, cu = 300, np.array([0, 230, 300])
    q, k, v = make(T, H_q, H_kv, dt, 4)
    k[190, 0, 3] = np.nan
    k[299, H_kv - 1] = np.nan
    fine = check(q, k, v, cu, dt, heads)
    assert fine[:190].all() and not fine[190:230, 0].any() and fine[230:299].all()


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("H_q,H_kv,heads", CASES)
def test_whole_tokens(H_q, H_kv, heads, dt):
    """Padding behind a prompt's real tokens, within its offsets: queries, keys and
    values of NaN, of infinities, and of the type's largest number."""
    T, cu = 400, np.array([0, 150, 400])
    q, k, v = make(T, H_q, H_kv, dt, 5)
    for x in (q, k, v):
        x[100:150] = np.nan
        x[330:350] = np.inf
        x[350:] = torch.finfo(DT[dt]).max
    fine = check(q, k, v, cu, dt, heads)
    assert fine[:100].all() and not fine[100:150].any() and fine[150:330].all()


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("H_q,H_kv,heads", CASES)
@pytest.mark.parametrize("fill", [3.3e38, -1e30])
def test_padding_of_large_numbers(fill, H_q, H_kv, heads, dt):
    """Finite ones behind the real tokens: rows before them are as without."""
    T, cu = 300, np.array([0, 27, 150, 300])
    q, k, v = make(T, H_q, H_kv, dt, 8)
    padding = [*range(17, 27), *range(100, 150), *range(285, 300)]
    for x in (q, k, v):
        x[padding] = dev(np.array(fill), DT[dt]).double().item()
    fine = check(q, k, v, cu, dt, heads, beyond=padding)
    assert fine[:17].all() and fine[27:100].all() and fine[150:285].all()


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("H_q,H_kv,heads", CASES[:2])
def test_queries(H_q, H_kv, heads, dt):
    T, cu = 100, np.array([0, 100])
    q, k, v = make(T, H_q, H_kv, dt, 6)
    q[40, 0, 5] = np.nan
    fine = check(q, k, v, cu, dt, heads)
    assert fine[np.arange(T) != 40].all() and not fine[40, 0].any()
