"""saki_attend_prompt of float32 where a row is made of small weights, or stands
beside values of another size: attention sinks, unattended keys of huge values,
scores that rise while values shrink.

Scores are products of one element with a power of two, exact in the kernel's
parts, so that what remains is what happens to weights and values.  u = 2^-24:
  scores   the scaling's constant and product and the exponent's argument:
           4 u max |s| + 4 u; softmax turns an error e into 2 e of sum p |v|
  sums     (T / 32 + 64) u of sum p |v|, and parts that leave 2^-21 of a product
  parts    a weight's step: 2^-31 of the row's largest p max |v| for each key;
           an element's: 2^-35 of its token's largest
"""
import numpy as np
import pytest

import oracle as O
from tests.test_gpu_serve import U, dev, host, ints, rounded

torch = pytest.importorskip("torch")
S = pytest.importorskip("paper_2608_03228_amd.saki")

pytestmark = pytest.mark.gpu


def check(s, v, heads):
    """s [T] the keys' scores (the same for every query), v [T, 128]; `heads`
    equal heads, which say how the rows are divided among work-groups."""
    T = len(s)
    k = np.zeros((T, 1, 128))
    k[:, 0, 0] = np.float32(s * np.sqrt(128))
    k[:, 0, 0] = np.round(k[:, 0, 0] * 2.0 ** 12) / 2.0 ** 12  # 22 bits of scores up to 2^9
    q = np.zeros((T, 1, 128))
    q[:, 0, 0] = 1.0
    v = rounded(v, "f32")[:, None]
    out = S.saki_attend_prompt(*(dev(np.repeat(x, heads, 1)) for x in (q, k, v)), ints([0, T]))
    assert all(torch.equal(out[:, :1], out[:, h:h + 1]) for h in range(heads))
    want, mass, _ = O.prompt_attend(q, k, v, [0, T])
    s = k[:, 0, 0] / np.sqrt(128)
    top = np.abs(v[:, 0]).max(1)
    bound = np.zeros((T, 128))
    for i in range(T):
        p = np.exp(s[:i + 1] - s[:i + 1].max())
        p /= p.sum()
        score = 4 * U * np.abs(s[:i + 1]).max() + 4 * U
        bound[i] = (2 * score + (T / 32 + 64) * U + 2.0 ** -21) * mass[i, 0] + U * np.abs(want[i, 0]) \
            + (i + 1) * 2.0 ** -31 * (p * top[:i + 1]).max() + 2.0 ** -35 * (p * top[:i + 1]).sum()
    err = np.abs(host(out[:, 0]) - want[:, 0])
    assert np.all(err <= bound), (np.max(err / np.maximum(bound, 1e-300)), np.argmax((err - bound).max(1)))


HEADS = [1, 64]  # halved work-groups, whole ones (of 1,024 tokens)
LOG2 = np.log(2.0)


@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("sink", [0.0, 1e-6, 1e-2])
@pytest.mark.parametrize("below", [18, 22, 26, 40, 90])
def test_rows_behind_a_sink(below, sink, heads):
    """The first key takes the weight, and its value is small or zero."""
    rng = np.random.default_rng(below)
    s = rng.standard_normal(1024) - below * LOG2
    s[0] = 0
    v = 1 + rng.standard_normal((1024, 128))
    v[0] *= sink
    check(s, v, heads)


@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("where", ["tile before", "key before", "key beside", "key behind"])
@pytest.mark.parametrize("power", [10, 17, 28, 60, 100, 122])
def test_rows_beside_values_of_another_size(power, where, heads):
    """Keys without weight (2^-78 and less), or not seen, whose values are larger
    by many powers of two."""
    rng = np.random.default_rng(power)
    s, v = rng.standard_normal(1024), rng.standard_normal((1024, 128))
    at = {"tile before": slice(0, 32), "key before": slice(5, 6), "key beside": slice(500, 501),
          "key behind": slice(1023, 1024)}[where]
    s[at] -= (78 + power) * LOG2
    v[at] *= 2.0 ** power
    check(s, v, heads)


@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("growth", [1, -1])
def test_scores_and_values_that_move_against_each_other(growth, sign, heads):
    rng = np.random.default_rng(5)
    at = np.linspace(-50, 50, 1024)
    check(sign * at * LOG2, rng.standard_normal((1024, 128)) * 2.0 ** (growth * at)[:, None], heads)


@pytest.mark.parametrize("heads", HEADS)
def test_sizes_that_differ_from_key_to_key(heads):
    """Values and scores of any size within each tile, zeros among them."""
    rng = np.random.default_rng(6)
    v = rng.standard_normal((1024, 128)) * 2.0 ** rng.integers(-40, 40, (1024, 1))
    v[rng.random(1024) < 0.1] = 0
    check(rng.uniform(-30, 30, 1024), v, heads)


@pytest.mark.parametrize("heads", HEADS)
def test_a_later_key_of_another_size_changes_no_row(heads):
    """A key that is not seen yet: rows before it are what they are without it, to
    the bound of their own."""
    rng = np.random.default_rng(7)
    s, v = rng.standard_normal(1024), rng.standard_normal((1024, 128))
    s[100::97] = -200.0
    v[100::97] *= 2.0 ** 90
    check(s, v, heads)
    v[100::97] *= 2.0 ** 32
    check(s, v, heads)
