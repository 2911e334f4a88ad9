"""CPU pins of the 4-bit cache's oracle: closed forms, bounds and round trips."""
import numpy as np
import pytest

import oracle as O


@pytest.mark.parametrize("top,e", [(7.0, 0), (np.nextafter(7.0, 8), 1), (3.5, -1), (0.0, -100), (7 * 2.0 ** -100, -100),
                                   (7 * 2.0 ** 120, 120), (2.0 ** 127, 120), (1.0, -2), (8.0, 1)])
def test_scale_is_the_least_power_of_two(top, e):
    assert O.cache4_scale(top) == e


def test_round_by_hand_ties_to_the_even_code_and_the_sign_of_zero():
    x = np.zeros(128)
    x[:20] = [7, 6, 5, 4.9, 3.5, 2.5, 2.6, 1.75, 1.25, 0.75, 0.25, 0.26, -0.25, -0.75, -7, -2.5, 0.0, -0.0, 0.5, 1.5]
    codes, e = O.cache4_round(x)
    assert codes[:20].tolist() == [7, 7, 6, 6, 6, 4, 5, 4, 2, 2, 0, 1, 8, 10, 15, 12, 0, 8, 1, 3]
    assert e.tolist() == [127, 27, 27, 27]


def test_round_is_within_half_a_step_of_the_group():
    rng = np.random.default_rng(0)
    x = np.exp(3 * rng.standard_normal((50, 1))) * rng.standard_normal((50, 128))
    codes, e = O.cache4_round(x)
    s = np.repeat(2.0 ** (e - 127.0), 32, -1)
    y = np.where(codes >= 8, -1, 1) * O.E2M1[codes & 7] * s
    # a quarter of the element, or of the scale below it (values under one step apart by half a scale)
    assert np.all(np.abs(x - y) <= np.maximum(np.abs(x) / 4, s / 4))
    top = np.abs(x).reshape(50, 4, 32).max(-1)
    assert np.all(top <= 7 * 2.0 ** (e - 127.0)) and np.all(top > 3.5 * 2.0 ** (e - 127.0))


def test_bytes_are_a_permutation_and_values_come_back():
    for w in range(2):
        seen = {O.cache4_byte(w, t, d) for t in range(64) for d in range(128)}
        assert len(seen) == 64 * 128 and max(b for b, _ in seen) == 4095
    # the values' order by an index expression: [token / 4][dim / 8][token % 4][4 bytes]
    order = np.arange(4096).reshape(16, 16, 4, 4).transpose(0, 2, 1, 3).reshape(64, 64)
    assert all(O.cache4_byte(1, t, d)[0] == order[t, d // 2] for t in range(64) for d in range(128))
    rng = np.random.default_rng(1)
    x = rng.standard_normal((3, 2, 128))
    x[1, 1, 40] = np.inf
    cache, scales = np.full((2, 2, 64, 64), 99, np.uint8), np.full((2, 2, 2, 64, 4), 88, np.uint8)
    for w in range(2):
        c, s = O.cache4_write(x, [5, 64 + 63, -1], cache, scales, w)
        v = O.cache4_values(c, s, w)
        codes, e = O.cache4_round(x)
        want = np.where(codes >= 8, -1, 1) * O.E2M1[codes & 7] * np.repeat(2.0 ** (e - 127.0), 32, -1)
        want[1, 1, 32:64] = np.nan
        np.testing.assert_array_equal(v[0, :, 5], want[0])
        np.testing.assert_array_equal(v[1, :, 63], want[1])
        assert (s[:, :, 1 - w] == 88).all() and (c != 99).sum() <= 256


def test_rows_by_hand():
    v = np.arange(3 * 64, dtype=float).reshape(3, 1, 64, 1) * np.ones(128)
    out, mine = O.cache4_rows(v, [[2, 0], [1, -1]], [1, 4, 6], [62, 63], 8)
    assert out[:, 0, 0].tolist() == [0, 2 * 64 + 62, 2 * 64 + 63, 0, 64 + 63, 0, 0, 0]
    assert mine.tolist() == [False] + [True] * 5 + [False] * 2


def test_prompt_is_the_packed_prompt_attention_and_a_chunk_its_end():
    rng = np.random.default_rng(2)
    n, H, Hk = 70, 2, 1
    k, v = rng.standard_normal((2, n, Hk, 128))
    q = rng.standard_normal((n, H, 128))
    blocks = np.zeros((2, 2, Hk, 64, 128))
    for w, x in enumerate((k, v)):
        blocks[w, 1, :, :] = x[:64].transpose(1, 0, 2)
        blocks[w, 0, :, :6] = x[64:].transpose(1, 0, 2)
    whole = O.prompt_attend(q, k, v, [0, n])[0]
    tab = np.array([[1, 0]])
    np.testing.assert_allclose(O.cache4_prompt(q, *blocks, tab, [n], [0, n])[0], whole, atol=1e-12)
    np.testing.assert_allclose(O.cache4_prompt(q[50:], *blocks, tab, [n], [0, 20])[0], whole[50:], atol=1e-12)
