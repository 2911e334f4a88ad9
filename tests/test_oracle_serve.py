"""CPU pins of the serving oracle: closed forms, identities and special cases."""
import numpy as np
import pytest

import oracle as O


def test_rope_axes_one_axis_is_rope_and_inverse_turns_back():
    rng = np.random.default_rng(0)
    x, pos = rng.standard_normal((7, 3, 128)), rng.integers(0, 100000, 7)
    one = O.rope_axes(x, pos[None], (64,))
    for t in range(7):
        for h in range(3):
            np.testing.assert_allclose(one[t, h], O.rope(x[t, h], pos[t]), atol=1e-9)
    three = np.stack([pos, pos // 7, pos % 13])
    y = O.rope_axes(x, three, (16, 24, 24))
    np.testing.assert_allclose(O.rope_axes(y, three, (16, 24, 24), inverse=True), x, atol=1e-12)
    # equal axes are one axis; a section's pairs follow its own axis alone
    np.testing.assert_allclose(O.rope_axes(x, np.stack([pos] * 3), (16, 24, 24)), one, atol=1e-12)
    other = three.copy()
    other[1] += 5
    same = O.rope_axes(x, other, (16, 24, 24)) == y
    assert same[..., :16].all() and same[..., 40:80].all() and not same[..., 16:40].any()


def test_block_tables_by_hand():
    free = [7, 3, 9]
    tab = [[5, -1, -1], [-1, -1, -1], [2, -1, -1]]
    t, slots, pos, cu, lens, counts = O.block_tables([63, 0, 10], [3, 65, 0], free, tab)
    assert t.tolist() == [[5, 7, -1], [3, 9, -1], [2, -1, -1]]
    assert slots[:3].tolist() == [5 * 64 + 63, 7 * 64, 7 * 64 + 1] and pos[:4].tolist() == [63, 64, 65, 0]
    assert slots[3] == 3 * 64 and slots[-1] == 9 * 64
    assert cu.tolist() == [0, 3, 68, 68] and lens.tolist() == [66, 65, 10] and counts.tolist() == [3, 0]
    # the list ends within the second request; a row holds three blocks
    t, slots, pos, cu, lens, counts = O.block_tables([63, 0], [3, 300], free, tab[:2])
    assert lens.tolist() == [66, 128] and counts.tolist() == [3, 3]
    assert (slots[3 + 128:] == -1).all() and slots.size == 303


@pytest.mark.parametrize("top,s", [(448.0, 1.0), (448.5, 2.0), (0.0, 2.0 ** -100), (7.0, 2.0 ** -6),
                                   (np.nextafter(7.0, 8.0), 2.0 ** -5)])
def test_cache_write_scale_is_the_least_power_of_two(top, s):
    x = np.zeros((1, 1, 128))
    x[0, 0, 5] = -top
    codes, scales = O.cache_write(x, [64 + 1], np.zeros((2, 1, 64, 128)), np.zeros((2, 1)))
    assert scales[1, 0] == s and scales[0, 0] == 0
    assert abs(codes[1, 0, 1, 5] * s + top) <= 2.0 ** -4 * top


def test_cache_write_growth_keeps_normal_codes():
    rng = np.random.default_rng(1)
    x = rng.uniform(1, 2, (5, 2, 128))
    codes, scales = O.cache_write(x, range(5), np.zeros((1, 2, 64, 128)), np.zeros((1, 2)))
    before = codes[0, :, :5] * scales[0][:, None, None]
    big = np.full((1, 2, 128), 300.0)
    codes, scales = O.cache_write(big, [5], codes, scales)
    np.testing.assert_array_equal(codes[0, :, :5] * scales[0][:, None, None], before)
    # a block's first slot starts a new scale
    codes, scales = O.cache_write(x[:1], [0], codes, scales)
    assert (scales[0] <= 2.0 / 448 * 2).all()


def test_attentions_agree_and_reduce_to_softmax():
    rng = np.random.default_rng(2)
    T, d = 70, 128
    k, v = rng.standard_normal((2, T, 1, d))
    q = rng.standard_normal((T, 2, d))
    table = [[1, 0]]
    kc, ks = O.cache_write(k, [64 + t if t < 64 else t - 64 for t in range(T)], np.zeros((2, 1, 64, d)), np.zeros((2, 1)))
    vc, vs = O.cache_write(v, [64 + t if t < 64 else t - 64 for t in range(T)], np.zeros((2, 1, 64, d)), np.zeros((2, 1)))
    sc = np.stack([ks, vs], -1)
    kr, ok = O.cache_rows(kc, ks, table[0], T, 0)
    vr, _ = O.cache_rows(vc, vs, table[0], T, 0)
    assert ok.all() and np.abs(kr - k[:, 0]).max() <= 2.0 ** -4 * np.abs(k).max()
    want, *_ = O.prompt_attend(q, kr[:, None], vr[:, None], [0, T])
    got, *_ = O.cache_attend(q[-3:].transpose(1, 0, 2)[None], kc, vc, sc, table, [T])
    np.testing.assert_allclose(got[0].transpose(1, 0, 2), want[-3:], atol=1e-12)
    every = np.broadcast_to(np.arange(T), (1, 2, 3, T))
    np.testing.assert_allclose(O.cache_attend(q[-3:].transpose(1, 0, 2)[None], kc, vc, sc, table, [T], every)[0], got,
                               atol=1e-12)
    np.testing.assert_array_equal(want[0], np.repeat(vr[:1], 2, 0))
    # two prompts do not see each other; rows outside stay zero
    two, *_ = O.prompt_attend(q, k, v, [0, 30, 60])
    np.testing.assert_array_equal(two[30:60], O.prompt_attend(q[30:60], k[30:60], v[30:60], [0, 30])[0])
    assert (two[60:] == 0).all()
    empty, *_ = O.cache_attend(q[:1].transpose(1, 0, 2)[None], kc, vc, sc, [[-1, -1]], [T])
    assert (empty == 0).all()
