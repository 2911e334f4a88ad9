"""float32 attention over the 4-bit cache takes queries and weights as three bf16
terms: the third one counts.

A request holds two keys: zeros, and ones in every dim; a query has one element x
that is not zero, so that with s = x / sqrt(128) the row is p / (1 + p) of the
second key's values, p = e^s.  Few operations are left to bound, u = 2^-24:
  score    a sum of three terms, a scaling, the exponent's argument: 8 u |s|
  weights  the exponential 2 ulp, 4 u: relative error d = (8 |s| + 4) u, in
           numerator and denominator: 2 d
  sums     three terms of a weight, two weights, a division, the output: 10 u
together (16 |s| + 18) u of the output, and half as much again for the order of
the operations.  Two terms of a query leave up to 2^-16 = 256 u of it, |s| times
that in the weight; two of a weight leave 256 u.
"""
import numpy as np
import pytest

import oracle as O

U = 2.0 ** -24
LOW, HIGH = 0.2, 8.0  # scores: a weight's terms show at the low end, a query's at the high end


def scores(shape, rng):
    """s < 0 (the first key's weight is one, the second's is any number), and x, a float32."""
    s = -np.where(rng.random(shape) < 0.5, rng.uniform(LOW, 2 * LOW, shape), rng.uniform(0.75 * HIGH, HIGH, shape))
    x = np.float32(s * np.sqrt(128)).astype(np.float64)
    return x / np.sqrt(128), x


def row(s):
    return np.exp(s) / (1 + np.exp(s))


def bound(s):
    return (24 * np.abs(s) + 27) * U * row(s)


def two_terms(x, rounded):
    """What is left of a float32 with its third bf16 term taken away (terms cut off, or rounded)."""
    def bf16(v):
        b = np.float32(v).view(np.uint32)
        if rounded:
            b = b + np.uint32(0x7fff) + (b >> np.uint32(16) & np.uint32(1))
        return (b & np.uint32(0xffff0000)).view(np.float32).astype(np.float64)
    first = bf16(x)
    return first + bf16(x - first)


@pytest.mark.parametrize("rounded", [False, True])
def test_two_terms_would_be_seen(rounded):
    s, x = scores(2000, np.random.default_rng(0))
    less = two_terms(x, rounded) / np.sqrt(128)
    queries = np.abs(row(less) - row(s)) / bound(s)
    p = np.exp(s).astype(np.float32).astype(np.float64)
    weights = np.abs(two_terms(p, rounded) / (1 + p) - row(s)) / bound(s)
    assert (queries > 1).mean() > 0.1 and (weights > 1).mean() > 0.1
    exact = p / (1 + p)
    assert (np.abs(exact - row(s)) <= bound(s)).all()


def two_keys(B, H, rng):
    """A cache of a block a request: tokens 0 (zeros) and 1 (ones), values 0 and any code but 0.  -> cache, v [B, H, 128]"""
    k, v = np.zeros((2, B, H, 64, 64), np.uint8)
    k[:, :, 1] = 0x22
    at = [O.cache4_byte(1, 1, d)[0] for d in range(0, 128, 2)]
    code = rng.integers(1, 8, (2, B, H, 64)) + 8 * rng.integers(0, 2, (2, B, H, 64))
    v.reshape(B, H, -1)[:, :, at] = code[0] | code[1] << 4
    scales = np.full((B, H, 2, 64, 4), 127, np.uint8)
    return (k, v, scales), O.cache4_values(v, scales, 1)[:, :, 1]


def queries(shape, rng):
    s, x = scores(shape, rng)
    q = np.zeros((*shape, 128))
    np.put_along_axis(q, rng.integers(0, 128, (*shape, 1)), x[..., None], -1)
    return q, s


def check(got, s, v):
    """got [..., 128], s [...], v as got"""
    err = np.abs(got - row(s)[..., None] * v) / (bound(s)[..., None] * np.abs(v))
    assert err.max() <= 1, err.max()


@pytest.mark.gpu
@pytest.mark.parametrize("width", [1, 70])   # a work-group a pair, and shares
@pytest.mark.parametrize("G,Q", [(1, 1), (3, 1), (2, 2), (7, 1), (4, 2), (13, 1), (5, 4)])  # 4, 8, 16 and more rows of a product
def test_attend(G, Q, width):
    import paper_2608_03228_amd.saki as S
    from tests.test_gpu_cache4 import dev, host, ints, on_gpu
    rng = np.random.default_rng(G + Q)
    B, H = 24, 2
    cache, v = two_keys(B, H, rng)
    q, s = queries((B, G * H, Q), rng)
    tab = np.full((B, width), -1)
    tab[:, 0] = np.arange(B)
    # all queries see both keys but the first of two and more, which see the first key or none
    got = host(S.saki_cache4_attend(dev(q), *on_gpu(cache), ints(tab), ints([2] * B)))
    assert (got[:, :, :-1] == 0).all()
    check(got[:, :, -1], s[:, :, -1], np.repeat(v, G, 1))
    got = host(S.saki_cache4_attend(dev(q[:, :, :1].copy()), *on_gpu(cache), ints(tab), ints([2] * B),
                                    top_idx=ints(np.broadcast_to([1, 0], (B, G * H, 1, 2)))))
    check(got[:, :, 0], s[:, :, 0], np.repeat(v, G, 1))


@pytest.mark.gpu
@pytest.mark.parametrize("B,H_q,H_kv,width", [(24, 4, 2, 1), (24, 4, 2, 100), (1, 3, 1, 400),  # 64 rows a work-group
                                              (341, 128, 1, 1)])                               # 128
def test_prompt(B, H_q, H_kv, width):
    import paper_2608_03228_amd.saki as S
    from tests.test_gpu_cache4 import dev, host, ints, on_gpu
    rng = np.random.default_rng(B + width)
    cache, v = two_keys(B, H_kv, rng)
    q, s = queries((B, H_q), rng)
    tab = np.full((B, width), -1)
    tab[:, 0] = np.arange(B)
    got = host(S.saki_cache4_prompt(dev(q), *on_gpu(cache), ints(tab), ints([2] * B), ints(range(B + 1))))
    check(got, s, np.repeat(v, H_q // H_kv, 1))
