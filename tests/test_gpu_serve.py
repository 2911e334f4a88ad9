"""GPU parity of the serving operators (rotary positions, block tables, the
8-bit cache, attention over it) against the float64 oracle.

Tolerances, before any run.  u = 2^-24 (float32 half step), bf16 half step 2^-8.
  rope       sin and cos within 2.5 u (Taylor remainder 2e-9, argument rounding
             0.79 u, a few roundings of the series); two products and a sum:
             (2.5 + 2) u (|x1| + |x2|), plus 2^-8 |y| for a bf16 output
  tables     equal
  write      codes and scales equal (scaling by a power of two is exact)
  attention  a score is a sum of up to 384 exact products in float32 and a
             scaling: off by 390 u S, S = the row's largest sum of |q_e k_e| /
             sqrt(d); exponent and its argument 4 u more; softmax turns a score
             error e into 2 e of sum p |v|; the weighted sums run over tiles of
             64 and then over N / 64 tiles, and their weights are split into
             terms that leave 2^-17 (bf16 outputs) or 2^-25; then the output's
             rounding
"""
import numpy as np
import pytest

import oracle as O

torch = pytest.importorskip("torch")
S = pytest.importorskip("paper_2608_03228_amd.saki")

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24
F8 = torch.float8_e4m3fn
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


def attention_bound(want, mass, size, N, dt):
    score = (390 * U * size + 4 * U)[..., None]
    return (2 * score + (N / 64 + 128) * U + (2.0 ** -17 if dt == "bf16" else 0)) * mass \
        + (2.0 ** -8 if dt == "bf16" else U) * np.abs(want) + 1e-30


# ---------------------------------------------------------------- rope

@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("T,H_q,H_kv,sections,inverse", [
    (1, 32, 8, (64,), False), (5, 28, 4, (16, 24, 24), True), (67, 3, 1, (10, 54), False),
    (300, 8, 8, (0, 64, 0), False), (4099, 5, 0, (64,), True), (2, 1, 1, (1, 62, 1), False),
])
def test_rope(T, H_q, H_kv, sections, inverse, dt):
    rng = np.random.default_rng(T)
    q, k = (rounded(3 * rng.standard_normal((T, h, 128)), dt) for h in (H_q, H_kv))
    pos = rng.integers(0, 1 << 20, (len(sections), T))
    pos[:, 0] = 0
    tk = dev(k, DT[dt]) if H_kv else None
    qo, ko = S.saki_rope(dev(q, DT[dt]), tk, ints(pos), sections=sections, inverse=inverse)
    for x, y in ((q, qo), (k, ko)):
        if y is None:
            continue
        want = O.rope_axes(x, pos, sections, inverse=inverse)
        size = np.abs(x[..., :64]) + np.abs(x[..., 64:])
        bound = 4.5 * U * np.concatenate([size, size], -1) + (2.0 ** -8 * np.abs(want) if dt == "bf16" else 0)
        assert np.all(np.abs(host(y) - want) <= bound), np.max(np.abs(host(y) - want) / bound)


def test_rope_far_and_negative_positions():
    """Angles up to 2^31: the frequencies (within 2^-51) and the oracle's float64
    product (2^-52) leave 1.5 * 2^-51 of the angle besides the bound of near ones."""
    rng = np.random.default_rng(5)
    pos = np.array([[2147483647, -2147483648, 2000000011, -1, -70001, 1 << 30]])
    x = rounded(rng.standard_normal((6, 2, 128)), "f32")
    got = host(S.saki_rope(dev(x), None, ints(pos))[0])
    want = O.rope_axes(x, pos, (64,))
    size = np.abs(x[..., :64]) + np.abs(x[..., 64:])
    angle = np.abs(pos[0])[:, None, None] * O.ROPE_THETA ** (-np.arange(64) / 64)
    bound = (4.5 * U + 1.5 * 2.0 ** -51 * angle) * size
    assert np.all(np.abs(got - want) <= np.concatenate([bound, bound], -1))


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_rope_in_place_in_a_fused_projection_and_back(dt):
    """q, k slices of one [T, (H_q + 2 H_kv) d] projection, rotated in place and
    back (the gradient); v between them is left as it was."""
    rng = np.random.default_rng(3)
    T, H_q, H_kv = 33, 6, 2
    x = rounded(rng.standard_normal((T, H_q + 2 * H_kv, 128)), dt)
    pos = ints(rng.integers(0, 5000, (3, T)))
    t = dev(x, DT[dt])
    q, k = t[:, :H_q], t[:, H_q + H_kv:]
    want = S.saki_rope(q.contiguous(), k.contiguous(), pos, sections=(16, 24, 24))
    got = S.saki_rope(q, k, pos, sections=(16, 24, 24), q_out=q, k_out=k)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    np.testing.assert_array_equal(host(t)[:, H_q:H_q + H_kv], x[:, H_q:H_q + H_kv])
    S.saki_rope(q, k, pos, sections=(16, 24, 24), inverse=True, q_out=q, k_out=k)
    size = np.abs(x[..., :64]) + np.abs(x[..., 64:])
    # two rotations, and for bf16 two roundings of values up to the pair's size
    tol = (18 * U if dt == "f32" else 18 * U + 2.0 ** -8 * 2.5) * np.concatenate([size, size], -1)
    assert np.all(np.abs(host(t) - x) <= tol)


def test_rope_inverse_is_the_gradient():
    """Against differences: the rotation is linear, so <g, rope(x + e) - rope(x)>
    = <inverse(g), e>."""
    rng = np.random.default_rng(4)
    x, g, e = (rng.standard_normal((9, 2, 128)) for _ in range(3))
    pos = ints(rng.integers(0, 3000, 9))
    f = lambda a, inv=False: host(S.saki_rope(dev(a), None, pos, inverse=inv)[0])  # noqa: E731
    left = ((f(x + e) - f(x)) * g).sum()
    right = (f(g, True) * e).sum()
    scale = np.abs(x).sum() + np.abs(e).sum()
    assert abs(left - right) <= 20 * U * scale * np.abs(g).max()


# ---------------------------------------------------------------- block tables

def tables_case(ctx, new, n_free, rows, T=None, seed=0):
    rng = np.random.default_rng(seed)
    held = [-(-min(max(c, 0), rows * 64) // 64) for c in ctx]
    ids = rng.permutation(sum(held) + n_free + 5)
    tab = np.full((len(ctx), rows), -9)
    at = 0
    for b, h in enumerate(held):
        tab[b, :h] = ids[at:at + h]
        at += h
    free = ids[at:at + n_free]
    want = O.block_tables(ctx, new, free, tab)
    n = want[3][-1]
    T = n if T is None else T
    slots, pos = ints(np.full(T, -77)), ints(np.full(T, -77))
    got = [host(t) for t in S.saki_block_tables(ints(ctx), ints(new), ints(free), ints(tab), slots, pos)]
    m = min(n, T)
    np.testing.assert_array_equal(got[0], want[0])
    for g, w, rest in ((got[1], want[1], -1), (got[2], want[2], 0)):
        np.testing.assert_array_equal(g[:m], w[:m])
        assert (g[m:] == rest).all()
    for g, w in zip(got[3:], want[3:]):
        np.testing.assert_array_equal(g, w)


@pytest.mark.parametrize("ctx,new,n_free,rows,T", [
    ([0], [1], 4, 4, None), ([0], [0], 0, 1, 3), ([64], [1], 4, 2, None), ([63], [1], 4, 2, None),
    ([63, 64, 0, 0, 130], [2, 64, 0, 129, 1], 40, 5, None),
    ([5, 0, 70], [100, 1000, 3], 9, 4, None),        # a row that is full
    ([5, 0, 70], [100, 200, 300], 4, 40, None),      # the list ends
    ([5, 0, 70], [100, 200, 300], 0, 40, None),
    ([10, 20], [100, 50], 9, 9, 70), ([10, 20], [100, 50], 9, 9, 200),
    ([-5, 1000], [-3, 9], 9, 3, 30),                 # below zero, past the row
])
def test_block_tables(ctx, new, n_free, rows, T):
    tables_case(ctx, new, n_free, rows, T)


@pytest.mark.parametrize("B", [255, 1024, 1025, 3000])
def test_block_tables_many_requests(B):
    rng = np.random.default_rng(B)
    tables_case(rng.integers(0, 300, B).tolist(), (rng.integers(0, 200, B) * (rng.random(B) < 0.7)).astype(int).tolist(),
                4 * B, 8, seed=B)


# ---------------------------------------------------------------- writing

def new_cache(n_blocks, H, rng):
    codes = O.fp8_round(100 * rng.standard_normal((2, n_blocks, H, 64, 128)))
    scales = 2.0 ** rng.integers(-7, -3, (n_blocks, H, 2))
    k, v = (dev(c).to(F8) for c in codes)
    return codes, scales, k, v, dev(scales)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("runs,H", [
    # (block, first slot, tokens), None: a token that is skipped
    ([(0, 0, 1)], 1), ([(3, 63, 1)], 3), ([(1, 0, 64)], 2),
    ([(2, 17, 40), None, (0, 5, 1), (4, 0, 64), (1, 0, 9), None, None, (3, 62, 2)], 2),
    ([(b, b % 64, 1) for b in range(70)], 1),
    ([(b, 0, 64) for b in range(66)] + [(70, 0, 33)], 1),     # over 4,096 tokens
    ([(b, 7 * b % 64, 1 + b % 3) for b in range(2100)], 1),
])
def test_cache_write(runs, H, dt):
    rng = np.random.default_rng(len(runs))
    slots = []
    for r in runs:
        slots += [-1] if r is None else [64 * r[0] + min(63, r[1]) + i for i in range(min(r[2], 64 - min(63, r[1])))]
    n_blocks = 1 + max(s // 64 for s in slots)
    codes, scales, kc, vc, sc = new_cache(n_blocks, H, rng)
    T = len(slots)
    size = np.exp(3 * rng.standard_normal((T, 1, 1)))
    size[rng.random(T) < 0.05] = 0
    k, v = (rounded(size * rng.standard_normal((T, H, 128)), dt) for _ in range(2))
    for i, s in enumerate(slots):
        if s < 0:
            k[i] = v[i] = np.nan  # a skipped token's contents have no effect
    S.saki_cache_write(dev(k, DT[dt]), dev(v, DT[dt]), ints(slots), kc, vc, sc)
    for i, (x, c) in enumerate(((k, kc), (v, vc))):
        want, ws = O.cache_write(x, slots, codes[i], scales[..., i])
        np.testing.assert_array_equal(host(sc)[..., i], ws)
        np.testing.assert_array_equal(host(c.float()), want)


def test_cache_write_every_code_and_tie():
    """Each E4M3 value and each midpoint between two, of both signs."""
    pos = np.array(sorted({float(v) for v in O.fp8_round(np.linspace(0, 448, 200001))} |
                          {i * 2.0 ** -9 for i in range(8)}))
    vals = np.concatenate([pos, (pos[1:] + pos[:-1]) / 2, pos * (1 + 2.0 ** -12), -pos])
    x = np.zeros((-(-vals.size // 127), 1, 128))
    x[:, :, 0] = 448.0  # the scale is one
    x[:, 0, 1:] = np.resize(vals, (x.shape[0], 127))
    x = x[:, :, :]
    assert x.shape[0] <= 64
    codes, scales, kc, vc, sc = new_cache(1, 1, np.random.default_rng(0))
    x = np.minimum(x, 448.0)
    S.saki_cache_write(dev(x), dev(x / 4), ints(range(x.shape[0])), kc, vc, sc)
    want = O.fp8_round(x[:, 0])
    np.testing.assert_array_equal(host(kc.float())[0, 0, :x.shape[0]], want)
    np.testing.assert_array_equal(host(vc.float())[0, 0, :x.shape[0]], want)
    assert host(sc)[0, 0].tolist() == [1.0, 0.25]


def test_cache_write_token_by_token_and_strided():
    """One token at a time, growing ones among them, out of a fused projection."""
    rng = np.random.default_rng(9)
    H, T = 2, 64
    codes, scales, kc, vc, sc = new_cache(2, H, rng)
    x = rounded(np.exp(np.linspace(-4, 6, T))[:, None, None] * rng.standard_normal((T, 3 * H, 128)), "bf16")
    t = dev(x, torch.bfloat16)
    wk, wv = codes[0], codes[1]
    sk, sv = scales[..., 0], scales[..., 1]
    for i in range(T):
        slot = [64 + i]
        S.saki_cache_write(t[i:i + 1, H:2 * H], t[i:i + 1, 2 * H:], ints(slot), kc, vc, sc)
        wk, sk = O.cache_write(x[i:i + 1, H:2 * H], slot, wk, sk)
        wv, sv = O.cache_write(x[i:i + 1, 2 * H:], slot, wv, sv)
    np.testing.assert_array_equal(host(kc.float()), wk)
    np.testing.assert_array_equal(host(vc.float()), wv)
    np.testing.assert_array_equal(host(sc), np.stack([sk, sv], -1))
    # all at once through strides: the same scales, codes rounded once
    S.saki_cache_write(t[:, H:2 * H], t[:, 2 * H:], ints(range(64)), kc, vc, sc)
    np.testing.assert_array_equal(host(kc.float())[0], O.cache_write(x[:, H:2 * H], range(64), wk, sk)[0][0])


def test_cache_write_slots_out_of_range_write_nothing():
    rng = np.random.default_rng(10)
    codes, scales, kc, vc, sc = new_cache(3, 1, rng)
    before = [t.clone() for t in (kc.view(torch.uint8), vc.view(torch.uint8), sc)]
    x = dev(rng.standard_normal((5, 1, 128)))
    S.saki_cache_write(x, x, ints([-1, 192, 2147483647, -2147483648, 500]), kc, vc, sc)
    for a, b in zip(before, (kc.view(torch.uint8), vc.view(torch.uint8), sc)):
        assert torch.equal(a, b)


# ---------------------------------------------------------------- attention over the cache

def attend_case(lens, H_q, H_kv, Q, dt, rows=None, seed=0, stale=True):
    rng = np.random.default_rng(seed + 17)
    held = [-(-max(n, 0) // 64) for n in lens]
    rows = max(1, max(held)) if rows is None else rows
    n_blocks = sum(held) + 2
    codes, scales, k, v, s = new_cache(n_blocks, H_kv, rng)
    ids = rng.permutation(n_blocks)
    tab = np.full((len(lens), rows), n_blocks + 7)  # never followed
    at = 0
    for b, h in enumerate(held):
        tab[b, :min(h, rows)] = ids[at:at + min(h, rows)]
        at += h
    if stale:  # slots behind a request's last key hold NaN codes
        for b, n in enumerate(lens):
            if n > 0 and n % 64 and n // 64 < rows:
                blk = int(tab[b, n // 64])
                k.view(torch.uint8)[blk, :, n % 64:] = 0x7F
                v.view(torch.uint8)[blk, :, n % 64:] = 0xFF
    q = rounded(0.5 * rng.standard_normal((len(lens), H_q, Q, 128)), dt)
    return q, codes, scales, (k, v, s), tab


def check_attend(case, lens, dt, top_idx=None, **kw):
    q, codes, scales, (k, v, s), tab = case
    out = S.saki_cache_attend(dev(q, DT[dt]), k, v, s, ints(tab), ints(lens),
                              top_idx=None if top_idx is None else ints(top_idx), **kw)
    want, mass, size = O.cache_attend(q, codes[0], codes[1], scales, tab, lens, top_idx)
    bound = attention_bound(want, mass, size, max(max(lens), 64), dt)
    err = np.abs(host(out) - want)
    assert np.all(err <= bound), (np.max(err / bound), np.unravel_index(np.argmax(err / bound), err.shape))


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("lens,H_q,H_kv,Q", [
    ([1], 1, 1, 1), ([63], 4, 1, 1), ([64], 8, 2, 1), ([65], 28, 4, 1), ([0, 5, 0], 4, 2, 1),
    ([0], 2, 1, 3), ([1000], 32, 8, 1), ([300, 1, 640, 129], 12, 1, 4), ([3, 200], 5, 5, 16),
    ([2], 4, 2, 16), ([700, 699], 17, 1, 1), ([-4, 70], 2, 1, 2), ([1500, 300], 4, 1, 1),
])
@pytest.mark.parametrize("rows", [None, 70])  # narrow tables: a work-group per pair; wide ones: shares, joined
def test_cache_attend(rows, lens, H_q, H_kv, Q, dt):
    check_attend(attend_case(lens, H_q, H_kv, Q, dt, rows), lens, dt)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("rows", [15, 70])
def test_cache_attend_many_requests(rows, dt):
    """More requests than one scan step takes, most of them short."""
    rng = np.random.default_rng(0)
    lens = rng.integers(0, 70, 530).tolist()
    lens[400] = 900
    check_attend(attend_case(lens, 2, 2, 1, dt, rows), lens, dt)


def test_cache_attend_table_entries_out_of_range():
    """Blocks that a table does not hold count as keys that are not there, and
    a length past the table's room ends with it."""
    lens = [500, 300, 400]
    q, codes, scales, c, tab = attend_case(lens, 4, 2, 1, "f32", stale=False)
    tab[0, 3], tab[0, 7], tab[1, :] = -1, 1 << 30, -5
    check_attend((q, codes, scales, c, tab), lens, "f32")
    check_attend((q, codes, scales, c, tab[:, :2].copy()), [1 << 30, 2147483647, 128], "f32")
    idx = np.tile(np.array([0, 200, 450, 2147483647, 499, -3]), (3, 4, 1, 1))
    check_attend((q, codes, scales, c, tab), lens, "f32", top_idx=idx)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("lens,H_q,H_kv,Q,k", [
    ([1], 1, 1, 1, 64), ([1000], 32, 8, 1, 64), ([300, 0, 640, 129], 12, 1, 4, 17), ([3, 200], 5, 5, 16, 1),
    ([64, 65], 28, 4, 1, 63),
])
def test_cache_attend_lists(lens, H_q, H_kv, Q, k, dt):
    rng = np.random.default_rng(k)
    case = attend_case(lens, H_q, H_kv, Q, dt)
    idx = rng.integers(-2, 1 + np.array(lens)[:, None, None, None], (len(lens), H_q, Q, k))  # repeats and unseen ones
    idx[0, 0, 0] = -1
    check_attend(case, lens, dt, top_idx=idx)


@pytest.mark.parametrize("top_idx", [False, True])
def test_cache_attend_peaked_rows(top_idx):
    """Scores of hundreds: one key takes all the weight."""
    lens = [400, 64]
    q, codes, scales, c, tab = attend_case(lens, 4, 2, 1, "f32")
    q = 40 * q
    idx = np.tile(np.arange(64), (2, 4, 1, 1)) if top_idx else None
    check_attend((q, codes, scales, c, tab), lens, "f32", top_idx=idx)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("rows,top_idx", [(None, False), (70, False), (None, True)])
def test_cache_attend_query_of_nan_stays_one(rows, top_idx, dt):
    """A row whose query is NaN is NaN whichever way the work is divided, and the
    other rows are what they are without it."""
    lens = [700, 0, 3]
    q, _, _, (k, v, s), tab = attend_case(lens, 4, 2, 2, dt, rows)
    idx = ints(np.tile(np.arange(3), (3, 4, 2, 1))) if top_idx else None
    clean = S.saki_cache_attend(dev(q, DT[dt]), k, v, s, ints(tab), ints(lens), top_idx=idx)
    bad = np.zeros(q.shape[:3], bool)
    bad[0, 1, 0] = bad[0, 3, 1] = bad[1, 2, 0] = bad[2, 0, 1] = True
    q[bad] = np.nan
    out = host(S.saki_cache_attend(dev(q, DT[dt]), k, v, s, ints(tab), ints(lens), top_idx=idx))
    np.testing.assert_array_equal(out[~bad], host(clean)[~bad])
    assert np.all(out[1] == 0)  # no key
    bad[1] = False
    assert np.all(np.isnan(out[bad]))


def test_cache_attend_is_the_same_every_time_and_on_another_stream():
    lens = [3000, 10, 700, 2500]
    q, codes, scales, (k, v, s), tab = attend_case(lens, 28, 4, 1, "bf16")
    assert tab.shape[1] > 16  # shares and their join
    args = (dev(q, torch.bfloat16), k, v, s, ints(tab), ints(lens))
    first = S.saki_cache_attend(*args)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    other = S.saki_cache_attend(*args, stream=side)
    side.synchronize()
    assert torch.equal(first, other) and torch.equal(first, S.saki_cache_attend(*args))


# ---------------------------------------------------------------- a step, as it is used

def step(s, x, pos, H_q, H_kv, idx=None):
    """One decode step: tables, rotation, write, attention; the outputs are s's."""
    S.saki_block_tables(s["ctx"], s["new"], s["free"], s["tab"], s["slots"], s["pos"], cu=s["cu"], lens=s["lens"],
                        counts=s["counts"])
    q, k, v = x[:, :H_q], x[:, H_q:H_q + H_kv], x[:, H_q + H_kv:]
    S.saki_rope(q, k, s["pos"], q_out=s["q"], k_out=s["k"])
    S.saki_cache_write(s["k"], v, s["slots"], *s["cache"])
    B = s["ctx"].numel()
    S.saki_cache_attend(s["q"].view(B, H_q, 1, 128), *s["cache"], s["tab"], s["lens"], out=s["out"], ws=s["ws"])
    if idx is not None:
        S.saki_cache_attend(s["q"].view(B, H_q, 1, 128), *s["cache"], s["tab"], s["lens"], top_idx=idx, out=s["out2"])


def step_state(ctx, H_q, H_kv, dt, rng, room=512):
    B, rows = len(ctx), room // 64
    held = [-(-c // 64) for c in ctx]
    n_blocks = B * rows
    codes, scales, k, v, sc = new_cache(n_blocks, H_kv, rng)
    ids = rng.permutation(n_blocks)
    tab = np.full((B, rows), -1)
    at = 0
    for b, h in enumerate(held):
        tab[b, :h] = ids[at:at + h]
        at += h
    z = lambda *n, d=torch.int32: torch.zeros(n, dtype=d, device=DEV)  # noqa: E731
    s = dict(ctx=ints(ctx), new=ints([1] * B), free=ints(ids[at:]), tab=ints(tab), slots=z(B), pos=z(B), cu=z(B + 1),
             lens=z(B), counts=z(2), q=z(B, H_q, 128, d=DT[dt]), k=z(B, H_kv, 128, d=DT[dt]), cache=(k, v, sc),
             out=z(B, H_q, 1, 128, d=DT[dt]), out2=z(B, H_q, 1, 128, d=DT[dt]),
             ws=z(S.saki_cache_attend_workspace_bytes(B, H_q, H_kv, 1, rows), d=torch.uint8))
    return s, codes, scales, tab, ids[at:]


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_step_of_all_operators(dt):
    rng = np.random.default_rng(21)
    ctx, H_q, H_kv = [0, 63, 64, 200, 191], 8, 2
    s, codes, scales, tab, free = step_state(ctx, H_q, H_kv, dt, rng)
    x = rounded(rng.standard_normal((5, H_q + 2 * H_kv, 128)), dt)
    idx = np.tile(np.where(np.arange(64) < 40, np.arange(64) * 3, -1), (5, H_q, 1, 1))
    step(s, dev(x, DT[dt]), None, H_q, H_kv, ints(idx))
    wt, slots, pos, cu, lens, counts = O.block_tables(ctx, [1] * 5, free, tab)
    np.testing.assert_array_equal(host(s["tab"]), wt)
    np.testing.assert_array_equal(host(s["slots"]), slots)
    # each part against the oracle on what the part before it gave
    q, k = host(s["q"]), host(s["k"])
    kc, ks = O.cache_write(k, slots, codes[0], scales[..., 0])
    vc, vs = O.cache_write(x[:, H_q + H_kv:], slots, codes[1], scales[..., 1])
    np.testing.assert_array_equal(host(s["cache"][0].float()), kc)
    np.testing.assert_array_equal(host(s["cache"][1].float()), vc)
    sc = np.stack([ks, vs], -1)
    for out, li in ((s["out"], None), (s["out2"], idx)):
        want, mass, size = O.cache_attend(q[:, :, None], kc, vc, sc, wt, lens, li)
        assert np.all(np.abs(host(out) - want) <= attention_bound(want, mass, size, 256, dt))


def test_step_captured_and_replayed():
    """The step in a graph, replayed with changed inputs and eager work between,
    against the eager step."""
    rng = np.random.default_rng(22)
    ctx, H_q, H_kv, dt = [5, 63, 130], 4, 2, "bf16"
    s, *_ = step_state(ctx, H_q, H_kv, dt, rng)
    e = {k: (tuple(x.clone() for x in v) if isinstance(v, tuple) else v.clone()) for k, v in s.items()}
    x = dev(rng.standard_normal((3, H_q + 2 * H_kv, 128)), torch.bfloat16)
    warm = {k: (tuple(y.clone() for y in v) if isinstance(v, tuple) else v.clone()) for k, v in s.items()}
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(warm, x, None, H_q, H_kv)
    torch.cuda.current_stream().wait_stream(side)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step(s, x, None, H_q, H_kv)
        s["ctx"].copy_(s["lens"])
    for i in range(5):
        new = dev(rng.standard_normal((3, H_q + 2 * H_kv, 128)), torch.bfloat16)
        x.copy_(new)
        g.replay()
        torch.cuda.synchronize()
        step(e, x, None, H_q, H_kv)
        e["ctx"].copy_(e["lens"])
        # the blocks taken leave the list (the same list for both)
        taken = int(e["counts"][0])
        for t in (s, e):
            rest = torch.cat([t["free"][taken:], t["free"][:taken]])
            t["free"].copy_(rest)
        torch.cuda.synchronize()
        for name in ("tab", "slots", "lens", "q", "k", "out"):
            assert torch.equal(s[name], e[name]), (i, name)
        for a, b in zip(s["cache"], e["cache"]):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8)), i


# ---------------------------------------------------------------- large arrays, calls at once

def test_offsets_past_32_bits():
    """Blocks beyond 4 GiB of a cache, token rows more than 4 GiB apart: writes,
    both attentions and the rotation."""
    rng = np.random.default_rng(30)
    H, n_blocks = 8, 1 + (5 << 30) // (8 * 8192)
    kc = torch.zeros(n_blocks, H, 64, 128, dtype=F8, device=DEV)
    vc = torch.zeros(n_blocks, H, 64, 128, dtype=F8, device=DEV)
    sc = torch.zeros(n_blocks, H, 2, device=DEV)
    ids = [n_blocks - 1, 3, n_blocks - 2]
    slots = [ids[t // 64] * 64 + t % 64 for t in range(150)]
    k, v = (rng.standard_normal((150, H, 128)) for _ in range(2))
    S.saki_cache_write(dev(k), dev(v), ints(slots), kc, vc, sc)
    near = [64 * i + t for i in range(3) for t in range(64)][:150]
    wk, sk = O.cache_write(dev(k).double().cpu().numpy(), near, np.zeros((3, H, 64, 128)), np.zeros((3, H)))
    wv, sv = O.cache_write(dev(v).double().cpu().numpy(), near, np.zeros((3, H, 64, 128)), np.zeros((3, H)))
    for i, b in enumerate(ids):
        np.testing.assert_array_equal(host(kc[b].float()), wk[i])
        np.testing.assert_array_equal(host(vc[b].float()), wv[i])
    q = rounded(rng.standard_normal((1, 2 * H, 1, 128)), "f32")
    scales = np.stack([sk, sv], -1)
    for idx in (None, np.tile(np.arange(0, 150, 3), (1, 2 * H, 1, 1))):
        for wide in (0, 80):  # both ways of dividing the work
            tab = ints([ids + [-1] * wide])
            out = S.saki_cache_attend(dev(q), kc, vc, sc, tab, ints([150]), top_idx=None if idx is None else ints(idx))
            want, mass, size = O.cache_attend(q, wk, wv, scales, [[0, 1, 2]], [150], idx)
            assert np.all(np.abs(host(out) - want) <= attention_bound(want, mass, size, 150, "f32"))
    del kc, vc
    x = torch.zeros(3, (3 << 30) // 128, 128, dtype=torch.bfloat16, device=DEV)[:, :2]  # rows 6 GiB apart
    y = rounded(rng.standard_normal((3, 2, 128)), "bf16")
    x.copy_(dev(y, torch.bfloat16))
    pos = ints([1, 70000, 5])
    want = S.saki_rope(dev(y, torch.bfloat16), None, pos)[0]
    S.saki_rope(x, None, pos, q_out=x)
    assert torch.equal(x, want)


def test_calls_at_once_on_two_streams():
    """Two batches, each with its own workspace, interleaved on two streams."""
    lens = [[3000, 100, 2500], [2100, 2900, 64]]
    runs = []
    for i in range(2):
        q, codes, scales, (k, v, s), tab = attend_case(lens[i], 8, 2, 1, "f32", seed=i)
        args = (dev(q), k, v, s, ints(tab), ints(lens[i]))
        ws = torch.empty(S.saki_cache_attend_workspace_bytes(3, 8, 2, 1, tab.shape[1]), dtype=torch.uint8, device=DEV)
        runs.append((args, ws, S.saki_cache_attend(*args), torch.empty_like(args[0]), torch.cuda.Stream()))
    torch.cuda.synchronize()
    for _ in range(20):
        for args, ws, want, out, stream in runs:
            S.saki_cache_attend(*args, out=out, ws=ws, stream=stream)
    torch.cuda.synchronize()
    for args, ws, want, out, stream in runs:
        assert torch.equal(out, want)


def test_arguments_of_other_kinds_are_refused():
    """Types, shapes, strides and devices that the calls do not take."""
    k = torch.zeros(4, 2, 64, 128, dtype=F8, device=DEV)
    s = torch.zeros(4, 2, 2, device=DEV)
    x = torch.zeros(5, 2, 128, device=DEV)
    i5, tab, lens = ints(range(5)), ints([[0, 1]]), ints([70])
    q = torch.zeros(1, 4, 1, 128, device=DEV)
    for call in (
            lambda: S.saki_cache_write(x.half(), x.half(), i5, k, k.clone(), s),
            lambda: S.saki_cache_write(x, x.bfloat16(), i5, k, k.clone(), s),
            lambda: S.saki_cache_write(x, x, i5[:4], k, k.clone(), s),
            lambda: S.saki_cache_write(x, x, i5.long(), k, k.clone(), s),
            lambda: S.saki_cache_write(x, x, i5.cpu(), k, k.clone(), s),
            lambda: S.saki_cache_write(x.transpose(0, 1), x, i5, k, k.clone(), s),
            lambda: S.saki_cache_write(x, x, i5, k.view(torch.uint8), k.clone(), s),
            lambda: S.saki_cache_write(x, x, i5, k[:, :, ::2], k.clone(), s),
            lambda: S.saki_cache_write(x, x, i5, k, k[:3], s),
            lambda: S.saki_cache_write(x, x, i5, k, k.clone(), s.double()),
            lambda: S.saki_cache_write(x, x, i5, k, k.clone(), s[:, :1]),
            lambda: S.saki_cache_attend(q, k, k, s, tab[0], lens),
            lambda: S.saki_cache_attend(q, k, k, s, tab, ints([70, 1])),
            lambda: S.saki_cache_attend(q[:, :, :, :64], k, k, s, tab, lens),
            lambda: S.saki_cache_attend(q, k, k, s, tab, lens, top_idx=ints([[[[0]]]])),
            lambda: S.saki_cache_attend(q, k, k, s, tab, lens, out=q.bfloat16()),
            lambda: S.saki_cache_attend(q.transpose(1, 2).expand(1, 4, 4, 128).transpose(1, 2), k, k, s, tab, lens),
            lambda: S.saki_rope(x, x[:4], i5),
            lambda: S.saki_rope(x, x, i5[:3]),
            lambda: S.saki_rope(x, x, ints([[1] * 5] * 2)),
            lambda: S.saki_rope(x, x, i5, q_out=x.flip(2)[:, :, ::2]),
            lambda: S.saki_rope(x.expand(5, 2, 128).as_strided((5, 2, 128), (0, 128, 1)), x, i5),
            lambda: S.saki_block_tables(lens, lens, i5, tab, i5, i5[:3]),
            lambda: S.saki_block_tables(lens, lens, i5, tab.long(), i5, i5),
            lambda: S.saki_attend_prompt(x, x, x, lens[:0]),
            lambda: S.saki_attend_prompt(x, x[:, :1], x, ints([0, 5])),
    ):
        with pytest.raises(ValueError):
            call()
    for call, status in (
            (lambda: S.saki_rope(x, x, i5, sections=(63,)), -1),
            (lambda: S.saki_rope(torch.zeros(5 * 2 * 128 + 1, device=DEV)[1:].view(5, 2, 128), x, i5), -1),
            (lambda: S.saki_rope(x, x, i5, rope_theta=0.0), -1),
            (lambda: S.saki_cache_attend(torch.zeros(1, 3, 1, 128, device=DEV), k, k, s, tab, lens), -1),
            (lambda: S.saki_cache_attend(torch.zeros(1, 2, 17, 128, device=DEV), k, k, s, tab, lens), -2),
            (lambda: S.saki_block_tables(lens, ints([1]), i5, tab, ints([0]), ints([0]), lens=lens), -1),
    ):
        with pytest.raises(S.SakiError) as e:
            call()
        assert e.value.status == status


def test_step_of_a_fixed_size_with_fewer_tokens():
    """A captured step for 4 requests and 8 tokens, replayed with fewer of both:
    what stands behind the last token is neither written to the cache nor read."""
    rng = np.random.default_rng(31)
    H_q, H_kv, B, T = 4, 2, 4, 8
    s, codes, scales, tab, free = step_state([70, 0, 10, 130], H_q, H_kv, "f32", rng)
    z = lambda *n, d=torch.int32: torch.zeros(n, dtype=d, device=DEV)  # noqa: E731
    s.update(slots=ints([5] * T), pos=ints([9] * T), q=z(T, H_q, 128, d=torch.float32),
             k=z(T, H_kv, 128, d=torch.float32))
    x = z(T, H_q + 2 * H_kv, 128, d=torch.float32)

    def run():
        S.saki_block_tables(s["ctx"], s["new"], s["free"], s["tab"], s["slots"], s["pos"], cu=s["cu"], lens=s["lens"],
                            counts=s["counts"])
        S.saki_rope(x[:, :H_q], x[:, H_q:H_q + H_kv], s["pos"], q_out=s["q"], k_out=s["k"])
        S.saki_cache_write(s["k"], x[:, H_q + H_kv:], s["slots"], *s["cache"])

    s["new"].zero_()
    x.fill_(float("nan"))
    before = [c.clone() for c in s["cache"]]
    run()  # no token at all
    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        run()
    assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(before, s["cache"]))
    kc, sk = codes[0], scales[..., 0]
    vc, sv = codes[1], scales[..., 1]
    for new in ([1, 0, 1, 0], [0, 3, 0, 1], [0, 0, 0, 0], [2, 2, 2, 2]):
        n = sum(new)
        y = rounded(rng.standard_normal((n, H_q + 2 * H_kv, 128)), "f32")
        x.fill_(float("nan"))
        x[:n].copy_(dev(y))
        s["new"].copy_(ints(new))
        g.replay()
        torch.cuda.synchronize()
        wt, slots, pos, cu, lens, counts = O.block_tables(host(s["ctx"]), new, free, tab)
        assert host(s["slots"]).tolist() == slots.tolist() + [-1] * (T - n)
        k = host(s["k"])[:n]
        kc, sk = O.cache_write(k, slots, kc, sk)
        vc, sv = O.cache_write(y[:, H_q + H_kv:], slots, vc, sv)
        np.testing.assert_array_equal(host(s["cache"][0].float()), kc)
        np.testing.assert_array_equal(host(s["cache"][1].float()), vc)


# ---------------------------------------------------------------- beside the index

def test_index_lists_read_from_the_cache():
    """The index's lists over the 8-bit cache against saki_attend over the exact
    keys: codes from unrotated keys, rotated keys in the cache."""
    import workloads as W
    N, H_q, H_kv, B = 1500, 8, 2, 2
    spec = W.SPECS["decode_1m"].with_(N=N, H_q=H_q, H_kv=H_kv, batch=B, Q=1)
    inp = W.make_layer(spec, with_values=True)
    cal = S.saki_calibrate(inp["q_cal"], inp["k_cal"], 32)
    keys, vals, q = dev(inp["keys"]), dev(inp["values"]), dev(inp["queries"])
    index = S.saki_build_index(keys, dev(cal["B_k"]), dev(cal["mu"]), 32, "bf16", H_q)
    idx, _ = S.saki_score_topk(index, "bf16", q, dev(cal["B_q"]), dev(cal["mu"]), H_kv, N, N, 32)
    exact = host(S.saki_attend(vals, q, idx, N, keys=keys))
    # the same tokens through tables, rotation and the cache
    rows = -(-N // 64)
    free = ints(np.random.default_rng(1).permutation(B * rows))
    slots, pos = (torch.empty(B * N, dtype=torch.int32, device=DEV) for _ in range(2))
    tab = torch.full((B, rows), -1, dtype=torch.int32, device=DEV)
    tab, slots, pos, cu, lens, counts = S.saki_block_tables(ints([0] * B), ints([N] * B), free, tab, slots, pos)
    k = keys.transpose(1, 2).reshape(B * N, H_kv, 128).contiguous()
    v = vals.transpose(1, 2).reshape(B * N, H_kv, 128).contiguous()
    _, kr = S.saki_rope(k[:, :1], k, pos)
    cache = (torch.zeros(B * rows, H_kv, 64, 128, dtype=F8, device=DEV),
             torch.zeros(B * rows, H_kv, 64, 128, dtype=F8, device=DEV), torch.zeros(B * rows, H_kv, 2, device=DEV))
    S.saki_cache_write(kr, v, slots, *cache)
    qr, _ = S.saki_rope(q.view(B, H_q, 128), None, ints([N - 1] * B))
    got = host(S.saki_cache_attend(qr.view(B, H_q, 1, 128), *cache, tab, lens, top_idx=idx))
    # exactly the attention of what the cache holds ...
    codes = [host(c.float()) for c in cache[:2]]
    want, mass, size = O.cache_attend(host(qr)[:, :, None], codes[0], codes[1], host(cache[2]), host(tab), [N] * B,
                                      host(idx))
    assert np.all(np.abs(got - want) <= attention_bound(want, mass, size, N, "f32"))
    # ... which holds keys and values to half an E4M3 step, 2^-4 of an element:
    # a score is off by 2^-4 size at most (and the rotation's 9 u), a value by 2^-4
    e = 2 * (2.0 ** -4 * size * 17 / 15)[..., None]
    top = np.abs(host(vals)).max()
    assert np.all(np.abs(got - exact) <= np.minimum(np.expm1(e), 2) * top + (2.0 ** -4 + 1e-4) * top)
