"""GPU parity of saki_attend_prompt against the float64 oracle.

Tolerances, before any run.  u = 2^-24, b = 2^-8 (half a bf16 step).
  scores     128 products, exact (bf16) or to 2^-21 = 8 u (float32: two fp16 parts
             an element), summed in float32, scaled, and the exponent with its
             argument: 140 u S + 4 u, S = the row's largest sum of |q_e k_e| /
             sqrt(d); softmax turns a score error e into 2 e of sum p |v|
  sums       (N / 32 + 64) u of sum p |v| (a tile, then tile by tile; float32
             weights and values to 8 u)
  bf16       weights rounded once before they meet the values: b of sum p |v|;
             the output's rounding: b of the output
"""
import numpy as np
import pytest

import oracle as O
from tests.test_gpu_serve import DT, U, dev, host, ints, rounded

torch = pytest.importorskip("torch")
S = pytest.importorskip("paper_2608_03228_amd.saki")

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def make(T, H_q, H_kv, dt, seed, size=0.7):
    rng = np.random.default_rng(seed)
    return [rounded(s * rng.standard_normal((T, h, 128)), dt) for s, h in ((size, H_q), (1, H_kv), (1, H_kv))]


def check(out, q, k, v, cu, dt):
    want, mass, size = O.prompt_attend(q, k, v, cu)
    n = max(np.diff(cu).max(), 64)
    score = (140 * U * size + 4 * U)[..., None]
    b = 2.0 ** -8 if dt == "bf16" else 0
    bound = (2 * score + (n / 32 + 64) * U + b) * mass + (b + U) * np.abs(want)
    got = host(out)
    inside = np.zeros(len(q), bool)
    for a, e in zip(cu[:-1], cu[1:]):
        inside[a:e] = True
    err = np.abs(got - want)[inside]
    assert np.all(err <= bound[inside]), (np.max(err / bound[inside]),
                                          np.unravel_index(np.argmax(err / bound[inside]), err.shape))
    return got, inside


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("lens,H_q,H_kv", [
    ([1], 1, 1), ([2], 32, 8), ([31, 33, 1], 4, 1), ([64], 8, 8), ([65, 0, 127, 128, 129], 4, 2),
    ([0, 0, 5], 28, 4), ([300], 12, 1), ([17, 400], 5, 5), ([1] * 40, 16, 2), ([255, 1, 256], 7, 1),
    # more blocks than halves are taken for: every work-group of 128 rows
    ([70, 1, 33, 130] * 3, 32, 8), ([5, 200] * 3, 40, 20),
])
def test_attend_prompt(lens, H_q, H_kv, dt):
    cu = np.concatenate([[0], np.cumsum(lens)])
    q, k, v = make(cu[-1], H_q, H_kv, dt, sum(lens))
    out = S.saki_attend_prompt(*(dev(x, DT[dt]) for x in (q, k, v)), ints(cu))
    check(out, q, k, v, cu, dt)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_attend_prompt_leaves_other_tokens_and_reads_none(dt):
    """Tokens before the first prompt and behind the last hold NaN and stay."""
    cu = np.array([3, 70, 70, 150])
    q, k, v = make(200, 4, 2, dt, 1)
    for x in (q, k, v):
        x[:3] = x[150:] = np.nan
    out = torch.full((200, 4, 128), 7.0, dtype=DT[dt], device=DEV)
    got = S.saki_attend_prompt(*(dev(x, DT[dt]) for x in (q, k, v)), ints(cu), out=out)
    for x in (q, k, v):
        x[:3] = x[150:] = 0
    got, inside = check(got, q, k, v, cu, dt)
    assert (got[~inside] == 7).all()


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_attend_prompt_behind_many_other_tokens(dt):
    """Row blocks that lie before the first prompt, and between the last one and
    the end, belong to none; more prompts than a search step tells apart."""
    cu = np.concatenate([[400], 400 + np.cumsum(np.arange(90) % 4)])
    T = cu[-1] + 333
    q, k, v = make(T, 4, 2, dt, 12)
    out = torch.full((T, 4, 128), 7.0, dtype=DT[dt], device=DEV)
    got = S.saki_attend_prompt(*(dev(x, DT[dt]) for x in (q, k, v)), ints(cu), out=out)
    got, inside = check(got, q, k, v, cu, dt)
    assert (got[~inside] == 7).all()


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_attend_prompt_of_a_fused_projection(dt):
    """q, k, v as slices of one [T, H_q + 2 H_kv, d] tensor."""
    H_q, H_kv, cu = 6, 2, np.array([0, 90, 131])
    q, k, v = make(131, H_q, H_kv, dt, 2)
    x = dev(np.concatenate([q, k, v], 1), DT[dt])
    out = S.saki_attend_prompt(x[:, :H_q], x[:, H_q:H_q + H_kv], x[:, H_q + H_kv:], ints(cu))
    check(out, q, k, v, cu, dt)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_attend_prompt_rising_and_peaked_scores(dt):
    """Every key's score passes the ones before it by far (the running maximum
    moves at every tile), and then falls."""
    T = 260
    q, k, v = make(T, 2, 1, dt, 3)
    up = np.concatenate([np.arange(130), np.arange(130)[::-1]])[:, None, None]
    u = np.sign(k[:1])
    k = rounded(0.05 * k + u * up * 0.02, dt)
    q = rounded(0.1 * q + u * 1.0, dt)
    out = S.saki_attend_prompt(*(dev(x, DT[dt]) for x in (q, k, v)), ints([0, T]))
    check(out, q, k, v, np.array([0, T]), dt)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_attend_prompt_offsets_that_do_not_ascend_stay_in_range(dt):
    """Such offsets are the caller's mistake: what is written to out is not
    specified, but nothing outside it is."""
    q, k, v = (dev(x, DT[dt]) for x in make(100, 4, 2, dt, 4))
    need = S.saki_attend_prompt_workspace_bytes(dt, 100, 2, 2)
    for cu in ([0, 2000000000, 50], [-5, 60, 1000], [90, 10, 95], [2147483647, -2147483648, 7]):
        out = torch.full((300, 4, 128), 7.0, dtype=DT[dt], device=DEV)
        ws = torch.full((need + 8192,), 9, dtype=torch.uint8, device=DEV)
        S.saki_attend_prompt(q, k, v, ints(cu), out=out[100:200], ws=ws[4096:4096 + need])
        assert (out[:100] == 7).all() and (out[200:] == 7).all()
        assert (ws[:4096] == 9).all() and (ws[4096 + need:] == 9).all()


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("H_q,H_kv", [(8, 2), (16, 4)])  # halved blocks, whole ones
def test_attend_prompt_long_rows_sampled(H_q, H_kv, dt):
    """A long prompt among short ones: sampled rows, against float64 on the GPU."""
    lens = [40, 5000, 1, 700]
    cu = np.concatenate([[0], np.cumsum(lens)])
    q, k, v = make(cu[-1], H_q, H_kv, dt, 5)
    tq, tk, tv = (dev(x, DT[dt]) for x in (q, k, v))
    got = host(S.saki_attend_prompt(tq, tk, tv, ints(cu)))
    rng = np.random.default_rng(6)
    for t in rng.choice(cu[-1], 60, replace=False).tolist() + [39, 40, 5039, 5040, 5041, cu[-1] - 1]:
        a = cu[np.searchsorted(cu, t, side="right") - 1]
        for h in (0, 7):
            kk, vv = k[a:t + 1, h // 4], v[a:t + 1, h // 4]
            s = kk @ q[t, h] / np.sqrt(128)
            p = np.exp(s - s.max())
            p /= p.sum()
            mass, want = p @ np.abs(vv), p @ vv
            b = 2.0 ** -8 if dt == "bf16" else 0
            score = 140 * U * (np.abs(kk) @ np.abs(q[t, h])).max() / np.sqrt(128) + 4 * U
            bound = (2 * score + (len(kk) / 32 + 64) * U + b) * mass + (b + U) * np.abs(want)
            assert np.all(np.abs(got[t, h] - want) <= bound), (t, h)


def test_attend_prompt_repeats_and_runs_on_another_stream():
    cu = ints([0, 700, 1500])
    x = [dev(a, torch.bfloat16) for a in make(1500, 28, 4, "bf16", 7)]
    first = S.saki_attend_prompt(*x, cu)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    other = S.saki_attend_prompt(*x, cu, stream=side)
    side.synchronize()
    assert torch.equal(first, other) and torch.equal(first, S.saki_attend_prompt(*x, cu))


def test_prompt_then_decode_steps():
    """Prompts through tables, rotation, prompt attention and the cache, then
    decode steps over that cache: the same attention to within the cache's
    8 bits."""
    rng = np.random.default_rng(8)
    H_q, H_kv, lens = 8, 2, [70, 1, 200]
    B, rows, n_blocks, dt = 3, 8, 24, "bf16"
    x = [dev(rng.standard_normal((n + 4, H_q + 2 * H_kv, 128)), DT[dt]) for n in lens]
    cache = (torch.zeros(n_blocks, H_kv, 64, 128, dtype=torch.float8_e4m3fn, device=DEV),
             torch.zeros(n_blocks, H_kv, 64, 128, dtype=torch.float8_e4m3fn, device=DEV),
             torch.zeros(n_blocks, H_kv, 2, device=DEV))
    free = ints(rng.permutation(n_blocks))
    tab = torch.full((B, rows), -1, dtype=torch.int32, device=DEV)
    ctx = ints([0] * B)
    for step in range(5):
        new = lens if step == 0 else [1] * B
        y = torch.cat([a[:n] if step == 0 else a[n + step - 1:n + step] for a, n in zip(x, lens)])
        T = y.shape[0]
        slots, pos = (torch.empty(T, dtype=torch.int32, device=DEV) for _ in range(2))
        tab, slots, pos, cu, ctx, counts = S.saki_block_tables(ctx, ints(new), free, tab, slots, pos)
        free = free[int(counts[0]):].contiguous()
        assert int(counts[1]) == 0
        q, k = S.saki_rope(y[:, :H_q], y[:, H_q:H_q + H_kv], pos)
        S.saki_cache_write(k, y[:, H_q + H_kv:], slots, *cache)
        if step == 0:
            S.saki_attend_prompt(q, k, y[:, H_q + H_kv:], cu)
            continue
        got = host(S.saki_cache_attend(q.view(B, H_q, 1, 128), *cache, tab, ctx))[:, :, 0]
        # the whole sequence so far as one prompt
        for b, n in enumerate(lens):
            z = x[b][:n + step]
            p = ints(range(n + step))
            qq, kk = S.saki_rope(z[:, :H_q].contiguous(), z[:, H_q:H_q + H_kv].contiguous(), p)
            vv = z[:, H_q + H_kv:]
            want = host(S.saki_attend_prompt(qq, kk, vv, ints([0, n + step])))[-1]
            # 8 bits: keys and values off by 2^-4 relative, and bf16 roundings
            s = np.einsum("hd,nhd->hn", np.abs(host(qq)[-1]), np.repeat(np.abs(host(kk)), 4, 1)) / np.sqrt(128)
            v_abs = np.abs(host(vv)).max()
            bound = (2 * 2.0 ** -4 * s.max(1, keepdims=True) + 2.0 ** -4 + 4 * 2.0 ** -8) * v_abs
            assert np.all(np.abs(got[b] - want) <= bound)
            # and on the whole much nearer: independent roundings average out
            assert np.linalg.norm(got[b] - want) <= 0.15 * np.linalg.norm(want)


@pytest.mark.parametrize("what", ["keys", "values", "queries", "zeros"])
def test_attend_prompt_f32_of_very_different_sizes(what):
    """Elements whose size changes by many powers of two from tile to tile (and
    tiles of zeros): each output against its own row's bound."""
    T = 230
    q, k, v = make(T, 4, 2, "f32", 11)
    g = 2.0 ** np.repeat(np.array([0, 30, -30, 5, -60, 12, 0, -3]), 32)[:T, None, None]
    if what == "keys":
        k, q = rounded(k / np.maximum(g, 1), "f32"), q
    elif what == "values":
        v = rounded(v * g, "f32")
    elif what == "queries":
        q = rounded(q * np.minimum(g, 8), "f32")
    else:
        v[:70] = 0
        k[64:128] = 0
        q[5] = 0
        q[100] *= 2.0 ** -100
    cu = np.array([0, T])
    out = S.saki_attend_prompt(dev(q), dev(k), dev(v), ints(cu))
    # two fp16 parts: 2^-21 of a product and 2^-38 of a tile's largest element more
    want, mass, size = O.prompt_attend(q, k, v, cu)
    score = ((140 * U + 2.0 ** -21) * size + 4 * U)[..., None]
    top = np.maximum.accumulate(np.abs(v).max(-1), 0).repeat(2, 1)[..., None]
    nxt = np.pad(np.abs(v).max(-1), ((0, 31), (0, 0)))
    nxt = np.stack([nxt[i:i + T] for i in range(32)]).max(0).repeat(2, 1)[..., None]  # a tile's later values
    bound = (2 * score + (T / 32 + 64) * U + 2.0 ** -21) * mass + 2.0 ** -37 * T * np.maximum(top, nxt) + U * np.abs(want)
    err = np.abs(host(out) - want)
    assert np.all(err <= bound), np.max(err / bound)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_attend_prompt_rows_far_apart(dt):
    """Token rows 2^22 elements apart: offsets of more than 4 GiB."""
    T, H_q, H_kv = 600, 2, 1
    q, k, v = make(T, H_q, H_kv, dt, 13)
    cu = np.array([0, 20, T])
    big = torch.empty(T * (1 << 22), dtype=DT[dt], device=DEV)
    far = []
    for i, x in enumerate((q, k, v)):
        t = big.as_strided(x.shape, (1 << 22, 128, 1), 512 * i)
        t.copy_(dev(x, DT[dt]))
        far.append(t)
    out = S.saki_attend_prompt(*far, ints(cu))
    assert torch.equal(out, S.saki_attend_prompt(*(dev(x, DT[dt]) for x in (q, k, v)), ints(cu)))
    check(out, q, k, v, cu, dt)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_attend_prompt_captured_and_replayed(dt):
    """In a graph, replayed with other offsets and inputs and eager work between."""
    T, H_q, H_kv = 400, 8, 2
    q, k, v = (dev(x, DT[dt]) for x in make(T, H_q, H_kv, dt, 14))
    cu, out = ints([0, 100, 400]), torch.zeros(T, H_q, 128, dtype=DT[dt], device=DEV)
    ws = torch.empty(S.saki_attend_prompt_workspace_bytes(dt, T, 2, H_kv), dtype=torch.uint8, device=DEV)
    S.saki_attend_prompt(q, k, v, cu, out=out, ws=ws)
    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        S.saki_attend_prompt(q, k, v, cu, out=out, ws=ws)
    rng = np.random.default_rng(15)
    for i in range(5):
        for t in (q, k, v):
            t.copy_(dev(rng.standard_normal(t.shape), DT[dt]))
        cu.copy_(ints([0, int(rng.integers(0, 400)), 400]))
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, S.saki_attend_prompt(q, k, v, cu)), i
