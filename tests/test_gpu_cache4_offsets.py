"""Chunks over the 4-bit cache that hold the first T of a step's tokens, as a step of
a fixed size does when saki_block_tables counted more: offsets go on past T, and
the tokens stand where they do in the whole.  Bounds of test_gpu_cache4.py."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
S = pytest.importorskip("paper_2608_03228_amd.saki")

from tests.cache4_rows import check_rows, chunk_case, picked, run  # noqa: E402
from tests.test_gpu_cache4 import DT, host, ints, on_gpu, random_cache, values  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("width", [None, 400])
@pytest.mark.parametrize("T", [130, 75, 40])
def test_offsets_past_the_tokens(T, width, dt):
    q, cache, tab, lens, cu = chunk_case([90, 33, 150], [40, 80, 20], 4, 2, dt, width)
    whole = run((q, cache, tab, lens, cu), dt)
    part = (q[:T], cache, tab, lens, cu)
    got = run(part, dt)
    rows = [(b, i, h) for b, i, h in picked([40, 80, 20], 2, 4, np.random.default_rng(0)) if cu[b] + i < T]
    check_rows(part, dt, got, rows)
    # every row: values are 3 at most, so that each side is off by 2^-8 (3 + 3) and little more
    np.testing.assert_allclose(got, whole[:T], rtol=0, atol=0.06)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_offsets_past_the_tokens_read_back_and_attended(dt):
    """What saki_block_tables gives for more tokens than the step holds."""
    rng = np.random.default_rng(5)
    ctx, new, T = [70, 10], [30, 50], 60
    cache, tab = random_cache(8, 2, rng), ints(np.full((2, 4), -1))
    tab[0, :2], tab[1, 0] = ints([6, 1]), 3
    slots, pos = ints([0] * T), ints([0] * T)
    _, _, _, cu, lens, _ = S.saki_block_tables(ints(ctx), ints(new), ints([5, 0, 2, 4, 7]), tab, slots, pos)
    assert host(cu).tolist() == [0, 30, 80]
    gpu = on_gpu(cache)
    q = rng.standard_normal((T, 4, 128))
    q = torch.from_numpy(q).to("cuda:0", DT[dt])
    out = host(S.saki_cache4_prompt(q, *gpu, tab, lens, cu))
    case = (host(q), cache, host(tab), host(lens), np.array([0, 30, 80]))
    assert host(pos)[59] == 10 + 29
    check_rows(case, dt, out, [(1, i, h) for i in (0, 1, 28, 29) for h in range(4)] + [(0, 29, 0), (0, 0, 3)])
    k = torch.zeros(T, 2, 128, device="cuda:0")
    S.saki_cache4_read(*gpu, tab, cu, k, None, starts=ints(ctx))
    vals = values(cache)[0]
    for t in (0, 29, 30, 59):
        b, p = int(t >= 30), int(host(pos)[t])
        np.testing.assert_array_equal(host(k)[t], vals[host(tab)[b, p // 64], :, p % 64])
