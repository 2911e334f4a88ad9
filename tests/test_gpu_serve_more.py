"""Serving calls at the ends of what they take."""
import numpy as np
import pytest

from tests.test_gpu_serve import DT, attend_case, dev, host, ints

torch = pytest.importorskip("torch")
S = pytest.importorskip("paper_2608_03228_amd.saki")

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("rows", [None, 70])
def test_cache_attend_lists_of_nothing(rows, dt):
    """Lists of no entry leave every row without a key: zeros, on any stream."""
    lens = [300, 0, 5]
    q, _, _, (k, v, s), tab = attend_case(lens, 4, 2, 2, dt, rows)
    args = (dev(q, DT[dt]), k, v, s, ints(tab), ints(lens))
    idx = torch.empty(3, 4, 2, 0, dtype=torch.int32, device=DEV)
    assert np.all(host(S.saki_cache_attend(*args, top_idx=idx)) == 0)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    out = torch.full_like(args[0], 7.0)
    side.wait_stream(torch.cuda.current_stream())
    S.saki_cache_attend(*args, top_idx=idx, out=out, stream=side)
    side.synchronize()
    assert np.all(host(out) == 0)
    with pytest.raises(ValueError):
        S.saki_cache_attend(*args, top_idx=idx[:2])


def test_rope_of_the_most_tokens():
    """2^26 - 4 tokens of one bf16 head (16 GiB), in place: sampled ones as in a
    call of their own."""
    T = (1 << 26) - 4
    x = torch.zeros(T, 1, 128, dtype=torch.bfloat16, device=DEV)
    pos = torch.arange(T, dtype=torch.int32, device=DEV)
    at = torch.tensor([0, 1, 12345678, T // 2, T - 2, T - 1], device=DEV)
    y = torch.randn(6, 1, 128, generator=torch.Generator(DEV).manual_seed(3), device=DEV).bfloat16()
    x[at] = y
    S.saki_rope(x, None, pos, q_out=x)
    assert torch.equal(x[at], S.saki_rope(y, None, pos[at])[0])
    x[at] = 0
    assert not x.any()


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_rope_of_keys_alone(dt):
    """Keys without queries, as the C entry point takes them."""
    x = torch.randn(9, 3, 128, generator=torch.Generator(DEV).manual_seed(4), device=DEV).to(DT[dt])
    pos = ints(range(100, 109))
    want, _ = S.saki_rope(x, None, pos)
    q, k = S.saki_rope(None, x, pos)
    assert q is None and torch.equal(k, want)
    out = torch.empty_like(x)
    assert S.saki_rope(None, x, pos, k_out=out)[1] is out and torch.equal(out, want)
    with pytest.raises(ValueError):
        S.saki_rope(None, None, pos)
