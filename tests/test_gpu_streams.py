"""Calls on a stream that is not the current one: the tensors and workspaces that
they make come from that stream's memory."""
import pytest

torch = pytest.importorskip("torch")
S = pytest.importorskip("paper_2608_03228_amd.saki")

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F8 = torch.float8_e4m3fn


@pytest.fixture
def made(monkeypatch):
    """Keeps what torch.empty makes."""
    kept, empty = [], torch.empty
    monkeypatch.setattr(torch, "empty", lambda *a, **k: kept.append(empty(*a, **k)) or kept[-1])
    return kept


def pool_of(t):
    """The stream from whose memory the tensor was taken."""
    p = t.data_ptr()
    return next(s["stream"] for s in torch.cuda.memory_snapshot()
                if s["address"] <= p < s["address"] + s["total_size"])


def zeros(*shape, dtype=torch.float32):
    return torch.zeros(shape, dtype=dtype, device=DEV)


def check_pools(made, call, n):
    torch.cuda.synchronize()
    del made[:]
    side = torch.cuda.Stream()
    call(side)
    side.synchronize()
    assert len(made) == n
    assert [pool_of(t) for t in made] == [side.cuda_stream] * n
    del made[:]
    call(None)
    assert [pool_of(t) for t in made] == [torch.cuda.current_stream().cuda_stream] * n


i32 = dict(dtype=torch.int32)
SERVING = {
    # name: arguments, keywords, tensors that the call makes
    "rope": lambda: (S.saki_rope, (zeros(5, 4, 128), zeros(5, 2, 128), zeros(5, **i32)), {}, 2),
    "tables": lambda: (S.saki_block_tables, (zeros(2, **i32), zeros(2, **i32), zeros(9, **i32), zeros(2, 3, **i32),
                                             zeros(4, **i32), zeros(4, **i32)), {}, 3),
    # wide tables: an output and a workspace
    "attend": lambda: (S.saki_cache_attend, (zeros(1, 4, 1, 128), zeros(2, 2, 64, 128, dtype=F8),
                                             zeros(2, 2, 64, 128, dtype=F8), zeros(2, 2, 2), zeros(1, 100, **i32),
                                             zeros(1, **i32) + 70), {}, 2),
    "prompt": lambda: (S.saki_attend_prompt, (zeros(9, 4, 128), zeros(9, 2, 128), zeros(9, 2, 128),
                                              torch.tensor([0, 9], device=DEV, **i32)), {}, 2),
}


@pytest.mark.parametrize("name", SERVING)
def test_serving_calls(name, made):
    f, args, kw, n = SERVING[name]()
    check_pools(made, lambda stream: f(*args, **kw, stream=stream), n)


def index_of(keys, B_k, mu):
    return S.saki_build_index(keys, B_k, mu, 16, "bf16", 4)


def index_arrays():
    """keys, factors and mean of one sequence, 4 / 2 heads, 200 keys, r = 16."""
    g = torch.Generator(DEV).manual_seed(1)
    keys, B_k, mu, q = (torch.randn(s, generator=g, device=DEV)
                        for s in ((1, 2, 200, 128), (4, 128, 16), (2, 128), (1, 4, 1, 128)))
    return keys, B_k, mu, q, torch.zeros(1, 4, 1, 8, device=DEV, **i32)


INDEX = {
    "moments": lambda k, b, mu, q, li: (S.saki_calibration_moments, (zeros(4, 64, 128), zeros(2, 64, 128)), {}, 3),
    "build": lambda k, b, mu, q, li: (S.saki_build_index, (k, b, mu, 16, "bf16", 4), {}, 1),
    "export": lambda k, b, mu, q, li: (S.saki_index_export, (index_of(k, b, mu), "bf16", 1, 4, 200, 16), {}, 1),
    "score": lambda k, b, mu, q, li: (S.saki_score_topk, (index_of(k, b, mu), "bf16", q, b, mu, 2, 200, 200, 16),
                                      dict(k=8), 3),
    "recall": lambda k, b, mu, q, li: (S.saki_recall, (k, q, li, 200), dict(k=8), 3),
    "attend": lambda k, b, mu, q, li: (S.saki_attend, (k, q, li, 200), dict(keys=k), 1),
}


@pytest.mark.parametrize("name", INDEX)
def test_index_calls(name, made):
    f, args, kw, n = INDEX[name](*index_arrays())
    check_pools(made, lambda stream: f(*args, **kw, stream=stream), n)
