"""CPU tests of what the entry points of the 4-bit cache refuse: nothing is launched."""
import ctypes as C

import pytest

S = pytest.importorskip("paper_2608_03228_amd.saki")
torch = pytest.importorskip("torch")

ARG, UNSUP, WS = -1, -2, -3
P = C.c_void_p(4096)     # never followed
ODD = C.c_void_p(4104)   # not on a 16-byte boundary
K, V, SC = C.c_void_p(0x100000), C.c_void_p(0x200000), C.c_void_p(0x300000)


@pytest.fixture(scope="module")
def lib():
    return S.lib()


def change(f, good, names, **kw):
    args = dict(zip(names, good))
    assert set(kw) <= set(args)
    args.update(kw)
    return f(*args.values())


WRITE = "k v dtype T H_kv d ld_k ld_v slots k_cache v_cache scales n_blocks stream".split()


@pytest.mark.parametrize("kw,status", [
    (dict(T=0), 0), (dict(n_blocks=0), 0), (dict(T=-1), ARG), (dict(H_kv=0), ARG), (dict(n_blocks=-1), ARG),
    (dict(d=0), ARG), (dict(d=64), UNSUP), (dict(dtype=2), UNSUP), (dict(T=(1 << 26) + 1), UNSUP),
    (dict(n_blocks=1 << 24), UNSUP), (dict(k=None), ARG), (dict(v=ODD), ARG), (dict(slots=None), ARG),
    (dict(k_cache=None), ARG), (dict(v_cache=ODD), ARG), (dict(scales=None), ARG), (dict(scales=ODD), ARG),
    (dict(ld_k=255), ARG), (dict(ld_v=260), ARG),
    # caches that overlap each other or their scales: 9 blocks of 2 heads are 0x12000 bytes, their scales 0x2400
    (dict(v_cache=K), ARG), (dict(v_cache=C.c_void_p(0x111ff0)), ARG), (dict(scales=C.c_void_p(0x100010)), ARG),
    (dict(scales=C.c_void_p(0x1fdc10)), ARG),
])
def test_write(lib, kw, status):
    good = [P, P, 1, 5, 2, 128, 256, 256, P, K, V, SC, 9, None]
    assert change(lib.saki_cache4_write, good, WRITE, **kw) == status


READ = ("k_cache v_cache scales n_blocks tables max_blocks starts cu B T H_kv d dtype k_out v_out ld_k ld_v "
        "stream").split()


@pytest.mark.parametrize("kw,status", [
    (dict(T=0), 0), (dict(B=0), 0), (dict(k_out=None, v_out=None), 0), (dict(T=-1), ARG), (dict(B=-1), ARG),
    (dict(d=0), ARG), (dict(max_blocks=0), ARG), (dict(H_kv=0), ARG), (dict(n_blocks=-1), ARG),
    (dict(d=256), UNSUP), (dict(dtype=2), UNSUP), (dict(T=(1 << 26) + 1), UNSUP), (dict(max_blocks=1 << 25), UNSUP),
    (dict(n_blocks=1 << 24), UNSUP), (dict(tables=None), ARG), (dict(cu=None), ARG), (dict(k_out=ODD), ARG),
    (dict(v_out=ODD), ARG), (dict(ld_k=255), ARG), (dict(ld_v=260), ARG), (dict(k_cache=None), ARG),
    (dict(v_cache=ODD), ARG), (dict(scales=ODD), ARG),
])
def test_read(lib, kw, status):
    good = [K, V, SC, 9, P, 4, None, P, 2, 5, 2, 128, 1, P, P, 256, 256, None]
    assert change(lib.saki_cache4_read, good, READ, **kw) == status


ATTEND = ("q dtype B H_q H_kv Q d k_cache v_cache scales n_blocks tables max_blocks lens top_idx k out ws ws_bytes "
          "stream").split()


@pytest.mark.parametrize("kw,status", [
    (dict(Q=0), 0), (dict(B=0), ARG), (dict(H_q=5), ARG), (dict(H_q=0), ARG), (dict(H_kv=0), ARG), (dict(Q=-1), ARG),
    (dict(Q=17), UNSUP), (dict(d=64), UNSUP), (dict(dtype=2), UNSUP), (dict(max_blocks=0), ARG),
    (dict(max_blocks=1 << 25), UNSUP), (dict(n_blocks=-1), ARG), (dict(n_blocks=1 << 24), UNSUP), (dict(k=3), ARG),
    (dict(top_idx=P), ARG), (dict(top_idx=P, k=65), UNSUP), (dict(k=-1), ARG), (dict(q=None), ARG), (dict(q=ODD), ARG),
    (dict(out=None), ARG), (dict(out=ODD), ARG), (dict(tables=None), ARG), (dict(lens=None), ARG),
    (dict(k_cache=None), ARG), (dict(scales=ODD), ARG), (dict(ws=None), WS), (dict(ws_bytes=100), WS),
    (dict(ws=ODD), WS), (dict(B=1 << 22), UNSUP),
])
def test_attend(lib, kw, status):
    need = lib.saki_cache4_attend_workspace_bytes(2, 4, 2, 1, 100, 0)
    assert need > 256
    good = [P, 1, 2, 4, 2, 1, 128, K, V, SC, 9, P, 100, P, None, 0, P, P, need, None]
    assert change(lib.saki_cache4_attend, good, ATTEND, **kw) == status


PROMPT = ("q dtype T B H_q H_kv d ld_q k_cache v_cache scales n_blocks tables max_blocks lens cu out ws ws_bytes "
          "stream").split()


@pytest.mark.parametrize("kw,status", [
    (dict(T=0), 0), (dict(B=0), 0), (dict(T=-1), ARG), (dict(B=-1), ARG), (dict(H_q=5), ARG), (dict(H_kv=0), ARG),
    (dict(d=0), ARG), (dict(d=64), UNSUP), (dict(dtype=2), UNSUP), (dict(max_blocks=0), ARG),
    (dict(max_blocks=1 << 25), UNSUP), (dict(n_blocks=-1), ARG), (dict(T=(1 << 26) + 1), UNSUP), (dict(q=None), ARG),
    (dict(q=ODD), ARG), (dict(ld_q=511), ARG), (dict(out=None), ARG), (dict(out=ODD), ARG), (dict(tables=None), ARG),
    (dict(lens=None), ARG), (dict(cu=None), ARG), (dict(k_cache=None), ARG), (dict(v_cache=ODD), ARG),
    (dict(scales=ODD), ARG), (dict(ws=None), WS), (dict(ws=ODD), WS), (dict(ws_bytes=100), WS),
])
def test_prompt(lib, kw, status):
    need = lib.saki_cache4_prompt_workspace_bytes(1, 5, 2, 4, 2, 100)
    assert need > 256
    good = [P, 1, 5, 2, 4, 2, 128, 512, K, V, SC, 9, P, 100, P, P, P, P, need, None]
    assert change(lib.saki_cache4_prompt, good, PROMPT, **kw) == status


def test_workspace_sizes(lib):
    assert lib.saki_cache4_attend_workspace_bytes(1, 4, 3, 1, 100, 0) == 0
    assert lib.saki_cache4_attend_workspace_bytes(1, 4, 2, 1, 100, 64) == 256
    assert 256 < lib.saki_cache4_attend_workspace_bytes(64, 32, 8, 1, 1 << 20, 0) <= 32 << 20
    assert lib.saki_cache4_prompt_workspace_bytes(1, 5, 2, 4, 3, 100) == 0
    assert lib.saki_cache4_prompt_workspace_bytes(2, 5, 2, 4, 2, 100) == 0
    assert lib.saki_cache4_prompt_workspace_bytes(1, 0, 2, 4, 2, 100) == 256
    assert lib.saki_cache4_prompt_workspace_bytes(0, 1 << 20, 2, 4, 2, 100) == 256
    # bounded, whatever the table's width
    assert lib.saki_cache4_prompt_workspace_bytes(1, 1, 1, 32, 8, 1 << 24) <= 128 << 20


@pytest.mark.parametrize("call", [
    lambda c: S.saki_cache4_write(torch.zeros(3, 2, 128), torch.zeros(3, 2, 128), torch.zeros(3, dtype=torch.int32), *c),
    lambda c: S.saki_cache4_read(*c, torch.zeros(1, 1, dtype=torch.int32), torch.zeros(2, dtype=torch.int32),
                                 torch.zeros(3, 2, 128), None),
    lambda c: S.saki_cache4_attend(torch.zeros(1, 4, 1, 128), *c, torch.zeros(1, 1, dtype=torch.int32),
                                   torch.zeros(1, dtype=torch.int32)),
    lambda c: S.saki_cache4_prompt(torch.zeros(3, 4, 128), *c, torch.zeros(1, 1, dtype=torch.int32),
                                   torch.zeros(1, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)),
])
def test_host_tensors_are_refused(call):
    cache = (torch.zeros(2, 2, 64, 64, dtype=torch.uint8), torch.zeros(2, 2, 64, 64, dtype=torch.uint8),
             torch.zeros(2, 2, 2, 64, 4, dtype=torch.uint8))
    with pytest.raises(ValueError, match="CUDA"):
        call(cache)
