"""CPU tests of what the serving entry points refuse: nothing is launched."""
import ctypes as C

import pytest

S = pytest.importorskip("paper_2608_03228_amd.saki")
torch = pytest.importorskip("torch")

ARG, UNSUP, WS = -1, -2, -3
P = C.c_void_p(4096)     # never followed
ODD = C.c_void_p(4104)   # not on a 16-byte boundary


@pytest.fixture(scope="module")
def lib():
    return S.lib()


def change(f, good, names, **kw):
    args = dict(zip(names, good))
    args.update(kw)
    return f(*args.values())


ROPE = "q k dtype T H_q H_kv d ld_q ld_k pos axes sections theta inverse q_out k_out ld_qo ld_ko stream".split()


@pytest.mark.parametrize("kw,status", [
    (dict(T=0), 0), (dict(H_q=0, H_kv=0), 0), (dict(T=-1), ARG), (dict(H_q=-1), ARG), (dict(d=0), ARG),
    (dict(d=64), UNSUP), (dict(dtype=2), UNSUP), (dict(axes=0), UNSUP), (dict(axes=4), UNSUP),
    (dict(T=(1 << 26) + 1), UNSUP), (dict(theta=0.0), ARG), (dict(theta=float("nan")), ARG),
    (dict(theta=float("inf")), ARG), (dict(sections=(C.c_int * 3)(16, 24, 23)), ARG),
    (dict(sections=(C.c_int * 3)(-1, 41, 24)), ARG), (dict(sections=(C.c_int * 3)(65, -1, 0)), ARG),
    (dict(sections=None), ARG), (dict(pos=None), ARG), (dict(q=None), ARG), (dict(k=None), ARG),
    (dict(q_out=None), ARG), (dict(q=ODD), ARG), (dict(k_out=ODD), ARG), (dict(ld_q=4 * 128 - 8), ARG),
    (dict(ld_k=257), ARG), (dict(ld_qo=4 * 128 + 4), ARG), (dict(ld_ko=1 << 62), ARG),
])
def test_rope(lib, kw, status):
    good = [P, P, 1, 5, 4, 2, 128, 512, 256, P, 3, (C.c_int * 3)(16, 24, 24), 1e4, 0, P, P, 512, 256, None]
    assert change(lib.saki_rope, good, ROPE, **kw) == status


A = [C.c_void_p(0x1000 * (i + 1)) for i in range(9)]  # arrays apart from one another
TABLES = "ctx new B free n_free tables max_blocks slots pos T cu lens counts stream".split()


@pytest.mark.parametrize("kw,status", [
    (dict(B=0), ARG), (dict(n_free=-1), ARG), (dict(max_blocks=0), ARG), (dict(T=-1), ARG), (dict(ctx=None), ARG),
    (dict(new=None), ARG), (dict(free=None), ARG), (dict(tables=None), ARG), (dict(slots=None), ARG),
    (dict(pos=None), ARG), (dict(cu=None), ARG), (dict(lens=None), ARG), (dict(counts=None), ARG),
    (dict(max_blocks=1 << 25), UNSUP),
    # outputs that overlap inputs: the lengths updated in place, a part of the free list
    (dict(lens=A[0]), ARG), (dict(lens=A[1]), ARG), (dict(cu=C.c_void_p(0x1000 - 8)), ARG),
    (dict(slots=C.c_void_p(0x3000 + 32)), ARG), (dict(tables=C.c_void_p(0x3000 - 28)), ARG), (dict(counts=A[0]), ARG),
])
def test_block_tables(lib, kw, status):
    good = [A[0], A[1], 2, A[2], 9, A[3], 4, A[4], A[5], 7, A[6], A[7], A[8], None]
    assert change(lib.saki_block_tables, good, TABLES, **kw) == status


WRITE = "k v dtype T H_kv d ld_k ld_v slots k_cache v_cache scales n_blocks stream".split()


@pytest.mark.parametrize("kw,status", [
    (dict(T=0), 0), (dict(n_blocks=0), 0), (dict(T=-1), ARG), (dict(H_kv=0), ARG), (dict(n_blocks=-1), ARG),
    (dict(d=0), ARG), (dict(d=64), UNSUP), (dict(dtype=2), UNSUP), (dict(T=(1 << 26) + 1), UNSUP),
    (dict(n_blocks=1 << 24), UNSUP), (dict(k=None), ARG), (dict(v=ODD), ARG), (dict(slots=None), ARG),
    (dict(k_cache=None), ARG), (dict(v_cache=ODD), ARG), (dict(scales=None), ARG), (dict(scales=C.c_void_p(4100)), ARG),
    (dict(ld_k=255), ARG), (dict(ld_v=260), ARG),
    # caches that overlap each other or their scales: 9 blocks of 2 heads are 0x24000 bytes
    (dict(v_cache=C.c_void_p(0x100000)), ARG), (dict(v_cache=C.c_void_p(0x123ff0)), ARG),
    (dict(scales=C.c_void_p(0x100010)), ARG), (dict(scales=C.c_void_p(0x1fff78)), ARG),
])
def test_cache_write(lib, kw, status):
    good = [P, P, 1, 5, 2, 128, 256, 256, P, C.c_void_p(0x100000), C.c_void_p(0x200000), C.c_void_p(0x300000), 9, None]
    assert change(lib.saki_cache_write, good, WRITE, **kw) == status


ATTEND = ("q dtype B H_q H_kv Q d k_cache v_cache scales n_blocks tables max_blocks lens top_idx k out ws ws_bytes "
          "stream").split()


@pytest.mark.parametrize("kw,status", [
    (dict(Q=0), 0), (dict(B=0), ARG), (dict(H_q=3), ARG), (dict(H_kv=0), ARG), (dict(Q=-1), ARG), (dict(Q=17), UNSUP),
    (dict(d=64), UNSUP), (dict(dtype=2), UNSUP), (dict(max_blocks=0), ARG), (dict(max_blocks=1 << 25), UNSUP),
    (dict(n_blocks=-1), ARG), (dict(n_blocks=1 << 25), UNSUP), (dict(q=None), ARG), (dict(q=ODD), ARG),
    (dict(out=None), ARG), (dict(out=ODD), ARG), (dict(tables=None), ARG), (dict(lens=None), ARG),
    (dict(k_cache=None), ARG), (dict(scales=None), ARG), (dict(top_idx=P), ARG), (dict(k=4), ARG), (dict(k=-1), ARG),
    (dict(top_idx=P, k=65), UNSUP), (dict(ws=None), WS), (dict(ws_bytes=100), WS), (dict(ws=ODD), WS),
    (dict(B=1 << 23), UNSUP), (dict(B=1 << 24, top_idx=P, k=4), UNSUP),
])
def test_cache_attend(lib, kw, status):
    good = [P, 1, 2, 4, 2, 1, 128, P, P, P, 9, P, 80, P, None, 0, P, P, 1 << 30, None]
    assert change(lib.saki_cache_attend, good, ATTEND, **kw) == status


def test_cache_attend_workspace():
    f = S.saki_cache_attend_workspace_bytes
    assert f(1, 4, 1, 1, 1) > 0 and f(1, 4, 1, 1, 1) <= f(8, 4, 1, 1, 2048) == f(64, 32, 8, 16, 1 << 24)
    assert f(64, 32, 8, 16, 1 << 24) <= 8.6e6 and f(2, 4, 2, 1, 8, 64) == 256
    for bad in ((0, 4, 1, 1, 1), (1, 3, 2, 1, 1), (1, 4, 1, 17, 1), (1, 4, 1, 1, 0), (1, 4, 1, -1, 1)):
        assert f(*bad) == 0
    assert f(1, 4, 1, 1, 1, 65) == 0


def test_cache_attend_workspace_of_more_pairs_than_an_int_holds():
    f = S.saki_cache_attend_workspace_bytes
    assert f(1 << 20, 4096, 4096, 1, 20) == f(1 << 19, 4096, 4096, 1, 20) == f(1 << 19, 4, 4, 1, 20) == 256


PROMPT = "q k v dtype T B H_q H_kv d ld_q ld_k ld_v cu out ws ws_bytes stream".split()


@pytest.mark.parametrize("kw,status", [
    (dict(T=0), 0), (dict(B=0), 0), (dict(T=-1), ARG), (dict(B=-1), ARG), (dict(H_q=3), ARG), (dict(H_kv=0), ARG),
    (dict(d=0), ARG), (dict(d=64), UNSUP), (dict(dtype=2), UNSUP), (dict(T=1 << 30), UNSUP),
    (dict(B=1 << 30), UNSUP), (dict(q=None), ARG), (dict(k=ODD), ARG), (dict(v=None), ARG), (dict(out=None), ARG),
    (dict(out=ODD), ARG), (dict(cu=None), ARG), (dict(ld_q=511), ARG), (dict(ld_k=128), ARG), (dict(ld_v=260), ARG), (dict(ld_q=(1 << 22) + 8), UNSUP),
    (dict(ws=None, dtype=0), WS), (dict(ws_bytes=1000, dtype=0), WS), (dict(ws=ODD, dtype=0), WS),
])
def test_attend_prompt(lib, kw, status):
    good = [P, P, P, 1, 5, 2, 4, 2, 128, 512, 256, 256, P, P, P, 1 << 30, None]
    assert change(lib.saki_attend_prompt, good, PROMPT, **kw) == status


def test_attend_prompt_workspace():
    f = S.saki_attend_prompt_workspace_bytes
    assert f("bf16", 1 << 20, 9, 8) == 256 and f("f32", 0, 1, 8) == 256
    # at least the parts of every token's keys and values, at most two tiles a prompt more
    assert 4 * 2 * 1000 * 3 * 128 <= f("f32", 1000, 5, 3) <= 4 * 2 * (1000 + 64 * 5 + 32) * 3 * 128
    assert f("f32", -1, 1, 1) == f("f32", 1, -1, 1) == f("f32", 1, 1, 0) == f("fp8", 1, 1, 1) == 0


def test_binding_refuses_host_tensors():
    x = torch.zeros(2, 4, 128)
    i = torch.zeros(2, dtype=torch.int32)
    c = torch.zeros(1, 4, 64, 128, dtype=torch.float8_e4m3fn)
    s = torch.zeros(1, 4, 2)
    with pytest.raises(ValueError):
        S.saki_rope(x, x, i)
    with pytest.raises(ValueError):
        S.saki_block_tables(i, i, i, torch.zeros(2, 3, dtype=torch.int32), i, i)
    with pytest.raises(ValueError):
        S.saki_cache_write(x, x, i, c, c, s)
    with pytest.raises(ValueError):
        S.saki_cache_attend(torch.zeros(1, 4, 1, 128), c, c, s, i[None], i[:1])
    with pytest.raises(ValueError):
        S.saki_attend_prompt(x, x, x, i)


def test_argument_module_checks_counts_and_ranges():
    m = S._args()
    with pytest.raises(TypeError):
        m.saki_block_tables(1, 2)
    with pytest.raises(OverflowError):
        m.saki_cache_attend_workspace_bytes(1 << 40, 4, 1, 1, 1, 0)
    with pytest.raises(OverflowError):
        m.saki_rope(0, 0, 1, 5, 4, 2, 128, -1, 256, 0, 1, 0, 1e4, 0, 0, 0, 512, 256, None)
    with pytest.raises(TypeError):
        m.saki_cache_attend_workspace_bytes("1", 4, 1, 1, 1, 0)
    assert m.saki_cache_attend_workspace_bytes(1, 4, 1, 1, 100, 0) == S.saki_cache_attend_workspace_bytes(1, 4, 1, 1, 100)
    x = torch.zeros(2, 3)
    for f in (m.array, m.rows):
        with pytest.raises(ValueError, match="must be a CUDA"):
            f(x, torch.float32, (2, 3), 0, "x")
        with pytest.raises(ValueError, match="must be a CUDA"):
            f(None, torch.float32, (2, 3), 0, "x")
        with pytest.raises(TypeError):
            f(x, torch.float32)


def test_rope_takes_the_tokens_that_a_launch_holds(lib):
    """A work-group of 256 takes four tokens, and a launch has fewer than 2^32
    threads: 2^26 - 4 tokens pass (the next check refuses them), one more do not."""
    good = [P, P, 1, 5, 4, 2, 128, 512, 256, None, 3, (C.c_int * 3)(16, 24, 24), 1e4, 0, P, P, 512, 256, None]
    most = (1 << 26) - 4
    assert (most + 3) // 4 * 256 < 1 << 32 <= (most + 4) // 4 * 256
    assert change(lib.saki_rope, good, ROPE, T=most) == ARG
    assert change(lib.saki_rope, good, ROPE, T=most + 1) == UNSUP
