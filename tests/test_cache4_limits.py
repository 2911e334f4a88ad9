"""CPU tests of the largest sizes that the 4-bit cache's entry points take: one more
is refused as unsupported, before anything is launched or read.  Sizes at a limit are
shown to be taken by the refusal that comes after it (a missing pointer)."""
import pytest

from tests.test_cache4_refusals import (  # noqa: F401  (lib: a fixture)
    ARG, ATTEND, K, P, PROMPT, READ, SC, UNSUP, V, WRITE, change, lib)


@pytest.mark.parametrize("kw,status", [
    (dict(T=1 << 26), ARG), (dict(T=(1 << 26) + 1), UNSUP), (dict(H_kv=32767, ld_k=32767 * 128, ld_v=32767 * 128), ARG),
    (dict(H_kv=32768, ld_k=32768 * 128, ld_v=32768 * 128), UNSUP), (dict(n_blocks=(1 << 24) - 1), ARG),
    (dict(n_blocks=1 << 24), UNSUP),
])
def test_write(lib, kw, status):  # noqa: F811
    good = [P, P, 1, 5, 2, 128, 256, 256, None, K, V, SC, 9, None]
    assert change(lib.saki_cache4_write, good, WRITE, **kw) == status


@pytest.mark.parametrize("kw,status", [
    (dict(T=1 << 26), ARG), (dict(T=(1 << 26) + 1), UNSUP), (dict(max_blocks=(1 << 25) - 2), ARG),
    (dict(max_blocks=(1 << 25) - 1), UNSUP), (dict(H_kv=32768), UNSUP), (dict(n_blocks=1 << 24), UNSUP),
])
def test_read(lib, kw, status):  # noqa: F811
    good = [K, V, SC, 9, P, 4, None, None, 2, 5, 2, 128, 1, P, P, 256, 256, None]
    assert change(lib.saki_cache4_read, good, READ, **kw) == status


@pytest.mark.parametrize("kw,status", [
    (dict(B=1 << 21), ARG), (dict(B=(1 << 21) + 1), UNSUP),                            # 2^22 groups of rows
    (dict(B=1 << 17, Q=16, H_q=16), ARG), (dict(B=(1 << 17) + 1, Q=16, H_q=16), UNSUP),  # 2^25 rows
    (dict(B=1 << 21, Q=4, H_q=4), ARG), (dict(B=1 << 20, Q=8, H_q=6), UNSUP),
    (dict(max_blocks=(1 << 25) - 2), ARG), (dict(max_blocks=(1 << 25) - 1), UNSUP),
    (dict(H_q=32768, H_kv=32768), UNSUP), (dict(n_blocks=1 << 24), UNSUP),
])
@pytest.mark.parametrize("k", [0, 64])
def test_attend(lib, k, kw, status):  # noqa: F811
    good = [P, 1, 2, 4, 2, 1, 128, K, V, SC, 9, P, 100, None, P if k else None, k, P, P, 1 << 40, None]
    assert change(lib.saki_cache4_attend, good, ATTEND, **kw) == status


@pytest.mark.parametrize("kw,status", [
    (dict(T=1 << 26), ARG), (dict(T=(1 << 26) + 1), UNSUP),
    (dict(H_q=65535, H_kv=1, ld_q=65535 * 128), ARG), (dict(H_q=65536, H_kv=2, ld_q=65536 * 128), UNSUP),
    (dict(T=(1 << 30) // 64 - 1, H_q=64, H_kv=1, ld_q=8192, B=1), UNSUP),              # T G = 2^30 - 64
    (dict(T=(1 << 22) - 1, H_q=128, H_kv=1, ld_q=16384, B=1), ARG),                    # (T G / 128 + B) H_kv = 2^22
    (dict(T=(1 << 22) - 1, H_q=128, H_kv=1, ld_q=16384, B=2), UNSUP),
    (dict(T=1 << 22, H_q=128, H_kv=1, ld_q=16384, B=1), UNSUP),
    (dict(B=(1 << 21) - 1), ARG), (dict(B=1 << 21), ARG), (dict(B=(1 << 21) + 1), UNSUP),
    (dict(max_blocks=(1 << 25) - 2), ARG), (dict(max_blocks=(1 << 25) - 1), UNSUP),
    (dict(H_q=32768, H_kv=32768, ld_q=32768 * 128), UNSUP), (dict(n_blocks=1 << 24), UNSUP),
])
def test_prompt(lib, kw, status):  # noqa: F811
    good = [P, 1, 5, 2, 4, 2, 128, 512, K, V, SC, 9, P, 100, P, None, P, P, 1 << 40, None]
    assert change(lib.saki_cache4_prompt, good, PROMPT, **kw) == status
