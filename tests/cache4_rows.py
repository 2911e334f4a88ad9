"""Single rows of a chunk over the 4-bit cache against the oracle, and how a call is divided."""
import numpy as np

import oracle as O
from tests.test_gpu_cache4 import DT, attention_bound, chunk_case, close, dev, host, ints, on_gpu, torch, values
from tests.test_gpu_cache4 import S

PART = 130  # floats of a part's row: sums, maximum, weight


def shared(case, dt, rows, shares):
    """Whether a chunk's call takes `rows` rows a work-group and `shares` of their keys (its workspace says so;
    one share: rows is not told)."""
    q, cache, tab, lens, cu = case
    T, H_q, H_kv, B = len(q), q.shape[1], cache[0].shape[1], len(lens)
    need = S.saki_cache4_prompt_workspace_bytes(dt, T, B, H_q, H_kv, tab.shape[1])
    return need == (256 if shares == 1 else (T * (H_q // H_kv) // rows + B) * H_kv * rows * PART * 4 * shares)


def picked(new, G, H_q, rng, n=10):
    """Some (request, token, head) rows: at the borders of waves and work-groups, at the ends, and any others."""
    out = set()
    for b, m in enumerate(new):
        rows = m * G
        at = {0, 31, 32, 63, 64, 95, 127, 128, 129, rows // 2, rows - 2, rows - 1, *rng.integers(0, max(rows, 1), n).tolist()}
        for r in at:
            if 0 <= r < rows:
                out.add((b, r // G, int(rng.integers(H_q // G)) * G + r % G))
    return sorted(out)


def run(case, dt, before=0, after=0, cu=None):
    """The chunk's output on the host; tokens of no request at the ends keep what they held."""
    q, cache, tab, lens, own = case
    full = np.concatenate([np.full((before, *q.shape[1:]), np.nan), q, np.full((after, *q.shape[1:]), np.nan)])
    out = torch.full(full.shape, -77.0, device="cuda:0", dtype=DT[dt])
    S.saki_cache4_prompt(dev(full, DT[dt]), *on_gpu(cache), ints(tab), ints(lens),
                         ints((own if cu is None else np.asarray(cu)) + before), out=out)
    got = host(out)
    assert (got[:before] == -77).all() and (got[before + len(q):] == -77).all()
    return got[before:before + len(q)]


def check_rows(case, dt, got, rows, new=None):
    """`rows` (request, token, head) of the output; new: tokens of the requests where they are not all given."""
    q, cache, tab, lens, cu = case
    G = q.shape[1] // cache[0].shape[1]
    new = np.diff(cu) if new is None else new
    k, v = values(cache)
    wants = []
    for b, i, h in rows:
        pos, one = int(lens[b]) - int(new[b]) + i, slice(h // G, h // G + 1)
        with np.errstate(invalid="ignore"):
            want, mass, size = O.cache4_prompt(q[cu[b] + i, h][None, None], k[:, one], v[:, one], tab[b:b + 1], [pos + 1],
                                               [0, 1])
        close(got[cu[b] + i, h], want[0, 0], attention_bound(want, mass, size, max(pos + 1, 64), dt, 2.0 ** -8)[0, 0])
        wants.append(want[0, 0])
    return np.array(wants)


__all__ = ["check_rows", "chunk_case", "picked", "run", "shared"]
