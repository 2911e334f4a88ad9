"""SAKI (score-aware low-rank key indexing) retrieval-index path for MI355X.

The compute lives in libsaki.so (host float64 calibration + gfx950 HIP
kernels, C ABI in include/saki.h): the index, and serving around it (rotary
positions, block tables, paged caches in 8 and 4 bits, their attention and that
of whole prompts).  ``paper_2608_03228_amd.saki`` is its thin ctypes binding.
Build with ``python -m paper_2608_03228_amd.build``.
"""
from . import saki  # noqa: F401
from .saki import (  # noqa: F401
    saki_attend, saki_attend_prompt, saki_attend_prompt_workspace_bytes, saki_block_tables,
    saki_build_index, saki_cache4_attend, saki_cache4_attend_workspace_bytes, saki_cache4_prompt,
    saki_cache4_prompt_workspace_bytes, saki_cache4_read, saki_cache4_write, saki_cache_attend,
    saki_cache_attend_workspace_bytes, saki_cache_write,
    saki_calibrate, saki_index_bytes, saki_index_export, saki_recall, saki_recall_workspace_bytes,
    saki_rope, saki_score_topk, saki_score_topk_workspace_bytes, saki_status_string, saki_sym_eig,
    saki_version, saki_weight_svd_factors,
)
