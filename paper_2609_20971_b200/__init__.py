"""RBS-Attention prefill hot path for NVIDIA B200: block statistics, dual-branch block selection and
causal block-sparse attention as hand-written sm_100a kernels behind a small C ABI (include/rbs.h), and the calls
around it in a serving engine: norm and rotation of queries and keys, a paged key/value cache, decode attention over it.

The Python names mirror the C entry points.  Importing this package does not load the CUDA library;
the first call does, and raises if it has not been built.
"""
from .binding import (BlockStats, PagedStep, RbsError, alloc_stats, alloc_step, load_library, load_native, paged_decode_workspace_bytes, rbs_block_stats,
                      rbs_block_stats_box, rbs_device_status, rbs_mask_group_union, rbs_paged_decode, rbs_paged_extend, rbs_qk_norm_rope,
                      rbs_qk_norm_rope_paged, rbs_select, rbs_select_box, rbs_select_chunk, rbs_select_static, rbs_sparse_prefill,
                      rbs_sparse_prefill_chunk, rbs_sparse_prefill_grouped, workspace_bytes)
from .paged import PagedCache, rope_frequencies

__all__ = ["BlockStats", "PagedCache", "PagedStep", "RbsError", "alloc_stats", "alloc_step", "load_library", "load_native", "paged_decode_workspace_bytes", "rbs_block_stats",
           "rbs_block_stats_box", "rbs_device_status", "rbs_mask_group_union", "rbs_paged_decode", "rbs_paged_extend", "rbs_qk_norm_rope",
           "rbs_qk_norm_rope_paged", "rbs_select", "rbs_select_box", "rbs_select_chunk", "rbs_select_static", "rbs_sparse_prefill",
           "rbs_sparse_prefill_chunk", "rbs_sparse_prefill_grouped", "rope_frequencies", "workspace_bytes"]
