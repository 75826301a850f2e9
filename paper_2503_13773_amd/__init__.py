"""Paged-KV decode hot path for MI355X: thin Python binding over libkvc_hip.so.

The operations (see include/kvc.h for the contract):
    paged_attention_decode  batched decode attention over a block-allocated KV cache
    kv_block_copy           bit-exact block gather/scatter between KV pools
    kv_cache_append         write one new token per sequence into the block-allocated cache
    paged_attention_prefill causal attention of many query positions (recompute / chunked prefill)
and what keeps the blocks around them:
    block_tables_extend     blocks and slots for the new tokens of every request, from their lengths
    kv_cache_write          many new tokens per sequence written through a slot map
    key_bounds_update       smallest and largest key of every block that new tokens filled
    block_select            the blocks that each query keeps, by a score from those bounds
    paged_attention_selected  attention over the blocks kept
Every step runs in the HIP kernels of the library; this package only marshals
arguments.  PyTorch supplies device memory and streams.
"""
from .binding import (  # noqa: F401
    KVC_F32, KVC_BF16, KERNEL_AUTO, KERNEL_VALU, KERNEL_MFMA, KERNEL_MFMA_LDS, KERNEL_MFMA_BALANCED,
    KvcError, AttnDesc, AttnPlan, Pool, lib, library_path, attn_desc, attn_plan,
    workspace_bytes, workspace_init, new_workspace, paged_attention_decode, paged_attention_decode_partial,
    paged_attention_decode_noalloc, NOALLOC_WORKSPACE_BYTES, schedule_bytes, attn_schedule_build,
    paged_attention_decode_scheduled,
    paged_attention_decode_merge, paged_attention_prefill, validate_attention_inputs, kv_block_copy, kv_cache_append,
    validate_block_mapping, pool_of, status_string, version, TableUpdate, new_table_update, block_tables_extend,
    kv_cache_write, new_key_bounds, key_bounds_update, new_select_workspace, block_select, new_selected_workspace,
    paged_attention_selected,
)
