"""CompressKV prefill-end KV-cache compression on one GB300 (sm_103a).

The compression path (window scoring with the SRH heads, pooling, budgeted
top-k, K/V gather), what stands in front of it (rotary positions, a paged cache
and attention over it) and behind it (a 4-bit cache) run in the CUDA kernels of
``libcompresskv``; this package holds the kernels' sources (``csrc/``), their nvcc build and a thin
ctypes binding of the C ABI in ``include/compresskv.h``.
"""
from . import compresskv  # noqa: F401
from .compresskv import (  # noqa: F401
    CompressKVError,
    LayerOutputs,
    PagedCache,
    Problem,
    Q4Cache,
    Rope,
    Trace,
    allocate_layer_budgets,
    compress_layer,
    compress_layer_head_budgets,
    compress_layer_lse,
    compress_layer_noalloc,
    compress_layers,
    compress_layers_lse,
    debug_stall_next_fused_call,
    debug_stall_next_paged_attend,
    debug_stall_next_q4_attend,
    gather,
    head_budget_layout,
    load,
    output_layout,
    paged_append,
    paged_attend,
    paged_cache,
    paged_gather,
    paged_workspace,
    paged_workspace_size,
    q4_append,
    q4_attend,
    q4_cache,
    q4_evict,
    q4_gather,
    q4_workspace,
    q4_workspace_size,
    read_device_status,
    rope_apply,
    rope_frequencies,
    score,
    select,
    status_string,
    workspace,
    workspace_size,
)
