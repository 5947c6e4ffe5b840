"""sbconv: sparse basis convolution on continuous domains for MI355X (gfx950).

The compute path is the HIP library libsbconv.so behind the C ABI declared in
include/sbconv.h; this package is its thin torch binding.
"""
from .ops import (CSC, CSR, Geometry, basis_eval, conv_backward, conv_forward,
                  conv_forward_noalloc, conv_forward_noalloc_max_bytes, conv_plan, conv_workspace_size, csr_transpose, csr_transpose_batched,
                  conv_decay_gradient, featureless_backward, featureless_forward, sample_points,
                  lif_sample_events, EventStream,
                  neighbour_search_events, neighbour_search_events_csc,
                  neighbour_search_points, resolve_order)
from .sequence import (cache_append, cache_slots, layer_norm_backward, layer_norm_forward,
                       linear_attention_backward, linear_attention_forward,
                       linear_attention_step, qk_norm_rotary_backward, qk_norm_rotary_forward,
                       rotary_backward, rotary_forward, softmax_attention_backward,
                       softmax_attention_forward, softmax_attention_paged)

__all__ = ["CSC", "CSR", "Geometry", "basis_eval", "conv_backward", "conv_forward",
           "conv_forward_noalloc", "conv_forward_noalloc_max_bytes", "conv_plan", "conv_workspace_size", "csr_transpose", "csr_transpose_batched",
           "conv_decay_gradient", "featureless_backward", "featureless_forward", "sample_points",
           "lif_sample_events", "EventStream",
           "neighbour_search_events", "neighbour_search_events_csc",
           "neighbour_search_points", "resolve_order",
           "layer_norm_backward", "layer_norm_forward", "linear_attention_backward",
           "linear_attention_forward", "linear_attention_step", "rotary_backward",
           "rotary_forward", "qk_norm_rotary_backward", "qk_norm_rotary_forward",
           "softmax_attention_backward", "softmax_attention_forward", "softmax_attention_paged",
           "cache_append", "cache_slots"]
