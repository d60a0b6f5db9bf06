"""MI355X-native MoE token shuffle with the layout transformation fused into the data movement.

The work is done by hand-written HIP kernels in libfusco.so behind the C boundary declared in
include/fusco.h; this package is a thin ctypes binding with the same names.  PyTorch supplies
device memory and streams only.  There is no CPU or PyTorch fallback: without the built library
every call raises.
"""
from .binding import (BF16, F32, DISPATCH_EXPERT, DISPATCH_WIRE, DISPATCH_TWO_HOP, DISPATCH_STREAMING, FuscoError, Layout, library_path,
                      ROUTE_TOKENS, ROUTE_TILES, ROUTE_BOTH_BY_TILES, ROUTE_TILES_THEN_TOKENS, WALK_PLAIN, WALK_STREAMING, WALK_THROUGH, PRODUCT_GATED, PRODUCT_LINEAR, PRODUCT_INPUT_GRAD, PRODUCT_INPUT_GRAD_ACTIVATION,
                      load_library, fusco_version, fusco_plan, fusco_plan_static, fusco_dispatch, fusco_dispatch_in_transfer_order, fusco_combine, fusco_plan_dispatch,
                      fusco_probe_copy, fusco_probe_rows, fusco_probe_pieces, fusco_probe_consume_slices, fusco_probe_time_next_call, fusco_probe_source_chunk_bytes, fusco_probe_dispatch_kernel, fusco_probe_dispatch_occupancy, fusco_probe_dispatch_pull, fusco_probe_dispatch_walk, fusco_probe_dispatch_route, fusco_probe_plan_through, fusco_probe_plan_dispatch_through, fusco_probe_segments_wide, fusco_probe_experts_tile_rows, fusco_probe_experts_tile_outputs,
                      fusco_combine_two_hop, fusco_balance_groups, fusco_cross_node_load, fusco_segments_scan,
                      fusco_segments_copy, fusco_disaggregated_plan, fusco_disaggregated_dispatch,
                      fusco_disaggregated_combine,
                      fusco_combine_backward, fusco_route, fusco_route_backward, fusco_norm_before, fusco_norm_after, fusco_norm_scratch_bytes,
                      fusco_norm_before_backward, fusco_norm_after_backward, SCORE_SOFTMAX, SCORE_SIGMOID, GATE_NONE, GATE_CHANNEL, GATE_TOKEN,
                      fusco_experts_gated, fusco_experts_linear, fusco_experts_input_grad, fusco_experts_weight_grad,
                      fusco_to_fp8, fusco_from_fp8, fusco_experts_gated_fp8, fusco_experts_linear_fp8, fusco_moe_few_scratch_bytes, fusco_moe_few)

__all__ = ["BF16", "F32", "DISPATCH_EXPERT", "DISPATCH_WIRE", "DISPATCH_TWO_HOP", "DISPATCH_STREAMING", "FuscoError", "Layout",
           "ROUTE_TOKENS", "ROUTE_TILES", "ROUTE_BOTH_BY_TILES", "ROUTE_TILES_THEN_TOKENS", "WALK_PLAIN", "WALK_STREAMING", "WALK_THROUGH", "PRODUCT_GATED", "PRODUCT_LINEAR", "PRODUCT_INPUT_GRAD", "PRODUCT_INPUT_GRAD_ACTIVATION",
           "library_path", "load_library", "fusco_version", "fusco_plan", "fusco_plan_static", "fusco_dispatch", "fusco_dispatch_in_transfer_order", "fusco_combine", "fusco_plan_dispatch",
           "fusco_probe_copy", "fusco_probe_rows", "fusco_probe_pieces", "fusco_probe_consume_slices", "fusco_probe_time_next_call", "fusco_probe_source_chunk_bytes", "fusco_probe_dispatch_kernel", "fusco_probe_dispatch_occupancy", "fusco_probe_dispatch_pull", "fusco_probe_dispatch_walk", "fusco_probe_dispatch_route", "fusco_probe_plan_through", "fusco_probe_plan_dispatch_through", "fusco_probe_segments_wide", "fusco_probe_experts_tile_rows", "fusco_probe_experts_tile_outputs", "fusco_combine_two_hop", "fusco_balance_groups", "fusco_cross_node_load",
           "fusco_segments_scan", "fusco_segments_copy", "fusco_disaggregated_plan", "fusco_disaggregated_dispatch",
           "fusco_disaggregated_combine",
           "fusco_combine_backward", "fusco_route", "fusco_route_backward", "fusco_norm_before", "fusco_norm_after", "fusco_norm_scratch_bytes",
           "fusco_norm_before_backward", "fusco_norm_after_backward", "SCORE_SOFTMAX", "SCORE_SIGMOID", "GATE_NONE", "GATE_CHANNEL", "GATE_TOKEN",
           "fusco_experts_gated", "fusco_experts_linear", "fusco_experts_input_grad", "fusco_experts_weight_grad",
           "fusco_to_fp8", "fusco_from_fp8", "fusco_experts_gated_fp8", "fusco_experts_linear_fp8", "fusco_moe_few_scratch_bytes", "fusco_moe_few"]
