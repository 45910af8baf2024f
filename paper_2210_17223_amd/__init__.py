"""MI355X-native one-GPU MoE-layer forward (libmoe) and its thin Python binding.

The HIP kernels live in csrc/ behind the C-ABI declared in include/moe.h and
include/moe_sched.h, include/moe_train.h, include/moe_offload.h, include/moe_comm.h,
include/moe_norm.h, include/moe_gated.h, include/moe_q8.h; this package only marshals arguments.  PyTorch is used for device memory and streams.
"""
from .binding import (ACT, DTYPE, MoeError, Shape, alloc_buffers, lib, lib_path,
                      moe_calib_copy, moe_calib_gemm, moe_calib_mfma, moe_capacity, moe_expert_gemm_kernel, moe_combine, moe_dispatch, moe_dispatch_static,
                      moe_dispatch_static_limit, moe_expert_ffn,
                      moe_last_error, moe_layer_chunked, moe_max_rows, moe_pack_gate, moe_path_calls,
                      moe_pack_weights, moe_packed_gate_bytes, moe_packed_weight_bytes,
                      moe_profile_enable, moe_profile_read, moe_route, moe_tune_ffn_group_rows,
                      moe_workspace_bytes,
                      STAGES)

from .sched_binding import (PathShape, moe_devices_for_expert, moe_path_count, moe_path_finalize,
                            moe_path_profile, moe_popularity_estimate, moe_schedule_experts,
                            moe_schedule_layer, moe_top_lists_identical)

from .offload_binding import (moe_expert_ffn_offloaded, moe_offload_staging_bytes,
                              moe_offload_workspace_bytes)
from .train_binding import (moe_backward_gemm_kernel, moe_backward_workspace_bytes, moe_layer_backward,
                            moe_layer_forward_keep)
from .gated_binding import (Q4Shape, moe_gated_backward_workspace_bytes, moe_gated_ffn, moe_gated_ffn_backward,
                            moe_gated_ffn_q4, moe_gated_gemm_kernel,
                            moe_gated_kept_backward_workspace_bytes, moe_gated_kept_workspace_bytes, moe_gated_packed_bytes, moe_gated_q4_workspace_bytes,
                            moe_gated_workspace_bytes, moe_pack_gated_weights, moe_q4_linear)
from .norm_binding import (NormShape, moe_norm_after, moe_norm_after_backward, moe_norm_before,
                           moe_norm_before_backward, moe_norm_workspace_bytes)
from .q8_binding import (Q8Shape, moe_dispatch_q8, moe_gated_ffn_q8, moe_gated_q8_kernel, moe_gated_q8_workspace_bytes,
                         moe_norm_after_q8, moe_norm_before_q8, moe_q8_linear, moe_q8_linear_kernel, moe_q8_rows, moe_q8_values)
from . import comm_binding as comm
from .comm_binding import moe_layer_padded, moe_padded_workspace_bytes

__all__ = ["Q8Shape", "moe_dispatch_q8", "moe_gated_ffn_q8", "moe_gated_q8_workspace_bytes", "moe_norm_after_q8", "moe_norm_before_q8",
           "moe_q8_linear", "moe_q8_linear_kernel", "moe_gated_q8_kernel", "moe_q8_rows", "moe_q8_values", "Q4Shape", "moe_gated_kept_workspace_bytes", "moe_gated_kept_backward_workspace_bytes", "moe_gated_gemm_kernel", "moe_gated_ffn_q4", "moe_gated_q4_workspace_bytes", "moe_q4_linear", "moe_gated_backward_workspace_bytes", "moe_gated_ffn", "moe_gated_ffn_backward", "moe_gated_packed_bytes",
           "moe_gated_workspace_bytes", "moe_pack_gated_weights", "NormShape", "moe_norm_after", "moe_norm_after_backward", "moe_norm_before",
           "moe_norm_before_backward", "moe_norm_workspace_bytes",
           "comm", "moe_layer_padded", "moe_padded_workspace_bytes", "moe_expert_ffn_offloaded", "moe_offload_staging_bytes", "moe_offload_workspace_bytes",
           "moe_backward_gemm_kernel", "moe_backward_workspace_bytes", "moe_layer_backward", "moe_layer_forward_keep", "PathShape", "moe_devices_for_expert", "moe_path_count", "moe_path_finalize",
           "moe_path_profile", "moe_popularity_estimate", "moe_schedule_experts",
           "moe_schedule_layer", "moe_top_lists_identical",
           "ACT", "DTYPE", "MoeError", "Shape", "alloc_buffers", "lib", "lib_path",
           "moe_calib_copy", "moe_calib_gemm", "moe_calib_mfma", "moe_capacity", "moe_expert_gemm_kernel", "moe_combine", "moe_dispatch", "moe_dispatch_static",
           "moe_dispatch_static_limit", "moe_expert_ffn",
           "moe_last_error", "moe_layer_chunked", "moe_max_rows", "moe_pack_gate", "moe_path_calls",
           "moe_pack_weights", "moe_packed_gate_bytes", "moe_packed_weight_bytes",
           "moe_profile_enable", "moe_profile_read", "moe_route", "moe_tune_ffn_group_rows",
           "moe_workspace_bytes",
           "STAGES"]
