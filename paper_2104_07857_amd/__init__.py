"""MI355X-native optimizer hot path for offloaded, partitioned mixed-precision training.

A thin binding over libzi.so (hand-written HIP for gfx950 behind a C ABI, see
include/zi.h and include/zi_fp8.h).  PyTorch is used by callers for device memory and streams only.
"""
from .binding import *  # noqa: F401,F403
from .binding import (EXPORTS, LIB_PATH, ZiError, fp8_layout, lib, make_config, make_file_tensors, make_fp8_matrix,
                      make_rms_norm, make_rms_norm_backward, make_tensors,
                      zi_adamw_config, zi_file_tensor, zi_fp8_matrix, zi_rms_norm_args, zi_rms_norm_backward_args,
                      zi_chunk_segment, zi_norm_result, zi_step_plan_item, zi_stream_stats, zi_tensor)
