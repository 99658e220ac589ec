// Acoustic-model operators: what the checks (am.cpp) and the kernels
// (am_norm.hip, am_layer_norm.hip, am_distill.hip, am_clip.hip,
// am_loglikes.hip, am_linear*.hip, am_gated*.hip) share.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "wfstdec.h"

namespace wfd {

// Launchers: arguments checked by the caller, no row count of zero unless
// said.  They return the launch's error.
hipError_t am_launch_linear(const wfst_am_linear_args &a, hipStream_t stream);
int64_t am_linear_backward_bytes(const wfst_am_linear_backward_args &a);
hipError_t am_launch_linear_backward(const wfst_am_linear_backward_args &a, hipStream_t stream);   // M >= 0
hipError_t am_launch_gated(const wfst_am_gated_args &a, hipStream_t stream);
int64_t am_gated_backward_bytes(const wfst_am_gated_backward_args &a);
hipError_t am_launch_gated_backward(const wfst_am_gated_backward_args &a, hipStream_t stream);     // M >= 0
hipError_t am_launch_norm(const wfst_am_norm_args &a, hipStream_t stream);
int64_t am_norm_backward_bytes(const wfst_am_norm_backward_args &a);
hipError_t am_launch_norm_backward(const wfst_am_norm_backward_args &a, hipStream_t stream);       // M >= 0
hipError_t am_launch_layer_norm(const wfst_am_layer_norm_args &a, hipStream_t stream);
int64_t am_layer_norm_backward_bytes(const wfst_am_layer_norm_backward_args &a);
hipError_t am_launch_layer_norm_backward(const wfst_am_layer_norm_backward_args &a, hipStream_t stream);   // M >= 0
hipError_t am_launch_distill(const wfst_am_distill_args &a, bool backward, hipStream_t stream);
int64_t am_clip_bytes(const wfst_am_clip_args &a);
hipError_t am_launch_clip(const wfst_am_clip_args &a, hipStream_t stream);   // count >= 0
hipError_t am_launch_loglikes(const wfst_am_loglikes_args &a, hipStream_t stream);

inline int64_t am_type_bytes(int32_t type)
{
    return type == WFST_F32 ? 4 : type == WFST_F8E4M3 ? 1 : 2;
}

constexpr float kE4m3Max = 448.0f;

}  // namespace wfd
