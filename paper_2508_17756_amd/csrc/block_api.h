// Launchers of the rotary positions, the gated norm and the 8-bit integer linear layer (each validates nothing: the API layer has already done so).
#pragma once
#include "sg_common.h"

namespace sg {

int launch_rotary(const sg_rotary_problem& p, int n_tiles, const void* const* q, const void* const* k, const double* frequencies,
                  const int32_t* origin, const int32_t* const* positions, const void* q_weight, const void* k_weight, const uint8_t* run,
                  void* const* q_out, void* const* k_out, hipStream_t s);
int launch_gated_norm(const sg_gated_norm_problem& p, int n_tiles, const void* const* x, const void* const* residual, const void* const* gate,
                      const void* post_weight, const void* weight, const void* const* scale, const void* const* shift, const uint8_t* run,
                      void* const* sum, void* const* out, float* const* out_scale, hipStream_t s);
int launch_int8_linear(const sg_int8_linear_problem& p, int n_tiles, const void* const* x, const float* const* x_scale, const void* w,
                       const float* w_scale, const void* bias, const uint8_t* run, void* const* out, hipStream_t s);

}  // namespace sg
