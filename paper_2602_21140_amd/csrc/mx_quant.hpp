// Quantisation of activations for the 4-bit expert FFN.
#pragma once

#include "ctx.hpp"

namespace revive {

// bf16 rows [rows, K] -> codes [rows][mx_code_row(K)], 64 bytes a step, and scales [rows][mx_scale_row(K)] in the order of mx_scale_at.
int launch_mx_quantize_tiled(revive_ctx*, const void* x, int64_t rows, int K, uint8_t* codes, uint8_t* scales, hipStream_t);

}  // namespace revive
