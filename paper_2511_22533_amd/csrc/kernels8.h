// Host entry points of the 8-bit operators' kernels (k_gemm8.hip, k_fp8rows.hip).
#pragma once

#include "kernels.h"

namespace f3c {

// Beside Dtype's and Epilogue's values, which the model's kernels take.
enum : int { DT_FP8 = 2, EPI_GELU_FP8 = 3 };
enum Norm { NORM_NONE = 0, NORM_LAYER = 1, NORM_RMS = 2 };

// launch_gemm on e4m3 operands with E8M0 scales: sa [M][ldsa] per 1 x 128 of A, sw
// [ceil(N/128)][ldsw] per 128 x 128 of W (row strides multiples of 4); bias may
// be null. EPI_GELU_FP8 writes out as e4m3 and so [M][ldso]. N, K and row strides
// of 8-bit operands multiples of 16.
hipError_t launch_gemm_fp8(int epi, int M, int N, int K, const void* A, int64_t lda, const void* sa, int64_t ldsa,
                           const void* W, int64_t ldw, const void* sw, int64_t ldsw, const float* bias,
                           const float* gate, void* out, int64_t ldo, void* so, int64_t ldso, float* resid,
                           int64_t ldr, hipStream_t s);

// e4m3 values and E8M0 scales of x [rows][K] (f32 or bf16) per block_rows (1 or
// 128) x 128; K a multiple of 8.
hipError_t launch_quant_fp8(int dt, int block_rows, int rows, int K, const void* x, int64_t ldx, void* q, int64_t ldq,
                            void* scale, int64_t lds, hipStream_t s);

// h += rs * gate * (post(y) * post_w) (y null: h as it is), out = (pre(h) *
// pre_w) * (1 + scale) + shift (out null: none) over the rows of the segments;
// gate, shift, scale [B][ldm]; null factors are left out. d a multiple of 8, at
// most 8192.
hipError_t launch_resid_norm(int dt, int out_dt, int post, int pre, float eps, float resid_scale, int d,
                             const Segs& rows, const void* y, int64_t ldy, const float* post_w, const float* gate,
                             float* h, int64_t ldh, const float* pre_w, const float* shift, const float* scale,
                             int64_t ldm, void* out, int64_t ldo, void* out_scale, int64_t lds, hipStream_t s);

}  // namespace f3c
