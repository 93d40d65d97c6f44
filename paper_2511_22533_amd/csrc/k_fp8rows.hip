// Row passes around the 8-bit projections: quantisation of rows and weights, and
// the pass between two blocks (norm of the block's output, gated and scaled
// residual update, norm and modulation of the next block's input). All of them
// read and write HBM once and are bound by it.
#include "fp8.h"
#include "kernels.h"

namespace f3c {

namespace {

struct Eight { float v[8]; };

__device__ __forceinline__ Eight load8(const float* p) {
  const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
  return {{a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w}};
}

__device__ __forceinline__ Eight load8(const bf16* p) {
  const bf16x8 a = *reinterpret_cast<const bf16x8*>(p);
  Eight r;
#pragma unroll
  for (int e = 0; e < 8; ++e) r.v[e] = (float)a[e];
  return r;
}

__device__ __forceinline__ void store8(float* p, const float (&v)[8]) {
  reinterpret_cast<float4*>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
  reinterpret_cast<float4*>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
}

__device__ __forceinline__ void store8(bf16* p, const float (&v)[8]) {
  bf16x8 o;
#pragma unroll
  for (int e = 0; e < 8; ++e) o[e] = (bf16)v[e];
  *reinterpret_cast<bf16x8*>(p) = o;
}

__device__ __forceinline__ float amax8(const float (&v)[8]) {
  float m = 0.0f;
#pragma unroll
  for (int e = 0; e < 8; ++e) m = fmaxf(m, finite_abs(v[e]));
  return m;
}

__device__ __forceinline__ void store8_fp8(uint8_t* p, const float (&v)[8], float scale) {
  float x[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) x[e] = fp8_no_inf(v[e]);
  *reinterpret_cast<u32x2*>(p) =
      u32x2{fp8_pack4(x[0], x[1], x[2], x[3], scale), fp8_pack4(x[4], x[5], x[6], x[7], scale)};
}

// Blocks of 1 x 128: a lane holds 8 columns, 16 lanes a block, a wave 512 columns
// of one row.
template <typename T>
__global__ __launch_bounds__(256) void k_quant_rows(const T* __restrict__ x, int64_t ldx, int rows, int K, int pieces,
                                                    uint8_t* __restrict__ q, int64_t ldq, uint8_t* __restrict__ scale,
                                                    int64_t lds) {
  const int64_t item = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int lane = threadIdx.x & 63;
  if (item >= (int64_t)rows * pieces) return;
  const int row = (int)(item / pieces), c = (int)(item - (int64_t)row * pieces) * 512 + lane * 8;
  const bool in = c < K;
  Eight r{};
  if (in) r = load8(x + row * ldx + c);
  const uint32_t byte = fp8_scale_byte(row16_max(amax8(r.v)));
  if (!in) return;
  store8_fp8(q + row * ldq + c, r.v, fp8_scale(byte));
  if ((lane & 15) == 0) scale[row * lds + c / kFp8Block] = (uint8_t)byte;
}

// Blocks of 128 x 128: one workgroup each, 16 threads a row, 8 rows a thread.
template <typename T>
__global__ __launch_bounds__(256) void k_quant_tiles(const T* __restrict__ x, int64_t ldx, int rows, int K,
                                                     uint8_t* __restrict__ q, int64_t ldq,
                                                     uint8_t* __restrict__ scale, int64_t lds) {
  __shared__ float part[4];
  const int kb = (K + kFp8Block - 1) / kFp8Block, bx = (int)(blockIdx.x % kb), by = (int)(blockIdx.x / kb);
  const int tid = threadIdx.x, c = bx * kFp8Block + (tid & 15) * 8;
  const int64_t r0 = (int64_t)by * kFp8Block + (tid >> 4);
  Eight r[8];
  float m = 0.0f;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    r[i] = Eight{};
    if (c < K && r0 + 16 * i < rows) r[i] = load8(x + (r0 + 16 * i) * ldx + c);
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) m = fmaxf(m, amax8(r[i].v));
  m = row16_max(m);
  m = fmaxf(m, __shfl_xor(m, 16));
  m = fmaxf(m, __shfl_xor(m, 32));
  if ((tid & 63) == 0) part[tid >> 6] = m;
  __syncthreads();
  const uint32_t byte = fp8_scale_byte(fmaxf(fmaxf(part[0], part[1]), fmaxf(part[2], part[3])));
  const float two_e = fp8_scale(byte);
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (c < K && r0 + 16 * i < rows) store8_fp8(q + (r0 + 16 * i) * ldq + c, r[i].v, two_e);
  if (tid == 0) scale[by * lds + bx] = (uint8_t)byte;
}

// The pass between two blocks. One wave holds a row in registers, 8 columns a
// lane and 512 a piece: p = post(y) post_w, h += rs gate p, u = pre(h) pre_w,
// out = u (1 + scale) + shift. Both norms take their statistics over the row in
// float32, the variance about the mean.
struct ResidNormArgs {
  Segs rows;
  int d, post, pre;
  float eps, rs;
  const void* y;
  int64_t ldy;
  const float* post_w;
  const float* gate;
  float* h;
  int64_t ldh;
  const float* pre_w;
  const float* shift;
  const float* scale;
  int64_t ldm;
  void* out;
  int64_t ldo;
  uint8_t* out_scale;
  int64_t lds;
};

template <int NP>
__device__ __forceinline__ void normalise(float (&v)[NP][8], int kind, int lane, int d, float eps) {
  if (kind == NORM_NONE) return;
  const float inv_d = 1.0f / (float)d;
  if (kind == NORM_LAYER) {
    float s = 0.0f;
#pragma unroll
    for (int j = 0; j < NP; ++j)
#pragma unroll
      for (int e = 0; e < 8; ++e) s += v[j][e];      // (0 past the row's end)
    const float mean = wave_sum(s) * inv_d;
#pragma unroll
    for (int j = 0; j < NP; ++j) {
      const bool in = j * 512 + lane * 8 < d;
#pragma unroll
      for (int e = 0; e < 8; ++e) v[j][e] = in ? v[j][e] - mean : 0.0f;
    }
  }
  float q = 0.0f;
#pragma unroll
  for (int j = 0; j < NP; ++j)
#pragma unroll
    for (int e = 0; e < 8; ++e) q += v[j][e] * v[j][e];
  const float r = rsqrtf(wave_sum(q) * inv_d + eps);
#pragma unroll
  for (int j = 0; j < NP; ++j)
#pragma unroll
    for (int e = 0; e < 8; ++e) v[j][e] *= r;
}

template <typename TY, int OUT, int NP>
__global__ __launch_bounds__(256) void k_resid_norm(ResidNormArgs p) {
  const int lane = threadIdx.x & 63;
  const uint32_t i = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (i >= (uint32_t)(p.rows.off[p.rows.B] - p.rows.off[0])) return;
  const int row = p.rows.off[0] + (int)i;
  const int64_t b = find_segment(p.rows.off, p.rows.B, row);
  float* hr = p.h + row * p.ldh;
  float h[NP][8];
#pragma unroll
  for (int j = 0; j < NP; ++j) {
    const int c = j * 512 + lane * 8;
    Eight r{};
    if (c < p.d) r = load8(hr + c);
#pragma unroll
    for (int e = 0; e < 8; ++e) h[j][e] = r.v[e];
  }
  if (p.y) {
    const TY* yr = reinterpret_cast<const TY*>(p.y) + row * p.ldy;
    float y[NP][8];
#pragma unroll
    for (int j = 0; j < NP; ++j) {
      const int c = j * 512 + lane * 8;
      Eight r{};
      if (c < p.d) r = load8(yr + c);
#pragma unroll
      for (int e = 0; e < 8; ++e) y[j][e] = r.v[e];
    }
    normalise<NP>(y, p.post, lane, p.d, p.eps);
#pragma unroll
    for (int j = 0; j < NP; ++j) {
      const int c = j * 512 + lane * 8;
      if (c >= p.d) continue;
      if (p.post_w) {
        const Eight w = load8(p.post_w + c);
#pragma unroll
        for (int e = 0; e < 8; ++e) y[j][e] *= w.v[e];
      }
      if (p.gate) {
        const Eight g = load8(p.gate + b * p.ldm + c);
#pragma unroll
        for (int e = 0; e < 8; ++e) y[j][e] *= g.v[e];
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) h[j][e] += p.rs * y[j][e];
      store8(hr + c, h[j]);
    }
  }
  if (!p.out) return;
  normalise<NP>(h, p.pre, lane, p.d, p.eps);
#pragma unroll
  for (int j = 0; j < NP; ++j) {
    const int c = j * 512 + lane * 8;
    if (c < p.d) {
      if (p.pre_w) {
        const Eight w = load8(p.pre_w + c);
#pragma unroll
        for (int e = 0; e < 8; ++e) h[j][e] *= w.v[e];
      }
      if (p.scale) {
        const Eight sc = load8(p.scale + b * p.ldm + c), sh = load8(p.shift + b * p.ldm + c);
#pragma unroll
        for (int e = 0; e < 8; ++e) h[j][e] = h[j][e] * (1.0f + sc.v[e]) + sh.v[e];
      }
    }
    if constexpr (OUT == DT_FP8) {
      const uint32_t byte = fp8_scale_byte(row16_max(amax8(h[j])));   // (0 past the row's end)
      if (c < p.d) {
        store8_fp8(reinterpret_cast<uint8_t*>(p.out) + row * p.ldo + c, h[j], fp8_scale(byte));
        if ((lane & 15) == 0) p.out_scale[row * p.lds + c / kFp8Block] = (uint8_t)byte;
      }
    } else if (c < p.d) {
      if constexpr (OUT == DT_BF16) store8(reinterpret_cast<bf16*>(p.out) + row * p.ldo + c, h[j]);
      else store8(reinterpret_cast<float*>(p.out) + row * p.ldo + c, h[j]);
    }
  }
}

template <typename TY, int OUT>
hipError_t launch_resid_norm_t(const ResidNormArgs& a, int rows, hipStream_t s) {
  const dim3 grid(((uint32_t)rows + 3) / 4), block(256);
  if (a.d <= 512) launch((k_resid_norm<TY, OUT, 1>), grid, block, 0, s, a);
  else if (a.d <= 1024) launch((k_resid_norm<TY, OUT, 2>), grid, block, 0, s, a);
  else if (a.d <= 2048) launch((k_resid_norm<TY, OUT, 4>), grid, block, 0, s, a);
  else if (a.d <= 4096) launch((k_resid_norm<TY, OUT, 8>), grid, block, 0, s, a);
  else launch((k_resid_norm<TY, OUT, 16>), grid, block, 0, s, a);
  return hipGetLastError();
}

template <typename TY>
hipError_t launch_resid_norm_y(const ResidNormArgs& a, int out_dt, int rows, hipStream_t s) {
  switch (out_dt) {
    case DT_F32: return launch_resid_norm_t<TY, DT_F32>(a, rows, s);
    case DT_BF16: return launch_resid_norm_t<TY, DT_BF16>(a, rows, s);
    case DT_FP8: return launch_resid_norm_t<TY, DT_FP8>(a, rows, s);
  }
  return hipErrorInvalidValue;
}

template <typename T>
hipError_t launch_quant_t(const T* x, int64_t ldx, int block_rows, int rows, int K, uint8_t* q, int64_t ldq,
                          uint8_t* scale, int64_t lds, hipStream_t s) {
  if (block_rows == 1) {
    const int pieces = (K + 511) / 512;
    launch((k_quant_rows<T>), dim3((uint32_t)(((int64_t)rows * pieces + 3) / 4)), dim3(256), 0, s, x, ldx, rows, K,
           pieces, q, ldq, scale, lds);
  } else {
    launch((k_quant_tiles<T>), dim3((uint32_t)((K + 127) / 128 * (((int64_t)rows + 127) / 128))), dim3(256), 0, s, x, ldx, rows, K, q, ldq,
           scale, lds);
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_quant_fp8(int dt, int block_rows, int rows, int K, const void* x, int64_t ldx, void* q, int64_t ldq,
                            void* scale, int64_t lds, hipStream_t s) {
  if (rows == 0) return hipSuccess;
  if (dt == DT_BF16)
    return launch_quant_t((const bf16*)x, ldx, block_rows, rows, K, (uint8_t*)q, ldq, (uint8_t*)scale, lds, s);
  return launch_quant_t((const float*)x, ldx, block_rows, rows, K, (uint8_t*)q, ldq, (uint8_t*)scale, lds, s);
}

hipError_t launch_resid_norm(int dt, int out_dt, int post, int pre, float eps, float resid_scale, int d,
                             const Segs& rows, const void* y, int64_t ldy, const float* post_w, const float* gate,
                             float* h, int64_t ldh, const float* pre_w, const float* shift, const float* scale,
                             int64_t ldm, void* out, int64_t ldo, void* out_scale, int64_t lds, hipStream_t s) {
  const int n = rows.off[rows.B] - rows.off[0];
  if (n == 0 || (!y && !out)) return hipSuccess;
  ResidNormArgs a{rows, d, post, pre, eps, resid_scale, y, ldy, post_w, gate, h, ldh, pre_w, shift, scale, ldm,
                  out, ldo, (uint8_t*)out_scale, lds};
  return dt == DT_BF16 ? launch_resid_norm_y<bf16>(a, out_dt, n, s) : launch_resid_norm_y<float>(a, out_dt, n, s);
}

}  // namespace f3c
