// Row passes around the 8-bit projections: quantisation of rows and weights, and
// the pass between two blocks (norm of the block's output, gated and scaled
// residual update, norm and modulation of the next block's input). All of them
// read and write HBM once and are bound by it (a 1 GiB copy moves 4.8 to 5.3 TB/s by
// card). On one, with a copy of 4.8: quantisation of 32768 x 4096 bf16 rows 79 us, 5.1
// TB/s, of a 16384 x 8192 bf16 weight 78 us, 5.1; the pass between blocks over 32768 x 1024
// bf16 to 8 bits 77 us, 4.8, with as much written as read. Under some 20 MB the 1.9 us of a
// launch and one or more trips to memory count as much: 9831 x 1024 quantised 5.8 us (6.9
// where two calls' rows take turns), 820 rows of the pass 5.3.
#include "fp8.h"
#include "kernels8.h"

namespace f3c {

namespace {

struct Eight { float v[8]; };

__device__ __forceinline__ Eight load8(const float* p) {
  const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
  return {{a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w}};
}

// Eight values as they are stored.
template <typename T> struct Raw8;
template <> struct Raw8<float> { Eight v; };
template <> struct Raw8<bf16> { bf16x8 v; };

__device__ __forceinline__ Raw8<float> raw8(const float* p) { return {load8(p)}; }
__device__ __forceinline__ Raw8<bf16> raw8(const bf16* p) { return {*reinterpret_cast<const bf16x8*>(p)}; }
__device__ __forceinline__ Eight widen(const Raw8<float>& a) { return a.v; }
__device__ __forceinline__ Eight widen(const Raw8<bf16>& a) {
  Eight r;
#pragma unroll
  for (int e = 0; e < 8; ++e) r.v[e] = (float)a.v[e];
  return r;
}

__device__ __forceinline__ Eight load8(const bf16* p) { return widen(raw8(p)); }

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

// Blocks of 1 x 128: a lane holds 8 columns, 16 lanes a block. WHOLE: a wave's four
// blocks are of one row; else each is found for itself (rows of few blocks would
// leave most lanes idle: 32000 rows of 136 8.6 -> 5.4 us).
template <typename T, bool WHOLE>
__global__ __launch_bounds__(256) void k_quant_rows(const T* __restrict__ x, int64_t ldx, int rows, int K, int pieces,
                                                    uint8_t* __restrict__ q, int64_t ldq, uint8_t* __restrict__ scale,
                                                    int64_t lds) {
  constexpr int LANES = WHOLE ? 64 : 16;           // of a piece, 8 columns each; `pieces` a row
  const uint32_t item = (blockIdx.x * 256u + threadIdx.x) / LANES;
  const uint32_t row = (WHOLE ? (uint32_t)__builtin_amdgcn_readfirstlane(item) : item) / (uint32_t)pieces;
  const int c = (int)(item - row * (uint32_t)pieces) * LANES * 8 + (int)(threadIdx.x % LANES) * 8;
  const bool in = row < (uint32_t)rows && c < K;
  Eight r{};
  if (in) r = load8(x + row * ldx + c);
  const uint32_t byte = fp8_scale_byte(row16_max(amax8(r.v)));
  if (!in) return;
  store8_fp8(q + row * ldq + c, r.v, fp8_scale(byte));
  if ((threadIdx.x & 15) == 0) scale[row * lds + c / kFp8Block] = (uint8_t)byte;
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

// The pass between two blocks: p = post(y) post_w, h += rs gate p, u = pre(h)
// pre_w, out = u (1 + scale) + shift. WPR waves hold a row in registers, 8 columns
// a lane and 512 or 1024 a wave; sums over a wave on DPP adds and half swaps, over
// more waves through LDS. Both norms take their statistics over the row in
// float32, the variance about the mean.
//
// A wave keeps its columns of the vectors, combined to three (rs gate post_w, pre_w
// (1 + scale), shift), in registers over the run of rows that it works off: read
// for each row they are up to 20 bytes a column beside the row's own 11.
struct ResidNormArgs {
  Segs rows;
  int d, post, pre, run;                           // run: rows that a workgroup (or wave) works off
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

template <typename TY, int OUT, int NP, int WPR>
__global__ __launch_bounds__(WPR == 1 ? 256 : 64 * WPR, WPR > 4 ? 4 : 1) void k_resid_norm(ResidNormArgs p) {
  __shared__ float part[2][WPR];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c0 = (WPR == 1 ? 0 : wave * NP * 512) + lane * 8;
  int turn = 0;
  auto row_sum = [&](float v) {
    v = wave_sum(v);
    if constexpr (WPR > 1) {
      // (two places in turn: whoever writes one again has passed the barrier behind
      // which everyone has read it)
      if (lane == 0) part[turn][wave] = v;
      __syncthreads();
      v = 0.0f;
#pragma unroll
      for (int w = 0; w < WPR; ++w) v += part[turn][w];
      turn ^= 1;
    }
    return v;
  };
  const float inv_d = 1.0f / (float)p.d;
  auto normalise = [&](float (&v)[NP][8], int kind) {   // returns the factor that is left to apply
    if (kind == NORM_NONE) return 1.0f;
    if (kind == NORM_LAYER) {
      float s = 0.0f;
#pragma unroll
      for (int j = 0; j < NP; ++j)
#pragma unroll
        for (int e = 0; e < 8; ++e) s += v[j][e];       // (0 past the row's end)
      const float mean = row_sum(s) * inv_d;
#pragma unroll
      for (int j = 0; j < NP; ++j)
#pragma unroll
        for (int e = 0; e < 8; ++e) v[j][e] = c0 + j * 512 < p.d ? v[j][e] - mean : 0.0f;
    }
    float q = 0.0f;
#pragma unroll
    for (int j = 0; j < NP; ++j)
#pragma unroll
      for (int e = 0; e < 8; ++e) q += v[j][e] * v[j][e];
    return rsqrtf(row_sum(q) * inv_d + p.eps);
  };
  const uint32_t total = (uint32_t)(p.rows.off[p.rows.B] - p.rows.off[0]);
  const uint32_t first = (WPR == 1 ? blockIdx.x * 4u + wave : blockIdx.x) * (uint32_t)p.run;
  if (first >= total) return;
  const uint32_t last = min(total - first, (uint32_t)p.run) + first;
  int b = find_segment(p.rows.off, p.rows.B, p.rows.off[0] + (int)first), end = 0;
  float fg[NP][8], fs[NP][8], sh[NP][8];           // rs gate post_w, pre_w (1 + scale), shift
  // a row's loads are issued a row ahead; of six and eight waves only one workgroup
  // would fit on a CU with the registers of that
  constexpr bool kAhead = WPR <= 4;
  Eight nh[NP];
  Raw8<TY> ny[NP];
  auto fetch = [&](int row) {
#pragma unroll
    for (int j = 0; j < NP; ++j) {
      const int c = c0 + j * 512;
      nh[j] = Eight{};
      ny[j] = Raw8<TY>{};
      if (c < p.d) {
        nh[j] = load8(p.h + row * p.ldh + c);
        if (p.y) ny[j] = raw8(reinterpret_cast<const TY*>(p.y) + row * p.ldy + c);
      }
    }
  };
  if (kAhead) fetch(p.rows.off[0] + (int)first);
  for (uint32_t i = first; i < last; ++i) {
    const int row = p.rows.off[0] + (int)i;
    float* hr = p.h + row * p.ldh;
    float h[NP][8], y[NP][8];
    if (!kAhead) fetch(row);
#pragma unroll
    for (int j = 0; j < NP; ++j) {
      const Eight t = widen(ny[j]);
#pragma unroll
      for (int e = 0; e < 8; ++e) h[j][e] = nh[j].v[e], y[j][e] = t.v[e];
    }
    if (kAhead && i + 1 < last) fetch(row + 1);
    if (row >= end) {                              // the first row, or another sample's
      while (p.rows.off[b + 1] <= row) ++b;
      end = p.rows.off[b + 1];
#pragma unroll
      for (int j = 0; j < NP; ++j) {
        const int c = c0 + j * 512;
        Eight g, w, v, z, t{};
#pragma unroll
        for (int e = 0; e < 8; ++e) g.v[e] = w.v[e] = v.v[e] = 1.0f, z.v[e] = 0.0f;
        if (c < p.d) {
          if (p.gate) g = load8(p.gate + b * p.ldm + c);
          if (p.post_w) w = load8(p.post_w + c);
          if (p.pre_w) v = load8(p.pre_w + c);
          if (p.scale) z = load8(p.scale + b * p.ldm + c), t = load8(p.shift + b * p.ldm + c);
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          fg[j][e] = p.rs * g.v[e] * w.v[e];
          fs[j][e] = v.v[e] * (1.0f + z.v[e]);
          sh[j][e] = t.v[e];
        }
      }
    }
    if (p.y) {
      const float r = normalise(y, p.post);
#pragma unroll
      for (int j = 0; j < NP; ++j) {
#pragma unroll
        for (int e = 0; e < 8; ++e) h[j][e] += y[j][e] * r * fg[j][e];
        if (c0 + j * 512 < p.d) store8(hr + c0 + j * 512, h[j]);
      }
    }
    if (!p.out) continue;
    const float r = normalise(h, p.pre);
#pragma unroll
    for (int j = 0; j < NP; ++j) {
      const int c = c0 + j * 512;
#pragma unroll
      for (int e = 0; e < 8; ++e) h[j][e] = h[j][e] * r * fs[j][e] + sh[j][e];
      if constexpr (OUT == DT_FP8) {
        const uint32_t byte = fp8_scale_byte(row16_max(c < p.d ? amax8(h[j]) : 0.0f));
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
}

template <typename TY, int OUT, int NP, int WPR>
hipError_t launch_resid_norm_w(ResidNormArgs a, int64_t rows, hipStream_t s) {
  // about twice as many waves as the chip holds, the rows in equal runs
  const int64_t workers = 8192 / WPR;
  a.run = (int)((rows + workers - 1) / workers);
  const int64_t used = (rows + a.run - 1) / a.run;
  launch((k_resid_norm<TY, OUT, NP, WPR>), dim3((uint32_t)(WPR == 1 ? (used + 3) / 4 : used)),
         dim3(WPR == 1 ? 256 : 64 * WPR), 0, s, a);
  return hipGetLastError();
}

// Waves per row: of 1024 columns, but of 512 (a lane's 8) up to 512 and from 1032 to
// 1536. With half the columns a wave waits for half the loads and holds half the
// registers: faster while a call's rows fit the last-level cache (256 MB). Beyond it
// more waves per row read memory less well, unless the wave of 1024 that they replace
// is half empty. us at 9831 / 65536 rows, bf16 to 8 bits: width 1024 in two of 512 21.6 /
// 164.1, in one of 1024 25.0 / 145.7; 1320 in three 27.2 / 216.3, in two of 1024 32.9 /
// 219.1; 1536 29.9 / 237.9 against 35.0 / 237.8; 2048 (at 32768 rows) in four 159.9, in
// two 155.0; 2560 (at 820 / 20000 rows, float32 to 8 bits) in five 7.9 / 147.5, in three
// of 1024 7.8 / 140.4. Beyond 4096 the number is even: width 4608 (bf16, 820 / 20000 rows)
// in six 15.3 / 245, in five 15.8 / 225 (few rows before many); 7168 in eight 18.5 / 328, in
// seven 18.8 / 358. Six and eight waves from float32 rows to 8 bits spill 36 bytes a lane.
template <typename TY, int OUT>
hipError_t launch_resid_norm_t(const ResidNormArgs& a, int rows, hipStream_t s) {
  if (a.d <= 512) return launch_resid_norm_w<TY, OUT, 1, 1>(a, rows, s);
  if (a.d > 1024 && a.d <= 1536) return launch_resid_norm_w<TY, OUT, 1, 3>(a, rows, s);
  switch ((a.d + 1023) / 1024) {                   // waves of 1024 columns
    case 1: return launch_resid_norm_w<TY, OUT, 2, 1>(a, rows, s);
    case 2: return launch_resid_norm_w<TY, OUT, 2, 2>(a, rows, s);
    case 3: return launch_resid_norm_w<TY, OUT, 2, 3>(a, rows, s);
    case 4: return launch_resid_norm_w<TY, OUT, 2, 4>(a, rows, s);
    case 5:
    case 6: return launch_resid_norm_w<TY, OUT, 2, 6>(a, rows, s);
  }
  return launch_resid_norm_w<TY, OUT, 2, 8>(a, rows, s);
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
    const int blocks = (K + kFp8Block - 1) / kFp8Block;
    const bool whole = blocks % 4 == 0;
    const int64_t threads = (int64_t)rows * (whole ? blocks / 4 * 64 : blocks * 16);
    const dim3 grid((uint32_t)((threads + 255) / 256));
    if (whole) launch((k_quant_rows<T, true>), grid, dim3(256), 0, s, x, ldx, rows, K, blocks / 4, q, ldq, scale, lds);
    else launch((k_quant_rows<T, false>), grid, dim3(256), 0, s, x, ldx, rows, K, blocks, q, ldq, scale, lds);
  } else {
    const int64_t tiles = ((int64_t)K + 127) / 128 * (((int64_t)rows + 127) / 128);
    launch((k_quant_tiles<T>), dim3((uint32_t)tiles), dim3(256), 0, s, x, ldx, rows, K, q, ldq, scale, lds);
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
  ResidNormArgs a{rows, d, post, pre, 1, eps, resid_scale, y, ldy, post_w, gate, h, ldh, pre_w, shift, scale, ldm,
                  out, ldo, (uint8_t*)out_scale, lds};
  return dt == DT_BF16 ? launch_resid_norm_y<bf16>(a, out_dt, n, s) : launch_resid_norm_y<float>(a, out_dt, n, s);
}

}  // namespace f3c
