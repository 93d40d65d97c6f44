// Quantisation of rows to 8-bit integers with a float32 scale each: s = max|x| / 127,
// rounded, at least 2^-126; q = the whole number nearest to the real quotient x / s, ties
// to even, so that a row has one right answer, bit for bit. A row that holds a NaN or an
// infinity gets the scale NaN (and zeros), which spoils its own row of a product.
//
// Bound by HBM: one read of x (kept in registers between its maximum and its rounding, up
// to 8192 columns), one write of q.
#include "common.h"
#include "kernels8.h"

namespace f3c {

namespace {

// Eight values as they are stored, and the largest of their magnitudes' bits so far (as
// whole numbers: infinities above all numbers, NaN above them).
template <typename T> struct Vec8;
template <> struct Vec8<float> {
  u32x4 w[2];
  __device__ __forceinline__ void load(const float* p) {
    w[0] = reinterpret_cast<const u32x4*>(p)[0];
    w[1] = reinterpret_cast<const u32x4*>(p)[1];
  }
  __device__ __forceinline__ uint32_t top(uint32_t m) const {
#pragma unroll
    for (int e = 0; e < 8; ++e) m = max(m, w[e / 4][e % 4] & 0x7fffffffu);
    return m;
  }
  __device__ __forceinline__ float at(int e) const { return __builtin_bit_cast(float, (uint32_t)w[e / 4][e % 4]); }
};
template <> struct Vec8<bf16> {
  u32x4 w;
  __device__ __forceinline__ void load(const bf16* p) { w = *reinterpret_cast<const u32x4*>(p); }
  __device__ __forceinline__ uint32_t top(uint32_t m) const {
#pragma unroll
    for (int e = 0; e < 4; ++e) m = max(m, max(w[e] << 16 & 0x7fffffffu, w[e] & 0x7fff0000u));
    return m;
  }
  __device__ __forceinline__ float at(int e) const {
    return __builtin_bit_cast(float, e % 2 ? w[e / 2] & 0xffff0000u : w[e / 2] << 16);
  }
};

// Eight quotients as bytes. x * (1 / s) is off by less than 127 * 2^-22, and the remainder
// x - n s exact (its bits fit: n s is a multiple of s's last place, and so is x or the
// remainder is x): where it is half a step or more, the quotient lies at a border and n
// is put right by it, or by evenness.
template <typename T>
__device__ __forceinline__ u32x2 quotients(const Vec8<T>& x, float s, float inv) {
  float n[8], far = 0.0f;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    n[e] = __builtin_rintf(x.at(e) * inv);
    far = fmaxf(far, __builtin_fabsf(__builtin_fmaf(-n[e], s, x.at(e))));
  }
  if (far + far >= s) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float r = __builtin_fmaf(-n[e], s, x.at(e)), d = __builtin_fabsf(r) + __builtin_fabsf(r);
      if (d > s || (d == s && ((int)n[e] & 1))) n[e] += __builtin_copysignf(1.0f, r);
    }
  }
  uint32_t w[2] = {0, 0};
#pragma unroll
  for (int e = 0; e < 8; ++e) w[e / 4] |= ((uint32_t)(int)n[e] & 0xffu) << (8 * (e % 4));
  return u32x2{w[0], w[1]};
}

// LANES lanes a row, 8 columns a lane at a time, N times in registers; what lies beyond
// those is read again.
template <typename T, int LANES, int N>
__global__ __launch_bounds__(256) void k_quant_i8(const T* __restrict__ x, int64_t ldx, int rows, int K,
                                                  uint8_t* __restrict__ q, int64_t ldq, float* __restrict__ scale) {
  __shared__ uint32_t part[4];
  const uint32_t row = blockIdx.x * (256u / LANES) + threadIdx.x / LANES;
  const int c = (int)(threadIdx.x % LANES) * 8;
  const bool in = row < (uint32_t)rows;
  x += (in ? row : 0) * ldx;
  q += (in ? row : 0) * ldq;
  Vec8<T> v[N];
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    v[i] = Vec8<T>{};
    if (in && c + i * LANES * 8 < K) v[i].load(x + c + i * LANES * 8);
  }
#pragma unroll
  for (int i = 0; i < N; ++i) m = v[i].top(m);
  for (int j = c + N * LANES * 8; in && j < K; j += LANES * 8) {
    Vec8<T> t;
    t.load(x + j);
    m = t.top(m);
  }
#pragma unroll
  for (int d = 1; d < (LANES < 64 ? LANES : 64); d *= 2) m = max(m, (uint32_t)__shfl_xor((int)m, d));
  if constexpr (LANES > 64) {
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = m;
    __syncthreads();
    m = max(max(part[0], part[1]), max(part[2], part[3]));
  }
  if (!in) return;
  const bool bad = m >= 0x7f800000u;
  const float s = bad ? __builtin_nanf("") : fmaxf(__builtin_bit_cast(float, m) / 127.0f, 0x1p-126f);
  const float inv = 1.0f / s;
  if (c == 0) scale[row] = s;
#pragma unroll
  for (int i = 0; i < N; ++i)
    if (c + i * LANES * 8 < K)
      *reinterpret_cast<u32x2*>(q + c + i * LANES * 8) = bad ? u32x2{0, 0} : quotients(v[i], s, inv);
  for (int j = c + N * LANES * 8; j < K; j += LANES * 8) {
    Vec8<T> t;
    t.load(x + j);
    *reinterpret_cast<u32x2*>(q + j) = bad ? u32x2{0, 0} : quotients(t, s, inv);
  }
}

template <typename T, int LANES, int N>
hipError_t launch_rows(const T* x, int64_t ldx, int rows, int K, uint8_t* q, int64_t ldq, float* scale, hipStream_t s) {
  launch((k_quant_i8<T, LANES, N>), dim3((uint32_t)(((int64_t)rows * LANES + 255) / 256)), dim3(256), 0, s, x, ldx,
         rows, K, q, ldq, scale);
  return hipGetLastError();
}

// As few lanes a row as hold it in 8 or 16 columns each, a workgroup beyond 1024 columns: of 20
// combinations of lanes and registers at 26 sizes the best or within 5% of it but for 1000 rows of
// 1024 (a workgroup a row 3.5 us, here 3.8). In us, bf16, here / the next best: 9831 x 1024 8.6 / 9.1
// (64 lanes of 32 columns; 3.5 TB/s with 2 us of dispatch), 20000 x 256 5.7 / 5.8 (a wave a row 7.7),
// 5000 x 2048 8.8 / 9.4 (a wave a row 10.1), 300 x 2048 3.3 / 3.4 (a wave a row 5.0), 2500 x 4096
// 9.0 / 9.6, 1320 x 5288 in float32 8.5 / 8.7 (64 lanes 10.1).
template <typename T>
hipError_t launch_t(const T* x, int64_t ldx, int rows, int K, uint8_t* q, int64_t ldq, float* scale, hipStream_t s) {
  if (K <= 128) return launch_rows<T, 16, 1>(x, ldx, rows, K, q, ldq, scale, s);
  if (K <= 256) return launch_rows<T, 32, 1>(x, ldx, rows, K, q, ldq, scale, s);
  if (K <= 512) return launch_rows<T, 64, 1>(x, ldx, rows, K, q, ldq, scale, s);
  if (K <= 1024) return launch_rows<T, 64, 2>(x, ldx, rows, K, q, ldq, scale, s);
  if (K <= 2048) return launch_rows<T, 256, 1>(x, ldx, rows, K, q, ldq, scale, s);
  if (K <= 4096) return launch_rows<T, 256, 2>(x, ldx, rows, K, q, ldq, scale, s);
  return launch_rows<T, 256, 4>(x, ldx, rows, K, q, ldq, scale, s);
}

}  // namespace

hipError_t launch_quant_i8(int dt, int rows, int K, const void* x, int64_t ldx, void* q, int64_t ldq, float* scale,
                           hipStream_t s) {
  if (rows == 0) return hipSuccess;
  if (dt == DT_BF16) return launch_t((const bf16*)x, ldx, rows, K, (uint8_t*)q, ldq, scale, s);
  return launch_t((const float*)x, ldx, rows, K, (uint8_t*)q, ldq, scale, s);
}

}  // namespace f3c
