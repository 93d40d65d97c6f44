// Dense projections on 8-bit operands: C = A W^T + bias, A = activations [M][K]
// and W = weights [N][K] in e4m3 (K contiguous) with power-of-two scales per 1 x
// 128 block of A and 128 x 128 block of W, on the scaled matrix instructions
// with float32 accumulators. Epilogues: bf16 store, GELU (tanh form) as bf16,
// gated residual update in float32, GELU as e4m3 with scales per 1 x 128.
//
// Numerics of the matrix core: it adds the products of 8 consecutive bytes of K
// after aligning them to the largest and drops what lies 2^14 below that; beyond
// these groups of 8 the sums and the accumulator are float32 (measured on MI355X
// with single products: one of 2^-13 of its group's largest is kept whole, one of
// 2^-14 lost, in another group all are kept). A sum is then 1.5e-5 off relative to
// its own size on normally distributed operands and 2.1e-5 behind a GELU, for K = 128
// to 8192 alike, over 1000 times below the operands' own rounding. No instruction
// that takes 8-bit operands does otherwise (16x16x32, 16x16x128 and 32x32x64 agree
// bit for bit on K in the same order).
//
// Every output is one workgroup's sum in the order of K, from the bias on, the same
// for every tile shape: the shape may follow the row count without changing a
// result.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "fp8.h"
#include "kernels8.h"

namespace f3c {

namespace {

struct Gemm8Args {
  int M, N, K;
  const uint8_t* A;
  int64_t lda;
  const uint8_t* sa;
  int64_t ldsa;
  const uint8_t* W;
  int64_t ldw;
  const uint8_t* sw;
  int64_t ldsw;
  const float* bias;
  const float* gate;
  void* out;
  int64_t ldo;
  uint8_t* so;
  int64_t ldso;
  float* resid;
  int64_t ldr;
  int xq;                             // column groups of the XCD tile partition
};

// GELU in its tanh form as x / (1 + 2^(x (a + b x^2))), a = -2 log2(e) sqrt(2/pi),
// b = 0.044715 a: five operations, an exponential and a reciprocal.
__device__ __forceinline__ float gelu_fast(float x) {
  const float z = x * __builtin_fmaf(x * x, -0.10294324f, -2.3022082f);
  return x * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(z));
}

// Eight e4m3 values times a scale, as bf16: no rounding (4 significant bits).
__device__ __forceinline__ bf16x8 widen8(int lo, int hi, float scale) {
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((uint32_t)lo, scale, false);
  const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((uint32_t)lo, scale, true);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((uint32_t)hi, scale, false);
  const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((uint32_t)hi, scale, true);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// A block's two scales (bytes; 255 is NaN) as one for widen8 on the activations, beside
// 2^27 on the weights. No value leaves bf16's range above: an exponent over 119 is
// taken for 119, whose products with any weight but 0 (2^-9 at least) leave float32's
// range all the same. Below, products under 2^-81 may be lost. (Each operand under its
// own scale, values over 2^128 became infinities and those under 2^-133 zeros,
// whatever the other operand's scale.)
constexpr float kWideWeightScale = 0x1p27f;
__device__ __forceinline__ float wide_row_scale(uint32_t sa, uint32_t sw) {
  sa &= 0xffu, sw &= 0xffu;
  const int e = min(max((int)(sa + sw) - 254 - 27, -126), 119);
  return __builtin_bit_cast(float, sa == 255 || sw == 255 ? 0x7fc00000u : (uint32_t)(e + 127) << 23);
}

// Epilogue through LDS, 32 rows of the wave at a time (a lane of the MFMA layout
// holds four columns here and there of one row; rows leave in whole pieces). The
// region is the wave's own and LDS operations of a wave keep their order. All of
// the workgroup's LDS is free to use.
template <int TM, int TN, int WTM, int WTN, int BM, int BN, int WGN, int OCC, int BYTES, int EPI>
__device__ __forceinline__ void gemm8_epilogue(const Gemm8Args& p, f32x16 (&acc)[TM][TN], char* lds, int m0, int n0,
                                               int wm, int wn, int lane) {
  const int g = lane >> 5, r32 = lane & 31, wave = wm * WGN + wn;
  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)lds;
  constexpr int NW = (BM / WTM) * WGN;
  if constexpr (EPI == EPI_GELU_FP8) {
    // A quantisation block is 128 columns of a row: the wave's own (WTN = 128), or
    // spread over 128 / WTN waves, which meet in LDS.
    constexpr int RS = WTN + 16;
    constexpr int PARTS = 128 / WTN;
    static_assert(NW * 32 * RS + WGN * BM * 4 <= BYTES && BN % 128 == 0, "epilogue buffer");
    const int c0 = n0 + wn * WTN;
    // largest magnitudes; an infinity among them (which a NaN cannot hide) is rare
    // and turns into NaN in a second look
    float top[TM];
    bool odd = false;
#pragma unroll
    for (int i = 0; i < TM; ++i) {
      float m = 0.0f;
#pragma unroll
      for (int j = 0; j < TN; ++j)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[i][j][e] = gelu_fast(acc[i][j][e]);
      if (n0 + BN > p.N) {
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
          for (int e = 0; e < 16; ++e)
            if (c0 + j * 32 + 8 * (e / 4) + 4 * g >= p.N) acc[i][j][e] = 0.0f;
      }
#pragma unroll
      for (int j = 0; j < TN; ++j)
#pragma unroll
        for (int e = 0; e < 16; e += 2)
          m = fmaxf(fmaxf(m, __builtin_fabsf(acc[i][j][e])), __builtin_fabsf(acc[i][j][e + 1]));
      top[i] = m;
      odd = odd || !(m < __builtin_inff());
    }
    if (__any(odd)) {
#pragma unroll
      for (int i = 0; i < TM; ++i) {
        float m = 0.0f;
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            m = fmaxf(m, finite_abs(acc[i][j][e]));
            acc[i][j][e] = fp8_no_inf(acc[i][j][e]);
          }
        top[i] = m;
      }
    }
#pragma unroll
    for (int i = 0; i < TM; ++i) top[i] = fmaxf(top[i], __shfl_xor(top[i], 32));
    if constexpr (PARTS > 1) {
      float* part = reinterpret_cast<float*>(lds + NW * 32 * RS);      // [WGN][BM]
      if (g == 0) {
#pragma unroll
        for (int i = 0; i < TM; ++i) part[wn * BM + wm * WTM + i * 32 + r32] = top[i];
      }
      __syncthreads();
#pragma unroll
      for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int x = 0; x < PARTS; ++x)
          top[i] = fmaxf(top[i], part[(wn / PARTS * PARTS + x) * BM + wm * WTM + i * 32 + r32]);
    }
    const uint32_t eb = lds0 + (uint32_t)(wave * 32 * RS);
    typedef __attribute__((address_space(3))) uint32_t lds_w;
    typedef __attribute__((address_space(3))) const u32x4 lds_r;
    constexpr int LPR = WTN / 16, RPI = 64 / LPR;
#pragma unroll
    for (int i = 0; i < TM; ++i) {
      const uint32_t byte = fp8_scale_byte(top[i]);
      const float two_e = fp8_scale(byte);
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
      for (int j = 0; j < TN; ++j)
#pragma unroll
        for (int q = 0; q < 4; ++q)
          *(lds_w*)(uintptr_t)(eb + (uint32_t)(r32 * RS + j * 32 + 8 * q + 4 * g)) =
              fp8_pack4(acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3], two_e);
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      const int row0 = m0 + wm * WTM + i * 32;
      if (g == 0 && wn % PARTS == 0 && row0 + r32 < p.M && c0 < p.N)
        p.so[(row0 + r32) * p.ldso + (c0 >> 7)] = (uint8_t)byte;
      const int ecol = c0 + (lane % LPR) * 16;
#pragma unroll
      for (int t = 0; t < 32 / RPI; ++t) {
        const int rr = t * RPI + lane / LPR, row = row0 + rr;
        const u32x4 v = *(lds_r*)(uintptr_t)(eb + (uint32_t)(rr * RS + (lane % LPR) * 16));
        if (row < p.M && ecol < p.N)
          *reinterpret_cast<u32x4*>(reinterpret_cast<uint8_t*>(p.out) + row * p.ldo + ecol) = v;
      }
    }
  } else {
  constexpr int RS = WTN * 4 + 16;
  static_assert(NW * 32 * RS <= BYTES, "epilogue buffer");
  typedef __attribute__((address_space(3))) f32x4 lds_f4;
  const uint32_t eb = lds0 + (uint32_t)(wave * 32 * RS);
  // columns per lane, lanes per row, rows per pass
  constexpr int VC = EPI == EPI_RESID ? 4 : 8, LPR = WTN / VC, RPI = 64 / LPR;
  const int ecol = n0 + wn * WTN + (lane % LPR) * VC;
  const bool in = ecol < p.N;                      // all VC columns or none
  float gv[VC];
#pragma unroll
  for (int e = 0; e < VC; e += 4) {
    float4 g4 = make_float4(1.0f, 1.0f, 1.0f, 1.0f);
    if (EPI == EPI_RESID && p.gate && in) g4 = *reinterpret_cast<const float4*>(p.gate + ecol + e);
    gv[e] = g4.x, gv[e + 1] = g4.y, gv[e + 2] = g4.z, gv[e + 3] = g4.w;
  }
  // Residual rows are read 32 rows ahead of their update, but where four workgroups
  // share the registers: 9831 x 1024 x 1024 25.6 -> 24.9 us, 9831 x 1024 x 2048 34.3 -> 33.7,
  // others as without (32768 x 1024 x 2048 90.8 / 91.8, 820 rows 7.6 / 7.7); four of 128 x 128
  // would spill: 32768 x 1024 x 1024 60.9 -> 82.6. The 256 x 256 tile spills 20 bytes a lane
  // here, behind its loop.
  constexpr int T = 32 / RPI;
  constexpr bool kAhead = OCC < 4;
  float4 hb[2][EPI == EPI_RESID ? T : 1];
  auto load_h = [&](int i) {
    if constexpr (EPI == EPI_RESID) {
#pragma unroll
      for (int t = 0; t < T; ++t) {
        const int row = m0 + wm * WTM + i * 32 + lane / LPR + t * RPI;
        if (row < p.M && in) hb[i & 1][t] = *reinterpret_cast<const float4*>(p.resid + row * p.ldr + ecol);
      }
    }
  };
  if (kAhead) load_h(0);
#pragma unroll
  for (int i = 0; i < TM; ++i) {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int q = 0; q < 4; ++q)
        *(lds_f4*)(uintptr_t)(eb + (uint32_t)(r32 * RS + (j * 32 + 8 * q + 4 * g) * 4)) =
            f32x4{acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    if (kAhead ? i + 1 < TM : true) load_h(kAhead ? i + 1 : i);   // (into the registers of what has just been written)
    const int row0 = m0 + wm * WTM + i * 32 + lane / LPR;
#pragma unroll
    for (int t = 0; t < T; ++t) {
      const int row = row0 + t * RPI;
      float v[VC];
#pragma unroll
      for (int e = 0; e < VC; e += 4) {
        const uint32_t at = eb + (uint32_t)((t * RPI + lane / LPR) * RS + ((lane % LPR) * VC + e) * 4);
        const f32x4 c4 = *(lds_f4*)(uintptr_t)at;
#pragma unroll
        for (int x = 0; x < 4; ++x) v[e + x] = c4[x];
      }
      if (row >= p.M || !in) continue;
      if constexpr (EPI == EPI_RESID) {
        float4 h = hb[i & 1][t];
        h.x += gv[0] * v[0];
        h.y += gv[1] * v[1];
        h.z += gv[2] * v[2];
        h.w += gv[3] * v[3];
        *reinterpret_cast<float4*>(p.resid + row * p.ldr + ecol) = h;
      } else {
        bf16x8 o;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          if constexpr (EPI == EPI_GELU) v[e] = gelu_fast(v[e]);
          o[e] = (bf16)v[e];
        }
        *reinterpret_cast<bf16x8*>(reinterpret_cast<bf16*>(p.out) + row * p.ldo + ecol) = o;
      }
    }
  }
  }
}

// K tiles of 128 bytes (one scale block) go HBM -> LDS by DMA into STAGES stages;
// each wave multiplies TM x TN tiles of 32 x 32 on 32x32x64 instructions, two
// K-steps per tile.
//
// The weight fragment is the instruction's A operand and the activation fragment
// its B operand (a tile of C^T), as in the bf16 kernels. A lane feeds 32 bytes of
// one row per instruction: 16-byte chunks g and g + 2 of the K-step's four, so
// that the instruction adds the 8-byte groups in the order of K.
//
// Activation fragments roll: fragment i of the next K-step is read as soon as its
// last product of this one is issued. Weight fragments, needed until the end, are
// read a K-step ahead into a second set.
//
// Scales come with their K tile: the dword of each row that holds the tile's byte,
// by DMA too, shifted into place as it is read. The loop over K tiles has no
// branch: the compiler would move products across it, out of their places
// between the reads.
//
// What bounds it. Long K, many rows: power. On such operands the matrix cores alone,
// from registers, sustain 3.5 to 3.8 PFLOP/s (4.9 on zeros); 8192 x 8192 x 8192 takes
// 410 to 470 us by card (2.7 to 2.35 PFLOP/s) at a clock of 1.6 GHz with the matrix
// pipes busy 69% of the cycles. 256 x 256 tiles read LDS least (16-byte K halves of a
// row as stages cost 10%: lines travel twice). Short K: no pipe alone; what one workgroup
// waits for (its stage, GELU's exponential and reciprocal, its stores) another's
// products have to hide. At 32768 x 4096 x 1024 into 8 bits matrix pipes and vector issue
// are busy 43% of the cycles each and LDS reads 32%; one 256 x 256 workgroup per CU takes
// 175 us, four of 128 x 128 in a single stage 157. On bf16 instructions (32768 x 1024 x
// 4096 into the residual, 232 us) matrix pipes 57%, vector issue 40%, most of it the
// widening. Few rows: the chain of K tiles, 0.2 to 0.5 us each, of LDS reads and dependent
// products, with every pipe below a quarter (820 x 1024 x 4096: on the 208 CUs that have a
// tile matrix 14%, vector issue 22%, LDS reads 8%).
// Against the bf16 projections on one card (us, bf16 / here): 32768 x 4096 x 1024 GELU
// 300 / 161 (out in 8 bits), 9831 x 2048 x 1024 55 / 29, 9831 x 1024 x 1024 gated residual 35 / 26;
// on exact products, gated residual: 32768 x 1024 x 4096 271 / 232, 9831 rows 91 / 86, 820 rows
// 18.6 / 18.7.
template <int BM, int BN, int WGM, int WGN, int STAGES, int OCC, int EPI, int DPI = 1, bool WIDE = false>
__global__ __launch_bounds__(64 * WGM * WGN, OCC) void k_gemm8_dma(Gemm8Args p) {
  constexpr int NW = WGM * WGN, WTM = BM / WGM, WTN = BN / WGN, TM = WTM / 32, TN = WTN / 32;
  constexpr int KTB = 128, ABUF = BM * KTB, SBUF = (BM + BN) * KTB;
  constexpr int DA = BM / 8, DB = BN / 8, DQ = (DA + DB) / NW;         // DMA blocks of 8 rows
  constexpr int SA = (BM + 63) / 64, SX = (SA + NW) / NW;              // scale DMAs of A; all, per wave
  constexpr int DT = DQ + SX;                                          // a wave's DMA instructions per K tile
  constexpr int SSET = 64 * NW * SX * 4;                               // bytes of a stage's scales
  static_assert(DA % NW == 0 && DB % NW == 0, "whole DMA blocks per wave");
  static_assert(BM % (32 * WGM) == 0 && BN % (32 * WGN) == 0 && WTN <= 128 && NW % 2 == 0, "tile shape");
  static_assert(STAGES > 1 || TM * TN > 2, "a single stage is refilled between the products of a K-step");
  constexpr int EB = EPI == EPI_GELU_FP8 ? NW * 32 * (WTN + 16) + WGN * BM * 4 : NW * 32 * (WTN * 4 + 16);
  constexpr int LDSB = STAGES * (SBUF + SSET) > EB ? STAGES * (SBUF + SSET) : EB;
  __shared__ __attribute__((aligned(16))) char lds[LDSB];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave / WGN, wn = wave % WGN;
  const int g = lane >> 5, r32 = lane & 31;
  int n0, m0;
  {
    const int gx = (p.N + BN - 1) / BN, gy = (p.M + BM - 1) / BM;
    const int l = xcd_logical_id(blockIdx.x, gx * gy);
    const int gq = gx / p.xq, per_group = gy * gq;
    const int grp = l / per_group, r = l - grp * per_group;
    const int y = r / gq;
    n0 = (grp * gq + (r - y * gq)) * BN;
    m0 = y * BM;
  }
  const int KT = (p.K + KTB - 1) / KTB;
  auto swizzle = [](int row) { return (row >> 1) & 7; };
  // Descriptors span 2 GiB: an offset of 2^31 is out of range and reads zeros
  // (chunks beyond K).
  auto descriptor = [](const void* base) {
    const uint64_t a = (uint64_t)base;
    return u32x4{(uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)a),
                 (uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)(a >> 32) & 0xffffu), 0x80000000u, 0x00020000u};
  };
  const u32x4 adesc = descriptor(p.A + m0 * p.lda), wdesc = descriptor(p.W + n0 * p.ldw);
  // DMA instruction q of this wave fills the 8 rows of block wave + NW q (A's
  // blocks first): lane l row l/8 at physical chunk l%8, with the logical chunk
  // that the row's swizzle maps there (the same for all q: a wave's blocks are all
  // even or all odd). Rows past the end re-read the last one (never stored).
  const int chunk = (lane % 8 ^ swizzle(8 * wave + lane / 8)) << 4;
  uint32_t dofs[DQ];
#pragma unroll
  for (int q = 0; q < DQ; ++q) {
    const int blk = wave + NW * q;
    if (q < DA / NW) dofs[q] = (uint32_t)min(8 * blk + lane / 8, p.M - 1 - m0) * (uint32_t)p.lda + chunk;
    else dofs[q] = (uint32_t)min(8 * (blk - DA) + lane / 8, p.N - 1 - n0) * (uint32_t)p.ldw + chunk;
    asm("" : "+v"(dofs[q]));
  }
  auto cut_tail = [&](int t) {                     // what of K tile t on lies beyond K
    const uint32_t m = t * KTB + chunk >= p.K ? 0x80000000u : 0u;
#pragma unroll
    for (int q = 0; q < DQ; ++q) dofs[q] |= m;
  };
  // Scale DMA x < SA: 64 rows of A from 64 x on; SA: the weight blocks of the
  // tile's columns (those beyond it repeat SA's in places of their own). Wave w
  // issues w, w + NW, ...
  u32x4 sdesc[SX];
  uint32_t sofs[SX];
#pragma unroll
  for (int y = 0; y < SX; ++y) {
    const int x = wave + NW * y;
    sdesc[y] = x < SA ? descriptor(p.sa + m0 * p.ldsa) : descriptor(p.sw + (n0 >> 7) * p.ldsw);
    sofs[y] = x < SA ? (uint32_t)min(64 * x + lane, p.M - 1 - m0) * (uint32_t)p.ldsa
                     : (uint32_t)min(lane, ((p.N - 1) >> 7) - (n0 >> 7)) * (uint32_t)p.ldsw;
  }
  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)lds;
  // DMA instruction q of K tile t (t < KT)
  auto fetch1 = [&](int q, int t, int stage) {
    const uint32_t k = (uint32_t)t * KTB;
    if (q < DQ) {
      const uint32_t dst = lds0 + (uint32_t)(stage * SBUF + (wave + NW * q) * 1024);
      if (q < DA / NW) {
        asm volatile("buffer_load_dwordx4 %0, %1, %2 offen lds"
                     : : "v"(dofs[q]), "s"(adesc), "s"(k), "{m0}"(dst) : "memory");
      } else {
        asm volatile("buffer_load_dwordx4 %0, %1, %2 offen lds"
                     : : "v"(dofs[q]), "s"(wdesc), "s"(k), "{m0}"(dst) : "memory");
      }
    } else {
      const int y = q - DQ;
      const uint32_t dst = lds0 + (uint32_t)(STAGES * SBUF + stage * SSET + (wave + NW * y) * 256);
      const uint32_t ks = (uint32_t)(t & ~3);
      asm volatile("buffer_load_dword %0, %1, %2 offen lds"
                   : : "v"(sofs[y]), "s"(sdesc[y]), "s"(ks), "{m0}"(dst) : "memory");
    }
  };
  typedef __attribute__((address_space(3))) const u32x4 lds_u32x4;
  typedef __attribute__((address_space(3))) const uint32_t lds_u32;
  uint32_t aad[2][2], wad[2][2];                   // K-step, chunk
#pragma unroll
  for (int ks = 0; ks < 2; ++ks)
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      const uint32_t ch = (uint32_t)(((4 * ks + 2 * x + g) ^ swizzle(r32)) << 4);
      aad[ks][x] = lds0 + (wm * WTM + r32) * KTB + ch;
      wad[ks][x] = lds0 + ABUF + (wn * WTN + r32) * KTB + ch;
      asm("" : "+v"(aad[ks][x]), "+v"(wad[ks][x]));
    }
  f32x16 acc[TM][TN];                              // from the bias on
#pragma unroll
  for (int j = 0; j < TN; ++j)
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int col = n0 + wn * WTN + j * 32 + 8 * q + 4 * g;
      f32x4 b{0.0f, 0.0f, 0.0f, 0.0f};
      if (p.bias && col < p.N) b = *reinterpret_cast<const f32x4*>(p.bias + col);
#pragma unroll
      for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[i][j][4 * q + e] = b[e];
    }
  union Frag { i32x8 v; u32x4 h[2]; };
  Frag fa[TM], fw[2][TN];
  uint32_t sa[TM], sw, nsa[TM], nsw;
  float wsa[TM];                                   // WIDE: scales of the activations for widen8
  auto fence = [] { __builtin_amdgcn_sched_barrier(0); };
  auto read_a = [&](int i, int ks) {
#pragma unroll
    for (int x = 0; x < 2; ++x) fa[i].h[x] = *(lds_u32x4*)(uintptr_t)(aad[ks][x] + (uint32_t)(i * 32 * KTB));
  };
  auto read_w = [&](int set, int j, int ks) {
#pragma unroll
    for (int x = 0; x < 2; ++x) fw[set][j].h[x] = *(lds_u32x4*)(uintptr_t)(wad[ks][x] + (uint32_t)(j * 32 * KTB));
  };
  const uint32_t sad = lds0 + (uint32_t)(STAGES * SBUF + (wm * WTM + r32) * 4);
  const uint32_t swd = lds0 + (uint32_t)(STAGES * SBUF + (64 * SA + (((n0 & 127) + wn * WTN) >> 7)) * 4);
  auto read_scales = [&](int stage) {
#pragma unroll
    for (int i = 0; i < TM; ++i) nsa[i] = *(lds_u32*)(uintptr_t)(sad + (uint32_t)(stage * SSET + i * 128));
    nsw = *(lds_u32*)(uintptr_t)(swd + (uint32_t)(stage * SSET));
  };
  auto take_scales = [&](int t) {                  // the byte of K tile t lowest
#pragma unroll
    for (int i = 0; i < TM; ++i) sa[i] = nsa[i] >> (8 * (t & 3));
    sw = nsw >> (8 * (t & 3));
    if constexpr (WIDE) {
#pragma unroll
      for (int i = 0; i < TM; ++i) wsa[i] = wide_row_scale(sa[i], sw);
    }
  };
  constexpr int GS = TM * TN;
  auto product = [&](int ks, int set, int i, int j) {
    if constexpr (WIDE) {
      // 8 of a lane's 32 values at a time, as bf16 with the blocks' scales (exact)
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        const bf16x8 a = widen8(fa[i].v[2 * x], fa[i].v[2 * x + 1], wsa[i]);
        const bf16x8 w = widen8(fw[set][j].v[2 * x], fw[set][j].v[2 * x + 1], kWideWeightScale);
        acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(w, a, acc[i][j], 0, 0, 0);
      }
      fence();
      return;
    }
    acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(fw[set][j].v, fa[i].v, acc[i][j], 0, 0, 0, (int)sw, 0,
                                                                (int)sa[i]);
    fence();
  };
  if constexpr (STAGES == 1) {
    // One stage: the wait for a tile is hidden by the CU's other workgroups, and each
    // fragment has one register set, read again as soon as its last product is
    // issued (more waves fit). Columns outermost: the weights are free first.
    auto open = [&](int t) {                       // K tile t has been issued: wait, read its first K-step
      wait_vm<0>();
      __builtin_amdgcn_s_barrier();
      fence();
      read_scales(0);
      read_w(0, 0, 0);
#pragma unroll
      for (int i = 0; i < TM; ++i) read_a(i, 0);
#pragma unroll
      for (int j = 1; j < TN; ++j) read_w(0, j, 0);
      take_scales(t);
      fence();
    };
    cut_tail(0);
#pragma unroll
    for (int q = 0; q < DT; ++q) fetch1(q, 0, 0);
    open(0);
    for (int kt = 0;; ++kt) {
#pragma unroll
      for (int j = 0; j < TN; ++j)
#pragma unroll
        for (int i = 0; i < TM; ++i) {
          product(0, 0, i, j);
          if (j == TN - 1) read_a(i, 1);
          if (i == TM - 1) read_w(0, j, 1);
          fence();
        }
#pragma unroll
      for (int n = 0; n < GS; ++n) {
        product(1, 0, n % TM, n / TM);
        if (n == 0 && GS > 1) {
          __builtin_amdgcn_s_waitcnt(0xc07f);      // lgkmcnt(0): this wave holds the tile's last fragments
          __builtin_amdgcn_s_barrier();
          fence();
          cut_tail(kt + 1);
        }
        if (n < GS - 1) {
#pragma unroll
          for (int q = 0; q < DT; ++q)
            if (n == (q / DPI < GS - 2 ? q / DPI : GS - 2)) fetch1(q, min(kt + 1, KT - 1), 0);
        }
        fence();
      }
      if (kt + 1 == KT) break;
      open(kt + 1);
    }
  } else {
  // Behind the barrier that frees tile kt's stage (before product TN of its second
  // K-step), tile kt + STAGES goes into it: over the rest of that K-step, and with
  // more than two stages over the next one as well.
  constexpr int HEAD = GS > TN ? GS - TN : 1, SLOTS = HEAD + (STAGES > 2 ? GS : 0);
  constexpr int FAST = (DT + DPI - 1) / DPI < SLOTS ? (DT + DPI - 1) / DPI : SLOTS;
  auto slot = [](int q) { return q * FAST / DT; };
  auto wpos = [](int f, int from) { return from + f * (GS - from) / TN; };
  int stage = 0, dstage = STAGES - 1, dt = min(STAGES - 1, KT - 1);
  constexpr int EARLY = [] {                       // a tile's instructions within its first K-step's slots
    int n = 0;
    for (int q = 0; q < DT; ++q) n += q * FAST / DT < HEAD;
    return n;
  }();
#pragma unroll
  for (int s = 0; s < STAGES; ++s) {
    cut_tail(s);
#pragma unroll
    for (int q = 0; q < DT; ++q)
      if (s < STAGES - 1 || q < EARLY) fetch1(q, min(s, KT - 1), s);
  }
  // (what stands for the first stage alone; ahead of the first product the compiler waits
  // for the bias, and with it for every stage in flight)
  wait_vm<(STAGES - 2) * DT + EARLY>();
  __syncthreads();
  // (in the loop's order, so that the compiler's waits in it are exact)
  read_scales(0);
#pragma unroll
  for (int n = TN; n < GS + TN; ++n) {
    if (n == TN) read_a(0, 0);
    if (n < GS && n % TN == TN - 1) read_a(n / TN, 0);
#pragma unroll
    for (int f = 0; f < TN; ++f)
      if (n == (GS > TN ? wpos(f, TN) : TN)) read_w(0, f, 0);
    fence();
  }
  take_scales(0);
  fence();
  // Products n0..n1 of K-step ks, the next K-step's fragment reads (next) and the
  // DMA (slots counted from the barrier) among them.
  auto products = [&](auto ks_, auto from_, auto to_, bool next) {
    constexpr int ks = decltype(ks_)::value, from = decltype(from_)::value, to = decltype(to_)::value;
#pragma unroll
    for (int n = from; n < to; ++n) {
      const int i = n / TN, j = n % TN, nxt = ks ^ 1;
      product(ks, ks, i, j);
      if (next) {
        // (behind the barrier the fragment of row block 0 is free already)
        if (ks == 1 && n == TN) read_a(0, nxt);
        if (j == TN - 1) read_a(i, nxt);
#pragma unroll
        for (int f = 0; f < TN; ++f)
          if (n == wpos(f, ks == 1 ? TN : 0)) read_w(nxt, f, nxt);
#pragma unroll
        for (int q = 0; q < DT; ++q)
          if (slot(q) == (ks == 1 ? n - TN : n + HEAD) && (ks == 1 || STAGES > 2)) fetch1(q, dt, dstage);
      }
      fence();
    }
  };
  constexpr std::integral_constant<int, 0> c0{};
  constexpr std::integral_constant<int, 1> c1{};
  constexpr std::integral_constant<int, TN> ctn{};
  constexpr std::integral_constant<int, GS> cgs{};
  products(c0, c0, cgs, true);
  products(c1, c0, ctn, false);
  for (int kt = 0; kt + 1 < KT; ++kt) {
    // Every wave holds tile kt's last fragments and tile kt + 1 has landed: one
    // barrier retires tile kt's stage and opens kt + 1's. The loop turns here, where
    // all reads are waited for anyway (at its other places the compiler would wait
    // for the reads just issued).
    __builtin_amdgcn_s_waitcnt(0xc07f);            // lgkmcnt(0)
    wait_vm<(STAGES - 2) * DT>();
    __builtin_amdgcn_s_barrier();
    fence();
    dstage = stage;
    dt = min(kt + STAGES, KT - 1);
    cut_tail(kt + STAGES);
    const uint32_t d = stage == STAGES - 1 ? (uint32_t)(-(STAGES - 1) * SBUF) : (uint32_t)SBUF;
    stage = stage == STAGES - 1 ? 0 : stage + 1;
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        aad[k][x] += d;
        wad[k][x] += d;
      }
    read_scales(stage);
    fence();
    if (GS == TN) {                                // (no product is left of this K-step)
      read_a(0, 0);
#pragma unroll
      for (int f = 0; f < TN; ++f) read_w(0, f, 0);
#pragma unroll
      for (int q = 0; q < DT; ++q)
        if (slot(q) == 0) fetch1(q, dt, dstage);
    }
    products(c1, ctn, cgs, true);
    take_scales(kt + 1);
    products(c0, c0, cgs, true);
    products(c1, c0, ctn, false);
  }
  products(c1, ctn, cgs, false);
  }
  wait_vm<0>();
  __syncthreads();                                 // no DMA in flight, every wave past its last fragment read
  gemm8_epilogue<TM, TN, WTM, WTN, BM, BN, WGN, OCC, LDSB, EPI>(p, acc, lds, m0, n0, wm, wn, lane);
}

// Column groups of the XCD tile partition (as the bf16 projections choose it).
inline int choose_xq(int M, int N, int K, int BM, int BN) {
  const int gx = (N + BN - 1) / BN;
  const double a = (double)M * K, w = (double)N * K, l2_share = 2.0 * 1024 * 1024;
  const double rounds = std::max(1.0, (double)((M + BM - 1) / BM) * gx / 256.0);
  int best = 1;
  double best_cost = 0.0;
  for (int q = 1; q <= 8; q *= 2) {
    if (gx % q) continue;
    const double cost = a * q + (w / q <= l2_share ? w * (8.0 / q) : 8.0 * rounds * (w / q));
    if (q == 1 || cost < best_cost) {
      best = q;
      best_cost = cost;
    }
  }
  return best;
}

template <int BM, int BN, int WGM, int WGN, int STAGES, int OCC, int EPI, int DPI, bool WIDE = false>
hipError_t launch_dma(const Gemm8Args& a0, hipStream_t s) {
  Gemm8Args a = a0;
  a.xq = choose_xq(a.M, a.N, a.K, BM, BN);
  const int64_t tiles = (int64_t)((a.N + BN - 1) / BN) * ((a.M + BM - 1) / BM);
  launch((k_gemm8_dma<BM, BN, WGM, WGN, STAGES, OCC, EPI, DPI, WIDE>), dim3((uint32_t)tiles), dim3(64 * WGM * WGN), 0,
         s, a);
  return hipGetLastError();
}

// Tile shapes by a cost model in us, as the bf16 projections': a fixed cost; per K
// tile of 128 a fixed cost, one per round of 256 x per_cu workgroups (a partial
// round costs a whole one), one per workgroup of the fullest CU and one per 256
// workgroups' load; per round, workgroup and load the epilogue. A least-squares fit
// to 1374 measured calls on MI355X (128 to 8192 columns, K = 128 to 8192, 1 to 32768
// rows, every epilogue), each tile where it is within 2.5 times of the best, larger
// calls weighing a little more: the pick is 0.5% slower than the best of eleven
// measured tiles in the mean, 25% at worst; for calls over 17 GFLOP 1.1% (with neither
// 192 x 256 nor 128 x 256 it was 5%: 9831 x 1024 x 4096 stored 48.1 -> 43.8 us).
struct Tile8Cost {
  int bm, bn, per_cu;
  double fixed, k, k_round, k_group, k_load, round, group, load_store, load_gelu, load_resid, load_fp8;
};
constexpr Tile8Cost kTile8Cost[] = {
    {256, 256, 1, 4.104, 0.078, 1.252, 0.000, 0.234, 0.500, 0.000, 5.760, 10.001, 22.848, 9.214},
    {192, 256, 1, 2.124, 0.185, 0.764, 0.000, 0.576, 2.823, 0.000, 1.843, 5.055, 13.074, 4.281},
    {128, 256, 1, 1.546, 0.073, 0.476, 0.000, 0.503, 3.348, 0.000, 0.489, 2.426, 6.972, 1.916},
    {128, 128, 4, 2.757, 0.594, 0.000, 0.000, 0.441, 0.000, 1.225, 0.000, 0.588, 3.526, 0.247},
    {64, 128, 2, 2.288, 0.127, 0.000, 0.170, 0.187, 0.631, 0.624, 0.000, 0.381, 1.609, 0.155},
    {32, 128, 2, 2.065, 0.089, 0.000, 0.140, 0.145, 0.933, 0.070, 0.000, 0.308, 0.600, 0.123},
    {64, 64, 2, 1.961, 0.087, 0.027, 0.110, 0.105, 0.727, 0.385, 0.000, 0.201, 0.704, 0.000},
    {32, 64, 2, 1.812, 0.000, 0.136, 0.053, 0.069, 1.162, 0.086, 0.000, 0.301, 0.380, 0.000},
    {128, 128, 1, 1.730, 0.094, 0.237, 0.000, 0.377, 2.182, 0.000, 0.000, 0.971, 3.287, 1.046},
};

// The same for products on bf16 instructions (residual epilogue, K beyond 2048): a fit to
// 272 calls with K = 4112 to 16384. It holds below as well: over 634 other calls with K =
// 2064 to 16144, 239 of them up to 4096, its pick is 0.3% from the best in the mean, 18% at
// worst (17606 x 544 x 14080), and a new fit over shorter K gains nothing.
constexpr Tile8Cost kTile8WideCost[] = {
    {256, 256, 1, 0.000, 0.000, 2.263, 0.000, 0.341, 6.636, 0.000, 0.000, 0.000, 24.990, 0.000},
    {128, 128, 2, 0.000, 0.653, 0.359, 0.000, 0.532, 0.000, 0.000, 0.000, 0.000, 4.247, 0.000},
    {64, 128, 2, 2.915, 0.134, 0.156, 0.281, 0.103, 0.869, 0.000, 0.000, 0.000, 3.612, 0.000},
    {64, 64, 2, 1.137, 0.146, 0.083, 0.196, 0.069, 2.302, 0.015, 0.000, 0.000, 1.024, 0.000},
    {32, 64, 2, 3.144, 0.045, 0.282, 0.075, 0.041, 0.000, 0.000, 0.000, 0.000, 1.114, 0.000},
};

template <int COUNT>
inline int choose_tiles(const Tile8Cost (&cost)[COUNT], int M, int N, int K, int epi) {
  int best = -1;
  double best_t = 0.0;
  for (int c = 0; c < COUNT; ++c) {
    const Tile8Cost& m = cost[c];
    if (epi == EPI_GELU_FP8 && m.bn < kFp8Block) continue;             // a quantisation block in one workgroup
    const double tiles = std::ceil((double)M / m.bm) * std::ceil((double)N / m.bn), load = tiles / 256.0;
    const double rounds = std::ceil(load / m.per_cu), groups = std::ceil(load), kt = std::ceil(K / 128.0);
    const double t = m.fixed + kt * (m.k + m.k_round * rounds + m.k_group * groups + m.k_load * load) +
                     m.round * rounds + m.group * groups +
                     (epi == EPI_STORE ? m.load_store : epi == EPI_GELU ? m.load_gelu :
                      epi == EPI_RESID ? m.load_resid : m.load_fp8) * load;
    if (best < 0 || t < best_t) {
      best = c;
      best_t = t;
    }
  }
  return best;
}

// The residual is float32, and v's own error (1.5e-5 of it, 2.1e-5 behind a GELU) reaches
// it times the gate, whose size only the device knows. v grows with sqrt(K): for
// normally distributed rows of size 1, weights of size 0.02 and no gate or one of size 1
// the residual is 8.0e-6 off at K = 1024 and 1.0e-5 (1.2e-5 in single rows) at 2048;
// behind a GELU 4.9e-6 and 6.8e-6. Beyond 2048 this epilogue multiplies on bf16
// instructions, exact products at half the rate: 7e-8 of the residual at K = 4096, 1.1e-7
// at 8192. (The other epilogues round to bf16 or e4m3 behind the sum, over 100 times as
// much.)
constexpr int kResidWideK = 2048;

template <int EPI>
hipError_t launch_epi(const Gemm8Args& a, hipStream_t s) {
  if constexpr (EPI == EPI_RESID) {
    if (a.K > kResidWideK) {
      switch (choose_tiles(kTile8WideCost, a.M, a.N, a.K, EPI)) {
        case 0: return launch_dma<256, 256, 2, 4, 2, 2, EPI, 1, true>(a, s);
        case 1: return launch_dma<128, 128, 2, 2, 1, 2, EPI, 4, true>(a, s);
        case 2: return launch_dma<64, 128, 2, 2, 3, 2, EPI, 2, true>(a, s);
        case 3: return launch_dma<64, 64, 2, 2, 4, 2, EPI, 4, true>(a, s);
        case 4: return launch_dma<32, 64, 1, 2, 5, 1, EPI, 4, true>(a, s);
      }
      return hipErrorInvalidValue;
    }
  }
  switch (choose_tiles(kTile8Cost, a.M, a.N, a.K, EPI)) {
    case 0: return launch_dma<256, 256, 2, 4, 2, 2, EPI, 1>(a, s);
    case 1: return launch_dma<192, 256, 2, 4, 2, 2, EPI, 1>(a, s);
    case 2: return launch_dma<128, 256, 2, 4, 3, 2, EPI, 1>(a, s);
    case 3: return launch_dma<128, 128, 2, 2, 1, 4, EPI, 4>(a, s);
    case 4: return launch_dma<64, 128, 2, 2, 3, 2, EPI, 2>(a, s);
    case 5: return launch_dma<32, 128, 1, 4, 3, 2, EPI, 4>(a, s);
    case 6:
      if constexpr (EPI != EPI_GELU_FP8) return launch_dma<64, 64, 2, 2, 4, 2, EPI, 4>(a, s);
      break;
    case 7:
      if constexpr (EPI != EPI_GELU_FP8) return launch_dma<32, 64, 1, 2, 5, 1, EPI, 4>(a, s);
      break;
    case 8: return launch_dma<128, 128, 2, 4, 4, 2, EPI, 1>(a, s);
  }
  return hipErrorInvalidValue;
}

}  // namespace

hipError_t launch_gemm_fp8(int epi, int M, int N, int K, const void* A, int64_t lda, const void* sa, int64_t ldsa,
                           const void* W, int64_t ldw, const void* sw, int64_t ldsw, const float* bias,
                           const float* gate, void* out, int64_t ldo, void* so, int64_t ldso, float* resid,
                           int64_t ldr, hipStream_t s) {
  if (M == 0) return hipSuccess;
  Gemm8Args a{M, N, K, (const uint8_t*)A, lda, (const uint8_t*)sa, ldsa, (const uint8_t*)W, ldw, (const uint8_t*)sw,
              ldsw, bias, gate, out, ldo, (uint8_t*)so, ldso, resid, ldr, 1};
  switch (epi) {
    case EPI_STORE: return launch_epi<EPI_STORE>(a, s);
    case EPI_GELU: return launch_epi<EPI_GELU>(a, s);
    case EPI_RESID: return launch_epi<EPI_RESID>(a, s);
    case EPI_GELU_FP8: return launch_epi<EPI_GELU_FP8>(a, s);
  }
  return hipErrorInvalidValue;
}

}  // namespace f3c
