// The cache of 8-bit keys and values (cache8.h): appending to it, and attention over it.
#include <algorithm>

#include "cache8.h"
#include "fp8.h"

namespace f3c {

namespace {

// ------------------------------------------------------------------------------ append

struct AppendArgs {
  Cache8 c;
  Lens len;
  Segs rows, pages;                                // pages: of the samples that the new tokens reach, counted through
  const void* k;
  const void* v;
  int64_t ldk, ldv;
};

template <typename T>
__device__ __forceinline__ void load8(float (&x)[8], const T* p) {
  if constexpr (sizeof(T) == 4) {
    const f32x4 a = reinterpret_cast<const f32x4*>(p)[0], b = reinterpret_cast<const f32x4*>(p)[1];
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = a[e], x[4 + e] = b[e];
  } else {
    const bf16x8 a = *reinterpret_cast<const bf16x8*>(p);
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = (float)a[e];
  }
}

// One workgroup per page, head, and K or V. A thread has four tokens of eight columns: of K
// tokens apart, so that 8-byte pieces of a row lie side by side; of V four in a row, which
// are a word of its tile. A page that holds tokens of before keeps its scale unless the new
// ones need a larger one; then those are rounded anew (a power of two less: exact but for
// e4m3's subnormals).
template <typename T, int HD>
__global__ __launch_bounds__(2 * HD) void k_cache8_append(AppendArgs p) {
  __shared__ float part[(2 * HD + 63) / 64];
  const int tid = threadIdx.x, heads = p.c.kv_heads;
  int item = blockIdx.x;
  const bool is_v = item & 1;
  item >>= 1;
  const int head = item % heads, pg = item / heads;
  const int b = find_segment(p.pages.off, p.pages.B, pg);
  const int n_old = p.len.n[b], r0 = p.rows.off[b], n_new = p.rows.off[b + 1] - r0;
  const int index = n_old / kPage + pg - p.pages.off[b];
  const int page = p.c.table[(int64_t)b * p.c.max_pages + index];
  if ((uint32_t)page >= (uint32_t)p.c.n_pages) return;
  const int t_old = max(n_old - index * kPage, 0);                     // tokens of before, of the page
  const int t_end = min(n_old + n_new - index * kPage, kPage);         // and those with the new ones
  const int64_t tile = (int64_t)page * heads + head;
  uint8_t* dst = (is_v ? p.c.v : p.c.k) + tile * (kPage * HD);
  uint8_t* sp = (is_v ? p.c.vs : p.c.ks) + tile;
  const T* src = reinterpret_cast<const T*>(is_v ? p.v : p.k) + (int64_t)head * HD;
  const int64_t ld = is_v ? p.ldv : p.ldk;
  const int64_t row0 = (int64_t)r0 + index * kPage - n_old;            // of the page's token 0

  const uint32_t was = t_old ? *sp : 0u;
  const int word = tid % 16;                                           // of V: tokens 16 (word % 4) + 4 (word / 4) + i
  const int col = is_v ? tid / 16 * 8 : tid % (HD / 8) * 8;
  int tok[4];
  float x[4][8];
  float m = 0.0f;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    tok[i] = is_v ? 16 * (word % 4) + 4 * (word / 4) + i : tid / (HD / 8) + 16 * i;
#pragma unroll
    for (int e = 0; e < 8; ++e) x[i][e] = 0.0f;
    if (tok[i] >= t_old && tok[i] < t_end) load8(x[i], src + (row0 + tok[i]) * ld + col);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int e = 0; e < 8; ++e) m = fmaxf(m, finite_abs(x[i][e]));
  m = row16_max(m);
  m = fmaxf(m, __shfl_xor(m, 16));
  m = fmaxf(m, __shfl_xor(m, 32));
  if constexpr (HD > 32) {
    if ((tid & 63) == 0) part[tid >> 6] = m;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < (2 * HD + 63) / 64; ++w) m = fmaxf(m, part[w]);
  }
  const uint32_t byte = max(fp8_scale_byte(m), was);
  const float scale = fp8_scale(byte);
  const bool grown = t_old && byte > was;
  // what is written: the new tokens, and all of them where the scale has grown
  const int first = grown ? 0 : t_old;
  if (grown) {
    const float up = fp8_scale(was);
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (tok[i] < t_old) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const uint32_t code = is_v ? dst[(col + e) * kPage + 4 * word + i] : dst[tok[i] * HD + col + e];
          x[i][e] = __builtin_amdgcn_cvt_f32_fp8((int)code, 0) * up;
        }
      }
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int e = 0; e < 8; ++e) x[i][e] = fp8_no_inf(x[i][e]);
  if (is_v) {
    const bool whole = tok[0] >= first && tok[3] < t_end;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const uint32_t w = fp8_pack4(x[0][e], x[1][e], x[2][e], x[3][e], scale);
      uint8_t* at = dst + (col + e) * kPage + 4 * word;
      if (whole) {
        *reinterpret_cast<uint32_t*>(at) = w;
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (tok[i] >= first && tok[i] < t_end) at[i] = (uint8_t)(w >> (8 * i));
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (tok[i] >= first && tok[i] < t_end)
        *reinterpret_cast<u32x2*>(dst + tok[i] * HD + col) =
            u32x2{fp8_pack4(x[i][0], x[i][1], x[i][2], x[i][3], scale),
                  fp8_pack4(x[i][4], x[i][5], x[i][6], x[i][7], scale)};
  }
  if (tid == 0) *sp = (uint8_t)byte;
}

// --------------------------------------------------------------------------- attention

struct Attn8Args {
  Cache8 c;
  Lens len;
  Segs rows, tiles;                                // tiles: of 16 rows (token, head of the group), counted through
  const bf16* q;
  bf16* o;
  int64_t ldq, ldo;
  int group, causal, splits;
  float scale;                                     // of the scores, to base 2
  float* part_o;                                   // [splits][tiles][kv_heads][16][hd]: unnormalised outputs
  float* part_ml;                                  // and [..][16][2]: reference max, sum
};

// Eight e4m3 values times a scale, as bf16: no rounding (4 significant bits).
__device__ __forceinline__ bf16x8 widen8(uint32_t lo, uint32_t hi, float scale) {
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false);
  const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false);
  const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// Bytes 0xff where a word's e4m3 bytes are NaN.
__device__ __forceinline__ uint32_t nan_bytes(uint32_t w) {
  const uint32_t top = ((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;     // 0x7f carries into its own top bit alone
  return (top >> 7) * 0xffu;
}

// 16 rows (queries of one key head's group) a workgroup, whose waves take its pages in
// turn; scores S^T = K Q^T, so that a lane holds one row's scores and its statistics.
template <int HD, int NW, bool SPLIT>
__global__ __launch_bounds__(64 * NW) void k_cache8_attn(Attn8Args p) {
  constexpr int NK = HD / 32, NV = HD / 16;        // K slices of 32 columns; output tiles of 16
  __shared__ __attribute__((aligned(16))) float so[NW][16][HD + 4];
  __shared__ float sm[NW][16], sl[NW][16];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int c = lane >> 4, r16 = lane & 15;
  const int n_tiles = p.tiles.off[p.tiles.B], kvh = p.c.kv_heads;
  int item = xcd_logical_id(blockIdx.x, n_tiles * kvh * p.splits);
  const int split = item % p.splits;
  item /= p.splits;
  const int head = item % kvh, tile = item / kvh;
  const int b = find_segment_wave(p.tiles.off, p.tiles.B, tile);
  const int q0 = p.rows.off[b], nq = p.rows.off[b + 1] - q0, n = p.len.n[b];
  const int row = (tile - p.tiles.off[b]) * 16 + r16, tok = row / p.group;
  const bool in = tok < nq;
  const int qcol = (head * p.group + row - tok * p.group) * HD;
  // a row sees keys below its limit; the tile those below the last row's
  const int lim = !in ? 0 : p.causal ? max(min(n, n - nq + tok + 1), 0) : n;
  const int tok_lo = (tile - p.tiles.off[b]) * 16 / p.group;
  const int tok_hi = min(((tile - p.tiles.off[b]) * 16 + 15) / p.group, nq - 1);
  const int lim_lo = p.causal ? n - nq + tok_lo + 1 : n, lim_hi = p.causal ? max(n - nq + tok_hi + 1, 0) : n;
  const int pages = (lim_hi + kPage - 1) / kPage;
  const int begin = (int)((int64_t)split * pages / p.splits), end = (int)((int64_t)(split + 1) * pages / p.splits);

  bf16x8 qf[NK];
#pragma unroll
  for (int s = 0; s < NK; ++s) {
    const int col = HD == 32 ? 8 * c : 64 * (s / 2) + 16 * c + 8 * (s % 2);
    u32x4 raw{0, 0, 0, 0};
    if (in) raw = *reinterpret_cast<const u32x4*>(p.q + (q0 + tok) * p.ldq + qcol + col);
    qf[s] = __builtin_bit_cast(bf16x8, raw);
  }
  f32x4 o[NV];
#pragma unroll
  for (int t = 0; t < NV; ++t) o[t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  float m = -INFINITY, l = 0.0f;

  for (int i = begin + wave; i < end; i += NW) {
    const int page = p.c.table[(int64_t)b * p.c.max_pages + i];
    if ((uint32_t)page >= (uint32_t)p.c.n_pages) continue;
    const int64_t at = (int64_t)page * kvh + head;
    const uint8_t* kp = p.c.k + at * (kPage * HD);
    const uint8_t* vp = p.c.v + at * (kPage * HD);
    const float ks = fp8_scale(p.c.ks[at]), vs = fp8_scale(p.c.vs[at]);
    u32x4 vr[NV];
#pragma unroll
    for (int t = 0; t < NV; ++t)
      vr[t] = *reinterpret_cast<const u32x4*>(vp + (16 * t + r16) * kPage + 16 * c);
    f32x4 s[4];
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const uint8_t* kr = kp + (16 * t + r16) * HD;
      s[t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
      if constexpr (HD == 32) {
        const u32x2 w = *reinterpret_cast<const u32x2*>(kr + 8 * c);
        s[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen8(w[0], w[1], ks), qf[0], s[t], 0, 0, 0);
      } else {
#pragma unroll
        for (int h = 0; h < NK / 2; ++h) {
          const u32x4 w = *reinterpret_cast<const u32x4*>(kr + 64 * h + 16 * c);
          s[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen8(w[0], w[1], ks), qf[2 * h], s[t], 0, 0, 0);
          s[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen8(w[2], w[3], ks), qf[2 * h + 1], s[t], 0, 0, 0);
        }
      }
    }
    const int k0 = i * kPage + 4 * c;
    const bool border = (i + 1) * kPage > lim_lo;                      // some row does not see all of the page
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        s[t][e] *= p.scale;
        if (border && k0 + 16 * t + e >= lim) s[t][e] = -INFINITY;
      }
    float mx = -INFINITY;
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int e = 0; e < 4; ++e) mx = fmaxf(mx, s[t][e]);
    mx = fmaxf(mx, __shfl_xor(mx, 16));
    mx = fmaxf(mx, __shfl_xor(mx, 32));
    if (__any(mx > m)) {
      const float to = fmaxf(m, mx), f = to == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m - to);
      m = to;
      l *= f;
#pragma unroll
      for (int t = 0; t < NV; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[t][e] *= f;
    }
    const float ref = m == -INFINITY ? 0.0f : m;
    bf16x8 pf[2];
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float x = __builtin_amdgcn_exp2f(s[t][e] - ref);
        l += x;
        pf[t / 2][4 * (t % 2) + e] = (bf16)x;
      }
    if (border) {
      // Tokens behind the sample's last one were never written; and a token that only some
      // rows see may hold NaN, which times a probability of 0 would be NaN: such values count as 0
      // in the product, and rows that see one get their NaN from a count of them.
      bool odd = false;
#pragma unroll
      for (int t = 0; t < NV; ++t)
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          const int left = n - (k0 + 16 * x);                          // written ones of the word's four
          const uint32_t w = vr[t][x] & (left >= 4 ? 0xffffffffu : left <= 0 ? 0u : (1u << (8 * left)) - 1u);
          const uint32_t nb = nan_bytes(w);
          odd = odd || nb;
          vr[t][x] = w;
        }
      if (__any(odd)) {
        bf16x8 sees[2];
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
          for (int e = 0; e < 4; ++e) sees[t / 2][4 * (t % 2) + e] = (bf16)(k0 + 16 * t + e < lim ? 1.0f : 0.0f);
#pragma unroll
        for (int t = 0; t < NV; ++t) {
          f32x4 count{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const uint32_t a = nan_bytes(vr[t][2 * h]), d = nan_bytes(vr[t][2 * h + 1]);
            count = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen8(a & 0x38383838u, d & 0x38383838u, 1.0f), sees[h], count,
                                                            0, 0, 0);
            vr[t][2 * h] &= ~a;
            vr[t][2 * h + 1] &= ~d;
          }
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (count[e] > 0.0f) o[t][e] = __builtin_nanf("");
        }
      }
    }
#pragma unroll
    for (int t = 0; t < NV; ++t)
#pragma unroll
      for (int h = 0; h < 2; ++h)
        o[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen8(vr[t][2 * h], vr[t][2 * h + 1], vs), pf[h], o[t], 0, 0, 0);
  }
  l += __shfl_xor(l, 16);
  l += __shfl_xor(l, 32);
#pragma unroll
  for (int t = 0; t < NV; ++t) *reinterpret_cast<f32x4*>(&so[wave][r16][16 * t + 4 * c]) = o[t];
  if (c == 0) {
    sm[wave][r16] = m;
    sl[wave][r16] = l;
  }
  __syncthreads();
  // The waves' results, joined; four columns a thread.
  for (int x = tid; x < 16 * HD / 4; x += 64 * NW) {
    const int r = x / (HD / 4), d = x % (HD / 4) * 4;
    float top = -INFINITY;
#pragma unroll
    for (int w = 0; w < NW; ++w) top = fmaxf(top, sm[w][r]);
    float sum = 0.0f;
    f32x4 v{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      const float f = sm[w][r] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(sm[w][r] - top);
      sum += sl[w][r] * f;
      const f32x4 ov = *reinterpret_cast<const f32x4*>(&so[w][r][d]);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] += ov[e] * f;
    }
    if constexpr (SPLIT) {
      const int64_t slot = (((int64_t)split * n_tiles + tile) * kvh + head) * 16 + r;
      *reinterpret_cast<f32x4*>(p.part_o + slot * HD + d) = v;
      if (d == 0) {
        p.part_ml[2 * slot] = top;
        p.part_ml[2 * slot + 1] = sum;
      }
    } else {
      const int rr = (tile - p.tiles.off[b]) * 16 + r, t = rr / p.group;
      if (t >= nq) continue;
      const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
      bf16x4 w;
#pragma unroll
      for (int e = 0; e < 4; ++e) w[e] = (bf16)(v[e] * inv);
      *reinterpret_cast<bf16x4*>(p.o + (q0 + t) * p.ldo + (head * p.group + rr - t * p.group) * HD + d) = w;
    }
  }
}

// The splits' results, joined in their order: a thread has four columns of a row.
template <int HD>
__global__ __launch_bounds__(256) void k_cache8_join(Attn8Args p) {
  const int n_tiles = p.tiles.off[p.tiles.B], kvh = p.c.kv_heads;
  const int64_t x = (int64_t)blockIdx.x * 256 + threadIdx.x, slot = x / (HD / 4), all = (int64_t)n_tiles * kvh * 16;
  if (slot >= all) return;
  const int d = (int)(x % (HD / 4)) * 4, r = (int)(slot % 16), head = (int)(slot / 16 % kvh);
  const int tile = (int)(slot / 16 / kvh), b = find_segment(p.tiles.off, p.tiles.B, tile);
  const int row = (tile - p.tiles.off[b]) * 16 + r, t = row / p.group, q0 = p.rows.off[b];
  if (t >= p.rows.off[b + 1] - q0) return;
  float top = -INFINITY;
  for (int s = 0; s < p.splits; ++s) top = fmaxf(top, p.part_ml[2 * (s * all + slot)]);
  float sum = 0.0f;
  f32x4 v{0.0f, 0.0f, 0.0f, 0.0f};
  for (int s = 0; s < p.splits; ++s) {
    const float m = p.part_ml[2 * (s * all + slot)];
    const float f = m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m - top);
    sum += p.part_ml[2 * (s * all + slot) + 1] * f;
    const f32x4 ov = *reinterpret_cast<const f32x4*>(p.part_o + (s * all + slot) * HD + d);
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] += ov[e] * f;
  }
  const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
  bf16x4 w;
#pragma unroll
  for (int e = 0; e < 4; ++e) w[e] = (bf16)(v[e] * inv);
  *reinterpret_cast<bf16x4*>(p.o + (q0 + t) * p.ldo + (head * p.group + row - t * p.group) * HD + d) = w;
}

struct Plan {
  Segs tiles;
  int splits;
  size_t bytes(const Cache8& c) const {
    return splits < 2 ? 0 : (size_t)splits * tiles.off[tiles.B] * c.kv_heads * 16 * (c.hd + 2) * 4;
  }
};

constexpr int kWaves = 4;

Plan plan(const Cache8& c, int heads, const Segs& rows, const Lens& len) {
  Plan r{};
  const int group = heads / c.kv_heads;
  r.tiles.B = rows.B;
  int pages = 0;
  for (int b = 0; b < rows.B; ++b) {
    const int64_t n = (int64_t)(rows.off[b + 1] - rows.off[b]) * group;
    r.tiles.off[b + 1] = r.tiles.off[b] + (int)((n + 15) / 16);
    if (n) pages = std::max(pages, (len.n[b] + kPage - 1) / kPage);
  }
  const int64_t items = (int64_t)r.tiles.off[rows.B] * c.kv_heads;
  r.splits = 1;
  if (items) r.splits = (int)std::max<int64_t>(1, std::min<int64_t>(1024 / items, pages / (2 * kWaves)));
  return r;
}

template <int HD>
hipError_t launch_attn8(const Attn8Args& a, hipStream_t s) {
  const int64_t items = (int64_t)a.tiles.off[a.tiles.B] * a.c.kv_heads;
  if (!items) return hipSuccess;
  if (a.splits < 2) {
    launch((k_cache8_attn<HD, kWaves, false>), dim3((uint32_t)items), dim3(64 * kWaves), 0, s, a);
    return hipGetLastError();
  }
  launch((k_cache8_attn<HD, kWaves, true>), dim3((uint32_t)(items * a.splits)), dim3(64 * kWaves), 0, s, a);
  launch((k_cache8_join<HD>), dim3((uint32_t)((items * 16 * (HD / 4) + 255) / 256)), dim3(256), 0, s, a);
  return hipGetLastError();
}

template <typename T>
hipError_t launch_append(const AppendArgs& a, hipStream_t s) {
  const dim3 grid((uint32_t)(2 * a.pages.off[a.pages.B] * a.c.kv_heads));
  switch (a.c.hd) {
    case 32: launch((k_cache8_append<T, 32>), grid, dim3(64), 0, s, a); break;
    case 64: launch((k_cache8_append<T, 64>), grid, dim3(128), 0, s, a); break;
    case 128: launch((k_cache8_append<T, 128>), grid, dim3(256), 0, s, a); break;
    default: return hipErrorInvalidValue;
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_cache8_append(const Cache8& c, int dt, const Lens& len, const Segs& rows, const void* k, int64_t ldk,
                                const void* v, int64_t ldv, hipStream_t s) {
  AppendArgs a{c, len, rows, {}, k, v, ldk, ldv};
  a.pages.B = rows.B;
  for (int b = 0; b < rows.B; ++b) {
    const int n = rows.off[b + 1] - rows.off[b];
    a.pages.off[b + 1] = a.pages.off[b] + (n ? (len.n[b] + n + kPage - 1) / kPage - len.n[b] / kPage : 0);
  }
  if (!a.pages.off[rows.B]) return hipSuccess;
  return dt == DT_F32 ? launch_append<float>(a, s) : launch_append<bf16>(a, s);
}

size_t cache8_attention_bytes(const Cache8& c, int heads, const Segs& rows, const Lens& len, bool causal) {
  return plan(c, heads, rows, len).bytes(c);
}

hipError_t launch_cache8_attention(const Cache8& c, int heads, const Segs& rows, const Lens& len, const void* q,
                                   int64_t ldq, void* o, int64_t ldo, bool causal, bool q_scaled, void* ws,
                                   size_t ws_bytes, hipStream_t s) {
  Plan pl = plan(c, heads, rows, len);
  while (pl.splits > 1 && pl.bytes(c) > ws_bytes) --pl.splits;
  const int64_t slots = (int64_t)pl.splits * pl.tiles.off[rows.B] * c.kv_heads * 16;
  Attn8Args a{c, len, rows, pl.tiles, (const bf16*)q, (bf16*)o, ldq, ldo, heads / c.kv_heads, causal, pl.splits,
              q_scaled ? 1.0f : attention_q_scale(c.hd), (float*)ws, (float*)ws + slots * c.hd};
  switch (c.hd) {
    case 32: return launch_attn8<32>(a, s);
    case 64: return launch_attn8<64>(a, s);
    case 128: return launch_attn8<128>(a, s);
  }
  return hipErrorInvalidValue;
}

}  // namespace f3c
