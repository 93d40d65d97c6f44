// The cache of 8-bit keys and values (cache8.h): appending to it, and attention over it.
#include <algorithm>
#include <cmath>
#include <type_traits>
#include <utility>

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
//
// Many tokens are bound by HBM, behind a workgroup's chain of table, rows, maximum and store: four
// samples of 1374 tokens, 16 heads of 64, take 8.9 us (27 MB, 5.3 us at a copy's rate), the
// next tokens of 32 sequences, 8 heads of 128, 5.0 us, all of it the chain.
template <typename T, int HD>
__global__ __launch_bounds__(2 * HD) void k_cache8_append(AppendArgs p) {
  __shared__ float part[(2 * HD + 63) / 64];
  const int tid = threadIdx.x, heads = p.c.kv_heads;
  int item = blockIdx.x;
  const bool is_v = item & 1;
  item >>= 1;
  const int head = item % heads, pg = item / heads;
  const int b = find_segment_wave(p.pages.off, p.pages.B, pg);
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
  Segs rows;
  // Samples by falling length: the y-th longest is order[y], its row tiles (of tile_rows rows: token,
  // head of the group) are tiles.off[y].., its items (tiles times splits of its pages)
  // items.off[y]..
  Segs tiles, items;
  uint8_t order[kMaxBatch];
  const bf16* q;
  bf16* o;
  int64_t ldq, ldo;
  int group, causal, tile_rows, split_pages;       // split_pages: of one split
  float scale;                                     // of the scores, to base 2
  float* part_o;                                   // [items][kv_heads][tile_rows][hd]: unnormalised outputs
  float* part_ml;                                  // and [..][tile_rows][2]: reference max, sum
};

// A workgroup's work. Workgroups go round the XCDs in turn: heads are fastest, so that an XCD
// (with its L2) sees few of them, and the longest items come first (later rows' under a
// causal mask, and longer samples').
struct Item {
  int item, head, b, tile, splits, split;
};
__device__ __forceinline__ Item item_of(const Attn8Args& p) {
  Item r;
  r.item = blockIdx.x / p.c.kv_heads;
  r.head = blockIdx.x - r.item * p.c.kv_heads;
  const int y = find_segment_wave(p.items.off, p.items.B, r.item);
  r.b = p.order[y];
  const int tiles = p.tiles.off[y + 1] - p.tiles.off[y], local = r.item - p.items.off[y];
  r.splits = (p.items.off[y + 1] - p.items.off[y]) / tiles;
  const int back = local / r.splits;
  r.tile = tiles - 1 - back;
  r.split = local - back * r.splits;
  return r;
}

// Eight e4m3 values times a scale, as bf16: no rounding (4 significant bits).
__device__ __forceinline__ bf16x8 widen8(uint32_t lo, uint32_t hi, float scale) {
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false);
  const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false);
  const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

typedef float f32x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ uint32_t pack2(float a, float b) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{a, b}), bf16x2));
}

// The largest of v over lanes l, l ^ 16, l ^ 32, l ^ 48, in all of them.
__device__ __forceinline__ float quarter_max(float v) {
  float w = v;
  asm("s_nop 1\n\tv_permlane16_swap_b32 %0, %1\n\ts_nop 1" : "+v"(v), "+v"(w));
  v = fmaxf(v, w);
  w = v;
  asm("s_nop 1\n\tv_permlane32_swap_b32 %0, %1\n\ts_nop 1" : "+v"(v), "+v"(w));
  return fmaxf(v, w);
}

// Bytes 0xff where a word's e4m3 bytes are NaN.
__device__ __forceinline__ uint32_t nan_bytes(uint32_t w) {
  const uint32_t top = ((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;     // 0x7f carries into its own top bit alone
  return (top >> 7) * 0xffu;
}

// 16 rows (queries of one key head's group) a workgroup, whose waves take its pages in
// turn, fragments straight from memory into registers, a page ahead; scores S^T = K Q^T, so
// that a lane holds one row's scores and its statistics.
//
// Single queries of long sequences are bound by HBM: 32 of up to 16384 tokens, 8 key heads of
// 128, 32 query heads, 147 us, 5.1 TB/s; a short one by latency: 16 heads of 64, 1374 tokens
// 7.6 us. Eight waves up to a workgroup for each CU, beyond that four: over 1374 tokens of 64
// columns 16 workgroups take 8.1 us with eight and 8.7 with four, 256 9.6 and 10.7, 304 14.4 and
// 12.0, 512 17.4 and 15.5.
template <int HD, int NW>
__global__ __launch_bounds__(64 * NW, HD == 128 ? 2 : 3) void k_cache8_attn(Attn8Args p) {
  constexpr int NK = HD / 32, NV = HD / 16;        // K slices of 32 columns; output tiles of 16
  constexpr int KR = HD == 32 ? 1 : HD / 64;       // 16-byte (of 32 columns 8-byte) pieces of K a lane has of 16 tokens
  typedef std::conditional_t<HD == 32, u32x2, u32x4> KPiece;
  __shared__ __attribute__((aligned(16))) float so[NW][16][HD + 4];
  __shared__ float sm[NW][16], sl[NW][16];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int c = lane >> 4, r16 = lane & 15;
  const Item it = item_of(p);
  const int kvh = p.c.kv_heads, b = it.b, head = it.head, item = it.item;
  const int q0 = p.rows.off[b], nq = p.rows.off[b + 1] - q0, n = p.len.n[b];
  const int row = it.tile * 16 + r16, tok = row / p.group;
  const bool in = tok < nq;
  const int qcol = (head * p.group + row - tok * p.group) * HD;
  // a row sees keys below its limit; the tile those below the last row's
  const int lim = !in ? 0 : p.causal ? max(min(n, n - nq + tok + 1), 0) : n;
  const int lim_lo = p.causal ? n - nq + it.tile * 16 / p.group + 1 : n;
  const int lim_hi = p.causal ? max(n - nq + min((it.tile * 16 + 15) / p.group, nq - 1) + 1, 0) : n;
  const int pages = (lim_hi + kPage - 1) / kPage;
  const int begin = min(it.split * p.split_pages, pages), end = min(begin + p.split_pages, pages);

  // This wave's pages, 64 of them at a time: one a lane, its number (or none) and scales.
  int pg = -1, base = 0;
  float pks = 0.0f, pvs = 0.0f;
  auto look = [&](int k) {
    base = k;
    pg = -1;
    const int i = begin + wave + (k + lane) * NW;
    if (i < end) pg = p.c.table[(int64_t)b * p.c.max_pages + i];
    if ((uint32_t)pg >= (uint32_t)p.c.n_pages) pg = -1;
    if (pg >= 0) {
      const int64_t x = (int64_t)pg * kvh + head;
      pks = fp8_scale(p.c.ks[x]);
      pvs = fp8_scale(p.c.vs[x]);
    }
  };
  const int mine = (end - begin - wave + NW - 1) / NW;               // pages (or none) of this wave
  if (mine > 0) look(0);
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

  // K of the next page is asked for as soon as this one's scores are taken, V at a page's
  // beginning. (A page that is none is passed over: its loads too.)
  KPiece kr[4 * KR];
  u32x4 vr[NV];
  auto page_of = [&](int k) { return __builtin_amdgcn_readlane(pg, k - base); };
  auto load_k = [&](int k) __attribute__((always_inline)) {
    const int page = page_of(k);
    if (page < 0) return;
    const uint8_t* kp = p.c.k + ((int64_t)page * kvh + head) * (kPage * HD);
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int h = 0; h < KR; ++h)
        kr[t * KR + h] = *reinterpret_cast<const KPiece*>(kp + (uint32_t)((16 * t + r16) * HD + 64 * h + (int)sizeof(KPiece) * c));
  };
  // What a page's scores s add to the rows: the maxima, probabilities, the product with V.
  auto take_page = [&](auto border_, int i, f32x4 (&s)[4], float vs) __attribute__((always_inline)) {
    constexpr bool BORDER = decltype(border_)::value;
    const int k0 = i * kPage + 4 * c;
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        s[t][e] *= p.scale;
        if (BORDER && k0 + 16 * t + e >= lim) s[t][e] = -INFINITY;
      }
    float mx = -INFINITY;
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int e = 0; e < 4; ++e) mx = fmaxf(mx, s[t][e]);
    mx = quarter_max(mx);
    const float to = fmaxf(m, mx);
    const float f = to == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m - to), ref = to == -INFINITY ? 0.0f : to;
    m = to;
    l *= f;
    u32x4 pf[2];
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      float x[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        x[e] = __builtin_amdgcn_exp2f(s[t][e] - ref);
        l += x[e];
      }
      pf[t / 2][2 * (t % 2)] = pack2(x[0], x[1]);
      pf[t / 2][2 * (t % 2) + 1] = pack2(x[2], x[3]);
    }
#pragma unroll
    for (int t = 0; t < NV; ++t) {
      u32x4 w = vr[t];
#pragma unroll
      for (int e = 0; e < 4; ++e) o[t][e] *= f;
      if constexpr (BORDER) {
        // Tokens behind the sample's last one were never written; and a token that only some
        // rows see may hold NaN, which times a probability of 0 would be NaN: such values count
        // as 0 in the product, and rows that see one get their NaN from a count of them.
        uint32_t odd = 0;
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          const int left = n - (k0 + 16 * x);                          // written ones of the word's four
          w[x] &= left >= 4 ? 0xffffffffu : left <= 0 ? 0u : (1u << (8 * left)) - 1u;
          odd |= nan_bytes(w[x]);
        }
        if (__any(odd)) {
          f32x4 count{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            bf16x8 sees;
#pragma unroll
            for (int e = 0; e < 8; ++e) sees[e] = (bf16)(k0 + 32 * h + 16 * (e / 4) + e % 4 < lim ? 1.0f : 0.0f);
            const uint32_t a = nan_bytes(w[2 * h]), d = nan_bytes(w[2 * h + 1]);
            count = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen8(a & 0x38383838u, d & 0x38383838u, 1.0f), sees, count, 0,
                                                            0, 0);
            w[2 * h] &= ~a;
            w[2 * h + 1] &= ~d;
          }
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (count[e] > 0.0f) o[t][e] = __builtin_nanf("");
        }
      }
#pragma unroll
      for (int h = 0; h < 2; ++h)
        o[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen8(w[2 * h], w[2 * h + 1], vs),
                                                       __builtin_bit_cast(bf16x8, pf[h]), o[t], 0, 0, 0);
    }
  };
  for (int k = 0; k < mine; ++k) {
    if (k % 64 == 0) {
      if (k) look(k);
      load_k(k);
    }
    const int page = page_of(k);
    if (page < 0) {
      if (k + 1 < mine && (k + 1) % 64) load_k(k + 1);
      continue;
    }
    {
      const uint8_t* vp = p.c.v + ((int64_t)page * kvh + head) * (kPage * HD);
#pragma unroll
      for (int t = 0; t < NV; ++t)
        vr[t] = *reinterpret_cast<const u32x4*>(vp + (uint32_t)((16 * t + r16) * kPage + 16 * c));
    }
    __builtin_amdgcn_sched_barrier(0);
    const int i = begin + wave + k * NW;
    const float ks = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, pks), k - base));
    const float vs = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, pvs), k - base));
    f32x4 s[4];
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      s[t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int h = 0; h < KR; ++h) {
        const KPiece w = kr[t * KR + h];
        s[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen8(w[0], w[1], ks), qf[HD == 32 ? 0 : 2 * h], s[t], 0, 0, 0);
        if constexpr (HD > 32)
          s[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen8(w[2], w[3], ks), qf[2 * h + 1], s[t], 0, 0, 0);
      }
    }
    __builtin_amdgcn_sched_barrier(0);
    if (k + 1 < mine && (k + 1) % 64) load_k(k + 1);
    __builtin_amdgcn_sched_barrier(0);
    if ((i + 1) * kPage > lim_lo) take_page(std::true_type{}, i, s, vs);           // some row does not see all of it
    else take_page(std::false_type{}, i, s, vs);
  }
  l = rows_sum(l);
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
    const int rr = it.tile * 16 + r, t = rr / p.group;
    if (t >= nq) continue;
    if (it.splits > 1) {
      const int64_t slot = ((int64_t)item * kvh + head) * 16 + r;
      *reinterpret_cast<f32x4*>(p.part_o + slot * HD + d) = v;
      if (d == 0) {
        p.part_ml[2 * slot] = top;
        p.part_ml[2 * slot + 1] = sum;
      }
    } else {
      const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
      bf16x4 w;
#pragma unroll
      for (int e = 0; e < 4; ++e) w[e] = (bf16)(v[e] * inv);
      *reinterpret_cast<bf16x4*>(p.o + (q0 + t) * p.ldo + (head * p.group + rr - t * p.group) * HD + d) = w;
    }
  }
}

// What lane ^ 32 holds beside v: the larger of the two, or their sum, in both.
__device__ __forceinline__ float half_max(float v) {
  float w = v;
  asm("s_nop 1\n\tv_permlane32_swap_b32 %0, %1\n\ts_nop 1" : "+v"(v), "+v"(w));
  return fmaxf(v, w);
}
__device__ __forceinline__ float half_sum(float v) {
  float w = v;
  asm("s_nop 1\n\tv_permlane32_swap_b32 %0, %1\n\ts_nop 1" : "+v"(v), "+v"(w));
  return v + w;
}

// f(std::integral_constant<int, I>) for I = 0 .. N - 1, unrolled.
template <typename F, int... I>
__device__ __forceinline__ void static_for_seq(F f, std::integer_sequence<int, I...>) {
  (f(std::integral_constant<int, I>{}), ...);
}
template <int N, typename F>
__device__ __forceinline__ void static_for(F f) {
  static_for_seq(f, std::make_integer_sequence<int, N>{});
}

// The largest of a tile's 16 scores, in dependent v_max3 (fmaxf would quiet each operand
// first). The first step is a builtin, for which the compiler waits until the matrix
// core has written the tile; it does not for what inline assembly reads. NaN is passed over
// (or makes the maximum infinite); its row is NaN all the same.
__device__ __forceinline__ float max16(const f32x16& v) {
  float r = __builtin_amdgcn_fmed3f(v[0], v[1], INFINITY);
  asm("v_max3_f32 %0, %0, %1, %2\n\t"
      "v_max3_f32 %0, %0, %3, %4\n\t"
      "v_max3_f32 %0, %0, %5, %6\n\t"
      "v_max3_f32 %0, %0, %7, %8\n\t"
      "v_max3_f32 %0, %0, %9, %10\n\t"
      "v_max3_f32 %0, %0, %11, %12\n\t"
      "v_max3_f32 %0, %0, %13, %14"
      : "+&v"(r)
      : "v"(v[2]), "v"(v[3]), "v"(v[4]), "v"(v[5]), "v"(v[6]), "v"(v[7]), "v"(v[8]), "v"(v[9]), "v"(v[10]), "v"(v[11]),
        "v"(v[12]), "v"(v[13]), "v"(v[14]), "v"(v[15]));
  return r;
}

typedef short s16x4 __attribute__((ext_vector_type(4)));

// What is read in place of a page that is none: zeros.
__device__ const u32x4 kNoPage[64] = {};

// Many rows: NW waves of 32 QB rows each share a page, which goes to LDS by DMA as it
// is, STAGES deep, its 16-byte chunks swizzled by row for conflict-free fragment reads;
// fragments are widened as they are read. Scores on 32 x 32 instructions, S^T = K Q^T.
//
// Pages that all rows of a wave see go in half steps of 32 keys: the matrix cores take the
// scores of the next 32 keys and the product with V of the 32 before while the vector
// unit takes the probabilities of these, instruction by instruction (a barrier to the
// compiler's scheduler behind each group; left alone it gathers the products and then the
// vector work, and both waves of a SIMD wait for the same unit). Pages at a row's limit, at
// most a few and the last, go one step after the other, with masks.
//
// NG groups of waves share the tile's pages, each with a ring of stages of its own, and are
// joined in LDS. One group alone on a CU has a wave a SIMD, which waits for its own matrix
// instructions: 1.5 us a page of 128 columns where two workgroups take 1.2 each. So few tiles
// take two groups (16 heads, 2048 queries over 5003 tokens, 128 columns: 117 us with one, 92
// with two), many tiles one, whose workgroups hide each other's beginnings and ends (4096
// over 4096: 145 against 149).
//
// Bound by vector issue: at 9831 queries over 32768 tokens, 16 heads of 64 (1371 us, 962 TFLOP/s),
// it is busy 63% of the cycles (exponentials and roundings to bf16 half of that, widening a
// quarter), the matrix pipes 46%; over 1374 tokens (32768 queries, 211 us, 873 TFLOP/s) the first
// and the last of 22 pages show. 64 rows a wave (QB 2) share each widening: 1744 us with 32 there.
template <int HD, int QB, int NW, int NG>
__global__ __launch_bounds__(64 * NW * NG, 2) void k_cache8_rows(Attn8Args p) {
  constexpr int ROWS = 32 * QB * NW, TILE = kPage * HD, STAGES = 5;
  constexpr int NS = HD / 32, NV = HD / 32;        // pairs of K slices of 16 columns; output tiles of 32
  constexpr int CPR = HD / 16;                     // 16-byte chunks of a row of K
  constexpr int DMA = TILE / 1024;                 // DMA instructions per tile
  constexpr int DQ = 2 * DMA / NW;                 // of both tiles, per wave
  static_assert(2 * DMA % NW == 0, "whole DMA blocks per wave");
  constexpr int RING = STAGES * 2 * TILE;
  constexpr int PARTS = 64 * NW * QB * (HD / 2 + 2) * 4;               // a group's results, for the join
  static_assert(NG == 1 || PARTS <= NG * RING, "the second group's sums fit");
  __shared__ __attribute__((aligned(16))) char lds[NG * RING];
  const int tid = threadIdx.x, lane = tid & 63, of_all = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wave = of_all % NW, group = of_all / NW;
  const int g = lane >> 5, r32 = lane & 31;
  const Item it = item_of(p);
  const int kvh = p.c.kv_heads, b = it.b, head = it.head, item = it.item;
  const int q0 = p.rows.off[b], nq = p.rows.off[b + 1] - q0, n = p.len.n[b];
  const int row_t = it.tile * ROWS, row_w = row_t + wave * 32 * QB;
  // A lane's row: its token and its columns (found anew for the output, not kept)
  auto place = [&](int lane_row, int& tok, int& col) {
    tok = (row_w + lane_row) / p.group;
    col = (head * p.group + row_w + lane_row - tok * p.group) * HD;
  };
  int lim[QB];
  bf16x8 qf[QB][2 * NS];
#pragma unroll
  for (int j = 0; j < QB; ++j) {
    int tok, col;
    place(r32 + 32 * j, tok, col);
    lim[j] = tok >= nq ? 0 : p.causal ? max(min(n, n - nq + tok + 1), 0) : n;
    // columns of a lane's fragment 2 i + h: 32 i + 16 g + 8 h on, as a chunk of K holds them
#pragma unroll
    for (int s = 0; s < 2 * NS; ++s) {
      u32x4 raw{0, 0, 0, 0};
      if (tok < nq)
        raw = *reinterpret_cast<const u32x4*>(p.q + (q0 + tok) * p.ldq + col + 32 * (s / 2) + 16 * g + 8 * (s % 2));
      qf[j][s] = __builtin_bit_cast(bf16x8, raw);
    }
  }
  // the wave's lowest limit, its highest, the workgroup's highest
  const int lim_lo = p.causal ? n - nq + row_w / p.group + 1 : n;
  const int lim_w = row_w >= nq * p.group ? 0
                    : p.causal ? max(n - nq + min((row_w + 32 * QB - 1) / p.group, nq - 1) + 1, 0) : n;
  const int lim_hi = p.causal ? max(n - nq + min((row_t + ROWS - 1) / p.group, nq - 1) + 1, 0) : n;
  const int pages = (lim_hi + kPage - 1) / kPage;
  // (a group's pages: as many for each, for the barriers that they meet at; from `held` on they
  // are none)
  const int begin0 = min(it.split * p.split_pages, pages), held = min(begin0 + p.split_pages, pages);
  const int share = (held - begin0 + NG - 1) / NG, begin = begin0 + group * share, end = begin + share;

  // o: outputs; m: the reference that probabilities are relative to, base 2; l: sums of a
  // lane's own keys. Where masks apply the reference is moved above 2^8 times it; in whole pages
  // no maximum is taken: a step whose probabilities bring a sum above kMost is taken
  // back and the reference moved to the maximum or what the sum stands for, the larger.
  // (Rounding is relative, so a reference far below the maximum costs nothing; sums of 2^24
  // leave outputs of values up to 2^100 within range. What is below 2^-102 of a row's largest
  // probability may count as none: exponentials end at 2^-126.)
  // Whole pages take their exponents by one fma, which rounds s c - m once, where m is a
  // rounded s c: the largest key's is half a last place of m off 0. Up to kNear that is 2^-13 at
  // most: nothing beside keys of the same score in pages that round s c first, as those with
  // masks do, and a step behind a moved reference adds less than 2^13 to a sum and is kept.
  // Rows further out (finite: infinite scores are NaN in any way) take their pages one step after
  // the other.
  constexpr float kMost = 0x1p24f, kNear = 0x1p12f;
  f32x16 o[QB][NV];
  float m[QB];
  f32x4 l[QB];
#pragma unroll
  for (int j = 0; j < QB; ++j) {
    m[j] = -INFINITY;
    l[j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int t = 0; t < NV; ++t)
#pragma unroll
      for (int e = 0; e < 16; ++e) o[j][t][e] = 0.0f;
  }
  // K: rows of CPR chunks, physical chunk = chunk ^ (row / (16 / CPR)) % CPR, so that 16
  // lanes reading a chunk of 16 rows meet 16 different places of 256 bytes; V: rows of 4.
  auto kswz = [](int row) { return row / (16 / CPR) & (CPR - 1); };
  auto vswz = [](int row) { return row >> 2 & 3; };
  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)lds + (uint32_t)(group * RING);
  // A lane's place within the 1 KiB that a DMA instruction reads (the same for all of a
  // wave's: blocks are NW apart, and only their parity enters, of 128 columns alone).
  static_assert(NW % 2 == 0, "a wave's blocks are all even or all odd");
  const uint32_t kdma = (uint32_t)(lane / CPR * HD + ((lane % CPR ^ kswz(64 / CPR * wave + lane / CPR)) << 4));
  const uint32_t vdma = (uint32_t)(lane / 4 * 64 + ((lane % 4 ^ vswz(lane / 4)) << 4));
  // Fragment reads: rows r32 (and 32 further) of the tiles, chunks 2 x + g.
  uint32_t kof[NS], vof[2];
#pragma unroll
  for (int x = 0; x < NS; ++x) kof[x] = lds0 + (uint32_t)(r32 * HD + ((2 * x + g ^ kswz(r32)) << 4));
#pragma unroll
  for (int x = 0; x < 2; ++x) vof[x] = lds0 + (uint32_t)(TILE + r32 * 64 + ((2 * x + g ^ vswz(r32)) << 4));
  typedef __attribute__((address_space(3))) const u32x4 lds_u32x4;
  typedef __attribute__((address_space(3))) const u32x2 lds_u32x2;
  auto read_k = [&](uint32_t at, int h, int x) { return *(lds_u32x4*)(uintptr_t)(kof[x] + at + (uint32_t)(h * 32 * HD)); };
  auto read_v = [&](uint32_t at, int h, int t, int x) {               // words of tokens 32 h on
    return *(lds_u32x2*)(uintptr_t)(vof[x] + at + (uint32_t)(t * 32 * 64 + 8 * h));
  };
  auto fence = [] { __builtin_amdgcn_sched_barrier(0); };
  const f32x16 zero = {};

  // The pages from `base` on, one a lane: its number (or none), its scales.
  int pg = -1, base = 0;
  float pks = 0.0f, pvs = 0.0f;
  auto look = [&](int at) {
    base = at;
    pg = -1;
    if (at + lane < held) pg = p.c.table[(int64_t)b * p.c.max_pages + at + lane];
    if ((uint32_t)pg >= (uint32_t)p.c.n_pages) pg = -1;
    const int64_t x = (int64_t)(pg < 0 ? 0 : pg) * kvh + head;
    pks = pg < 0 ? 1.0f : fp8_scale(p.c.ks[x]);
    pvs = pg < 0 ? 1.0f : fp8_scale(p.c.vs[x]);
  };
  auto lane_f = [](float v, int i) {
    return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), i));
  };
  // (s_nop: the load's base, a scalar write of M0, wants one wait state, which the compiler does not place before
  // inline assembly)
  auto fetch = [&](int i, int stage) {             // page i (of those looked up)
    const int page = __builtin_amdgcn_readlane(pg, i - base);
    const int64_t at = ((int64_t)page * kvh + head) * TILE;
#pragma unroll
    for (int q = 0; q < DQ; ++q) {
      const int blk = wave + NW * q, of = blk < DMA ? blk : blk - DMA;
      const uint8_t* from = page < 0 ? reinterpret_cast<const uint8_t*>(kNoPage)
                                     : (blk < DMA ? p.c.k : p.c.v) + at + of * 1024;
      const uint32_t to = lds0 + (uint32_t)(stage * 2 * TILE + blk * 1024);
      asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %0, %1"
                   : : "v"(blk < DMA ? kdma : vdma), "s"(from), "{m0}"(to) : "memory");
    }
  };
  // The reference of block j moves to `to`: what was summed up is scaled.
  auto rescale = [&](int j, float to) __attribute__((always_inline)) {
    const float f = to == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m[j] - to);
    m[j] = to;
#pragma unroll
    for (int e = 0; e < 4; ++e) l[j][e] *= f;
#pragma unroll
    for (int t = 0; t < NV; ++t)
#pragma unroll
      for (int e = 0; e < 16; ++e) o[j][t][e] *= f;
  };
  auto row_sum = [](const bf16x8& f, f32x4 acc) {  // of a lane's own values: 4 x 4 blocks, ones on the left
    const s16x4 one = {0x3f80, 0x3f80, 0x3f80, 0x3f80};
    union { bf16x8 b; s16x4 h[2]; } u{f};
    acc = __builtin_amdgcn_mfma_f32_4x4x4bf16_1k(one, u.h[0], acc, 0, 0, 0);
    return __builtin_amdgcn_mfma_f32_4x4x4bf16_1k(one, u.h[1], acc, 0, 0, 0);
  };

  // Scores of the 32 keys at kat, not interleaved with anything.
  auto scores = [&](uint32_t kat, float ks, f32x16 (&s)[QB]) __attribute__((always_inline)) {
#pragma unroll
    for (int x = 0; x < NS; ++x) {
      const u32x4 w = read_k(kat, 0, x);
      const bf16x8 a = widen8(w[0], w[1], ks), c = widen8(w[2], w[3], ks);
#pragma unroll
      for (int j = 0; j < QB; ++j) {
        s[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, qf[j][2 * x], x ? s[j] : zero, 0, 0, 0);
        s[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(c, qf[j][2 * x + 1], s[j], 0, 0, 0);
      }
      fence();
    }
  };
  // A page with masks (or its second half), one step after the other; none for keys behind all of the wave's limits
  // (1374 tokens end 30 into a page: 32768 queries 244 -> 235 us).
  auto masked_page = [&](int i, int half, uint32_t at, float ks, float vs) __attribute__((always_inline)) {
    // (tokens counted from the lane's first; opaque, or the compiler keeps 64 sums over all pages)
    const int from = i * kPage + 32 * half + 4 * g;
    int there = n - from, seen[QB];
    asm("" : "+v"(there));
#pragma unroll
    for (int j = 0; j < QB; ++j) {
      seen[j] = lim[j] - from;
      asm("" : "+v"(seen[j]));
    }
#pragma unroll 1
    for (int h = half; h < 2 && i * kPage + 32 * h < lim_w; ++h) {
      f32x16 s[QB];
      scores(at + (uint32_t)(h * 32 * HD), ks, s);
      u32x4 pf[QB][2];
#pragma unroll
      for (int j = 0; j < QB; ++j) {
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if (8 * (e / 4) + e % 4 >= seen[j]) s[j][e] = -INFINITY;
        const float mx = half_max(max16(s[j])) * p.scale;
        if (__any(mx - m[j] > 8.0f)) rescale(j, fmaxf(m[j], mx));      // (a difference: m + 8 may be m)
        // (the product rounded as the reference was: what an fma leaves of a score of 2^33 is 2^8, and
        // the largest key's probability 0 or infinite)
        const float ref = m[j] == -INFINITY ? 0.0f : m[j];
#pragma unroll
        for (int e = 0; e < 16; e += 2)
          pf[j][e / 8][e / 2 % 4] = pack2(__builtin_amdgcn_exp2f(s[j][e] * p.scale - ref),
                                          __builtin_amdgcn_exp2f(s[j][e + 1] * p.scale - ref));
#pragma unroll
        for (int u = 0; u < 2; ++u) l[j] = row_sum(__builtin_bit_cast(bf16x8, pf[j][u]), l[j]);
        fence();
      }
#pragma unroll
      for (int t = 0; t < NV; ++t) {
        u32x2 v[2];
        // (as for 16 rows: what was never written counts as 0, and NaN where it is seen)
        uint32_t odd = 0;
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          v[x] = read_v(at, h, t, x);
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            const int left = there - 16 * u - 8 * x;
            v[x][u] &= left >= 4 ? 0xffffffffu : left <= 0 ? 0u : (1u << (8 * left)) - 1u;
            odd |= nan_bytes(v[x][u]);
          }
        }
        if (__any(odd)) {
#pragma unroll
          for (int j = 0; j < QB; ++j) {
            f32x16 count = zero;
#pragma unroll
            for (int u = 0; u < 2; ++u) {
              bf16x8 sees;
#pragma unroll
              for (int e = 0; e < 8; ++e)
                sees[e] = (bf16)(16 * u + 8 * (e / 4) + e % 4 < seen[j] ? 1.0f : 0.0f);
              count = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
                  widen8(nan_bytes(v[0][u]) & 0x38383838u, nan_bytes(v[1][u]) & 0x38383838u, 1.0f), sees, count, 0, 0, 0);
            }
#pragma unroll
            for (int e = 0; e < 16; ++e)
              if (count[e] > 0.0f) o[j][t][e] = __builtin_nanf("");
            fence();
          }
#pragma unroll
          for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int u = 0; u < 2; ++u) v[x][u] &= ~nan_bytes(v[x][u]);
        }
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const bf16x8 vf = widen8(v[0][u], v[1][u], vs);
#pragma unroll
          for (int j = 0; j < QB; ++j)
            o[j][t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, __builtin_bit_cast(bf16x8, pf[j][u]), o[j][t], 0, 0, 0);
        }
        fence();
      }
      there -= 32;
#pragma unroll
      for (int j = 0; j < QB; ++j) seen[j] -= 32;
    }
  };

  // Half step: scores `next` of the 32 keys at `kat`, probabilities pc of `cur` (against the
  // reference -ref), the product of pp with the 32 tokens of V at `vat`.
  auto product_v = [&](uint32_t vat, float vs, const u32x4 (&pp)[QB][2]) __attribute__((always_inline)) {
#pragma unroll
    for (int t = 0; t < NV; ++t) {
      const u32x2 a = read_v(vat, 0, t, 0), c = read_v(vat, 0, t, 1);
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const bf16x8 vf = widen8(a[u], c[u], vs);
#pragma unroll
        for (int j = 0; j < QB; ++j)
          o[j][t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, __builtin_bit_cast(bf16x8, pp[j][u]), o[j][t], 0, 0, 0);
      }
      fence();
    }
  };
  auto half_step = [&](uint32_t kat, float ks, uint32_t vat, float vs, const float (&ref)[QB], const f32x16 (&cur)[QB],
                       f32x16 (&next)[QB], const u32x4 (&pp)[QB][2], u32x4 (&pc)[QB][2]) __attribute__((always_inline)) {
    // Fragments (K and V in turn), groups of one product each, probabilities. A fragment is
    // widened a group before its first product, a wave's next product issued only when the
    // matrix core is about done with the one before (in order, it would hold up what follows).
    constexpr int F = 4 * NS, G = F * QB, N = 16 * QB;
    u32x4 kr[2];                                   // raw fragments of K (a pair of slices each)
    u32x2 vr[2][2];                                // and of V (an output tile each)
    bf16x8 frag[2];
    float ex[N];
    auto widen = [&](auto xc) {
      constexpr int x = decltype(xc)::value, a = x / 2;
      if constexpr (x % 2 == 0) frag[0] = widen8(kr[a / 2 % 2][2 * (a % 2)], kr[a / 2 % 2][2 * (a % 2) + 1], ks);
      else frag[1] = widen8(vr[a / 2 % 2][0][a % 2], vr[a / 2 % 2][1][a % 2], vs);
    };
    kr[0] = read_k(kat, 0, 0);
    vr[0][0] = read_v(vat, 0, 0, 0);
    vr[0][1] = read_v(vat, 0, 0, 1);
    widen(std::integral_constant<int, 0>{});
    fence();
    static_for<G>([&](auto nc) {
      constexpr int y = decltype(nc)::value, x = y / QB, j = y % QB, a = x / 2;
      if constexpr (j == 0 && x % 4 == 0 && x + 4 < F) {
        kr[(a / 2 + 1) % 2] = read_k(kat, 0, a / 2 + 1);
        vr[(a / 2 + 1) % 2][0] = read_v(vat, 0, a / 2 + 1, 0);
        vr[(a / 2 + 1) % 2][1] = read_v(vat, 0, a / 2 + 1, 1);
      }
      if constexpr (x % 2 == 0)
        next[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag[0], qf[j][a], a ? next[j] : zero, 0, 0, 0);
      else
        o[j][a / 2] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag[1], __builtin_bit_cast(bf16x8, pp[j][a % 2]), o[j][a / 2],
                                                              0, 0, 0);
      // exponentials, converted a group later
      constexpr int E0 = y * N / G, E1 = (y + 1) * N / G, C0 = y ? (y - 1) * N / G & ~1 : 0,
                    C1 = y + 1 == G ? N : E0 & ~1;
      static_for<E1 - E0>([&](auto k) {
        constexpr int i = E0 + decltype(k)::value;
        ex[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(cur[i / 16][i % 16], p.scale, ref[i / 16]));
      });
      if constexpr (j == QB - 1 && x + 1 < F) widen(std::integral_constant<int, x + 1>{});
      static_for<(C1 - C0) / 2>([&](auto k) {
        constexpr int i = C0 + 2 * decltype(k)::value;
        pc[i / 16][i / 8 % 2][i / 2 % 4] = pack2(ex[i], ex[i + 1]);
        if constexpr (i % 8 == 6) l[i / 16] = row_sum(__builtin_bit_cast(bf16x8, pc[i / 16][i / 8 % 2]), l[i / 16]);
      });
      fence();
    });
  };

  for (int first = begin; first < end; first += 64) {
    const int last = min(first + 64, end);
    __syncthreads();                               // every wave past its reads of the last stages
    look(first);
    wait_vm<0>();
#pragma unroll
    for (int i = 0; i < STAGES - 2; ++i) fetch(min(first + i, last - 1), i);
    wait_vm<(STAGES - 3) * DQ>();
    __builtin_amdgcn_s_barrier();                  // the first page has landed
    fence();
    int stage = 0;                                 // of page i
    int synced = -1;                               // the last page that the next was called for
    auto sync = [&](int i) {                       // page i + 1 has landed, the stage of i - 2 is free
      synced = i;
      wait_vm<(STAGES - 4) * DQ>();
      __builtin_amdgcn_s_barrier();
      fence();
      fetch(min(i + STAGES - 2, last - 1), stage >= 2 ? stage - 2 : stage + STAGES - 2);
    };
    auto none = [&](int i) { return __builtin_amdgcn_readlane(pg, i - base) < 0; };
    auto at_stage = [&](int s) { return (uint32_t)(s * 2 * TILE); };
    auto after = [&](int s) { return s == STAGES - 1 ? 0 : s + 1; };
    // Pages that all of the wave's rows see, in half steps. A segment of them ends where the
    // reference has to move (a branch within the loop would copy the outputs at every step):
    // it starts with scores of its own and no probabilities before them. Where a reference is
    // beyond kNear, the rest of the pages looked up go like those with masks.
    const int whole = row_w >= nq * p.group ? first : min(max(lim_lo / kPage, first), last);
    int t = 2 * first;
    while (t < 2 * whole) {
      int i = t / 2;
      f32x16 s0[QB];
      scores(at_stage(stage) + (uint32_t)(32 * HD * (t % 2)), lane_f(pks, i - base), s0);
      bool far = false;
#pragma unroll
      for (int j = 0; j < QB; ++j) {
        const float mx = half_max(max16(s0[j])) * p.scale, sum = half_sum(l[j][0]);
        if (!none(i) && __any(mx > m[j] + 8.0f || sum > 0x1p12f))
          rescale(j, fmaxf(fmaxf(m[j], mx), m[j] + __builtin_amdgcn_logf(sum)));
        const float off = __builtin_fabsf(m[j]);
        far = far || (off > kNear && off < INFINITY);
      }
      if (__any(far)) break;
      f32x16 s1[QB];
      u32x4 p0[QB][2], p1[QB][2];                  // (pairs, as bf16)
#pragma unroll
      for (int j = 0; j < QB; ++j) p1[j][0] = p1[j][1] = u32x4{0, 0, 0, 0};
      uint32_t vat = at_stage(stage) + (uint32_t)(8 * (t % 2));      // (zeros times V of this page, which every row sees)
      float vsb = lane_f(pvs, i - base);
      // A half step at t, then whether the segment ends. Where it has ended already (behind the
      // first of a pair: the loop has one exit, or the outputs would be copied at it), it is
      // no step: the product with pp and no probabilities.
      bool done = false;
      auto step = [&](const f32x16 (&cur)[QB], f32x16 (&next)[QB], const u32x4 (&pp)[QB][2], u32x4 (&pc)[QB][2])
                      __attribute__((always_inline)) {
        const bool second = t % 2;
        if (!done && !second && synced != i) sync(i);
        // (behind the last half step scores of this page again: the next one may hold NaN that not
        // all rows see, which no step may take)
        const bool next_page = second && t + 1 < 2 * whole;
        const int nx = next_page ? i + 1 : i;
        const uint32_t here = at_stage(stage), kat = next_page ? at_stage(after(stage)) : here + 32 * HD;
        // (a page that is none: its scores are 0 and its probabilities 0)
        float ref[QB], before[QB];
#pragma unroll
        for (int j = 0; j < QB; ++j) {
          ref[j] = done || none(i) ? -INFINITY : -m[j];
          before[j] = l[j][0];
        }
        half_step(kat, lane_f(pks, nx - base), vat, vsb, ref, cur, next, pp, pc);
        bool much = false;
#pragma unroll
        for (int j = 0; j < QB; ++j) much = much || l[j][0] > kMost;
        if (__any(much)) {                         // rare; the step is taken again in the next segment
#pragma unroll
          for (int j = 0; j < QB; ++j) {
            l[j][0] = before[j];
            pc[j][0] = pc[j][1] = u32x4{0, 0, 0, 0};
          }
          done = true;
        } else if (!done) {
          vat = here + (uint32_t)(8 * (t % 2));
          vsb = lane_f(pvs, i - base);
          if (second) ++i, stage = after(stage);
          done = ++t == 2 * whole;
        }
      };
      do {
        step(s0, s1, p1, p0);
        step(s1, s0, p0, p1);
      } while (!done);
      product_v(vat, vsb, p1);
    }
    for (int i = t / 2, half = t % 2; i < last; ++i, half = 0) {
      if (synced != i) sync(i);
      const uint32_t at = at_stage(stage);
      stage = after(stage);
      if (!none(i) && i * kPage < lim_w) masked_page(i, half, at, lane_f(pks, i - base), lane_f(pvs, i - base));
    }
  }
  wait_vm<0>();                                    // no DMA into LDS that another workgroup may get
  float sums[QB];
#pragma unroll
  for (int j = 0; j < QB; ++j) sums[j] = half_sum(l[j][0]);
  if constexpr (NG > 1) {                          // the second group's results, into the first's
    typedef __attribute__((address_space(3))) f32x4 lds_f4;
    typedef __attribute__((address_space(3))) float lds_f;
    const uint32_t all = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)lds;
    const uint32_t at4 = all + (uint32_t)((wave * QB * NV * 256 + lane) * 16);
    const uint32_t at1 = all + (uint32_t)(NW * QB * NV * 4096 + (wave * QB * 128 + lane) * 4);
    __syncthreads();
    if (group) {
#pragma unroll
      for (int j = 0; j < QB; ++j) {
#pragma unroll
        for (int t = 0; t < NV; ++t)
#pragma unroll
          for (int e = 0; e < 16; e += 4)
            *(lds_f4*)(uintptr_t)(at4 + (uint32_t)((j * NV + t) * 4096 + e * 256)) =
                f32x4{o[j][t][e], o[j][t][e + 1], o[j][t][e + 2], o[j][t][e + 3]};
        *(lds_f*)(uintptr_t)(at1 + (uint32_t)(j * 512)) = m[j];
        *(lds_f*)(uintptr_t)(at1 + (uint32_t)(j * 512 + 256)) = sums[j];
      }
    }
    __syncthreads();
    if (group) return;
#pragma unroll
    for (int j = 0; j < QB; ++j) {
      const float m1 = *(lds_f*)(uintptr_t)(at1 + (uint32_t)(j * 512)), top = fmaxf(m[j], m1);
      const float f0 = m[j] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m[j] - top);
      const float f1 = m1 == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m1 - top);
      m[j] = top;
      sums[j] = sums[j] * f0 + *(lds_f*)(uintptr_t)(at1 + (uint32_t)(j * 512 + 256)) * f1;
#pragma unroll
      for (int t = 0; t < NV; ++t)
#pragma unroll
        for (int e = 0; e < 16; e += 4) {
          const f32x4 v = *(lds_f4*)(uintptr_t)(at4 + (uint32_t)((j * NV + t) * 4096 + e * 256));
#pragma unroll
          for (int x = 0; x < 4; ++x) o[j][t][e + x] = o[j][t][e + x] * f0 + v[x] * f1;
        }
    }
  }
#pragma unroll
  for (int j = 0; j < QB; ++j) {
    const float sum = sums[j];
    int again = r32 + 32 * j, tok, col;
    asm("" : "+v"(again));
    place(again, tok, col);
    if (tok >= nq) continue;
    if (it.splits > 1) {
      const int64_t slot = ((int64_t)item * kvh + head) * ROWS + wave * 32 * QB + again;
#pragma unroll
      for (int t = 0; t < NV; ++t)
#pragma unroll
        for (int e = 0; e < 16; e += 4)
          *reinterpret_cast<f32x4*>(p.part_o + slot * HD + 32 * t + 2 * e + 4 * g) =
              f32x4{o[j][t][e], o[j][t][e + 1], o[j][t][e + 2], o[j][t][e + 3]};
      if (g == 0) {
        p.part_ml[2 * slot] = m[j];
        p.part_ml[2 * slot + 1] = sum;
      }
    } else {
      const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
      bf16* out = p.o + (q0 + tok) * p.ldo + col;
#pragma unroll
      for (int t = 0; t < NV; ++t)
#pragma unroll
        for (int e = 0; e < 16; e += 4) {
          bf16x4 w;
#pragma unroll
          for (int x = 0; x < 4; ++x) w[x] = (bf16)(o[j][t][e + x] * inv);
          *reinterpret_cast<bf16x4*>(out + 32 * t + 2 * e + 4 * g) = w;
        }
    }
  }
}

// The splits' results, joined in their order: a thread has four columns of a row. (A wave's
// rows are of one tile.)
template <int HD>
__global__ __launch_bounds__(256) void k_cache8_join(Attn8Args p) {
  const int kvh = p.c.kv_heads, x = blockIdx.x * 256 + threadIdx.x, d = x % (HD / 4) * 4, y = x / (HD / 4);
  const int r = y % p.tile_rows, z = __builtin_amdgcn_readfirstlane(y / p.tile_rows), head = z % kvh, tile = z / kvh;
  if (tile >= p.tiles.off[p.tiles.B]) return;
  const int s0 = find_segment_wave(p.tiles.off, p.tiles.B, tile), b = p.order[s0], q0 = p.rows.off[b];
  const int tiles = p.tiles.off[s0 + 1] - p.tiles.off[s0], splits = (p.items.off[s0 + 1] - p.items.off[s0]) / tiles;
  const int back = tile - p.tiles.off[s0], row = (tiles - 1 - back) * p.tile_rows + r, t = row / p.group;
  if (splits < 2 || t >= p.rows.off[b + 1] - q0) return;
  const int64_t step = (int64_t)kvh * p.tile_rows;
  const int64_t slot = ((int64_t)(p.items.off[s0] + back * splits) * kvh + head) * p.tile_rows + r;
  float top = -INFINITY;
  for (int s = 0; s < splits; ++s) top = fmaxf(top, p.part_ml[2 * (slot + s * step)]);
  float sum = 0.0f;
  f32x4 v{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 4
  for (int s = 0; s < splits; ++s) {
    const float m = p.part_ml[2 * (slot + s * step)];
    const float f = m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m - top);
    sum += p.part_ml[2 * (slot + s * step) + 1] * f;
    const f32x4 ov = *reinterpret_cast<const f32x4*>(p.part_o + (slot + s * step) * HD + d);
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] += ov[e] * f;
  }
  const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
  bf16x4 w;
#pragma unroll
  for (int e = 0; e < 4; ++e) w[e] = (bf16)(v[e] * inv);
  *reinterpret_cast<bf16x4*>(p.o + (q0 + t) * p.ldo + (head * p.group + row - t * p.group) * HD + d) = w;
}

// How a call is cut: row tiles, and splits of the pages of their sample.
struct Plan {
  Segs tiles, items;
  uint8_t order[kMaxBatch];
  int rows, groups, split_pages;                   // rows: of a tile; groups: that share a tile's pages
  bool split;                                      // some sample's pages are split
  size_t bytes(const Cache8& c) const {
    return split ? (size_t)items.off[items.B] * c.kv_heads * rows * (c.hd + 2) * 4 : 0;
  }
};

// What a form of the kernel takes, in us on MI355X: a page of one workgroup's rows while a CU has
// one of them (first) or more (page, each), and what a workgroup costs beside its pages (own).
// Of 16 rows, page is a CU's throughput and first the time from page to page of one wave.
// Fitted to 33000 timings of all forms and up to 64 splits over 3060 calls (1 to 32 samples of 64 to
// 40000 tokens, 1 to 9000 queries, 1 to 16 key heads, groups of 1 to 7, causal or not): the
// pick takes 1% longer than the best of them in the mean, 6% or less in 95 of 100 calls, 32% at
// worst (ragged calls of a few pieces for each CU).
struct FormCost {
  int rows, hd, groups;
  double first, page, own;
};
constexpr FormCost kForms[] = {
    {16, 32, 1, 0.78, 0.101, 0.35}, {16, 64, 1, 1.32, 0.155, 0.53}, {16, 128, 1, 2.99, 0.431, 1.23},
    {128, 32, 1, 0.97, 0.425, 0.63}, {128, 64, 1, 0.92, 0.658, 1.3}, {128, 128, 1, 1.38, 1.075, 3.5},
    {128, 32, 2, 0.61, 0.447, 1.5}, {128, 64, 2, 0.63, 0.772, 3.3}, {128, 128, 2, 0.96, 1.229, 7.5},
    {256, 32, 1, 1.05, 0.893, 2.1}, {256, 64, 1, 1.63, 1.101, 3.3},
    {256, 32, 2, 0.82, 0.903, 3.3}, {256, 64, 2, 0.97, 1.171, 4.7},
};
constexpr double kLaunchUs = 5.5, kJoinUs = 3.0, kJoinSplitUs = 0.29, kPartialBytesPerUs = 7.5e6, kReadBytesPerUs = 5e6;
constexpr double kSplitRounds = 1.1;               // splits of what fills the CUs without: partial results in their way
constexpr int kLeastSplit = 8;                     // pages

Plan plan(const Cache8& c, int heads, const Segs& rows, const Lens& len, bool causal, size_t ws_bytes) {
  Plan best{};
  const int group = heads / c.kv_heads, B = rows.B;
  int pages[kMaxBatch];
  int64_t most_rows = 0;
  for (int b = 0; b < B; ++b) {
    pages[b] = (len.n[b] + kPage - 1) / kPage;
    best.order[b] = (uint8_t)b;
    most_rows = std::max(most_rows, (int64_t)(rows.off[b + 1] - rows.off[b]) * group);
  }
  std::stable_sort(best.order, best.order + B, [&](int x, int y) { return pages[x] > pages[y]; });
  bool ragged = causal;                            // pieces of different length
  for (int b = 1; b < B; ++b) ragged = ragged || len.n[b] != len.n[0];
  int longest = 1;
  for (int y = B - 1; y >= 0; --y)
    if (rows.off[best.order[y] + 1] > rows.off[best.order[y]]) longest = std::max(pages[best.order[y]], 1);
  double best_t = 0.0;
  for (const FormCost& f : kForms) {
    if (f.hd != c.hd || (f.rows > 16 && most_rows <= 16)) continue;
    int tiles[kMaxBatch];
    double work = 0.0, read = 0.0, whole = 0.0;    // pages of all tiles and heads; bytes; items without splits
    for (int y = 0; y < B; ++y) {
      const int b = best.order[y], nq = rows.off[b + 1] - rows.off[b];
      tiles[y] = (int)(((int64_t)nq * group + f.rows - 1) / f.rows);
      const double unseen = !causal || !nq ? 0.0                       // in the mean of its rows
                            : nq <= len.n[b] ? nq / (2.0 * kPage)
                                             : pages[b] - pages[b] * (double)len.n[b] / (2.0 * nq);
      const double seen = pages[b] - unseen;
      work += tiles[y] * std::max(seen, 0.5) * c.kv_heads;
      whole += (double)tiles[y] * c.kv_heads;
      if (tiles[y]) read += 2.0 * pages[b] * kPage * c.hd * c.kv_heads;
    }
    for (int k = 1; k <= 128; k = k < 4 ? k + 1 : k * 2) {
      const int p = (longest + k - 1) / k;
      if (k > 1 && p < kLeastSplit) break;
      int64_t all = 0;
      for (int y = 0; y < B; ++y) all += (int64_t)tiles[y] * std::max(1, (pages[best.order[y]] + p - 1) / p);
      const double items = (double)all * c.kv_heads, need = k < 2 ? 0.0 : items * f.rows * (c.hd + 2) * 4.0;
      // (a launch has fewer than 2^32 threads; the join's count is 32 bits and signed)
      if (k > 1 && (need > (double)ws_bytes || items >= (1 << 23) || items * f.rows * (c.hd / 4) >= 2147483648.0)) break;
      const double per_cu = items / 256.0, load = work / 256.0;
      double t;
      if (f.rows == 16) {
        t = std::max({load * f.page + per_cu * f.own, p * f.first / (items <= 256.0 ? 8.0 : 4.0), read / kReadBytesPerUs});
      } else if (per_cu <= 1.0) {
        t = p * f.first + f.own;
      } else {
        double longest_cu;                         // pages of the CU that has most
        if (ragged) {
          // lengths evenly from p down to `least`: one workgroup at a time, the 256th and the next
          // share a CU; two at a time, the first and the 257th
          const double mean = load / per_cu, least = std::max(2.0 * mean - p, 0.0), next = p - (p - least) / per_cu;
          longest_cu = std::max(f.groups > 1 ? 2.0 * next : p + next, load + (f.groups > 1 ? 0.33 : 0.38) * mean);
        } else {
          longest_cu = load * (1.0 + (std::ceil(per_cu) / per_cu - 1.0) * (f.groups > 1 ? 0.89 : 0.97));
        }
        t = std::max(p * f.first, longest_cu * f.page) + per_cu * f.own;
      }
      t += kLaunchUs + (k > 1 ? kJoinUs + kJoinSplitUs * k + 2.0 * need / kPartialBytesPerUs : 0.0);
      if (k > 1 && f.rows > 16 && whole > 256.0) t *= kSplitRounds;
      if (best_t == 0.0 || t < best_t) {
        best_t = t;
        best.rows = f.rows;
        best.groups = f.groups;
        best.split_pages = p;
      }
    }
  }
  best.tiles.B = best.items.B = B;
  for (int y = 0; y < B; ++y) {
    const int b = best.order[y];
    const int n = (int)(((int64_t)(rows.off[b + 1] - rows.off[b]) * group + best.rows - 1) / best.rows);
    const int splits = std::max(1, (pages[b] + best.split_pages - 1) / best.split_pages);
    best.tiles.off[y + 1] = best.tiles.off[y] + n;
    best.items.off[y + 1] = best.items.off[y] + n * splits;
    best.split = best.split || (splits > 1 && n);
  }
  return best;
}

template <int HD, int QB>
void launch_rows(const Attn8Args& a, const Plan& pl, uint32_t items, hipStream_t s) {
  if (pl.groups == 2) launch((k_cache8_rows<HD, QB, 4, 2>), dim3(items), dim3(512), 0, s, a);
  else launch((k_cache8_rows<HD, QB, 4, 1>), dim3(items), dim3(256), 0, s, a);
}

template <int HD>
hipError_t launch_attn8(const Attn8Args& a, const Plan& pl, hipStream_t s) {
  const int64_t items = (int64_t)a.items.off[a.items.B] * a.c.kv_heads;
  if (!items) return hipSuccess;
  if (pl.rows == 256) {
    if constexpr (HD < 128) launch_rows<HD, 2>(a, pl, (uint32_t)items, s);
  } else if (pl.rows == 128) launch_rows<HD, 1>(a, pl, (uint32_t)items, s);
  else if (items <= 256) launch((k_cache8_attn<HD, 8>), dim3((uint32_t)items), dim3(512), 0, s, a);
  else launch((k_cache8_attn<HD, 4>), dim3((uint32_t)items), dim3(256), 0, s, a);
  if (pl.split) {
    const int64_t threads = (int64_t)a.tiles.off[a.tiles.B] * a.c.kv_heads * pl.rows * (HD / 4);
    launch((k_cache8_join<HD>), dim3((uint32_t)((threads + 255) / 256)), dim3(256), 0, s, a);
  }
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
  return plan(c, heads, rows, len, causal, ~(size_t)0).bytes(c);
}

hipError_t launch_cache8_attention(const Cache8& c, int heads, const Segs& rows, const Lens& len, const void* q,
                                   int64_t ldq, void* o, int64_t ldo, bool causal, bool q_scaled, void* ws,
                                   size_t ws_bytes, hipStream_t s) {
  const Lens held = c.n_pages ? len : Lens{};      // no pages: no tokens
  const Plan pl = plan(c, heads, rows, held, causal, ws_bytes);
  const int64_t slots = (int64_t)pl.items.off[rows.B] * c.kv_heads * pl.rows;
  Attn8Args a{c, held, rows, pl.tiles, pl.items, {}, (const bf16*)q, (bf16*)o, ldq, ldo, heads / c.kv_heads, causal,
              pl.rows, pl.split_pages, q_scaled ? 1.0f : attention_q_scale(c.hd), (float*)ws,
              (float*)ws + slots * c.hd};
  std::copy(pl.order, pl.order + rows.B, a.order);
  switch (c.hd) {
    case 32: return launch_attn8<32>(a, pl, s);
    case 64: return launch_attn8<64>(a, pl, s);
    case 128: return launch_attn8<128>(a, pl, s);
  }
  return hipErrorInvalidValue;
}

}  // namespace f3c
