// Keys and values in 8 bits: pages of 64 tokens, for each key head a tile of K and a
// tile of V in e4m3 with one power-of-two scale each (E8M0 bytes, as fp8.h's blocks).
//
// A tile of K is [64 tokens][hd]. A tile of V is transposed, [hd][64], its tokens in
// the order in which a lane of the matrix cores takes them: the scores' accumulators
// hold, for each of four lane groups c, keys 16t + 4c + e (e < 4), and the product with
// V wants a group's keys side by side, so that token 16t + 4c + e lies at 16c + 4t + e:
// 16 bytes a lane, one load, no transposition of V or of the probabilities.
#pragma once

#include "kernels.h"

namespace f3c {

constexpr int kPage = 64;                          // tokens

struct Cache8 {
  uint8_t* k;                                      // [n_pages][kv_heads][64][hd]
  uint8_t* v;                                      // [n_pages][kv_heads][hd][64]
  uint8_t* ks;                                     // [n_pages][kv_heads]
  uint8_t* vs;
  const int32_t* table;                            // [batch][max_pages]: a sample's pages in order
  int kv_heads, hd, n_pages, max_pages;
};

// Tokens that each sample's cache holds, by value.
struct Lens {
  int n[kMaxBatch];
};

// rows.off[b]..rows.off[b+1] of k and v (f32 or bf16, head h at columns h * hd) become
// tokens len[b].. of sample b.
hipError_t launch_cache8_append(const Cache8& c, int dt, const Lens& len, const Segs& rows, const void* k, int64_t ldk,
                                const void* v, int64_t ldv, hipStream_t s);

// Bytes of workspace that the launch below makes use of (0: none).
size_t cache8_attention_bytes(const Cache8& c, int heads, const Segs& rows, const Lens& len, bool causal);

// o = softmax(q K^T scale) V in bf16 for the queries of rows, head h over key head h /
// (heads / kv_heads); causal: a sample's queries are its last tokens. q_scaled: the
// queries hold the softmax scale (attention_q_scale).
hipError_t launch_cache8_attention(const Cache8& c, int heads, const Segs& rows, const Lens& len, const void* q,
                                   int64_t ldq, void* o, int64_t ldo, bool causal, bool q_scaled, void* ws,
                                   size_t ws_bytes, hipStream_t s);

}  // namespace f3c
