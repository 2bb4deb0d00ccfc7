// What the attention kernels share: arguments, the sequences' ranges, and how rows are cut.
//
// The rows of a sequence and key head are its new tokens times the g query heads that share the key head, row r being token r / g,
// head r % g, so that cached keys and values are read once for all of them.  The cached tokens of a sequence start at the first
// that any of its rows sees, rounded down to 64, and may be cut into splits of `chunk` tokens, each with its own softmax statistics; a
// second kernel joins them.
//
// Statistics are kept in units that take the scale of the values along: with x = log2(e) scale q k + e_v (e_v: exponent of the scale of v
// in j's page) the accumulators hold  o = sum 2^(x - m) v8,  l = sum 2^(x - m - e_v),  so that a page's scale costs no work on
// the accumulators, and the weights, fp16 for the second product, are largest where their product with v is.  The reference m
// only moves when a tile's largest x is more than 8 above it (weights reach 2^8, far from fp16's largest number); the result is o / l.
// Exponents of pages differ by up to 120: beside a page of huge values 2^(x - m) of a page of zeros or tiny ones may be no fp32 number where its part of l still counts.  Rows that
// met an exponent below kTiny therefore form l once more at their end, as the sum of 2^(x - e_v - m), from the keys alone.  (Above kTiny what is lost is below 2^-46 of l.  Formed in
// each tile, even behind a branch, it cost 4 % of 64 sequences of 8192.)
#pragma once
#include "ccq_layer.h"

namespace ccq {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8_t;
typedef __attribute__((ext_vector_type(8))) _Float16 f16x8_t;

struct AttnArgs {
  const uint8_t *k, *v, *ks, *vs;
  const uint16_t* q;
  uint16_t* out;
  int64_t q_token, q_head, o_token, o_head;
  const int32_t *offsets, *lens, *table;
  int64_t ld_table;
  float* part_o;    // [split][token row][q head][D]
  float* part_ml;   // [split][token row][q head][2]
  uint8_t* images;        // [batch][kv head][image_tiles], for the kernel for many rows
  float* image_scales;    // the same, eight numbers each
  int32_t pages, page_shift, kv_heads, q_heads, group, table_width, batch, tokens, max_new, max_len;
  int32_t causal, window;
  int32_t splits;   // at most so many pieces
  int32_t row_tiles, tile_rows, image_tiles;
  float c;          // scale * log2(e)
};

constexpr float kLowest = -3.0e38f;   // the reference before any token is seen
constexpr float kRise = 8.f;
constexpr int kTiny = -20;
// l times 2^d, where 2^d alone may be no fp32 number.
__device__ __forceinline__ float rescaled(float l, float d) {
  const float half = __builtin_amdgcn_exp2f(0.5f * d);
  return l * half * half;
}

struct AttnSequence {
  int first, n, old, len;   // first token row, new tokens, tokens before them, cached tokens with them
};
__device__ __forceinline__ int first_seen(const AttnArgs& a, int p) { return a.window > 0 ? max(0, p - a.window + 1) : 0; }
__device__ __forceinline__ AttnSequence attn_sequence(const AttnArgs& a, int b) {
  AttnSequence s;
  s.first = max(a.offsets[b], 0);
  s.n = min(a.offsets[b + 1], a.tokens) - s.first;
  s.len = a.lens[b];
  s.old = s.len - s.n;
  s.n = min(s.n, a.max_new);
  s.len = min(min(s.len, a.max_len), (int)min((int64_t)a.table_width << a.page_shift, (int64_t)0x7FFFFFFF));
  return s;
}
// Cached tokens [first, second) that the row at position p sees.
__device__ __forceinline__ int seen_end(const AttnArgs& a, const AttnSequence& s, int p) { return a.causal ? min(max(p + 1, 0), s.len) : s.len; }

// Rows [first_row, last_row] of a tile and what they see: any of them, all of them; the tokens from `begin` on in `splits` pieces of `chunk`.  The pieces go by
// the sequence's own length, not by the bound that the grid was made for: a program whose max_len is what its page table holds has them too.
constexpr int kUnit = 256;   // tokens of the smallest piece
struct AttnTile {
  int first_row, last_row;
  int any_lo, any_hi, all_lo, all_hi, begin;
  int chunk, splits;
};
__device__ __forceinline__ AttnTile attn_tile(const AttnArgs& a, const AttnSequence& s, int first_row, int rows) {
  AttnTile t;
  t.first_row = first_row;
  t.last_row = min(first_row + rows, s.n * a.group) - 1;
  const int p_first = s.old + t.first_row / a.group, p_last = s.old + t.last_row / a.group;
  t.any_lo = first_seen(a, p_first);
  t.any_hi = seen_end(a, s, p_last);
  t.all_lo = first_seen(a, p_last);
  t.all_hi = seen_end(a, s, p_first);
  t.begin = min(t.any_lo, max(s.len, 0)) & ~63;
  const int units = (max(t.any_hi - t.begin, 1) - 1) / kUnit + 1, per = (units - 1) / a.splits + 1;
  t.chunk = per > 0x7FFFFFFF / kUnit ? 0x7FFFFFFF : per * kUnit;
  t.splits = (units - 1) / per + 1;
  return t;
}

__device__ __forceinline__ f16x8_t values_f16(uint32_t lo, uint32_t hi) {
  typedef __attribute__((ext_vector_type(2))) _Float16 pair;
  const pair a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)lo, 1.f, false), b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)lo, 1.f, true);
  const pair c = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)hi, 1.f, false), d = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)hi, 1.f, true);
  return f16x8_t{a.x, a.y, b.x, b.y, c.x, c.y, d.x, d.y};
}
__device__ __forceinline__ bf16x8_t values_bf16(uint32_t lo, uint32_t hi, float scale) {
  typedef __attribute__((ext_vector_type(2))) __bf16 pair;
  const pair a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)lo, scale, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)lo, scale, true);
  const pair c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)hi, scale, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)hi, scale, true);
  return bf16x8_t{a.x, a.y, b.x, b.y, c.x, c.y, d.x, d.y};
}
// A scale's byte.  Pages that no row sees (missing: the first page's is read in their place; in a tile that starts before the window) may hold any byte, and what is masked has to
// stay finite beside it: 0 would make a masked score of -inf times 0, 255 a sum of weights of 0 times infinity.
__device__ __forceinline__ int cache_byte(int byte) { return min(max(byte, 127 - kCacheExp), 127 + kCacheExp); }
// Whether one of the pages of tokens [from, to) has tiny values (kTiny): looked at where a kernel met a small exponent, which may be that of a page no row sees.
__device__ __forceinline__ bool tiny_pages(const AttnArgs& a, int b, int head, int lane, int from, int to) {
  bool tiny = false;
  for (int i = (from >> a.page_shift) + lane; i <= (to - 1) >> a.page_shift; i += 64) {
    const int page = a.table[b * a.ld_table + i];
    if (page < 0 || page >= a.pages) continue;
    const int byte = a.vs[(int64_t)page * a.kv_heads + head];
    tiny |= byte >= 127 - kCacheExp && byte < 127 + kTiny;
  }
  return __any(tiny);
}
// The bytes of 16 neighbouring slots from token t0 on whose tokens lie in [lo, hi); the others become zero.
__device__ __forceinline__ u32x4_t keep_tokens(u32x4_t v, int t0, int lo, int hi) {
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const int from = min(max(lo - t0 - 4 * w, 0), 4), to = min(max(hi - t0 - 4 * w, 0), 4);
    const uint32_t below_to = (uint32_t)((1ull << (8 * to)) - 1), below_from = (uint32_t)((1ull << (8 * from)) - 1);
    v[w] &= below_to & ~below_from;
  }
  return v;
}

// The kernels for many rows, of 128 dimensions: workgroups of kManyRows; a.row_tiles counts them.  Before it the tiles of 64 cached tokens that a sequence's
// rows see, from image_begin on, are converted to images of kImageBytes.
constexpr int kManyRows = 256, kImageBytes = 64 * 128 * 4;
__device__ __forceinline__ int image_begin(const AttnArgs& a, const AttnSequence& s) { return min(first_seen(a, s.old), max(s.len, 0)) & ~63; }
int launch_attention_rows(const AttnArgs& a, void* stream);

}  // namespace ccq
