// Shared by the two forms of the attention over an 8-bit paged cache: few query rows per KV head
// (serve_attn.cu) and many (serve_attn_tc.cu).
#pragma once
#include "serve_cache.cuh"
#include "tc.cuh"
#include <cuda_fp16.h>

constexpr int ATTN_HD = 128;
constexpr int ATTN_MAX_CHUNK = 16384;       // tokens of a CTA
// References of a row: m near its largest score, and d near the largest score - m + log2 of the value scale.  d is
// held relative to m, so that scores whose size leaves no bits for the value scale's log2 do not lose it.
// A weight is 2^SHIFT at the reference m + d and at most 2^(SHIFT + SLACK), below the largest fp16.
constexpr float ATTN_SHIFT = 8.f, ATTN_SLACK = 7.f;
constexpr float ATTN_NOTHING = -3.402823466e38f;   // m before the first visible token: no score is lower
constexpr float ATTN_NO_VALUE = -1e30f;     // d before the first visible token whose page has values, and its floor
constexpr float ATTN_SCALE = 0.12751743074602467f;   // log2(e) / sqrt(128)

// The part 2^e of a weight that its token's page and the references give.  e passes CAP only where the row's top
// score lies on pages whose values vanish beside this one's; a token's own part is 2^-105 or less there, and
// its weight counts for nothing, but infinity times zero would make the row NaN.  (A NaN of e passes through.)
constexpr float ATTN_CAP = 120.f;
__device__ __forceinline__ float attn_factor(float e) {
  asm("min.NaN.f32 %0, %0, %1;" : "+f"(e) : "f"(ATTN_CAP));
  return tc::ex2(e);
}

struct AttnArgs {
  omq_kv_cache c;
  int total_q, max_q; const int32_t* cu_q; int max_kv, n_heads;
  const __nv_bfloat16* Q; int64_t ldq;
  float* Of; __nv_bfloat16* Ob; int64_t ldo; float* lse;
  float* wo; float2* wl;                    // partial results of the splits (n_split > 1) and their log-sum-exp (attn_part)
  int chunk, n_split, row_tiles;
  int32_t* status;
  const uint32_t* seen; int words;          // draft trees (serve_tree.cuh): bits of the newest tokens that each row sees
};

// Draft trees: the newest tokens that a row sees, from node d of its sequence (d below zero: context, which every row
// sees) on, as 64 bits.  bits: the row's words.
__device__ __forceinline__ uint64_t attn_window(const uint32_t* bits, int words, int nq, int d) {
  if (d <= -64) return ~0ull;
  if (d >= nq) return 0ull;
  auto word = [&](int w) { return w < words ? (uint64_t)__ldg(bits + w) : 0ull; };
  uint64_t x;
  const int w = max(d, 0) >> 5, s = max(d, 0) & 31;
  x = (word(w) | word(w + 1) << 32) >> s;
  if (s) x |= word(w + 2) << (64 - s);
  const int left = nq - max(d, 0);                            // nodes from there on
  if (left < 64) x &= (1ull << left) - 1;
  return d < 0 ? x << -d | ((1ull << -d) - 1) : x;
}


// two codes (bytes 0, 1 or 2, 3 of w) as fp16 integers code - 128
__device__ __forceinline__ uint32_t codes_lo(uint32_t w) {
  const uint32_t u = __byte_perm(w, 0x64646464u, 0x4140);
  const __half2 h = __hsub2(*reinterpret_cast<const __half2*>(&u), __half2half2(__ushort_as_half(0x6480)));
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ uint32_t codes_hi(uint32_t w) {
  const uint32_t u = __byte_perm(w, 0x64646464u, 0x4342);
  const __half2 h = __hsub2(*reinterpret_cast<const __half2*>(&u), __half2half2(__ushort_as_half(0x6480)));
  return *reinterpret_cast<const uint32_t*>(&h);
}

__device__ __forceinline__ uint32_t pack_half2(float lo, float hi) {
  const __half2 h = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}

// Four channels (4 lane ..) of query row `row` of KV head g (zeros from `rows` on) times 2^*sh: the power of two that puts the
// row's largest magnitude in [2^13, 2^14) (capped where 2^sh would overflow).  Warp-collective.
__device__ __forceinline__ void attn_query4(const AttnArgs& a, const SeqRows& s, int g, int rep, int row, int rows, int lane,
                                            float (&v)[4], int* sh) {
  uint2 u = make_uint2(0, 0);
  if (row < rows)
    u = __ldg(reinterpret_cast<const uint2*>(a.Q + (int64_t)(s.row0 + row / rep) * a.ldq + (g * rep + row % rep) * ATTN_HD + 4 * lane));
  v[0] = __uint_as_float(u.x << 16); v[1] = __uint_as_float(u.x & 0xffff0000u);
  v[2] = __uint_as_float(u.y << 16); v[3] = __uint_as_float(u.y & 0xffff0000u);
  uint32_t big = 0;
#pragma unroll
  for (int e = 0; e < 4; ++e) big = max(big, __float_as_uint(v[e]) & 0x7fffffffu);
  big = __reduce_max_sync(0xffffffffu, big);
  *sh = big == 0 ? 0 : min(13 + 127 - (int)(big >> 23), 126);
  const float up = __uint_as_float((uint32_t)(127 + *sh) << 23);
#pragma unroll
  for (int e = 0; e < 4; ++e) v[e] *= up;
}

// Log-sum-exp of a part of a row's tokens (reference m, sum L), and what its rounding to fp32 left out.  Parts are weighed by
// 2^ of it: from 4096 on the rounding would count beside the fp16 weights' 2^-11, and at 2^24 a part of ten tokens with the top
// score would weigh what a part of one does.  Below, the rest is taken as nothing.
__device__ __forceinline__ float2 attn_part(float m, float L) {
  if (L == 0.f) return make_float2(-INFINITY, 0.f);           // (a NaN score is not an empty row)
  const float lg = log2f(L), lse = m + lg;
  return make_float2(lse, fabsf(lse) < 4096.f ? 0.f : lg - (lse - m));
}

// page record i of a chunk that starts at page `first`: id (-1 and the status word where it is out of range),
// key scale times log2(e) / sqrt(128), log2 of the value scale
__device__ __forceinline__ void attn_page(const AttnArgs& a, int b, int g, int page, int* id_out, float* ks, float* lv) {
  int id = page < a.c.max_pages ? __ldg(a.c.page_table + (int64_t)b * a.c.max_pages + page) : -1;
  if (id < 0 || id >= a.c.n_pages) {
    omq_set_status(a.status, OMQ_ERR_INVALID_ARG);
    id = -1;
  }
  *id_out = id;
  const int64_t at = (int64_t)(id < 0 ? 0 : id) * a.c.n_kv + g;
  *ks = __ldg(a.c.k_scale + at) * ATTN_SCALE;
  *lv = log2f(__ldg(a.c.v_scale + at));
}

// the launch for many query rows per KV head
omq_status attn_tc_launch(cudaStream_t st, const AttnArgs& a);
constexpr int ATTN_TC_ROWS = 128;           // its query rows per CTA
