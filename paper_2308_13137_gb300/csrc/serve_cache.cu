// Write of new tokens into the pages of an 8-bit cache (omq_kv_append): rotary positions, the
// [Q, K] LET scale and the per-(page, head) quantizer in one launch.
//
// A CTA owns one (sequence, page, KV head, K or V): it holds the page's new tokens in registers,
// takes their largest magnitude over the block, settles the scale, rounds the older codes of the page
// again where the scale grew, and writes the new ones; so no value is read twice and no two CTAs
// touch one scale.  The other CTAs of the launch turn the q rows.  The bound is HBM for prompts
// (rows in, q / k / v values and codes out): 2048 rows of 32 + 2 x 32 fp32 heads 38.5 us, 4.4 TB/s; 64 single
// tokens of 32 + 2 x 8 heads 7.6 us, of which 4 us are the launch and the chain length -> page -> scale -> rows.
// Eight threads to a token: with sixteen, of half the channels and 8-byte stores, the rotary loads and the
// addresses were a larger part of the instructions (44.0 us; fp32 pages of 128 tokens 63.0 against 53.1 us).
//
// Every operation is one fp32 rounding (no fused multiply-add), so that the codes and scales are
// the same as those of any implementation that rounds in the stated order.
#include "attn.cuh"
#include "serve_cache.cuh"

namespace {

constexpr int HD = 128;
constexpr int NT = 256;              // eight threads per token or q head, 8 + 8 channels (j, j + 64) each
constexpr int GRP = NT / 8;          // tokens or heads per pass
constexpr int QPASS = 2;             // q heads per eight threads

struct AppendArgs {
  omq_kv_cache c;
  int total_q, max_q; const int32_t* cu_q; int n_heads;
  const void* QKV; int64_t ld;
  const float2* rope; int n_pos; const float* sa;
  __nv_bfloat16* Qo; int64_t ldq; __nv_bfloat16 *Ko, *Vo; int64_t ldkv;
  int kv_units;
  int32_t* status;
};

template <bool BF>
__device__ __forceinline__ void load8(const void* base, int64_t off, float (&v)[8]) {
  if (BF) {
    unpack_bf16x8(__ldg(reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(base) + off)), v);
  } else {
    const float4* p = reinterpret_cast<const float4*>(static_cast<const float*>(base) + off);
    const float4 a = __ldg(p), b = __ldg(p + 1);
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
  }
}

// rotate-half pair of channels j .. j+7 and j+64 .. j+71 at position pos
__device__ __forceinline__ void turn(const float2* rope, int pos, int j, float (&a)[8], float (&b)[8]) {
  const float4* p = reinterpret_cast<const float4*>(rope + (int64_t)pos * 64 + j);
  float4 u[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) u[i] = __ldg(p + i);
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float c = e & 1 ? u[e >> 1].z : u[e >> 1].x, s = e & 1 ? u[e >> 1].w : u[e >> 1].y;
    const float x = a[e], y = b[e];
    a[e] = __fsub_rn(__fmul_rn(x, c), __fmul_rn(y, s));
    b[e] = __fadd_rn(__fmul_rn(y, c), __fmul_rn(x, s));
  }
}

template <bool BF>
__device__ __forceinline__ void q_unit(const AppendArgs& a, const SeqRows& s, int unit) {
  const int grp = threadIdx.x >> 3, j = 8 * (threadIdx.x & 7);
  const int rep = a.n_heads / a.c.n_kv;
#pragma unroll
  for (int p = 0; p < QPASS; ++p) {
    const int idx = (unit * QPASS + p) * GRP + grp;
    const int i = idx / a.n_heads, h = idx - i * a.n_heads;
    if (i >= s.nq) return;
    const int64_t row = s.row0 + i;
    float x[8], y[8];
    load8<BF>(a.QKV, row * a.ld + h * HD + j, x);
    load8<BF>(a.QKV, row * a.ld + h * HD + j + 64, y);
    turn(a.rope, s.len - s.nq + i, j, x, y);
    if (a.sa) {
      float u[8], w[8];
      load8<false>(a.sa, (h / rep) * HD + j, u);
      load8<false>(a.sa, (h / rep) * HD + j + 64, w);
#pragma unroll
      for (int e = 0; e < 8; ++e) { x[e] = __fdiv_rn(x[e], u[e]); y[e] = __fdiv_rn(y[e], w[e]); }
    }
    __nv_bfloat16* o = a.Qo + row * a.ldq + h * HD + j;
    *reinterpret_cast<uint4*>(o) = pack_bf16x8(x);
    *reinterpret_cast<uint4*>(o + 64) = pack_bf16x8(y);
  }
}

// new code of a value under a positive scale, moved by 128
__device__ __forceinline__ float code_of(float v, float scale) {
  return fminf(fmaxf(rintf(__fdiv_rn(v, scale)), -127.f), 127.f);
}

template <bool BF, int NP>
__global__ void __launch_bounds__(NT) kv_append_kernel(const AppendArgs a) {
  __shared__ uint32_t red[NT / 32];
  const int b = blockIdx.y;
  const SeqRows s = seq_rows(a.c, a.cu_q, a.max_q, a.total_q, b);
  const int start = s.len - s.nq;                      // position of the first new token
  if (!s.ok || (s.nq > 0 && (start < 0 || s.len > a.n_pos))) {
    if (threadIdx.x == 0) omq_set_status(a.status, OMQ_ERR_INVALID_ARG);
    return;
  }
  if (s.nq == 0) return;
  if ((int)blockIdx.x >= a.kv_units) {
    q_unit<BF>(a, s, blockIdx.x - a.kv_units);
    return;
  }
  const int G = a.c.n_kv, P = a.c.page;
  const bool is_v = blockIdx.x & 1;
  const int g = (blockIdx.x >> 1) % G;
  const int pg = start / P + (blockIdx.x >> 1) / G;    // page of the sequence
  if ((int64_t)pg * P >= s.len) return;
  const int id = pg < a.c.max_pages ? __ldg(a.c.page_table + (int64_t)b * a.c.max_pages + pg) : -1;
  if (id < 0 || id >= a.c.n_pages) {
    if (threadIdx.x == 0) omq_set_status(a.status, OMQ_ERR_INVALID_ARG);
    return;
  }
  const int kept = max(start - pg * P, 0);             // the page's tokens from before this call
  const int n_new = min(s.len, (pg + 1) * P) - pg * P - kept;
  const int grp = threadIdx.x >> 3, j = 8 * (threadIdx.x & 7);
  const int64_t head = (int64_t)id * G + g;
  float* scale_at = (is_v ? a.c.v_scale : a.c.k_scale) + head;
  uint8_t* codes = (is_v ? a.c.v : a.c.k) + head * P * HD;
  const float before = kept > 0 ? *scale_at : 0.f;
  const int64_t col = (int64_t)(a.n_heads + (is_v ? G : 0) + g) * HD + j;

  float x[NP][8], y[NP][8];
  uint32_t big = 0;              // largest magnitude as its bits: ordered as the values, a NaN on top
#pragma unroll
  for (int p = 0; p < NP; ++p) {
    const int i = p * GRP + grp;                 // new token of the page
    if (i < n_new) {
      const int pos = pg * P + kept + i;
      const int64_t row = s.row0 + (pos - start);
      load8<BF>(a.QKV, row * a.ld + col, x[p]);
      load8<BF>(a.QKV, row * a.ld + col + 64, y[p]);
      if (!is_v) {
        turn(a.rope, pos, j, x[p], y[p]);
        if (a.sa) {
          float u[8], w[8];
          load8<false>(a.sa, g * HD + j, u);
          load8<false>(a.sa, g * HD + j + 64, w);
#pragma unroll
          for (int e = 0; e < 8; ++e) { x[p][e] = __fmul_rn(x[p][e], u[e]); y[p][e] = __fmul_rn(y[p][e], w[e]); }
        }
      }
#pragma unroll
      for (int e = 0; e < 8; ++e)
        big = max(big, max(__float_as_uint(x[p][e]) & 0x7fffffffu, __float_as_uint(y[p][e]) & 0x7fffffffu));
    }
  }
  big = __reduce_max_sync(0xffffffffu, big);
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = big;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < NT / 32; ++w) big = max(big, red[w]);
  const float want = __fdiv_rn(__uint_as_float(big), 127.f);
  const float after = before >= want || before != before ? before : want;

  if (kept > 0 && after > before) {                    // the older tokens, on the new scale
    const float ratio = __fdiv_rn(before, after);
    for (int v = threadIdx.x; v < kept * (HD / 16); v += NT) {
      uint4* at = reinterpret_cast<uint4*>(codes) + v;
      uint4 u = *at;
      uint32_t* w = reinterpret_cast<uint32_t*>(&u);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        uint32_t o = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float c = (float)((int)((w[k] >> (8 * e)) & 255u) - 128);
          o |= ((uint32_t)((int)rintf(__fmul_rn(c, ratio)) + 128) & 255u) << (8 * e);
        }
        w[k] = o;
      }
      *at = u;
    }
  }
  if (threadIdx.x == 0) *scale_at = after;
  __nv_bfloat16* out = is_v ? a.Vo : a.Ko;
#pragma unroll
  for (int p = 0; p < NP; ++p) {
    const int i = p * GRP + grp;
    if (i < n_new) {
      uint32_t lo[2] = {0, 0}, hi[2] = {0, 0};
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float cx = after > 0.f ? code_of(x[p][e], after) : 0.f;
        const float cy = after > 0.f ? code_of(y[p][e], after) : 0.f;
        lo[e >> 2] |= (uint32_t)((int)cx + 128) << (8 * (e & 3));
        hi[e >> 2] |= (uint32_t)((int)cy + 128) << (8 * (e & 3));
        x[p][e] = __fmul_rn(cx, after);
        y[p][e] = __fmul_rn(cy, after);
      }
      uint8_t* at = codes + (kept + i) * HD + j;
      *reinterpret_cast<uint2*>(at) = make_uint2(lo[0], lo[1]);
      *reinterpret_cast<uint2*>(at + 64) = make_uint2(hi[0], hi[1]);
      if (out) {
        __nv_bfloat16* o = out + (int64_t)(s.row0 + pg * P + kept + i - start) * a.ldkv + g * HD + j;
        *reinterpret_cast<uint4*>(o) = pack_bf16x8(x[p]);
        *reinterpret_cast<uint4*>(o + 64) = pack_bf16x8(y[p]);
      }
    }
  }
}

template <bool BF>
omq_status append_launch(cudaStream_t st, const AppendArgs& a, const dim3& grid) {
  if (a.c.page <= 32) kv_append_kernel<BF, 1><<<grid, NT, 0, st>>>(a);
  else if (a.c.page == 64) kv_append_kernel<BF, 2><<<grid, NT, 0, st>>>(a);
  else kv_append_kernel<BF, 4><<<grid, NT, 0, st>>>(a);
  OMQ_LAUNCH_CHECK();
  return OMQ_OK;
}

}  // namespace

extern "C" {

omq_status omq_rope_table(omq_stream_t stream, int32_t n_pos, float theta, float* out) {
  OMQ_REQUIRE(n_pos > 0, OMQ_ERR_SHAPE);
  OMQ_REQUIRE(out && theta > 0.f, OMQ_ERR_INVALID_ARG);
  return rope_table((cudaStream_t)stream, n_pos, HD, theta, out);
}

omq_status omq_kv_append(omq_stream_t stream, const omq_kv_cache* cache, int32_t total_q, int32_t max_q,
                         const int32_t* cu_q, int32_t n_heads, const void* QKV, int32_t dtype, int64_t ld,
                         const float* rope, int32_t n_pos, const float* sa, void* Qo, int64_t ldq, void* Ko, void* Vo,
                         int64_t ldkv, int32_t* dev_status) {
  OMQ_TRY(kv_check(cache, total_q, max_q, cu_q, n_heads));
  OMQ_REQUIRE(QKV && rope && Qo && !Ko == !Vo, OMQ_ERR_INVALID_ARG);
  OMQ_REQUIRE(dtype == OMQ_F32 || dtype == OMQ_BF16, OMQ_ERR_INVALID_ARG);
  OMQ_REQUIRE(n_pos > 0 && ld >= (int64_t)(n_heads + 2 * cache->n_kv) * HD && ldq >= (int64_t)n_heads * HD &&
                  (!Ko || ldkv >= (int64_t)cache->n_kv * HD),
              OMQ_ERR_SHAPE);
  OMQ_REQUIRE(ld % 8 == 0 && ldq % 8 == 0 && (!Ko || ldkv % 8 == 0), OMQ_ERR_ALIGN);
  OMQ_REQUIRE(omq_aligned16(QKV) && omq_aligned16(rope) && omq_aligned16(sa) && omq_aligned16(Qo) && omq_aligned16(Ko) &&
                  omq_aligned16(Vo),
              OMQ_ERR_ALIGN);
  AppendArgs a{*cache, total_q, max_q, cu_q, n_heads, QKV, ld, (const float2*)rope, n_pos, sa, (__nv_bfloat16*)Qo, ldq,
               (__nv_bfloat16*)Ko, (__nv_bfloat16*)Vo, ldkv, 0, dev_status};
  const int64_t pages = ((int64_t)max_q + cache->page - 2) / cache->page + 1;    // that max_q tokens can touch
  const int64_t kv_units = 2 * pages * cache->n_kv;
  const int64_t q_units = ((int64_t)max_q * n_heads + QPASS * GRP - 1) / (QPASS * GRP);
  OMQ_REQUIRE(kv_units + q_units < (1ll << 31), OMQ_ERR_SHAPE);
  a.kv_units = (int)kv_units;
  const dim3 grid((unsigned)(kv_units + q_units), (unsigned)cache->B);
  return dtype == OMQ_BF16 ? append_launch<true>((cudaStream_t)stream, a, grid)
                           : append_launch<false>((cudaStream_t)stream, a, grid);
}

}  // extern "C"
