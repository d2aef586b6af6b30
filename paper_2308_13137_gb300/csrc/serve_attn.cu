// Attention of the newest tokens over an 8-bit paged cache (omq_kv_attention).
//
// O = softmax(q k^T / sqrt(128)) v with k = (ck - 128) sk, v = (cv - 128) sv, sk and sv one number per
// (page, KV head).  The cache read is the bound (2 x 128 bytes per token and KV head; every query head
// of the group and every new token of the sequence is served by one read), so the work is split over
// the tokens: a CTA takes (sequence, KV head, a chunk of tokens), its warps take 16-token tiles, and
// their partial results are joined through shared memory and, between CTAs, by a second small kernel.
//
// Per tile a warp forms S^T = K q^T (16 tokens x 8 query rows) and O^T += V^T P by mma.sync m16n8k16 with
// fp16 operands and fp32 sums.  The tokens are the M dimension of the first product and the channels
// of the second, so a single query row costs an eighth of a tile and not a sixteenth.  tcgen05 has
// nothing to offer here: its smallest tile is 64 or 128 rows, and the products take 0.2 of the
// instruction issue of the loop.  A code becomes an fp16 integer in registers, exactly: the byte under
// the exponent of 1024 (0x6400 | c = 1024 + c), minus 1152.  Channels and tokens are numbered inside
// the products so that each thread's operand values are 16 consecutive bytes of the page.
//
// Precision: the codes are exact; q (bf16) is exact after a power-of-two scale per row that puts
// its largest value in [2^13, 2^14); scores, sums and accumulators are fp32.  The weight of a token,
// p sv, is rounded to fp16 against a running reference M >= log2(p sv) with 14 bits of headroom, so
// that a weight keeps 11 bits down to 2^-28 of the largest; p's own sum stays fp32 against its own
// running maximum m (V's scales differ by page, so the two references differ).
#include "serve_cache.cuh"
#include "tc.cuh"
#include <cuda_fp16.h>

namespace {

constexpr int HD = 128;
constexpr int TILE = 16;                    // tokens of a warp's tile
constexpr int MAX_CHUNK = 16384;
constexpr float SHIFT = 14.f;               // headroom of the fp16 weights, in powers of two
constexpr int OPAD = 132;                   // floats per row of the joining buffer

struct AttnArgs {
  omq_kv_cache c;
  int total_q, max_q; const int32_t* cu_q; int max_kv, n_heads;
  const __nv_bfloat16* Q; int64_t ldq;
  float* Of; __nv_bfloat16* Ob; int64_t ldo; float* lse;
  float* wo; float* wl;                     // partial results of the splits (n_split > 1)
  int chunk, n_split, row_tiles, rg;        // rg: row groups of a CTA
  int32_t* status;
};

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

__device__ __forceinline__ void mma16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                         uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

__device__ __forceinline__ uint32_t transpose8x8(uint32_t v) {
  uint32_t d;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(v));
  return d;
}

__device__ __forceinline__ uint32_t pack_half2(float lo, float hi) {
  const __half2 h = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}

__device__ __forceinline__ uint32_t u4(const uint4& v, int i) { return i == 0 ? v.x : (i == 1 ? v.y : (i == 2 ? v.z : v.w)); }

struct Tile { uint4 k[4], v[4]; };

// shared memory of a CTA: query fragments | row factors | page records | joining buffers
template <int W, int NT>
struct Smem {
  static constexpr int QF = 4 * NT * 8 * 32 * 8;              // up to 4 row groups: [rg][NT][8][32] uint2
  static constexpr int QS = 4 * NT * 8 * 4;
  static constexpr int STAT = 3 * W * NT * 8 * 4;
  static constexpr int JOIN = W * 8 * OPAD * 4;
  static constexpr int PAGES_OFF = QF + QS + STAT + JOIN;
  static int bytes(int chunk, int page) { return PAGES_OFF + chunk / page * 12; }
};

template <int W, int NT, int MIN_CTAS>
__global__ void __launch_bounds__(W * 32, MIN_CTAS) kv_attention_kernel(const AttnArgs a) {
  using S = Smem<W, NT>;
  extern __shared__ __align__(16) uint8_t smem[];
  uint2* qf = reinterpret_cast<uint2*>(smem);
  float* qs = reinterpret_cast<float*>(smem + S::QF);
  float* st_m = reinterpret_cast<float*>(smem + S::QF + S::QS);
  float* st_M = st_m + W * NT * 8;
  float* st_l = st_M + W * NT * 8;
  float* join = reinterpret_cast<float*>(smem + S::QF + S::QS + S::STAT);
  int* pid = reinterpret_cast<int*>(smem + S::PAGES_OFF);
  const int P = a.c.page, per_chunk = a.chunk / P;
  float* pks = reinterpret_cast<float*>(pid + per_chunk);     // key scale, times log2(e) / sqrt(128)
  float* plv = pks + per_chunk;                               // log2 of the value scale

  const int b = blockIdx.z, split = blockIdx.x;
  const int g = blockIdx.y / a.row_tiles, rt = blockIdx.y % a.row_tiles;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, lg = lane >> 2, lt = lane & 3;
  const int rep = a.n_heads / a.c.n_kv;
  SeqRows s = seq_rows(a.c, a.cu_q, a.max_q, a.total_q, b);
  if (!s.ok || s.len > a.max_kv) {
    if (threadIdx.x == 0) omq_set_status(a.status, OMQ_ERR_INVALID_ARG);
    s.len = 0;                                                // its rows read as empty
  }
  const int R = s.nq * rep;                                   // query rows of this KV head
  const int rows_cta = a.rg * NT * 8;
  const int r0 = rt * rows_cta;
  if (r0 >= R) return;
  const int start = s.len - s.nq;
  const int r_last = min(R, r0 + rows_cta) - 1;
  const int kv_end = max(0, min(s.len, start + r_last / rep + 1));   // keys that some row of the CTA sees
  const int t_begin = split * a.chunk;
  const int t_end = min(kv_end, t_begin + a.chunk);
  if (split > 0 && t_begin >= kv_end) return;

  // ---- page records of the chunk, query fragments and row factors ----
  const int np = t_end > t_begin ? (t_end - t_begin + P - 1) / P : 0;
  for (int i = threadIdx.x; i < np; i += W * 32) {
    const int pg = t_begin / P + i;
    int id = pg < a.c.max_pages ? __ldg(a.c.page_table + (int64_t)b * a.c.max_pages + pg) : -1;
    if (id < 0 || id >= a.c.n_pages) {
      omq_set_status(a.status, OMQ_ERR_INVALID_ARG);
      id = -1;
    }
    pid[i] = id;
    const int64_t at = (int64_t)(id < 0 ? 0 : id) * a.c.n_kv + g;
    pks[i] = __ldg(a.c.k_scale + at) * 0.12751743074602467f;  // log2(e) / sqrt(128)
    plv[i] = log2f(__ldg(a.c.v_scale + at));
  }
  for (int r = warp; r < rows_cta; r += W) {
    const int row = r0 + r;
    float v[4] = {0.f, 0.f, 0.f, 0.f};
    if (row < R) {
      const uint2 u = __ldg(reinterpret_cast<const uint2*>(
          a.Q + (int64_t)(s.row0 + row / rep) * a.ldq + (g * rep + row % rep) * HD + 4 * lane));
      v[0] = __uint_as_float(u.x << 16); v[1] = __uint_as_float(u.x & 0xffff0000u);
      v[2] = __uint_as_float(u.y << 16); v[3] = __uint_as_float(u.y & 0xffff0000u);
    }
    uint32_t big = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) big = max(big, __float_as_uint(v[e]) & 0x7fffffffu);
    big = __reduce_max_sync(0xffffffffu, big);
    // 2^sh puts the largest magnitude in [2^13, 2^14) (sh capped where 2^sh would overflow)
    const int sh = big == 0 ? 0 : min(13 + 127 - (int)(big >> 23), 126);
    const float up = __uint_as_float((uint32_t)(127 + sh) << 23);
    const int nt = r >> 3, q = r & 7;
    const int w = (lane & 3) + (lane < 16 ? 0 : 4), t = (lane >> 2) & 3;
    qf[(nt * 8 + w) * 32 + q * 4 + t] = make_uint2(pack_half2(v[0] * up, v[1] * up), pack_half2(v[2] * up, v[3] * up));
    if (lane == 0) qs[r] = __uint_as_float((uint32_t)(127 - sh) << 23);
  }
  __syncthreads();

  const int rgi = warp % a.rg, tw = warp / a.rg, n_tw = W / a.rg;   // row group and token group of this warp
  const uint2* qfw = qf + rgi * NT * 8 * 32 + lane;
  float f[NT][2], m[NT][2], M[NT][2], l[NT][2];
  int lim[NT][2];
  float acc[NT][8][4];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt)
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int r = rgi * NT * 8 + nt * 8 + 2 * lt + e, row = r0 + r;
      f[nt][e] = qs[r];
      lim[nt][e] = row < R ? min(s.len, start + row / rep + 1) : 0;
      m[nt][e] = -INFINITY; M[nt][e] = -INFINITY; l[nt][e] = 0.f;
    }
#pragma unroll
  for (int nt = 0; nt < NT; ++nt)
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[nt][i][e] = 0.f;

  const int64_t page_bytes = (int64_t)P * HD, pool_stride = page_bytes * a.c.n_kv;
  const uint8_t* kbase = a.c.k + g * page_bytes + lg * HD + lt * 16;
  const uint8_t* vbase = a.c.v + g * page_bytes + 2 * lt * HD + lg * 16;
  const int pshift = 31 - __clz(P);
  auto load = [&](int t0, Tile& T) {
    const int id = pid[(t0 - t_begin) >> pshift];
    const int64_t off = (int64_t)max(id, 0) * pool_stride + (t0 & (P - 1)) * HD;
    const uint4* k = reinterpret_cast<const uint4*>(kbase + off);
    const uint4* v = reinterpret_cast<const uint4*>(vbase + off);
    T.k[0] = __ldg(k); T.k[1] = __ldg(k + 4); T.k[2] = __ldg(k + 64); T.k[3] = __ldg(k + 68);
    T.v[0] = __ldg(v); T.v[1] = __ldg(v + 8); T.v[2] = __ldg(v + 64); T.v[3] = __ldg(v + 72);
  };
  auto compute = [&](int t0, const Tile& T) {
    const int pi = (t0 - t_begin) >> pshift;
    const float ks = pks[pi], lv = plv[pi];
    const bool there = pid[pi] >= 0;
    float sc[NT][4];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int e = 0; e < 4; ++e) sc[nt][e] = 0.f;
#pragma unroll
    for (int w = 0; w < 8; ++w) {
      const uint32_t x = u4(T.k[w >> 2], w & 3), y = u4(T.k[2 + (w >> 2)], w & 3);
      const uint32_t a0 = codes_lo(x), a1 = codes_lo(y), a2 = codes_hi(x), a3 = codes_hi(y);
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        const uint2 q = qfw[(nt * 8 + w) * 32];
        mma16816(sc[nt], a0, a1, a2, a3, q.x, q.y);
      }
    }
    uint32_t p0[NT], p1[NT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      float x[4], top[2];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int t = t0 + lg + 8 * (e >> 1);
        x[e] = t < lim[nt][e & 1] && there ? sc[nt][e] * (ks * f[nt][e & 1]) : -INFINITY;
      }
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        top[e] = fmaxf(x[e], x[e + 2]);
        top[e] = fmaxf(top[e], __shfl_xor_sync(0xffffffffu, top[e], 4));
        top[e] = fmaxf(top[e], __shfl_xor_sync(0xffffffffu, top[e], 8));
        top[e] = fmaxf(top[e], __shfl_xor_sync(0xffffffffu, top[e], 16));
      }
      float grow[2], pw[4];
      bool moved = false;
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const float mn = fmaxf(m[nt][e], top[e]), mr = mn == -INFINITY ? 0.f : mn;
        l[nt][e] = l[nt][e] * tc::ex2(m[nt][e] - mr) + (tc::ex2(x[e] - mr) + tc::ex2(x[e + 2] - mr));
        m[nt][e] = mn;
        const float Mn = fmaxf(M[nt][e], top[e] + lv), Mr = Mn == -INFINITY ? 0.f : Mn;
        grow[e] = tc::ex2(M[nt][e] - Mr);
        moved = moved || Mn != M[nt][e];
        M[nt][e] = Mn;
        const float ref = lv - Mr + SHIFT;
        pw[e] = tc::ex2(x[e] + ref);
        pw[e + 2] = tc::ex2(x[e + 2] + ref);
      }
      if (__any_sync(0xffffffffu, moved)) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[nt][i][e] *= grow[e & 1];
      }
      p0[nt] = transpose8x8(pack_half2(pw[0], pw[1]));
      p1[nt] = transpose8x8(pack_half2(pw[2], pw[3]));
    }
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const uint32_t va = u4(T.v[0], w), vb = u4(T.v[1], w), vc = u4(T.v[2], w), vd = u4(T.v[3], w);
      const uint32_t x0 = __byte_perm(va, vb, 0x5140), x1 = __byte_perm(vc, vd, 0x5140);
      const uint32_t y0 = __byte_perm(va, vb, 0x7362), y1 = __byte_perm(vc, vd, 0x7362);
      const uint32_t a0 = codes_lo(x0), a1 = codes_hi(x0), a2 = codes_lo(x1), a3 = codes_hi(x1);
      const uint32_t c0 = codes_lo(y0), c1 = codes_hi(y0), c2 = codes_lo(y1), c3 = codes_hi(y1);
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        mma16816(acc[nt][2 * w], a0, a1, a2, a3, p0[nt], p1[nt]);
        mma16816(acc[nt][2 * w + 1], c0, c1, c2, c3, p0[nt], p1[nt]);
      }
    }
  };

  // the next tile's loads are in flight while the current one is computed
  const int step = TILE * n_tw;
  int t0 = t_begin + TILE * tw;
  Tile cur, nxt;
  if (t0 < t_end) load(t0, cur);
  while (t0 < t_end) {
    if (t0 + step < t_end) load(t0 + step, nxt);
    compute(t0, cur);
    cur = nxt;
    t0 += step;
  }

  // ---- join the token groups of each row group ----
#pragma unroll
  for (int nt = 0; nt < NT; ++nt)
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      float v = l[nt][e];
      v += __shfl_xor_sync(0xffffffffu, v, 4);
      v += __shfl_xor_sync(0xffffffffu, v, 8);
      v += __shfl_xor_sync(0xffffffffu, v, 16);
      if (lg == 0) {
        const int at = (warp * NT + nt) * 8 + 2 * lt + e;
        st_m[at] = m[nt][e]; st_M[at] = M[nt][e]; st_l[at] = v;
      }
    }
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    __syncthreads();
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      float4* o = reinterpret_cast<float4*>(join + (warp * 8 + 2 * lt + e) * OPAD + 16 * lg);
#pragma unroll
      for (int i = 0; i < 4; ++i)
        o[i] = make_float4(acc[nt][2 * i][e], acc[nt][2 * i][e + 2], acc[nt][2 * i + 1][e], acc[nt][2 * i + 1][e + 2]);
    }
    __syncthreads();
    for (int rq = warp; rq < a.rg * 8; rq += W) {             // one query row per warp, 4 channels per lane
      const int gi = rq >> 3, q = rq & 7;
      const int row = r0 + gi * NT * 8 + nt * 8 + q;
      if (row >= R) continue;
      float mm = -INFINITY, MM = -INFINITY;
      for (int k = 0; k < n_tw; ++k) {
        const int at = ((k * a.rg + gi) * NT + nt) * 8 + q;
        mm = fmaxf(mm, st_m[at]);
        MM = fmaxf(MM, st_M[at]);
      }
      const float mr = mm == -INFINITY ? 0.f : mm, Mr = MM == -INFINITY ? 0.f : MM;
      float L = 0.f;
      float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
      for (int k = 0; k < n_tw; ++k) {
        const int wk = k * a.rg + gi, at = (wk * NT + nt) * 8 + q;
        L += st_l[at] * tc::ex2(st_m[at] - mr);
        const float c = tc::ex2(st_M[at] - Mr);
        const float4 x = *reinterpret_cast<const float4*>(join + (wk * 8 + q) * OPAD + 4 * lane);
        o.x = fmaf(x.x, c, o.x); o.y = fmaf(x.y, c, o.y); o.z = fmaf(x.z, c, o.z); o.w = fmaf(x.w, c, o.w);
      }
      const bool empty = mm == -INFINITY && L == 0.f;         // a NaN score is not an empty row
      const float c = empty ? 0.f : tc::ex2(Mr - mr - SHIFT) / L;
      const float lse = empty ? -INFINITY : mr + log2f(L);
      o.x *= c; o.y *= c; o.z *= c; o.w *= c;
      const int64_t tok = s.row0 + row / rep;
      const int head = g * rep + row % rep;
      if (a.n_split > 1) {
        const int64_t at = (tok * a.n_heads + head) * a.n_split + split;
        *reinterpret_cast<float4*>(a.wo + at * HD + 4 * lane) = o;
        if (lane == 0) a.wl[at] = lse;
      } else {
        if (a.Of) *reinterpret_cast<float4*>(a.Of + tok * a.ldo + head * HD + 4 * lane) = o;
        if (a.Ob) {
          uint2 u;
          __nv_bfloat162* h = reinterpret_cast<__nv_bfloat162*>(&u);
          h[0] = __floats2bfloat162_rn(o.x, o.y);
          h[1] = __floats2bfloat162_rn(o.z, o.w);
          *reinterpret_cast<uint2*>(a.Ob + tok * a.ldo + head * HD + 4 * lane) = u;
        }
        if (a.lse && lane == 0) a.lse[tok * a.n_heads + head] = lse;
      }
    }
  }
}

// O = sum_s O_s 2^(lse_s - lse) over the splits that hold keys of the row, in split order; one warp per
// (row, head)
__global__ void __launch_bounds__(256) kv_attention_join_kernel(const AttnArgs a) {
  const int b = blockIdx.y, lane = threadIdx.x & 31;
  const int idx = blockIdx.x * 8 + (threadIdx.x >> 5);
  SeqRows s = seq_rows(a.c, a.cu_q, a.max_q, a.total_q, b);
  if (!s.ok || s.len > a.max_kv) s.len = 0;
  const int i = idx / a.n_heads, head = idx % a.n_heads;
  if (i >= s.nq) return;
  const int seen = max(0, min(s.len, s.len - s.nq + i + 1));
  const int nv = (seen + a.chunk - 1) / a.chunk;
  const int64_t tok = s.row0 + i, at = (tok * a.n_heads + head) * a.n_split;
  float top = -INFINITY;
  for (int k = lane; k < nv; k += 32) top = fmaxf(top, a.wl[at + k]);
#pragma unroll
  for (int off = 16; off > 0; off >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, off));
  const float ref = top == -INFINITY ? 0.f : top;
  float L = 0.f;
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
  for (int k = 0; k < nv; ++k) {
    const float c = tc::ex2(a.wl[at + k] - ref);
    const float4 x = *reinterpret_cast<const float4*>(a.wo + (at + k) * HD + 4 * lane);
    L += c;
    o.x = fmaf(x.x, c, o.x); o.y = fmaf(x.y, c, o.y); o.z = fmaf(x.z, c, o.z); o.w = fmaf(x.w, c, o.w);
  }
  const float c = L == 0.f ? 0.f : 1.f / L;
  o.x *= c; o.y *= c; o.z *= c; o.w *= c;
  if (a.Of) *reinterpret_cast<float4*>(a.Of + tok * a.ldo + head * HD + 4 * lane) = o;
  if (a.Ob) {
    uint2 u;
    __nv_bfloat162* h = reinterpret_cast<__nv_bfloat162*>(&u);
    h[0] = __floats2bfloat162_rn(o.x, o.y);
    h[1] = __floats2bfloat162_rn(o.z, o.w);
    *reinterpret_cast<uint2*>(a.Ob + tok * a.ldo + head * HD + 4 * lane) = u;
  }
  if (a.lse && lane == 0) a.lse[tok * a.n_heads + head] = L == 0.f ? -INFINITY : ref + log2f(L);
}

struct Plan { int nt, rg, row_tiles, chunk, n_split; };

// How a call is cut.  Rows per CTA: 8 (one new token of up to 8 query heads per KV head), 16, 32 or 64;
// tokens per CTA: as many chunks as give every SM two rounds of CTAs, none under 256 tokens.
Plan plan_of(int64_t B, int max_q, int max_kv, int n_heads, int n_kv) {
  Plan p;
  const int64_t rows = (int64_t)max_q * (n_heads / n_kv);
  p.nt = rows <= 8 ? 1 : 2;
  p.rg = rows <= 16 ? 1 : (rows <= 32 ? 2 : 4);
  const int64_t per = 8ll * p.nt * p.rg;
  p.row_tiles = (int)((rows + per - 1) / per);
  const int64_t units = B * n_kv * p.row_tiles;
  const int64_t slots = (int64_t)omq_num_sms() * (p.nt == 1 ? 2 : 3);
  int64_t n = (2 * slots + units - 1) / units;
  const int64_t most = (max_kv + 255) / 256;
  if (n > most) n = most;
  if (n < 1) n = 1;
  int64_t chunk = ((max_kv + n - 1) / n + 127) / 128 * 128;
  if (chunk > MAX_CHUNK) chunk = MAX_CHUNK;
  p.chunk = (int)chunk;
  p.n_split = (int)((max_kv + chunk - 1) / chunk);
  return p;
}

size_t plan_workspace(const Plan& p, int64_t total_q, int64_t n_heads) {
  if (p.n_split <= 1) return 0;
  const size_t parts = (size_t)total_q * n_heads * p.n_split;
  return parts * HD * sizeof(float) + (parts * sizeof(float) + 255) / 256 * 256;
}

template <int W, int NT, int MIN_CTAS>
omq_status attn_launch(cudaStream_t st, const AttnArgs& a) {
  auto kern = kv_attention_kernel<W, NT, MIN_CTAS>;
  const int bytes = Smem<W, NT>::bytes(a.chunk, a.c.page);
  static bool set = false;
  if (!set) {
    if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, Smem<W, NT>::bytes(MAX_CHUNK, 16)) !=
        cudaSuccess)
      return OMQ_ERR_CUDA;
    set = true;
  }
  kern<<<dim3(a.n_split, a.c.n_kv * a.row_tiles, a.c.B), W * 32, bytes, st>>>(a);
  OMQ_LAUNCH_CHECK();
  return OMQ_OK;
}

}  // namespace

extern "C" {

size_t omq_kv_attention_workspace_size(int32_t B, int32_t total_q, int32_t max_q, int32_t max_kv, int32_t n_heads,
                                       int32_t n_kv) {
  if (B <= 0 || total_q <= 0 || max_q <= 0 || max_kv <= 0 || n_kv <= 0 || n_heads <= 0 || n_heads % n_kv) return 0;
  return plan_workspace(plan_of(B, max_q, max_kv, n_heads, n_kv), total_q, n_heads);
}

omq_status omq_kv_attention(omq_stream_t stream, const omq_kv_cache* cache, int32_t total_q, int32_t max_q,
                            const int32_t* cu_q, int32_t max_kv, int32_t n_heads, const void* Q, int64_t ldq, float* Of,
                            void* Ob, int64_t ldo, float* lse, void* workspace, size_t ws_bytes, int32_t* dev_status) {
  OMQ_TRY(kv_check(cache, total_q, max_q, cu_q, n_heads));
  OMQ_REQUIRE(Q && (Of || Ob), OMQ_ERR_INVALID_ARG);
  OMQ_REQUIRE(max_kv > 0 && ldq >= (int64_t)n_heads * HD && ldo >= (int64_t)n_heads * HD, OMQ_ERR_SHAPE);
  OMQ_REQUIRE(ldq % 8 == 0 && ldo % 8 == 0, OMQ_ERR_ALIGN);
  OMQ_REQUIRE(omq_aligned16(Q) && omq_aligned16(Of) && omq_aligned16(Ob) && omq_aligned16(lse) &&
                  omq_aligned16(workspace),
              OMQ_ERR_ALIGN);
  const Plan p = plan_of(cache->B, max_q, max_kv, n_heads, cache->n_kv);
  OMQ_REQUIRE((int64_t)cache->n_kv * p.row_tiles <= 65535, OMQ_ERR_SHAPE);
  const size_t need = plan_workspace(p, total_q, n_heads);
  OMQ_REQUIRE(need == 0 || (workspace && ws_bytes >= need), OMQ_ERR_WORKSPACE);
  AttnArgs a{*cache, total_q, max_q, cu_q, max_kv, n_heads, (const __nv_bfloat16*)Q, ldq, Of, (__nv_bfloat16*)Ob, ldo,
             lse, nullptr, nullptr, p.chunk, p.n_split, p.row_tiles, p.rg, dev_status};
  if (p.n_split > 1) {
    a.wo = (float*)workspace;
    a.wl = a.wo + (size_t)total_q * n_heads * p.n_split * HD;
  }
  cudaStream_t st = (cudaStream_t)stream;
  OMQ_TRY(p.nt == 1 ? (attn_launch<8, 1, 2>(st, a)) : (attn_launch<4, 2, 3>(st, a)));
  if (p.n_split > 1) {
    const int64_t pairs = (int64_t)max_q * n_heads;
    kv_attention_join_kernel<<<dim3((unsigned)((pairs + 7) / 8), cache->B), 256, 0, st>>>(a);
    OMQ_LAUNCH_CHECK();
  }
  return OMQ_OK;
}

}  // extern "C"
