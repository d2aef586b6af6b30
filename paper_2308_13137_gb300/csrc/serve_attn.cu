// Attention of the newest tokens over an 8-bit paged cache (omq_kv_attention).
//
// O = softmax(q k^T / sqrt(128)) v with k = (ck - 128) sk, v = (cv - 128) sv, sk and sv one number per
// (page, KV head).  The cache read is the bound (2 x 128 bytes per token and KV head; every query head
// of the group and every new token of the sequence is served by one read), so the work is split over
// the tokens: a CTA takes (sequence, KV head, a chunk of tokens), its warps take 16-token tiles, and
// their partial results are joined through shared memory and, between CTAs, by a second small kernel.
//
// This file holds the form for few query rows per KV head (up to 16: decoding).  Every warp keeps its own
// ring of 16-token tiles in flight (TMA, 2 KB of K and of V each, 128-byte swizzle) and refills a slot as
// soon as it has used it: no barrier between warps.  Per tile a warp forms S^T = K q^T (16 tokens x 8 query
// rows) and O^T += V^T P by mma.sync m16n8k16 with fp16 operands and fp32 sums.  The tokens are the M
// dimension of the first product and the channels of the second, so a single query row costs an eighth of
// a tile and not a sixteenth.  tcgen05 has nothing to offer here: its smallest tile is 64 or 128 rows, and
// the products are a tenth of the loop's instructions (serve_attn_tc.cu has the form for more rows).  A code
// becomes an fp16 integer in registers, exactly: the byte under the exponent of 1024 (0x6400 | c = 1024 + c),
// minus 1152.  Channels are numbered inside the products so that a thread's operand values are 16 consecutive
// bytes of the page; row g of a product is token g ^ ((g & 1) << 2) of its eight, which puts the eight
// lanes of every load phase, of K and of V, on eight distinct 16-byte bank groups.
// Measured: 4 sequences of 62108 to 131072 tokens (400 K in all), 8 rows on each of 8 KV heads, 136 us, 6.0 TB/s; 16
// of up to 4096 tokens, one row on each of 32 heads, 66 us, 5.2 TB/s; one sequence of 2048 tokens 11 us, of which 7
// are the two launches and the first loads.  (Here and below "n x t tokens" are n sequences between t / 4 and t long.)
//
// Precision: the codes are exact; q (bf16) is fp16 after a power-of-two scale per row that puts
// its largest value in [2^13, 2^14): exact but for elements 2^-30 of that and less, whose last bits go; scores,
// sums and accumulators are fp32.  The weight of a token, p sv, is rounded to fp16 (the products' operand, 2^-11
// relative, whatever the output's type) against a reference m + d near the largest log2(p sv), so that a weight keeps 11
// bits down to 2^-22 of the largest; p's own sum stays fp32 against its own reference m (V's scales
// differ by page, so the two references differ).  A reference moves, and the accumulator with it,
// only when a score passes it by more than 2^7: few tiles do, and the others need no maximum across
// lanes at all, only a vote.
#include "serve_attn.cuh"

namespace {

using namespace tc;

constexpr int HD = ATTN_HD;
constexpr int TILE = 16;                    // tokens of a warp's tile
constexpr int TILE_BYTES = 2 * TILE * HD;   // K and V
constexpr float SHIFT = ATTN_SHIFT, SLACK = ATTN_SLACK, NOTHING = ATTN_NOTHING, NO_VALUE = ATTN_NO_VALUE;
constexpr int OPAD = 132;                   // floats per row of the joining buffer

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

__device__ __forceinline__ uint32_t u4(const uint4& v, int i) { return i == 0 ? v.x : (i == 1 ? v.y : (i == 2 ? v.z : v.w)); }

// shared memory of a CTA: rings (the joining buffers after the loop) | query fragments | per row: factor,
// keys seen | references and sums | barriers | page records
constexpr int W = 8;                        // warps
template <int NT>
struct Smem {
  static constexpr int DEPTH = 3, SLOTS = DEPTH * W;                 // ring tiles, DEPTH per warp
  static constexpr int RING = SLOTS * TILE_BYTES;
  static constexpr int ROWS = NT * 8;
  static constexpr int QF = ROWS * HD * 2;                            // [NT][8][32] uint2
  static constexpr int QS_OFF = RING + QF;
  static constexpr int STAT_OFF = QS_OFF + 2 * ROWS * 4;
  static constexpr int BAR_OFF = STAT_OFF + 3 * W * NT * 8 * 4;
  static constexpr int PAGES_OFF = BAR_OFF + SLOTS * 8 + 16;
  static_assert(W * 8 * OPAD * 4 <= RING, "the joining buffer fits the ring");
  static int bytes(int chunk, int page) { return PAGES_OFF + chunk / page * 12 + 1024; }
};

template <int NT>
__global__ void __launch_bounds__(W * 32, 2)
    kv_attention_kernel(const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV, const AttnArgs a) {
  using S = Smem<NT>;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  float* join = reinterpret_cast<float*>(smem);
  uint2* qf = reinterpret_cast<uint2*>(smem + S::RING);
  float* qs = reinterpret_cast<float*>(smem + S::QS_OFF);
  int* lims = reinterpret_cast<int*>(qs + S::ROWS);
  float* st_m = reinterpret_cast<float*>(smem + S::STAT_OFF);
  float* st_d = st_m + W * NT * 8;
  float* st_l = st_d + W * NT * 8;
  uint64_t* full = reinterpret_cast<uint64_t*>(smem + S::BAR_OFF);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(full + S::SLOTS);
  int* pid = reinterpret_cast<int*>(smem + S::PAGES_OFF);
  const int P = a.c.page, per_chunk = a.chunk / P, pshift = 31 - __clz(P);
  float* pks = reinterpret_cast<float*>(pid + per_chunk);     // key scale, times log2(e) / sqrt(128)
  float* plv = pks + per_chunk;                               // log2 of the value scale

  const int b = blockIdx.y, split = blockIdx.x % a.n_split, gr = blockIdx.x / a.n_split;
  const int g = gr / a.row_tiles, rt = gr % a.row_tiles;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, lg = lane >> 2, lt = lane & 3;
  const int rep = a.n_heads / a.c.n_kv;
  SeqRows s = seq_rows(a.c, a.cu_q, a.max_q, a.total_q, b);
  if (!s.ok || s.len > a.max_kv) {
    if (threadIdx.x == 0) omq_set_status(a.status, OMQ_ERR_INVALID_ARG);
    s.len = 0;                                                // its rows read as empty
  }
  const int R = s.nq * rep;                                   // query rows of this KV head
  constexpr int ROWS = S::ROWS;
  const int r0 = rt * ROWS;
  if (r0 >= R) return;
  const int start = s.len - s.nq;
  const int r_last = min(R, r0 + ROWS) - 1;
  const int kv_end = max(0, min(s.len, start + r_last / rep + 1));   // keys that some row of the CTA sees
  const int t_begin = split * a.chunk;
  const int t_end = min(kv_end, t_begin + a.chunk);
  if (split > 0 && t_begin >= kv_end) return;
  const int np = t_end > t_begin ? (t_end - t_begin + P - 1) >> pshift : 0;
  const int tiles = t_end > t_begin ? (t_end - t_begin + TILE - 1) / TILE : 0;

  // ---- page records of the chunk, query fragments and row factors ----
  for (int i = threadIdx.x; i < np; i += W * 32) {
    attn_page(a, b, g, (t_begin >> pshift) + i, pid + i, pks + i, plv + i);
  }
  if (threadIdx.x == 0) {
    for (int i = 0; i < S::SLOTS; ++i) mbar_init(&full[i], 1);
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  for (int r = warp; r < ROWS; r += W) {
    const int row = r0 + r;
    float v[4];
    int sh;
    attn_query4(a, s, g, rep, row, R, lane, v, &sh);
    const int nt = r >> 3, q = r & 7;
    const int w = (lane & 3) + (lane < 16 ? 0 : 4), t = (lane >> 2) & 3;
    qf[(nt * 8 + w) * 32 + q * 4 + t] = make_uint2(pack_half2(v[0], v[1]), pack_half2(v[2], v[3]));
    if (lane == 0) {
      qs[r] = __uint_as_float((uint32_t)(127 - sh) << 23);
      lims[r] = row < R ? min(s.len, start + row / rep + 1) : 0;
    }
  }
  __syncthreads();

  float m[NT][2], d[NT][2], l[NT][2], acc[NT][8][4];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
    for (int e = 0; e < 2; ++e) { m[nt][e] = NOTHING; d[nt][e] = NO_VALUE; l[nt][e] = 0.f; }
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[nt][i][e] = 0.f;
  }

  // this warp's ring: its n-th tile is tile warp + n W of the chunk, in slot n % DEPTH
  constexpr int DEPTH = S::DEPTH;
  const int mine = tiles > warp ? (tiles - warp + W - 1) / W : 0;
  uint64_t* wfull = full + warp * DEPTH;
  const uint32_t ring = smem_u32(smem + warp * DEPTH * TILE_BYTES);
  auto fill = [&](const int n, const int slot) {              // the converged warp; one lane issues
    const int t = (warp + n * W) * TILE, id = pid[t >> pshift];
    uint8_t* dst = smem + (warp * DEPTH + slot) * TILE_BYTES;
    const int row = (id * a.c.n_kv + g) * P + (t & (P - 1));
    if (elect_one()) {
      if (id < 0) {
        mbar_arrive(&wfull[slot]);                            // its tokens read as unseen
      } else {
        mbar_expect_tx(&wfull[slot], TILE_BYTES);
        tma_load_3d(&tmK, &wfull[slot], dst, 0, row, 0);
        tma_load_3d(&tmV, &wfull[slot], dst + TILE * HD, 0, row, 0);
      }
    }
    __syncwarp();
  };
  int filled = min(DEPTH, mine);
  for (int n = 0; n < filled; ++n) fill(n, n);

  {
    const uint2* qfw = qf + lane;
    uint2 qr[NT == 1 ? 8 : 1];               // one row tile: its fragments stay in registers
    if (NT == 1) {
#pragma unroll
      for (int w = 0; w < 8; ++w) qr[NT == 1 ? w : 0] = qfw[w * 32];
    }
    const int lim_min = __reduce_min_sync(0xffffffffu, lane < ROWS && r0 + lane < R ? lims[lane] : 0x7fffffff);
    const int n_here = (min(ROWS, R - r0) + 7) >> 3;          // row tiles that hold rows
    const float2* f2 = reinterpret_cast<const float2*>(qs) + lt;
    const int2* lim2 = reinterpret_cast<const int2*>(lims) + lt;
    const int row_k = lg ^ ((lg & 1) << 2);                   // token of product row lg among its eight
    const int row_v0 = 2 * lt, row_v1 = (2 * lt + 1) ^ 4;     // tokens of the product columns 2 lt, 2 lt + 1
    const uint32_t k_off = row_k * HD, kx0 = (uint32_t)(lt ^ row_k) << 4, kx1 = (uint32_t)((lt + 4) ^ row_k) << 4;
    const uint32_t v_off0 = TILE * HD + row_v0 * HD + ((uint32_t)(lg ^ row_v0) << 4);
    const uint32_t v_off1 = TILE * HD + row_v1 * HD + ((uint32_t)(lg ^ row_v1) << 4);

    auto tile = [&](const uint32_t base, const int t0) {
      const int pi = (t0 - t_begin) >> pshift;
      if (pid[pi] < 0) return;
      const float ks = pks[pi], lv = plv[pi];
      float sc[NT][4];
      {
        uint4 k[4];
        k[0] = lds128(base + k_off + kx0); k[1] = lds128(base + k_off + kx1);
        k[2] = lds128(base + k_off + 8 * HD + kx0); k[3] = lds128(base + k_off + 8 * HD + kx1);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int e = 0; e < 4; ++e) sc[nt][e] = 0.f;
#pragma unroll
        for (int w = 0; w < 8; ++w) {
          const uint32_t x = u4(k[w >> 2], w & 3), y = u4(k[2 + (w >> 2)], w & 3);
          const uint32_t a0 = codes_lo(x), a1 = codes_lo(y), a2 = codes_hi(x), a3 = codes_hi(y);
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
            if (nt > 0 && nt >= n_here) break;
            const uint2 q = NT == 1 ? qr[NT == 1 ? w : 0] : qfw[(nt * 8 + w) * 32];
            mma16816(sc[nt], a0, a1, a2, a3, q.x, q.y);
          }
        }
      }
      uint4 v[4];
      auto values = [&]() {
        v[0] = lds128(base + v_off0); v[1] = lds128(base + v_off1);
        v[2] = lds128(base + v_off0 + 8 * HD); v[3] = lds128(base + v_off1 + 8 * HD);
      };
      if (NT == 1) values();                 // (two row tiles have no registers for them before the weights)
      uint32_t p0[NT], p1[NT];
      const bool cut = t0 + TILE > lim_min;                   // some row does not see all of the tile
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        if (nt > 0 && nt >= n_here) break;
        const float2 f = f2[4 * nt];
        const float fk[2] = {ks * f.x, ks * f.y};
        float x[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = sc[nt][e] * fk[e & 1];
        if (cut) {
          const int2 lm = lim2[4 * nt];
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (t0 + row_k + 8 * (e >> 1) >= (e & 1 ? lm.y : lm.x)) x[e] = -INFINITY;
        }
        const float t0m = fmaxf(x[0], x[2]), t1m = fmaxf(x[1], x[3]);
        const float u0 = t0m - m[nt][0], u1 = t1m - m[nt][1];
        const bool over = u0 > SLACK || u1 > SLACK || u0 + (lv - d[nt][0]) > SLACK || u1 + (lv - d[nt][1]) > SLACK;
        if (__any_sync(0xffffffffu, over)) {
          float top[2] = {t0m, t1m}, grow[2];
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            top[e] = fmaxf(top[e], __shfl_xor_sync(0xffffffffu, top[e], 4));
            top[e] = fmaxf(top[e], __shfl_xor_sync(0xffffffffu, top[e], 8));
            top[e] = fmaxf(top[e], __shfl_xor_sync(0xffffffffu, top[e], 16));
            const float mn = fmaxf(m[nt][e], top[e]), drop = m[nt][e] - mn;
            const float dn = fmaxf(fmaxf(d[nt][e] + drop, (top[e] - mn) + lv), NO_VALUE);
            l[nt][e] *= ex2(drop);
            grow[e] = ex2((d[nt][e] - dn) + drop);
            m[nt][e] = mn;
            d[nt][e] = dn;
          }
#pragma unroll
          for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[nt][i][e] *= grow[e & 1];
        }
        float pw[4];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const float c = attn_factor(lv - d[nt][e] + SHIFT);
          pw[e] = ex2(x[e] - m[nt][e]);
          pw[e + 2] = ex2(x[e + 2] - m[nt][e]);
          l[nt][e] += pw[e] + pw[e + 2];
          pw[e] *= c;
          pw[e + 2] *= c;
        }
        if (cut) {                            // nothing unseen weighs, even where the page's scale is not finite
          const int2 lm = lim2[4 * nt];
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (t0 + row_k + 8 * (e >> 1) >= (e & 1 ? lm.y : lm.x)) pw[e] = 0.f;
        }
        p0[nt] = transpose8x8(pack_half2(pw[0], pw[1]));
        p1[nt] = transpose8x8(pack_half2(pw[2], pw[3]));
      }
      if (NT > 1) values();
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const uint32_t va = u4(v[0], w), vb = u4(v[1], w), vc = u4(v[2], w), vd = u4(v[3], w);
        const uint32_t x0 = __byte_perm(va, vb, 0x5140), x1 = __byte_perm(vc, vd, 0x5140);
        const uint32_t y0 = __byte_perm(va, vb, 0x7362), y1 = __byte_perm(vc, vd, 0x7362);
        const uint32_t a0 = codes_lo(x0), a1 = codes_hi(x0), a2 = codes_lo(x1), a3 = codes_hi(x1);
        const uint32_t c0 = codes_lo(y0), c1 = codes_hi(y0), c2 = codes_lo(y1), c3 = codes_hi(y1);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          if (nt > 0 && nt >= n_here) break;
          mma16816(acc[nt][2 * w], a0, a1, a2, a3, p0[nt], p1[nt]);
          mma16816(acc[nt][2 * w + 1], c0, c1, c2, c3, p0[nt], p1[nt]);
        }
      }
    };

    int slot = 0, turn = 0;                  // of tile n
    for (int n = 0; n < mine; ++n) {
      if (!warp_wait(&wfull[slot], turn)) {
        omq_set_status(a.status, OMQ_ERR_TIMEOUT); *abort_flag = 1; break;
      }
      tile(ring + slot * TILE_BYTES, t_begin + (warp + n * W) * TILE);
      __syncwarp();                          // every lane has read the tile
      if (filled < mine) fill(filled++, slot);
      if (++slot == DEPTH) { slot = 0; turn ^= 1; }
    }
    if (lane == 0 && *abort_flag)            // no copy may land after this CTA has left
      for (int j = max(0, filled - DEPTH); j < filled; ++j)
        if (!wait_phase(&wfull[j % DEPTH], (j / DEPTH) & 1)) break;
  }

  // ---- join the warps ----
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
        st_m[at] = m[nt][e]; st_d[at] = d[nt][e]; st_l[at] = v;
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
    {                                                         // one query row per warp, 4 channels per lane
      const int q = warp, row = r0 + nt * 8 + q;
      if (row >= R) continue;
      float mm = NOTHING, dd = NO_VALUE;
      for (int k = 0; k < W; ++k) mm = fmaxf(mm, st_m[(k * NT + nt) * 8 + q]);
      for (int k = 0; k < W; ++k) {
        const int at = (k * NT + nt) * 8 + q;
        dd = fmaxf(dd, (st_m[at] - mm) + st_d[at]);
      }
      float L = 0.f;
      float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
      for (int k = 0; k < W; ++k) {
        const int at = (k * NT + nt) * 8 + q;
        L += st_l[at] * ex2(st_m[at] - mm);
        const float c = ex2((st_m[at] - mm) + st_d[at] - dd);
        const float4 x = *reinterpret_cast<const float4*>(join + (k * 8 + q) * OPAD + 4 * lane);
        o.x = fmaf(x.x, c, o.x); o.y = fmaf(x.y, c, o.y); o.z = fmaf(x.z, c, o.z); o.w = fmaf(x.w, c, o.w);
      }
      const bool none = L == 0.f;                             // a NaN score is not an empty row
      const float c = none ? 0.f : ex2(dd - SHIFT) / L;
      const float lse = none ? -INFINITY : mm + log2f(L);
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
    const float c = ex2(a.wl[at + k] - ref);
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

struct Plan { int form, row_tiles, chunk, n_split; };   // form: rows per CTA, 8 or 16 (this file) or 128 (tcgen05)

// How a call is cut.  Up to 16 query rows per KV head take this file's form, more the tcgen05 tiles (16 rows,
// 16 x 4096 tokens: 37 us here, 42 us there).  Tokens per CTA: as many chunks as fill one wave, none under 256
// tokens; a second wave costs more than it balances (4 x 131072 tokens of 8 rows 136 us on one wave, 148 us on
// two; 8 x 8192 tokens of 128 rows 65 and 77 us; 16 x 4096 tokens of 24 rows 43 and 54 us).
Plan plan_of(int64_t B, int max_q, int max_kv, int n_heads, int n_kv) {
  Plan p;
  const int64_t rows = (int64_t)max_q * (n_heads / n_kv);
  p.form = rows <= 8 ? 8 : (rows <= 16 ? 16 : ATTN_TC_ROWS);
  p.row_tiles = (int)((rows + p.form - 1) / p.form);
  const int64_t units = B * n_kv * p.row_tiles;
  const int64_t slots = omq_num_sms() * (p.form == ATTN_TC_ROWS ? 1ll : 2ll);
  int64_t n = slots / units;
  const int64_t most = (max_kv + 255) / 256;
  if (n > most) n = most;
  if (n < 1) n = 1;
  int64_t chunk = ((max_kv + n - 1) / n + 127) / 128 * 128;
  if (chunk > ATTN_MAX_CHUNK) chunk = ATTN_MAX_CHUNK;
  p.chunk = (int)chunk;
  p.n_split = (int)((max_kv + chunk - 1) / chunk);
  return p;
}

size_t plan_workspace(const Plan& p, int64_t total_q, int64_t n_heads) {
  if (p.n_split <= 1) return 0;
  const size_t parts = (size_t)total_q * n_heads * p.n_split;
  return parts * HD * sizeof(float) + (parts * sizeof(float) + 255) / 256 * 256;
}

template <int NT>
omq_status attn_launch(cudaStream_t st, const AttnArgs& a) {
  using S = Smem<NT>;
  auto kern = kv_attention_kernel<NT>;
  static std::atomic<uint64_t> allowed{0};
  OMQ_TRY(omq_allow_smem(allowed, kern, S::bytes(ATTN_MAX_CHUNK, 16)));
  CUtensorMap tk, tv;
  const int64_t rows = (int64_t)a.c.n_pages * a.c.n_kv * a.c.page;
  if (!omq_make_map_u8(&tk, a.c.k, HD, rows, HD, TILE, HD) || !omq_make_map_u8(&tv, a.c.v, HD, rows, HD, TILE, HD))
    return OMQ_ERR_UNSUPPORTED;
  kern<<<dim3(a.n_split * a.c.n_kv * a.row_tiles, a.c.B), W * 32, S::bytes(a.chunk, a.c.page), st>>>(tk, tv, a);
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
  OMQ_REQUIRE((int64_t)cache->n_kv * p.row_tiles * p.n_split < (1ll << 31), OMQ_ERR_SHAPE);
  OMQ_REQUIRE((int64_t)cache->n_pages * cache->n_kv * cache->page < (1ll << 31), OMQ_ERR_SHAPE);   // TMA coordinates
  const size_t need = plan_workspace(p, total_q, n_heads);
  OMQ_REQUIRE(need == 0 || (workspace && ws_bytes >= need), OMQ_ERR_WORKSPACE);
  AttnArgs a{*cache, total_q, max_q, cu_q, max_kv, n_heads, (const __nv_bfloat16*)Q, ldq, Of, (__nv_bfloat16*)Ob, ldo,
             lse, nullptr, nullptr, p.chunk, p.n_split, p.row_tiles, dev_status};
  if (p.n_split > 1) {
    a.wo = (float*)workspace;
    a.wl = a.wo + (size_t)total_q * n_heads * p.n_split * HD;
  }
  cudaStream_t st = (cudaStream_t)stream;
  OMQ_TRY(p.form == 8 ? attn_launch<1>(st, a) : (p.form == 16 ? attn_launch<2>(st, a) : attn_tc_launch(st, a)));
  if (p.n_split > 1) {
    const int64_t pairs = (int64_t)max_q * n_heads;
    kv_attention_join_kernel<<<dim3((unsigned)((pairs + 7) / 8), cache->B), 256, 0, st>>>(a);
    OMQ_LAUNCH_CHECK();
  }
  return OMQ_OK;
}

}  // extern "C"
