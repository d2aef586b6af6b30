// Attention over an 8-bit paged cache for many query rows per KV head (several new tokens times the
// query heads of a group): tcgen05 tiles of 128 rows x 64 tokens.
//
// The mathematics and the precision are those of serve_attn.cu.  With more than 16 rows per KV head the
// conversion of the codes, done once per 8 rows of a warp there, and the per-warp softmax bound that form; here
// a 64-token tile is converted once for 128 rows.  Roles of a CTA's 20 warps:
//   0, 3    TMA: raw code tiles of K and of V [64 x 128] (128-byte swizzle)
//   1, 2    issue S = Q K^T (128 x 64 x 128) and O += P V (128 x 128 x 64).  An issuing warp spends 150 cycles on a
//           wait that is already over, 180 on a commit and 150 on the products, so each has one wait and one
//           commit per tile: "ready" barriers count the converters and the softmax warps together, and
//           the commit that hands a result on also frees the operands
//   4..7, 16..19   softmax, one row per thread, the even and the odd tiles: scores from tensor memory, weights to
//           shared memory as the A operand of P V.  The two groups have their own references, sums and
//           accumulators in tensor memory, joined at the end, so neither waits for the other; a row's
//           references move, and its O is rescaled, only when a score passes them by more than 2^7
//   8..15   convert: K (8..11) and V (12..15) to fp16, one half row of 64 codes per thread; K is read K-major, V
//           MN-major, both from [half][64 tokens][128 bytes] swizzled tiles
// Warps without a row of the call do not take part.  Bound: the latency of a tile's way through the
// softmax threads, 1700 cycles per tile and group with 64 exponentials each (half of them in the waits and the
// fences around the exponentials), where the tile's 16 KB come from HBM in 700: 8 sequences of up to 8192 tokens, 128 rows on
// each of 8 KV heads, 67 us, 0.52 PFLOP/s, 1.4 TB/s.
#include "serve_attn.cuh"

namespace {

using namespace tc;

constexpr int HD = ATTN_HD, BMR = ATTN_TC_ROWS, TT = 64;
constexpr int RAW = 4;                               // ring depth of raw tiles (K | V); converted tiles: two of each
constexpr int RAW_BYTES = 2 * TT * HD;               // K | V codes
constexpr int HALF = TT * HD;                        // one 64-channel half of a converted tile: 64 rows x 128 bytes
constexpr int OP_BYTES = 2 * HALF;                   // a converted tile of K or V
constexpr int P_BYTES = BMR * TT * 2;
constexpr int Q_OFF = 0, Q_BYTES = BMR * HD * 2;
constexpr int CONV_OFF = Q_OFF + Q_BYTES;
constexpr int P_OFF = CONV_OFF + 4 * OP_BYTES;       // converted: K K | V V
constexpr int RAW_OFF = P_OFF + 2 * P_BYTES;
constexpr int ROW_OFF = RAW_OFF + RAW * RAW_BYTES;   // per row: factor, keys seen
constexpr int REF_OFF = ROW_OFF + 2 * BMR * 4;      // per group and row: m, d, l
constexpr int BAR_OFF = REF_OFF + 2 * 3 * BMR * 4;
constexpr int PAGES_OFF = BAR_OFF + 256;
constexpr int THREADS = 640;

int tc_smem(int chunk, int page) { return PAGES_OFF + chunk / page * 12 + 1024; }

// 16 codes to fp16, into two swizzled 16-byte chunks of a 128-byte row
__device__ __forceinline__ void put16(uint32_t row, int c, uint32_t x, const uint4& u) {
  sts128(row + (((2 * c) ^ x) << 4), make_uint4(codes_lo(u.x), codes_hi(u.x), codes_lo(u.y), codes_hi(u.y)));
  sts128(row + (((2 * c + 1) ^ x) << 4), make_uint4(codes_lo(u.z), codes_hi(u.z), codes_lo(u.w), codes_hi(u.w)));
}

// CP: copies of a row.  Rows that fit a half or a quarter of the tile's 128 are held two or four times, each copy
// with its own half or quarter of every tile's tokens: a softmax thread's 64 exponentials become 32 or 16.
template <int CP>
__global__ void __launch_bounds__(THREADS, 1)
    kv_attention_tc_kernel(const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV, const AttnArgs a) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  float* qs = reinterpret_cast<float*>(smem + ROW_OFF);
  int* lims = reinterpret_cast<int*>(qs + BMR);
  float* refs = reinterpret_cast<float*>(smem + REF_OFF);
  uint64_t* raw_full = reinterpret_cast<uint64_t*>(smem + BAR_OFF);
  uint64_t* raw_empty = raw_full + RAW;
  uint64_t* s_ready = raw_empty + RAW;               // [2] K of the tile converted, the buffer's last scores read
  uint64_t* s_full = s_ready + 2;                    // [2] scores formed (K's slot is free)
  uint64_t* p_ready = s_full + 2;                    // [2] V of the tile converted, its weights written
  uint64_t* p_done = p_ready + 2;                    // [2] product formed (V's slot and the weights are free)
  uint64_t* drain = p_done + 2;                      // [2]
  uint32_t* tmem_holder = reinterpret_cast<uint32_t*>(drain + 2);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_holder + 1);
  int* pid = reinterpret_cast<int*>(smem + PAGES_OFF);
  const int P = a.c.page, per_chunk = a.chunk / P, pshift = 31 - __clz(P);
  float* pks = reinterpret_cast<float*>(pid + per_chunk);
  float* plv = pks + per_chunk;

  const int b = blockIdx.y, split = blockIdx.x % a.n_split, gr = blockIdx.x / a.n_split;
  const int g = gr / a.row_tiles, rt = gr % a.row_tiles;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rep = a.n_heads / a.c.n_kv;
  SeqRows s = seq_rows(a.c, a.cu_q, a.max_q, a.total_q, b);
  if (!s.ok || s.len > a.max_kv) {
    if (threadIdx.x == 0) omq_set_status(a.status, OMQ_ERR_INVALID_ARG);
    s.len = 0;                                                // its rows read as empty
  }
  const int R = s.nq * rep, r0 = rt * BMR;
  if (r0 >= R) return;
  const int start = s.len - s.nq, r_last = min(R, r0 + BMR) - 1;
  const int kv_end = max(0, min(s.len, start + r_last / rep + 1));
  const int t_begin = split * a.chunk, t_end = min(kv_end, t_begin + a.chunk);
  if (split > 0 && t_begin >= kv_end) return;
  const int np = t_end > t_begin ? (t_end - t_begin + P - 1) >> pshift : 0;
  const int tiles = t_end > t_begin ? (t_end - t_begin + TT - 1) / TT : 0;

  constexpr int SPAN = BMR / CP, TW = TT / CP;                // rows held, tokens of a softmax thread
  const int row_warps = CP > 1 ? 4 : min(4, (R - r0 + 31) >> 5);     // softmax warps of a group that hold rows

  // ---- page records, the query operand (fp16, K-major, 128-byte swizzle, two halves of 64 channels) ----
  for (int i = threadIdx.x; i < np; i += THREADS) attn_page(a, b, g, (t_begin >> pshift) + i, pid + i, pks + i, plv + i);
  if (threadIdx.x == 0) {
    for (int i = 0; i < RAW; ++i) { mbar_init(&raw_full[i], 2); mbar_init(&raw_empty[i], 8); }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&s_ready[i], 4 + row_warps); mbar_init(&s_full[i], 1);
      mbar_init(&p_ready[i], 4 + row_warps); mbar_init(&p_done[i], 1);
      mbar_init(&drain[i], 1);
    }
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) tmem_alloc(tmem_holder, 512);
  for (int i = warp; i < SPAN; i += THREADS / 32) {
    float v[4];
    int sh;
    attn_query4(a, s, g, rep, r0 + i, R, lane, v, &sh);
    const uint2 u = make_uint2(pack_half2(v[0], v[1]), pack_half2(v[2], v[3]));
    for (int r = i; r < BMR; r += SPAN) {
      uint8_t* row = smem + Q_OFF + (lane >> 4) * (BMR * 128) + r * 128;
      *reinterpret_cast<uint2*>(row + (((lane & 15) >> 1 ^ (r & 7)) << 4) + (lane & 1) * 8) = u;
      if (lane == 0) {
        qs[r] = __uint_as_float((uint32_t)(127 - sh) << 23);
        lims[r] = r0 + i < R ? min(s.len, start + (r0 + i) / rep + 1) : 0;
      }
    }
  }
  fence_async_smem();                                         // the query tile -> visible to the tensor core
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_holder;
  constexpr uint32_t O_COL = 128;                             // S: columns 0 and 64; O: 128 and 256
  auto fail = [&]() { omq_set_status(a.status, OMQ_ERR_TIMEOUT); *abort_flag = 1; };

  // registers: 128 x 48 + 256 x 64 + 256 x 144 of the launch's 640 x 96
  if (warp < 4) asm volatile("setmaxnreg.dec.sync.aligned.u32 48;");
  if (warp == 0 || warp == 3) {
    // ---------------- the raw ring, K and V: the whole warp runs the loop, one lane issues ----------------
    const bool is_v = warp == 3;
    const CUtensorMap* const tm = is_v ? &tmV : &tmK;
    const int box = min(P, TT), per = TT / box;
    int i = 0;
    for (; i < tiles; ++i) {
      const int st = i % RAW, t0 = i * TT;
      // row of the pool of each box that holds tokens, one lane each (-1: none, or a page out of range)
      const int tk = t0 + lane * box, id = lane < per && tk < t_end - t_begin ? pid[tk >> pshift] : -1;
      const int row = id < 0 ? -1 : (id * a.c.n_kv + g) * P + (tk & (P - 1));
      const uint32_t bytes = __popc(__ballot_sync(0xffffffffu, row >= 0)) * box * HD;
      if (!warp_wait(&raw_empty[st], ((i / RAW) & 1) ^ 1)) { fail(); break; }
      uint8_t* dst = smem + RAW_OFF + st * RAW_BYTES + (is_v ? TT * HD : 0);
      if (elect_one()) mbar_expect_tx(&raw_full[st], bytes);
      for (int k = 0; k < per; ++k) {
        const int rk = __shfl_sync(0xffffffffu, row, k);
        if (rk >= 0 && elect_one()) tma_load_3d(tm, &raw_full[st], dst + k * box * HD, 0, rk, 0);
      }
      __syncwarp();
    }
    if (__any_sync(0xffffffffu, *abort_flag))        // no copy may land after this CTA has left
      for (int j = i > RAW ? i - RAW : 0; j < i; ++j)
        if (!wait_phase(&raw_full[j % RAW], (j / RAW) & 1)) break;
  } else if (warp == 1 || warp == 2) {
    // ---------------- issue: the whole warp runs the loop, one lane issues ----------------
    const bool scores = warp == 1;
    constexpr uint32_t idS = idesc_f16(BMR, TT), idO = idesc_f16(BMR, HD) | (1u << 16);        // V is MN-major
    const uint64_t dq = sdesc(smem_u32(smem + Q_OFF), 16, 1024), dk = sdesc(smem_u32(smem + CONV_OFF), 16, 1024);
    const uint64_t dp = sdesc(smem_u32(smem + P_OFF), 16, 1024);
    const uint64_t dv = sdesc(smem_u32(smem + CONV_OFF + 2 * OP_BYTES), HALF, 1024);
    for (int j = 0; j < tiles; ++j) {
      if (!warp_wait(scores ? &s_ready[j & 1] : &p_ready[j & 1], (j >> 1) & 1)) { fail(); break; }
      tc_fence_after();
      if (elect_one()) {
        if (scores) {
          const uint64_t k0 = dk + (uint64_t)((j & 1) * (OP_BYTES >> 4));
#pragma unroll
          for (int k = 0; k < HD / 16; ++k)
            umma_bf16(tmem + (j & 1) * TT, dq + (((k >> 2) * (BMR * 128) + (k & 3) * 32) >> 4),
                      k0 + (((k >> 2) * HALF + (k & 3) * 32) >> 4), idS, k != 0);
          umma_commit(&s_full[j & 1]);
        } else {
          const uint64_t p0 = dp + (uint64_t)((j & 1) * (P_BYTES >> 4)), v0 = dv + (uint64_t)((j & 1) * (OP_BYTES >> 4));
#pragma unroll
          for (int k = 0; k < TT / 16; ++k)
            umma_bf16(tmem + O_COL + (j & 1) * HD, p0 + ((k * 32) >> 4), v0 + ((k * 2048) >> 4), idO, j > 1 || k != 0);
          umma_commit(&p_done[j & 1]);
        }
      }
      __syncwarp();
    }
    if (__any_sync(0xffffffffu, *abort_flag)) {   // products in flight end before the tensor memory is released
      if (elect_one()) umma_commit(&drain[scores]);
      wait_phase(&drain[scores], 0);
    }
  } else if (warp >= 8 && warp < 16) {
    // ---------------- convert ----------------
    asm volatile("setmaxnreg.dec.sync.aligned.u32 64;");
    const bool is_v = warp >= 12;
    const int t = threadIdx.x & 127, r = t & 63, h = t >> 6;  // token, half of its channels
    const uint32_t x = r & 7, src0 = smem_u32(smem + RAW_OFF) + (is_v ? TT * HD : 0) + r * HD;
    const uint32_t dst0 = smem_u32(smem + CONV_OFF) + (is_v ? 2 * OP_BYTES : 0) + h * HALF + r * 128;
    uint64_t *ready = is_v ? p_ready : s_ready, *freed = is_v ? p_done : s_full;
    for (int j = 0; j < tiles; ++j) {
      const int rs = j % RAW;
      if (!warp_wait(&raw_full[rs], (j / RAW) & 1)) { fail(); break; }
      uint4 u[4];
#pragma unroll
      for (int c = 0; c < 4; ++c) u[c] = lds128(src0 + rs * RAW_BYTES + (((4 * h + c) ^ x) << 4));
      if (j > 1 && !warp_wait(&freed[j & 1], ((j >> 1) & 1) ^ 1)) { fail(); break; }
#pragma unroll
      for (int c = 0; c < 4; ++c) put16(dst0 + (j & 1) * OP_BYTES, c, x, u[c]);
      fence_async_smem();                    // the converted tile -> visible to the tensor core
      __syncwarp();
      if (lane == 0) { mbar_arrive(&raw_empty[rs]); mbar_arrive(&ready[j & 1]); }
    }
  } else if (warp >= 4) {
    // ---------------- softmax: one row per thread, every other tile ----------------
    asm volatile("setmaxnreg.inc.sync.aligned.u32 144;");
    const int sg = warp >= 16, r = (warp & 3) * 32 + lane;
    const uint32_t lanes = tmem + ((uint32_t)((warp & 3) * 32) << 16), o_col = lanes + O_COL + sg * HD;
    const bool holds = (warp & 3) < row_warps, mine = r0 + (r & (SPAN - 1)) < R;
    const uint32_t prow = smem_u32(smem + P_OFF + sg * P_BYTES) + r * 128;
    float m = ATTN_NOTHING, d = ATTN_NO_VALUE, l = 0.f;
    bool ok = true;
    if (CP > 1)                                               // the weights of the other copies' tokens
      for (int c = 0; c < 8; ++c) sts128(prow + (c << 4), make_uint4(0, 0, 0, 0));
    if (holds && lane == 0) mbar_arrive(&s_ready[sg]);        // the first scores overwrite nothing
    const int w0 = r / SPAN * TW;                             // this copy's tokens of a tile
    const float f = qs[r];
    const int lim = lims[r], lim_min = __reduce_min_sync(0xffffffffu, mine ? lim : 0x7fffffff);
    uint32_t turn = 0;
    for (int j = sg; j < tiles && holds; j += 2, turn ^= 1) {
      // the 16-token quarters, each of one page: score factor, log2 of the value scale; the tokens that
      // this row sees, as bits
      const int t0 = t_begin + j * TT + w0;
      float fk[TW / 16], lv[TW / 16];
      uint64_t seen = lim - t0 >= TW ? ~0ull : (lim <= t0 ? 0ull : (1ull << (lim - t0)) - 1);
      bool whole = t0 + TW <= min(t_end, lim_min);
#pragma unroll
      for (int q = 0; q < TW / 16; ++q) {
        const int pi = min((j * TT + w0 + 16 * q) >> pshift, np - 1);
        fk[q] = pks[pi] * f;
        lv[q] = plv[pi];
        if (pid[pi] < 0) {
          whole = false;
          seen &= ~(0xffffull << (16 * q));
        }
      }
      if (!whole) {                          // a page that the row does not see weighs nothing, whatever its scale
#pragma unroll
        for (int q = 0; q < TW / 16; ++q)
          if (((uint32_t)(seen >> (16 * q)) & 0xffffu) == 0) { fk[q] = 0.f; lv[q] = -INFINITY; }
      }
      ok = warp_wait(&s_full[sg], turn);
      if (!ok) { fail(); break; }
      tc_fence_after();
      float x[TW];
      if (TW == 16) {
        tmem_ld16(lanes + sg * TT + w0, x);
      } else {
#pragma unroll
        for (int c = 0; c < TW; c += 32) tmem_ld32(lanes + sg * TT + w0 + c, x + c);
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&s_ready[sg]);
      // the row's largest score (factors are not negative), and how far it passes m + d with the value scale
      float top = -INFINITY, far = -INFINITY, xm[TW / 16];
#pragma unroll
      for (int q = 0; q < TW / 16; ++q) {
        float mx[4];
        if (whole) {
#pragma unroll
          for (int i = 0; i < 4; ++i) mx[i] = fmaxf(fmaxf(x[16 * q + i], x[16 * q + 4 + i]), fmaxf(x[16 * q + 8 + i], x[16 * q + 12 + i]));
        } else {
          const uint32_t sb = (uint32_t)(seen >> (16 * q));
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            mx[i] = -INFINITY;
#pragma unroll
            for (int k = 0; k < 4; ++k)
              if ((sb >> (4 * k + i)) & 1) mx[i] = fmaxf(mx[i], x[16 * q + 4 * k + i]);
          }
        }
        const float mq = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3]));
        xm[q] = mq == -INFINITY ? -INFINITY : mq * fk[q];
        top = fmaxf(top, xm[q]);
        far = fmaxf(far, (xm[q] - m) + (lv[q] - d));
      }
      if (j > 1) {                                            // this group's last product: it has read P and written O
        ok = warp_wait(&p_done[sg], turn ^ 1);
        if (!ok) { fail(); break; }
        tc_fence_after();
      }
      if (__any_sync(0xffffffffu, top - m > ATTN_SLACK || far > ATTN_SLACK)) {
        const float mn = fmaxf(m, top), drop = m - mn;
        float dn = fmaxf(d + drop, ATTN_NO_VALUE);
#pragma unroll
        for (int q = 0; q < TW / 16; ++q) dn = fmaxf(dn, (xm[q] - mn) + lv[q]);
        const float grow = ex2((d - dn) + drop);
        l *= ex2(drop);
        m = mn;
        d = dn;
        if (j > 1) {
#pragma unroll 1
          for (int c = 0; c < HD; c += 32) {
            float v[32];
            tmem_ld32(o_col + c, v);
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] *= grow;
            tmem_st32(o_col + c, v);
          }
        }
      }
      // x fk - m below is one operation, whose exact product differs from the rounded one in m by up to
      // 2^-25 |m|: scores of such size are rounded first
      if (fabsf(m) > 1048576.f) {
#pragma unroll
        for (int q = 0; q < TW / 16; ++q) {
#pragma unroll
          for (int i = 0; i < 16; ++i) x[16 * q + i] *= fk[q];
          fk[q] = 1.f;
        }
      }
      float2 ls = make_float2(0.f, 0.f), lt = ls;
      const float2 nm = make_float2(-m, -m);
#pragma unroll
      for (int q = 0; q < TW / 16; ++q) {
        const uint32_t sb = (uint32_t)(seen >> (16 * q));
        const float c = attn_factor(lv[q] - d + ATTN_SHIFT);
        const float2 c2 = make_float2(c, c), f2 = make_float2(fk[q], fk[q]);
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) {
          uint32_t w[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int k = 8 * hf + 2 * i;
            const float2 u = omq_fma2(make_float2(x[16 * q + k], x[16 * q + k + 1]), f2, nm);
            float2 p = make_float2(ex2(u.x), ex2(u.y));
            if (!whole) {
              if (!((sb >> k) & 1)) p.x = 0.f;
              if (!((sb >> (k + 1)) & 1)) p.y = 0.f;
            }
            if (i & 1) lt = omq_add2(lt, p);
            else ls = omq_add2(ls, p);
            const float2 e = omq_mul2(p, c2);
            w[i] = pack_half2(e.x, e.y);
          }
          sts128(prow + (((w0 / 8 + 2 * q + hf) ^ (r & 7)) << 4), make_uint4(w[0], w[1], w[2], w[3]));
        }
      }
      ls = omq_add2(ls, lt);
      l += ls.x + ls.y;
      fence_async_smem();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&p_ready[sg]);
    }
    // ---- join the two groups and the copies: the sums go through the converted tiles' buffers ----
    refs[(sg * 3 + 0) * BMR + r] = m;
    refs[(sg * 3 + 1) * BMR + r] = d;
    refs[(sg * 3 + 2) * BMR + r] = l;
    // each group waits for the last product into its own O, whose phases it has followed (the other's barrier may
    // be two phases behind for it); the barrier of the two orders both against what follows
    if (ok && holds && tiles > sg) {
      ok = warp_wait(&p_done[sg], ((tiles - sg + 1) / 2 - 1) & 1);
      if (!ok) fail();
      tc_fence_after();
    }
    tc_fence_before();
    asm volatile("bar.sync 1, 256;" ::: "memory");            // the references are written, the operands read
    tc_fence_after();
    const uint32_t sums = smem_u32(smem + CONV_OFF);          // [128][32] chunks of four channels, moved by the row
    if (ok && holds) {
      float mm = ATTN_NOTHING, dd = ATTN_NO_VALUE, L = 0.f;
      for (int c = 0; c < CP; ++c)
#pragma unroll
        for (int k = 0; k < 2; ++k) mm = fmaxf(mm, refs[k * 3 * BMR + c * SPAN + (r & (SPAN - 1))]);
      for (int c = 0; c < CP; ++c)
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const int at = k * 3 * BMR + c * SPAN + (r & (SPAN - 1));
          dd = fmaxf(dd, (refs[at] - mm) + refs[at + BMR]);
          L += refs[at + 2 * BMR] * ex2(refs[at] - mm);
        }
      const bool none = L == 0.f;                             // a NaN score is not an empty row
      const float c = none ? 0.f : ex2(dd - ATTN_SHIFT) / L;
      const float c0 = c * ex2((refs[r] - mm) + refs[BMR + r] - dd), c1 = c * ex2((refs[3 * BMR + r] - mm) + refs[4 * BMR + r] - dd);
      if (mine && sg == 0 && r < SPAN) {
        const int row = r0 + r;
        const int64_t at = (s.row0 + row / rep) * a.n_heads + g * rep + row % rep;
        const float lse = none ? -INFINITY : mm + log2f(L);
        if (a.n_split > 1) a.wl[at * a.n_split + split] = attn_part(mm, L);
        else if (a.lse) a.lse[at] = lse;
      }
#pragma unroll 1
      for (int ch = sg * 64; ch < sg * 64 + 64; ch += 32) {
        float v[32], u[32];
        if (tiles > 0) tmem_ld32(lanes + O_COL + ch, v);
        if (tiles > 1) tmem_ld32(lanes + O_COL + HD + ch, u);
#pragma unroll
        for (int i = 0; i < 32; ++i) {
          const float o = none ? 0.f : v[i] * c0;
          v[i] = none || tiles < 2 ? o : fmaf(u[i], c1, o);
        }
#pragma unroll
        for (int i = 0; i < 32; i += 4)
          sts128(sums + r * 512 + ((((ch + i) >> 2) ^ (r & 7)) << 4), make_uint4(__float_as_uint(v[i]), __float_as_uint(v[i + 1]),
                                                                             __float_as_uint(v[i + 2]), __float_as_uint(v[i + 3])));
      }
    }
    asm volatile("bar.sync 1, 256;" ::: "memory");
    const int n_rows = *abort_flag ? 0 : min(SPAN, R - r0);
    for (int q = (warp & 3) + 4 * sg; q < n_rows; q += 8) {   // a row per warp, four channels per lane
      float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
      for (int c = 0; c < CP; ++c) {
        const int at = c * SPAN + q;
        const uint4 w = lds128(sums + at * 512 + ((lane ^ (at & 7)) << 4));
        o.x += __uint_as_float(w.x); o.y += __uint_as_float(w.y); o.z += __uint_as_float(w.z); o.w += __uint_as_float(w.w);
      }
      const int row = r0 + q, head = g * rep + row % rep;
      const int64_t tok = s.row0 + row / rep;
      if (a.n_split > 1) {
        *reinterpret_cast<float4*>(a.wo + ((tok * a.n_heads + head) * a.n_split + split) * HD + 4 * lane) = o;
      } else {
        if (a.Of) *reinterpret_cast<float4*>(a.Of + tok * a.ldo + head * HD + 4 * lane) = o;
        if (a.Ob) {
          uint2 w;
          __nv_bfloat162* h = reinterpret_cast<__nv_bfloat162*>(&w);
          h[0] = __floats2bfloat162_rn(o.x, o.y);
          h[1] = __floats2bfloat162_rn(o.z, o.w);
          *reinterpret_cast<uint2*>(a.Ob + tok * a.ldo + head * HD + 4 * lane) = w;
        }
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem, 512);
  }
}

}  // namespace

template <int CP>
static omq_status launch(cudaStream_t st, const AttnArgs& a) {
  auto kern = kv_attention_tc_kernel<CP>;
  static std::atomic<uint64_t> allowed{0};
  OMQ_TRY(omq_allow_smem(allowed, kern, tc_smem(ATTN_MAX_CHUNK, 16)));
  CUtensorMap tk, tv;
  const int64_t rows = (int64_t)a.c.n_pages * a.c.n_kv * a.c.page;
  const int box = a.c.page < TT ? a.c.page : TT;
  if (!omq_make_map_u8(&tk, a.c.k, HD, rows, HD, box, HD) || !omq_make_map_u8(&tv, a.c.v, HD, rows, HD, box, HD))
    return OMQ_ERR_UNSUPPORTED;
  kern<<<dim3(a.n_split * a.c.n_kv * a.row_tiles, a.c.B), THREADS, tc_smem(a.chunk, a.c.page), st>>>(tk, tv, a);
  OMQ_LAUNCH_CHECK();
  return OMQ_OK;
}

// By the most rows that a KV head has in the call (16 x 4096 tokens of 24 rows 42 us with four copies, 53 with
// one; 64 ragged sequences of up to 40 rows 133 us with two, 144 with one).
omq_status attn_tc_launch(cudaStream_t st, const AttnArgs& a) {
  const int64_t rows = (int64_t)a.max_q * (a.n_heads / a.c.n_kv);
  if (rows <= BMR / 4) return launch<4>(st, a);
  if (rows <= BMR / 2) return launch<2>(st, a);
  return launch<1>(st, a);
}
