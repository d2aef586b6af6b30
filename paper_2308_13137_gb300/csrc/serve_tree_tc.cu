// Attention of draft trees over an 8-bit paged cache for more than 16 query rows per KV head: tcgen05 tiles of 128 rows x
// 64 tokens, on CTAs that share the tokens of all sequences evenly (serve_tree.cuh).
//
// The mathematics and the precision are those of serve_attn.cu.  A CTA holds one tile of 128 query rows, whose even and odd
// token tiles go to its two groups of softmax warps, or two tiles of rows, one for each group, which read the same
// converted token tiles (a unit of more than 128 rows).  Roles of the 20 warps:
//   0        TMA: raw code tiles of K and V (128-byte swizzle); it also walks the CTA's share
//   1, 2     issue S = Q K^T (128 x 64 x 128), one group each
//   3        issues O += P V (128 x 128 x 64) of both groups
//   4..7, 16..19   softmax, a row per thread: scores from tensor memory, weights in fp16 back to the columns that
//            the scores had, from where the second product reads them as its A operand
//   8..15    convert: K (8..11) and V (12..15) to fp16, one half row of 64 codes per thread; K is read K-major, V MN-major
// A group's scores have two buffers, so the product of its next tile runs while it works, and a tile costs it one
// wait.  Every barrier belongs to one group, and the groups differ only in which tiles they take.
#include "serve_tree.cuh"

namespace {

using namespace tc;

constexpr int HD = ATTN_HD, BMR = 128, TT = 64;
constexpr int RAW = 4;                               // ring depth of raw tiles (K | V); converted tiles: two of each
constexpr int RAW_BYTES = 2 * TT * HD;
constexpr int HALF = TT * HD;                        // one 64-channel half of a converted tile: 64 rows x 128 bytes
constexpr int OP_BYTES = 2 * HALF;
constexpr int Q_BYTES = BMR * HD * 2;
constexpr int WIN = 1024;                            // pages whose records are held at a time
constexpr int THREADS = 640;
constexpr int FIRST = 1, LAST = 2, DUAL = 4, DONE = 8;

struct Window {                                      // what warp 0 posts: tokens [t0, t1) of a piece
  TreePiece p;
  int t0, t1, flags;
};

template <int TILES>
struct Smem {
  static constexpr int CONV = TILES * Q_BYTES;       // K K | V V
  static constexpr int RAWS = CONV + 4 * OP_BYTES;
  static constexpr int ROW = RAWS + RAW * RAW_BYTES; // per row: factor, row among all
  static constexpr int REF = ROW + 2 * TILES * BMR * 4;                 // per group and row: m, d, l
  static constexpr int BAR = REF + 2 * 3 * BMR * 4;
  static constexpr int WINDOW = BAR + 256;
  static constexpr int SCAN = WINDOW + 2 * 64;
  static constexpr int PAGES = SCAN + (THREADS / 32 + 4) * 8;
  static constexpr int BYTES = PAGES + WIN * 12 + 1024;
};
static_assert(sizeof(Window) <= 64 && Smem<2>::BYTES <= 232448, "shared memory");

// 16 codes to fp16, into two swizzled 16-byte chunks of a 128-byte row
__device__ __forceinline__ void put16(uint32_t row, int c, uint32_t x, const uint4& u) {
  sts128(row + (((2 * c) ^ x) << 4), make_uint4(codes_lo(u.x), codes_hi(u.x), codes_lo(u.y), codes_hi(u.y)));
  sts128(row + (((2 * c + 1) ^ x) << 4), make_uint4(codes_lo(u.z), codes_hi(u.z), codes_lo(u.w), codes_hi(u.w)));
}

// D += A B with A (fp16, K-major: a 32-bit column holds two steps of K) in tensor memory
__device__ __forceinline__ void umma_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t bdesc, uint32_t idesc, uint32_t accum) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
      ::"r"(d_tmem), "r"(a_tmem), "l"(bdesc), "r"(idesc), "r"(accum)
      : "memory");
}

// eight 32-bit columns from registers into tensor memory (warp-collective; not waited for)
__device__ __forceinline__ void tmem_st8(uint32_t taddr, const uint32_t (&v)[8]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"r"(taddr), "r"(v[0]), "r"(v[1]),
               "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7])
               : "memory");
}

__device__ __forceinline__ void cta_sync() { asm volatile("bar.sync 0, 640;" ::: "memory"); }
__device__ __forceinline__ void group_sync(int id, int n) { asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(n) : "memory"); }

// CP: copies of a row (serve_attn_tc.cu); TILES: tiles of 128 rows that a CTA has room for
template <int CP, int TILES>
__global__ void __launch_bounds__(THREADS, 1)
    kv_attention_tree_tc_kernel(const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV, const TreeArgs t) {
  using S = Smem<TILES>;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  const AttnArgs& a = t.a;
  float* qs = reinterpret_cast<float*>(smem + S::ROW);
  int* token = reinterpret_cast<int*>(qs + TILES * BMR);
  float* refs = reinterpret_cast<float*>(smem + S::REF);
  uint64_t* raw_full = reinterpret_cast<uint64_t*>(smem + S::BAR);
  uint64_t* raw_empty = raw_full + RAW;
  uint64_t* k_ready = raw_empty + RAW;               // [2] K of a tile converted
  uint64_t* s_full = k_ready + 2;                    // [group][2] scores formed
  uint64_t* pv_ready = s_full + 4;                   // [group][2] V of the tile converted and its weights written
  uint64_t* pv_done = pv_ready + 4;                  // [group][2] product formed: weights (and scores) consumed
  uint64_t* drain = pv_done + 4;                     // [3] of the issuing warps
  uint32_t* tmem_holder = reinterpret_cast<uint32_t*>(drain + 3);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_holder + 1);
  Window* windows = reinterpret_cast<Window*>(smem + S::WINDOW);        // 64 bytes apart
  int* pid = reinterpret_cast<int*>(smem + S::PAGES);
  float* pks = reinterpret_cast<float*>(pid + WIN);
  float* plv = pks + WIN;
  const int P = a.c.page, pshift = 31 - __clz(P);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rep = a.n_heads / a.c.n_kv;

  const TreeShare share = tree_share<THREADS>(t, reinterpret_cast<int64_t*>(smem + S::SCAN));
  if (share.hi <= share.lo) return;
  if (threadIdx.x == 0) {
    for (int i = 0; i < RAW; ++i) { mbar_init(&raw_full[i], 1); mbar_init(&raw_empty[i], 8); }
    for (int i = 0; i < 2; ++i) mbar_init(&k_ready[i], 4);
    for (int i = 0; i < 4; ++i) { mbar_init(&s_full[i], 1); mbar_init(&pv_ready[i], 8); mbar_init(&pv_done[i], 1); }
    for (int i = 0; i < 3; ++i) mbar_init(&drain[i], 1);
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) tmem_alloc(tmem_holder, 512);
  tc_fence_before();
  cta_sync();
  tc_fence_after();
  const uint32_t tmem = *tmem_holder;
  constexpr uint32_t O_COL = 256;                    // scores: group g, buffer b at column 128 g + 64 b; O: 256 + 128 g
  auto fail = [&]() { omq_set_status(a.status, OMQ_ERR_TIMEOUT); *abort_flag = 1; };
  auto window = [&](int k) -> Window& { return *reinterpret_cast<Window*>(reinterpret_cast<uint8_t*>(windows) + (k & 1) * 64); };
  // items (token tiles) of a group in a window, and the group and item of a tile
  auto items_of = [](int tiles, bool dual, int g) { return dual ? tiles : (tiles + 1 - g) >> 1; };

  // Every role: for each window the barrier that ends the one before, its set-up, the barrier that starts it, its tiles.  A
  // role whose wait runs out sets the flag, which all see behind the next barrier.  J, N: tiles and items of the windows
  // before, which give the phases.
  // registers: 128 x 56 + 256 x 48 + 256 x 160 of the launch's 640 x 96
  if (warp < 4) asm volatile("setmaxnreg.dec.sync.aligned.u32 56;");
  if (warp == 0) {
    TreeWalk walk;
    walk.start(t, share);
    Window w;
    w.t1 = 0; w.flags = LAST;
    int J = 0;
    for (int k = 0;; ++k) {
      if (w.flags & LAST) {
        if (walk.next(t, &w.p)) {
          w.flags = FIRST | (TILES > 1 && w.p.R - w.p.r0 > BMR ? DUAL : 0);
          w.t1 = w.p.t0;
        } else {
          w.flags = DONE;
        }
      } else {
        w.flags &= ~FIRST;
      }
      if (!(w.flags & DONE)) {
        w.t0 = w.t1;
        w.t1 = min(w.p.t1, w.t0 + WIN * P);
        if (w.t1 == w.p.t1) w.flags |= LAST;
      }
      if (lane == 0) window(k) = w;
      cta_sync();
      if ((w.flags & DONE) || *abort_flag) break;
      cta_sync();
      const int tiles = (w.t1 - w.t0 + TT - 1) / TT, box = min(P, TT), per = TT / box;
      int i = 0;
      for (; i < tiles; ++i) {
        const int st = (J + i) % RAW;
        // row of the pool of each box that holds tokens, one lane each (-1: none, or a page out of range)
        const int tk = i * TT + lane * box, id = lane < per && tk < w.t1 - w.t0 ? pid[tk >> pshift] : -1;
        const int row = id < 0 ? -1 : (id * a.c.n_kv + w.p.g) * P + (tk & (P - 1));
        const uint32_t bytes = __popc(__ballot_sync(0xffffffffu, row >= 0)) * box * HD * 2;
        if (!warp_wait(&raw_empty[st], (((J + i) / RAW) & 1) ^ 1)) { fail(); break; }
        uint8_t* dst = smem + S::RAWS + st * RAW_BYTES;
        if (elect_one()) mbar_expect_tx(&raw_full[st], bytes);
        __syncwarp();
        for (int b = 0; b < per; ++b) {
          const int rb = __shfl_sync(0xffffffffu, row, b);
          if (rb >= 0 && elect_one()) {
            tma_load_3d(&tmK, &raw_full[st], dst + b * box * HD, 0, rb, 0);
            tma_load_3d(&tmV, &raw_full[st], dst + TT * HD + b * box * HD, 0, rb, 0);
          }
        }
        __syncwarp();
      }
      if (__any_sync(0xffffffffu, *abort_flag))      // no copy may land after this CTA has left
        for (int j = max(0, i - RAW); j < i; ++j)
          if (!wait_phase(&raw_full[(J + j) % RAW], ((J + j) / RAW) & 1)) break;
      J += tiles;
    }
  } else if (warp == 1 || warp == 2) {
    // ---------------- S of one group: the whole warp runs the loop, one lane issues ----------------
    const int g = warp - 1;
    constexpr uint32_t idS = idesc_f16(BMR, TT);
    const uint64_t dk = sdesc(smem_u32(smem + S::CONV), 16, 1024);
    int J = 0, N = 0;
    for (int k = 0;; ++k) {
      cta_sync();
      const Window& w = window(k);
      if ((w.flags & DONE) || *abort_flag) break;
      cta_sync();
      tc_fence_after();
      const bool dual = w.flags & DUAL;
      const int tiles = (w.t1 - w.t0 + TT - 1) / TT, items = items_of(tiles, dual, g);
      const uint64_t dq = sdesc(smem_u32(smem + (dual ? g * Q_BYTES : 0)), 16, 1024);
      for (int n = 0; n < items; ++n) {
        const int j = J + (dual ? n : 2 * n + g), b = (N + n) & 1;
        if (!warp_wait(&k_ready[j & 1], (j >> 1) & 1) || !warp_wait(&pv_done[2 * g + b], (((N + n) >> 1) & 1) ^ 1)) { fail(); break; }
        tc_fence_after();
        if (elect_one()) {
          const uint64_t k0 = dk + (uint64_t)((j & 1) * (OP_BYTES >> 4));
#pragma unroll
          for (int c = 0; c < HD / 16; ++c)
            umma_bf16(tmem + g * 128 + b * TT, dq + (((c >> 2) * (BMR * 128) + (c & 3) * 32) >> 4),
                      k0 + (((c >> 2) * HALF + (c & 3) * 32) >> 4), idS, c != 0);
          umma_commit(&s_full[2 * g + b]);
        }
        __syncwarp();
      }
      J += tiles;
      N += items;
    }
    if (*abort_flag) {                        // products in flight end before the tensor memory is released
      if (elect_one()) umma_commit(&drain[g]);
      wait_phase(&drain[g], 0);
    }
  } else if (warp == 3) {
    // ---------------- P V of both groups ----------------
    constexpr uint32_t idO = idesc_f16(BMR, HD) | (1u << 16);           // V is MN-major
    const uint64_t dv = sdesc(smem_u32(smem + S::CONV + 2 * OP_BYTES), HALF, 1024);
    int J = 0, N[2] = {0, 0};
    bool some[2] = {false, false};            // the group's O holds tiles of this piece
    for (int k = 0;; ++k) {
      cta_sync();
      const Window& w = window(k);
      if ((w.flags & DONE) || *abort_flag) break;
      if (w.flags & FIRST) some[0] = some[1] = false;
      cta_sync();
      tc_fence_after();
      const bool dual = w.flags & DUAL;
      const int tiles = (w.t1 - w.t0 + TT - 1) / TT;
      bool ok = true;
      for (int j = 0; j < tiles && ok; ++j) {
#pragma unroll
        for (int g = 0; g < 2; ++g) {
          if (!dual && (j & 1) != g) continue;
          const int n = N[g] + (dual ? j : j >> 1), b = n & 1;
          ok = ok && warp_wait(&pv_ready[2 * g + b], (n >> 1) & 1);
          if (!ok) break;
          tc_fence_after();
          if (elect_one()) {
            const uint64_t v0 = dv + (uint64_t)(((J + j) & 1) * (OP_BYTES >> 4));
#pragma unroll
            for (int c = 0; c < TT / 16; ++c)
              umma_ts(tmem + O_COL + g * HD, tmem + g * 128 + b * TT + c * 8, v0 + ((c * 2048) >> 4), idO, some[g] || c != 0);
            umma_commit(&pv_done[2 * g + b]);
          }
          some[g] = true;
          __syncwarp();
        }
      }
      J += tiles;
      for (int g = 0; g < 2; ++g) {           // a window ends with its products, so that the next one finds all free
        const int items = items_of(tiles, dual, g);
        N[g] += items;
        if (ok && items > 0) ok = warp_wait(&pv_done[2 * g + ((N[g] - 1) & 1)], ((N[g] - 1) >> 1) & 1);
      }
      if (!ok) fail();
    }
    if (*abort_flag) {
      if (elect_one()) umma_commit(&drain[2]);
      wait_phase(&drain[2], 0);
    }
  } else if (warp >= 8 && warp < 16) {
    // ---------------- convert ----------------
    asm volatile("setmaxnreg.dec.sync.aligned.u32 48;");
    const bool is_v = warp >= 12;
    const int tid = threadIdx.x & 127, r = tid & 63, h = tid >> 6;      // token, half of its channels
    const uint32_t x = r & 7, src0 = smem_u32(smem + S::RAWS) + (is_v ? TT * HD : 0) + r * HD;
    const uint32_t dst0 = smem_u32(smem + S::CONV) + (is_v ? 2 * OP_BYTES : 0) + h * HALF + r * 128;
    const uint64_t* freed = is_v ? pv_done : s_full;
    int J = 0, N[2] = {0, 0};
    for (int k = 0;; ++k) {
      cta_sync();
      const Window& w = window(k);
      if ((w.flags & DONE) || *abort_flag) break;
      const int np = (w.t1 - w.t0 + P - 1) >> pshift;
      for (int i = threadIdx.x - 256; i < np; i += 256) attn_page(a, w.p.b, w.p.g, (w.t0 >> pshift) + i, pid + i, pks + i, plv + i);
      cta_sync();
      const bool dual = w.flags & DUAL;
      const int tiles = (w.t1 - w.t0 + TT - 1) / TT;
      for (int j = 0; j < tiles; ++j) {
        const int rs = (J + j) % RAW, slot = (J + j) & 1;
        if (!warp_wait(&raw_full[rs], ((J + j) / RAW) & 1)) { fail(); break; }
        uint4 u[4];
#pragma unroll
        for (int c = 0; c < 4; ++c) u[c] = lds128(src0 + rs * RAW_BYTES + (((4 * h + c) ^ x) << 4));
        if (j > 1) {                          // the slot's last tile has been read
          bool ok = true;
          const int i = j - 2;
#pragma unroll
          for (int g = 0; g < 2; ++g)
            if (dual || (i & 1) == g) {
              const int n = N[g] + (dual ? i : i >> 1);
              ok = ok && warp_wait(const_cast<uint64_t*>(&freed[2 * g + (n & 1)]), (n >> 1) & 1);
            }
          if (!ok) { fail(); break; }
        }
#pragma unroll
        for (int c = 0; c < 4; ++c) put16(dst0 + slot * OP_BYTES, c, x, u[c]);
        fence_async_smem();                   // the converted tile -> visible to the tensor core
        __syncwarp();
        if (lane == 0) {
          mbar_arrive(&raw_empty[rs]);
          if (!is_v) {
            mbar_arrive(&k_ready[slot]);
          } else {
#pragma unroll
            for (int g = 0; g < 2; ++g)
              if (dual || (j & 1) == g) mbar_arrive(&pv_ready[2 * g + ((N[g] + (dual ? j : j >> 1)) & 1)]);
          }
        }
      }
      J += tiles;
      for (int g = 0; g < 2; ++g) N[g] += items_of(tiles, dual, g);
    }
  } else {
    // ---------------- softmax: one row per thread ----------------
    asm volatile("setmaxnreg.inc.sync.aligned.u32 160;");
    constexpr int SPAN = BMR / CP, TW = TT / CP;              // rows held, tokens of a thread
    const int sg = warp >= 16, qw = warp & 3, r = qw * 32 + lane;
    const uint32_t lanes = tmem + ((uint32_t)(qw * 32) << 16), s_col = lanes + sg * 128;
    const int w0 = r / SPAN * TW;                             // this copy's tokens of a tile
    float m = ATTN_NOTHING, d = ATTN_NO_VALUE, l = 0.f;
    int N = 0, n_piece = 0;                                   // items of the windows before, of the piece's
    for (int k = 0;; ++k) {
      cta_sync();
      const Window& w = window(k);
      if ((w.flags & DONE) || *abort_flag) break;
      const bool dual = w.flags & DUAL;
      const int start = w.p.len - w.p.nq, np = (w.t1 - w.t0 + P - 1) >> pshift;
      if (w.flags & FIRST) {
        // the query operand: fp16, K-major, 128-byte swizzle, two halves of 64 channels; a warp's rows in batches
        m = ATTN_NOTHING; d = ATTN_NO_VALUE; l = 0.f;
        n_piece = 0;
        const SeqRows s{w.p.row0, w.p.nq, w.p.len, true};
        const int held = TILES > 1 && dual ? 2 * BMR : SPAN;
        const int wid = sg * 4 + qw;
        for (int i0 = wid * 8; i0 < held; i0 += 64) {
          uint2 u[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) u[e] = attn_query_raw(a, s, w.p.g, rep, w.p.r0 + i0 + e, i0 + e < held ? w.p.R : 0, lane);
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const int i = i0 + e;
            if (i >= held) break;
            float v[4];
            int sh;
            attn_query_scaled(u[e], v, &sh);
            const uint2 h = make_uint2(pack_half2(v[0], v[1]), pack_half2(v[2], v[3]));
            const int tile = TILES > 1 ? i >> 7 : 0;
            for (int rr = i & (BMR - 1); rr < BMR; rr += SPAN) {
              uint8_t* row = smem + tile * Q_BYTES + (lane >> 4) * (BMR * 128) + rr * 128;
              *reinterpret_cast<uint2*>(row + (((lane & 15) >> 1 ^ (rr & 7)) << 4) + (lane & 1) * 8) = h;
              if (lane == 0) {
                qs[tile * BMR + rr] = __uint_as_float((uint32_t)(127 - sh) << 23);
                token[tile * BMR + rr] = w.p.row0 + min(w.p.r0 + i, w.p.R - 1) / rep;
              }
            }
          }
        }
        fence_async_smem();
      }
      cta_sync();
      const int at = (dual ? sg * BMR : 0) + r;               // the thread's row of those held
      const int row = w.p.r0 + (dual ? sg * BMR : 0) + (r & (SPAN - 1));
      const bool mine = row < w.p.R, idle = __all_sync(0xffffffffu, !mine);
      const float f = qs[at];
      const uint32_t* const bits = a.seen + (int64_t)token[at] * a.words;
      const int items = items_of((w.t1 - w.t0 + TT - 1) / TT, dual, sg);
      bool ok = true;
      for (int n = 0; n < items; ++n) {
        // the 16-token quarters, each of one page: score factor, log2 of the value scale; the tokens that
        // this row sees, as bits
        const int j = dual ? n : 2 * n + sg, b = (N + n) & 1, t0 = w.t0 + j * TT + w0;
        const uint32_t col = s_col + b * TT;
        float fk[TW / 16], lv[TW / 16];
        uint64_t seen = ~0ull;
        bool whole = t0 + TW <= start;
        if (!whole) seen = attn_window(bits, mine ? a.words : 0, w.p.nq, t0 - start);
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
        ok = warp_wait(&s_full[2 * sg + b], ((N + n) >> 1) & 1);
        if (!ok) { fail(); break; }
        tc_fence_after();
        if (!idle) {
        float x[TW];
        if (TW == 16) {
          tmem_ld16(col + w0, x);
        } else {
#pragma unroll
          for (int c = 0; c < TW; c += 32) tmem_ld32(col + w0 + c, x + c);
        }
        if (!whole) {
          // what the row does not see: minus infinity under any positive factor.  A page without a token that it sees gets
          // the factor 1 and no value scale, whatever it has; a factor of zero makes way for one that changes no score
#pragma unroll
          for (int q = 0; q < TW / 16; ++q) {
            const uint32_t sb = (uint32_t)(seen >> (16 * q)) & 0xffffu;
            if (sb == 0) { fk[q] = 1.f; lv[q] = -INFINITY; }
            else if (fk[q] == 0.f) fk[q] = 1e-30f;
#pragma unroll
            for (int i = 0; i < 16; ++i)
              if (!((sb >> i) & 1)) x[16 * q + i] = -INFINITY;
          }
        }
        // the row's largest score (factors are not negative), and how far it passes m + d with the value scale
        float top = -INFINITY, far = -INFINITY, xm[TW / 16];
#pragma unroll
        for (int q = 0; q < TW / 16; ++q) {
          float mx[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) mx[i] = fmaxf(fmaxf(x[16 * q + i], x[16 * q + 4 + i]), fmaxf(x[16 * q + 8 + i], x[16 * q + 12 + i]));
          const float mq = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3]));
          xm[q] = mq == -INFINITY ? -INFINITY : mq * fk[q];
          top = fmaxf(top, xm[q]);
          far = fmaxf(far, (xm[q] - m) + (lv[q] - d));
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
          if (n_piece + n > 0) {              // O of the tiles before
            const int last = N + n - 1;
            ok = warp_wait(&pv_done[2 * sg + (last & 1)], (last >> 1) & 1);
            if (!ok) { fail(); break; }
            tc_fence_after();
#pragma unroll 1
            for (int c = 0; c < HD; c += 16) {
              float v[16];
              tmem_ld16(lanes + O_COL + sg * HD + c, v);
#pragma unroll
              for (int i = 0; i < 16; ++i) v[i] *= grow;
              tmem_st8(lanes + O_COL + sg * HD + c, reinterpret_cast<const uint32_t(&)[8]>(v[0]));
              tmem_st8(lanes + O_COL + sg * HD + c + 8, reinterpret_cast<const uint32_t(&)[8]>(v[8]));
            }
            asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
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
          uint32_t pw[8];
          const float c = attn_factor(lv[q] - d + ATTN_SHIFT);
          const float2 c2 = make_float2(c, c), f2 = make_float2(fk[q], fk[q]);
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const float2 u = omq_fma2(make_float2(x[16 * q + 2 * i], x[16 * q + 2 * i + 1]), f2, nm);
            const float2 p = make_float2(ex2(u.x), ex2(u.y));
            if (i & 1) lt = omq_add2(lt, p);
            else ls = omq_add2(ls, p);
            const float2 e = omq_mul2(p, c2);
            pw[i] = pack_half2(e.x, e.y);
          }
          tmem_st8(col + w0 / 2 + 8 * q, pw);                 // to the scores' first 32 columns
        }
        ls = omq_add2(ls, lt);
        l += ls.x + ls.y;
        if (CP > 1) {                         // the other copies' tokens weigh nothing here
          const uint32_t zero[8] = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
          for (int c = 0; c < TT / 16; ++c)
            if (c / (TW / 16) != r / SPAN) tmem_st8(col + 8 * c, zero);
        }
        asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&pv_ready[2 * sg + b]);
      }
      N += items;
      n_piece += items;
      if (!(w.flags & LAST)) continue;

      // ---- the piece's end: O over the sum of weights, to the outputs or the partial results ----
      if (ok && items > 0) {
        const int last = N - 1;
        ok = warp_wait(&pv_done[2 * sg + (last & 1)], (last >> 1) & 1);
        if (!ok) fail();
      }
      tc_fence_after();
      float c0, c1 = 0.f, lse;
      if (TILES > 1 && dual) {
        const bool none = l == 0.f;                           // a NaN score is not an empty row
        c0 = none ? 0.f : ex2(d - ATTN_SHIFT) / l;
        lse = none ? -INFINITY : m + log2f(l);
        if (none || n_piece == 0) c0 = 0.f;
      } else {
        refs[(sg * 3 + 0) * BMR + r] = m;
        refs[(sg * 3 + 1) * BMR + r] = d;
        refs[(sg * 3 + 2) * BMR + r] = l;
        tc_fence_before();
        group_sync(3, 256);                                   // both groups' references, and their products are done
        tc_fence_after();
        float mm = ATTN_NOTHING, dd = ATTN_NO_VALUE, L = 0.f;
        for (int c = 0; c < CP; ++c)
#pragma unroll
          for (int g = 0; g < 2; ++g) mm = fmaxf(mm, refs[g * 3 * BMR + c * SPAN + (r & (SPAN - 1))]);
        for (int c = 0; c < CP; ++c)
#pragma unroll
          for (int g = 0; g < 2; ++g) {
            const int i = g * 3 * BMR + c * SPAN + (r & (SPAN - 1));
            dd = fmaxf(dd, (refs[i] - mm) + refs[i + BMR]);
            L += refs[i + 2 * BMR] * ex2(refs[i] - mm);
          }
        const bool none = L == 0.f;
        const float c = none ? 0.f : ex2(dd - ATTN_SHIFT) / L;
        c0 = none ? 0.f : c * ex2((refs[r] - mm) + refs[BMR + r] - dd);
        c1 = none ? 0.f : c * ex2((refs[3 * BMR + r] - mm) + refs[4 * BMR + r] - dd);
        lse = none ? -INFINITY : mm + log2f(L);
      }
      const int n_a = dual ? n_piece : (sg == 0 ? n_piece : (w.p.t1 - w.p.t0 + 2 * TT - 1) / (2 * TT));      // group 0's tiles
      const int n_b = dual ? 0 : (w.p.t1 - w.p.t0 + TT - 1) / TT - n_a;
      const int first = w.p.r0 + (dual ? sg * BMR : 0), rows = min(dual ? BMR : SPAN, w.p.R - first);
      if (mine && (dual || sg == 0) && r < SPAN) {
        if (w.p.part >= 0) t.pl[(int64_t)w.p.part * t.cost.rows + (dual ? sg * BMR : 0) + r] = lse;
        else if (a.lse) a.lse[(int64_t)(w.p.row0 + row / rep) * a.n_heads + w.p.g * rep + row % rep] = lse;
      }
      // 64 channels at a time through shared memory (the queries' own tile: its last product is done), rows of 256 bytes
      const uint32_t stage = smem_u32(dual ? smem + sg * Q_BYTES : (sg == 0 ? smem : smem + S::CONV));
      for (int hf = dual ? 0 : sg; hf < (dual ? 2 : sg + 1); ++hf) {
#pragma unroll 1
        for (int ch = 0; ch < 64; ch += 32) {
          float v[32], u[32];
          const uint32_t o = lanes + O_COL + hf * 64 + ch;
          if (n_a > 0) tmem_ld32(o + (dual ? sg * HD : 0), v);
          if (n_b > 0) tmem_ld32(o + HD, u);
#pragma unroll
          for (int i = 0; i < 32; ++i) {
            const float y = n_a > 0 && c0 != 0.f ? v[i] * c0 : 0.f;
            v[i] = n_b > 0 && c1 != 0.f ? fmaf(u[i], c1, y) : y;
          }
#pragma unroll
          for (int i = 0; i < 32; i += 4)
            sts128(stage + r * 256 + ((((ch + i) >> 2) ^ (r & 15)) << 4),
                   make_uint4(__float_as_uint(v[i]), __float_as_uint(v[i + 1]), __float_as_uint(v[i + 2]), __float_as_uint(v[i + 3])));
        }
        group_sync(1 + sg, 128);
        const int n_rows = *abort_flag ? 0 : rows;
        for (int q = 2 * qw + (lane >> 4); q < n_rows; q += 8) {        // half a row per half warp
          float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
          for (int c = 0; c < CP; ++c) {
            const int i = c * SPAN + q;
            const uint4 y = lds128(stage + i * 256 + (((lane & 15) ^ (i & 15)) << 4));
            o.x += __uint_as_float(y.x); o.y += __uint_as_float(y.y); o.z += __uint_as_float(y.z); o.w += __uint_as_float(y.w);
          }
          const int rw = first + q, ch = hf * 64 + 4 * (lane & 15);
          if (w.p.part >= 0) {
            *reinterpret_cast<float4*>(t.po + ((int64_t)w.p.part * t.cost.rows + (rw - w.p.r0)) * HD + ch) = o;
          } else {
            const int64_t to = (int64_t)(w.p.row0 + rw / rep) * a.ldo + (w.p.g * rep + rw % rep) * HD + ch;
            if (a.Of) *reinterpret_cast<float4*>(a.Of + to) = o;
            if (a.Ob) {
              uint2 y;
              __nv_bfloat162* h = reinterpret_cast<__nv_bfloat162*>(&y);
              h[0] = __floats2bfloat162_rn(o.x, o.y);
              h[1] = __floats2bfloat162_rn(o.z, o.w);
              *reinterpret_cast<uint2*>(a.Ob + to) = y;
            }
          }
        }
        group_sync(1 + sg, 128);
      }
      tc_fence_before();
    }
  }
  tc_fence_before();
  cta_sync();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem, 512);
  }
}

template <int CP, int TILES>
omq_status launch(cudaStream_t st, const TreeArgs& t, int n_ctas) {
  auto kern = kv_attention_tree_tc_kernel<CP, TILES>;
  static std::atomic<uint64_t> allowed{0};
  OMQ_TRY(omq_allow_smem(allowed, kern, Smem<TILES>::BYTES));
  CUtensorMap tk, tv;
  const omq_kv_cache& c = t.a.c;
  const int64_t rows = (int64_t)c.n_pages * c.n_kv * c.page;
  const int box = c.page < TT ? c.page : TT;
  if (!omq_make_map_u8(&tk, c.k, HD, rows, HD, box, HD) || !omq_make_map_u8(&tv, c.v, HD, rows, HD, box, HD))
    return OMQ_ERR_UNSUPPORTED;
  kern<<<n_ctas, THREADS, Smem<TILES>::BYTES, st>>>(tk, tv, t);
  OMQ_LAUNCH_CHECK();
  return OMQ_OK;
}

}  // namespace

// By the most rows that a KV head has in the call.
omq_status tree_tc_launch(cudaStream_t st, const TreeArgs& t, int n_ctas) {
  const int64_t rows = (int64_t)t.a.max_q * (t.a.n_heads / t.a.c.n_kv);
  if (rows <= BMR / 4) return launch<4, 1>(st, t, n_ctas);
  if (rows <= BMR / 2) return launch<2, 1>(st, t, n_ctas);
  if (rows <= BMR) return launch<1, 1>(st, t, n_ctas);
  return launch<1, 2>(st, t, n_ctas);
}
