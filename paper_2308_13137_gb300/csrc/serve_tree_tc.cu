// Attention of draft trees over an 8-bit paged cache for more than 16 query rows per KV head: tcgen05 tiles of 128 rows x
// 64 tokens, on CTAs that share the tokens of all sequences evenly (serve_tree.cuh).
//
// The mathematics and the precision are those of serve_attn.cu.  Shared memory sets the layout: its 128 bytes a cycle carry the
// converted tiles in and the products' operands out.  So the queries and the weights, the A operands, lie in tensor
// memory, and a tile of 64 tokens costs 768 cycles there (codes in and out, converted in and out), 517 on the tensor
// cores, and its 16 KB of codes 725 from HBM.  Roles of the 28 warps:
//   0, 3     issue S = Q K^T (128 x 64 x 128), of one group each (an issue and the waits before it are 700 cycles)
//   1        issues O += P V (128 x 128 x 64)
//   2        walks the CTA's share: chunks of up to 1024 tokens, with the records of their pages
//   4..11    softmax, a row per thread, two groups (even and odd tiles) with their own references, sums and accumulators:
//            scores from tensor memory, weights in fp16 to columns of their own, so that the group's next scores are
//            formed meanwhile
//   12..27   convert K and V to fp16, two sets (even and odd tiles), from rings of their own that bulk copies fill.  K is
//            read K-major, V MN-major, both from [half][64 tokens][128 bytes] swizzled tiles
// Tile j's converted V lies in the place j % 3, its K in one of its group's two places, its scores and weights in its group's.
// Barriers of what one warp does in order of tiles go by place; the scores of the two groups come in no order, so theirs
// belong to a group (a phase may be waited for only when the one before it is known to be over).  Chunks of a piece follow one
// another without a stop; between pieces the next one's queries are written, and its first scores formed, before the last one's
// output is, by the softmax warps themselves.
// Time: a tile of 128 rows takes 1250 cycles.  Of these a scheduler issues for 635 (64 scores of its two softmax warps' rows 345,
// the exponentials alone 267; the maximum 80; the conversion 210) and shared memory works for 768; the rest are waits between the
// roles, a latency and no limit of the chip.  With copies of rows (32 or 16 scores per thread) a tile takes about 1000.  A piece costs about
// 13000 cycles beside its tiles (queries, joining, output), which short sequences feel.  Measured: 16 sequences of up to 8192 tokens,
// 512 rows on each of 8 KV heads, 209 us, 0.82 PFLOP/s (235 us with pages of 16 tokens); 64 of up to 4099 tokens, up to 104 rows,
// 137 us; 16 of up to 8192, 64 rows, 57 us; 4 of up to 131072 tokens, 32 rows, 190 us, 4.4 TB/s, and 64 rows, 168 us.
// No role may spill much: local memory passes the small rest of the L1 here, and a softmax that reloads a dozen registers in every
// tile took half again as long.  What is spilled now: 84 bytes with four pages per tile, 28 with one, 4 with copies of rows.  Two threads per
// row (16 softmax warps): 290 us where one took 265, bound by issue.
#include <type_traits>

#include "serve_tree.cuh"

namespace {

using namespace tc;

constexpr int HD = ATTN_HD, BMR = 128, TT = 64;
constexpr int HALF = TT * HD;                        // one 64-channel half of a converted tile: 64 rows x 128 bytes
constexpr int OP_BYTES = 2 * HALF;
constexpr int BUF = 3, KBUF = 4;                     // places of V and of K
constexpr int CHUNK = 1024, PAGES = CHUNK / 16, RING = 8;      // tokens, pages at most of a chunk; chunks in flight
constexpr int RAW_BYTES = 16 * HD, DEPTH = 2;        // a warp's share of a tile's codes, its two slots
constexpr int THREADS = 896;
constexpr int FIRST = 1, LAST = 2, DONE = 4;         // of a piece; the share's end
constexpr uint32_t Q_COL = 0, S_COL = 64, P_COL = 192, O_COL = 256;       // tensor memory: Q | of the two groups: scores | weights | O

struct __align__(16) Chunk {                         // tokens [t0, t1) of a piece
  TreePiece p;
  int t0, t1, flags;
  float4 page[PAGES];                                // score factor, log2 of the value scale, place of its rows in the pool (-1: none)
};

constexpr int K_CONV = 0, V_CONV = K_CONV + KBUF * OP_BYTES, STAGE = V_CONV + BUF * OP_BYTES;
constexpr int RAW = STAGE + BMR * HD * 2;            // the stage: queries in fp16, or 32 channels of O from each group
constexpr int ROW = RAW + 16 * DEPTH * RAW_BYTES;    // factor of each row
constexpr int REF = ROW + BMR * 4;                   // [group][m, d, l]
constexpr int BAR = REF + 2 * 3 * BMR * 4, SCAN = BAR + 768, CHUNKS = SCAN + (THREADS / 32 + 4) * 8;
constexpr int SMEM = CHUNKS + RING * (int)sizeof(Chunk) + 1024;
static_assert(SMEM <= 232448 && CHUNKS % 16 == 0, "shared memory");

// D += A B with A (fp16, K-major: a 32-bit column holds two steps of K) in tensor memory
__device__ __forceinline__ void umma_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t bdesc, uint32_t idesc, uint32_t accum) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
      ::"r"(d_tmem), "r"(a_tmem), "l"(bdesc), "r"(idesc), "r"(accum)
      : "memory");
}

// mbarriers by their shared addresses (32 bits: the roles here have few registers)
__device__ __forceinline__ bool bar_test(uint32_t bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(ok)
      : "r"(bar), "r"(parity)
      : "memory");
  return ok != 0;
}
// A converged warp's bounded wait.  The phase is mostly over already: a test costs 50 cycles, a wait 120.  A try without a time
// hint suspends the warp until the phase completes, or for 3.8 us (measured: a wait that nothing ends), and costs one instruction;
// with a hint it is a loop of polls, and those of this kernel's 28 warps were more than half of all its instructions.
__device__ __forceinline__ bool wait_tries(uint32_t bar, uint32_t parity, uint32_t tries) {
  bool ok = bar_test(bar, parity);
  for (uint32_t i = 0; !__all_sync(0xffffffffu, ok); ++i) {
    if (i == tries) return false;
    uint32_t p;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(p)
        : "r"(bar), "r"(parity)
        : "memory");
    ok = p != 0;
  }
  return true;
}
__device__ __forceinline__ void bar_arrive(uint32_t bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void arrive(uint32_t bar, int lane) {          // of a warp
  __syncwarp();
  if (lane == 0) bar_arrive(bar);
}
__device__ __forceinline__ void commit(uint32_t bar) {                    // tcgen05 products so far
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
// bytes of global memory on their way to shared memory, counted on bar (16-byte aligned)
__device__ __forceinline__ void fetch_bytes(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
               ::"r"(dst), "l"(reinterpret_cast<uint64_t>(src)), "r"(bytes), "r"(bar)
               : "memory");
}

// 32 lanes x 32 consecutive 32-bit columns into registers (warp-collective; not waited for)
__device__ __forceinline__ void tmem_ld32_async(uint32_t taddr, float* v) {
  uint32_t* r = reinterpret_cast<uint32_t*>(v);
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
      "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
        "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]),
        "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]),
        "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(taddr));
}
__device__ __forceinline__ float max3(float a, float b, float c) {
  float d;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}
__device__ __forceinline__ float min_nan(float a, float b) {
  asm("min.NaN.f32 %0, %0, %1;" : "+f"(a) : "f"(b));
  return a;
}
__device__ __forceinline__ float max_nan(float a, float b) {
  asm("max.NaN.f32 %0, %0, %1;" : "+f"(a) : "f"(b));
  return a;
}

// eight 32-bit columns from registers into tensor memory (warp-collective; not waited for)
__device__ __forceinline__ void tmem_st8(uint32_t taddr, const uint32_t (&v)[8]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"r"(taddr), "r"(v[0]), "r"(v[1]),
               "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7])
               : "memory");
}

// place j % 3 of a tile and the parity of j / 3
struct Place {
  int b; uint32_t ph;
  __device__ __forceinline__ void move(int n) {      // n <= 3
    b += n;
    if (b >= BUF) { b -= BUF; ph ^= 1; }
  }
  __device__ __forceinline__ Place before() const { return b >= 2 ? Place{b - 2, ph} : Place{b + BUF - 2, ph ^ 1}; }      // of tile j - 2
};

// CP: copies of a row (serve_attn_tc.cu); NQ: pages (at most) that a softmax thread's 64 / CP tokens of a tile lie on; TEST: the
// waits' limit and the chunk that never comes are the self-test's (a limit from memory, 16 x 64 rows 210 us in place of 207)
template <int CP, int NQ, bool TEST>
__global__ void __launch_bounds__(THREADS, 1) kv_attention_tree_tc_kernel(const TreeArgs t) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* const smem = smem_raw + (-smem_u32(smem_raw) & 1023u);
  const AttnArgs& a = t.a;
  const uint32_t bars = smem_u32(smem + BAR);
  const uint32_t k_full = bars;                      // [4] K of a tile converted
  const uint32_t s_full = k_full + 8 * KBUF;         // [4] scores formed (K consumed)
  const uint32_t pv_ready = s_full + 8 * KBUF;       // [3] V of the tile converted and its weights written
  const uint32_t pv_done = pv_ready + 8 * BUF;       // [3] product formed: weights and V consumed
  const uint32_t s_free = pv_done + 8 * BUF;         // [2] scores read
  const uint32_t o_free = s_free + 16;               // both accumulators read
  const uint32_t q_ready = o_free + 8;               // the piece's queries lie in tensor memory
  const uint32_t meet = q_ready + 8;                 // of the softmax warps
  const uint32_t chunk_full = meet + 8;              // [RING]
  const uint32_t chunk_empty = chunk_full + 8 * RING;                     // [RING]
  const uint32_t raw_full = chunk_empty + 8 * RING;  // [converting warp][DEPTH]
  const uint32_t q_seen = raw_full + 8 * 16 * DEPTH; // both issuing warps have come to the piece
  const uint32_t drain = q_seen + 8;                 // [4] of the issuing warps
  constexpr int N_BAR = 2 * KBUF + 2 * BUF + 5 + 2 * RING + 16 * DEPTH + 5;
  uint32_t* tmem_holder = reinterpret_cast<uint32_t*>(smem + BAR + 8 * N_BAR);
  static_assert(8 * N_BAR + 8 <= SCAN - BAR, "");
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_holder + 1);
  Chunk* chunks = reinterpret_cast<Chunk*>(smem + CHUNKS);
  const int P = a.c.page, pshift = 31 - __clz(P);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  const TreeShare share = tree_share<THREADS>(t, reinterpret_cast<int64_t*>(smem + SCAN));
  if (share.hi <= share.lo) return;
  if (threadIdx.x < N_BAR) {                  // (one thread after the other's barrier: 170 cycles each)
    const uint32_t at = bars + 8 * threadIdx.x;
    const uint32_t count = at < s_full ? 4 : (at < pv_ready ? 1 : (at < pv_done ? 8 : (at < s_free ? 1 : (at < o_free ? 4 :
                           (at < chunk_full ? 8 : (at < chunk_empty ? 1 : (at < raw_full ? 27 : (at == q_seen ? 2 : 1))))))));
    mbar_init(reinterpret_cast<uint64_t*>(smem + BAR) + threadIdx.x, count);
    if (threadIdx.x == 0) *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) tmem_alloc(tmem_holder, 512);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_holder;
  // a role whose wait runs out sets the flag and leaves; those that wait for it follow.  All meet at the end
  auto fail = [&]() { omq_set_status(a.status, OMQ_ERR_TIMEOUT); *abort_flag = 1; };
  auto soon = [&](uint32_t bar, uint32_t parity) { return wait_tries(bar, parity, TEST ? t.tries : TREE_TRIES); };
  // for what is in flight when a role leaves, whatever the limit of its waits
  auto landed = [&](uint32_t bar, uint32_t parity) { return wait_tries(bar, parity, TREE_TRIES); };
  auto chunk_at = [&](int k) -> Chunk& { return chunks[k % RING]; };
  auto chunk_wait = [&](int k) { return soon(chunk_full + 8 * (k % RING), (k / RING) & 1); };
  auto tiles_of = [](const Chunk& w) { return (w.t1 - w.t0 + TT - 1) / TT; };

  // registers: 128 x 56 + 256 x 144 + 512 x 40 of the launch's 896 x 72; with copies of rows 128 x 56 + 256 x 120 + 512 x 48
  if (warp < 4) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 56;");
    if (warp == 0 || warp == 3) {
      // ---------------- S of one group: the whole warp runs the loop, one lane issues ----------------
      constexpr uint32_t idS = idesc_f16(BMR, TT);
      const uint64_t dk = sdesc(smem_u32(smem + K_CONV), 16, 1024);
      const int g = warp == 3;
      int i = g, n = 0;                       // the next tile in the chunk, the group's tiles so far
      uint32_t q_ph = 0;
      bool ok = true;
      for (int k = 0; ok; ++k) {
        ok = chunk_wait(k);
        if (!ok) break;
        const Chunk& w = chunk_at(k);
        if (w.flags & DONE) break;
        const int tiles = tiles_of(w);
        if (w.flags & FIRST) {                // (with a tile of it or without: a phase that nobody waits for can be missed)
          ok = soon(q_ready, q_ph);
          q_ph ^= 1;
          arrive(q_seen, lane);
        }
        for (; i < tiles && ok; i += 2) {
          const int b = 2 * g + (n & 1);
          ok = soon(k_full + 8 * b, (n >> 1) & 1) && soon(s_free + 8 * g, (n & 1) ^ 1);
          if (!ok) break;
          tc_fence_after();
          if (elect_one()) {
            const uint64_t k0 = dk + (uint64_t)(b * (OP_BYTES >> 4));
#pragma unroll
            for (int c = 0; c < HD / 16; ++c)
              umma_ts(tmem + S_COL + g * TT, tmem + Q_COL + c * 8, k0 + (((c >> 2) * HALF + (c & 3) * 32) >> 4), idS, c != 0);
            commit(s_full + 8 * b);
          }
          __syncwarp();
          ++n;
        }
        i -= tiles;                           // of the next chunk
        arrive(chunk_empty + 8 * (k % RING), lane);
      }
      if (!ok) fail();
    } else if (warp == 1) {
      // ---------------- P V ----------------
      constexpr uint32_t idO = idesc_f16(BMR, HD) | (1u << 16);           // V is MN-major
      const uint64_t dv = sdesc(smem_u32(smem + V_CONV), HALF, 1024);
      Place at{0, 0};
      int g = 0;                              // the tile's group
      bool ok = true, some[2] = {false, false};                           // the group's O holds tiles of this piece
      for (int k = 0; ok; ++k) {
        ok = chunk_wait(k);
        if (!ok) break;
        const Chunk& w = chunk_at(k);
        if (w.flags & DONE) break;
        if (w.flags & FIRST) some[0] = some[1] = false;
        const int tiles = tiles_of(w);
        for (int i = 0; i < tiles && ok; ++i) {
          ok = soon(pv_ready + 8 * at.b, at.ph);
          if (!ok) break;
          tc_fence_after();
          if (elect_one()) {
            const uint64_t v0 = dv + (uint64_t)(at.b * (OP_BYTES >> 4));
#pragma unroll
            for (int c = 0; c < TT / 16; ++c)
              umma_ts(tmem + O_COL + g * HD, tmem + P_COL + g * 32 + c * 8, v0 + ((c * 2048) >> 4), idO,
                      (g ? some[1] : some[0]) || c != 0);
            commit(pv_done + 8 * at.b);
          }
          __syncwarp();
          some[0] |= g == 0; some[1] |= g == 1;
          at.move(1);
          g ^= 1;
        }
        arrive(chunk_empty + 8 * (k % RING), lane);
      }
      if (!ok) fail();
    } else if (warp == 2) {
      // ---------------- the walk ----------------
      TreeWalk walk;
      walk.start(t, share);
      TreePiece p;
      int t1 = 0, flags = LAST;
      for (int k = 0;; ++k) {
        if (flags & LAST) {
          flags = walk.next(t, &p) ? FIRST : DONE;
          t1 = p.t0;
        } else {
          flags = 0;
        }
        const int t0 = t1;
        if (!(flags & DONE)) {
          t1 = min(p.t1, t0 + CHUNK);
          if (t1 == p.t1) flags |= LAST;
        }
        if (TEST && k == t.withhold) break;   // this chunk never comes
        if (!soon(chunk_empty + 8 * (k % RING), ((k / RING) & 1) ^ 1)) { fail(); break; }
        Chunk& w = chunk_at(k);
        if (flags & FIRST) {                  // the unit's queries to L2, by tokens
          const int rep = t.rep, i0 = p.r0 / rep, i1 = (min(p.R, p.r0 + BMR) + rep - 1) / rep;
          for (int i = i0 + lane; i < i1; i += 32)
            asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(reinterpret_cast<uint64_t>(a.Q + (int64_t)(p.row0 + i) * a.ldq + p.g * rep * HD)), "r"(rep * HD * 2) : "memory");
        }
        if (!(flags & DONE)) {
          const int np = (t1 - t0 + P - 1) >> pshift;
          for (int i = lane; i < np; i += 32) {
            int id;
            float4 x;
            attn_page(a, p.b, p.g, (t0 >> pshift) + i, &id, &x.x, &x.y);
            x.z = __int_as_float(id < 0 ? -1 : (id * a.c.n_kv + p.g) * P);          // (below 2^31: attention_check)
            x.w = 0.f;
            w.page[i] = x;
          }
        }
        if (lane == 0) { w.p = p; w.t0 = t0; w.t1 = t1; w.flags = flags; }
        arrive(chunk_full + 8 * (k % RING), lane);
        if (flags & DONE) break;
      }
    }
    // The products end before the tensor memory is released.  (Without a condition: a wait of another role may run out, and
    // end the CTA, after this one has issued all it had.)
    __syncwarp();
    if (warp != 2) {
      if (elect_one()) commit(drain + 8 * warp);
      landed(drain + 8 * warp, 0);
    }
  } else if (warp >= 12) {
    // ---------------- convert ----------------
    if (CP > 1) asm volatile("setmaxnreg.dec.sync.aligned.u32 48;");
    else asm volatile("setmaxnreg.dec.sync.aligned.u32 40;");
    const int cw = warp - 12, set = cw >> 3, q = warp & 3;
    const bool is_v = cw & 4;
    // 16 codes of channels 16 c .. of tokens 16 q + r + 4 e.  The eight lanes of a load or store phase have the first half of
    // one token's row and the second half of its neighbour's, whose swizzle differs in the lowest bit: eight
    // 16-byte bank groups both times
    const int r = (lane >> 2 & 1) | lane >> 4 << 1, c = (lane & 3) | ((lane >> 2 ^ lane >> 3) & 1) << 2;
    const uint32_t dst0 = smem_u32(smem + (is_v ? V_CONV : K_CONV)) + (c >> 2) * HALF + (16 * q + r) * 128;
    const uint32_t x0 = 2 * (c & 3) ^ r;      // chunk of the row, swizzled with r + 4 e
    const uint8_t* const pool = is_v ? a.c.v : a.c.k;
    const uint32_t slots = smem_u32(smem + RAW) + cw * (DEPTH * RAW_BYTES), mine = r * HD + c * 16;
    const uint32_t full = is_v ? pv_ready : k_full, freed = is_v ? pv_done : s_full, got = raw_full + 8 * cw * DEPTH;
    bool ok = true, done = false;
    int k = 0, tiles = -1, i = set;           // the chunk fetched from, its tiles (-1: not looked at), the next one of this set's
    int slot = 0, on_way = 0;                 // the slot to convert, tiles on their way
    uint32_t ph = 0;
    Place at{is_v ? set : 2 * set, 0};
    while (true) {
      while (on_way < DEPTH && !done) {       // the next tiles' rows on their way
        if (tiles < 0) {
          // while a tile is on its way the next chunk is not waited for: it may come only once that tile's chunk is over
          if (on_way == 0) ok = chunk_wait(k);
          else if (!__all_sync(0xffffffffu, bar_test(chunk_full + 8 * (k % RING), (k / RING) & 1))) break;
          if (!ok) break;
          done = chunk_at(k).flags & DONE;
          if (done) break;
          tiles = tiles_of(chunk_at(k));
        }
        if (i >= tiles) {
          arrive(chunk_empty + 8 * (k % RING), lane);
          ++k;
          i -= tiles;                         // of the next chunk
          tiles = -1;
          continue;
        }
        const Chunk& w = chunk_at(k);
        const int tk = i * TT + 16 * q, at0 = tk < w.t1 - w.t0 ? __float_as_int(w.page[tk >> pshift].z) : -1, s = slot ^ on_way;
        if (elect_one()) {
          if (at0 < 0) {
            bar_arrive(got + 8 * s);          // unseen, whatever the slot holds
          } else {
            fetch_bytes(slots + s * RAW_BYTES, pool + ((int64_t)at0 + (tk & (P - 1))) * HD, RAW_BYTES, got + 8 * s);
          }
        }
        __syncwarp();
        i += 2;
        ++on_way;
      }
      if (!ok || on_way == 0) break;
      ok = soon(got + 8 * slot, ph) && soon(freed + 8 * at.b, at.ph ^ 1);
      if (!ok) break;
      const uint32_t src = slots + mine + slot * RAW_BYTES, dst = dst0 + at.b * OP_BYTES;
#pragma unroll
      for (int e = 0; e < 4; e += 2) {
        const uint4 u = lds128(src + e * 4 * HD), v = lds128(src + (e + 1) * 4 * HD);
        const uint32_t to = dst + e * 4 * 128;
        sts128(to + (x0 << 4), make_uint4(codes_lo(u.x), codes_hi(u.x), codes_lo(u.y), codes_hi(u.y)));
        sts128(to + ((x0 ^ 1) << 4), make_uint4(codes_lo(u.z), codes_hi(u.z), codes_lo(u.w), codes_hi(u.w)));
        sts128(to + 4 * 128 + ((x0 ^ 4) << 4), make_uint4(codes_lo(v.x), codes_hi(v.x), codes_lo(v.y), codes_hi(v.y)));
        sts128(to + 4 * 128 + ((x0 ^ 5) << 4), make_uint4(codes_lo(v.z), codes_hi(v.z), codes_lo(v.w), codes_hi(v.w)));
      }
      slot ^= 1;
      ph ^= slot == 0;
      --on_way;
      fence_async_smem();                     // the converted tile -> visible to the tensor core
      arrive(full + 8 * at.b, lane);          // (and the slot has been read)
      if (is_v) {
        at.move(2);
      } else {
        at.b ^= 1;
        at.ph ^= at.b == 2 * set;
      }
    }
    if (!ok) {                                // no copy may land after this CTA has left
      fail();
      for (int s = slot; on_way > 0; --on_way, s ^= 1, ph ^= s == 0) landed(got + 8 * s, ph);
    }
  } else {
    // ---------------- softmax: one row per thread ----------------
    if (CP > 1) asm volatile("setmaxnreg.inc.sync.aligned.u32 120;");
    else asm volatile("setmaxnreg.inc.sync.aligned.u32 144;");
    constexpr int SPAN = BMR / CP, TW = TT / CP, QT = TW / NQ;          // rows held, tokens of a thread, of them on a page
    const int rep = t.rep;
    auto by_rep = [&](int row) { return rep == 1 ? row : (int)__umulhi((uint32_t)row, t.rep_inv); };            // row / rep
    const int sg = warp >= 8, qw = warp & 3, r = qw * 32 + lane;
    const uint32_t lanes = tmem + ((uint32_t)(qw * 32) << 16), o_col = lanes + O_COL + sg * HD;
    const int w0 = r / SPAN * TW;                             // this copy's tokens of a tile
    const uint32_t s_col = lanes + S_COL + sg * TT, p_col = lanes + P_COL + sg * 32;
    uint32_t meet_ph = 0;
    auto all_meet = [&]() { arrive(meet, lane); meet_ph ^= 1; return soon(meet, meet_ph ^ 1); };

    // the piece's rows
    float m = ATTN_NOTHING, d = ATTN_NO_VALUE, l = 0.f, f = 0.f;
    int token = -1;                                           // its row of the packed arrays; -1: none
    int J = 0;                                                // tiles before
    uint32_t seen_ph = 1;
    auto queries = [&](const Chunk& w) {
      // Rows in fp16 under a power of two, 16 lanes per row, through shared memory to the row's two threads, 64 channels each
      constexpr int RW = SPAN / 8;
      const int r0 = (sg * 4 + qw) * RW;
      uint4 u[RW / 2];
      {
        int row = w.p.r0 + r0 + (lane >> 4);
        const int tok = by_rep(row);
        int h = row - tok * rep;
        const __nv_bfloat16* from = a.Q + (int64_t)(w.p.row0 + tok) * a.ldq + w.p.g * rep * HD + 8 * (lane & 15);
#pragma unroll
        for (int e = 0; e < RW / 2; ++e) {
          u[e] = row < w.p.R ? __ldg(reinterpret_cast<const uint4*>(from + h * HD)) : make_uint4(0, 0, 0, 0);
          row += 2;
          h += 2;
#pragma unroll
          for (int z = 0; z < 2; ++z)
            if (h >= rep) { h -= rep; from += a.ldq; }
        }
      }
      if (!all_meet()) return false;                          // the stage has been read
      const uint32_t rows = smem_u32(smem + STAGE);
      float* const factor = reinterpret_cast<float*>(smem + ROW);
#pragma unroll
      for (int e = 0; e < RW / 2; ++e) {
        const uint32_t y[4] = {u[e].x, u[e].y, u[e].z, u[e].w};
        uint32_t big = 0;
#pragma unroll
        for (int z = 0; z < 4; ++z) big = max(big, max(y[z] << 16 & 0x7fffffffu, y[z] & 0x7fff0000u));
#pragma unroll
        for (int o = 8; o > 0; o >>= 1) big = max(big, __shfl_xor_sync(0xffffffffu, big, o));
        const int sh = big == 0 ? 0 : min(13 + 127 - (int)(big >> 23), 126), i = r0 + 2 * e + (lane >> 4);
        const float up = __uint_as_float((uint32_t)(127 + sh) << 23);         // as attn_query4
        uint32_t z[4];
#pragma unroll
        for (int o = 0; o < 4; ++o) z[o] = pack_half2(__uint_as_float(y[o] << 16) * up, __uint_as_float(y[o] & 0xffff0000u) * up);
        sts128(rows + i * 256 + (((lane & 15) ^ (i & 15)) << 4), make_uint4(z[0], z[1], z[2], z[3]));
        if ((lane & 15) == 0) factor[i] = __uint_as_float((uint32_t)(127 - sh) << 23);
      }
      if (!all_meet()) return false;
      const int i = r & (SPAN - 1), row = w.p.r0 + i;
      token = row < w.p.R ? w.p.row0 + by_rep(row) : -1;
      f = factor[i];
      // (the scores of the piece before are all formed: both groups have met here)
      if (!soon(q_seen, seen_ph)) return false;
      seen_ph ^= 1;
      tc_fence_after();
#pragma unroll
      for (int c = 8 * sg; c < 8 * sg + 8; c += 2) {
        const uint4 x = lds128(rows + i * 256 + ((c ^ (i & 15)) << 4)), y = lds128(rows + i * 256 + (((c + 1) ^ (i & 15)) << 4));
        const uint32_t z[8] = {x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w};
        tmem_st8(lanes + Q_COL + c * 4, z);
      }
      asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
      tc_fence_before();
      arrive(q_ready, lane);
      return true;
    };

    // a tile's scores to weights
    auto tile = [&](const Chunk& w, const int i, const int before, const int seen_all, const int np, const Place at, const int n) {
      const Place prev = at.before();         // of the group's last tile (before the first: a phase that is over)
      // score factor and log2 of the value scale of each page; the tokens that this row sees, as bits
      const int o = i * TT + w0;
      float fk[NQ], lv[NQ];
      uint64_t seen = ~0ull;
      bool whole = o + TW <= seen_all;
      if (!whole) seen = attn_window(a.seen + (int64_t)max(token, 0) * a.words, token >= 0 ? a.words : 0, w.p.nq, o - seen_all);
#pragma unroll
      for (int q = 0; q < NQ; ++q) {
        const float4 pg = w.page[min((o + QT * q) >> pshift, np - 1)];
        fk[q] = pg.x * f;
        lv[q] = pg.y;
        if (__float_as_int(pg.z) < 0) {
          whole = false;
          seen &= ~(((1ull << (QT - 1) << 1) - 1) << (QT * q));
        }
      }
      if (!soon(s_full + 8 * (2 * sg + (n & 1)), (n >> 1) & 1)) return false;
      tc_fence_after();
      if (__any_sync(0xffffffffu, token >= 0)) {
        float x[TW];
        if (TW == 16) {
          tmem_ld16(s_col + w0, x);
        } else {
#pragma unroll
          for (int c = 0; c < TW; c += 32) tmem_ld32_async(s_col + w0 + c, x + c);
          asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
          for (int c = 0; c < TW; ++c) asm volatile("" : "+f"(x[c]));
        }
        tc_fence_before();
        arrive(s_free + 8 * sg, lane);
        if (!whole) {                         // what the row does not see
#pragma unroll
          for (int c = 0; c < TW; ++c)
            if (!((seen >> c) & 1)) x[c] = -INFINITY;
          // the unseen stay minus infinity under any positive factor.  A page without a token that the row sees gets
          // the factor 1 and no value scale, whatever it has; a factor of zero makes way for one that changes no score
#pragma unroll
          for (int q = 0; q < NQ; ++q) {
            if ((seen >> (QT * q) & ((1ull << (QT - 1) << 1) - 1)) == 0) { fk[q] = 1.f; lv[q] = -INFINITY; }
            else if (fk[q] == 0.f) fk[q] = 1e-30f;
          }
        }
        // the row's largest score (factors are not negative), and how far it passes m + d with the value scale
        float top = -INFINITY, far = -INFINITY, xm[NQ];
#pragma unroll
        for (int q = 0; q < NQ; ++q) {
          float mx[4];
#pragma unroll
          for (int c = 0; c < 4; ++c) mx[c] = x[QT * q + c];
#pragma unroll
          for (int c = 4; c + 8 <= QT; c += 8)
#pragma unroll
            for (int e = 0; e < 4; ++e) mx[e] = max3(mx[e], x[QT * q + c + e], x[QT * q + c + 4 + e]);
          static_assert(QT % 8 == 0, "");
#pragma unroll
          for (int e = 0; e < 4; ++e) mx[e] = fmaxf(mx[e], x[QT * q + QT - 4 + e]);
          const float mq = fmaxf(max3(mx[0], mx[1], mx[2]), mx[3]);
          xm[q] = mq == -INFINITY ? -INFINITY : mq * fk[q];
          top = fmaxf(top, xm[q]);
          far = fmaxf(far, (xm[q] - m) + (lv[q] - d));
        }
        // the weights and the accumulator of the group's last tile are done with
        if (!soon(pv_done + 8 * prev.b, prev.ph)) return false;
        tc_fence_after();
        if (__any_sync(0xffffffffu, top - m > ATTN_SLACK || far > ATTN_SLACK)) {
          const float mn = fmaxf(m, top), drop = m - mn;
          float dn = fmaxf(d + drop, ATTN_NO_VALUE);
#pragma unroll
          for (int q = 0; q < NQ; ++q) dn = fmaxf(dn, (xm[q] - mn) + lv[q]);
          const float grow = ex2((d - dn) + drop);
          l *= ex2(drop);
          m = mn;
          d = dn;
          if (before + i > 1) {               // O of the group's tiles before
#pragma unroll 1
            for (int c = 0; c < HD; c += 16) {
              float v[16];
              tmem_ld16(o_col + c, v);
#pragma unroll
              for (int e = 0; e < 16; ++e) v[e] *= grow;
              tmem_st8(o_col + c, reinterpret_cast<const uint32_t(&)[8]>(v[0]));
              tmem_st8(o_col + c + 8, reinterpret_cast<const uint32_t(&)[8]>(v[8]));
            }
          }
        }
        // A weight is p = 2^(x fk - m) times c = 2^e for its page's value scale, l the sum of p.  Where e and m are moderate c goes
        // into the exponent, and the sum is divided by it: one product less per pair.  e - m and the exponents that count, those
        // near e, round to 2^-19 below 64; beyond (large scores, pages whose values vanish beside the others') p and c stay apart.
        float e[NQ];
#pragma unroll
        for (int q = 0; q < NQ; ++q) e[q] = lv[q] - d + ATTN_SHIFT;
        float lo = e[0], hi = e[0];           // (a NaN stays)
#pragma unroll
        for (int q = 1; q < NQ; ++q) { lo = min_nan(lo, e[q]); hi = max_nan(hi, e[q]); }
        const bool apart = !(lo > fmaxf(m, 0.f) - 64.f && hi < fminf(m, 0.f) + 64.f);
        auto weights = [&](auto kind) {
          constexpr bool together = decltype(kind)::value;
#pragma unroll
          for (int q = 0; q < NQ; ++q) {
            const float cq = together ? 0.f : attn_factor(e[q]), s = together ? e[q] - m : -m;
            const float2 f2 = make_float2(fk[q], fk[q]), s2 = make_float2(s, s);
            constexpr int BW = QT < 16 ? QT : 16;
            float2 ls[4];
#pragma unroll
            for (int h = 0; h < 4; ++h) ls[h] = make_float2(0.f, 0.f);
#pragma unroll
            for (int o = 0; o < QT; o += BW) {
              float2 y[BW / 2];
#pragma unroll
              for (int h = 0; h < BW / 2; ++h) y[h] = omq_fma2(make_float2(x[QT * q + o + 2 * h], x[QT * q + o + 2 * h + 1]), f2, s2);
#pragma unroll
              for (int h = 0; h < BW / 2; ++h) y[h] = make_float2(ex2(y[h].x), ex2(y[h].y));
#pragma unroll
              for (int h = 0; h < BW / 2; ++h) ls[h & 3] = omq_add2(ls[h & 3], y[h]);
              if (!together) {
#pragma unroll
                for (int h = 0; h < BW / 2; ++h) { y[h].x *= cq; y[h].y *= cq; }
              }
              uint32_t pw[8];
#pragma unroll
              for (int h = 0; h < BW / 2; ++h) pw[h] = pack_half2(y[h].x, y[h].y);
              tmem_st8(p_col + (w0 + QT * q + o) / 2, pw);
            }
            ls[0] = omq_add2(omq_add2(ls[0], ls[1]), omq_add2(ls[2], ls[3]));
            l = together ? fmaf(ls[0].x + ls[0].y, ex2(-e[q]), l) : l + (ls[0].x + ls[0].y);
          }
        };
        if (!__any_sync(0xffffffffu, apart)) {
          weights(std::true_type());
        } else {
          // x fk - m is one operation, whose exact product differs from the rounded one in m by up to 2^-25 |m|: scores of such
          // size are rounded first
          if (fabsf(m) > 1048576.f) {
#pragma unroll
            for (int q = 0; q < NQ; ++q) {
#pragma unroll
              for (int h = 0; h < QT; ++h) x[QT * q + h] *= fk[q];
              fk[q] = 1.f;
            }
          }
          weights(std::false_type());
        }
        asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
      } else {
        arrive(s_free + 8 * sg, lane);
        if (!soon(pv_done + 8 * prev.b, prev.ph)) return false;
      }
      tc_fence_before();
      arrive(pv_ready + 8 * at.b, lane);
      return true;
    };

    if (CP > 1) {                             // the other copies' tokens weigh nothing here
      const uint32_t zero[8] = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
      for (int c = 0; c < 32; c += 8) tmem_st8(p_col + c, zero);
      asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
    }
    uint32_t o_ph = 1;
    Place at{sg, 0};                          // of the group's next tile
    int n = 0;                                // the group's tiles so far
    bool ok = chunk_wait(0);
    if (ok && !(chunk_at(0).flags & DONE)) ok = queries(chunk_at(0));
    for (int k = 0; ok; ++k) {
      const Chunk& w = chunk_at(k);
      if (w.flags & DONE) break;
      const int first = (w.p.t1 - w.p.t0 + TT - 1) / TT;      // tiles of the piece
      const int piece0 = (w.t0 - w.p.t0) / TT;                // its tiles before this chunk
      const int J0 = J - piece0, tiles = tiles_of(w), seen_all = w.p.len - w.p.nq - w.t0, np = (w.t1 - w.t0 + P - 1) >> pshift;
      if (w.flags & FIRST) {
        m = ATTN_NOTHING; d = ATTN_NO_VALUE; l = 0.f;
        ok = soon(o_free, o_ph);              // the piece before has read its accumulators
        o_ph ^= 1;
      }
      for (int i = (J ^ sg) & 1; i < tiles && ok; i += 2) {
        ok = tile(w, i, piece0, seen_all, np, at, n++);
        at.move(2);
      }
      J += tiles;
      if (!ok) break;
      if (!(w.flags & LAST)) { arrive(chunk_empty + 8 * (k % RING), lane); ok = chunk_wait(k + 1); continue; }
      // what the piece's end needs of this piece's rows
      const bool mine_now = token >= 0;
      const int row = w.p.r0 + (r & (SPAN - 1));
      // the next piece's queries, once this one's scores are all formed
      ok = chunk_wait(k + 1);
      if (ok && !(chunk_at(k + 1).flags & DONE)) ok = queries(chunk_at(k + 1));
      if (!ok) break;

      // ---- the piece's end: O over the sum of weights, to the outputs or the partial results ----
      const int n_a = (first + ((J0 & 1) == 0)) >> 1, n_b = first - n_a;  // tiles of the two groups
      if (sg == 0 ? n_a > 0 : n_b > 0) {
        const Place prev = at.before();
        ok = soon(pv_done + 8 * prev.b, prev.ph);
        if (!ok) break;
      }
      tc_fence_after();
      float* const refs = reinterpret_cast<float*>(smem + REF);
      refs[(sg * 3 + 0) * BMR + r] = m;
      refs[(sg * 3 + 1) * BMR + r] = d;
      refs[(sg * 3 + 2) * BMR + r] = l;
      tc_fence_before();
      ok = all_meet();                                        // both groups' references, and their products are done
      if (!ok) break;
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
      const bool none = L == 0.f;                             // a NaN score is not an empty row
      const float c = none ? 0.f : ex2(dd - ATTN_SHIFT) / L;
      const float c0 = none ? 0.f : c * ex2((refs[r] - mm) + refs[BMR + r] - dd);
      const float c1 = none ? 0.f : c * ex2((refs[3 * BMR + r] - mm) + refs[4 * BMR + r] - dd);
      const float lse = none ? -INFINITY : mm + log2f(L);
      if (mine_now && sg == 0 && r < SPAN) {
        if (w.p.part >= 0) t.pl[(int64_t)w.p.part * t.cost.rows + r] = attn_part(mm, L);
        else if (a.lse) a.lse[(int64_t)(w.p.row0 + by_rep(row)) * a.n_heads + w.p.g * rep + row - by_rep(row) * rep] = lse;
      }
      // 64 channels of each group, 32 at a time: each thread its row's, or, with copies of a row to add up, through shared
      // memory to rows of 128 bytes
      constexpr int RO = SPAN / 4;                            // rows that a warp writes
      const int q0 = CP == 1 ? r : qw * RO + (lane >> 3), rows = min(min(SPAN, w.p.R - w.p.r0), (qw + 1) * RO);
      const uint32_t stage = smem_u32(smem + STAGE) + sg * (BMR * 128);
      const int tok0 = by_rep(w.p.r0 + q0), h0 = w.p.r0 + q0 - tok0 * rep;
      auto put = [&](const float4& o, int64_t to) {
        if (a.Of) *reinterpret_cast<float4*>(a.Of + to) = o;
        if (a.Ob) {
          uint2 y;
          __nv_bfloat162* b2 = reinterpret_cast<__nv_bfloat162*>(&y);
          b2[0] = __floats2bfloat162_rn(o.x, o.y);
          b2[1] = __floats2bfloat162_rn(o.z, o.w);
          *reinterpret_cast<uint2*>(a.Ob + to) = y;
        }
      };
#pragma unroll 1
      for (int ch = sg * 64; ch < sg * 64 + 64; ch += 32) {
        if (CP > 1 && (ch & 32)) ok = all_meet();             // the stage has been read
#pragma unroll
        for (int b = 0; b < 32; b += 16) {
          float v[16], u[16];
          const uint32_t o = lanes + O_COL + ch + b;
          if (n_a > 0) tmem_ld16(o, v);
          if (n_b > 0) tmem_ld16(o + HD, u);
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const float y = n_a > 0 && c0 != 0.f ? v[i] * c0 : 0.f;
            v[i] = n_b > 0 && c1 != 0.f ? fmaf(u[i], c1, y) : y;
          }
          if (CP > 1) {
#pragma unroll
            for (int i = 0; i < 16; i += 4)
              sts128(stage + r * 128 + ((((b + i) >> 2) ^ (r & 7)) << 4),
                     make_uint4(__float_as_uint(v[i]), __float_as_uint(v[i + 1]), __float_as_uint(v[i + 2]), __float_as_uint(v[i + 3])));
          } else if (mine_now) {
            if (w.p.part >= 0) {
              float* const to = t.po + ((int64_t)w.p.part * BMR + r) * HD + ch + b;
#pragma unroll
              for (int i = 0; i < 16; i += 4) *reinterpret_cast<float4*>(to + i) = make_float4(v[i], v[i + 1], v[i + 2], v[i + 3]);
            } else {
              const int64_t to = (int64_t)(w.p.row0 + tok0) * a.ldo + (w.p.g * rep + h0) * HD + ch + b;
              if (a.Of) {
#pragma unroll
                for (int i = 0; i < 16; i += 4) *reinterpret_cast<float4*>(a.Of + to + i) = make_float4(v[i], v[i + 1], v[i + 2], v[i + 3]);
              }
              if (a.Ob) {
#pragma unroll
                for (int i = 0; i < 16; i += 8) {
                  uint4 y;
                  __nv_bfloat162* b2 = reinterpret_cast<__nv_bfloat162*>(&y);
#pragma unroll
                  for (int e = 0; e < 4; ++e) b2[e] = __floats2bfloat162_rn(v[i + 2 * e], v[i + 2 * e + 1]);
                  *reinterpret_cast<uint4*>(a.Ob + to + i) = y;
                }
              }
            }
          }
        }
        if (ch & 32) {                                        // the accumulators have been read
          tc_fence_before();
          arrive(o_free, lane);
        }
        if (CP == 1) continue;
        ok = ok && all_meet();
        if (!ok) break;
        int h = h0;
        int64_t to = (int64_t)(w.p.row0 + tok0) * a.ldo + w.p.g * rep * HD + ch + 4 * (lane & 7);
        const int step_t = by_rep(4), step_h = 4 - step_t * rep;
#pragma unroll
        for (int n = 0; n < RO / 4; ++n) {                    // a row per eight lanes
          const int q = q0 + 4 * n;
          if (q < rows) {
            float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int c = 0; c < CP; ++c) {
              const int i = c * SPAN + q;
              const uint4 y = lds128(stage + i * 128 + (((lane & 7) ^ (i & 7)) << 4));
              o.x += __uint_as_float(y.x); o.y += __uint_as_float(y.y); o.z += __uint_as_float(y.z); o.w += __uint_as_float(y.w);
            }
            if (w.p.part >= 0) *reinterpret_cast<float4*>(t.po + ((int64_t)w.p.part * BMR + q) * HD + ch + 4 * (lane & 7)) = o;
            else put(o, to + h * HD);
          }
          to += step_t * a.ldo;
          h += step_h;
          if (h >= rep) { h -= rep; to += a.ldo; }
        }
      }
      if (!ok) break;
      arrive(chunk_empty + 8 * (k % RING), lane);
    }
    if (!ok) fail();
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem, 512);
  }
}

template <int CP, int NQ, bool TEST>
omq_status launch(cudaStream_t st, const TreeArgs& t, int n_ctas) {
  auto kern = kv_attention_tree_tc_kernel<CP, NQ, TEST>;
  static std::atomic<uint64_t> allowed{0};
  OMQ_TRY(omq_allow_smem(allowed, kern, SMEM));
  kern<<<n_ctas, THREADS, SMEM, st>>>(t);
  OMQ_LAUNCH_CHECK();
  return OMQ_OK;
}

// By the most rows that a KV head has in the call.
template <bool TEST>
omq_status launch_form(cudaStream_t st, const TreeArgs& t, int n_ctas) {
  const int64_t rows = (int64_t)t.a.max_q * (t.a.n_heads / t.a.c.n_kv);
  const int page = t.a.c.page;
  if (rows <= BMR / 4) return launch<4, 1, TEST>(st, t, n_ctas);
  if (rows <= BMR / 2) return page >= 32 ? launch<2, 1, TEST>(st, t, n_ctas) : launch<2, 2, TEST>(st, t, n_ctas);
  return page >= TT ? launch<1, 1, TEST>(st, t, n_ctas) : launch<1, 4, TEST>(st, t, n_ctas);
}

}  // namespace

omq_status tree_tc_launch(cudaStream_t st, const TreeArgs& t, int n_ctas) {
  return t.tries != TREE_ORDINARY ? launch_form<true>(st, t, n_ctas) : launch_form<false>(st, t, n_ctas);
}
