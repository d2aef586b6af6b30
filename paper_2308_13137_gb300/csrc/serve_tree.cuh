// How the attention of draft trees is shared out (omq_kv_attention_tree).
//
// A unit of work is (sequence, KV head, a tile of its query rows); it goes over all of the sequence's tokens, whose number
// only the device knows.  Sequences differ in length by orders of magnitude, so a grid of units leaves most SMs
// waiting for the longest ones.  Here the units lie one after another on a line, each as long as it costs (its
// start, then one per 128 tokens), and CTA c of n takes the c-th n-th of the line, cutting units where they lie
// across a border.  A unit that one CTA has whole is written straight away; of a cut one each CTA leaves a partial result,
// and the joining launch adds them in order of tokens.
#pragma once
#include "serve_attn.cuh"

constexpr int TREE_SLOT = 128;              // tokens: whole pages and whole tiles of both forms
// limit of a wait of the tcgen05 form, in tries of 3.8 us (wait_tries); one that came back at once would still leave it 10 ms
constexpr uint32_t tree_tries(uint64_t limit_ns) { return (uint32_t)(limit_ns / 4000u); }
constexpr uint32_t TREE_TRIES = tree_tries(OMQ_WAIT_LIMIT_NS), TREE_ORDINARY = ~0u;

// query rows of a unit, at most, and what its start costs, in 128-token slots
struct TreeCost { int rows, start; };

// In the workspace, for the joining launch: the cut unit whose first tokens a CTA has.  It lies in `parts` partial results:
// `first`, then the first ones of the CTAs behind.  parts 0: none
struct TreeCut { int row0, g, r0, R, first, parts; };

struct TreeArgs {
  AttnArgs a;
  TreeCost cost;
  int64_t min_share;                        // of the line, per CTA
  int rep; uint32_t rep_inv;                // query heads per KV head, and 2^32 over it rounded up: row / rep for rows below 2^20
  TreeCut* cut;                             // [n]
  float* po; float2* pl;                    // partial results: [2 n][rows][128] and their log-sum-exp (attn_part)
  uint32_t tries;                           // self-test of the tcgen05 form: limit of a wait (else TREE_ORDINARY),
  int withhold;                             // and the chunk of each share that never comes (-1: none)
};

struct TreeSeq {
  int row0, nq, len, R, tiles, slots;       // R: query rows of a KV head, in `tiles` units
  bool ok;
  int64_t unit, head;                       // cost of a unit, of all units of a head
};

__device__ __forceinline__ TreeSeq tree_seq(const TreeArgs& t, int b) {
  const SeqRows s = seq_rows(t.a.c, t.a.cu_q, t.a.max_q, t.a.total_q, b);
  TreeSeq q;
  q.ok = s.ok && s.len <= t.a.max_kv && s.len <= 0x7ff00000;      // (rounded up without overflow)
  q.row0 = s.row0; q.nq = s.nq;
  q.len = q.ok ? s.len : 0;                                    // its rows read as empty
  q.R = s.nq * t.rep;
  q.tiles = (q.R + t.cost.rows - 1) / t.cost.rows;
  q.slots = (q.len + TREE_SLOT - 1) / TREE_SLOT;
  q.unit = t.cost.start + (int64_t)q.slots;
  q.head = q.tiles * q.unit;
  return q;
}

// slots of the unit at `at` on the line that lie before x
__device__ __forceinline__ int tree_slots(const TreeArgs& t, const TreeSeq& q, int64_t at, int64_t x) {
  const int64_t k = x - at - t.cost.start;
  return k <= 0 ? 0 : (k >= q.slots ? q.slots : (int)k);
}
__device__ __forceinline__ int64_t tree_border(int64_t total, int64_t n, int64_t c) { return total * c / n; }

// Share of this CTA on the line: [lo, hi), and the sequence that lo lies in.  Block-wide, THREADS of it; `scratch` holds
// THREADS / 32 + 4 numbers.
struct TreeShare { int64_t lo, hi, before, total, n; int b; };
template <int THREADS>
__device__ __forceinline__ TreeShare tree_share(const TreeArgs& t, int64_t* scratch) {
  constexpr int NW = THREADS / 32;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  int64_t total = 0;
  auto scan = [&](int base, int64_t* mine) {                  // inclusive, within THREADS sequences
    const int b = base + threadIdx.x;
    int64_t v = 0;
    if (b < t.a.c.B) {
      const TreeSeq q = tree_seq(t, b);
      if (!q.ok && blockIdx.x == 0) omq_set_status(t.a.status, OMQ_ERR_INVALID_ARG);
      v = q.head * t.a.c.n_kv;
    }
    *mine = v;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int64_t u = __shfl_up_sync(0xffffffffu, v, d);
      if (lane >= d) v += u;
    }
    __syncthreads();
    if (lane == 31) scratch[warp] = v;
    __syncthreads();
    int64_t all = 0;
    for (int k = 0; k < NW; ++k) {
      if (k < warp) v += scratch[k];
      all += scratch[k];
    }
    total += all;
    return v + total - all;
  };
  int64_t mine, end = 0;
  const bool once = t.a.c.B <= THREADS;
  for (int base = 0; base < t.a.c.B; base += THREADS) end = scan(base, &mine);
  const int64_t sum = total;
  const int64_t n = max((int64_t)1, min((int64_t)gridDim.x, sum / t.min_share));
  if (threadIdx.x == 0) t.cut[blockIdx.x].parts = 0;
  TreeShare r{0, 0, 0, sum, n, 0};
  if (blockIdx.x >= n || sum == 0) return r;
  r.lo = tree_border(sum, n, blockIdx.x);
  r.hi = tree_border(sum, n, blockIdx.x + 1);
  total = 0;
  for (int base = 0; base < t.a.c.B; base += THREADS) {
    if (!once) end = scan(base, &mine);
    if (mine > 0 && end - mine <= r.lo && r.lo < end) {
      scratch[NW] = base + threadIdx.x;
      scratch[NW + 1] = end - mine;
    }
  }
  __syncthreads();
  r.b = (int)scratch[NW];
  r.before = scratch[NW + 1];
  return r;
}

// The pieces of a CTA's share in order.  Uniform: every thread that calls it gets the same.
struct TreePiece {
  int b, row0, nq, len, R, g, r0;           // sequence and its rows; KV head, first query row of the unit
  int t0, t1;                               // tokens
  int part;                                 // place of the partial result; -1: the unit is whole
};
struct TreeWalk {
  TreeShare s;
  TreeSeq q;
  int g, tile;
  int64_t at;                               // of the unit on the line

  __device__ __forceinline__ void start(const TreeArgs& t, const TreeShare& share) {
    s = share;
    if (s.hi <= s.lo) return;
    q = tree_seq(t, s.b);
    const int64_t k = s.lo - s.before;
    g = (int)(k / q.head);
    tile = (int)((k - g * q.head) / q.unit);
    at = s.before + g * q.head + tile * q.unit;
  }
  __device__ __forceinline__ bool next(const TreeArgs& t, TreePiece* p) {
    while (at < s.hi && s.hi > s.lo) {
      const int a = tree_slots(t, q, at, s.lo), z = tree_slots(t, q, at, s.hi);
      const bool take = z > a || (q.slots == 0 && at >= s.lo);
      *p = TreePiece{s.b, q.row0, q.nq, q.len, q.R, g, tile * t.cost.rows, a * TREE_SLOT, min(q.len, z * TREE_SLOT),
                     a == 0 && z == q.slots ? -1 : (int)(2 * blockIdx.x + (at >= s.lo))};
      if (take && p->part >= 0 && a == 0) {                   // the CTA that has the end: as many borders lie before it
        const int last = (int)(((at + q.unit) * s.n - 1) / s.total);
        t.cut[blockIdx.x] = TreeCut{q.row0, g, tile * t.cost.rows, q.R, p->part, last - (int)blockIdx.x + 1};
      }
      at += q.unit;
      if (++tile == q.tiles) {
        tile = 0;
        if (++g == t.a.c.n_kv) {
          g = 0;
          do {
            if (++s.b >= t.a.c.B) { at = s.hi; break; }
            q = tree_seq(t, s.b);
          } while (q.tiles == 0);
        }
      }
      if (take) return true;
    }
    return false;
  }
};

omq_status tree_tc_launch(cudaStream_t st, const TreeArgs& t, int n_ctas);
