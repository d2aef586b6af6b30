// Drafted tokens: what the nodes of a draft tree see (omq_draft_tree), the walk that accepts or rejects them against
// the target's probabilities (omq_verify_drafts), and the accepted path's place in the caches (omq_kv_keep).
#include "serve_cache.cuh"
#include "tc.cuh"

namespace {

// ------------------------------------------------------------------------------------------------
// omq_draft_tree: one CTA per sequence, a thread per node, bits in shared memory.  Depths by pointer doubling: after round k
// a node has a jump over its 2^k nearest ancestors, so the chain of dependent steps is log2(depth) long.  The bits of
// trees up to WALK deep are set by walking up, one word for each ancestor; those of deeper ones by doubling too: a
// node takes over the bits of the node that it jumps to.  (A node whose bits grow in the same round passes on more than its 2^k
// ancestors: they are ancestors of the reader too.)  Bound: the launch and the round trips to the parents and back: 4.1 us
// for one tree, of which the launch is nearly all, 8.2 us for 384 of 509 nodes (by doubling throughout 10.2).
// ------------------------------------------------------------------------------------------------
constexpr int WALK = 24;
constexpr int MAX_NODES = 1024;

struct NodeArgs {
  int total_q, max_q; const int32_t* cu_q; const int32_t* parent; int32_t* depth; uint32_t* seen; int words;
  int32_t* status;
};

// rows of sequence b, checked
__device__ __forceinline__ bool node_rows(const int32_t* cu_q, int max_q, int total_q, int b, int* row0, int* n) {
  if (!cu_q) { *row0 = b * max_q; *n = max_q; return true; }
  const int lo = __ldg(cu_q + b), hi = __ldg(cu_q + b + 1);
  *row0 = lo; *n = hi - lo;
  return lo >= 0 && hi >= lo && hi <= total_q && hi - lo <= max_q;
}

__global__ void __launch_bounds__(MAX_NODES) draft_tree_kernel(const NodeArgs a) {
  extern __shared__ uint32_t tree_smem[];
  int row0, n;
  if (!node_rows(a.cu_q, a.max_q, a.total_q, blockIdx.x, &row0, &n)) {
    if (threadIdx.x == 0) omq_set_status(a.status, OMQ_ERR_INVALID_ARG);
    return;
  }
  const int i = threadIdx.x, W = (a.max_q + 31) >> 5, ld = W | 1;      // an odd row length: no bank conflicts
  uint32_t* bits = tree_smem;                                            // [max_q][ld]
  int2* hop = reinterpret_cast<int2*>(bits + ((a.max_q * ld + 1) & ~1));    // [2][max_q]: jump, ancestors up to it
  for (int k = i; k < (n * ld + 1) / 2; k += blockDim.x) reinterpret_cast<uint2*>(bits)[k] = make_uint2(0, 0);
  int up = -1;
  if (i < n) {
    up = __ldg(a.parent + row0 + i);
    if (up < -1 || up >= i) { omq_set_status(a.status, OMQ_ERR_INVALID_ARG); up = -1; }
    hop[i] = make_int2(up, up >= 0);
  }
  __syncthreads();
  int2 h = make_int2(up, up >= 0);
  int k = 0;
  for (;; k ^= 1) {
    const int2* const now = hop + k * a.max_q;
    int2* const next = hop + (k ^ 1) * a.max_q;
    bool more = false;
    if (i < n) {
      if (h.x >= 0) {
        const int2 j = now[h.x];
        h = make_int2(j.x, h.y + j.y);
        more = j.x >= 0;
      }
      next[i] = h;
    }
    if (!__syncthreads_or(more)) break;
  }
  if (i < n) a.depth[row0 + i] = h.y;
  uint32_t* const mine = bits + i * ld;
  if (i < n) mine[i >> 5] = 1u << (i & 31);
  // every thread has its last round's jumps behind it: the first array takes the parents again
  if (i < n) hop[i].x = up;
  if (!__syncthreads_or(i < n && h.y > WALK)) {
    if (i < n)
      for (int j = up; j >= 0; j = hop[j].x) mine[j >> 5] |= 1u << (j & 31);
  } else {
    int j = up;
    for (k = 0;; k ^= 1) {
      const int2* const now = hop + k * a.max_q;
      int2* const next = hop + (k ^ 1) * a.max_q;
      if (i < n) {
        if (j >= 0) {
          for (int w = 0; w <= j >> 5; ++w) mine[w] |= bits[j * ld + w];
          j = now[j].x;
        }
        next[i].x = j;
      }
      if (!__syncthreads_or(i < n && j >= 0)) break;
    }
  }
  __syncthreads();
  // rows of `words` words, consecutive threads on consecutive words
  const int step_r = blockDim.x / a.words, step_w = blockDim.x - step_r * a.words;
  for (int r = i / a.words, w = i - r * a.words; r < n;) {
    a.seen[((int64_t)row0 + r) * a.words + w] = w < W ? bits[r * ld + w] : 0u;
    r += step_r;
    w += step_w;
    if (w >= a.words) { w -= a.words; ++r; }
  }
}

size_t tree_smem_bytes(int max_q) {
  const int ld = ((max_q + 31) >> 5) | 1;
  return (size_t)((max_q * ld + 1) & ~1) * 4 + (size_t)max_q * 2 * sizeof(int2);
}


// ------------------------------------------------------------------------------------------------
// omq_verify_drafts.  At a node r with the children c_1, c_2, .. the weights are R = p_r and T = 1; child c (token x) is
// accepted when u_c T q(x) < R(x).  After a rejection the residual max(r - q, 0) of the normalised weights
// r = R / T takes their place: max(R / T - q, 0) = max(R - T q, 0) / T, and as R is itself max(p - a q, 0),
// that is max(p - (a + T) q, 0).  So one number a per node holds all its rejections, and a pass over the row
// gives the next T = sum max(p - a q, 0).
//
// The outcome is whole numbers, and a comparison next to its border must not depend on the order of a sum: terms
// are taken in 64-bit fixed point (2^-60, truncated), sums are exact, and the scalar tests are in double.  The new token is
// the first index whose running sum passes floor(u S): the 64-bit formula's, unless u S lies within V 2^-60 of a
// running sum.  Sums of 8 and more, which only rows that are far from adding up to one can have, are marked and reported, not held.
//
// A cluster of CTAs per sequence.  CTA 0 walks: every node's p(x) and q(x) are fetched at the start, all at once, so a
// walk that accepts first children touches shared memory only.  For a pass it posts (row, a) to all CTAs, each sums
// its slice of the vocabulary (the second pass over a row finds it in L1), and the parts meet in CTA 0.  Every CTA
// does what CTA 0 posts and decides nothing itself, so no input can make them disagree at a barrier.
//
// Bound: the passes of the longest walk, one after the other, each a read of the row (from the caches after the first), 30
// integer instructions per token, and two cluster barriers: 2 us and 2.5 for 32000 tokens, 6 and 2.5 for 128256.  64
// sequences of up to 15 rows, 128256 tokens, 35 to 46 us (bf16 41 to 54), one of 26 rows, 32000 tokens, 10 to 25 us, by the length of
// the longest walk; with chosen drafts (one pass per sequence at most) 20 and 10 to 12 us.  All clusters of 64 sequences are
// resident (four CTAs per SM, hence the registers); CTAs of 512 threads, in two waves, 61 us.
// ------------------------------------------------------------------------------------------------
constexpr int VT = 256, VW = VT / 32;       // threads, warps
constexpr int BATCH = 2;                    // 128-token steps whose loads a warp has in flight
constexpr int VMAX_CLUSTER = 8;
constexpr int VMAX_V = 1 << 20;

struct VerifyArgs {
  int total_q, max_q; const int32_t* cu_q; const int32_t* parent; const int32_t* tokens;
  int V, slice; const void* P; const void* Q; int64_t ldp, ldq; const float* u;
  int steps; int32_t* out_tokens; int32_t* out_path; int32_t* out_count;
  bool wide;                                // rows start on 16-byte (bf16: 8-byte) boundaries
  int32_t* status;
};

__device__ __forceinline__ float probability(float p) { return fminf(fmaxf(p, 0.f), 1.f); }    // NaN: 0

__device__ __forceinline__ float number(float u) { return fminf(fmaxf(u, 0.f), 0.99999994f); }  // in [0, 1)

// a q times 2^60, truncated, for q in [0, 1] and a = a52 2^-52 below 8: the product of significand and a52, less 15 bits, is
// that for an exponent of 127 and has 64 bits; back by 127 less the exponent.  (a52's last 15 bits are zero after a node's first
// rejection, a = 1)
__device__ __forceinline__ uint64_t times60(float q, uint64_t a52) {
  const uint32_t b = __float_as_uint(q), m = (b & 0x7fffffu) | 0x800000u, rest = (uint32_t)a52 & 0x7fffu;
  const uint64_t a37 = a52 >> 15;
  uint64_t w = (uint64_t)m * (uint32_t)a37 + ((uint64_t)(m * (uint32_t)(a37 >> 32)) << 32);
  if (rest) w += (uint64_t)m * rest >> 15;
  asm("shr.u64 %0, %0, %1;" : "+l"(w) : "r"(127u - (b >> 23)));            // (64 and more: zero)
  return w;
}
// p times 2^60, truncated
__device__ __forceinline__ uint64_t fixed60(float p) {
  uint64_t w = (uint64_t)((__float_as_uint(p) & 0x7fffffu) | 0x800000u) << 37;
  asm("shr.u64 %0, %0, %1;" : "+l"(w) : "r"(127u - (__float_as_uint(p) >> 23)));
  return w;
}

// the same for a = a52 2^-52 of any size: 88 bits of product and a shift; all ones when it passes 2^63
__device__ __forceinline__ uint64_t scaled60(float q, uint64_t a52) {
  const uint32_t b = __float_as_uint(q), e = b >> 23;
  const uint32_t m = e ? (b & 0x7fffffu) | 0x800000u : 0u;
  const uint64_t lo = (uint64_t)m * (uint32_t)a52, hi = (uint64_t)m * (uint32_t)(a52 >> 32) + (lo >> 32);   // hi : low half of lo
  const int s = 142 - (int)e;               // right shift, 15 or more: of both words below 32, else of hi alone (64 and more: zero)
  uint64_t far = hi, near = hi;
  asm("shr.u64 %0, %0, %1;" : "+l"(far) : "r"((uint32_t)max(s - 32, 0)));
  asm("shl.b64 %0, %0, %1;" : "+l"(near) : "r"((uint32_t)max(32 - s, 0)));
  near |= (uint32_t)lo >> (s & 31);
  if (hi >> min(31 + s, 63)) near = ~0ull;
  return s >= 32 ? far : near;
}

__device__ __forceinline__ float prob_at(const void* base, bool bf, int64_t at) {
  return probability(bf ? __bfloat162float(__ldg(static_cast<const __nv_bfloat16*>(base) + at)) : __ldg(static_cast<const float*>(base) + at));
}

// values i .. i + 3 of a row (zero from n on)
template <bool BF>
__device__ __forceinline__ float4 prob4(const void* row, int i, int n, bool wide) {
  float4 f = make_float4(0.f, 0.f, 0.f, 0.f);
  if (wide && i + 4 <= n) {
    if (BF) {
      const uint2 w = __ldg(reinterpret_cast<const uint2*>(static_cast<const __nv_bfloat16*>(row) + i));
      f = make_float4(__uint_as_float(w.x << 16), __uint_as_float(w.x & 0xffff0000u), __uint_as_float(w.y << 16),
                      __uint_as_float(w.y & 0xffff0000u));
    } else {
      f = __ldg(reinterpret_cast<const float4*>(static_cast<const float*>(row) + i));
    }
  } else {
    float* v = reinterpret_cast<float*>(&f);
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (i + k < n)
        v[k] = BF ? __bfloat162float(__ldg(static_cast<const __nv_bfloat16*>(row) + i + k)) : __ldg(static_cast<const float*>(row) + i + k);
  }
  return f;
}

// what CTA 0 posts: the row of p and q, a, and how many tokens the sequence has with the new one
struct Order { int32_t row, kind, count, pad; uint64_t a52; };
// PASS: sum the residual.  DRAW: the new token, from the last pass's residual; DRAW_PASS: from a residual that is to be
// summed first; DRAW_WHOLE: from p as it is
enum { PASS = 0, DRAW = 1, DRAW_PASS = 2, DRAW_WHOLE = 3 };

struct __align__(16) VerifySmem {
  Order order;
  uint64_t part[VMAX_CLUSTER];              // the CTAs' sums, in every CTA
  uint64_t warp_sum[VW], step_sum[VW];
  int32_t parent[MAX_NODES], token[MAX_NODES];
  float u[MAX_NODES], p[MAX_NODES], q[MAX_NODES];
  uint32_t gone[VMAX_V / VMAX_CLUSTER / 32];          // tokens of the slice that were rejected (no draft distribution)
};

// p and q of N x 128 tokens of a warp, four of each to a lane: all on their way before the first is used
template <bool BF, int N>
__device__ __forceinline__ void fetch(const VerifyArgs& a, int64_t row, bool both, int at, int hi, float4 (&p)[N], float4 (&q)[N]) {
  const char* const pr = static_cast<const char*>(a.P) + row * a.ldp * (BF ? 2 : 4);
#pragma unroll
  for (int k = 0; k < N; ++k) p[k] = prob4<BF>(pr, at + 128 * k, hi, a.wide);
  if (both) {
    const char* const qr = static_cast<const char*>(a.Q) + row * a.ldq * (BF ? 2 : 4);
#pragma unroll
    for (int k = 0; k < N; ++k) q[k] = prob4<BF>(qr, at + 128 * k, hi, a.wide);
  }
}

// the weights of four tokens of the slice
__device__ __forceinline__ void weights4(const VerifySmem& s, const float4& p, const float4& q, uint64_t a52, bool cut, int i, int lo,
                                         int hi, uint64_t (&w)[4]) {
  w[0] = fixed60(probability(p.x)); w[1] = fixed60(probability(p.y)); w[2] = fixed60(probability(p.z)); w[3] = fixed60(probability(p.w));
  if (a52) {
    const float f[4] = {probability(q.x), probability(q.y), probability(q.z), probability(q.w)};
    if (a52 < 8ull << 52) {                 // (more only after eight rejections)
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const uint64_t d = times60(f[k], a52);
        w[k] = w[k] > d ? w[k] - d : 0ull;
      }
    } else {
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const uint64_t d = scaled60(f[k], a52);
        w[k] = w[k] > d ? w[k] - d : 0ull;
      }
    }
  }
  if (cut && i < hi) {
    const uint32_t g = s.gone[(i - lo) >> 5] >> ((i - lo) & 31);
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if ((g >> k) & 1) w[k] = 0;
  }
}

// A sum of weights that comes to 8 (2^63) or more keeps its top bit from there on, whatever is added: 2^63 - 1 and a term of up
// to 2^63 do not pass 64 bits, and a sum with the bit is not looked at further.
constexpr uint64_t HEAVY = 1ull << 63;
__device__ __forceinline__ uint64_t add_held(uint64_t a, uint64_t b) { return (a + b) | ((a | b) & HEAVY); }

// of a warp, in digits of 24 bits and the 16 above them: three reductions (five steps of marked sums of
// shuffled values cost 64 x 128256 up to 1.5 us)
__device__ __forceinline__ uint64_t warp_sum64(uint64_t v) {
  const uint64_t low = ((uint64_t)__reduce_add_sync(0xffffffffu, (uint32_t)(v >> 24) & 0xffffffu) << 24) +
                       __reduce_add_sync(0xffffffffu, (uint32_t)v & 0xffffffu);
  const uint32_t top = __reduce_add_sync(0xffffffffu, (uint32_t)(v >> 48)) + (uint32_t)(low >> 48);
  return (low & 0xffffffffffffull) | (uint64_t)top << 48 | (top >> 15 ? HEAVY : 0ull);
}

// to this CTA's shared variable and its like in the other CTAs of the cluster
__device__ __forceinline__ void put64(uint64_t* at, int rank, int C, uint64_t v) {
  if (C == 1) *at = v;
  else asm volatile("st.shared::cluster.b64 [%0], %1;" ::"r"(tc::mapa_shared(tc::smem_u32(at), rank)), "l"(v) : "memory");
}

template <bool BF>
__global__ void __launch_bounds__(VT, 4) verify_kernel(const VerifyArgs a, const int C) {
  __shared__ VerifySmem s;
  const int b = blockIdx.x / C, rank = blockIdx.x - b * C, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int lo = min(a.V, rank * a.slice), hi = min(a.V, lo + a.slice);
  const int share = (a.slice + VW * 128 - 1) / (VW * 128) * 128;             // tokens of a warp, in order
  const int w_lo = min(hi, lo + warp * share), w_hi = min(hi, w_lo + share);
  int32_t* const tokens = a.out_tokens + (int64_t)b * a.steps;
  int row0, n;
  if (!node_rows(a.cu_q, a.max_q, a.total_q, b, &row0, &n)) {
    if (rank == 0 && threadIdx.x == 0) omq_set_status(a.status, OMQ_ERR_INVALID_ARG);
    row0 = n = 0;
  }
  auto sync = [&]() {
    __syncwarp();
    if (C > 1) tc::cluster_sync();
    else __syncthreads();
  };

  // ---- CTA 0: the nodes, with p and q of their tokens at their parents ----
  int32_t* const path = a.out_path + (int64_t)b * a.steps;
  if (rank == 0) {
    for (int i = threadIdx.x; i < n; i += VT) {
      int p = __ldg(a.parent + row0 + i);
      const int x = __ldg(a.tokens + row0 + i);
      if (i == 0 ? p != -1 : (p < -1 || p >= i || x < 0 || x >= a.V)) {
        omq_set_status(a.status, OMQ_ERR_INVALID_ARG);
        p = -1;                             // nobody's child
      }
      const bool child = i > 0 && p >= 0;
      s.parent[i] = p;
      s.token[i] = x;
      s.u[i] = number(__ldg(a.u + row0 + i));
      s.p[i] = child ? prob_at(a.P, BF, (int64_t)(row0 + p) * a.ldp + x) : 0.f;
      s.q[i] = child && a.Q ? prob_at(a.Q, BF, (int64_t)(row0 + p) * a.ldq + x) : 1.f;
    }
    for (int j = threadIdx.x; j < a.steps; j += VT) { tokens[j] = -1; path[j] = j == 0 && n > 0 ? 0 : -1; }
  }
  sync();                                   // the nodes are there; every CTA runs, so its shared memory can be written

  // ---- the walk: one warp, since its tests are in double, of which an SM has few units ----
  int cur = 0, count = 1, i = 0;            // node, tokens with the new one, last child tested
  double A = 0.0, T = 1.0;
  bool fresh = false;                       // the last pass's sums are those of (cur, A)
  Order o;
  while (true) {
    if (rank == 0 && warp == 0) {
      o = Order{n > 0 ? row0 + cur : -1, DRAW_WHOLE, 0, 0, 0ull};
      while (n > 0 && count < a.steps && T >= 0.0) {         // (below zero: a row without a sum, see below)
        uint32_t m = 0;
        int base = (i + 1) & ~31;
        for (; base < n && !m; base += 32) {
          const int k = base + lane;
          m = __ballot_sync(0xffffffffu, k > i && k < n && s.parent[min(k, MAX_NODES - 1)] == cur);
        }
        o.kind = fresh ? DRAW : DRAW_PASS;
        if (!m) break;                      // no child, or all rejected
        i = base - 32 + __ffs(m) - 1;
        const int x = s.token[i];
        const double p = (double)s.p[i], q = (double)s.q[i];
        double R = p;
        if (a.Q) {
          R = fmax(__dsub_rn(p, __dmul_rn(A, q)), 0.0);
        } else {                            // a token that a sibling before it had weighs nothing any more
          bool again = false;
          for (int k = cur + 1 + lane; k < i; k += 32) again |= s.parent[k] == cur && s.token[k] == x;
          if (__any_sync(0xffffffffu, again)) R = 0.0;
        }
        if (__dmul_rn(__dmul_rn((double)s.u[i], T), q) < R) {
          if (threadIdx.x == 0) { tokens[count - 1] = x; path[count] = i; }
          cur = i; ++count; A = 0.0; T = 1.0; fresh = false;
          o.kind = DRAW_WHOLE;
        } else if (a.Q) {
          A = __dadd_rn(A, T);
          o.kind = PASS;
          break;
        } else {
          T = __dsub_rn(T, R);
        }
      }
      if (n > 0) o.row = row0 + cur;
      o.count = count;
      o.a52 = A < 4095.0 ? (uint64_t)(A * 4503599627370496.0) : 0xfff0000000000000ull;
      if (threadIdx.x < C) {
        put64(reinterpret_cast<uint64_t*>(&s.order), threadIdx.x, C, (uint64_t)(uint32_t)o.row | (uint64_t)(uint32_t)o.kind << 32);
        put64(reinterpret_cast<uint64_t*>(&s.order) + 1, threadIdx.x, C, (uint64_t)(uint32_t)o.count);
        put64(&s.order.a52, threadIdx.x, C, o.a52);
      }
    }
    sync();
    o = s.order;
    if (o.row < 0) break;
    bool cut = o.kind == DRAW_PASS && !a.Q;
    if (cut) {                              // the node's children were all rejected: their tokens weigh nothing
      for (int k = threadIdx.x; k < (a.slice + 31) / 32; k += VT) s.gone[k] = 0;
      __syncthreads();
      for (int k = threadIdx.x + 1; k < n; k += VT) {
        const int x = __ldg(a.tokens + row0 + k);
        if (k > o.row - row0 && __ldg(a.parent + row0 + k) == o.row - row0 && x >= lo && x < hi)
          atomicOr(&s.gone[(x - lo) >> 5], 1u << ((x - lo) & 31));
      }
      __syncthreads();
    }
    uint64_t total, before;
    while (true) {
      if (o.kind != DRAW) {
        uint64_t sum = 0;
        uint32_t high = 0;                  // of all sums so far: a batch adds 2^63 at most
        static_assert(BATCH <= 2, "");
        for (int at = w_lo + 4 * lane; at < w_hi; at += 128 * BATCH) {
          float4 p[BATCH], q[BATCH];
          fetch<BF, BATCH>(a, o.row, o.a52 != 0, at, w_hi, p, q);
#pragma unroll
          for (int k = 0; k < BATCH; ++k) {
            uint64_t w[4];
            weights4(s, p[k], q[k], o.a52, cut, at + 128 * k, lo, w_hi, w);
            sum += (w[0] + w[1]) + (w[2] + w[3]);
          }
          high |= (uint32_t)(sum >> 32);
        }
        sum = warp_sum64(sum | ((uint64_t)high << 32 & HEAVY));
        if (lane == 0) s.warp_sum[warp] = sum;
        __syncthreads();
        if (threadIdx.x < C) {
          uint64_t mine = 0;
#pragma unroll
          for (int k = 0; k < VW; ++k) mine = add_held(mine, s.warp_sum[k]);
          put64(&s.part[rank], threadIdx.x, C, mine);
        }
        sync();
      }
      total = before = 0;
      for (int k = 0; k < C; ++k) {
        if (k < rank) before += s.part[k];
        total = add_held(total, s.part[k]);
      }
      if (total != 0 || o.kind == PASS || o.kind == DRAW_WHOLE) break;
      // nothing is left of the weights (rows that do not sum to one): the new token comes from p as it is
      o.kind = DRAW_WHOLE;
      o.a52 = 0;
      cut = false;
      sync();                               // every CTA has read the parts
    }
    const bool heavy = total & HEAVY;       // the weights add up to 8 or more: no distribution, and no sum to draw from
    if (o.kind == PASS) {
      if (rank == 0 && warp == 0) {
        T = heavy ? -1.0 : (double)total * (1.0 / 1152921504606846976.0);
        if (heavy) A = 0.0;                 // p itself is posted next, and adds up to no less
      }
      fresh = true;
      continue;
    }
    // ---- the new token: the first one whose running sum passes floor(u total) ----
    if (rank == 0 && threadIdx.x == 0) {
      a.out_count[b] = o.count;
      if (total == 0 || heavy) { omq_set_status(a.status, OMQ_ERR_INVALID_ARG); tokens[o.count - 1] = 0; }
    }
    if (heavy) return;
    const uint64_t t = __umul64hi((uint64_t)((double)number(__ldg(a.u + row0)) * 18446744073709551616.0), total);
    // the warp share that t falls into, if this CTA has it
    uint64_t run = before;
    int own = -1;
#pragma unroll
    for (int k = 0; k < VW; ++k) {
      if (own < 0 && t >= run && t - run < s.warp_sum[k]) own = k;
      if (own < 0) run += s.warp_sum[k];
    }
    if (own < 0) return;
    // a part of that share for each warp
    const int part = share / VW;            // (a multiple of 4)
    const int p_lo = min(hi, lo + own * share + warp * part), p_hi = min(hi, p_lo + part);
    uint64_t sum = 0;
    for (int at = p_lo + 4 * lane; at < p_hi; at += 128 * 2) {
      float4 p[2], q[2];
      fetch<BF, 2>(a, o.row, o.a52 != 0, at, p_hi, p, q);
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        uint64_t w[4];
        weights4(s, p[k], q[k], o.a52, cut, at + 128 * k, lo, p_hi, w);
        sum += (w[0] + w[1]) + (w[2] + w[3]);
      }
    }
    sum = warp_sum64(sum);
    if (lane == 0) s.step_sum[warp] = sum;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < VW; ++k)
      if (k < warp) run += s.step_sum[k];
    if (t >= run && t - run < sum) {
      for (int base = p_lo; base < p_hi; base += 128) {
        float4 p[1], q[1];
        uint64_t w[4];
        fetch<BF, 1>(a, o.row, o.a52 != 0, base + 4 * lane, p_hi, p, q);
        weights4(s, p[0], q[0], o.a52, cut, base + 4 * lane, lo, p_hi, w);
        uint64_t in = (w[0] + w[1]) + (w[2] + w[3]);
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
          const uint64_t v = __shfl_up_sync(0xffffffffu, in, d);
          if (lane >= d) in += v;
        }
        const uint32_t past = __ballot_sync(0xffffffffu, t < run + in);
        if (past) {
          if (lane == __ffs(past) - 1) {
            uint64_t c = run + in;
            int x = 3;                      // back from the lane's last token while the sum before it passes t too
            for (; x > 0; --x) {
              c -= w[x];
              if (c <= t) break;
            }
            tokens[o.count - 1] = base + 4 * lane + x;
          }
          break;
        }
        run += __shfl_sync(0xffffffffu, in, 31);
      }
    }
    return;
  }
  if (rank == 0 && threadIdx.x == 0) a.out_count[b] = 0;      // a sequence without rows
}

// 16 codes under a scale that is 1 / r of theirs
__device__ __forceinline__ uint4 again16(uint4 u, float r) {
  uint32_t* w = reinterpret_cast<uint32_t*>(&u);
  if (r == 1.f) {                           // all whole numbers already: only the clamp of code 0
#pragma unroll
    for (int k = 0; k < 4; ++k) w[k] = __vmaxu4(w[k], 0x01010101u);
    return u;
  }
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    uint32_t o = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float c = (float)((int)((w[k] >> (8 * e)) & 255u) - 128);
      const float v = fminf(fmaxf(rintf(__fmul_rn(c, r)), -127.f), 127.f);
      o |= (uint32_t)((int)v + 128) << (8 * e);
    }
    w[k] = o;
  }
  return u;
}

// ------------------------------------------------------------------------------------------------
// omq_kv_keep.  Place j of a sequence's drafted tokens takes the codes of node path[j], which lies at j or behind it, so in
// order of j no place is written before what it held has been read.  A page's scale grows where a token comes in from a
// page of larger values, and the codes of the page are rounded again then, as in the append; tokens that move within
// the page are rounded like those that stay.  A warp per (sequence, KV head, layer), four tokens' K and V at a time, eight lanes
// each; the CTA's eight warps share the path.  Bound: the chain of path, page, scale and codes; few registers and no barrier
// between warps keep 32 of them on an SM: 64 sequences of 8 heads in 40 layers, 34 to 55 tokens of which move, 13.4 us, one of 32
// heads in 32 layers (none or one moves) 4.1 to 8.  (A CTA of four warps for each head and each of K and V, with the moved tokens in
// registers, 51.2 us; a warp for each 17.8, bound by the instructions around the moves.)  Where seven tokens of every sequence come
// from other pages to both sides of a page's end: 34.8 and 10.2 us; where both pages grow, 203 and 59 us, since one warp rounds a
// page's K and V (745 MB and 71 MB in all: 112 and 11 us).
// ------------------------------------------------------------------------------------------------
constexpr int KT = 256, KW = KT / 32;       // threads, warps
constexpr int KEEP_LAYERS = 128;            // caches of a launch

struct KeepCache {
  uint8_t *k, *v; float *k_scale, *v_scale; const int32_t *page_table, *kv_len; int32_t* status;
  int32_t n_pages, max_pages;
};
template <int L>
struct KeepArgs {
  int total_q, max_q; const int32_t* cu_q; const int32_t* path; int steps; const int32_t* count;
  int n_kv, page;
  KeepCache c[L];
};

template <int L>
__global__ void __launch_bounds__(KT) kv_keep_kernel(const __grid_constant__ KeepArgs<L> a) {
  __shared__ int32_t path[MAX_NODES];
  const KeepCache& c = a.c[blockIdx.z];
  const int b = blockIdx.y, lane = threadIdx.x & 31, g = blockIdx.x * KW + (threadIdx.x >> 5);
  const int P = a.page, shift = 31 - __clz(P);
  const int32_t* const my_path = a.path + (int64_t)b * a.steps;
  const int ahead = (int)threadIdx.x < a.steps ? __ldg(my_path + threadIdx.x) : 0;     // asked for beside the lengths
  int row0, nq;
  const bool rows = node_rows(a.cu_q, a.max_q, a.total_q, b, &row0, &nq);
  const int len = __ldg(c.kv_len + b), n = __ldg(a.count + b), start = len - nq;
  bool bad = !rows || n < 0 || n > a.steps || n > nq || (n > 0 && start < 0);
  if (!bad) {
    for (int j = threadIdx.x; j < n; j += KT) path[j] = j < KT ? ahead : __ldg(my_path + j);
  }
  __syncthreads();
  if (!bad)
    for (int j = threadIdx.x; j < n; j += KT) bad |= path[j] >= nq || path[j] < 0 || (j > 0 && path[j - 1] >= path[j]);
  if (__syncthreads_or(bad)) {
    if (threadIdx.x == 0) omq_set_status(c.status, OMQ_ERR_INVALID_ARG);
    return;
  }
  if (g >= a.n_kv) return;
  uint8_t* const codes[2] = {c.k, c.v};
  float* const scales[2] = {c.k_scale, c.v_scale};
  auto page_id = [&](int pg) {
    const int id = pg < c.max_pages ? __ldg(c.page_table + (int64_t)b * c.max_pages + pg) : -1;
    if (id >= 0 && id < c.n_pages) return id;
    omq_set_status(c.status, OMQ_ERR_INVALID_ARG);
    return -1;
  };
  const int sub = lane >> 3, at16 = 16 * (lane & 7);          // token of four, its bytes
  int j0 = 0;
  while (j0 < n && path[j0] == j0) ++j0;    // these lie where they belong
  while (j0 < n) {
    const int pg = (start + j0) >> shift, j1 = min(n, ((pg + 1) << shift) - start);
    // four tokens' codes of K and V; whether they come from another page, and under which scales; nothing for one that stays, or
    // whose page is out of range
    auto get = [&](int j, uint4 (&u)[2], float (&from)[2], bool* other) {
      if (j >= j1 || path[j] == j) return false;
      const int at = start + path[j], src = page_id(at >> shift);
      if (src < 0) return false;
      const int64_t head = (int64_t)src * a.n_kv + g, place = (head * P + (at & (P - 1))) * 128 + at16;
      *other = at >> shift != pg;
#pragma unroll
      for (int v = 0; v < 2; ++v) {
        u[v] = *reinterpret_cast<const uint4*>(codes[v] + place);
        from[v] = scales[v][head];
      }
      return true;
    };
    const int id = page_id(pg);
    if (id < 0) { j0 = j1; continue; }
    const int64_t head = (int64_t)id * a.n_kv + g, dst = head * P * 128 + at16;
    const float before[2] = {scales[0][head], scales[1][head]};
    uint32_t big[2] = {0, 0};
    uint4 u0[2];
    float from0[2];
    bool other0 = false, got0 = false;
    for (int jb = j0; jb < j1; jb += 4) {
      uint4 u[2];
      float from[2];
      bool other;
      const bool got = get(jb + sub, u, from, &other);
      if (got && other) {
#pragma unroll
        for (int v = 0; v < 2; ++v) {       // largest |code - 128|, four bytes at a time
          uint32_t four = __vmaxu4(__vmaxu4(__vabsdiffu4(u[v].x, 0x80808080u), __vabsdiffu4(u[v].y, 0x80808080u)),
                                   __vmaxu4(__vabsdiffu4(u[v].z, 0x80808080u), __vabsdiffu4(u[v].w, 0x80808080u)));
          four = __vmaxu4(four, four >> 16);
          const uint32_t top = max(four & 255u, four >> 8 & 255u);
          big[v] = max(big[v], __float_as_uint(__fmul_rn((float)top, from[v])) & 0x7fffffffu);
        }
      }
      if (jb == j0) {
        other0 = other; got0 = got;
#pragma unroll
        for (int v = 0; v < 2; ++v) { u0[v] = u[v]; from0[v] = from[v]; }
      }
    }
    float after[2];
    bool any = false;
#pragma unroll
    for (int v = 0; v < 2; ++v) {
      const float want = __fdiv_rn(__uint_as_float(__reduce_max_sync(0xffffffffu, big[v])), 127.f);
      const bool grows = !(before[v] >= want) && before[v] == before[v];
      after[v] = grows ? want : before[v];
      if (grows) {
        const float r = __fdiv_rn(before[v], after[v]);
        for (int k = sub; k < P; k += 4) {
          uint4* at = reinterpret_cast<uint4*>(codes[v] + dst + k * 128);
          *at = again16(*at, r);
        }
        if (lane == 0) scales[v][head] = after[v];
        any = true;
      }
    }
    if (any) __syncwarp();
    for (int jb = j0; jb < j1; jb += 4) {
      uint4 u[2] = {u0[0], u0[1]};
      float from[2] = {from0[0], from0[1]};
      bool other = other0, got = got0;
      // (what moves within a page that grew has been rounded by now, but for the first four, read before)
      if (jb > j0) got = get(jb + sub, u, from, &other);
      if (got) {
#pragma unroll
        for (int v = 0; v < 2; ++v)
          u[v] = again16(u[v], after[v] > 0.f ? __fdiv_rn(other || jb == j0 ? from[v] : after[v], after[v]) : 0.f);
      }
      __syncwarp();
      if (got) {
#pragma unroll
        for (int v = 0; v < 2; ++v)
          *reinterpret_cast<uint4*>(codes[v] + dst + (start + jb + sub - (pg << shift)) * 128) = u[v];
      }
      __syncwarp();
    }
    j0 = j1;
  }
}

template <int L>
omq_status keep_launch(cudaStream_t st, const omq_kv_cache* const* caches, int32_t* const* status, int n, int total_q, int max_q,
                       const int32_t* cu_q, const int32_t* path, int steps, const int32_t* count) {
  KeepArgs<L> a;
  a.total_q = total_q; a.max_q = max_q; a.cu_q = cu_q; a.path = path; a.steps = steps; a.count = count;
  a.n_kv = caches[0]->n_kv; a.page = caches[0]->page;
  for (int i = 0; i < L; ++i) {
    const omq_kv_cache& c = *caches[i < n ? i : 0];
    a.c[i] = KeepCache{c.k, c.v, c.k_scale, c.v_scale, c.page_table, c.kv_len, status ? status[i < n ? i : 0] : nullptr, c.n_pages,
                       c.max_pages};
  }
  kv_keep_kernel<L><<<dim3((a.n_kv + KW - 1) / KW, caches[0]->B, n), KT, 0, st>>>(a);
  OMQ_LAUNCH_CHECK();
  return OMQ_OK;
}

}  // namespace

extern "C" {

omq_status omq_draft_tree(omq_stream_t stream, int32_t B, int32_t total_q, int32_t max_q, const int32_t* cu_q,
                          const int32_t* parent, int32_t* depth, uint32_t* seen, int32_t words, int32_t* dev_status) {
  OMQ_REQUIRE(parent && depth && seen, OMQ_ERR_INVALID_ARG);
  OMQ_REQUIRE(B > 0 && B <= 65535 && total_q > 0 && max_q > 0 && max_q <= total_q && max_q <= MAX_NODES, OMQ_ERR_SHAPE);
  OMQ_REQUIRE(cu_q || (int64_t)B * max_q == total_q, OMQ_ERR_SHAPE);
  OMQ_REQUIRE(words >= (max_q + 31) / 32 && words <= MAX_NODES, OMQ_ERR_SHAPE);
  OMQ_REQUIRE(omq_aligned4(cu_q) && omq_aligned4(parent) && omq_aligned4(depth) && omq_aligned4(seen), OMQ_ERR_ALIGN);
  static std::atomic<uint64_t> allowed{0};
  OMQ_TRY(omq_allow_smem(allowed, draft_tree_kernel, (int)tree_smem_bytes(MAX_NODES)));
  const NodeArgs a{total_q, max_q, cu_q, parent, depth, seen, words, dev_status};
  draft_tree_kernel<<<B, (max_q + 31) / 32 * 32, tree_smem_bytes(max_q), (cudaStream_t)stream>>>(a);
  OMQ_LAUNCH_CHECK();
  return OMQ_OK;
}

omq_status omq_verify_drafts(omq_stream_t stream, int32_t B, int32_t total_q, int32_t max_q, const int32_t* cu_q,
                             const int32_t* parent, const int32_t* tokens, int64_t V, const void* P, const void* Q,
                             int32_t dtype, int64_t ldp, int64_t ldq, const float* u, int32_t steps, int32_t* out_tokens,
                             int32_t* out_path, int32_t* out_count, int32_t* dev_status) {
  OMQ_REQUIRE(parent && tokens && P && u && out_tokens && out_path && out_count, OMQ_ERR_INVALID_ARG);
  OMQ_REQUIRE(dtype == OMQ_F32 || dtype == OMQ_BF16, OMQ_ERR_INVALID_ARG);
  OMQ_REQUIRE(B > 0 && B <= 65535 && total_q > 0 && max_q > 0 && max_q <= total_q && max_q <= MAX_NODES, OMQ_ERR_SHAPE);
  OMQ_REQUIRE(cu_q || (int64_t)B * max_q == total_q, OMQ_ERR_SHAPE);
  OMQ_REQUIRE(steps > 0 && steps <= MAX_NODES, OMQ_ERR_SHAPE);
  OMQ_REQUIRE(V > 0 && V <= VMAX_V && ldp >= V && (!Q || ldq >= V), OMQ_ERR_SHAPE);
  const int size = dtype == OMQ_BF16 ? 2 : 4;
  OMQ_REQUIRE(omq_aligned4(cu_q) && omq_aligned4(parent) && omq_aligned4(tokens) && omq_aligned4(u) && omq_aligned4(out_tokens) &&
                  omq_aligned4(out_path) && omq_aligned4(out_count) && (uintptr_t)P % size == 0 && (uintptr_t)Q % size == 0,
              OMQ_ERR_ALIGN);
  VerifyArgs a{total_q, max_q, cu_q, parent, tokens, (int)V, 0, P, Q, ldp, ldq, u, steps, out_tokens, out_path, out_count,
               false, dev_status};
  a.wide = (uintptr_t)P % (4 * size) == 0 && (uintptr_t)Q % (4 * size) == 0 && ldp % 4 == 0 && (!Q || ldq % 4 == 0);
  const int C = V > 4096 ? VMAX_CLUSTER : 1;
  a.slice = (int)((V + C * 128 - 1) / (C * 128) * 128);
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(B * C), 1, 1);
  cfg.blockDim = dim3(VT, 1, 1);
  cfg.stream = (cudaStream_t)stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = C; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = C > 1 ? 1 : 0;
  auto kern = dtype == OMQ_BF16 ? verify_kernel<true> : verify_kernel<false>;
  if (cudaLaunchKernelEx(&cfg, kern, a, C) != cudaSuccess) { cudaGetLastError(); return OMQ_ERR_CUDA; }
  OMQ_LAUNCH_CHECK();
  return OMQ_OK;
}

omq_status omq_kv_keep(omq_stream_t stream, const omq_kv_cache* const* caches, int32_t* const* dev_status, int32_t n_caches,
                       int32_t total_q, int32_t max_q, const int32_t* cu_q, const int32_t* path, int32_t steps,
                       const int32_t* count) {
  OMQ_REQUIRE(caches && n_caches > 0 && path && count, OMQ_ERR_INVALID_ARG);
  OMQ_REQUIRE(steps > 0 && steps <= MAX_NODES, OMQ_ERR_SHAPE);
  OMQ_REQUIRE(omq_aligned4(path) && omq_aligned4(count), OMQ_ERR_ALIGN);
  for (int32_t i = 0; i < n_caches; ++i) {
    OMQ_REQUIRE(caches[i], OMQ_ERR_INVALID_ARG);
    OMQ_TRY(kv_check(caches[i], total_q, max_q, cu_q, caches[i]->n_kv));
    OMQ_REQUIRE(caches[i]->n_kv == caches[0]->n_kv && caches[i]->page == caches[0]->page && caches[i]->B == caches[0]->B,
                OMQ_ERR_SHAPE);
    for (int32_t j = 0; j < i; ++j)         // a cache that is named twice would be moved twice at once
      OMQ_REQUIRE(caches[j]->k != caches[i]->k && caches[j]->v != caches[i]->v, OMQ_ERR_INVALID_ARG);
  }
  for (int32_t i = 0; i < n_caches; i += KEEP_LAYERS) {
    const int32_t n = n_caches - i < KEEP_LAYERS ? n_caches - i : KEEP_LAYERS;
    OMQ_TRY(n <= 4 ? keep_launch<4>((cudaStream_t)stream, caches + i, dev_status ? dev_status + i : nullptr, n, total_q, max_q, cu_q,
                                    path, steps, count)
                   : keep_launch<KEEP_LAYERS>((cudaStream_t)stream, caches + i, dev_status ? dev_status + i : nullptr, n, total_q,
                                              max_q, cu_q, path, steps, count));
  }
  return OMQ_OK;
}

}  // extern "C"
