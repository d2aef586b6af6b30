// Product of 8-bit codes with a step and zero point per token and output channel (omq_qgemm_i8).
//
// sum_k (a - za)(b - zb) is formed from the codes moved by 128 (a' = a - 128, b' = b - 128) as
//   sum a'b' - za' sum b' - zb' sum a' + K za' zb',   za' = za - 128, zb' = zb - 128,
// each sum an exact integer; the combination is taken in 64 bits and rounded once to fp32.
//
// sm_103a has no integer form of tcgen05.mma and a small integer rate elsewhere, so sum a'b' runs on
// the fp16 tensor path, exactly: |a'|, |b'| <= 128 are fp16 integers, a product is below 2^14, and fp32
// sums of up to 1024 of them stay at or below 2^24, where every integer is an fp32 number.  Every 1024
// steps of K the accumulator is added to 32-bit integers.
#include "common.cuh"
#include "tc.cuh"
#include <cuda_fp16.h>
#include <cstring>

namespace {

using namespace tc;

struct QgemmArgs {
  int M, N, K;
  const uint8_t* A; int64_t lda; const float* ah; const int32_t* az;
  const uint8_t* B; int64_t ldb; const float* bh; const int32_t* bz;
  const float* bias;
  float* Cf; __nv_bfloat16* Cb; int64_t ldc;
  int32_t* status;
  // K split over S work items per tile (S > 1): integer partial sums, joined by qgemm_join_kernel
  int splits, kb_per_split;
  int32_t* part;              // [S, M, N]
  int32_t* part_sb;           // [S, N]
  int m_fast;
  __half* wide;               // [M, K] activation codes as fp16 integers, written by qgemm_widen_kernel
  int32_t* sum_a;             // [M] their row sums
  uint32_t wait_ns;           // limit of a wait of the register form
  int withhold;               // self-test only: its first tile is never loaded, so the wait for it runs out
};

// two of the four codes of a word as fp16 integers code - 128: the byte under the exponent of 1024
// (0x6400 | c = 1024 + c), minus 1152
__device__ __forceinline__ uint32_t half_codes(uint32_t w, uint32_t sel) {
  const uint32_t u = __byte_perm(w, 0x64646464u, sel);
  const __half2 h = __hsub2(*reinterpret_cast<const __half2*>(&u), __half2half2(__ushort_as_half(0x6480)));
  return *reinterpret_cast<const uint32_t*>(&h);
}

// s + the sum of 16 codes
__device__ __forceinline__ int code_sum(const uint4& u, int s) {
  uint32_t v = (uint32_t)s;
  v = __dp4a(u.x, 0x01010101u, v);
  v = __dp4a(u.y, 0x01010101u, v);
  v = __dp4a(u.z, 0x01010101u, v);
  return (int)__dp4a(u.w, 0x01010101u, v);
}

// h_a h_b (integer sum) + bias, each step one fp32 rounding
__device__ __forceinline__ float finish(int acc, long long za, long long zb, int sa, int sb, int K, float ah, float bh,
                                        bool zeros) {
  float s;
  if (zeros) s = __ll2float_rn((long long)acc - za * sb - zb * ((long long)sa - (long long)K * za));
  else s = __int2float_rn(acc);
  return __fmul_rn(__fmul_rn(s, ah), bh);
}

// ================================================================================================
// many rows: CTA pairs on the tensor cores
// ================================================================================================
// The activation codes are widened to fp16 once per call (qgemm_widen_kernel: M K codes, an N-th of the
// conversions that the product's tiles would repeat); the weights stay 8-bit in HBM and are converted
// on their way to the MMA.  A pair of CTAs computes a 256 x 256 tile with one tcgen05.mma of cta_group::2 per
// 16 steps of K; each CTA holds 128 rows of A and 128 of B.  Roles of a CTA's 20 warps:
//   0       TMA: raw weight code tiles [128 x 128] into a ring (128-byte swizzle)
//   1       leader CTA: issues the MMAs
//   2       TMA: fp16 tiles of A into the operand ring (128-byte swizzle)
//   4..11   drain: warps w and w + 4 own the 32 accumulator rows of lane quadrant w % 4, half the columns
//           each; every 1024 steps of K they add the fp32 accumulator to integers in registers
//   12..19  convert: 128 codes of a weight row per thread to fp16 in the 128-byte swizzled layout the MMA
//           reads; warps 12..15 take the even stages and 16..19 the odd ones, so that one group's waits
//           and proxy fence overlap the other's work.  They also form the rows' code sums for the
//           zero points
// The tensor memory holds two accumulators, so the drain overlaps the MMAs of the next 1024 steps.
// What bounds it is the hand-offs between the roles, then the tensor rate: 2048 x 22016 x 4096 in 255 to 260 us,
// 1.43 PFLOP/s; its 688 tiles are nine rounds of the 76 pairs and four tiles, which take a tenth round.
constexpr int BM = 128, BN = 256, BK = 128;
// Ring depths: raw weight tiles (they come from HBM), operand stages (A | converted B).  Stages of 128
// codes: the signals between the roles, not the work, set the pace (2048 x 22016 x 4096: 356 us with 64 and 277
// with 128; 273 with one barrier for both operands of a stage).
constexpr int RAW = 4, OPS = 2;
constexpr int CHUNK_KB = 1024 / BK;               // k blocks per exact accumulation
constexpr int TC_THREADS = 640;
constexpr int RAW_BYTES = 128 * BK, OP_BYTES = 128 * BK * 2;      // a raw tile, an fp16 tile of A or B
constexpr int RAW_OFF = 2 * OPS * OP_BYTES;
constexpr int SUM_OFF = RAW_OFF + RAW * RAW_BYTES;      // code sums of B: 2 tiles x 2 groups x [256]
constexpr int COL_OFF = SUM_OFF + 4 * 256 * 4;                    // drain warps: [8][4][128] column operands
constexpr int BAR_OFF = COL_OFF + 8 * 4 * 128 * 4;
constexpr int TC_SMEM = BAR_OFF + 512 + 1024;
static_assert(TC_SMEM <= 227 * 1024, "shared memory per CTA");

struct Item { int m0, n0, kb0, nkb, split; };

__device__ __forceinline__ Item item_of(const QgemmArgs& p, int i, int mt, int nt) {
  const int tiles = mt * nt, t = i % tiles;
  Item it;
  it.split = i / tiles;
  const int mi = p.m_fast ? t % mt : t / nt, ni = p.m_fast ? t / mt : t % nt;
  it.m0 = mi * 2 * BM;
  it.n0 = ni * BN;
  const int all = (p.K + BK - 1) / BK;
  it.kb0 = it.split * p.kb_per_split;
  it.nkb = min(all, it.kb0 + p.kb_per_split) - it.kb0;
  return it;
}

__device__ __forceinline__ void sts_cluster(uint32_t addr, int v) {
  asm volatile("st.shared::cluster.b32 [%0], %1;" ::"r"(addr), "r"(v) : "memory");
}

// 32 bytes of one row, two rows of 16 where the output is only 16-byte aligned
__device__ __forceinline__ void store32(void* at, const uint32_t (&v)[8], bool wide) {
  if (wide) {
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(at), "r"(v[0]), "r"(v[1]), "r"(v[2]),
                 "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7])
                 : "memory");
  } else {
    reinterpret_cast<uint4*>(at)[0] = make_uint4(v[0], v[1], v[2], v[3]);
    reinterpret_cast<uint4*>(at)[1] = make_uint4(v[4], v[5], v[6], v[7]);
  }
}

// A drain thread's 128 integer sums (row m, columns n0 ..) to the outputs.  MODE 0: no zero points; 1: 32-bit
// combination; 2: 64-bit.  A thread writes whole 32-byte sectors where the alignment allows it.
template <int MODE>
__device__ __forceinline__ void tc_store(const QgemmArgs& p, const int (&acc)[BN / 2], int m, int n0, float ah, int za, int sa,
                                         const float* col_h, const int* col_z, const int* col_s, const float* col_b) {
  if (m >= p.M) return;
  const int64_t at = (int64_t)m * p.ldc + n0;
  const bool wide_f = ((uintptr_t)p.Cf & 31) == 0;                              // ldc is a multiple of 8
  const bool wide_b = ((uintptr_t)p.Cb & 31) == 0 && p.ldc % 16 == 0;
  const uint32_t ta = (uint32_t)sa - (uint32_t)p.K * (uint32_t)za;               // MODE 1: modulo 2^32
  const long long ta64 = (long long)sa - (long long)p.K * za;
#pragma unroll
  for (int j = 0; j < BN / 2; j += 16) {
    if (n0 + j >= p.N) break;
    float y[16];
#pragma unroll
    for (int e = 0; e < 16; e += 4) {
      const float4 h = *reinterpret_cast<const float4*>(col_h + j + e);
      const float hv[4] = {h.x, h.y, h.z, h.w};
      int4 z = make_int4(0, 0, 0, 0), s = z;
      if (MODE != 0) { z = *reinterpret_cast<const int4*>(col_z + j + e); s = *reinterpret_cast<const int4*>(col_s + j + e); }
      const int zv[4] = {z.x, z.y, z.z, z.w}, sv[4] = {s.x, s.y, s.z, s.w};
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        float f;
        if (MODE == 2) f = __ll2float_rn((long long)acc[j + e + k] - (long long)za * sv[k] - zv[k] * ta64);
        else if (MODE == 1) f = __int2float_rn((int)((uint32_t)acc[j + e + k] - (uint32_t)za * (uint32_t)sv[k] - (uint32_t)zv[k] * ta));
        else f = __int2float_rn(acc[j + e + k]);
        y[e + k] = __fmul_rn(__fmul_rn(f, ah), hv[k]);
      }
    }
    if (p.bias) {
#pragma unroll
      for (int e = 0; e < 16; e += 4) {
        const float4 b = *reinterpret_cast<const float4*>(col_b + j + e);
        y[e] = __fadd_rn(y[e], b.x); y[e + 1] = __fadd_rn(y[e + 1], b.y);
        y[e + 2] = __fadd_rn(y[e + 2], b.z); y[e + 3] = __fadd_rn(y[e + 3], b.w);
      }
    }
    const bool both = n0 + j + 8 < p.N;                      // N is a multiple of 8
    if (p.Cf) {
#pragma unroll
      for (int hlf = 0; hlf < 2; ++hlf) {
        uint32_t v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = __float_as_uint(y[8 * hlf + e]);
        if (hlf == 0 || both) store32(p.Cf + at + j + 8 * hlf, v, wide_f);
      }
    }
    if (p.Cb) {
      float lo[8], hi[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) { lo[e] = y[e]; hi[e] = y[8 + e]; }
      const uint4 a = pack_bf16x8(lo), b = pack_bf16x8(hi);
      const uint32_t v[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
      if (both) store32(p.Cb + at + j, v, wide_b);
      else *reinterpret_cast<uint4*>(p.Cb + at + j) = a;
    }
  }
}

__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(TC_THREADS, 1)
    qgemm_tc_kernel(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB, const QgemmArgs p) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint8_t* a_ring = smem;                                        // 1024-aligned (swizzle atom)
  uint8_t* conv_ring = smem + OPS * OP_BYTES;
  uint8_t* raw_ring = smem + RAW_OFF;
  int* sum_b = reinterpret_cast<int*>(smem + SUM_OFF);           // [tile parity][group][column of the pair's tile]
  uint64_t* raw_full = reinterpret_cast<uint64_t*>(smem + BAR_OFF);
  uint64_t* raw_empty = raw_full + RAW;
  uint64_t* ready = raw_empty + RAW;                             // leader's: both CTAs' A landed and B converted
  uint64_t* freed = ready + OPS;                                 // the stage's products are formed
  uint64_t* acc_full = freed + OPS;                              // [2]
  uint64_t* acc_empty = acc_full + 2;                            // [2], leader's
  uint64_t* sum_full = acc_empty + 2;                            // [2]
  uint64_t* sum_empty = sum_full + 2;                            // [2]
  uint64_t* drain = sum_empty + 2;
  uint32_t* tmem_holder = reinterpret_cast<uint32_t*>(drain + 1);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_holder + 1);

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rank = (int)cluster_ctarank();
  const bool leader = rank == 0;
  const int mt = (p.M + 2 * BM - 1) / (2 * BM), nt = (p.N + BN - 1) / BN;
  const int total = mt * nt * p.splits, first = blockIdx.x >> 1, step = gridDim.x >> 1;
  const bool zeros = p.az || p.bz;

  if (threadIdx.x == 0) {
    for (int s = 0; s < RAW; ++s) { mbar_init(&raw_full[s], 1); mbar_init(&raw_empty[s], 4); }
    // one barrier tells the issuing warp everything about a stage, and one commit frees it: each wait and
    // each commit costs that warp 150 cycles and more
    for (int s = 0; s < OPS; ++s) { mbar_init(&ready[s], 1 + 8); mbar_init(&freed[s], 1); }
    for (int b = 0; b < 2; ++b) {
      mbar_init(&acc_full[b], 1); mbar_init(&acc_empty[b], 16);
      mbar_init(&sum_full[b], 16); mbar_init(&sum_empty[b], 16);
    }
    mbar_init(drain, 1);
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) tmem_alloc_pair(tmem_holder, 512);
  tc_fence_before();
  __syncthreads();
  cluster_sync();                            // both CTAs' barriers initialised before any remote use
  tc_fence_after();
  const uint32_t tmem = *tmem_holder;
  auto fail = [&]() { omq_set_status(p.status, OMQ_ERR_TIMEOUT); *abort_flag = 1; };

  if (warp < 4) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 32;");
    // (each of the three: the whole warp runs the loop, one lane issues)
    if (warp == 0) {
      // ---------------- raw weight code tiles ----------------
      uint32_t it = 0;
      bool ok = true;
      for (int i = first; i < total && ok; i += step) {
        const Item w = item_of(p, i, mt, nt);
        for (int kb = 0; kb < w.nkb; ++kb, ++it) {
          const int s = it % RAW;
          ok = warp_wait(&raw_empty[s], ((it / RAW) & 1) ^ 1);
          if (!ok) { fail(); break; }
          if (elect_one()) {
            mbar_expect_tx(&raw_full[s], RAW_BYTES);
            tma_load_3d(&tmB, &raw_full[s], raw_ring + s * RAW_BYTES, (w.kb0 + kb) * BK, w.n0 + rank * 128, 0);
          }
          __syncwarp();
        }
      }
      if (__any_sync(0xffffffffu, *abort_flag)) {    // no copy may land after this CTA has left
        const uint32_t from = it > (uint32_t)RAW ? it - RAW : 0u;
        for (uint32_t j = from; j < it; ++j)
          if (!wait_phase(&raw_full[j % RAW], (j / RAW) & 1)) break;
      }
    } else if (warp == 2) {
      // ---------------- A tiles: both CTAs' loads complete on the leader's barrier ----------------
      uint32_t it = 0;
      bool ok = true;
      for (int i = first; i < total && ok; i += step) {
        const Item w = item_of(p, i, mt, nt);
        for (int kb = 0; kb < w.nkb; ++kb, ++it) {
          const int s = it % OPS;
          ok = warp_wait(&freed[s], ((it / OPS) & 1) ^ 1);
          if (!ok) { fail(); break; }
          if (elect_one()) {
            if (leader) mbar_expect_tx(&ready[s], 2 * OP_BYTES);
#pragma unroll
            for (int h = 0; h < 2; ++h)
              tma_load_3d_pair(&tmA, mapa_shared(smem_u32(&ready[s]), 0), a_ring + s * OP_BYTES + h * OP_BYTES / 2,
                               (w.kb0 + kb) * BK + 64 * h, w.m0 + rank * BM, 0);
          }
          __syncwarp();
        }
      }
      if (__any_sync(0xffffffffu, *abort_flag) && leader) {   // (the peer leaves with the leader)
        const uint32_t from = it > (uint32_t)OPS ? it - OPS : 0u;
        for (uint32_t j = from; j < it; ++j)
          if (!wait_phase(&ready[j % OPS], (j / OPS) & 1)) break;
      }
    } else if (warp == 1 && leader) {
      // ---------------- MMA issuer: the whole warp runs the loop, one lane issues ----------------
      constexpr uint32_t idesc = idesc_f16(2 * BM, BN);
      const uint64_t da = sdesc(smem_u32(a_ring), 16, 1024), db = sdesc(smem_u32(conv_ring), 16, 1024);
      uint32_t it = 0, ch = 0;
      bool ok = true;
      for (int i = first; i < total && ok; i += step) {
        const Item w = item_of(p, i, mt, nt);
        for (int kb = 0; kb < w.nkb; ++kb, ++it) {
          const uint32_t buf = ch & 1, s = it % OPS;
          ok = (kb % CHUNK_KB != 0 || warp_wait(&acc_empty[buf], ((ch >> 1) & 1) ^ 1)) &&
               warp_wait(&ready[s], (it / OPS) & 1);
          if (!ok) { fail(); break; }
          tc_fence_after();
          const bool last = kb % CHUNK_KB == CHUNK_KB - 1 || kb == w.nkb - 1;
          if (elect_one()) {
            const uint64_t a0 = da + (uint64_t)(s * (OP_BYTES >> 4)), b0 = db + (uint64_t)(s * (OP_BYTES >> 4));
#pragma unroll
            for (int k = 0; k < BK / 16; ++k)
              umma_bf16_pair(tmem + buf * BN, a0 + (((k >> 2) * (OP_BYTES / 2) + (k & 3) * 32) >> 4),
                             b0 + (((k >> 2) * (OP_BYTES / 2) + (k & 3) * 32) >> 4), idesc, kb % CHUNK_KB != 0 || k != 0);
            umma_commit_pair(&freed[s], 0x3);
            if (last) umma_commit_pair(&acc_full[buf], 0x3);
          }
          __syncwarp();
          if (last) ++ch;
        }
      }
      if (__any_sync(0xffffffffu, *abort_flag)) {   // products in flight end before the tensor memory is released
        if (elect_one()) umma_commit_pair(drain, 0x1);
        wait_phase(drain, 0);
      }
    }
  } else if (warp < 12) {
    // ---------------- drain: fp32 accumulators -> integers -> outputs ----------------
    asm volatile("setmaxnreg.inc.sync.aligned.u32 160;");
    const int q = warp & 3, c0 = warp >= 8 ? BN / 2 : 0;
    // this warp's copy of its 128 columns' step, zero point - 128, code sum and bias
    float* col_h = reinterpret_cast<float*>(smem + COL_OFF) + (warp - 4) * 512;
    int* col_z = reinterpret_cast<int*>(col_h + 128);
    int* col_s = col_z + 128;
    float* col_b = reinterpret_cast<float*>(col_s + 128);
    uint32_t ch = 0, tile = 0;
    for (int i = first; i < total; i += step, ++tile) {
      const Item w = item_of(p, i, mt, nt);
      int acc[BN / 2];
#pragma unroll
      for (int j = 0; j < BN / 2; ++j) acc[j] = 0;
      bool ok = true;
      for (int kb = 0; kb < w.nkb; kb += CHUNK_KB, ++ch) {
        const uint32_t buf = ch & 1;
        ok = warp_wait(&acc_full[buf], (ch >> 1) & 1);
        if (!ok) { fail(); break; }
        tc_fence_after();
#pragma unroll
        for (int j = 0; j < BN / 2; j += 16) {
          float v[16];
          tmem_ld16(tmem + buf * BN + ((uint32_t)(q * 32) << 16) + c0 + j, v);
#pragma unroll
          for (int e = 0; e < 16; ++e) acc[j + e] += __float2int_rn(v[e]);
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive_cluster(mapa_shared(smem_u32(&acc_empty[buf]), 0));
      }
      if (!ok) break;
      const uint32_t sbuf = tile & 1;
      const int* sumB = sum_b + sbuf * 512;
      const int row_l = q * 32 + lane, m = w.m0 + rank * BM + row_l;
      int sa = 0;
      if (zeros) {
        ok = __all_sync(0xffffffffu, mbar_wait_cluster(&sum_full[sbuf], (tile >> 1) & 1));
        if (!ok) { fail(); break; }
        if (p.bz && m < p.M) sa = p.sum_a[m];
      }
      if (p.splits > 1) {
        if (m < p.M) {
          int32_t* out = p.part + ((int64_t)w.split * p.M + m) * p.N + w.n0 + c0;
#pragma unroll
          for (int j = 0; j < BN / 2; j += 4)
            if (w.n0 + c0 + j < p.N) *reinterpret_cast<int4*>(out + j) = make_int4(acc[j], acc[j + 1], acc[j + 2], acc[j + 3]);
        }
        if (zeros && w.m0 == 0 && rank == 0 && q == 0) {
#pragma unroll
          for (int j = 0; j < BN / 2; j += 32)
            if (w.n0 + c0 + j + lane < p.N) 
              p.part_sb[(int64_t)w.split * p.N + w.n0 + c0 + j + lane] = sumB[c0 + j + lane] + sumB[256 + c0 + j + lane];
        }
      } else {
        int zmax = 0;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const int c = 32 * k + lane, n = w.n0 + c0 + c;
          const bool in = n < p.N;
          col_h[c] = in ? __ldg(p.bh + n) : 0.f;
          col_b[c] = in && p.bias ? __ldg(p.bias + n) : 0.f;
          if (zeros) {
            const int z = in && p.bz ? __ldg(p.bz + n) - 128 : 0;
            zmax = max(zmax, abs(z));
            col_z[c] = z;
            col_s[c] = sumB[c0 + c] + sumB[256 + c0 + c];
          }
        }
        zmax = (int)__reduce_max_sync(0xffffffffu, (unsigned)zmax);
        __syncwarp();
        const float ah = m < p.M ? __ldg(p.ah + m) : 0.f;
        const int za = p.az && m < p.M ? __ldg(p.az + m) - 128 : 0;
        // |sum| <= K (128 + |za'|)(128 + |zb'|): where that is below 2^31, 32-bit arithmetic (modulo 2^32)
        // gives it, and the 64-bit form is left to rows or columns far from zero
        const bool narrow = (unsigned long long)p.K * (128u + abs(za)) * (128u + zmax) < (1ull << 31);
        if (!zeros) tc_store<0>(p, acc, m, w.n0 + c0, ah, za, sa, col_h, col_z, col_s, col_b);
        else if (__all_sync(0xffffffffu, narrow)) tc_store<1>(p, acc, m, w.n0 + c0, ah, za, sa, col_h, col_z, col_s, col_b);
        else tc_store<2>(p, acc, m, w.n0 + c0, ah, za, sa, col_h, col_z, col_s, col_b);
        __syncwarp();                        // the column operands are rewritten by the next tile
      }
      if (zeros) {
        __syncwarp();
        if (lane < 2) mbar_arrive_cluster(mapa_shared(smem_u32(&sum_empty[sbuf]), lane));
      }
    }
  } else {
    // ---------------- convert ----------------
    asm volatile("setmaxnreg.dec.sync.aligned.u32 64;");
    const int grp = (warp - 12) >> 2, r = threadIdx.x & 127;
    const uint32_t src0 = smem_u32(raw_ring) + r * BK, dst0 = smem_u32(conv_ring) + r * 128;
    const uint32_t cx = r & 7;
    uint32_t it = 0, tile = 0;
    bool ok = true;
    for (int i = first; i < total && ok; i += step, ++tile) {
      const Item w = item_of(p, i, mt, nt);
      int sb = 0, codes = 0;                 // sum of this group's codes and their number per row
      for (int kb = 0; kb < w.nkb; ++kb, ++it) {
        if ((int)(it & 1) != grp) continue;
        const int rs = it % RAW, cs = it % OPS;
        ok = warp_wait(&raw_full[rs], (it / RAW) & 1);
        if (!ok) { fail(); break; }
        uint4 u[8];
#pragma unroll
        for (int c = 0; c < 8; ++c) u[c] = lds128(src0 + rs * RAW_BYTES + ((c ^ cx) << 4));
        if (zeros) {
          codes += min(BK, p.K - (w.kb0 + kb) * BK);       // beyond K the tile holds zeros, which add nothing
#pragma unroll
          for (int c = 0; c < 8; ++c) sb = code_sum(u[c], sb);
        }
        ok = warp_wait(&freed[cs], ((it / OPS) & 1) ^ 1);
        if (!ok) { fail(); break; }
#pragma unroll
        for (int c = 0; c < 8; ++c) {        // (beyond K they are -128, and A is zero there)
          const uint32_t dst = dst0 + cs * OP_BYTES + (c >> 2) * (OP_BYTES / 2);
          sts128(dst + (((2 * (c & 3)) ^ cx) << 4), make_uint4(half_codes(u[c].x, 0x4140), half_codes(u[c].x, 0x4342),
                                                               half_codes(u[c].y, 0x4140), half_codes(u[c].y, 0x4342)));
          sts128(dst + (((2 * (c & 3) + 1) ^ cx) << 4), make_uint4(half_codes(u[c].z, 0x4140), half_codes(u[c].z, 0x4342),
                                                                   half_codes(u[c].w, 0x4140), half_codes(u[c].w, 0x4342)));
        }
        fence_async_smem();                  // the converted tile -> visible to this SM's tensor core
        __syncwarp();
        if (lane == 0) {
          mbar_arrive(&raw_empty[rs]);
          mbar_signal_cluster(mapa_shared(smem_u32(&ready[cs]), 0));
        }
      }
      if (!ok) break;
      if (zeros) {
        const uint32_t sbuf = tile & 1;
        ok = __all_sync(0xffffffffu, mbar_wait_cluster(&sum_empty[sbuf], ((tile >> 1) & 1) ^ 1));
        if (!ok) { fail(); break; }
        sb -= 128 * codes;                   // the codes moved by 128
        // this CTA's 128 columns of the tile, to both CTAs
        const uint32_t at = smem_u32(sum_b + sbuf * 512 + grp * 256 + rank * 128 + r);
        sts_cluster(mapa_shared(at, 0), sb);
        sts_cluster(mapa_shared(at, 1), sb);
        __syncwarp();
        if (lane < 2) mbar_arrive_cluster(mapa_shared(smem_u32(&sum_full[sbuf]), lane));
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  cluster_sync();                            // no CTA leaves while its peer may still signal it
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc_pair(tmem, 512);
  }
}

// A's codes -> fp16 integers code - 128, and the row sums of those; one CTA per row
__global__ void __launch_bounds__(256) qgemm_widen_kernel(const QgemmArgs p) {
  __shared__ int red[8];
  const int m = blockIdx.x, nv = p.K >> 4;
  int s = 0;
  for (int i = threadIdx.x; i < nv; i += 256) {
    const uint4 u = __ldg(reinterpret_cast<const uint4*>(p.A + (int64_t)m * p.lda) + i);
    s = code_sum(u, s) - 128 * 16;
    uint4* o = reinterpret_cast<uint4*>(p.wide + (int64_t)m * p.K) + 2 * i;
    o[0] = make_uint4(half_codes(u.x, 0x4140), half_codes(u.x, 0x4342), half_codes(u.y, 0x4140), half_codes(u.y, 0x4342));
    o[1] = make_uint4(half_codes(u.z, 0x4140), half_codes(u.z, 0x4342), half_codes(u.w, 0x4140), half_codes(u.w, 0x4342));
  }
  if (!p.bz) return;
  s = __reduce_add_sync(0xffffffffu, s);
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = s;
  __syncthreads();
  if (threadIdx.x == 0) {
#pragma unroll
    for (int w = 1; w < 8; ++w) s += red[w];
    p.sum_a[m] = s;
  }
}

// sums of the splits -> outputs; four columns per thread
__global__ void __launch_bounds__(256) qgemm_join_kernel(const QgemmArgs p) {
  const int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
  const int nv = p.N >> 2;
  if (i >= (int64_t)p.M * nv) return;
  const int m = (int)(i / nv), n = (int)(i % nv) * 4;
  const bool zeros = p.az || p.bz;
  int a[4] = {}, b[4] = {};
  const int sa = p.bz ? p.sum_a[m] : 0;
  for (int s = 0; s < p.splits; ++s) {
    const int4 v = *reinterpret_cast<const int4*>(p.part + ((int64_t)s * p.M + m) * p.N + n);
    a[0] += v.x; a[1] += v.y; a[2] += v.z; a[3] += v.w;
    if (zeros) {
      const int4 t = *reinterpret_cast<const int4*>(p.part_sb + (int64_t)s * p.N + n);
      b[0] += t.x; b[1] += t.y; b[2] += t.z; b[3] += t.w;
    }
  }
  const float ah = __ldg(p.ah + m);
  const long long za = p.az ? (long long)__ldg(p.az + m) - 128 : 0;
  float y[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const long long zb = p.bz ? (long long)__ldg(p.bz + n + e) - 128 : 0;
    y[e] = finish(a[e], za, zb, sa, b[e], p.K, ah, __ldg(p.bh + n + e), zeros);
    if (p.bias) y[e] = __fadd_rn(y[e], __ldg(p.bias + n + e));
  }
  const int64_t at = (int64_t)m * p.ldc + n;
  if (p.Cf) *reinterpret_cast<float4*>(p.Cf + at) = make_float4(y[0], y[1], y[2], y[3]);
  if (p.Cb) {
    uint2 u;
    __nv_bfloat162* h = reinterpret_cast<__nv_bfloat162*>(&u);
    h[0] = __floats2bfloat162_rn(y[0], y[1]);
    h[1] = __floats2bfloat162_rn(y[2], y[3]);
    *reinterpret_cast<uint2*>(p.Cb + at) = u;
  }
}

// ================================================================================================
// few rows: the weight read is the bound
// ================================================================================================
// A CTA owns BN = 64 or 128 output channels and a share of K; a cluster of 1 to 8 CTAs covers K and joins its
// integer sums through distributed shared memory.  One thread keeps a ring of 16 KB weight tiles [BN
// channels x 16384 / BN codes] and the matching codes of 8 NT tokens in flight (TMA); eight warps, each on
// 32 channels and a 64-code slice of a tile, form 32 channels x 8 NT tokens by mma.sync m16n8k16.  The weight
// rows are the M dimension, so one token costs an eighth of a tile, and the codes are converted in registers
// between the shared-memory load and the product: no converted copy is written.  K is numbered inside the
// products so that a thread's operand values are 16 consecutive codes of its row; row 8 i + g of a product
// is tile row 8 i + (g % 2) 4 + g / 2, so that the eight lanes of a load phase hit eight distinct 16-byte
// bank groups of the 128-byte swizzle.
// Measured: 1 x 12288 x 4096 (192 CTAs, no cluster) 13.4 us, 17 x 5120 x 13824 (clusters of 3) 22 us, 3.8 and 3.2 TB/s
// of weight codes.  What is not the read is the start, the first tiles and the epilogue, about 6 us, and, from 17
// rows on, the conversion.
constexpr int FEW_WARPS = 8;

__device__ __forceinline__ void mma16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                         uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

__device__ __forceinline__ uint32_t pick(const uint4& v, int i) { return i == 0 ? v.x : (i == 1 ? v.y : (i == 2 ? v.z : v.w)); }

// 16 codes 128 (value 0): what lies beyond K
__device__ __forceinline__ uint4 no_codes() { return make_uint4(0x80808080u, 0x80808080u, 0x80808080u, 0x80808080u); }

__device__ __forceinline__ int lds_cluster(uint32_t addr) {
  int v;
  asm volatile("ld.shared::cluster.b32 %0, [%1];" : "=r"(v) : "r"(addr) : "memory");
  return v;
}

template <int NT, int FEW_N>
struct Few {
  static constexpr int TOK = 8 * NT, FEW_K = 16384 / FEW_N;
  static constexpr int STAGES = NT <= 2 ? 5 : 4;
  static constexpr int STAGE = (FEW_N + TOK) * FEW_K;                 // bytes
  static constexpr int RED_OFF = STAGES * STAGE;                      // [TOK][FEW_N] integer sums
  static constexpr int SUM_OFF = RED_OFF + TOK * FEW_N * 4;           // code sums: [TOK] of A, [FEW_N] of B
  static constexpr int BAR_OFF = SUM_OFF + (TOK + FEW_N) * 4;
  static constexpr int BYTES = BAR_OFF + 2 * STAGES * 8 + 16 + 1024;
};

template <int NT, int FEW_N>
__global__ void __launch_bounds__((FEW_WARPS + 1) * 32, 2)
    qgemm_few_kernel(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB, const QgemmArgs p,
                     const int ck, const int k_share) {
  using F = Few<NT, FEW_N>;
  constexpr int FEW_K = F::FEW_K, FEW_GROUPS = FEW_N / 32;
  extern __shared__ uint8_t few_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(few_raw) + 1023) & ~uintptr_t(1023));
  int* red = reinterpret_cast<int*>(smem + F::RED_OFF);
  int* red_a = reinterpret_cast<int*>(smem + F::SUM_OFF);
  int* red_b = red_a + F::TOK;
  uint64_t* full = reinterpret_cast<uint64_t*>(smem + F::BAR_OFF);
  uint64_t* empty = full + F::STAGES;
  volatile int* abort_flag = reinterpret_cast<volatile int*>(empty + F::STAGES);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int rank = ck > 1 ? (int)cluster_ctarank() : 0;
  const int n0 = (blockIdx.x / ck) * FEW_N, m0 = blockIdx.y * F::TOK;
  const int k_begin = rank * k_share, k_end = min(p.K, k_begin + k_share);
  const int steps = k_end > k_begin ? (k_end - k_begin + FEW_K - 1) / FEW_K : 0;
  const bool sum_b = p.az != nullptr, sum_a = p.bz != nullptr;
  for (int i = threadIdx.x; i < F::TOK * FEW_N + F::TOK + FEW_N; i += (FEW_WARPS + 1) * 32) red[i] = 0;   // and the code sums
  if (threadIdx.x == 0) {
    for (int s = 0; s < F::STAGES; ++s) { mbar_init(&full[s], 1); mbar_init(&empty[s], FEW_WARPS); }
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  __syncthreads();
  if (warp == FEW_WARPS) {
    int i = 0;                               // the whole warp runs the loop, one lane issues
    for (; i < steps; ++i) {
      const int s = i % F::STAGES;
      if (p.withhold && i == 0) continue;            // self-test: the first tile never comes
      if (!warp_wait(&empty[s], ((i / F::STAGES) & 1) ^ 1, p.wait_ns)) {
        omq_set_status(p.status, OMQ_ERR_TIMEOUT); *abort_flag = 1; break;
      }
      uint8_t* dst = smem + s * F::STAGE;
      if (elect_one()) {
        mbar_expect_tx(&full[s], F::STAGE);
#pragma unroll
        for (int b = 0; b < FEW_K / 128; ++b) {
          tma_load_3d(&tmB, &full[s], dst + b * FEW_N * 128, k_begin + i * FEW_K + 128 * b, n0, 0);
          tma_load_3d(&tmA, &full[s], dst + FEW_N * FEW_K + b * F::TOK * 128, k_begin + i * FEW_K + 128 * b, m0, 0);
        }
      }
      __syncwarp();
    }
    if (__any_sync(0xffffffffu, *abort_flag))        // no copy may land after this CTA has left
      for (int j = i > F::STAGES ? i - F::STAGES : 0; j < i; ++j)
        if (!(p.withhold && j == 0) && !wait_phase(&full[j % F::STAGES], (j / F::STAGES) & 1, p.wait_ns)) break;
  } else {
    // channel group, 64-code slice of the tile, this thread's 16-code chunk of its rows' 128 bytes
    const int cw = warp % FEW_GROUPS, kq = warp / FEW_GROUPS, c = t + 4 * (kq & 1);
    int sb[4] = {0, 0, 0, 0}, sa[NT] = {};           // code sums: of the weight rows, of the token tiles that this warp counts
    float d[2][NT][4];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) d[i][j][e] = 0.f;
    const int row = (g & 1) * 4 + (g >> 1);          // tile row of product row g
    for (int i = 0; i < steps; ++i) {
      const int s = i % F::STAGES;
      if (!warp_wait(&full[s], (i / F::STAGES) & 1, p.wait_ns)) {
        omq_set_status(p.status, OMQ_ERR_TIMEOUT); *abort_flag = 1; break;
      }
      const uint32_t wb = smem_u32(smem + s * F::STAGE) + ((kq >> 1) * FEW_N + 32 * cw + row) * 128 + ((c ^ row) << 4);
      const uint32_t ab = smem_u32(smem + s * F::STAGE) + FEW_N * FEW_K + ((kq >> 1) * F::TOK + row) * 128 + ((c ^ row) << 4);
      uint4 w[4], x[NT];
#pragma unroll
      for (int q = 0; q < 4; ++q) w[q] = lds128(wb + 8 * q * 128);
#pragma unroll
      for (int j = 0; j < NT; ++j) x[j] = lds128(ab + 8 * j * 128);
      if (i == steps - 1 && 128 * (kq >> 1) + 16 * c >= k_end - (k_begin + i * FEW_K)) {   // beyond K
#pragma unroll
        for (int q = 0; q < 4; ++q) w[q] = no_codes();
#pragma unroll
        for (int j = 0; j < NT; ++j) x[j] = no_codes();
      }
      if (sum_b) {
#pragma unroll
        for (int q = 0; q < 4; ++q) sb[q] = code_sum(w[q], sb[q]);
      }
      if (sum_a) {
#pragma unroll
        for (int j = 0; j < NT; ++j)
          if (j % FEW_GROUPS == cw) sa[j / FEW_GROUPS] = code_sum(x[j], sa[j / FEW_GROUPS]);
      }
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        uint32_t b0[NT], b1[NT];
#pragma unroll
        for (int j = 0; j < NT; ++j) { b0[j] = half_codes(pick(x[j], q), 0x4140); b1[j] = half_codes(pick(x[j], q), 0x4342); }
#pragma unroll
        for (int mt = 0; mt < 2; ++mt) {
          const uint32_t u = pick(w[2 * mt], q), v = pick(w[2 * mt + 1], q);
          const uint32_t f0 = half_codes(u, 0x4140), f1 = half_codes(v, 0x4140), f2 = half_codes(u, 0x4342),
                         f3 = half_codes(v, 0x4342);
#pragma unroll
          for (int j = 0; j < NT; ++j) mma16816(d[mt][j], f0, f1, f2, f3, b0[j], b1[j]);
        }
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(&empty[s]);
      // every 1024 codes of this warp's slices the fp32 sums, still exact, go to integers in shared memory
      // (several warps add to each: integer sums do not depend on the order)
      if (i % 16 == 15 || i == steps - 1) {
#pragma unroll
        for (int mt = 0; mt < 2; ++mt)
#pragma unroll
          for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              // column e & 1 of the pair is token 2 t + (e & 1) as a product column: tile row of A
              const int col = 2 * t + (e & 1), tok = 8 * j + (col & 1) * 4 + (col >> 1);
              atomicAdd(red + tok * FEW_N + 32 * cw + 16 * mt + 8 * (e >> 1) + row, __float2int_rn(d[mt][j][e]));
              d[mt][j][e] = 0.f;
            }
      }
    }
    const int moved = 128 * 16 * steps;              // the codes moved by 128: each thread summed 16 per stage
    if (sum_b) {
#pragma unroll
      for (int q = 0; q < 4; ++q) atomicAdd(red_b + 32 * cw + 8 * q + row, sb[q] - moved);
    }
    if (sum_a) {
#pragma unroll
      for (int j = 0; j < NT; ++j)
        if (j % FEW_GROUPS == cw) atomicAdd(red_a + 8 * j + row, sa[j / FEW_GROUPS] - moved);
    }
  }
  __syncthreads();
  if (ck > 1) cluster_sync();                                         // release / acquire over the cluster
  // CTA `rank` finishes its share of the channels over the cluster's sums
  const int share = (FEW_N + ck - 1) / ck, rows = min(F::TOK, p.M - m0);
  for (int i = threadIdx.x; i < share * rows; i += (FEW_WARPS + 1) * 32) {
    const int c = rank * share + i % share, m = i / share, n = n0 + c;
    if (c >= FEW_N || n >= p.N) continue;
    int s = 0, ta = 0, tb = 0;
    if (ck > 1) {
      const uint32_t ar = smem_u32(red + m * FEW_N + c), aa = smem_u32(red_a + m), ab = smem_u32(red_b + c);
      for (int r = 0; r < ck; ++r) {
        s += lds_cluster(mapa_shared(ar, r));
        if (sum_a) ta += lds_cluster(mapa_shared(aa, r));
        if (sum_b) tb += lds_cluster(mapa_shared(ab, r));
      }
    } else {
      s = red[m * FEW_N + c]; ta = red_a[m]; tb = red_b[c];
    }
    const int mg = m0 + m;
    const long long za = p.az ? (long long)__ldg(p.az + mg) - 128 : 0, zb = p.bz ? (long long)__ldg(p.bz + n) - 128 : 0;
    float y = finish(s, za, zb, ta, tb, p.K, __ldg(p.ah + mg), __ldg(p.bh + n), sum_a || sum_b);
    if (p.bias) y = __fadd_rn(y, __ldg(p.bias + n));
    if (p.Cf) p.Cf[(int64_t)mg * p.ldc + n] = y;
    if (p.Cb) p.Cb[(int64_t)mg * p.ldc + n] = f_to_bf16(y);
  }
  if (ck > 1) cluster_sync();                                         // no CTA leaves while its sums may be read
}

template <int NT, int FEW_N>
omq_status few_launch(cudaStream_t st, const QgemmArgs& p) {
  using F = Few<NT, FEW_N>;
  auto kern = qgemm_few_kernel<NT, FEW_N>;
  static std::atomic<uint64_t> allowed{0};
  OMQ_TRY(omq_allow_smem(allowed, kern, F::BYTES));
  CUtensorMap ta, tb;
  if (!omq_make_map_u8(&ta, p.A, p.K, p.M, p.lda, F::TOK, 128) || !omq_make_map_u8(&tb, p.B, p.K, p.N, p.ldb, FEW_N, 128))
    return OMQ_ERR_UNSUPPORTED;
  // One wave of CTAs, two per SM: the start of a CTA (tile ring, signals, joining) costs about 4 us, so a
  // second wave loses more than an idle SM (4096 x 4096, one row: 6.6 us on 256 CTAs, 10.9 us on 512).
  // Within that K is split as far as it goes, no share under 512 codes; clusters of 5 and 7 fill the SMs
  // badly (5120 x 13824: 16.7 us with 6, 24.5 us with 7).
  const int gy = (p.M + F::TOK - 1) / F::TOK, blocks = (p.N + FEW_N - 1) / FEW_N, cand[6] = {8, 6, 4, 3, 2, 1};
  int ck = 1;
  for (int c : cand)
    if (blocks * gy * c <= 2 * omq_num_sms() && p.K >= 512 * c) { ck = c; break; }
  const int k_share = ((p.K + ck - 1) / ck + F::FEW_K - 1) / F::FEW_K * F::FEW_K;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(blocks * ck), (unsigned)gy, 1);
  cfg.blockDim = dim3((FEW_WARPS + 1) * 32, 1, 1);
  cfg.dynamicSmemBytes = F::BYTES;
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = ck; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = ck > 1 ? 1 : 0;
  if (cudaLaunchKernelEx(&cfg, kern, ta, tb, p, ck, k_share) != cudaSuccess) { cudaGetLastError(); return OMQ_ERR_CUDA; }
  OMQ_LAUNCH_CHECK();
  return OMQ_OK;
}

// ------------------------------------------------------------------------------------------------
// The register form.  64 channels per CTA while that is one wave, else 128 (22016 x 4096, one row: 22.9 against 25.8
// us); with 17 rows and more the conversion of the tokens counts and 64 stays the faster (34.4 against 40.5 us).
// Rows of a block from 17 on: 24 where that makes no more blocks than 32 (17 x 5120 x 13824: 22.0 against 25.0 us,
// 48 x 22016 x 4096: 48.4 against 53.8).
omq_status few_rows(cudaStream_t st, const QgemmArgs& p) {
  const bool wide = (p.N + 63) / 64 > 2 * omq_num_sms();
  if (p.M <= 8) return wide ? few_launch<1, 128>(st, p) : few_launch<1, 64>(st, p);
  if (p.M <= 16) return wide ? few_launch<2, 128>(st, p) : few_launch<2, 64>(st, p);
  return (p.M + 23) / 24 == (p.M + 31) / 32 ? few_launch<3, 64>(st, p) : few_launch<4, 64>(st, p);
}

// ------------------------------------------------------------------------------------------------
struct QPlan { int splits, kb_per_split; double us; };

// K split of the tensor-core form.  The work items (tiles x splits) run in rounds over the CTA pairs; a split
// shortens an item and can fill the last round, and costs the partial sums' way through memory and a joining
// launch.  Estimated with what the kernel measured: 0.8 us per 128 codes of K, 3 us per item, 3 us per joining
// launch and 1 us per million partial sums (64 x 22016 x 4096: 76 us in 2 rounds of 86 tiles, 63 us
// split).  No piece under 512 codes.
QPlan plan_of(int64_t M, int64_t N, int64_t K) {
  const int64_t tiles = ((M + 255) / 256) * ((N + 255) / 256), pairs = omq_num_sms() / 2, kbs = (K + BK - 1) / BK;
  QPlan best{1, (int)kbs, 1e30};
  for (int64_t s = 1; s <= 16 && (s == 1 || kbs / s >= 512 / BK); ++s) {
    const int64_t per = (kbs + s - 1) / s, n = (kbs + per - 1) / per, rounds = (tiles * n + pairs - 1) / pairs;
    const double us = rounds * (0.8 * per + 3.0) + (n > 1 ? 3.0 + 1e-6 * n * M * N : 0.0);
    if (us < best.us) best = {(int)n, (int)per, us};
  }
  return best;
}

// Which form: up to 32 rows the first; beyond, by estimates that both measured.  The tensor-core form costs its
// plan and 7.5 us for the widening launch and its own start (64 x 4096 x 4096: 21.8 us, 64 x 12288 x 4096: 35.8);
// the register form 6 us and, for each block of rows, the weight codes at 3.4 TB/s (15.4 and 36.7 us; 128 rows
// 23.6 and 64 us; 128 x 1024 x 4096: 9.8 against 22.5 us).  (Blocks of 24 reach 3.9 TB/s where K is split, but
// 33 x 5120 x 13824 takes 48.3 us in them, unsplit, and 38.8 in the tensor-core form.)
bool use_few(int64_t M, int64_t N, int64_t K) {
  if (M <= 32) return true;
  if ((M + 31) / 32 > 65535) return false;       // its row blocks are the grid's second axis
  return 6.0 + (double)((M + 31) / 32) * N * K / 3.4e6 < plan_of(M, N, K).us + 7.5;
}

// workspace of the tensor-core form: fp16 A | its row sums | partial sums of the K split (and of B's codes);
// every part a multiple of 16 bytes
struct QSpace { size_t sum_a, part, part_sb, bytes; };
QSpace space_of(int64_t M, int64_t N, int64_t K, int splits) {
  QSpace w;
  w.sum_a = (size_t)M * K * 2;
  w.part = w.sum_a + (size_t)((M + 3) / 4 * 4) * 4;
  w.part_sb = w.part + (splits > 1 ? (size_t)splits * M * N * 4 : 0);
  w.bytes = w.part_sb + (splits > 1 ? (size_t)splits * N * 4 : 0);
  return w;
}

}  // namespace

extern "C" size_t omq_qgemm_i8_workspace_size(int64_t M, int64_t N, int64_t K) {
  if (M <= 0 || N <= 0 || K <= 0 || use_few(M, N, K)) return 0;
  return space_of(M, N, K, plan_of(M, N, K).splits).bytes;
}

extern "C" omq_status omq_qgemm_i8(omq_stream_t stream, int64_t M, int64_t N, int64_t K, const uint8_t* A, int64_t lda,
                                   const float* a_h, const int32_t* a_z, const uint8_t* B, int64_t ldb, const float* b_h,
                                   const int32_t* b_z, const float* bias, float* Cf, void* Cb, int64_t ldc,
                                   void* workspace, size_t ws_bytes, int32_t* dev_status) {
  OMQ_REQUIRE(M > 0 && N > 0 && K > 0 && M < (1 << 22) && N < (1 << 24) && K <= 65536, OMQ_ERR_SHAPE);
  OMQ_REQUIRE(A && B && a_h && b_h && (Cf || Cb), OMQ_ERR_INVALID_ARG);
  OMQ_REQUIRE(lda >= K && ldb >= K && ldc >= N, OMQ_ERR_SHAPE);
  OMQ_REQUIRE(K % 16 == 0 && lda % 16 == 0 && ldb % 16 == 0 && N % 8 == 0 && ldc % 8 == 0, OMQ_ERR_ALIGN);
  OMQ_REQUIRE(omq_aligned16(A) && omq_aligned16(B) && omq_aligned16(a_h) && omq_aligned16(b_h) && omq_aligned16(a_z) &&
                  omq_aligned16(b_z) && omq_aligned16(bias) && omq_aligned16(Cf) && omq_aligned16(Cb) &&
                  omq_aligned16(workspace),
              OMQ_ERR_ALIGN);
  const size_t need = omq_qgemm_i8_workspace_size(M, N, K);
  OMQ_REQUIRE(need == 0 || (workspace && ws_bytes >= need), OMQ_ERR_WORKSPACE);
  cudaStream_t st = (cudaStream_t)stream;
  QgemmArgs p{};
  p.M = (int)M; p.N = (int)N; p.K = (int)K;
  p.A = A; p.lda = lda; p.ah = a_h; p.az = a_z;
  p.B = B; p.ldb = ldb; p.bh = b_h; p.bz = b_z;
  p.bias = bias; p.Cf = Cf; p.Cb = (__nv_bfloat16*)Cb; p.ldc = ldc; p.status = dev_status;
  p.wait_ns = (uint32_t)OMQ_WAIT_LIMIT_NS;
  if (use_few(M, N, K)) return few_rows(st, p);
  const QPlan q = plan_of(M, N, K);
  p.splits = q.splits; p.kb_per_split = q.kb_per_split;
  const QSpace sp = space_of(M, N, K, q.splits);
  uint8_t* const space = (uint8_t*)workspace;
  p.wide = (__half*)space;
  p.sum_a = (int32_t*)(space + sp.sum_a);
  p.part = (int32_t*)(space + sp.part);
  p.part_sb = (int32_t*)(space + sp.part_sb);
  p.m_fast = (double)M > 1.5 * (double)N ? 0 : 1;               // keep the smaller operand in L2
  CUtensorMap ta, tb;
  if (!omq_make_map_bf16(&ta, p.wide, K, M, 1, K, 0, 64, 128) || !omq_make_map_u8(&tb, B, K, N, ldb, 128, BK))
    return OMQ_ERR_UNSUPPORTED;              // (a map of any 16-bit type moves fp16)
  static std::atomic<uint64_t> allowed{0};
  OMQ_TRY(omq_allow_smem(allowed, qgemm_tc_kernel, TC_SMEM));
  qgemm_widen_kernel<<<(unsigned)M, 256, 0, st>>>(p);
  OMQ_LAUNCH_CHECK();
  const int64_t items = ((M + 255) / 256) * ((N + 255) / 256) * q.splits, pairs = omq_num_sms() / 2;
  qgemm_tc_kernel<<<(unsigned)(2 * (items < pairs ? items : pairs)), TC_THREADS, TC_SMEM, st>>>(ta, tb, p);
  OMQ_LAUNCH_CHECK();
  if (q.splits > 1) {
    const int64_t n = M * (N / 4);
    qgemm_join_kernel<<<(unsigned)((n + 255) / 256), 256, 0, st>>>(p);
    OMQ_LAUNCH_CHECK();
  }
  return OMQ_OK;
}

// Failure-detection self-test: the register form with every wait bounded by wait_limit_ns, and optionally
// without its first tile, so that the wait for it runs out.
extern "C" omq_status omq_selftest_qgemm_wait(omq_stream_t stream, int64_t M, int64_t N, int64_t K, const uint8_t* A,
                                              const float* a_h, const uint8_t* B, const float* b_h, float* C,
                                              uint64_t wait_limit_ns, int32_t withhold, int32_t* dev_status) {
  OMQ_REQUIRE(M > 0 && M <= 32 && N > 0 && N <= 65536 && K > 0 && K <= 65536, OMQ_ERR_SHAPE);
  OMQ_REQUIRE(A && a_h && B && b_h && C, OMQ_ERR_INVALID_ARG);
  OMQ_REQUIRE(withhold == 0 || withhold == 1, OMQ_ERR_INVALID_ARG);
  OMQ_REQUIRE(wait_limit_ns >= 1000ull && wait_limit_ns <= OMQ_WAIT_LIMIT_NS, OMQ_ERR_INVALID_ARG);
  OMQ_REQUIRE(K % 16 == 0 && N % 8 == 0, OMQ_ERR_ALIGN);
  OMQ_REQUIRE(omq_aligned16(A) && omq_aligned16(B) && omq_aligned16(a_h) && omq_aligned16(b_h) && omq_aligned16(C),
              OMQ_ERR_ALIGN);
  QgemmArgs p{};
  p.M = (int)M; p.N = (int)N; p.K = (int)K;
  p.A = A; p.lda = K; p.ah = a_h; p.B = B; p.ldb = K; p.bh = b_h; p.Cf = C; p.ldc = N;
  p.status = dev_status;
  p.wait_ns = (uint32_t)wait_limit_ns;
  p.withhold = withhold;
  return few_rows((cudaStream_t)stream, p);
}
