// Residual addition + RMSNorm + per-token Q_a in one pass (omq_rmsnorm_quant).
//
// One CTA owns one token row at a time and keeps it in registers: t = x + r, the block sum of t^2,
// y = t rstd gain + bias, the block max / min of y, Eq. 2 on every element; the next row is on its way
// to L2, or to shared memory, meanwhile.  Nothing of the row is read twice; the bound is HBM (x, r in; codes, values, residual sum
// out): 8192 x 8192, bf16 in, fp32 residual, 147 us, 5.95 TB/s.  Elements are worked on in pairs, and the
// roundings of Eq. 2 are additions of 1.5 * 2^23 instead of conversions, which halves the instructions
// per element.
#include "common.cuh"
#include "tc.cuh"

namespace {

using namespace tc;

struct NormArgs {
  const void* X; int64_t ldx;
  const void* R; void* H; int64_t ldr;
  const float* gain; const float* bias;
  float rms_eps;
  int64_t T; int C;
  uint8_t* codes; __nv_bfloat16* Xq; float* h; int32_t* z;
  int abits; float h_eps;
};

// eight consecutive elements, widened exactly
template <bool BF>
__device__ __forceinline__ void widen8(const uint4& a, const uint4& b, float2 (&v)[4]) {
  if (BF) {
    v[0] = make_float2(__uint_as_float(a.x << 16), __uint_as_float(a.x & 0xffff0000u));
    v[1] = make_float2(__uint_as_float(a.y << 16), __uint_as_float(a.y & 0xffff0000u));
    v[2] = make_float2(__uint_as_float(a.z << 16), __uint_as_float(a.z & 0xffff0000u));
    v[3] = make_float2(__uint_as_float(a.w << 16), __uint_as_float(a.w & 0xffff0000u));
  } else {
    v[0] = make_float2(__uint_as_float(a.x), __uint_as_float(a.y));
    v[1] = make_float2(__uint_as_float(a.z), __uint_as_float(a.w));
    v[2] = make_float2(__uint_as_float(b.x), __uint_as_float(b.y));
    v[3] = make_float2(__uint_as_float(b.z), __uint_as_float(b.w));
  }
}

template <bool BF>
__device__ __forceinline__ void staged8(uint32_t base, int i, float2 (&v)[4]) {
  const uint32_t at = base + i * (BF ? 2 : 4);
  const uint4 a = lds128(at);
  uint4 b = a;
  if (!BF) b = lds128(at + 16);
  widen8<BF>(a, b, v);
}

// RO: through the read-only path.  The residual is not: R and H may be one buffer.
template <bool BF, bool RO>
__device__ __forceinline__ void load8(const void* base, int64_t off, float2 (&v)[4]) {
  const uint4* p = reinterpret_cast<const uint4*>(static_cast<const char*>(base) + off * (BF ? 2 : 4));
  const uint4 a = RO ? __ldg(p) : *p;
  uint4 b = a;
  if (!BF) b = RO ? __ldg(p + 1) : p[1];
  widen8<BF>(a, b, v);
}

__device__ __forceinline__ uint32_t bf16x2(float2 v) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(v.x, v.y);
  return *reinterpret_cast<const uint32_t*>(&h);
}

template <bool BF>
__device__ __forceinline__ void store8(void* base, int64_t off, const float2 (&v)[4]) {
  uint4* p = reinterpret_cast<uint4*>(static_cast<char*>(base) + off * (BF ? 2 : 4));
  if (BF) {
    *p = make_uint4(bf16x2(v[0]), bf16x2(v[1]), bf16x2(v[2]), bf16x2(v[3]));
  } else {
    reinterpret_cast<float4*>(p)[0] = make_float4(v[0].x, v[0].y, v[1].x, v[1].y);
    reinterpret_cast<float4*>(p)[1] = make_float4(v[2].x, v[2].y, v[3].x, v[3].y);
  }
}

// max / min of three that return NaN where an operand is one
__device__ __forceinline__ float max3_nan(float a, float b, float c) {
  float d;
  asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}
__device__ __forceinline__ float min3_nan(float a, float b, float c) {
  float d;
  asm("min.NaN.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}

// block max and min, NaN where the row holds one.  smem >= 64 floats.
__device__ __forceinline__ void block_extremes(float& M, float& m, float* smem) {
  const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5, nw = (blockDim.x + 31) >> 5;
#pragma unroll
  for (int off = 16; off > 0; off >>= 1) {
    M = max3_nan(M, __shfl_xor_sync(0xffffffffu, M, off), -INFINITY);
    m = min3_nan(m, __shfl_xor_sync(0xffffffffu, m, off), INFINITY);
  }
  if (lane == 0) { smem[wid] = M; smem[32 + wid] = m; }
  __syncthreads();
  M = lane < nw ? smem[lane] : -INFINITY;
  m = lane < nw ? smem[32 + lane] : INFINITY;
#pragma unroll
  for (int off = 16; off > 0; off >>= 1) {
    M = max3_nan(M, __shfl_xor_sync(0xffffffffu, M, off), -INFINITY);
    m = min3_nan(m, __shfl_xor_sync(0xffffffffu, m, off), INFINITY);
  }
}

// block sum; smem >= 32 floats
__device__ __forceinline__ float block_sum(float a, float* smem) {
  const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5, nw = (blockDim.x + 31) >> 5;
  a = warp_sum(a);
  if (lane == 0) smem[wid] = a;
  __syncthreads();
  return warp_sum(lane < nw ? smem[lane] : 0.f);
}

constexpr float ROUND = 12582912.f;            // 1.5 * 2^23: x + ROUND holds the integer nearest to x, |x| < 2^22

// Eq. 2 on a pair, as omq_fakequant2, with the roundings by the addition of ROUND (half to even, like
// rint): for |y / h| and |z| below 2^21.  Returns the value; *w = code + ROUND.
struct Fast { float2 rh, nh, h, round, back, zr, nzr; float lo, hi; };
__device__ __forceinline__ float2 quant2(const float2 y, const Fast& q, float2* w) {
  const float2 k = omq_add2(omq_add2(omq_mul2(y, q.rh), q.round), q.back);
  const float2 r = omq_mul2(omq_fma2(k, q.nh, y), q.rh);
  const float2 c = omq_add2(omq_add2(omq_add2(omq_add2(r, q.round), q.back), k), q.zr);     // round(y / h) + z + ROUND
  w->x = fminf(fmaxf(c.x, q.lo), q.hi);
  w->y = fminf(fmaxf(c.y, q.lo), q.hi);
  return omq_mul2(omq_add2(*w, q.nzr), q.h);
}

// ST: the next row's x and r come by bulk copy into shared memory, not by prefetch into L2
template <bool XB, bool RB, int V, int MAX_THREADS, int MIN_CTAS, bool ST>
__global__ void __launch_bounds__(MAX_THREADS, MIN_CTAS) rmsnorm_quant_kernel(const NormArgs a) {
  __shared__ float red[2][96];                   // by row parity: one barrier fewer per row
  __shared__ uint64_t landed;
  __shared__ int late;
  extern __shared__ __align__(16) uint8_t stage[];         // the raw row of x and of r
  const int tid = threadIdx.x, nt = blockDim.x, nvec = a.C >> 3;
  const uint32_t x_bytes = a.C * (XB ? 2 : 4), r_bytes = a.R ? a.C * (RB ? 2 : 4) : 0;
  bool staged = ST;
  auto fetch = [&](int64_t t) {                  // one thread
    mbar_expect_tx(&landed, x_bytes + r_bytes);
    bulk_g2s(stage, (const char*)a.X + t * a.ldx * (XB ? 2 : 4), x_bytes, &landed);
    if (a.R) bulk_g2s(stage + x_bytes, (const char*)a.R + t * a.ldr * (RB ? 2 : 4), r_bytes, &landed);
  };
  if (ST) {
    if (tid == 0) {
      late = 0;
      mbar_init(&landed, 1);
      asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
      fetch(blockIdx.x);
    }
    __syncthreads();
  }
  int par = 0;
  for (int64_t t = blockIdx.x; t < a.T; t += gridDim.x, par ^= 1) {
    float2 v[V][4];
    // a copy that has not come within the limit: this row and the rest without staging; the CTA leaves only
    // after another wait for the copy
    const bool here = staged && wait_phase(&landed, par);
    if (staged && !here) { late = 1; wait_phase(&landed, par); }
    if (!ST && tid == 0 && t + gridDim.x < a.T) {       // the next row of this CTA, into L2
      omq_l2_prefetch((const char*)a.X + (t + gridDim.x) * a.ldx * (XB ? 2 : 4), (uint64_t)a.C * (XB ? 2 : 4));
      if (a.R) omq_l2_prefetch((const char*)a.R + (t + gridDim.x) * a.ldr * (RB ? 2 : 4), (uint64_t)a.C * (RB ? 2 : 4));
    }
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const int vi = j * nt + tid;
#pragma unroll
      for (int e = 0; e < 4; ++e) v[j][e] = make_float2(0.f, 0.f);
      if (vi < nvec) {
        if (here) staged8<XB>(smem_u32(stage), 8 * vi, v[j]);
        else load8<XB, true>(a.X, t * a.ldx + 8 * vi, v[j]);
      }
    }
    if (a.R) {
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const int vi = j * nt + tid;
        if (vi < nvec) {
          float2 r[4];
          if (here) staged8<RB>(smem_u32(stage) + x_bytes, 8 * vi, r);
          else load8<RB, false>(a.R, t * a.ldr + 8 * vi, r);
#pragma unroll
          for (int e = 0; e < 4; ++e) v[j][e] = omq_add2(v[j][e], r[e]);
        }
      }
    }
    float2 ss = make_float2(0.f, 0.f);
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const int vi = j * nt + tid;
      if (a.H && vi < nvec) store8<RB>(a.H, t * a.ldr + 8 * vi, v[j]);
#pragma unroll
      for (int e = 0; e < 4; ++e) ss = omq_fma2(v[j][e], v[j][e], ss);
    }
    const float tot = block_sum(ss.x + ss.y, red[par]);
    if (ST) {                                    // the row is in registers: its buffer takes the next one
      staged = staged && *(volatile int*)&late == 0;
      if (staged && tid == 0 && t + gridDim.x < a.T) fetch(t + gridDim.x);
    }
    const float rstd = 1.0f / sqrtf(tot / (float)a.C + a.rms_eps);
    const float2 rs = make_float2(rstd, rstd);
    float M = -INFINITY, m = INFINITY;
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const int vi = j * nt + tid;
      if (vi < nvec) {
        float2 g[4], b[4];
        if (a.gain) load8<false, true>(a.gain, 8 * vi, g);
        if (a.bias) load8<false, true>(a.bias, 8 * vi, b);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          float2 y = omq_mul2(v[j][e], rs);
          if (a.gain) y = omq_mul2(y, g[e]);
          if (a.bias) y = omq_add2(y, b[e]);
          v[j][e] = y;
          M = max3_nan(M, y.x, y.y);
          m = min3_nan(m, y.x, y.y);
        }
      }
    }
    if (a.abits < 16) {
      const float Q = (float)((1 << a.abits) - 1);
      block_extremes(M, m, red[par] + 32);
      const bool bad = !(M < INFINITY && m > -INFINITY);
      const QState qs = omq_qstate(bad ? 0.f : M, bad ? 0.f : m, 1.f, 1.f, Q, a.h_eps);
      if (tid == 0) { a.h[t] = bad ? NAN : qs.h; a.z[t] = bad ? 0 : (int32_t)qs.z; }
      uint8_t* cr = a.codes ? a.codes + t * a.C : nullptr;
      __nv_bfloat16* xr = a.Xq ? a.Xq + t * a.C : nullptr;
      const bool near = fmaxf(fabsf(M), fabsf(m)) * qs.rh < 2097152.f && fabsf(qs.z) < 2097152.f;
      if (near) {                                // every row but those far from zero in steps
        Fast q;
        q.rh = make_float2(qs.rh, qs.rh); q.nh = make_float2(-qs.h, -qs.h); q.h = make_float2(qs.h, qs.h);
        q.round = make_float2(ROUND, ROUND); q.back = make_float2(-ROUND, -ROUND);
        q.zr = make_float2(qs.z + ROUND, qs.z + ROUND); q.nzr = make_float2(-(qs.z + ROUND), -(qs.z + ROUND));
        q.lo = ROUND; q.hi = ROUND + Q;
#pragma unroll
        for (int j = 0; j < V; ++j) {
          const int vi = j * nt + tid;
          if (vi >= nvec) continue;
          uint32_t c[8];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            float2 w;
            v[j][e] = quant2(v[j][e], q, &w);
            c[2 * e] = __float_as_uint(w.x);       // the code is the low byte
            c[2 * e + 1] = __float_as_uint(w.y);
          }
          if (cr)
            *reinterpret_cast<uint2*>(cr + 8 * vi) =
                make_uint2(__byte_perm(__byte_perm(c[0], c[1], 0x0040), __byte_perm(c[2], c[3], 0x0040), 0x5410),
                           __byte_perm(__byte_perm(c[4], c[5], 0x0040), __byte_perm(c[6], c[7], 0x0040), 0x5410));
          if (xr) store8<true>(xr, 8 * vi, v[j]);
        }
      } else {
#pragma unroll 1
        for (int j = 0; j < V; ++j) {
          const int vi = j * nt + tid;
          if (vi >= nvec) continue;
          float2 y[4];
#pragma unroll
          for (int k = 0; k < V; ++k)
            if (k == j) { y[0] = v[k][0]; y[1] = v[k][1]; y[2] = v[k][2]; y[3] = v[k][3]; }
          uint32_t p[2] = {0, 0};
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            float2 c2;
            const float2 w = omq_fakequant2(y[e], qs, Q, &c2);
            y[e] = bad ? make_float2(NAN, NAN) : w;
            if (!bad) p[e >> 1] |= ((uint32_t)c2.x | ((uint32_t)c2.y << 8)) << (16 * (e & 1));
          }
          if (cr) *reinterpret_cast<uint2*>(cr + 8 * vi) = make_uint2(p[0], p[1]);
          if (xr) store8<true>(xr, 8 * vi, y);
        }
      }
    } else {
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const int vi = j * nt + tid;
        if (vi < nvec) store8<true>(a.Xq, t * a.C + 8 * vi, v[j]);
      }
    }
  }
}

template <bool XB, bool RB, int V, int MAX_THREADS, int MIN_CTAS, bool ST = false>
omq_status norm_run(cudaStream_t st, const NormArgs& a) {
  auto kern = rmsnorm_quant_kernel<XB, RB, V, MAX_THREADS, MIN_CTAS, ST>;
  const int smem = ST ? a.C * ((XB ? 2 : 4) + (a.R ? (RB ? 2 : 4) : 0)) : 0;
  if (ST) {
    static std::atomic<uint64_t> allowed{0};
    OMQ_TRY(omq_allow_smem(allowed, kern, 8 * V * MAX_THREADS * 8));
  }
  const int nt = ((a.C / 8 + V - 1) / V + 31) / 32 * 32;
  int per = 1;
  cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per, kern, nt, smem);
  const int64_t most = (int64_t)omq_num_sms() * (per > 0 ? per : 1);
  kern<<<(unsigned)(a.T < most ? a.T : most), nt, smem, st>>>(a);
  OMQ_LAUNCH_CHECK();
  return OMQ_OK;
}

// Eight-element vectors per thread.  Up to one row per SM the row's own latency counts and more threads win
// (1 x 4096: 3.8 us with one vector, 4.4 with four; 1 x 8192: 5.1, 5.3); with more rows fewer threads leave
// room for a second CTA (2048 x 5120 30.5 us with two, 38.1 with one) and, from 6 K columns on, four
// vectors amortise the two block reductions better (8192 x 8192: 146.6 us against 153.1 with two).  From six rows per
// SM on the shorter rows are staged (2048 x 4096, bf16 with fp32 residual: 22.4 against 25.4 us; 8192 x 4096: 70.9,
// 77.6; 700 x 4096: 13.2, 11.9); longer ones lose more than they gain (8192 x 8192: 182 us staged).
template <bool XB, bool RB>
omq_status norm_launch(cudaStream_t st, const NormArgs& a) {
  const int nvec = a.C / 8;
  const bool few = a.T <= omq_num_sms();
  if (few && nvec <= 1024) return norm_run<XB, RB, 1, 1024, 1>(st, a);
  if (few && nvec <= 2048) return norm_run<XB, RB, 2, 1024, 1>(st, a);
  if (nvec <= 768 && a.T > 6 * omq_num_sms()) return norm_run<XB, RB, 2, 512, 2, true>(st, a);
  if (nvec <= 768) return norm_run<XB, RB, 2, 512, 2>(st, a);
  if (nvec <= 2048) return norm_run<XB, RB, 4, 512, 1>(st, a);
  return norm_run<XB, RB, 8, 512, 1>(st, a);
}

}  // namespace

extern "C" omq_status omq_rmsnorm_quant(omq_stream_t stream, int64_t T, int64_t C, const void* X, int32_t x_dtype,
                                        int64_t ldx, const void* R, void* H, int32_t r_dtype, int64_t ldr,
                                        const float* gain, const float* bias, float rms_eps, uint8_t* codes, void* Xq,
                                        float* h, int32_t* z, const omq_qcfg* cfg) {
  OMQ_TRY(omq_check_cfg(cfg));
  const bool quant = cfg->abits < 16;
  OMQ_REQUIRE(T > 0 && C > 0 && C <= 32768, OMQ_ERR_SHAPE);
  OMQ_REQUIRE(X && (Xq || (codes && quant)), OMQ_ERR_INVALID_ARG);
  OMQ_REQUIRE(!quant || (h && z), OMQ_ERR_INVALID_ARG);
  OMQ_REQUIRE((x_dtype == OMQ_F32 || x_dtype == OMQ_BF16) && (r_dtype == OMQ_F32 || r_dtype == OMQ_BF16),
              OMQ_ERR_INVALID_ARG);
  OMQ_REQUIRE(rms_eps >= 0.f, OMQ_ERR_INVALID_ARG);
  OMQ_REQUIRE(ldx >= C && ((!R && !H) || ldr >= C), OMQ_ERR_SHAPE);
  OMQ_REQUIRE(C % 8 == 0 && ldx % 8 == 0 && ((!R && !H) || ldr % 8 == 0), OMQ_ERR_ALIGN);
  OMQ_REQUIRE(omq_aligned16(X) && omq_aligned16(R) && omq_aligned16(H) && omq_aligned16(gain) && omq_aligned16(bias) &&
                  omq_aligned16(codes) && omq_aligned16(Xq) && omq_aligned16(h) && omq_aligned16(z),
              OMQ_ERR_ALIGN);
  NormArgs a{X, ldx, R, H, ldr, gain, bias, rms_eps, T, (int)C, codes, (__nv_bfloat16*)Xq, h, z, cfg->abits, cfg->h_eps};
  if (!quant) a.codes = nullptr;
  cudaStream_t st = (cudaStream_t)stream;
  if (x_dtype == OMQ_BF16) return r_dtype == OMQ_BF16 ? norm_launch<true, true>(st, a) : norm_launch<true, false>(st, a);
  return r_dtype == OMQ_BF16 ? norm_launch<false, true>(st, a) : norm_launch<false, false>(st, a);
}
