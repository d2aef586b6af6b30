// Residual addition + RMSNorm + per-token Q_a in one pass (omq_rmsnorm_quant).
//
// One CTA owns one token row at a time and keeps it in registers: t = x + r, the block sum of t^2,
// y = t rstd gain + bias, the block max / min of y, Eq. 2 on every element.  Nothing of the row is
// read twice; the bound is HBM (x, r in; codes, values, residual sum out).
#include "common.cuh"

namespace {

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
__device__ __forceinline__ void load8(const void* base, int64_t off, float (&v)[8]) {
  if (BF) {
    const uint4 u = __ldg(reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(base) + off));
    unpack_bf16x8(u, v);
  } else {
    const float4* p = reinterpret_cast<const float4*>(static_cast<const float*>(base) + off);
    const float4 a = __ldg(p), b = __ldg(p + 1);
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
  }
}

// R and H may be one buffer: plain loads (no read-only path) for the residual
template <bool BF>
__device__ __forceinline__ void load8_rw(const void* base, int64_t off, float (&v)[8]) {
  if (BF) {
    const uint4 u = *reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(base) + off);
    unpack_bf16x8(u, v);
  } else {
    const float4* p = reinterpret_cast<const float4*>(static_cast<const float*>(base) + off);
    const float4 a = p[0], b = p[1];
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
  }
}

template <bool BF>
__device__ __forceinline__ void store8(void* base, int64_t off, const float (&v)[8]) {
  if (BF) {
    *reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(base) + off) = pack_bf16x8(v);
  } else {
    float4* p = reinterpret_cast<float4*>(static_cast<float*>(base) + off);
    p[0] = make_float4(v[0], v[1], v[2], v[3]);
    p[1] = make_float4(v[4], v[5], v[6], v[7]);
  }
}

// block max and min; an unordered value was turned into +inf by the caller.  smem >= 64 floats.
__device__ __forceinline__ void block_extremes(float& M, float& m, float* smem) {
  const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5, nw = (blockDim.x + 31) >> 5;
#pragma unroll
  for (int off = 16; off > 0; off >>= 1) {
    M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, off));
    m = fminf(m, __shfl_xor_sync(0xffffffffu, m, off));
  }
  if (lane == 0) { smem[wid] = M; smem[32 + wid] = m; }
  __syncthreads();
  M = lane < nw ? smem[lane] : -INFINITY;
  m = lane < nw ? smem[32 + lane] : INFINITY;
#pragma unroll
  for (int off = 16; off > 0; off >>= 1) {
    M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, off));
    m = fminf(m, __shfl_xor_sync(0xffffffffu, m, off));
  }
}

template <bool XB, bool RB, int V>
__global__ void __launch_bounds__(1024) rmsnorm_quant_kernel(const NormArgs a) {
  __shared__ float red[128];
  const int tid = threadIdx.x, nt = blockDim.x, nvec = a.C >> 3;
  for (int64_t t = blockIdx.x; t < a.T; t += gridDim.x) {
    float v[V][8];
    float ss = 0.f;
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const int vi = j * nt + tid;
#pragma unroll
      for (int e = 0; e < 8; ++e) v[j][e] = 0.f;
      if (vi < nvec) load8<XB>(a.X, t * a.ldx + 8 * vi, v[j]);
    }
    if (a.R) {
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const int vi = j * nt + tid;
        if (vi < nvec) {
          float r[8];
          load8_rw<RB>(a.R, t * a.ldr + 8 * vi, r);
#pragma unroll
          for (int e = 0; e < 8; ++e) v[j][e] += r[e];
        }
      }
    }
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const int vi = j * nt + tid;
      if (a.H && vi < nvec) store8<RB>(a.H, t * a.ldr + 8 * vi, v[j]);
#pragma unroll
      for (int e = 0; e < 8; ++e) ss = fmaf(v[j][e], v[j][e], ss);
    }
    const float2 tot = block_sum2(ss, 0.f, red);
    const float rstd = 1.0f / sqrtf(tot.x / (float)a.C + a.rms_eps);
    float M = -INFINITY, m = INFINITY;
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const int vi = j * nt + tid;
      if (vi < nvec) {
        float g[8], b[8];
        if (a.gain) load8<false>(a.gain, 8 * vi, g);
        if (a.bias) load8<false>(a.bias, 8 * vi, b);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          float y = v[j][e] * rstd;
          if (a.gain) y *= g[e];
          if (a.bias) y += b[e];
          v[j][e] = y;
          M = fmaxf(M, fabsf(y) < INFINITY ? y : INFINITY);   // a NaN or an infinity shows as +inf
          m = fminf(m, y);
        }
      }
    }
    if (a.abits < 16) {
      const float Q = (float)((1 << a.abits) - 1);
      block_extremes(M, m, red + 64);
      const bool bad = !(M < INFINITY);
      QState qs = omq_qstate(bad ? 0.f : M, bad ? 0.f : m, 1.f, 1.f, Q, a.h_eps);
      if (tid == 0) { a.h[t] = bad ? NAN : qs.h; a.z[t] = bad ? 0 : (int32_t)qs.z; }
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const int vi = j * nt + tid;
        if (vi >= nvec) continue;
        float cd[8];
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
          float2 c2;
          const float2 w = omq_fakequant2(make_float2(v[j][e], v[j][e + 1]), qs, Q, &c2);
          v[j][e] = bad ? NAN : w.x; v[j][e + 1] = bad ? NAN : w.y;
          cd[e] = bad ? 0.f : c2.x; cd[e + 1] = bad ? 0.f : c2.y;
        }
        if (a.codes) {
          uint32_t p[2];
#pragma unroll
          for (int k = 0; k < 2; ++k)
            p[k] = (uint32_t)cd[4 * k] | ((uint32_t)cd[4 * k + 1] << 8) | ((uint32_t)cd[4 * k + 2] << 16) |
                   ((uint32_t)cd[4 * k + 3] << 24);
          *reinterpret_cast<uint2*>(a.codes + t * a.C + 8 * vi) = make_uint2(p[0], p[1]);
        }
        if (a.Xq) *reinterpret_cast<uint4*>(a.Xq + t * a.C + 8 * vi) = pack_bf16x8(v[j]);
      }
    } else {
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const int vi = j * nt + tid;
        if (vi < nvec) *reinterpret_cast<uint4*>(a.Xq + t * a.C + 8 * vi) = pack_bf16x8(v[j]);
      }
    }
    __syncthreads();                             // the reduction scratch is reused by the next row
  }
}

template <bool XB, bool RB>
omq_status norm_launch(cudaStream_t st, const NormArgs& a) {
  const int nvec = a.C / 8;
  const int V = nvec <= 1024 ? 1 : (nvec <= 2048 ? 2 : 4);
  const int nt = ((nvec + V - 1) / V + 31) / 32 * 32;
  const unsigned grid = (unsigned)(a.T < 65536 ? a.T : 65536);
  if (V == 1) rmsnorm_quant_kernel<XB, RB, 1><<<grid, nt, 0, st>>>(a);
  else if (V == 2) rmsnorm_quant_kernel<XB, RB, 2><<<grid, nt, 0, st>>>(a);
  else rmsnorm_quant_kernel<XB, RB, 4><<<grid, nt, 0, st>>>(a);
  OMQ_LAUNCH_CHECK();
  return OMQ_OK;
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
