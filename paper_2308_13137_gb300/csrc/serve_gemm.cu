// Product of 8-bit codes with a step and zero point per token and output channel (omq_qgemm_i8).
//
// sum_k (a - za)(b - zb) is formed from the codes moved by 128 (a' = a - 128 fits a signed byte) as
//   sum a'b' - za' sum b' - zb' sum a' + K za' zb',   za' = za - 128, zb' = zb - 128,
// each sum an exact integer; the combination is taken in 64 bits and rounded once to fp32.
#include "common.cuh"

namespace {

struct QgemmArgs {
  int M, N, K;
  const uint8_t* A; int64_t lda; const float* ah; const int32_t* az;
  const uint8_t* B; int64_t ldb; const float* bh; const int32_t* bz;
  const float* bias;
  float* Cf; __nv_bfloat16* Cb; int64_t ldc;
  int32_t* status;
};

// 64 x 64 outputs per CTA, 4 x 4 per thread, 64 codes of K at a time through shared memory
__global__ void __launch_bounds__(256) qgemm_tile_kernel(const QgemmArgs p) {
  __shared__ int As[64][17], Bs[64][17];
  const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4;
  const int m0 = blockIdx.y * 64, n0 = blockIdx.x * 64;
  int acc[4][4] = {}, sa[4] = {}, sb[4] = {};
  const int lr = tid >> 2, lc = tid & 3;                 // row and 16-byte chunk this thread loads
  for (int k0 = 0; k0 < p.K; k0 += 64) {
    const int k = k0 + 16 * lc;
    uint4 a = make_uint4(0, 0, 0, 0), b = a;             // beyond the matrix: a' = b' = 0
    const uint32_t s = 0x80808080u;
    if (k < p.K && m0 + lr < p.M) {
      a = __ldg(reinterpret_cast<const uint4*>(p.A + (int64_t)(m0 + lr) * p.lda + k));
      a.x ^= s; a.y ^= s; a.z ^= s; a.w ^= s;
    }
    if (k < p.K && n0 + lr < p.N) {
      b = __ldg(reinterpret_cast<const uint4*>(p.B + (int64_t)(n0 + lr) * p.ldb + k));
      b.x ^= s; b.y ^= s; b.z ^= s; b.w ^= s;
    }
    __syncthreads();
    As[lr][4 * lc] = a.x; As[lr][4 * lc + 1] = a.y; As[lr][4 * lc + 2] = a.z; As[lr][4 * lc + 3] = a.w;
    Bs[lr][4 * lc] = b.x; Bs[lr][4 * lc + 1] = b.y; Bs[lr][4 * lc + 2] = b.z; Bs[lr][4 * lc + 3] = b.w;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < 16; ++w) {
      int av[4], bv[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) { av[i] = As[ty + 16 * i][w]; bv[i] = Bs[tx + 16 * i][w]; }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        sa[i] = __dp4a(av[i], 0x01010101, sa[i]);
        sb[i] = __dp4a(bv[i], 0x01010101, sb[i]);
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = __dp4a(av[i], bv[j], acc[i][j]);
      }
    }
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int m = m0 + ty + 16 * i;
    if (m >= p.M) continue;
    const int za = p.az ? p.az[m] - 128 : 0;
    const float ah = p.ah[m];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int n = n0 + tx + 16 * j;
      if (n >= p.N) continue;
      const int zb = p.bz ? p.bz[n] - 128 : 0;
      const long long s = (long long)acc[i][j] - (long long)za * sb[j] - (long long)zb * sa[i] +
                          (long long)p.K * za * zb;
      float y = __fmul_rn(__fmul_rn(__ll2float_rn(s), ah), p.bh[n]);
      if (p.bias) y = __fadd_rn(y, p.bias[n]);
      if (p.Cf) p.Cf[(int64_t)m * p.ldc + n] = y;
      if (p.Cb) p.Cb[(int64_t)m * p.ldc + n] = f_to_bf16(y);
    }
  }
}

}  // namespace

extern "C" omq_status omq_qgemm_i8(omq_stream_t stream, int64_t M, int64_t N, int64_t K, const uint8_t* A, int64_t lda,
                                   const float* a_h, const int32_t* a_z, const uint8_t* B, int64_t ldb, const float* b_h,
                                   const int32_t* b_z, const float* bias, float* Cf, void* Cb, int64_t ldc,
                                   int32_t* dev_status) {
  OMQ_REQUIRE(M > 0 && N > 0 && K > 0 && M < (1 << 22) && N < (1 << 30) && K <= 65536, OMQ_ERR_SHAPE);
  OMQ_REQUIRE(A && B && a_h && b_h && (Cf || Cb), OMQ_ERR_INVALID_ARG);
  OMQ_REQUIRE(lda >= K && ldb >= K && ldc >= N, OMQ_ERR_SHAPE);
  OMQ_REQUIRE(K % 16 == 0 && lda % 16 == 0 && ldb % 16 == 0 && N % 8 == 0 && ldc % 8 == 0, OMQ_ERR_ALIGN);
  OMQ_REQUIRE(omq_aligned16(A) && omq_aligned16(B) && omq_aligned16(a_h) && omq_aligned16(b_h) && omq_aligned16(a_z) &&
                  omq_aligned16(b_z) && omq_aligned16(bias) && omq_aligned16(Cf) && omq_aligned16(Cb),
              OMQ_ERR_ALIGN);
  const QgemmArgs p{(int)M, (int)N, (int)K, A, lda, a_h, a_z, B, ldb, b_h, b_z, bias, Cf, (__nv_bfloat16*)Cb, ldc, dev_status};
  const dim3 grid((unsigned)((N + 63) / 64), (unsigned)((M + 63) / 64));
  qgemm_tile_kernel<<<grid, 256, 0, (cudaStream_t)stream>>>(p);
  OMQ_LAUNCH_CHECK();
  return OMQ_OK;
}
