// General kernel of the e4m3 product with block scales: operands of any alignment, dense, by experts'
// rows, or by experts' depth.
//
//   C[m][n] = sum over blocks b of 128 depth values of  SA[b][m] * SB(n, b) * sum_k a(m, k) b(n, k)
//
// 64 x 64 tiles, 4 x 4 values per thread.  A block's product is summed in binary32 by itself and then
// scaled and added, so it is the tensor-core kernels' arithmetic up to the order inside a block.
// Bound: FP32 multiply-adds; the aligned problems go to the tensor-core kernels.
#include <cuda_fp8.h>

#include "q4_f8.cuh"

namespace q4 {
namespace f8 {

__device__ __forceinline__ float value_of(uint8_t code)
{
    return __half2float(__half(__nv_cvt_fp8_to_halfraw(code, __NV_E4M3)));
}

__device__ __forceinline__ void store_c(const GemmF8Params& p, int64_t row, int n, float v)
{
    const int64_t at = row * p.ldc + n;
    if (p.c_type == Q4_F32) static_cast<float*>(p.C)[at] = v;
    else if (p.c_type == Q4_BF16) static_cast<__nv_bfloat16*>(p.C)[at] = __float2bfloat16_rn(v);
    else static_cast<__half*>(p.C)[at] = __float2half_rn(v);
}

constexpr int TILE = 64, KS = 32;

__global__ void __launch_bounds__(256)
gemm_f8_simt_kernel(const GemmF8Params p)
{
    __shared__ float sa[KS][TILE + 4], sb[KS][TILE + 4];
    const int e = blockIdx.z;
    int m_lo = 0, m_hi = p.M, k_lo = 0, k_hi = p.K;
    int64_t brow0 = 0, crow0 = 0, sbrow0 = 0;
    if (p.mode == kExpertRows) {
        m_lo = min(max(p.starts[e], 0), p.M);
        m_hi = min(max(p.starts[e + 1], m_lo), p.M);
        brow0 = (int64_t)e * p.N;
        sbrow0 = e * blocks_of(p.N);
    } else if (p.mode == kExpertDepth) {
        k_lo = min(max(p.starts[e], 0), p.K);
        k_hi = min(max(p.starts[e + 1], k_lo), p.K);
        if (k_lo < k_hi) {                     // an empty segment stays empty where the depth ends inside a block
            k_lo = k_lo / BLK * BLK;
            if (k_hi != p.K) k_hi = k_hi / BLK * BLK;
        }
        crow0 = (int64_t)e * p.M;
    }
    const int n0 = blockIdx.x * TILE;
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    for (int64_t m0 = (int64_t)m_lo + (int64_t)blockIdx.y * TILE; m0 < m_hi; m0 += (int64_t)gridDim.y * TILE) {
        float acc[4][4] = {};
        for (int kb = k_lo; kb < k_hi; kb += BLK) {
            const int64_t b = kb / BLK;
            float part[4][4] = {};
            for (int ks = kb; ks < min(kb + BLK, k_hi); ks += KS) {
                __syncthreads();
                for (int i = threadIdx.x; i < TILE * KS; i += 256) {
                    const int k = i % KS, r = i / KS;
                    const bool in = ks + k < k_hi;
                    sa[k][r] = in && m0 + r < m_hi ? value_of(p.A[(m0 + r) * p.lda + ks + k]) : 0.0f;
                    sb[k][r] = in && n0 + r < p.N ? value_of(p.Bt[(brow0 + n0 + r) * p.ldb + ks + k]) : 0.0f;
                }
                __syncthreads();
#pragma unroll 8
                for (int k = 0; k < KS; ++k)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
#pragma unroll
                        for (int j = 0; j < 4; ++j)
                            part[i][j] = fmaf(sa[k][ty * 4 + i], sb[k][tx * 4 + j], part[i][j]);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int64_t m = m0 + ty * 4 + i;
                const float s = m < m_hi ? p.SA[b * p.ldsa + m] : 0.0f;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int n = n0 + tx * 4 + j;
                    if (n >= p.N) continue;
                    const float t = p.b_rows ? p.SB[b * p.ldsb + n] : p.SB[(sbrow0 + n / BLK) * p.ldsb + b];
                    acc[i][j] = fmaf(part[i][j] * t, s, acc[i][j]);
                }
            }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int64_t m = m0 + ty * 4 + i;
                const int n = n0 + tx * 4 + j;
                if (m < m_hi && n < p.N) store_c(p, crow0 + m, n, acc[i][j]);
            }
    }
}

}  // namespace f8

cudaError_t launch_gemm_f8_simt(const f8::GemmF8Params& p, cudaStream_t st)
{
    const unsigned gx = (unsigned)((p.N + f8::TILE - 1) / f8::TILE);
    const int64_t mt = ((int64_t)p.M + f8::TILE - 1) / f8::TILE;
    // rows of one expert are walked by the tiles of grid.y in turn: most experts own few of the M rows
    const unsigned gy = (unsigned)(p.mode == f8::kExpertRows ? (mt < 64 ? mt : 64) : mt < 65535 ? mt : 65535);
    f8::gemm_f8_simt_kernel<<<dim3(gx, gy, (unsigned)(p.mode == f8::kDense ? 1 : p.E)), 256, 0, st>>>(p);
    count_launch();
    return cudaGetLastError();
}

}  // namespace q4
