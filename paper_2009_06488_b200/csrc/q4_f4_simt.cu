// General kernels of the 4-bit float operators: operands of any alignment and any size.
//
// Products: 64 x 64 tiles, 4 x 4 values per thread; codes become scaled binary32 values as they are staged (a code
// times a scale is exact), and the sum over the depth is binary32.  Bound: FP32 multiply-adds.
//
// Expert layer: a warp per value, lanes along the depth.  Kernel 1: h = act(W1 x) of every pair of a token and an
// expert, in binary32; kernel 2: Out = sum over a token's pairs of w * (W2 h).  Bound: one warp reads one row of codes
// byte by byte.
#include "q4_f4.cuh"

namespace q4 {
namespace f4 {

__device__ __forceinline__ float code_value(uint32_t code)
{
    uint32_t h[4];
    values8(code, h);
    return floats2(h[0]).x;
}
// value k of a row of codes whose words of scales are [word][rows], without the factor
template <bool BY16>
__device__ __forceinline__ float value_at(const uint8_t* row, const uint32_t* words, int64_t lds, int k)
{
    const uint32_t byte = row[k >> 1], word = words[(int64_t)(k / word_cols(BY16)) * lds];
    return code_value(byte >> (4 * (k & 1)) & 15u) * scale_value<BY16>(word >> (8 * (k / group_of(BY16) % 4)) & 255u);
}

constexpr int TILE = 64, KS = 32;

template <bool BY16>
__global__ void __launch_bounds__(256)
gemm_f4_simt_kernel(const GemmParams p)
{
    __shared__ float sa[KS][TILE + 4], sb[KS][TILE + 4];
    const int e = blockIdx.z;
    int m_lo = 0, m_hi = p.M;
    if (p.E) {
        m_lo = min(max(p.starts[e], 0), p.M);
        m_hi = min(max(p.starts[e + 1], m_lo), p.M);
    }
    const int64_t brow0 = (int64_t)e * p.N;
    const float f = (p.FA ? *p.FA : 1.0f) * (p.FB ? p.FB[e] : 1.0f);
    const int n0 = blockIdx.x * TILE;
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    for (int64_t m0 = (int64_t)m_lo + (int64_t)blockIdx.y * TILE; m0 < m_hi; m0 += (int64_t)gridDim.y * TILE) {
        float acc[4][4] = {};
        for (int ks = 0; ks < p.K; ks += KS) {
            __syncthreads();
            for (int i = threadIdx.x; i < TILE * KS; i += 256) {
                const int k = i % KS, r = i / KS;
                const bool in = ks + k < p.K;
                const int64_t m = m0 + r, n = brow0 + n0 + r;
                sa[k][r] = in && m < m_hi ? value_at<BY16>(p.A + m * p.lda, p.SA + m, p.ldsa, ks + k) : 0.0f;
                sb[k][r] = in && n0 + r < p.N ? value_at<BY16>(p.Bt + n * p.ldb, p.SB + n, p.ldsb, ks + k) : 0.0f;
            }
            __syncthreads();
#pragma unroll 8
            for (int k = 0; k < KS; ++k)
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        acc[i][j] = fmaf(sa[k][ty * 4 + i], sb[k][tx * 4 + j], acc[i][j]);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int64_t m = m0 + ty * 4 + i;
                const int n = n0 + tx * 4 + j;
                if (m < m_hi && n < p.N) store_value(p.C, m * p.ldc + n, p.c_type, acc[i][j] * f);
            }
    }
}

__device__ __forceinline__ float warp_sum(float v)
{
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
    return v;
}

// grid: x over groups of 8 values of a row, y over pairs (kernel 1) or tokens (kernel 2)
template <bool BY16>
__global__ void __launch_bounds__(256)
layer_up_simt_kernel(const LayerParams p, float* hidden)
{
    const int lane = threadIdx.x & 31, h = blockIdx.x * 8 + (threadIdx.x >> 5);
    const int64_t pairs = (int64_t)p.tokens * p.topk;
    for (int64_t pair = blockIdx.y; pair < pairs; pair += gridDim.y) {
        const int e = p.ids[pair];
        if ((unsigned)e >= (unsigned)p.E || h >= p.H) continue;
        const int64_t x0 = pair / p.topk * p.ldx, r = (int64_t)e * (p.gated ? 2 : 1) * p.H + h;
        float g = 0.0f, u = 0.0f;
        for (int k = lane; k < p.D; k += 32) {
            const float x = load_value(p.X, x0 + k, p.type);
            g = fmaf(x, value_at<BY16>(p.W1 + r * p.ldw1, p.S1 + r, p.lds1, k), g);
            if (p.gated) u = fmaf(x, value_at<BY16>(p.W1 + (r + p.H) * p.ldw1, p.S1 + r + p.H, p.lds1, k), u);
        }
        const float f = p.F1 ? p.F1[e] : 1.0f;
        g = warp_sum(g) * f;
        u = p.gated ? warp_sum(u) * f : 1.0f;
        if (lane == 0) hidden[pair * p.H + h] = g / (1.0f + expf(-g)) * u;
    }
}
template <bool BY16>
__global__ void __launch_bounds__(256)
layer_down_simt_kernel(const LayerParams p, const float* hidden)
{
    const int lane = threadIdx.x & 31, d = blockIdx.x * 8 + (threadIdx.x >> 5);
    if (d >= p.D) return;
    for (int t = blockIdx.y; t < p.tokens; t += gridDim.y) {
        float out = 0.0f;
        for (int j = 0; j < p.topk; ++j) {
            const int64_t pair = (int64_t)t * p.topk + j;
            const int e = p.ids[pair];
            if ((unsigned)e >= (unsigned)p.E) continue;
            const int64_t r = (int64_t)e * p.D + d;
            float y = 0.0f;
            for (int k = lane; k < p.H; k += 32)
                y = fmaf(hidden[pair * p.H + k], value_at<BY16>(p.W2 + r * p.ldw2, p.S2 + r, p.lds2, k), y);
            out = fmaf(p.w ? p.w[pair] : 1.0f, warp_sum(y) * (p.F2 ? p.F2[e] : 1.0f), out);
        }
        if (lane == 0) store_value(p.Out, t * p.ldo + d, p.type, out);
    }
}

}  // namespace f4

using namespace f4;

cudaError_t launch_gemm_f4_simt(const f4::GemmParams& p, bool by16, cudaStream_t st)
{
    const unsigned gx = (unsigned)(((int64_t)p.N + TILE - 1) / TILE);
    const int64_t mt = ((int64_t)p.M + TILE - 1) / TILE;
    // rows of one expert are walked by the tiles of grid.y in turn: most experts own few of the M rows
    const unsigned gy = (unsigned)(p.E ? (mt < 64 ? mt : 64) : mt < 65535 ? mt : 65535);
    const dim3 grid(gx, gy, (unsigned)(p.E ? p.E : 1));
    if (by16) gemm_f4_simt_kernel<true><<<grid, 256, 0, st>>>(p);
    else gemm_f4_simt_kernel<false><<<grid, 256, 0, st>>>(p);
    count_launch();
    return cudaGetLastError();
}

cudaError_t launch_expert_layer_f4_simt(const f4::LayerParams& p, bool by16, cudaStream_t st)
{
    const int64_t pairs = (int64_t)p.tokens * p.topk;
    float* hidden = static_cast<float*>(p.ws);
    const dim3 up((unsigned)(((int64_t)p.H + 7) / 8), (unsigned)(pairs < 65535 ? pairs : 65535));
    const dim3 down((unsigned)(((int64_t)p.D + 7) / 8), (unsigned)(p.tokens < 65535 ? p.tokens : 65535));
    if (by16) {
        layer_up_simt_kernel<true><<<up, 256, 0, st>>>(p, hidden);
        layer_down_simt_kernel<true><<<down, 256, 0, st>>>(p, hidden);
    } else {
        layer_up_simt_kernel<false><<<up, 256, 0, st>>>(p, hidden);
        layer_down_simt_kernel<false><<<down, 256, 0, st>>>(p, hidden);
    }
    count_launch(2);
    return cudaGetLastError();
}

}  // namespace q4
