// e4m3 product with block scales for few rows of A (tokens being decoded): every weight is read once,
// straight from memory into the registers of warp-level matrix instructions.
//
//   C[m][n] = sum over blocks b of 128 depth values of  SA[b][m] * SB(n, b) * sum_k a(m, k) b(n, k)
//
// The matrix instruction (16 x 8 x 32) has Bt's rows as its 16 and the rows of A as its 8.  A block of 8 warps
// owns 16 * R rows of Bt; each warp takes every eighth depth block and keeps scaled binary32 sums, which are
// added over the warps, in order, through shared memory.  The order of depth values inside a block is
// free as long as both operands share it: lane (g, t) takes the 32 bytes t * 32 .. of the rows it
// needs, so a quad of lanes reads a row's 128 bytes, and no operand passes through shared memory.
// Bound: HBM.  The tensor memory path would first stage the same bytes in shared memory and drain a 128-row
// accumulator per block for a handful of rows.
#include "q4_f8.cuh"

namespace q4 {
namespace f8 {

constexpr int NWARP = 8;

struct Chunk { uint4 lo, hi; };           // 32 consecutive depth values

// Depth values x .. x + 31 of a row; those at or past `end` read 0 (the bytes may hold anything).
__device__ __forceinline__ Chunk load_chunk(const uint8_t* row, int x, int end, bool on)
{
    Chunk c;
    c.lo = c.hi = make_uint4(0, 0, 0, 0);
    if (!on) return c;
    if (x < end) c.lo = __ldg(reinterpret_cast<const uint4*>(row + x));
    if (x + 16 < end) c.hi = __ldg(reinterpret_cast<const uint4*>(row + x + 16));
    return c;
}
__device__ __forceinline__ void mask_word(uint32_t& w, int valid)        // valid bytes of a word
{
    if (valid <= 0) w = 0;
    else if (valid < 4) w &= (1u << (8 * valid)) - 1u;
}
__device__ __forceinline__ void mask_chunk(Chunk& c, int valid)
{
    mask_word(c.lo.x, valid);      mask_word(c.lo.y, valid - 4);  mask_word(c.lo.z, valid - 8);  mask_word(c.lo.w, valid - 12);
    mask_word(c.hi.x, valid - 16); mask_word(c.hi.y, valid - 20); mask_word(c.hi.z, valid - 24); mask_word(c.hi.w, valid - 28);
}
__device__ __forceinline__ void mma_e4m3(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k32.row.col.f32.e4m3.e4m3.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
                 "{%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// R: groups of 16 rows of Bt per block; NT: groups of 8 rows of A per pass.
template <int R, int NT>
__global__ void __launch_bounds__(NWARP * 32, R == 2 ? 2 : 3)
gemm_f8_few_kernel(const GemmF8Params p)
{
    constexpr int NB = 16 * R, MB = 8 * NT;
    __shared__ float part[NWARP][MB][NB + 4];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
    const int n0 = blockIdx.x * NB, e = blockIdx.y;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    int m_lo = 0, m_hi = p.M;
    int64_t brow = n0, sbrow = n0 / BLK;
    if (p.mode == kExpertRows) {
        m_lo = min(max(p.starts[e], 0), p.M);
        m_hi = min(max(p.starts[e + 1], m_lo), p.M);
        brow += (int64_t)e * p.N;
        sbrow += e * blocks_of(p.N);
    }
    const int nkb = (p.K + BLK - 1) / BLK;
    const int rows_n = min(NB, p.N - n0);
    const uint8_t* wrow = p.Bt + (brow + g) * p.ldb + t * 32;

    for (int m0 = m_lo; m0 < m_hi; m0 += MB) {
        const int rows_m = min(MB, m_hi - m0);
        float acc[R][NT][4] = {};
        const uint8_t* arow = p.A + (int64_t)(m0 + g) * p.lda + t * 32;
#pragma unroll (R * NT == 1 ? 2 : 1)
        for (int b = warp; b < nkb; b += NWARP) {
            const int x = b * BLK, left = p.K - x - t * 32;       // depth values left from my first
            Chunk w[R][2];
#pragma unroll
            for (int r = 0; r < R; ++r)
#pragma unroll
                for (int h = 0; h < 2; ++h)
                    w[r][h] = load_chunk(wrow + (int64_t)(16 * r + 8 * h) * p.ldb + x, 0, left, 16 * r + 8 * h + g < rows_n);
            Chunk a[NT];
            float sa[NT][2], sb[R][2];
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                a[j] = load_chunk(arow + (int64_t)(8 * j) * p.lda + x, 0, left, 8 * j + g < rows_m);
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    const int m = 8 * j + 2 * t + c;
                    sa[j][c] = m < rows_m ? __ldg(p.SA + b * p.ldsa + m0 + m) : 0.0f;
                }
            }
#pragma unroll
            for (int r = 0; r < R; ++r)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int n = 16 * r + 8 * h + g;
                    sb[r][h] = n >= rows_n ? 0.0f : p.b_rows ? __ldg(p.SB + b * p.ldsb + n0 + n) : __ldg(p.SB + sbrow * p.ldsb + b);
                }
            if (x + BLK > p.K) {
#pragma unroll
                for (int r = 0; r < R; ++r) { mask_chunk(w[r][0], left); mask_chunk(w[r][1], left); }
#pragma unroll
                for (int j = 0; j < NT; ++j) mask_chunk(a[j], left);
            }
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                if (8 * j >= rows_m) break;
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    float d[4] = {};
                    const Chunk& u = w[r][0];
                    const Chunk& v = w[r][1];
                    mma_e4m3(d, u.lo.x, v.lo.x, u.lo.y, v.lo.y, a[j].lo.x, a[j].lo.y);
                    mma_e4m3(d, u.lo.z, v.lo.z, u.lo.w, v.lo.w, a[j].lo.z, a[j].lo.w);
                    mma_e4m3(d, u.hi.x, v.hi.x, u.hi.y, v.hi.y, a[j].hi.x, a[j].hi.y);
                    mma_e4m3(d, u.hi.z, v.hi.z, u.hi.w, v.hi.w, a[j].hi.z, a[j].hi.w);
#pragma unroll
                    for (int i = 0; i < 4; ++i) acc[r][j][i] = fmaf(d[i] * sb[r][i >> 1], sa[j][i & 1], acc[r][j][i]);
                }
            }
        }
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int r = 0; r < R; ++r)
#pragma unroll
                for (int i = 0; i < 4; ++i) part[warp][8 * j + 2 * t + (i & 1)][16 * r + 8 * (i >> 1) + g] = acc[r][j][i];
        __syncthreads();
        for (int u = threadIdx.x; u < rows_m * NB; u += NWARP * 32) {
            const int m = u / NB, n = u % NB;
            if (n >= rows_n) continue;
            float v = 0.0f;
#pragma unroll
            for (int k = 0; k < NWARP; ++k) v += part[k][m][n];
            const int64_t at = (int64_t)(m0 + m) * p.ldc + n0 + n;
            if (p.c_type == Q4_F32) static_cast<float*>(p.C)[at] = v;
            else if (p.c_type == Q4_BF16) static_cast<__nv_bfloat16*>(p.C)[at] = __float2bfloat16_rn(v);
            else static_cast<__half*>(p.C)[at] = __float2half_rn(v);
        }
        __syncthreads();
    }
}

template <int R, int NT>
static q4_status launch_few(const GemmF8Params& p, cudaStream_t st)
{
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)((p.N + 16 * R - 1) / (16 * R)), (unsigned)(p.mode == kExpertRows ? p.E : 1));
    cfg.blockDim = dim3(NWARP * 32);
    cfg.stream = st;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, gemm_f8_few_kernel<R, NT>, p);
    count_launch();
    return e == cudaSuccess ? Q4_OK : Q4_ERR_CUDA;
}

}  // namespace f8

using namespace f8;

bool gemm_f8_few_supported(const GemmF8Params& g)
{
    if ((uintptr_t)g.A % 16 || (uintptr_t)g.Bt % 16 || g.lda % 16 || g.ldb % 16) return false;
    return g.mode == kExpertRows ? g.M <= 8 * (int64_t)g.E : g.mode == kDense && g.M <= 16;
}

q4_status launch_gemm_f8_few(const GemmF8Params& p, cudaStream_t st)
{
    if (p.mode == kExpertRows) return launch_few<2, 2>(p, st);
    return p.M <= 8 ? launch_few<1, 1>(p, st) : launch_few<1, 2>(p, st);
}

}  // namespace q4
