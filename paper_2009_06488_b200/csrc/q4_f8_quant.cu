// Quantizer to e4m3 codes with a scale per 128 values.
//
//   groups (default): a = max |x| over 128 consecutive columns of a row
//   blocks:           a = max |x| over 128 x 128 values
//   s = max(a, 2^-60) / 448, with pow2 rounded up to a power of two; code = e4m3(x * (1/s))
// where 1/s is 448 / max(a, 2^-60), or the exact power of two.  All steps are binary32 with round to
// nearest even, so a code -- decided by floating-point arithmetic -- is reproducible.  The floor on a
// keeps 1/s finite; a block of zeros gets codes 0.  Maxima are taken on the bit patterns of |x| as
// unsigned integers, which order NaN above infinity above every number: a block that holds either gets
// a scale that is not finite, and what is multiplied with it becomes NaN rather than a wrong number.
//
// The transposed output (codes of X^T, groups along 128 rows of a column) comes from the same read.
//
// Layout: a thread holds 8 consecutive columns of RT rows; 16 threads span the 128 columns of a block
// and 16 such rows of threads a tile of 16 * RT rows.  Straight groups alone take RT = 2 (32 rows: the
// tile's scales are one 128-byte line of S), everything else RT = 8 (a 128 x 128 tile).  A row's
// maximum is a 4-step shuffle over 16 lanes; columns' maxima go through shared memory.  The transposed
// codes are put together in a 16 KB shared tile whose 8-byte pieces are swizzled by the column, so that
// both the 8-row pieces written and the rows read back spread over all banks.
// Bound: HBM (each value is read once, each code written once).
#include "q4_f8.cuh"

namespace q4 {
namespace f8 {

__device__ __forceinline__ uint32_t abs_bits(float v) { return __float_as_uint(v) & 0x7FFFFFFFu; }

// Scale of a block whose largest |x| has the bit pattern `a`, and its inverse.
__device__ __forceinline__ void scale_of(uint32_t a, int pow2, float& s, float& inv)
{
    const float m = __uint_as_float(max(a, 0x21800000u));       // 2^-60
    s = __fdiv_rn(m, 448.0f);
    if (!pow2) {
        inv = __fdiv_rn(448.0f, m);
        return;
    }
    if (a <= 0x7F800000u) s = __uint_as_float((__float_as_uint(s) + 0x7FFFFFu) & 0xFF800000u);
    inv = __fdiv_rn(1.0f, s);
}
// two codes, `lo` in the low byte
__device__ __forceinline__ uint32_t cvt2(float lo, float hi)
{
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ uint2 cvt8(const float (&v)[8], float inv)
{
    return make_uint2(cvt2(v[0] * inv, v[1] * inv) | (cvt2(v[2] * inv, v[3] * inv) << 16),
                      cvt2(v[4] * inv, v[5] * inv) | (cvt2(v[6] * inv, v[7] * inv) << 16));
}

template <int TYPE, int RT, bool BLOCKS>
__global__ void __launch_bounds__(256)
quantize_kernel(const QuantizeParams p)
{
    using T = typename Elem<TYPE>::T;
    constexpr int TR = 16 * RT;                            // rows of the tile
    __shared__ uint32_t col_max[RT == 8 ? 8 : 1][BLK];     // per warp; blocks: [0][warp]
    __shared__ float row_scale[TR];
    __shared__ __align__(16) uint8_t tile[RT == 8 ? BLK * BLK : 16];

    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int cx = threadIdx.x & 15, ry = threadIdx.x >> 4;
    const int ncb = (p.cols + BLK - 1) / BLK;
    const int rb = blockIdx.x / ncb, cb = blockIdx.x - rb * ncb;
    const int64_t r0 = (int64_t)rb * TR + ry * RT;             // my first row
    const int c0 = cb * BLK + cx * 8;
    const int nc = min(8, max(0, p.cols - c0));

    float v[RT][8];
#pragma unroll
    for (int i = 0; i < RT; ++i) {
        int64_t r = r0 + i;
        bool on = r < p.rows;
        if (on && p.source) {
            const int s = p.source[r];
            r = s / p.topk;
            on = s >= 0 && r < p.x_rows;
        }
        load8(static_cast<const T*>(p.X) + (on ? r * p.ldx + c0 : 0), on ? nc : 0, p.x_vec, v[i]);
    }

    uint32_t block_max = 0;
    if (BLOCKS) {
#pragma unroll
        for (int i = 0; i < RT; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) block_max = max(block_max, abs_bits(v[i][j]));
        block_max = __reduce_max_sync(0xFFFFFFFFu, block_max);
        if (lane == 0) col_max[0][warp] = block_max;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < 8; ++w) block_max = max(block_max, col_max[0][w]);
    }
    float bs = 0.0f, binv = 0.0f;
    if (BLOCKS) {
        scale_of(block_max, p.pow2, bs, binv);
        if (threadIdx.x == 0) {
            if (p.S) p.S[(int64_t)rb * p.lds + cb] = bs;
            if (p.St) p.St[(int64_t)cb * p.ldst + rb] = bs;
        }
    }

    if (p.Q) {
#pragma unroll
        for (int i = 0; i < RT; ++i) {
            float inv = binv;
            if (!BLOCKS) {
                uint32_t a = 0;
#pragma unroll
                for (int j = 0; j < 8; ++j) a = max(a, abs_bits(v[i][j]));
#pragma unroll
                for (int o = 8; o; o >>= 1) a = max(a, __shfl_xor_sync(0xFFFFFFFFu, a, o));
                float s;
                scale_of(a, p.pow2, s, inv);
                if (cx == 0) row_scale[ry * RT + i] = s;
            }
            if (r0 + i < p.rows && nc > 0) {
                const uint2 q = cvt8(v[i], inv);
                uint8_t* dst = p.Q + (r0 + i) * p.ldq + c0;
                if (nc == 8 && p.q_vec) {
                    *reinterpret_cast<uint2*>(dst) = q;
                } else {
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        if (j < nc) dst[j] = (uint8_t)((j < 4 ? q.x >> (8 * j) : q.y >> (8 * (j - 4))) & 0xFFu);
                }
            }
        }
        if (!BLOCKS) {
            __syncthreads();
            const int64_t r = (int64_t)rb * TR + threadIdx.x;
            if (threadIdx.x < TR && r < p.rows) p.S[(int64_t)cb * p.lds + r] = row_scale[threadIdx.x];
        }
    }

    if (RT == 8 && p.Qt) {
        float inv[8];
        if (!BLOCKS) {
            // maxima of my 8 columns: over my rows, the warp's other row of threads, the other warps
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                uint32_t a = 0;
#pragma unroll
                for (int i = 0; i < RT; ++i) a = max(a, abs_bits(v[i][j]));
                a = max(a, __shfl_xor_sync(0xFFFFFFFFu, a, 16));
                if (lane < 16) col_max[RT == 8 ? warp : 0][cx * 8 + j] = a;
            }
            __syncthreads();
            if (threadIdx.x < BLK) {
                uint32_t a = 0;
#pragma unroll
                for (int w = 0; w < (RT == 8 ? 8 : 1); ++w) a = max(a, col_max[w][threadIdx.x]);
                float s, iv;
                scale_of(a, p.pow2, s, iv);
                const int c = cb * BLK + threadIdx.x;
                if (c < p.cols) p.St[(int64_t)rb * p.ldst + c] = s;
                col_max[0][threadIdx.x] = __float_as_uint(iv);
            }
            __syncthreads();
#pragma unroll
            for (int j = 0; j < 8; ++j) inv[j] = __uint_as_float(col_max[0][cx * 8 + j]);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) inv[j] = binv;
        }
        // column c's 128 codes: 16 pieces of 8 bytes, piece q at q ^ (c / 8)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            float t[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) t[i] = v[i < RT ? i : 0][j];
            *reinterpret_cast<uint2*>(&tile[(cx * 8 + j) * BLK + ((ry ^ cx) << 3)]) = cvt8(t, inv[j]);
        }
        __syncthreads();
        const int64_t rt0 = (int64_t)rb * BLK;
#pragma unroll
        for (int it = 0; it < 4; ++it) {
            const int u = it * 256 + threadIdx.x;
            const int c = u >> 3, h = u & 7;                    // 16 codes of column c, from row 16 h
            const int n = (int)min((int64_t)16, p.rows - (rt0 + 16 * h));
            if (cb * BLK + c >= p.cols || n <= 0) continue;
            const uint2 lo = *reinterpret_cast<const uint2*>(&tile[c * BLK + (((2 * h) ^ (c >> 3)) << 3)]);
            const uint2 hi = *reinterpret_cast<const uint2*>(&tile[c * BLK + (((2 * h + 1) ^ (c >> 3)) << 3)]);
            uint8_t* dst = p.Qt + (int64_t)(cb * BLK + c) * p.ldqt + rt0 + 16 * h;
            if (n == 16 && p.qt_vec) {
                *reinterpret_cast<uint4*>(dst) = make_uint4(lo.x, lo.y, hi.x, hi.y);
            } else {
                const uint32_t w[4] = {lo.x, lo.y, hi.x, hi.y};
#pragma unroll
                for (int j = 0; j < 16; ++j) if (j < n) dst[j] = (uint8_t)((w[j >> 2] >> (8 * (j & 3))) & 0xFFu);
            }
        }
    }
}

template <int TYPE>
static void launch_typed(const QuantizeParams& p, bool blocks, cudaStream_t st)
{
    // column blocks vary fastest: neighbouring tiles read neighbouring pieces of the same rows
    const unsigned tiles = (unsigned)(blocks_of(p.cols) * (blocks || p.Qt ? blocks_of(p.rows) : (p.rows + 31) / 32));
    if (blocks) quantize_kernel<TYPE, 8, true><<<tiles, 256, 0, st>>>(p);
    else if (p.Qt) quantize_kernel<TYPE, 8, false><<<tiles, 256, 0, st>>>(p);
    else quantize_kernel<TYPE, 2, false><<<tiles, 256, 0, st>>>(p);
}

}  // namespace f8

cudaError_t launch_f8_quantize(const f8::QuantizeParams& p, int x_type, bool blocks, cudaStream_t st)
{
    if (x_type == Q4_F32) f8::launch_typed<Q4_F32>(p, blocks, st);
    else if (x_type == Q4_BF16) f8::launch_typed<Q4_BF16>(p, blocks, st);
    else f8::launch_typed<Q4_F16>(p, blocks, st);
    count_launch();
    return cudaGetLastError();
}

}  // namespace q4
