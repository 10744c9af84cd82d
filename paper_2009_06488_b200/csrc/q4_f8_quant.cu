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
// Layout: a thread holds 8 consecutive columns of RT rows as they lie in memory; 16 threads span the 128 columns of
// a block and 16 such rows of threads a tile of 16 * RT rows.  RT = 8 is a 128 x 128 tile, the unit of blocks and of
// the transposed output; straight groups alone take RT = 2 below 128 such tiles, where more and smaller thread
// blocks start sooner (128 x 4096: 1.8 against 2.0 us; 512 x 4096: 3.0 against 2.8).  Maxima stay packed: an
// element-wise maximum over words, then shuffles that halve the rows as they double the threads, so that a row's
// scale is computed once.  Columns' maxima go through shared memory.  The transposed codes are put together in a
// 16 KB shared tile whose 8-byte pieces are swizzled by the column, so that both the 8-row pieces written and the
// rows read back spread over all banks.
// Bound: HBM (each value is read once, each code written once), with instruction issue close behind (73 % before
// whole tiles ran without conditions).  8192 x 4096 bf16: one way 17.6 us = 5.8 TB/s, both ways 25.0 us = 5.4
// TB/s; float32 27.6 and 37.4 us.  Rows that do not begin on multiples of 16 bytes (VEC false) are read in aligned pieces
// and cut: 8192 x 4092 both ways 38.8 us (value by value 47.6), float32 8192 x 4091 52.8.
#include "q4_f8.cuh"

namespace q4 {
namespace f8 {

// Maxima of |x| on the values' own bit patterns: element-wise over the words of eight values, then of
// all eight as the pattern of a binary32 number.
template <typename T> __device__ __forceinline__ uint32_t max_words(uint32_t a, uint32_t b);
template <> __device__ __forceinline__ uint32_t max_words<float>(uint32_t a, uint32_t b) { return max(a, b & 0x7FFFFFFFu); }
template <> __device__ __forceinline__ uint32_t max_words<__nv_bfloat16>(uint32_t a, uint32_t b) { return __vmaxu2(a, b & 0x7FFF7FFFu); }
template <> __device__ __forceinline__ uint32_t max_words<__half>(uint32_t a, uint32_t b) { return __vmaxu2(a, b & 0x7FFF7FFFu); }
template <typename T> __device__ __forceinline__ uint32_t pattern(const Eight<T>& e, int i) { return __float_as_uint(e.get(i)); }
template <typename T> __device__ __forceinline__ uint32_t max_of(const Eight<T>& e)
{
    Eight<T> m;
    m.w[0] = max_words<T>(0, e.w[0]);
#pragma unroll
    for (int k = 1; k < Eight<T>::NW; ++k) m.w[0] = max_words<T>(m.w[0], e.w[k]);
    return sizeof(T) == 4 ? m.w[0] : max(pattern(m, 0), pattern(m, 1));
}

// Scale of a block whose largest |x| has the bit pattern `a`, and its inverse.
__device__ __forceinline__ void scale_of(uint32_t a, int pow2, float& s, float& inv)
{
    const float m = __uint_as_float(max(a, 0x21800000u));       // 2^-60
    s = __fdiv_rn(m, 448.0f);
    if (!pow2) {
        inv = __fdiv_rn(448.0f, m);
        return;
    }
    if (a > 0x7F800000u) {                                      // NaN
        inv = s;
        return;
    }
    const uint32_t up = (__float_as_uint(s) + 0x7FFFFFu) & 0xFF800000u;
    s = __uint_as_float(up);
    inv = a == 0x7F800000u ? 0.0f : __uint_as_float(0x7F000000u - up);      // exponents of inverses add up to 254
}
// two codes, `lo` in the low byte
__device__ __forceinline__ uint32_t cvt2(float lo, float hi)
{
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ uint32_t cvt4(float a, float b, float c, float d) { return cvt2(a, b) | (cvt2(c, d) << 16); }

// VEC: every row of X begins on a multiple of 16 bytes and cols is a multiple of 8.
template <int TYPE, int RT, bool BLOCKS, bool VEC>
__global__ void __launch_bounds__(256, RT == 2 ? 1 : !VEC || TYPE == Q4_F32 ? 2 : 4)
quantize_kernel(const QuantizeParams p)
{
    using T = typename Elem<TYPE>::T;
    constexpr int TR = 16 * RT;                            // rows of the tile
    constexpr int NW = Eight<T>::NW;
    __shared__ uint32_t col_max[RT == 8 ? 8 : 1][BLK];     // per warp; blocks: [0][warp]
    __shared__ float row_scale[TR];
    __shared__ __align__(16) uint8_t tile[RT == 8 ? BLK * BLK : 16];

    wait_for_predecessor();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int cx = threadIdx.x & 15, ry = threadIdx.x >> 4;
    const int ncb = (p.cols + BLK - 1) / BLK;
    const int rb = blockIdx.x / ncb, cb = blockIdx.x - rb * ncb;
    const int64_t r0 = (int64_t)rb * TR + ry * RT;             // my first row
    const int c0 = cb * BLK + cx * 8;
    const int nc = min(8, max(0, p.cols - c0));

    // the tile lies inside: no conditions in the loops (a tenth of the kernel's instructions, and issue binds it)
    const bool whole = (int64_t)(rb + 1) * TR <= p.rows && (cb + 1) * BLK <= p.cols;
    Coming<VEC, T> x[RT];
    Eight<T> v[RT];
    if (whole && !p.source) {
        const T* src = static_cast<const T*>(p.X) + r0 * p.ldx + c0;
#pragma unroll
        for (int i = 0; i < RT; ++i) x[i].load(src + i * p.ldx, 8, careful_at(r0 + i, p.x_rows, c0, p.cols - c0, p.cols));
#pragma unroll
        for (int i = 0; i < RT; ++i) v[i] = x[i].get(src + i * p.ldx, 8);
    } else {
        int64_t from = -1;
        if (cx < RT && r0 + cx < p.rows) {
            // a thread of each row finds where it comes from
            from = r0 + cx;
            if (p.source) {
                const int s = __ldg(p.source + from);
                from = s >= 0 && s / p.topk < p.x_rows ? s / p.topk : -1;
            }
        }
#pragma unroll
        for (int i = 0; i < RT; ++i) {
            const int64_t r = __shfl_sync(0xFFFFFFFFu, from, (lane & 16) + i);
            x[i].load(static_cast<const T*>(p.X) + (r >= 0 ? r * p.ldx + c0 : 0), r >= 0 ? nc : 0,
                      careful_at(r, p.x_rows, c0, p.cols - c0, p.cols));
        }
#pragma unroll
        for (int i = 0; i < RT; ++i) {
            const int64_t r = VEC ? 0 : __shfl_sync(0xFFFFFFFFu, from, (lane & 16) + i);
            v[i] = x[i].get(static_cast<const T*>(p.X) + r * p.ldx + c0, r >= 0 ? nc : 0);
        }
    }

    float binv = 0.0f;
    if (BLOCKS) {
        uint32_t a = 0;
#pragma unroll
        for (int i = 0; i < RT; ++i) a = max(a, max_of(v[i]));
        a = __reduce_max_sync(0xFFFFFFFFu, a);
        if (lane == 0) col_max[0][warp] = a;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < 8; ++w) a = max(a, col_max[0][w]);
        float s;
        scale_of(a, p.pow2, s, binv);
        if (threadIdx.x == 0) {
            if (p.S) p.S[(int64_t)rb * p.lds + cb] = s;
            if (p.St) p.St[(int64_t)cb * p.ldst + rb] = s;
        }
    }

    if (p.Q) {
        // Maxima of my RT rows over the 16 threads that span them: each step hands half of the rows to the
        // neighbour, so that thread cx ends with row cx % RT and takes that row's scale alone (a scale costs about
        // forty instructions; every thread taking all of its rows' was a third of the kernel's).
        float inv_mine = binv;
        if (!BLOCKS) {
            uint32_t a[RT];
#pragma unroll
            for (int i = 0; i < RT; ++i) a[i] = max_of(v[i]);
#pragma unroll
            for (int w = RT / 2; w; w >>= 1) {
                const bool up = cx & w;
#pragma unroll
                for (int i = 0; i < RT / 2; ++i) {
                    if (i >= w) break;
                    const uint32_t give = up ? a[i] : a[i + w], keep = up ? a[i + w] : a[i];
                    a[i] = max(keep, __shfl_xor_sync(0xFFFFFFFFu, give, w));
                }
            }
#pragma unroll
            for (int o = RT; o < 16; o <<= 1) a[0] = max(a[0], __shfl_xor_sync(0xFFFFFFFFu, a[0], o));
            float s;
            scale_of(a[0], p.pow2, s, inv_mine);
            if (cx < RT) row_scale[ry * RT + cx] = s;
        }
        auto row_codes = [&](int i) {
            const float inv = BLOCKS ? binv : __shfl_sync(0xFFFFFFFFu, inv_mine, (lane & 16) + i);
            return make_uint2(cvt4(v[i].get(0) * inv, v[i].get(1) * inv, v[i].get(2) * inv, v[i].get(3) * inv),
                              cvt4(v[i].get(4) * inv, v[i].get(5) * inv, v[i].get(6) * inv, v[i].get(7) * inv));
        };
        uint8_t* dst = p.Q + r0 * p.ldq + c0;
        if (whole && p.q_vec) {
#pragma unroll
            for (int i = 0; i < RT; ++i, dst += p.ldq) *reinterpret_cast<uint2*>(dst) = row_codes(i);
        } else {
#pragma unroll
            for (int i = 0; i < RT; ++i, dst += p.ldq) {
                const uint2 q = row_codes(i);
                if (r0 + i >= p.rows) continue;
                if (nc == 8 && p.q_vec) {
                    *reinterpret_cast<uint2*>(dst) = q;
                } else {
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        if (j < nc) dst[j] = (uint8_t)(((j < 4 ? q.x : q.y) >> (8 * (j & 3))) & 0xFFu);
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
            Eight<T> m;
            m.zero();
#pragma unroll
            for (int i = 0; i < RT; ++i)
#pragma unroll
                for (int k = 0; k < NW; ++k) m.w[k] = max_words<T>(m.w[k], v[i].w[k]);
#pragma unroll
            for (int k = 0; k < NW; ++k) m.w[k] = max_words<T>(m.w[k], __shfl_xor_sync(0xFFFFFFFFu, m.w[k], 16));
            if (lane < 16) {
                uint4* at = reinterpret_cast<uint4*>(&col_max[RT == 8 ? warp : 0][cx * 8]);
                at[0] = make_uint4(pattern(m, 0), pattern(m, 1), pattern(m, 2), pattern(m, 3));
                at[1] = make_uint4(pattern(m, 4), pattern(m, 5), pattern(m, 6), pattern(m, 7));
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
            uint32_t q[2];
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const int i = RT == 8 ? 4 * k : 0;
                q[k] = cvt4(v[i].get(j) * inv[j], v[RT == 8 ? i + 1 : 0].get(j) * inv[j], v[RT == 8 ? i + 2 : 0].get(j) * inv[j],
                            v[RT == 8 ? i + 3 : 0].get(j) * inv[j]);
            }
            *reinterpret_cast<uint2*>(&tile[(cx * 8 + j) * BLK + ((ry ^ cx) << 3)]) = make_uint2(q[0], q[1]);
        }
        __syncthreads();
        const int h = threadIdx.x & 7;
        const int64_t rt0 = (int64_t)rb * BLK + 16 * h;
        const int n = (int)min((int64_t)16, p.rows - rt0);
        uint8_t* dst = p.Qt + (int64_t)(cb * BLK + (int)(threadIdx.x >> 3)) * p.ldqt + rt0;
#pragma unroll
        for (int it = 0; it < 4; ++it, dst += 32 * p.ldqt) {
            const int c = it * 32 + (int)(threadIdx.x >> 3);    // 16 codes of column c, from row 16 h
            if (cb * BLK + c >= p.cols || n <= 0) continue;
            // pieces 2 h and 2 h + 1 lie together, in either order
            const uint4 two = *reinterpret_cast<const uint4*>(&tile[c * BLK + ((h ^ (c >> 4)) << 4)]);
            const bool turned = (c >> 3) & 1;
            const uint2 lo = turned ? make_uint2(two.z, two.w) : make_uint2(two.x, two.y);
            const uint2 hi = turned ? make_uint2(two.x, two.y) : make_uint2(two.z, two.w);
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

template <int TYPE, bool VEC>
static cudaError_t launch_typed(const QuantizeParams& p, bool blocks, cudaStream_t st)
{
    // column blocks vary fastest: neighbouring tiles read neighbouring pieces of the same rows (RT: see above)
    const int64_t t128 = blocks_of(p.cols) * blocks_of(p.rows);
    const bool large = blocks || p.Qt || t128 >= 128;
    const unsigned tiles = (unsigned)(large ? t128 : blocks_of(p.cols) * (((int64_t)p.rows + 31) / 32));
    if (blocks) return launch(quantize_kernel<TYPE, 8, true, VEC>, tiles, 256, 0, st, p);
    if (large) return launch(quantize_kernel<TYPE, 8, false, VEC>, tiles, 256, 0, st, p);
    return launch(quantize_kernel<TYPE, 2, false, VEC>, tiles, 256, 0, st, p);
}

}  // namespace f8

cudaError_t launch_f8_quantize(const f8::QuantizeParams& p, int x_type, bool blocks, cudaStream_t st)
{
    using namespace f8;
    if (x_type == Q4_F32) return p.x_vec ? launch_typed<Q4_F32, true>(p, blocks, st) : launch_typed<Q4_F32, false>(p, blocks, st);
    if (x_type == Q4_BF16) return p.x_vec ? launch_typed<Q4_BF16, true>(p, blocks, st) : launch_typed<Q4_BF16, false>(p, blocks, st);
    return p.x_vec ? launch_typed<Q4_F16, true>(p, blocks, st) : launch_typed<Q4_F16, false>(p, blocks, st);
}

}  // namespace q4
