// Quantizer to e2m1 codes with microscales, and the read-back.
//
//   a = max |x| of a group of 32 (16) columns of a row
//   by 32: s = the smallest power of two >= max(a, 2^-60) / 6,         code = e2m1(x / s)
//   by 16: r = 1 / factor, s = max(e4m3(a * (r / 6)), 2^-9),           code = e2m1(x * (r / s))
// All steps are binary32 with round to nearest even, so a code -- decided by floating-point arithmetic -- is
// reproducible.  Quotients past binary32's largest number are that number: a matrix of zeros has the factor 0 by
// max |X| / 2688, and a zero times an infinite r would be NaN.  s never is below a group's need by more than its own rounding: codes saturate at 6 only there.  Maxima
// are taken on the bit patterns of |x|, which order NaN above infinity above every number: a group that holds either
// gets the scale NaN.
//
// The transposed output (codes of X^T, groups along the rows of a column) comes from the same read.
//
// Layout: a thread holds 8 consecutive columns of RT rows as they lie in memory; 16 threads span 128 columns and 16
// such rows of threads a tile of 16 * RT rows.  RT = 8 is the unit of the transposed output; straight codes alone mostly
// take RT = 2, where more and smaller thread blocks start sooner.  A group is 4 (2) threads of a
// row: its maximum goes round them by shuffles that halve the rows as they double the threads, so that each of a
// thread's rows has its scale computed once.  Along columns a group is 4 (2) rows of threads.
// Bound: HBM, with instruction issue close behind.
#include "q4_f4.cuh"

namespace q4 {
namespace f4 {

using f8::Coming;
using f8::Eight;
using f8::Elem;

constexpr int TC = 128;                 // columns of a tile

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

__device__ __forceinline__ float at_most_largest(float v) { return v > 3.402823466e38f ? 3.402823466e38f : v; }      // (NaN stays)

// Scale byte of a group whose largest |x| has the bit pattern `a`, and what its values are multiplied with.
// r = 1 / factor, r6 = r / 6.
template <bool BY16> __device__ __forceinline__ uint32_t scale_of(uint32_t a, float r, float r6, float& inv)
{
    if (BY16) {
        uint32_t byte = __nv_cvt_float_to_fp8(__uint_as_float(a) * r6, __NV_SATFINITE, __NV_E4M3);
        byte = a > 0x7F7FFFFFu ? 0x7Fu : max(byte, 1u);
        inv = at_most_largest(__fdiv_rn(r, e4m3_value(byte)));
        return byte;
    }
    // a / 6 = (m / 1.5) 2^(e - 2): the next power of two is 2^(e - 2) where the mantissa is at most 1.5
    const uint32_t byte = ((max(a, 0x21800000u) + 0x3FFFFFu) >> 23) - 2u;
    inv = __uint_as_float((254u - byte) << 23);
    return a > 0x7F7FFFFFu ? 255u : byte;
}

// VEC: every row of X begins on a multiple of 16 bytes and cols is a multiple of 8.
template <int TYPE, int RT, bool BY16, bool VEC>
__global__ void __launch_bounds__(256, RT == 2 ? 1 : !VEC || TYPE == Q4_F32 ? 2 : 4)
quantize_kernel(const QuantizeParams p)
{
    using T = typename Elem<TYPE>::T;
    constexpr int TR = 16 * RT;                            // rows of the tile
    constexpr int NW = Eight<T>::NW;
    constexpr int GT = group_of(BY16) / 8;                 // threads (or rows of threads) of a group
    constexpr int GC = TC / group_of(BY16);                // groups of a tile's row (RT == 8: of its columns too)
    constexpr int WC = GC / 4;                             // their words
    __shared__ uint32_t scales[TR * WC];                   // [word][row] straight, then [word][column]
    __shared__ uint32_t col_max[RT == 8 ? 8 : 1][TC];      // [warp][column]: maxima, then what the values are multiplied with
    __shared__ __align__(16) uint32_t tile[RT == 8 ? TC * 16 : 4];      // [column][eight rows]

    f8::wait_for_predecessor();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int cx = threadIdx.x & 15, ry = threadIdx.x >> 4;
    const int ncb = (p.cols + TC - 1) / TC;
    const int rb = blockIdx.x / ncb, cb = blockIdx.x - rb * ncb;
    const int64_t r0 = (int64_t)rb * TR + ry * RT;             // my first row
    const int c0 = cb * TC + cx * 8;
    const int nc = min(8, max(0, p.cols - c0));
    float r = 1.0f, r6 = 1.0f;
    if (BY16) {
        if (p.factor) r = at_most_largest(__fdiv_rn(1.0f, __ldg(p.factor)));
        r6 = __fdiv_rn(r, 6.0f);
    }

    // the tile lies inside: no conditions in the loops
    const bool whole = (int64_t)(rb + 1) * TR <= p.rows && (cb + 1) * TC <= p.cols;
    Coming<VEC, T> x[RT];
    Eight<T> v[RT];
    if (whole && !p.source) {
        const T* src = static_cast<const T*>(p.X) + r0 * p.ldx + c0;
#pragma unroll
        for (int i = 0; i < RT; ++i) x[i].load(src + i * p.ldx, 8, f8::careful_at(r0 + i, p.x_rows, c0, p.cols - c0, p.cols));
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
            const int64_t at = __shfl_sync(0xFFFFFFFFu, from, (lane & 16) + i);
            x[i].load(static_cast<const T*>(p.X) + (at >= 0 ? at * p.ldx + c0 : 0), at >= 0 ? nc : 0,
                      f8::careful_at(at, p.x_rows, c0, p.cols - c0, p.cols));
        }
#pragma unroll
        for (int i = 0; i < RT; ++i) {
            const int64_t at = VEC ? 0 : __shfl_sync(0xFFFFFFFFu, from, (lane & 16) + i);
            v[i] = x[i].get(static_cast<const T*>(p.X) + at * p.ldx + c0, at >= 0 ? nc : 0);
        }
    }

    if (p.Q) {
        // maxima of my RT rows over the GT threads of my group; thread cx ends with rows base .. base + OWN - 1
        constexpr int OWN = RT >= GT ? RT / GT : 1;
        uint32_t a[RT];
#pragma unroll
        for (int i = 0; i < RT; ++i) a[i] = max_of(v[i]);
        int have = RT, base = 0;
#pragma unroll
        for (int w = GT / 2; w; w >>= 1) {
            const bool up = cx & w;
            if (have > 1) {
                have /= 2;
                base += up ? have : 0;
#pragma unroll
                for (int i = 0; i < RT / 2; ++i) {
                    if (i >= have) break;
                    const uint32_t give = up ? a[i] : a[i + have], keep = up ? a[i + have] : a[i];
                    a[i] = max(keep, __shfl_xor_sync(0xFFFFFFFFu, give, w));
                }
            } else {
                a[0] = max(a[0], __shfl_xor_sync(0xFFFFFFFFu, a[0], w));
            }
        }
        float inv[OWN];
        uint8_t* const bytes = reinterpret_cast<uint8_t*>(scales);
        const int grp = cx / GT;
#pragma unroll
        for (int i = 0; i < OWN; ++i) {
            const uint32_t b = scale_of<BY16>(a[i], r, r6, inv[i]);
            // (where a group has more threads than rows, two of them write the same)
            bytes[((grp >> 2) * TR + ry * RT + base + i) * 4 + (grp & 3)] = (uint8_t)(cb * TC + grp * group_of(BY16) < p.cols ? b : 0u);
        }
        uint8_t* dst = p.Q + r0 * p.ldq + (c0 >> 1);
#pragma unroll
        for (int i = 0; i < RT; ++i, dst += p.ldq) {
            // row i's: its bits from the top say which thread of the group has it
            int owner = 0, left = RT, at = i;
#pragma unroll
            for (int w = GT / 2; w; w >>= 1)
                if (left > 1) {
                    left /= 2;
                    if (at >= left) { owner |= w; at -= left; }
                }
            const float iv = __shfl_sync(0xFFFFFFFFu, inv[at], (lane & ~(GT - 1)) + owner);
            float y[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) y[j] = v[i].get(j) * iv;
            const uint32_t q = codes8(y);
            if (whole && p.q_vec) {
                *reinterpret_cast<uint32_t*>(dst) = q;
            } else if (r0 + i < p.rows) {
                if (nc == 8 && p.q_vec) {
                    *reinterpret_cast<uint32_t*>(dst) = q;
                } else {
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        if (2 * j < nc) dst[j] = (uint8_t)(q >> (8 * j) & (2 * j + 1 < nc ? 0xFFu : 0x0Fu));
                }
            }
        }
        __syncthreads();
        for (int i = threadIdx.x; i < TR * WC; i += 256) {
            const int64_t row = (int64_t)rb * TR + i % TR, word = (int64_t)cb * WC + i / TR;
            if (row < p.rows && word < words_of(p.cols, BY16)) p.S[word * p.lds + row] = scales[i];
        }
    }

    if (RT == 8 && p.Qt) {
        // maxima of my 8 columns over my rows and the warp's other row of threads
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
        __syncthreads();                                       // the straight scales have been written out, too
        uint8_t* const bytes = reinterpret_cast<uint8_t*>(scales);
        for (int i = threadIdx.x; i < TC * GC; i += 256) {
            const int c = i % TC, g = i / TC;                  // a group is one warp's rows, or two warps'
            constexpr int WG = 8 / GC;
            uint32_t a = col_max[RT == 8 ? g * WG : 0][c];
            if (WG == 2) a = max(a, col_max[RT == 8 ? g * WG + 1 : 0][c]);
            float iv;
            const uint32_t b = scale_of<BY16>(a, r, r6, iv);
            bytes[((g >> 2) * TC + c) * 4 + (g & 3)] = (uint8_t)((int64_t)rb * TC + g * group_of(BY16) < p.rows ? b : 0u);
            col_max[RT == 8 ? g * WG : 0][c] = __float_as_uint(iv);
        }
        __syncthreads();
        float inv[8];
        const int g = ry / GT * (GT / 2);                      // the group's first warp
#pragma unroll
        for (int j = 0; j < 8; ++j) inv[j] = __uint_as_float(col_max[RT == 8 ? g : 0][cx * 8 + j]);
        // column c's 128 codes: 16 words of eight rows, word q at q ^ (c / 8)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            float y[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) y[i] = v[RT == 8 ? i : 0].get(j) * inv[j];
            tile[RT == 8 ? (cx * 8 + j) * 16 + (ry ^ cx) : 0] = codes8(y);
        }
        __syncthreads();
        for (int i = threadIdx.x; i < TC * WC; i += 256) {
            const int c = i % TC;
            const int64_t word = (int64_t)rb * WC + i / TC;
            if (cb * TC + c < p.cols && word < words_of(p.rows, BY16)) p.St[word * p.ldst + cb * TC + c] = scales[i];
        }
        const int h = threadIdx.x & 3;                          // 32 codes of a column from row 32 h
        const int64_t rt0 = (int64_t)rb * TC + 32 * h;
        const int n = (int)min((int64_t)32, p.rows - rt0);
#pragma unroll
        for (int it = 0; it < 2; ++it) {
            const int c = it * 64 + (int)(threadIdx.x >> 2);
            if (cb * TC + c >= p.cols || n <= 0) continue;
            uint32_t w[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) w[k] = tile[RT == 8 ? c * 16 + ((4 * h + k) ^ (c >> 3)) : 0];
            uint8_t* const dst = p.Qt + (int64_t)(cb * TC + c) * p.ldqt + (rt0 >> 1);
            if (n == 32 && p.qt_vec) {
                *reinterpret_cast<uint4*>(dst) = make_uint4(w[0], w[1], w[2], w[3]);
            } else {
#pragma unroll
                for (int j = 0; j < 16; ++j)
                    if (2 * j < n) dst[j] = (uint8_t)(w[j >> 2] >> (8 * (j & 3)) & (2 * j + 1 < n ? 0xFFu : 0x0Fu));
            }
        }
    }
}

// Read-back: 16 threads span 128 columns of a row, a block 16 rows at a time and DR in all.
constexpr int DR = 64;
template <int TYPE, bool BY16, bool VEC>
__global__ void __launch_bounds__(256)
dequantize_kernel(const DequantizeParams p)
{
    using T = typename Elem<TYPE>::T;
    f8::wait_for_predecessor();
    const int cx = threadIdx.x & 15, ry = threadIdx.x >> 4;
    const int ncb = (p.cols + TC - 1) / TC;
    const int rb = blockIdx.x / ncb, cb = blockIdx.x - rb * ncb;
    const int c0 = cb * TC + cx * 8, nc = min(8, max(0, p.cols - c0));
    const float f = p.factor ? __ldg(p.factor) : 1.0f;
    uint32_t q[DR / 16], s[DR / 16];
#pragma unroll
    for (int i = 0; i < DR / 16; ++i) {
        const int64_t row = (int64_t)rb * DR + i * 16 + ry;
        q[i] = s[i] = 0;
        if (row >= p.rows || nc <= 0) continue;
        const uint8_t* src = p.Q + row * p.ldq + (c0 >> 1);
        if (nc == 8 && p.q_vec) {
            q[i] = __ldcs(reinterpret_cast<const unsigned int*>(src));
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) if (2 * j < nc) q[i] |= (uint32_t)src[j] << (8 * j);
        }
        s[i] = __ldg(p.S + (int64_t)(c0 / word_cols(BY16)) * p.lds + row) >> (8 * (c0 / group_of(BY16) % 4));
    }
#pragma unroll
    for (int i = 0; i < DR / 16; ++i) {
        const int64_t row = (int64_t)rb * DR + i * 16 + ry;
        uint32_t h[4];
        values8(q[i], h);
        const float sc = scale_value<BY16>(s[i] & 255u);
        float y[8];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float2 t = floats2(h[j]);
            y[2 * j] = t.x * sc * f;
            y[2 * j + 1] = t.y * sc * f;
        }
        Eight<T> e;
        f8::pack8(e, y);
        f8::store8<VEC, T>(static_cast<T*>(p.Y) + row * p.ldy + c0, row < p.rows ? p.cols - c0 : 0, e, cx, 16);
    }
}

template <int TYPE, bool BY16, bool VEC>
static cudaError_t launch_quantize(const QuantizeParams& p, cudaStream_t st)
{
    // column tiles vary fastest: neighbouring tiles read neighbouring pieces of the same rows
    const int64_t nc = ((int64_t)p.cols + TC - 1) / TC, t128 = nc * (((int64_t)p.rows + 127) / 128);
    // Straight codes alone: the small tiles, with more threads per SM, win for binary32 (2048 x 2048 and read back 9.4 -> 8.0 us,
    // 4096 x 4096 23.0 -> 21.6) and below two tiles per SM for 16 bits (2048 x 1024 5.8 -> 5.4; 2048 x 4096 9.8 against 10.3).
    if (p.Qt || (TYPE != Q4_F32 && t128 >= 4 * f8_pairs_of_device())) return f8::launch(quantize_kernel<TYPE, 8, BY16, VEC>, (unsigned)t128, 256, 0, st, p);
    return f8::launch(quantize_kernel<TYPE, 2, BY16, VEC>, (unsigned)(nc * (((int64_t)p.rows + 31) / 32)), 256, 0, st, p);
}
template <int TYPE>
static cudaError_t quantize_typed(const QuantizeParams& p, bool by16, cudaStream_t st)
{
    if (by16) return p.x_vec ? launch_quantize<TYPE, true, true>(p, st) : launch_quantize<TYPE, true, false>(p, st);
    return p.x_vec ? launch_quantize<TYPE, false, true>(p, st) : launch_quantize<TYPE, false, false>(p, st);
}
template <int TYPE>
static cudaError_t dequantize_typed(const DequantizeParams& p, bool by16, cudaStream_t st)
{
    const unsigned n = (unsigned)((((int64_t)p.cols + TC - 1) / TC) * (((int64_t)p.rows + DR - 1) / DR));
    if (by16) return p.y_vec ? f8::launch(dequantize_kernel<TYPE, true, true>, n, 256, 0, st, p)
                             : f8::launch(dequantize_kernel<TYPE, true, false>, n, 256, 0, st, p);
    return p.y_vec ? f8::launch(dequantize_kernel<TYPE, false, true>, n, 256, 0, st, p)
                   : f8::launch(dequantize_kernel<TYPE, false, false>, n, 256, 0, st, p);
}

}  // namespace f4

cudaError_t launch_f4_quantize(const f4::QuantizeParams& p, int x_type, bool by16, cudaStream_t st)
{
    if (x_type == Q4_F32) return f4::quantize_typed<Q4_F32>(p, by16, st);
    if (x_type == Q4_BF16) return f4::quantize_typed<Q4_BF16>(p, by16, st);
    return f4::quantize_typed<Q4_F16>(p, by16, st);
}
cudaError_t launch_f4_dequantize(const f4::DequantizeParams& p, int y_type, bool by16, cudaStream_t st)
{
    if (y_type == Q4_F32) return f4::dequantize_typed<Q4_F32>(p, by16, st);
    if (y_type == Q4_BF16) return f4::dequantize_typed<Q4_BF16>(p, by16, st);
    return f4::dequantize_typed<Q4_F16>(p, by16, st);
}

}  // namespace q4
