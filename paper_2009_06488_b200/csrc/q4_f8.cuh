// Shared pieces of the e4m3 (8-bit float) kernels with a scale per 128 values and of the
// expert-layer kernels: element types, eight-at-a-time loads and stores, launch parameters.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "q4_common.cuh"

namespace q4 {
namespace f8 {

constexpr int BLK = 128;                 // values under one scale

__host__ __device__ inline int64_t blocks_of(int64_t n) { return (n + BLK - 1) / BLK; }

template <int TYPE> struct Elem;
template <> struct Elem<Q4_F32>  { using T = float; };
template <> struct Elem<Q4_BF16> { using T = __nv_bfloat16; };
template <> struct Elem<Q4_F16>  { using T = __half; };

__device__ __forceinline__ float to_f(float v) { return v; }
__device__ __forceinline__ float to_f(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_f(__half v) { return __half2float(v); }
template <typename T> __device__ __forceinline__ T from_f(float v);
template <> __device__ __forceinline__ float from_f<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half from_f<__half>(float v) { return __float2half_rn(v); }

// Eight consecutive values as they lie in memory (NW 32-bit words), so that many of them can be in flight
// or held at a register cost of the type's own size.
template <typename T> struct Eight {
    static constexpr int NW = 2 * (int)sizeof(T);
    uint32_t w[NW];
    __device__ __forceinline__ float get(int i) const;          // i is a constant after unrolling
    __device__ __forceinline__ void zero()
    {
#pragma unroll
        for (int k = 0; k < NW; ++k) w[k] = 0;
    }
};
template <> __device__ __forceinline__ float Eight<float>::get(int i) const { return __uint_as_float(w[i]); }
template <> __device__ __forceinline__ float Eight<__nv_bfloat16>::get(int i) const
{
    return __uint_as_float(i & 1 ? w[i >> 1] & 0xFFFF0000u : w[i >> 1] << 16);
}
template <> __device__ __forceinline__ float Eight<__half>::get(int i) const
{
    const __half2 h = *reinterpret_cast<const __half2*>(&w[i >> 1]);
    return i & 1 ? __high2float(h) : __low2float(h);
}

__device__ __forceinline__ uint32_t pack2(float lo, float hi, const __nv_bfloat16*)
{
    const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ uint32_t pack2(float lo, float hi, const __half*)
{
    const __half2 h = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ void pack8(Eight<float>& e, const float (&v)[8])
{
#pragma unroll
    for (int i = 0; i < 8; ++i) e.w[i] = __float_as_uint(v[i]);
}
template <typename H> __device__ __forceinline__ void pack8(Eight<H>& e, const float (&v)[8])
{
#pragma unroll
    for (int i = 0; i < 4; ++i) e.w[i] = pack2(v[2 * i], v[2 * i + 1], (const H*)nullptr);
}

// Bytes off .. off + 15 of the 32 bytes a, b (0 <= off < 16).
__device__ __forceinline__ uint4 cut16(const uint4& a, const uint4& b, int off)
{
    const bool two = off & 8, one = off & 4;
    const uint32_t s0 = two ? a.z : a.x, s1 = two ? a.w : a.y, s2 = two ? b.x : a.z, s3 = two ? b.y : a.w, s4 = two ? b.z : b.x,
                   s5 = two ? b.w : b.y;
    const uint32_t t0 = one ? s1 : s0, t1 = one ? s2 : s1, t2 = one ? s3 : s2, t3 = one ? s4 : s3, t4 = one ? s5 : s4;
    const unsigned sh = 8u * ((unsigned)off & 3u);
    return make_uint4(__funnelshift_r(t0, t1, sh), __funnelshift_r(t1, t2, sh), __funnelshift_r(t2, t3, sh), __funnelshift_r(t3, t4, sh));
}

// Rows that need not begin on multiples of 16 bytes are read in the aligned pieces that hold their values, and cut
// afterwards.  A piece may hold bytes of a row's neighbours, never bytes before the matrix's first value or behind its
// last: `careful` values, the first and last eights of those rows, are read one by one.
__device__ __forceinline__ bool careful_at(int64_t row, int64_t rows, int c, int left, int cols)
{
    return (c == 0 && row == 0) || (left < 16 && row == rows - 1) || cols < 16;
}
template <typename T> __device__ __noinline__ uint4 piece_by_values(uintptr_t at, uintptr_t lo, uintptr_t hi)
{
    constexpr int ES = (int)sizeof(T);
    uint32_t v[16 / ES], w[4];
#pragma unroll
    for (int i = 0; i < 16 / ES; ++i) {            // all under way before one is used
        const uintptr_t from = at + ES * i;
        v[i] = 0;
        if (from >= lo && from < hi) v[i] = ES == 4 ? *reinterpret_cast<const uint32_t*>(from) : *reinterpret_cast<const uint16_t*>(from);
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) w[k] = ES == 4 ? v[k] : v[2 * k % (16 / ES)] | v[(2 * k + 1) % (16 / ES)] << 16;
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// Eight values on their way.  VEC: all eight exist (n > 0, or none) at an address that is a multiple of 16
// bytes; else n of them (0..8) anywhere.  What does not exist reads 0.
template <bool VEC, typename T> struct Coming;
template <typename T> struct Coming<true, T> {
    Eight<T> e;
    // The data is streamed: read once.
    __device__ __forceinline__ void load(const T* p, int n, bool)
    {
        e.zero();
        if (n > 0) {
#pragma unroll
            for (int k = 0; k < Eight<T>::NW / 4; ++k)
                asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];"
                             : "=r"(e.w[4 * k]), "=r"(e.w[4 * k + 1]), "=r"(e.w[4 * k + 2]), "=r"(e.w[4 * k + 3])
                             : "l"(reinterpret_cast<const uint4*>(p) + k));
        }
    }
    template <bool CAREFUL = true> __device__ __forceinline__ const Eight<T>& get(const T*, int) { return e; }
};
template <typename T> struct Coming<false, T> {
    static constexpr int G = Eight<T>::NW / 4 + 1;
    uint4 g[G];
    int off;                                       // of the values in the first piece; + 16: `careful`, not loaded yet
    __device__ __forceinline__ void load(const T* p, int n, bool careful)
    {
        off = (int)((uintptr_t)p & 15);
        const uintptr_t at = (uintptr_t)p - off;
        const int end = n > 0 && !careful ? off + n * (int)sizeof(T) : 0;
#pragma unroll
        for (int k = 0; k < G; ++k) {
            g[k] = make_uint4(0, 0, 0, 0);
            asm volatile("{\n\t.reg .pred q;\n\tsetp.gt.s32 q, %5, 0;\n\t@q ld.global.nc.v4.u32 {%0, %1, %2, %3}, [%4];\n\t}"
                         : "+r"(g[k].x), "+r"(g[k].y), "+r"(g[k].z), "+r"(g[k].w) : "l"(at + 16 * k), "r"(end - 16 * k));
        }
        if (careful && n > 0) off += 16;
    }
    // CAREFUL = false: load() was given no `careful` values.
    template <bool CAREFUL = true> __device__ __forceinline__ Eight<T> get(const T* p, int n)
    {
        Eight<T> e;
        if (CAREFUL && off > 15) {                 // here, not in load(): a call there would hold up the loads behind it
#pragma unroll
            for (int k = 0; k < G; ++k)
                if (n > 0) g[k] = piece_by_values<T>(((uintptr_t)p & ~(uintptr_t)15) + 16 * k, (uintptr_t)p, (uintptr_t)(p + n));
            off -= 16;
        }
#pragma unroll
        for (int k = 0; k + 1 < G; ++k) {
            const uint4 c = cut16(g[k], g[k + 1], off);
            e.w[4 * k] = c.x;
            e.w[4 * k + 1] = c.y;
            e.w[4 * k + 2] = c.z;
            e.w[4 * k + 3] = c.w;
        }
        if (n < 8) {
#pragma unroll
            for (int k = 0; k < Eight<T>::NW; ++k) {
                if (sizeof(T) == 4) e.w[k] = k < n ? e.w[k] : 0;
                else e.w[k] = 2 * k + 1 < n ? e.w[k] : 2 * k < n ? e.w[k] & 0xFFFFu : 0;
            }
        }
        return e;
    }
};

// The first `left` (any number; at most 8) of a lane's eight values to p.  VEC as above.  Else: called by whole warps; the
// lane is place tx of the TX (a power of two) that share a row, each with the eight values behind the lane before.
// Aligned pieces of 16 bytes are put together with the lane before; what is left at the ends is written by values.
template <bool VEC, typename T>
__device__ __forceinline__ void store8(T* p, int left, const Eight<T>& e, int tx, int TX)
{
    constexpr int NW = Eight<T>::NW, ES = (int)sizeof(T);
    if constexpr (VEC) {
        if (left > 0) {
#pragma unroll
            for (int k = 0; k < NW / 4; ++k)
                __stcs(reinterpret_cast<uint4*>(p) + k, make_uint4(e.w[4 * k], e.w[4 * k + 1], e.w[4 * k + 2], e.w[4 * k + 3]));
        }
    } else {
        const int off = (int)((uintptr_t)p & 15);
        const bool first = (tx & 31) == 0, last = ((tx + 1) & (min(TX, 32) - 1)) == 0;    // of the warp's part of the row
        uint4 s[NW / 4 + 1];
        s[0] = make_uint4(__shfl_up_sync(0xFFFFFFFFu, e.w[NW - 4], 1), __shfl_up_sync(0xFFFFFFFFu, e.w[NW - 3], 1),
                          __shfl_up_sync(0xFFFFFFFFu, e.w[NW - 2], 1), __shfl_up_sync(0xFFFFFFFFu, e.w[NW - 1], 1));
#pragma unroll
        for (int k = 0; k < NW / 4; ++k) s[k + 1] = make_uint4(e.w[4 * k], e.w[4 * k + 1], e.w[4 * k + 2], e.w[4 * k + 3]);
        unsigned done = 0;                         // pieces that are written whole, the last one by the next lane
#pragma unroll
        for (int k = 0; k < NW / 4; ++k) {
            if (min(left, 8) * ES < 16 * (k + 1) - off || (k == 0 && off && first)) continue;
            done |= 1u << k;
            const uint4 v = off ? cut16(s[k], s[k + 1], 16 - off) : s[k + 1];
            __stcs(reinterpret_cast<uint4*>((uintptr_t)p - off) + k, v);
        }
        if (ES == 2 && TX >= 32 && left - 8 * (31 - (tx & 31)) >= 16) {
            // one row, which goes on behind the warp: the 16 bytes at its ends by eight lanes
            if (off == 0) return;
            const int lane = tx & 31, k = lane & 7, from = 2 * k < 16 - off ? 0 : 31;
            const uint32_t w0 = __shfl_sync(0xFFFFFFFFu, e.w[0], from), w1 = __shfl_sync(0xFFFFFFFFu, e.w[1], from),
                           w2 = __shfl_sync(0xFFFFFFFFu, e.w[2], from), w3 = __shfl_sync(0xFFFFFFFFu, e.w[3], from);
            const uint32_t w = k & 4 ? (k & 2 ? w3 : w2) : (k & 2 ? w1 : w0);
            if (lane < 8) reinterpret_cast<uint16_t*>(p)[8 * (from - lane) + k] = (uint16_t)(w >> (16 * (k & 1)));
            return;
        }
        if (!last && min(left - 8, 8) * ES >= 16 - off) done |= 1u << (NW / 4);
        if (done == (2u << (NW / 4)) - 1u || (off == 0 && done == (1u << (NW / 4)) - 1u)) return;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (i >= left || (done >> ((off + i * ES) >> 4) & 1u)) continue;
            if (ES == 4) reinterpret_cast<uint32_t*>(p)[i] = e.w[i % NW];
            else reinterpret_cast<uint16_t*>(p)[i] = (uint16_t)(e.w[i >> 1] >> (16 * (i & 1)));
        }
    }
}

// Launch with programmatic stream serialization: the kernel's start overlaps its predecessor's end; it calls
// wait_for_predecessor() before it touches memory.
template <typename... P, typename... A>
cudaError_t launch(void (*kernel)(P...), dim3 grid, unsigned threads, size_t smem, cudaStream_t st, A... args)
{
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, P(args)...);
    count_launch();
    return e;
}
__device__ __forceinline__ void wait_for_predecessor()
{
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}

inline size_t type_size(int type) { return type == Q4_F32 ? 4 : 2; }

struct QuantizeParams {
    const void* X;
    int64_t ldx;
    int32_t rows, cols;            // of the output
    const int32_t* source;         // NULL, or row r comes from X's row source[r] / topk (-1: zeros)
    int32_t topk, x_rows;
    uint8_t* Q;  int64_t ldq;  float* S;  int64_t lds;       // both or neither
    uint8_t* Qt; int64_t ldqt; float* St; int64_t ldst;      // both or neither
    int32_t pow2;
    int32_t x_vec;                 // rows of X begin on multiples of 16 bytes and cols is a multiple of 8
    int32_t q_vec, qt_vec;         // 8-byte stores to Q / 16-byte stores to Qt are aligned
};

// One product, dense or grouped.
enum GroupMode { kDense = 0, kExpertRows = 1, kExpertDepth = 2 };
struct GemmF8Params {
    const uint8_t* A;  int64_t lda;  const float* SA; int64_t ldsa;     // SA [block of K][row of A]
    const uint8_t* Bt; int64_t ldb;  const float* SB; int64_t ldsb;     // see b_rows
    int32_t b_rows;                // SB: 0 = [block of N][block of K], 1 = [block of K][row of Bt]
    void* C; int64_t ldc; int32_t c_type;
    int32_t M, N, K;
    int32_t mode, E;
    const int32_t* starts;         // E + 1 row (kExpertRows) or depth (kExpertDepth) positions
    unsigned* status;
};

}  // namespace f8

cudaError_t launch_f8_quantize(const f8::QuantizeParams& p, int x_type, bool blocks, cudaStream_t st);
cudaError_t launch_gemm_f8_simt(const f8::GemmF8Params& p, cudaStream_t st);
int         f8_pairs_of_device();              // SMs / 2 of the current device
bool        gemm_f8_few_supported(const f8::GemmF8Params& p);
q4_status   launch_gemm_f8_few(const f8::GemmF8Params& p, cudaStream_t st);
bool        gemm_f8_pair_supported(const f8::GemmF8Params& p);
q4_status   launch_gemm_f8_pair(const f8::GemmF8Params& p, cudaStream_t st);

size_t      expert_sort_ws_bytes(int64_t n, int32_t E);
cudaError_t launch_expert_sort(const int32_t* ids, int32_t n, int32_t E, int32_t align, int32_t* starts, int32_t* source,
                               int32_t rows, int32_t* slot, void* ws, cudaStream_t st);
struct ExpertRowsParams {
    int32_t type, topk, D;
    int32_t tokens, rows;
    const void* Y; int64_t ldy;        // rows of the experts' side
    const void* X; int64_t ldx;        // rows of the tokens' side (the output's gradient, or the gather's input)
    const int32_t* slot;               // [tokens][topk] row of each pair, negative = none
    const int32_t* source;             // [rows] pair of each row, negative = none
    const float* w;                    // [tokens][topk] or NULL (= 1)
    void* out; int64_t ldo;
    float* dw;                         // [tokens][topk] (gradient only)
    int32_t vec;                       // rows begin on multiples of 16 bytes and D is a multiple of 8
};
cudaError_t launch_expert_gather(const ExpertRowsParams& p, cudaStream_t st);
cudaError_t launch_expert_combine(const ExpertRowsParams& p, cudaStream_t st);
cudaError_t launch_expert_combine_grad(const ExpertRowsParams& p, cudaStream_t st);

}  // namespace q4
