// Shared pieces of the 4-bit float (e2m1) kernels with microscales: formats, code conversions, launch parameters.
//
// x ~= factor * scale * code.  A group is 32 columns with a power of two as its scale (a byte, exponent + 127, 255 = NaN)
// or, BY16, 16 columns with an e4m3 number.  The scales of four neighbouring groups of a row lie in one 32-bit word, the
// first in its low byte; words are stored [word of columns][row], so that the words of a tile's rows lie together.
#pragma once

#include <cuda_fp8.h>

#include "q4_f8.cuh"

namespace q4 {
namespace f4 {

__host__ __device__ constexpr int group_of(bool by16) { return by16 ? 16 : 32; }
__host__ __device__ constexpr int word_cols(bool by16) { return by16 ? 64 : 128; }      // columns under one word of scales
__host__ __device__ inline int64_t words_of(int64_t cols, bool by16) { return (cols + word_cols(by16) - 1) / word_cols(by16); }

// Eight codes of eight values (nearest even, saturating), the first in the low four bits.
__device__ __forceinline__ uint32_t codes8(const float (&v)[8])
{
    uint32_t r;
    asm("{\n\t.reg .b8 a, b, c, d;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n\t"
        "mov.b32 %0, {a, b, c, d};\n\t}"
        : "=r"(r) : "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]));
    return r;
}
// The values of eight codes as pairs of binary16 numbers, in order.
__device__ __forceinline__ void values8(uint32_t codes, uint32_t (&h)[4])
{
    asm("{\n\t.reg .b8 a, b, c, d;\n\t"
        "mov.b32 {a, b, c, d}, %4;\n\t"
        "cvt.rn.f16x2.e2m1x2 %0, a;\n\t"
        "cvt.rn.f16x2.e2m1x2 %1, b;\n\t"
        "cvt.rn.f16x2.e2m1x2 %2, c;\n\t"
        "cvt.rn.f16x2.e2m1x2 %3, d;\n\t}"
        : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3]) : "r"(codes));
}
__device__ __forceinline__ float2 floats2(uint32_t h) { return __half22float2(*reinterpret_cast<const __half2*>(&h)); }

__device__ __forceinline__ float e4m3_value(uint32_t byte)
{
    return __half2float(__half(__nv_cvt_fp8_to_halfraw((__nv_fp8_storage_t)byte, __NV_E4M3)));
}
// 2^(byte - 127); 255 is NaN
__device__ __forceinline__ float pow2_value(uint32_t byte)
{
    return __uint_as_float(byte == 255u ? 0x7FFFFFFFu : byte ? byte << 23 : 0x00400000u);
}
template <bool BY16> __device__ __forceinline__ float scale_value(uint32_t byte)
{
    return BY16 ? e4m3_value(byte & 0x7Fu) : pow2_value(byte);
}

__device__ __forceinline__ int clamp_to(int v, int lo, int hi) { return min(max(v, lo), hi); }

// The bytes that exist of a word of scales with `cols_left` columns from its first on.
__device__ __forceinline__ uint32_t valid_bytes(int cols_left, int group)
{
    const int n = (cols_left + group - 1) / group;
    return n >= 4 ? 0xFFFFFFFFu : n <= 0 ? 0u : (1u << (8 * n)) - 1u;
}

struct QuantizeParams {
    const void* X; int64_t ldx;
    int32_t rows, cols;                // of the output
    const int32_t* source;             // NULL, or row r comes from X's row source[r] / topk (-1: zeros)
    int32_t topk, x_rows;
    const float* factor;               // BY16: device, or NULL (= 1)
    uint8_t* Q;  int64_t ldq;  uint32_t* S;  int64_t lds;    // both or neither
    uint8_t* Qt; int64_t ldqt; uint32_t* St; int64_t ldst;   // both or neither
    int32_t x_vec;                     // rows of X begin on multiples of 16 bytes and cols is a multiple of 8
    int32_t q_vec, qt_vec;             // 4-byte stores to Q / 16-byte stores to Qt are aligned
};
struct DequantizeParams {
    const uint8_t* Q; int64_t ldq;
    const uint32_t* S; int64_t lds;
    int32_t rows, cols;
    const float* factor;               // or NULL (= 1)
    void* Y; int64_t ldy;
    int32_t q_vec, y_vec;              // 4-byte loads of Q / 16-byte stores to Y are aligned
};

// One product, dense or by experts' rows.
struct GemmParams {
    const uint8_t* A;  int64_t lda; const uint32_t* SA; int64_t ldsa;
    const uint8_t* Bt; int64_t ldb; const uint32_t* SB; int64_t ldsb;
    const float* FA; const float* FB;  // one factor / one per expert, or NULL (= 1)
    void* C; int64_t ldc; int32_t c_type;
    int32_t M, N, K;
    int32_t E;                         // 0: dense
    const int32_t* starts;             // E + 1 row positions
    unsigned* status;
};

// The expert layer.
struct LayerParams {
    const void* X; int64_t ldx; int32_t type;
    int32_t tokens, topk, D, H, E, gated;
    const int32_t* ids;                // [tokens][topk]
    const float* w;                    // [tokens][topk] or NULL (= 1)
    const uint8_t* W1; int64_t ldw1; const uint32_t* S1; int64_t lds1; const float* F1;
    const uint8_t* W2; int64_t ldw2; const uint32_t* S2; int64_t lds2; const float* F2;
    void* Out; int64_t ldo;
    void* ws;
    unsigned* status;
};

template <typename T> __device__ __forceinline__ void store_value(void* base, int64_t at, int type, T v)
{
    if (type == Q4_F32) static_cast<float*>(base)[at] = v;
    else if (type == Q4_BF16) static_cast<__nv_bfloat16*>(base)[at] = __float2bfloat16_rn(v);
    else static_cast<__half*>(base)[at] = __float2half_rn(v);
}
__device__ __forceinline__ float load_value(const void* base, int64_t at, int type)
{
    if (type == Q4_F32) return static_cast<const float*>(base)[at];
    if (type == Q4_BF16) return __bfloat162float(static_cast<const __nv_bfloat16*>(base)[at]);
    return __half2float(static_cast<const __half*>(base)[at]);
}

}  // namespace f4

cudaError_t launch_f4_quantize(const f4::QuantizeParams& p, int x_type, bool by16, cudaStream_t st);
cudaError_t launch_f4_dequantize(const f4::DequantizeParams& p, int y_type, bool by16, cudaStream_t st);
cudaError_t launch_gemm_f4_simt(const f4::GemmParams& p, bool by16, cudaStream_t st);
bool        gemm_f4_few_supported(const f4::GemmParams& p);
q4_status   launch_gemm_f4_few(const f4::GemmParams& p, bool by16, cudaStream_t st);
bool        gemm_f4_pair_supported(const f4::GemmParams& p);
q4_status   launch_gemm_f4_pair(const f4::GemmParams& p, bool by16, cudaStream_t st);
bool        expert_layer_f4_stream_supported(const f4::LayerParams& p, bool by16);
q4_status   launch_expert_layer_f4_stream(const f4::LayerParams& p, bool by16, cudaStream_t st);
cudaError_t launch_expert_layer_f4_simt(const f4::LayerParams& p, bool by16, cudaStream_t st);
int64_t     expert_layer_f4_ws_bytes(int64_t pairs, int32_t D, int32_t H);

}  // namespace q4
