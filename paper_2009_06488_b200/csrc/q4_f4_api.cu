// C ABI of the 4-bit float products with microscales and of the expert layer for a few tokens (declared in q4.h):
// argument validation, kernel selection, launch.  No allocation, no synchronization.
#include "q4_f4.cuh"

namespace q4 {
unsigned* device_status_ptr();
int kernel_variant();
}

using namespace q4;

namespace {

bool type_ok(int32_t t) { return t == Q4_F32 || t == Q4_BF16 || t == Q4_F16; }
bool aligned(const void* p, size_t a) { return (uintptr_t)p % a == 0; }
cudaStream_t stream_of(void* s) { return static_cast<cudaStream_t>(s); }
q4_status done(cudaError_t e) { return e == cudaSuccess ? Q4_OK : Q4_ERR_CUDA; }
int64_t bytes_of(int64_t cols) { return (cols + 1) / 2; }
// (the kernels' indexes pass a size by less than a tile)
constexpr int32_t MOST = INT32_MAX - 512;
// A tile's depth by experts is one block's, and its end is waited for for 4e9 clk at most: 2^22 stages of 500 to 720 clk.  (A dense
// product that deep has few rows, whose depth goes to eight blocks.)
constexpr int32_t DEEPEST_BY_EXPERTS = 1 << 30;

q4_status run_product(f4::GemmParams& p, int32_t flags, const char* call, void* stream)
{
    const bool by16 = flags & Q4_F4_BY16;
    const int64_t c_rows = p.E ? p.E : p.M, b_rows = (int64_t)p.N * (p.E ? p.E : 1);
    if (p.M < 0 || p.N < 0 || p.K < 1 || !type_ok(p.c_type)) return Q4_ERR_INVALID_ARG;
    if (p.lda < bytes_of(p.K) || p.ldb < bytes_of(p.K) || p.ldc < p.N || p.ldsa < p.M || p.ldsb < b_rows) return Q4_ERR_INVALID_ARG;
    if (p.M == 0 || p.N == 0 || c_rows == 0) return Q4_OK;
    if (!p.A || !p.Bt || !p.SA || !p.SB || !p.C) return Q4_ERR_INVALID_ARG;
    if (!aligned(p.SA, 4) || !aligned(p.SB, 4) || !aligned(p.FA, 4) || !aligned(p.FB, 4) || !aligned(p.starts, 4) ||
        !aligned(p.C, f8::type_size(p.c_type))) return Q4_ERR_ALIGNMENT;
    if (p.N > MOST || p.K > MOST || (p.E && p.K > DEEPEST_BY_EXPERTS)) return Q4_ERR_RANGE;
    p.status = device_status_ptr();
    if (!p.status) return Q4_ERR_CUDA;
    const int variant = kernel_variant();
    if ((variant == 0 || variant == 3) && gemm_f4_few_supported(p)) {
        log_choice(call, "few-rows kernel");
        return launch_gemm_f4_few(p, by16, stream_of(stream));
    }
    if (variant != 1 && gemm_f4_pair_supported(p)) {
        log_choice(call, "CTA-pair tcgen05 kernel");
        return launch_gemm_f4_pair(p, by16, stream_of(stream));
    }
    log_choice(call, "general kernel");
    return done(launch_gemm_f4_simt(p, by16, stream_of(stream)));
}

}  // namespace

extern "C" {

q4_status q4_f4_quantize(const void* X, int32_t x_type, int64_t ldx, int32_t rows, int32_t cols,
                         const int32_t* source, int32_t topk, int32_t x_rows, int32_t flags, const float* factor,
                         uint8_t* Q, int64_t ldq, uint32_t* S, int64_t lds,
                         uint8_t* Qt, int64_t ldqt, uint32_t* St, int64_t ldst, void* stream)
{
    if (!type_ok(x_type) || rows < 0 || cols < 0 || ldx < cols || (flags & ~Q4_F4_BY16)) return Q4_ERR_INVALID_ARG;
    if (source && (topk < 1 || x_rows < 0)) return Q4_ERR_INVALID_ARG;
    if (!Q != !S || !Qt != !St || (!Q && !Qt)) return Q4_ERR_INVALID_ARG;
    if (factor && !(flags & Q4_F4_BY16)) return Q4_ERR_INVALID_ARG;
    if (Q && (ldq < bytes_of(cols) || lds < rows)) return Q4_ERR_INVALID_ARG;
    if (Qt && (ldqt < bytes_of(rows) || ldst < cols)) return Q4_ERR_INVALID_ARG;
    if (rows == 0 || cols == 0) return Q4_OK;
    if (!X && !(source && x_rows == 0)) return Q4_ERR_INVALID_ARG;         // an empty matrix to pick from: every row is absent
    if (!aligned(X, f8::type_size(x_type)) || !aligned(S, 4) || !aligned(St, 4) || !aligned(source, 4) || !aligned(factor, 4))
        return Q4_ERR_ALIGNMENT;
    if (rows > MOST || cols > MOST || ((int64_t)cols + 127) / 128 * (((int64_t)rows + 31) / 32) > INT32_MAX) return Q4_ERR_RANGE;
    f4::QuantizeParams p{};
    p.X = X; p.ldx = ldx; p.rows = rows; p.cols = cols;
    p.source = source; p.topk = source ? topk : 1; p.x_rows = source ? x_rows : rows;
    p.factor = factor;
    p.Q = Q; p.ldq = ldq; p.S = S; p.lds = lds;
    p.Qt = Qt; p.ldqt = ldqt; p.St = St; p.ldst = ldst;
    p.x_vec = cols % 8 == 0 && aligned(X, 16) && ldx * (int64_t)f8::type_size(x_type) % 16 == 0;
    p.q_vec = aligned(Q, 4) && ldq % 4 == 0;
    p.qt_vec = aligned(Qt, 16) && ldqt % 16 == 0;
    return done(launch_f4_quantize(p, x_type, flags & Q4_F4_BY16, stream_of(stream)));
}

q4_status q4_f4_dequantize(const uint8_t* Q, int64_t ldq, const uint32_t* S, int64_t lds, int32_t rows, int32_t cols,
                           int32_t flags, const float* factor, void* Y, int32_t y_type, int64_t ldy, void* stream)
{
    if (!type_ok(y_type) || rows < 0 || cols < 0 || ldq < bytes_of(cols) || lds < rows || ldy < cols || (flags & ~Q4_F4_BY16))
        return Q4_ERR_INVALID_ARG;
    if (rows == 0 || cols == 0) return Q4_OK;
    if (!Q || !S || !Y) return Q4_ERR_INVALID_ARG;
    if (!aligned(S, 4) || !aligned(factor, 4) || !aligned(Y, f8::type_size(y_type))) return Q4_ERR_ALIGNMENT;
    if (rows > MOST || cols > MOST || ((int64_t)cols + 127) / 128 * (((int64_t)rows + 63) / 64) > INT32_MAX) return Q4_ERR_RANGE;
    f4::DequantizeParams p{Q, ldq, S, lds, rows, cols, factor, Y, ldy, 0, 0};
    p.q_vec = aligned(Q, 4) && ldq % 4 == 0;
    p.y_vec = cols % 8 == 0 && aligned(Y, 16) && ldy * (int64_t)f8::type_size(y_type) % 16 == 0;
    return done(launch_f4_dequantize(p, y_type, flags & Q4_F4_BY16, stream_of(stream)));
}

q4_status q4_gemm_f4(const uint8_t* A, int64_t lda, const uint32_t* SA, int64_t ldsa,
                     const uint8_t* Bt, int64_t ldb, const uint32_t* SB, int64_t ldsb, int32_t flags,
                     const float* FA, const float* FB,
                     void* C, int32_t c_type, int64_t ldc, int32_t M, int32_t N, int32_t K, void* stream)
{
    if (flags & ~Q4_F4_BY16) return Q4_ERR_INVALID_ARG;
    f4::GemmParams p{A, lda, SA, ldsa, Bt, ldb, SB, ldsb, FA, FB, C, ldc, c_type, M, N, K, 0, nullptr, nullptr};
    return run_product(p, flags, "q4_gemm_f4", stream);
}

q4_status q4_gemm_f4_experts(const uint8_t* A, int64_t lda, const uint32_t* SA, int64_t ldsa,
                             const uint8_t* Bt, int64_t ldb, const uint32_t* SB, int64_t ldsb, int32_t flags,
                             const float* FA, const float* FB, const int32_t* starts, int32_t E,
                             void* C, int32_t c_type, int64_t ldc, int32_t M, int32_t N, int32_t K, void* stream)
{
    if (E < 0 || (flags & ~Q4_F4_BY16)) return Q4_ERR_INVALID_ARG;
    if (E > Q4_MAX_EXPERTS || (int64_t)E * N > INT32_MAX) return Q4_ERR_RANGE;
    if (E == 0) return Q4_OK;
    f4::GemmParams p{A, lda, SA, ldsa, Bt, ldb, SB, ldsb, FA, FB, C, ldc, c_type, M, N, K, E, starts, nullptr};
    if (M > 0 && N > 0 && !starts) return Q4_ERR_INVALID_ARG;
    return run_product(p, flags, "q4_gemm_f4_experts", stream);
}

size_t q4_expert_layer_f4_workspace_bytes(int32_t tokens, int32_t topk, int32_t D, int32_t H)
{
    if (tokens < 1 || topk < 1 || D < 1 || H < 1) return 0;
    return (size_t)expert_layer_f4_ws_bytes((int64_t)tokens * topk, D, H);
}

q4_status q4_expert_layer_f4(const void* X, int64_t ldx, int32_t type, int32_t tokens, int32_t D, int32_t H,
                             const int32_t* ids, const float* w, int32_t topk, int32_t E, int32_t flags,
                             const uint8_t* W1, int64_t ldw1, const uint32_t* S1, int64_t lds1, const float* F1,
                             const uint8_t* W2, int64_t ldw2, const uint32_t* S2, int64_t lds2, const float* F2,
                             void* Out, int64_t ldo, void* ws, size_t ws_bytes, void* stream)
{
    const int32_t up = flags & Q4_F4_GATED ? 2 : 1;
    if (!type_ok(type) || tokens < 0 || D < 1 || H < 1 || topk < 1 || E < 1 || (flags & ~(Q4_F4_BY16 | Q4_F4_GATED)))
        return Q4_ERR_INVALID_ARG;
    if (E > Q4_MAX_EXPERTS || (int64_t)E * D > INT32_MAX || (int64_t)E * up * H > INT32_MAX || D > MOST || H > MOST || (int64_t)tokens * topk > INT32_MAX)
        return Q4_ERR_RANGE;
    if (ldx < D || ldo < D || ldw1 < bytes_of(D) || ldw2 < bytes_of(H) || lds1 < (int64_t)E * up * H || lds2 < (int64_t)E * D)
        return Q4_ERR_INVALID_ARG;
    if (tokens == 0) return Q4_OK;
    if (!X || !ids || !W1 || !S1 || !W2 || !S2 || !Out) return Q4_ERR_INVALID_ARG;
    const size_t z = f8::type_size(type);
    if (!aligned(X, z) || !aligned(Out, z) || !aligned(ids, 4) || !aligned(w, 4) || !aligned(S1, 4) || !aligned(S2, 4) ||
        !aligned(F1, 4) || !aligned(F2, 4)) return Q4_ERR_ALIGNMENT;
    if (!ws || !aligned(ws, 256) || ws_bytes < q4_expert_layer_f4_workspace_bytes(tokens, topk, D, H)) return Q4_ERR_WORKSPACE;
    f4::LayerParams p{X, ldx, type, tokens, topk, D, H, E, up == 2, ids, w, W1, ldw1, S1, lds1, F1, W2, ldw2, S2, lds2, F2,
                      Out, ldo, ws, device_status_ptr()};
    if (!p.status) return Q4_ERR_CUDA;
    if (kernel_variant() != 1 && expert_layer_f4_stream_supported(p, flags & Q4_F4_BY16)) {
        log_choice("q4_expert_layer_f4", "streaming kernels");
        return launch_expert_layer_f4_stream(p, flags & Q4_F4_BY16, stream_of(stream));
    }
    log_choice("q4_expert_layer_f4", "general kernels");
    return done(launch_expert_layer_f4_simt(p, flags & Q4_F4_BY16, stream_of(stream)));
}

}  // extern "C"
