// C ABI of the e4m3 products with block scales and of the expert layer (declared in q4.h): argument
// validation, kernel selection, launch.  No allocation, no synchronization.
#include "q4_f8.cuh"

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

// A, Bt and their scales, C: what every product checks.  Sets the kernel's parameters.
q4_status check_product(f8::GemmF8Params& p, int64_t c_rows, int64_t sa_pitch, int64_t sb_pitch)
{
    if (p.M < 0 || p.N < 0 || p.K < 1 || !type_ok(p.c_type)) return Q4_ERR_INVALID_ARG;
    if (p.lda < p.K || p.ldb < p.K || p.ldc < p.N || p.ldsa < sa_pitch || p.ldsb < sb_pitch) return Q4_ERR_INVALID_ARG;
    if (p.M == 0 || p.N == 0 || c_rows == 0) return Q4_OK;
    if (!p.A || !p.Bt || !p.SA || !p.SB || !p.C) return Q4_ERR_INVALID_ARG;
    if (!aligned(p.SA, 4) || !aligned(p.SB, 4) || !aligned(p.C, f8::type_size(p.c_type))) return Q4_ERR_ALIGNMENT;
    return Q4_OK;
}

q4_status run_product(f8::GemmF8Params& p, const char* call, void* stream)
{
    p.status = device_status_ptr();
    if (!p.status) return Q4_ERR_CUDA;
    const int variant = kernel_variant();
    if ((variant == 0 || variant == 3) && gemm_f8_few_supported(p)) {
        log_choice(call, "few-rows kernel");
        return launch_gemm_f8_few(p, stream_of(stream));
    }
    if (variant != 1 && gemm_f8_pair_supported(p)) {
        log_choice(call, "CTA-pair tcgen05 kernel");
        return launch_gemm_f8_pair(p, stream_of(stream));
    }
    log_choice(call, "general kernel");
    return done(launch_gemm_f8_simt(p, stream_of(stream)));
}

q4_status check_rows(const ExpertRowsParams& p)
{
    if (!type_ok(p.type) || p.D < 0 || p.tokens < 0 || p.rows < 0 || p.topk < 1) return Q4_ERR_INVALID_ARG;
    if ((int64_t)p.tokens * p.topk > INT32_MAX) return Q4_ERR_RANGE;
    return Q4_OK;
}

}  // namespace

extern "C" {

q4_status q4_f8_quantize(const void* X, int32_t x_type, int64_t ldx, int32_t rows, int32_t cols,
                         const int32_t* source, int32_t topk, int32_t x_rows, int32_t flags,
                         uint8_t* Q, int64_t ldq, float* S, int64_t lds,
                         uint8_t* Qt, int64_t ldqt, float* St, int64_t ldst, void* stream)
{
    if (!type_ok(x_type) || rows < 0 || cols < 0 || ldx < cols || (flags & ~(Q4_F8_BLOCKS | Q4_F8_POW2)))
        return Q4_ERR_INVALID_ARG;
    if (source && (topk < 1 || x_rows < 0)) return Q4_ERR_INVALID_ARG;
    if (!Q != !S || !Qt != !St || (!Q && !Qt)) return Q4_ERR_INVALID_ARG;
    const bool blocks = flags & Q4_F8_BLOCKS;
    if (Q && (ldq < cols || lds < (blocks ? f8::blocks_of(cols) : rows))) return Q4_ERR_INVALID_ARG;
    if (Qt && (ldqt < rows || ldst < (blocks ? f8::blocks_of(rows) : cols))) return Q4_ERR_INVALID_ARG;
    if (rows == 0 || cols == 0) return Q4_OK;
    if (!X && !(source && x_rows == 0)) return Q4_ERR_INVALID_ARG;         // an empty matrix to pick from: every row is absent
    if (!aligned(X, f8::type_size(x_type)) || !aligned(S, 4) || !aligned(St, 4) || !aligned(source, 4))
        return Q4_ERR_ALIGNMENT;
    if (f8::blocks_of(cols) * (((int64_t)rows + 31) / 32) > INT32_MAX) return Q4_ERR_RANGE;
    f8::QuantizeParams p{};
    p.X = X; p.ldx = ldx; p.rows = rows; p.cols = cols;
    p.source = source; p.topk = source ? topk : 1; p.x_rows = source ? x_rows : rows;
    p.Q = Q; p.ldq = ldq; p.S = S; p.lds = lds;
    p.Qt = Qt; p.ldqt = ldqt; p.St = St; p.ldst = ldst;
    p.pow2 = (flags & Q4_F8_POW2) ? 1 : 0;
    p.x_vec = cols % 8 == 0 && aligned(X, 16) && ldx * (int64_t)f8::type_size(x_type) % 16 == 0;
    p.q_vec = aligned(Q, 8) && ldq % 8 == 0;
    p.qt_vec = aligned(Qt, 16) && ldqt % 16 == 0;
    return done(launch_f8_quantize(p, x_type, blocks, stream_of(stream)));
}

q4_status q4_gemm_f8(const uint8_t* A, int64_t lda, const float* SA, int64_t ldsa,
                     const uint8_t* Bt, int64_t ldb, const float* SB, int64_t ldsb, int32_t flags,
                     void* C, int32_t c_type, int64_t ldc, int32_t M, int32_t N, int32_t K, void* stream)
{
    if (flags & ~Q4_F8_B_ROWS) return Q4_ERR_INVALID_ARG;
    f8::GemmF8Params p{A, lda, SA, ldsa, Bt, ldb, SB, ldsb, flags & Q4_F8_B_ROWS ? 1 : 0, C, ldc, c_type,
                       M, N, K, f8::kDense, 1, nullptr, nullptr};
    const q4_status s = check_product(p, M, M, p.b_rows ? N : f8::blocks_of(K));
    if (s != Q4_OK || M == 0 || N == 0) return s;
    return run_product(p, "q4_gemm_f8", stream);
}

q4_status q4_gemm_f8_experts(const uint8_t* A, int64_t lda, const float* SA, int64_t ldsa,
                             const uint8_t* Bt, int64_t ldb, const float* SB, int64_t ldsb,
                             const int32_t* starts, int32_t E,
                             void* C, int32_t c_type, int64_t ldc, int32_t M, int32_t N, int32_t K, void* stream)
{
    if (E < 0) return Q4_ERR_INVALID_ARG;
    if (E > Q4_MAX_EXPERTS || (int64_t)E * N > INT32_MAX) return Q4_ERR_RANGE;
    f8::GemmF8Params p{A, lda, SA, ldsa, Bt, ldb, SB, ldsb, 0, C, ldc, c_type,
                       M, N, K, f8::kExpertRows, E, starts, nullptr};
    const q4_status s = check_product(p, E, M, f8::blocks_of(K));
    if (s != Q4_OK || M == 0 || N == 0 || E == 0) return s;
    if (!starts) return Q4_ERR_INVALID_ARG;
    if (!aligned(starts, 4)) return Q4_ERR_ALIGNMENT;
    return run_product(p, "q4_gemm_f8_experts", stream);
}

q4_status q4_gemm_f8_experts_wgrad(const uint8_t* A, int64_t lda, const float* SA, int64_t ldsa,
                                   const uint8_t* Bt, int64_t ldb, const float* SB, int64_t ldsb,
                                   const int32_t* starts, int32_t E,
                                   void* C, int32_t c_type, int64_t ldc, int32_t M, int32_t N, int32_t K, void* stream)
{
    if (E < 0) return Q4_ERR_INVALID_ARG;
    if (E > Q4_MAX_EXPERTS || (int64_t)E * M > INT32_MAX) return Q4_ERR_RANGE;
    f8::GemmF8Params p{A, lda, SA, ldsa, Bt, ldb, SB, ldsb, 1, C, ldc, c_type,
                       M, N, K, f8::kExpertDepth, E, starts, nullptr};
    const q4_status s = check_product(p, E, M, N);
    if (s != Q4_OK || M == 0 || N == 0 || E == 0) return s;
    if (!starts) return Q4_ERR_INVALID_ARG;
    if (!aligned(starts, 4)) return Q4_ERR_ALIGNMENT;
    return run_product(p, "q4_gemm_f8_experts_wgrad", stream);
}

size_t q4_expert_sort_workspace_bytes(int32_t n, int32_t E)
{
    return n < 0 || E < 1 || E > Q4_MAX_EXPERTS ? 0 : expert_sort_ws_bytes(n, E);
}

int64_t q4_expert_sort_rows(int32_t n, int32_t E, int32_t align)
{
    if (n < 0 || E < 1 || align < 1) return 0;
    return ((int64_t)n + (int64_t)(n < E ? n : E) * (align - 1)) / align * align;
}

q4_status q4_expert_sort(const int32_t* ids, int32_t n, int32_t E, int32_t align, int32_t* starts,
                         int32_t* source, int32_t rows, int32_t* slot, void* ws, size_t ws_bytes, void* stream)
{
    if (n < 0 || E < 1 || align < 1 || rows < 0) return Q4_ERR_INVALID_ARG;
    if (E > Q4_MAX_EXPERTS || align > 65536 || q4_expert_sort_rows(n, E, align) > INT32_MAX) return Q4_ERR_RANGE;
    if (rows < q4_expert_sort_rows(n, E, align)) return Q4_ERR_INVALID_ARG;
    if (!starts || (n > 0 && (!ids || !slot)) || (rows > 0 && !source)) return Q4_ERR_INVALID_ARG;
    if (!aligned(ids, 4) || !aligned(starts, 4) || !aligned(source, 4) || !aligned(slot, 4)) return Q4_ERR_ALIGNMENT;
    const size_t need = expert_sort_ws_bytes(n, E);
    if (need && (!ws || !aligned(ws, 4) || ws_bytes < need)) return Q4_ERR_WORKSPACE;
    return done(launch_expert_sort(ids, n, E, align, starts, source, rows, slot, ws, stream_of(stream)));
}

q4_status q4_expert_gather(const void* X, int64_t ldx, int32_t type, int32_t D, int32_t tokens, int32_t topk,
                           const int32_t* source, int32_t rows, const float* w, void* Xs, int64_t ldxs, void* stream)
{
    ExpertRowsParams p{type, topk, D, tokens, rows, nullptr, 0, X, ldx, nullptr, source, w, Xs, ldxs, nullptr, 0};
    const q4_status s = check_rows(p);
    if (s != Q4_OK) return s;
    if (ldx < D || ldxs < D) return Q4_ERR_INVALID_ARG;
    if (rows == 0 || D == 0) return Q4_OK;
    if ((tokens > 0 && !X) || !source || !Xs) return Q4_ERR_INVALID_ARG;
    const size_t z = f8::type_size(type);
    if (!aligned(X, z) || !aligned(Xs, z) || !aligned(source, 4) || !aligned(w, 4)) return Q4_ERR_ALIGNMENT;
    p.vec = D % 8 == 0 && aligned(X, 16) && aligned(Xs, 16) && ldx * z % 16 == 0 && ldxs * z % 16 == 0;
    return done(launch_expert_gather(p, stream_of(stream)));
}

q4_status q4_expert_combine(const void* Y, int64_t ldy, int32_t type, int32_t D, int32_t rows,
                            const int32_t* slot, const float* w, int32_t tokens, int32_t topk,
                            void* Out, int64_t ldo, void* stream)
{
    ExpertRowsParams p{type, topk, D, tokens, rows, Y, ldy, nullptr, 0, slot, nullptr, w, Out, ldo, nullptr, 0};
    const q4_status s = check_rows(p);
    if (s != Q4_OK) return s;
    if (ldy < D || ldo < D) return Q4_ERR_INVALID_ARG;
    if (tokens == 0 || D == 0) return Q4_OK;
    if ((rows > 0 && !Y) || !slot || !Out) return Q4_ERR_INVALID_ARG;
    const size_t z = f8::type_size(type);
    if (!aligned(Y, z) || !aligned(Out, z) || !aligned(slot, 4) || !aligned(w, 4)) return Q4_ERR_ALIGNMENT;
    p.vec = D % 8 == 0 && aligned(Y, 16) && aligned(Out, 16) && ldy * z % 16 == 0 && ldo * z % 16 == 0;
    return done(launch_expert_combine(p, stream_of(stream)));
}

q4_status q4_expert_combine_grad(const void* dOut, int64_t ldd, const void* Y, int64_t ldy, int32_t type, int32_t D,
                                 int32_t rows, const int32_t* source, const int32_t* slot, const float* w,
                                 int32_t tokens, int32_t topk, void* dY, int64_t lddy, float* dw, void* stream)
{
    ExpertRowsParams p{type, topk, D, tokens, rows, Y, ldy, dOut, ldd, slot, source, w, dY, lddy, dw, 0};
    const q4_status s = check_rows(p);
    if (s != Q4_OK) return s;
    if (ldd < D || ldy < D || lddy < D) return Q4_ERR_INVALID_ARG;
    if (tokens == 0 && (rows == 0 || D == 0)) return Q4_OK;
    // (rows of no values have no address; dw is 0 for every pair then)
    if ((rows > 0 && ((D > 0 && (!Y || !dY)) || !source)) || (tokens > 0 && ((D > 0 && !dOut) || !slot || !dw))) return Q4_ERR_INVALID_ARG;
    const size_t z = f8::type_size(type);
    if (!aligned(dOut, z) || !aligned(Y, z) || !aligned(dY, z) || !aligned(slot, 4) || !aligned(source, 4) ||
        !aligned(w, 4) || !aligned(dw, 4)) return Q4_ERR_ALIGNMENT;
    p.vec = D % 8 == 0 && aligned(dOut, 16) && aligned(Y, 16) && aligned(dY, 16) && ldd * z % 16 == 0 && ldy * z % 16 == 0 &&
            lddy * z % 16 == 0;
    return done(launch_expert_combine_grad(p, stream_of(stream)));
}

}  // extern "C"
