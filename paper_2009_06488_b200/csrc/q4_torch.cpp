// Argument marshalling of the e4m3, 4-bit float and expert-layer calls for torch tensors: checks types, shapes, strides and
// devices, takes pointers and pitches, and calls the C ABI on the tensors' device and its current stream.
// The same in Python took 3 to 4 us of a call whose kernel may take two; this takes about half of one.
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <sstream>
#include <stdexcept>
#include <string>

#include "q4.h"

namespace {

struct Error {
    PyObject* type;
    std::string text;
};

template <typename... A> [[noreturn]] void fail(PyObject* type, const A&... a)
{
    std::ostringstream s;
    (s << ... << a);
    throw Error{type, s.str()};
}

const at::Tensor& tensor(PyObject* o, const char* name)
{
    if (!THPVariable_Check(o)) fail(PyExc_TypeError, name, " must be a tensor");
    return THPVariable_Unpack(o);
}
const at::Tensor* optional(PyObject* o, const char* name) { return o == Py_None ? nullptr : &tensor(o, name); }

int64_t integer(PyObject* o)
{
    const int64_t v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) throw Error{nullptr, ""};
    return v;
}
int32_t int32(PyObject* o, const char* name)
{
    const int64_t v = integer(o);
    if (v < INT32_MIN || v > INT32_MAX) fail(PyExc_ValueError, name, " does not fit 32 bits");
    return (int32_t)v;
}
int32_t int32(int64_t v, const char* name)
{
    if (v > INT32_MAX) fail(PyExc_ValueError, name, " does not fit 32 bits");
    return (int32_t)v;
}

// The CUDA device that all of the tensors are on.
template <typename... T> c10::Device device_of(const at::Tensor& first, const T*... others)
{
    if (!first.is_cuda()) fail(PyExc_ValueError, "CUDA tensors are needed");
    const c10::Device d = first.device();
    (void)((others == nullptr || others->device() == d ||
            (fail(PyExc_ValueError, "tensors on ", d.str(), " and ", others->device().str()), true)) && ...);
    return d;
}

enum Kind { kCode, kFloat, kReal };
bool is(const at::Tensor& t, Kind k)
{
    const auto s = t.scalar_type();
    if (k == kCode) return s == at::kFloat8_e4m3fn || s == at::kByte;
    return s == at::kFloat || (k == kReal && (s == at::kBFloat16 || s == at::kHalf));
}
int32_t type_of(const at::Tensor& t)
{
    return t.scalar_type() == at::kFloat ? Q4_F32 : t.scalar_type() == at::kBFloat16 ? Q4_BF16 : Q4_F16;
}

// Row pitch, in elements, of a tensor of at least rows x cols elements with contiguous rows.
int64_t pitch(const at::Tensor& t, const char* name, Kind kind, int64_t rows, int64_t cols)
{
    if (!is(t, kind))
        fail(PyExc_TypeError, name, " must be ", kind == kCode ? "float8_e4m3fn or uint8" : kind == kFloat ? "float32" : "float32, bfloat16 or float16");
    if (t.dim() != 2 || t.size(0) < rows || t.size(1) < cols)
        fail(PyExc_ValueError, name, " must be 2-D and at least ", rows, " x ", cols);
    if (t.stride(1) != 1 && t.size(1) > 1) fail(PyExc_ValueError, name, " must have contiguous rows");
    return t.size(0) > 1 ? t.stride(0) : std::max(t.stride(0), t.size(1));
}

template <typename T = int32_t>
T* flat(const at::Tensor* t, const char* name, at::ScalarType type, int64_t n)
{
    if (!t) return nullptr;
    if (t->scalar_type() != type) fail(PyExc_TypeError, name, " must be ", type == at::kInt ? "int32" : "float32");
    if (!t->is_contiguous() || t->numel() < n) fail(PyExc_ValueError, name, " must be contiguous and hold at least ", n, " elements");
    return static_cast<T*>(t->data_ptr());
}

int64_t blocks(int64_t n) { return (n + 127) / 128; }
uint8_t* bytes(const at::Tensor* t) { return t ? static_cast<uint8_t*>(t->data_ptr()) : nullptr; }
float* floats(const at::Tensor* t) { return t ? static_cast<float*>(t->data_ptr()) : nullptr; }

// Runs a call on the tensors' device and its current stream.
template <typename F> PyObject* on(c10::Device d, F&& call)
{
    const c10::cuda::CUDAGuard guard(d);
    return PyLong_FromLong(call((void*)c10::cuda::getCurrentCUDAStream(d.index()).stream()));
}

// Every entry: a fixed number of positional arguments; C++ exceptions become Python's.
template <int N, typename F> PyObject* entry(PyObject* const* a, Py_ssize_t n, F&& body)
{
    try {
        if (n != N) fail(PyExc_TypeError, "expected ", N, " arguments");
        return body(a);
    } catch (const Error& e) {
        if (e.type) PyErr_SetString(e.type, e.text.c_str());
    } catch (const std::exception& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
    } catch (...) {
        PyErr_SetString(PyExc_RuntimeError, "unknown C++ exception");
    }
    return nullptr;
}

// X, Q, S, Qt, St, source, topk, flags
PyObject* f8_quantize(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    return entry<8>(a, n, [](PyObject* const* a) {
        const at::Tensor& X = tensor(a[0], "X");
        const at::Tensor *Q = optional(a[1], "Q"), *S = optional(a[2], "S"), *Qt = optional(a[3], "Qt"), *St = optional(a[4], "St");
        const at::Tensor* source = optional(a[5], "source");
        const int32_t topk = int32(a[6], "topk"), flags = int32(a[7], "flags");
        const c10::Device d = device_of(X, Q, S, Qt, St, source);
        if (!Q != !S || !Qt != !St || (!Q && !Qt))
            fail(PyExc_ValueError, "codes come with their scales: give Q and S, Qt and St, or both pairs");
        const int64_t ldx = pitch(X, "X", kReal, 0, 0), x_rows = X.size(0), cols = X.size(1);
        const int64_t rows = source ? source->numel() : x_rows;
        const bool bl = flags & Q4_F8_BLOCKS;
        int64_t ldq = 0, lds = 0, ldqt = 0, ldst = 0;
        if (Q) {
            ldq = pitch(*Q, "Q", kCode, rows, cols);
            lds = bl ? pitch(*S, "S", kFloat, blocks(rows), blocks(cols)) : pitch(*S, "S", kFloat, blocks(cols), rows);
        }
        if (Qt) {
            ldqt = pitch(*Qt, "Qt", kCode, cols, rows);
            ldst = bl ? pitch(*St, "St", kFloat, blocks(cols), blocks(rows)) : pitch(*St, "St", kFloat, blocks(rows), cols);
        }
        const int32_t* src = flat(source, "source", at::kInt, rows);
        return on(d, [&](void* st) {
            return q4_f8_quantize(X.data_ptr(), type_of(X), ldx, int32(rows, "rows"), int32(cols, "cols"), src, topk,
                                  int32(x_rows, "rows of X"), flags, bytes(Q), ldq, floats(S), lds, bytes(Qt), ldqt, floats(St), ldst, st);
        });
    });
}

// A, SA, Bt, SB, C, M, N, K, flags
PyObject* gemm_f8(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    return entry<9>(a, n, [](PyObject* const* a) {
        const at::Tensor &A = tensor(a[0], "A"), &SA = tensor(a[1], "SA"), &B = tensor(a[2], "Bt"), &SB = tensor(a[3], "SB"), &C = tensor(a[4], "C");
        const int32_t M = int32(a[5], "M"), N = int32(a[6], "N"), K = int32(a[7], "K"), flags = int32(a[8], "flags");
        const c10::Device d = device_of(A, &SA, &B, &SB, &C);
        const int64_t kb = blocks(K);
        const int64_t lda = pitch(A, "A", kCode, M, K), ldb = pitch(B, "Bt", kCode, N, K), ldc = pitch(C, "C", kReal, M, N);
        const int64_t ldsa = pitch(SA, "SA", kFloat, kb, M);
        const int64_t ldsb = flags & Q4_F8_B_ROWS ? pitch(SB, "SB", kFloat, kb, N) : pitch(SB, "SB", kFloat, blocks(N), kb);
        return on(d, [&](void* st) {
            return q4_gemm_f8(bytes(&A), lda, floats(&SA), ldsa, bytes(&B), ldb, floats(&SB), ldsb, flags, C.data_ptr(), type_of(C),
                              ldc, M, N, K, st);
        });
    });
}

// A, SA, Bt, SB, starts, C, M, N, K, weight gradient
PyObject* gemm_f8_experts(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    return entry<10>(a, n, [](PyObject* const* a) {
        const at::Tensor &A = tensor(a[0], "A"), &SA = tensor(a[1], "SA"), &B = tensor(a[2], "Bt"), &SB = tensor(a[3], "SB"),
                         &starts = tensor(a[4], "starts"), &C = tensor(a[5], "C");
        const int32_t M = int32(a[6], "M"), N = int32(a[7], "N"), K = int32(a[8], "K");
        const bool wgrad = integer(a[9]) != 0;
        const c10::Device d = device_of(A, &SA, &B, &SB, &starts, &C);
        const int64_t E = starts.numel() - 1, kb = blocks(K);
        const int64_t lda = pitch(A, "A", kCode, M, K), ldb = pitch(B, "Bt", kCode, wgrad ? N : E * N, K);
        const int64_t ldc = pitch(C, "C", kReal, wgrad ? E * M : M, N), ldsa = pitch(SA, "SA", kFloat, kb, M);
        const int64_t ldsb = wgrad ? pitch(SB, "SB", kFloat, kb, N) : pitch(SB, "SB", kFloat, E * blocks(N), kb);
        const int32_t* at = flat(&starts, "starts", at::kInt, 1);
        return on(d, [&](void* st) {
            return (wgrad ? q4_gemm_f8_experts_wgrad : q4_gemm_f8_experts)(bytes(&A), lda, floats(&SA), ldsa, bytes(&B), ldb, floats(&SB), ldsb,
                                                                           at, int32(E, "experts"), C.data_ptr(), type_of(C), ldc, M, N, K, st);
        });
    });
}

// ids, E, align, starts, source, slot, ws
PyObject* expert_sort(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    return entry<7>(a, n, [](PyObject* const* a) {
        const at::Tensor &ids = tensor(a[0], "ids"), &starts = tensor(a[3], "starts"), &source = tensor(a[4], "source"), &slot = tensor(a[5], "slot");
        const int32_t E = int32(a[1], "E"), align = int32(a[2], "align");
        const at::Tensor* ws = optional(a[6], "ws");
        const c10::Device d = device_of(ids, &starts, &source, &slot, ws);
        if (ws && !ws->is_contiguous()) fail(PyExc_ValueError, "ws must be contiguous");
        const int64_t pairs = ids.numel();
        const int32_t* i = flat(&ids, "ids", at::kInt, 0);
        int32_t *s = flat(&starts, "starts", at::kInt, (int64_t)E + 1), *src = flat(&source, "source", at::kInt, 0), *sl = flat(&slot, "slot", at::kInt, pairs);
        return on(d, [&](void* st) {
            return q4_expert_sort(i, int32(pairs, "pairs"), E, align, s, src, int32(source.numel(), "rows"), sl, ws ? ws->data_ptr() : nullptr,
                                  ws ? (size_t)ws->numel() * ws->element_size() : 0, st);
        });
    });
}

void same_rows(const at::Tensor& first, const at::Tensor& other)
{
    if (other.scalar_type() != first.scalar_type() || other.dim() != 2 || other.size(1) != first.size(1))
        fail(PyExc_ValueError, "rows of one type and width are needed");
}

// X, source, topk, Xs, w
PyObject* expert_gather(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    return entry<5>(a, n, [](PyObject* const* a) {
        const at::Tensor &X = tensor(a[0], "X"), &source = tensor(a[1], "source"), &Xs = tensor(a[3], "Xs");
        const int32_t topk = int32(a[2], "topk");
        const at::Tensor* w = optional(a[4], "w");
        const c10::Device d = device_of(X, &source, &Xs, w);
        const int64_t ldx = pitch(X, "X", kReal, 0, 0), rows = source.numel(), ldxs = pitch(Xs, "Xs", kReal, rows, X.size(1));
        same_rows(X, Xs);
        const int32_t* src = flat(&source, "source", at::kInt, rows);
        const float* pw = flat<float>(w, "w", at::kFloat, X.size(0) * topk);
        return on(d, [&](void* st) {
            return q4_expert_gather(X.data_ptr(), ldx, type_of(X), int32(X.size(1), "width"), int32(X.size(0), "tokens"), topk, src,
                                    int32(rows, "rows"), pw, Xs.data_ptr(), ldxs, st);
        });
    });
}

// Y, slot, w, Out
PyObject* expert_combine(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    return entry<4>(a, n, [](PyObject* const* a) {
        const at::Tensor &Y = tensor(a[0], "Y"), &slot = tensor(a[1], "slot"), &Out = tensor(a[3], "Out");
        const at::Tensor* w = optional(a[2], "w");
        const c10::Device d = device_of(Y, &slot, w, &Out);
        if (slot.dim() != 2) fail(PyExc_ValueError, "slot must be [tokens, topk]");
        const int64_t tokens = slot.size(0), topk = slot.size(1);
        const int64_t ldy = pitch(Y, "Y", kReal, 0, 0), ldo = pitch(Out, "Out", kReal, tokens, Y.size(1));
        same_rows(Y, Out);
        const int32_t* sl = flat(&slot, "slot", at::kInt, 0);
        const float* pw = flat<float>(w, "w", at::kFloat, tokens * topk);
        return on(d, [&](void* st) {
            return q4_expert_combine(Y.data_ptr(), ldy, type_of(Y), int32(Y.size(1), "width"), int32(Y.size(0), "rows"), sl, pw,
                                     int32(tokens, "tokens"), int32(topk, "topk"), Out.data_ptr(), ldo, st);
        });
    });
}

// dOut, Y, slot, w, source, dY, dw
PyObject* expert_combine_grad(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    return entry<7>(a, n, [](PyObject* const* a) {
        const at::Tensor &G = tensor(a[0], "dOut"), &Y = tensor(a[1], "Y"), &slot = tensor(a[2], "slot"), &source = tensor(a[4], "source"),
                         &dY = tensor(a[5], "dY"), &dw = tensor(a[6], "dw");
        const at::Tensor* w = optional(a[3], "w");
        const c10::Device d = device_of(G, &Y, &slot, w, &source, &dY, &dw);
        if (slot.dim() != 2) fail(PyExc_ValueError, "slot must be [tokens, topk]");
        const int64_t tokens = slot.size(0), topk = slot.size(1), ldy = pitch(Y, "Y", kReal, 0, 0), rows = Y.size(0);
        const int64_t ldg = pitch(G, "dOut", kReal, tokens, Y.size(1)), lddy = pitch(dY, "dY", kReal, rows, Y.size(1));
        same_rows(Y, G);
        same_rows(Y, dY);
        const int32_t *src = flat(&source, "source", at::kInt, rows), *sl = flat(&slot, "slot", at::kInt, 0);
        const float* pw = flat<float>(w, "w", at::kFloat, tokens * topk);
        float* pdw = flat<float>(&dw, "dw", at::kFloat, tokens * topk);
        return on(d, [&](void* st) {
            return q4_expert_combine_grad(G.data_ptr(), ldg, Y.data_ptr(), ldy, type_of(Y), int32(Y.size(1), "width"), int32(rows, "rows"), src,
                                          sl, pw, int32(tokens, "tokens"), int32(topk, "topk"), dY.data_ptr(), lddy, pdw, st);
        });
    });
}

// ---- 4-bit floats: codes uint8 (two per byte), words of scales int32 [word of columns][row]

int64_t words(int64_t cols, int32_t flags) { return flags & Q4_F4_BY16 ? (cols + 63) / 64 : blocks(cols); }

// Row pitch of codes of rows x cols values, in bytes.
int64_t code_pitch(const at::Tensor& t, const char* name, int64_t rows, int64_t cols)
{
    if (t.scalar_type() != at::kByte) fail(PyExc_TypeError, name, " must be uint8");
    return pitch(t, name, kCode, rows, (cols + 1) / 2);
}
// Pitch of their words of scales.
int64_t word_pitch(const at::Tensor& t, const char* name, int64_t rows, int64_t cols, int32_t flags)
{
    if (t.scalar_type() != at::kInt) fail(PyExc_TypeError, name, " must be int32");
    const int64_t n = words(cols, flags);
    if (t.dim() != 2 || t.size(0) < n || t.size(1) < rows) fail(PyExc_ValueError, name, " must be 2-D and at least ", n, " x ", rows);
    if (t.stride(1) != 1 && t.size(1) > 1) fail(PyExc_ValueError, name, " must have contiguous rows");
    return t.size(0) > 1 ? t.stride(0) : std::max(t.stride(0), t.size(1));
}
uint32_t* word_data(const at::Tensor* t) { return t ? static_cast<uint32_t*>(t->data_ptr()) : nullptr; }

// X, Q, S, Qt, St, source, topk, flags, factor
PyObject* f4_quantize(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    return entry<9>(a, n, [](PyObject* const* a) {
        const at::Tensor& X = tensor(a[0], "X");
        const at::Tensor *Q = optional(a[1], "Q"), *S = optional(a[2], "S"), *Qt = optional(a[3], "Qt"), *St = optional(a[4], "St");
        const at::Tensor *source = optional(a[5], "source"), *factor = optional(a[8], "factor");
        const int32_t topk = int32(a[6], "topk"), flags = int32(a[7], "flags");
        const c10::Device d = device_of(X, Q, S, Qt, St, source, factor);
        if (!Q != !S || !Qt != !St || (!Q && !Qt))
            fail(PyExc_ValueError, "codes come with their scales: give Q and S, Qt and St, or both pairs");
        const int64_t ldx = pitch(X, "X", kReal, 0, 0), x_rows = X.size(0), cols = X.size(1);
        const int64_t rows = source ? source->numel() : x_rows;
        int64_t ldq = 0, lds = 0, ldqt = 0, ldst = 0;
        if (Q) {
            ldq = code_pitch(*Q, "Q", rows, cols);
            lds = word_pitch(*S, "S", rows, cols, flags);
        }
        if (Qt) {
            ldqt = code_pitch(*Qt, "Qt", cols, rows);
            ldst = word_pitch(*St, "St", cols, rows, flags);
        }
        const int32_t* src = flat(source, "source", at::kInt, rows);
        const float* f = flat<float>(factor, "factor", at::kFloat, 1);
        return on(d, [&](void* st) {
            return q4_f4_quantize(X.data_ptr(), type_of(X), ldx, int32(rows, "rows"), int32(cols, "cols"), src, topk,
                                  int32(x_rows, "rows of X"), flags, f, bytes(Q), ldq, word_data(S), lds, bytes(Qt), ldqt, word_data(St),
                                  ldst, st);
        });
    });
}

// Q, S, Y, flags, factor
PyObject* f4_dequantize(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    return entry<5>(a, n, [](PyObject* const* a) {
        const at::Tensor &Q = tensor(a[0], "Q"), &S = tensor(a[1], "S"), &Y = tensor(a[2], "Y");
        const int32_t flags = int32(a[3], "flags");
        const at::Tensor* factor = optional(a[4], "factor");
        const c10::Device d = device_of(Y, &Q, &S, factor);
        const int64_t ldy = pitch(Y, "Y", kReal, 0, 0), rows = Y.size(0), cols = Y.size(1);
        const int64_t ldq = code_pitch(Q, "Q", rows, cols), lds = word_pitch(S, "S", rows, cols, flags);
        const float* f = flat<float>(factor, "factor", at::kFloat, 1);
        return on(d, [&](void* st) {
            return q4_f4_dequantize(bytes(&Q), ldq, word_data(&S), lds, int32(rows, "rows"), int32(cols, "cols"), flags, f, Y.data_ptr(),
                                    type_of(Y), ldy, st);
        });
    });
}

// A, SA, Bt, SB, C, M, N, K, flags, FA, FB, starts (None: dense)
PyObject* gemm_f4(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    return entry<12>(a, n, [](PyObject* const* a) {
        const at::Tensor &A = tensor(a[0], "A"), &SA = tensor(a[1], "SA"), &B = tensor(a[2], "Bt"), &SB = tensor(a[3], "SB"), &C = tensor(a[4], "C");
        const int32_t M = int32(a[5], "M"), N = int32(a[6], "N"), K = int32(a[7], "K"), flags = int32(a[8], "flags");
        const at::Tensor *FA = optional(a[9], "FA"), *FB = optional(a[10], "FB"), *starts = optional(a[11], "starts");
        const c10::Device d = device_of(A, &SA, &B, &SB, &C, FA, FB, starts);
        const int32_t* at = flat(starts, "starts", at::kInt, 1);
        const int64_t E = starts ? starts->numel() - 1 : 1;
        const int64_t lda = code_pitch(A, "A", M, K), ldb = code_pitch(B, "Bt", E * N, K), ldc = pitch(C, "C", kReal, M, N);
        const int64_t ldsa = word_pitch(SA, "SA", M, K, flags), ldsb = word_pitch(SB, "SB", E * N, K, flags);
        const float *fa = flat<float>(FA, "FA", at::kFloat, 1), *fb = flat<float>(FB, "FB", at::kFloat, E);
        return on(d, [&](void* st) {
            if (starts)
                return q4_gemm_f4_experts(bytes(&A), lda, word_data(&SA), ldsa, bytes(&B), ldb, word_data(&SB), ldsb, flags, fa, fb, at,
                                          int32(E, "experts"), C.data_ptr(), type_of(C), ldc, M, N, K, st);
            return q4_gemm_f4(bytes(&A), lda, word_data(&SA), ldsa, bytes(&B), ldb, word_data(&SB), ldsb, flags, fa, fb, C.data_ptr(),
                              type_of(C), ldc, M, N, K, st);
        });
    });
}

// X, ids, w, W1, S1, W2, S2, Out, E, H, ws, flags, F1, F2
PyObject* expert_layer_f4(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    return entry<14>(a, n, [](PyObject* const* a) {
        const at::Tensor &X = tensor(a[0], "X"), &ids = tensor(a[1], "ids"), &W1 = tensor(a[3], "W1"), &S1 = tensor(a[4], "S1"),
                         &W2 = tensor(a[5], "W2"), &S2 = tensor(a[6], "S2"), &Out = tensor(a[7], "Out"), &ws = tensor(a[10], "ws");
        const at::Tensor *w = optional(a[2], "w"), *F1 = optional(a[12], "F1"), *F2 = optional(a[13], "F2");
        const int32_t E = int32(a[8], "E"), H = int32(a[9], "H"), flags = int32(a[11], "flags");
        const c10::Device d = device_of(X, &ids, w, &W1, &S1, &W2, &S2, &Out, &ws, F1, F2);
        if (ids.dim() != 2) fail(PyExc_ValueError, "ids must be [tokens, topk]");
        if (!ws.is_contiguous()) fail(PyExc_ValueError, "ws must be contiguous");
        const int64_t ldx = pitch(X, "X", kReal, 0, 0), tokens = X.size(0), D = X.size(1), topk = ids.size(1);
        if (ids.size(0) != tokens) fail(PyExc_ValueError, "ids must have a row per token");
        const int64_t ldo = pitch(Out, "Out", kReal, tokens, D), rows1 = (int64_t)E * (flags & Q4_F4_GATED ? 2 : 1) * H, rows2 = (int64_t)E * D;
        same_rows(X, Out);
        const int64_t ldw1 = code_pitch(W1, "W1", rows1, D), lds1 = word_pitch(S1, "S1", rows1, D, flags);
        const int64_t ldw2 = code_pitch(W2, "W2", rows2, H), lds2 = word_pitch(S2, "S2", rows2, H, flags);
        const int32_t* i = flat(&ids, "ids", at::kInt, 0);
        const float *pw = flat<float>(w, "w", at::kFloat, tokens * topk), *f1 = flat<float>(F1, "F1", at::kFloat, E),
                    *f2 = flat<float>(F2, "F2", at::kFloat, E);
        return on(d, [&](void* st) {
            return q4_expert_layer_f4(X.data_ptr(), ldx, type_of(X), int32(tokens, "tokens"), int32(D, "width"), H, i, pw,
                                      int32(topk, "topk"), E, flags, bytes(&W1), ldw1, word_data(&S1), lds1, f1, bytes(&W2), ldw2,
                                      word_data(&S2), lds2, f2, Out.data_ptr(), ldo, ws.data_ptr(),
                                      (size_t)ws.numel() * ws.element_size(), st);
        });
    });
}

#define Q4_ENTRY(name) {#name, (PyCFunction)(void (*)(void))name, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {Q4_ENTRY(f8_quantize), Q4_ENTRY(gemm_f8), Q4_ENTRY(gemm_f8_experts), Q4_ENTRY(expert_sort),
                         Q4_ENTRY(expert_gather), Q4_ENTRY(expert_combine), Q4_ENTRY(expert_combine_grad),
                         Q4_ENTRY(f4_quantize), Q4_ENTRY(f4_dequantize), Q4_ENTRY(gemm_f4), Q4_ENTRY(expert_layer_f4), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_q4_torch", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

extern "C" PyObject* PyInit__q4_torch(void)
{
    PyObject* m = PyModule_Create(&module);
    if (m && PyModule_AddStringConstant(m, "built_for", Q4_TORCH_VERSION) < 0) {
        Py_DECREF(m);
        return nullptr;
    }
    return m;
}
