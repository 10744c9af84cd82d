"""Argument checks of the e4m3 products and of the expert layer: nothing here needs a device, every call is
refused (or empty) before any launch."""
import ctypes

import pytest

fake = 0x1000       # never dereferenced
INVALID, ALIGN, RANGE, WORKSPACE = 1, 2, 3, 4


@pytest.fixture(scope="module")
def lib():
    from paper_2009_06488_b200 import build
    build.build()
    from paper_2009_06488_b200 import binding       # sets the argument types
    return binding._lib


def test_quantizer(lib):
    def f(X=fake, t=1, ldx=256, rows=8, cols=256, src=None, topk=1, xr=8, flags=0, Q=fake, ldq=256, S=fake, lds=8,
          Qt=None, ldqt=0, St=None, ldst=0):
        return lib.q4_f8_quantize(X, t, ldx, rows, cols, src, topk, xr, flags, Q, ldq, S, lds, Qt, ldqt, St, ldst, None)
    assert f(t=3) == INVALID and f(t=-1) == INVALID and f(rows=-1) == INVALID and f(ldx=255) == INVALID and f(flags=4) == INVALID
    assert f(S=None) == INVALID and f(Q=None) == INVALID and f(Q=None, S=None) == INVALID and f(X=None) == INVALID
    assert f(ldq=255) == INVALID and f(lds=7) == INVALID and f(Qt=fake, St=None) == INVALID
    assert f(Qt=fake, St=fake, ldqt=7, ldst=256) == INVALID and f(Qt=fake, St=fake, ldqt=8, ldst=255) == INVALID
    assert f(flags=1, lds=1) == INVALID                               # blocks: two blocks of columns
    assert f(src=fake, topk=0) == INVALID and f(src=fake, xr=-1) == INVALID
    assert f(X=fake + 1) == ALIGN and f(t=0, X=fake + 2) == ALIGN and f(S=fake + 2) == ALIGN and f(src=fake + 2) == ALIGN
    assert f(rows=0, lds=0) == 0 and f(cols=0) == 0
    assert f(rows=2 ** 31 - 1, cols=2 ** 12, ldx=2 ** 12, ldq=2 ** 12, lds=2 ** 31) == RANGE


def test_products(lib):
    def f(A=fake, lda=256, SA=fake, ldsa=8, B=fake, ldb=256, SB=fake, ldsb=2, flags=0, C=fake, t=0, ldc=16, M=8, N=16, K=256):
        return lib.q4_gemm_f8(A, lda, SA, ldsa, B, ldb, SB, ldsb, flags, C, t, ldc, M, N, K, None)
    assert f(M=-1) == INVALID and f(N=-1) == INVALID and f(K=0) == INVALID and f(t=3) == INVALID and f(flags=1) == INVALID
    assert f(lda=255) == INVALID and f(ldb=255) == INVALID and f(ldsa=7) == INVALID and f(ldsb=1) == INVALID and f(ldc=15) == INVALID
    assert f(flags=4, ldsb=15) == INVALID
    assert f(A=None) == INVALID and f(SA=None) == INVALID and f(SB=None) == INVALID and f(C=None) == INVALID and f(B=None) == INVALID
    assert f(SA=fake + 2) == ALIGN and f(SB=fake + 1) == ALIGN and f(C=fake + 2) == ALIGN and f(t=1, C=fake + 1) == ALIGN
    assert f(M=0, ldsa=0) == 0 and f(N=0) == 0

    def g(fn, starts=fake, E=4, A=fake, lda=256, SA=fake, ldsa=256, B=fake, ldb=256, SB=fake, ldsb=16, C=fake, t=0, ldc=16, M=8,
          N=16, K=256):
        return fn(A, lda, SA, ldsa, B, ldb, SB, ldsb, starts, E, C, t, ldc, M, N, K, None)
    for fn in (lib.q4_gemm_f8_experts, lib.q4_gemm_f8_experts_wgrad):
        assert g(fn, E=-1) == INVALID and g(fn, E=1025) == RANGE and g(fn, starts=None) == INVALID and g(fn, starts=fake + 2) == ALIGN
        assert g(fn, K=0) == INVALID and g(fn, lda=255) == INVALID and g(fn, ldsa=7) == INVALID and g(fn, ldsb=1) == INVALID
        assert g(fn, C=None) == INVALID and g(fn, A=None) == INVALID and g(fn, t=7) == INVALID and g(fn, ldc=15) == INVALID
        assert g(fn, E=0) == 0 and g(fn, M=0) == 0
    assert g(lib.q4_gemm_f8_experts, E=1024, N=1 << 22, ldc=1 << 22) == RANGE
    assert g(lib.q4_gemm_f8_experts_wgrad, E=1024, M=1 << 22, ldsa=1 << 22) == RANGE


def test_expert_layer(lib):
    assert lib.q4_expert_sort_rows(100, 8, 1) == 100 and lib.q4_expert_sort_rows(100, 8, 16) == 208
    assert lib.q4_expert_sort_rows(3, 8, 128) == 384 and lib.q4_expert_sort_rows(0, 8, 128) == 0
    assert lib.q4_expert_sort_rows(-1, 8, 1) == 0 and lib.q4_expert_sort_workspace_bytes(-1, 8) == 0
    big = 1 << 20
    need = lib.q4_expert_sort_workspace_bytes(big, 64)
    assert need > 0 and lib.q4_expert_sort_workspace_bytes(64, 64) == 0

    def s(ids=fake, n=100, E=8, align=16, starts=fake, source=fake, rows=208, slot=fake, ws=None, wsb=0):
        return lib.q4_expert_sort(ids, n, E, align, starts, source, rows, slot, ws, wsb, None)
    assert s(n=-1) == INVALID and s(E=0) == INVALID and s(align=0) == INVALID and s(rows=207) == INVALID
    assert s(E=1025, rows=10 ** 9) == RANGE and s(align=65537, rows=10 ** 9) == RANGE
    assert s(n=2 ** 31 - 1, align=128, rows=2 ** 31 - 1) == RANGE     # more rows than an int32 can count
    assert s(ids=None) == INVALID and s(slot=None) == INVALID and s(starts=None) == INVALID and s(source=None) == INVALID
    assert s(ids=fake + 1) == ALIGN and s(starts=fake + 2) == ALIGN
    assert s(n=big, E=64, align=1, rows=big) == WORKSPACE
    assert s(n=big, E=64, align=1, rows=big, ws=fake, wsb=need - 1) == WORKSPACE

    def ga(X=fake, ldx=64, t=1, D=64, T=4, k=2, src=fake, rows=8, Xs=fake, ldxs=64):
        return lib.q4_expert_gather(X, ldx, t, D, T, k, src, rows, None, Xs, ldxs, None)

    def co(Y=fake, ldy=64, t=1, D=64, rows=8, slot=fake, T=4, k=2, O=fake, ldo=64):
        return lib.q4_expert_combine(Y, ldy, t, D, rows, slot, None, T, k, O, ldo, None)

    def gr(G=fake, ldd=64, Y=fake, ldy=64, t=1, D=64, rows=8, src=fake, slot=fake, T=4, k=2, dY=fake, lddy=64, dw=fake):
        return lib.q4_expert_combine_grad(G, ldd, Y, ldy, t, D, rows, src, slot, None, T, k, dY, lddy, dw, None)
    for f in (ga, co, gr):
        assert f(t=3) == INVALID and f(k=0) == INVALID and f(T=-1) == INVALID and f(rows=-1) == INVALID and f(D=-1) == INVALID
        assert f(T=2 ** 30, k=4) == RANGE
    assert ga(X=None) == INVALID and ga(src=None) == INVALID and ga(Xs=None) == INVALID and ga(ldx=63) == INVALID and ga(ldxs=63) == INVALID
    assert co(Y=None) == INVALID and co(slot=None) == INVALID and co(O=None) == INVALID and co(ldo=63) == INVALID
    assert gr(G=None) == INVALID and gr(dw=None) == INVALID and gr(dY=None) == INVALID and gr(lddy=63) == INVALID and gr(src=None) == INVALID
    assert ga(X=fake + 1) == ALIGN and co(O=fake + 1) == ALIGN and gr(dw=fake + 2) == ALIGN
    assert ga(rows=0) == 0 and co(T=0) == 0 and gr(T=0, rows=0) == 0


def test_the_binding_refuses_what_does_not_fit():
    import torch
    from paper_2009_06488_b200 import binding as q4
    x = torch.zeros(4, 128)
    with pytest.raises(ValueError):                                   # host tensors
        q4.q4_f8_quantize(x, torch.zeros(4, 128, dtype=torch.uint8), torch.zeros(1, 4))
    with pytest.raises(ValueError):
        q4.q4_gemm_f8(x, x, x, x, x, 4, 4, 128)
    with pytest.raises(ValueError):
        q4.q4_expert_combine(x, torch.zeros(4, 1, dtype=torch.int32), None, x)
