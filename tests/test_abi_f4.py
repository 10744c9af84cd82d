"""Argument checks of the 4-bit float products and of their expert layer: nothing here needs a device, every call is
refused (or empty) before any launch."""
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
    def f(X=fake, t=1, ldx=257, rows=9, cols=257, src=None, topk=1, xr=9, flags=0, fac=None, Q=fake, ldq=129, S=fake, lds=9,
          Qt=None, ldqt=0, St=None, ldst=0):
        return lib.q4_f4_quantize(X, t, ldx, rows, cols, src, topk, xr, flags, fac, Q, ldq, S, lds, Qt, ldqt, St, ldst, None)
    assert f(t=3) == INVALID and f(t=-1) == INVALID and f(rows=-1) == INVALID and f(ldx=256) == INVALID and f(flags=2) == INVALID
    assert f(S=None) == INVALID and f(Q=None) == INVALID and f(Q=None, S=None) == INVALID and f(X=None) == INVALID
    assert f(ldq=128) == INVALID and f(lds=8) == INVALID and f(Qt=fake, St=None) == INVALID
    assert f(Qt=fake, St=fake, ldqt=4, ldst=257) == INVALID and f(Qt=fake, St=fake, ldqt=5, ldst=256) == INVALID
    assert f(fac=fake) == INVALID                                     # a factor belongs to scales per 16
    assert f(src=fake, topk=0) == INVALID and f(src=fake, xr=-1) == INVALID
    assert f(X=fake + 1) == ALIGN and f(t=0, X=fake + 2) == ALIGN and f(S=fake + 2) == ALIGN and f(src=fake + 2) == ALIGN
    assert f(flags=1, fac=fake + 1) == ALIGN
    assert f(rows=0, lds=0) == 0 and f(cols=0) == 0
    assert f(rows=2 ** 31 - 1, cols=2 ** 12, ldx=2 ** 12, ldq=2 ** 12, lds=2 ** 31) == RANGE


def test_read_back(lib):
    def f(Q=fake, ldq=129, S=fake, lds=9, rows=9, cols=257, flags=0, fac=None, Y=fake, t=1, ldy=257):
        return lib.q4_f4_dequantize(Q, ldq, S, lds, rows, cols, flags, fac, Y, t, ldy, None)
    assert f(t=3) == INVALID and f(ldq=128) == INVALID and f(lds=8) == INVALID and f(ldy=256) == INVALID and f(flags=2) == INVALID
    assert f(Q=None) == INVALID and f(S=None) == INVALID and f(Y=None) == INVALID and f(rows=-1) == INVALID
    assert f(S=fake + 2) == ALIGN and f(Y=fake + 1) == ALIGN and f(fac=fake + 2) == ALIGN
    assert f(rows=0) == 0 and f(cols=0) == 0


def test_products(lib):
    def f(A=fake, lda=129, SA=fake, ldsa=8, B=fake, ldb=129, SB=fake, ldsb=16, flags=0, FA=None, FB=None, C=fake, t=0, ldc=16, M=8,
          N=16, K=257):
        return lib.q4_gemm_f4(A, lda, SA, ldsa, B, ldb, SB, ldsb, flags, FA, FB, C, t, ldc, M, N, K, None)
    assert f(M=-1) == INVALID and f(N=-1) == INVALID and f(K=0) == INVALID and f(t=3) == INVALID and f(flags=2) == INVALID
    assert f(lda=128) == INVALID and f(ldb=128) == INVALID and f(ldsa=7) == INVALID and f(ldsb=15) == INVALID and f(ldc=15) == INVALID
    assert f(A=None) == INVALID and f(SA=None) == INVALID and f(SB=None) == INVALID and f(C=None) == INVALID and f(B=None) == INVALID
    assert f(SA=fake + 2) == ALIGN and f(SB=fake + 1) == ALIGN and f(C=fake + 2) == ALIGN and f(t=1, C=fake + 1) == ALIGN
    assert f(FA=fake + 2) == ALIGN and f(FB=fake + 1) == ALIGN
    assert f(M=0, ldsa=0) == 0 and f(N=0) == 0

    def g(starts=fake, E=4, A=fake, lda=129, SA=fake, ldsa=8, B=fake, ldb=129, SB=fake, ldsb=64, C=fake, t=0, ldc=16, M=8, N=16,
          K=257, flags=1):
        return lib.q4_gemm_f4_experts(A, lda, SA, ldsa, B, ldb, SB, ldsb, flags, None, None, starts, E, C, t, ldc, M, N, K, None)
    assert g(E=-1) == INVALID and g(E=1025) == RANGE and g(starts=None) == INVALID and g(starts=fake + 2) == ALIGN
    assert g(K=0) == INVALID and g(lda=128) == INVALID and g(ldsa=7) == INVALID and g(ldsb=63) == INVALID and g(flags=2) == INVALID
    assert g(C=None) == INVALID and g(A=None) == INVALID and g(t=7) == INVALID and g(ldc=15) == INVALID
    assert g(E=0) == 0 and g(M=0) == 0
    assert g(E=1024, N=1 << 22, ldc=1 << 22) == RANGE


def test_layer(lib):
    need = lib.q4_expert_layer_f4_workspace_bytes(4, 2, 64, 33)
    assert need > 0 and lib.q4_expert_layer_f4_workspace_bytes(0, 2, 64, 33) == 0
    assert lib.q4_expert_layer_f4_workspace_bytes(1, 0, 64, 33) == 0 and lib.q4_expert_layer_f4_workspace_bytes(1, 1, 64, -1) == 0

    def f(X=fake, ldx=64, t=1, T=4, D=64, H=33, ids=fake, w=None, topk=2, E=8, flags=2, W1=fake, ldw1=32, S1=fake, lds1=528, F1=None,
          W2=fake, ldw2=17, S2=fake, lds2=512, F2=None, O=fake, ldo=64, ws=fake, wsb=need):
        return lib.q4_expert_layer_f4(X, ldx, t, T, D, H, ids, w, topk, E, flags, W1, ldw1, S1, lds1, F1, W2, ldw2, S2, lds2, F2,
                                      O, ldo, ws, wsb, None)
    assert f(t=3) == INVALID and f(T=-1) == INVALID and f(D=0) == INVALID and f(H=0) == INVALID and f(topk=0) == INVALID
    assert f(E=0) == INVALID and f(flags=4) == INVALID and f(ldx=63) == INVALID and f(ldo=63) == INVALID
    assert f(ldw1=31) == INVALID and f(ldw2=16) == INVALID and f(lds1=527) == INVALID and f(lds2=511) == INVALID
    for k in ("X", "ids", "W1", "S1", "W2", "S2", "O"):
        assert f(**{k: None}) == INVALID
    assert f(E=1025, lds1=10 ** 9, lds2=10 ** 9) == RANGE and f(T=2 ** 30, topk=4) == RANGE
    assert f(E=1024, H=1 << 21, ldw2=1 << 21, lds1=1 << 40) == RANGE
    assert f(X=fake + 1) == ALIGN and f(O=fake + 1) == ALIGN and f(S1=fake + 2) == ALIGN and f(F2=fake + 2) == ALIGN and f(w=fake + 1) == ALIGN
    assert f(ws=None) == WORKSPACE and f(wsb=need - 1) == WORKSPACE and f(ws=fake + 16) == WORKSPACE
    assert f(T=0, ws=None) == 0


def test_sizes_at_the_end_of_32_bits(lib):
    """Indexes that run past a size by a part of a tile would leave 32 bits."""
    big, half = 2 ** 31 - 100, 2 ** 30
    assert lib.q4_f4_quantize(fake, 1, big, 1, big, None, 1, 1, 0, None, fake, half, fake, 1, None, 0, None, 0, None) == RANGE
    assert lib.q4_f4_quantize(fake, 1, 1, big, 1, None, 1, big, 0, None, fake, 1, fake, big, None, 0, None, 0, None) == RANGE
    assert lib.q4_f4_dequantize(fake, half, fake, 1, 1, big, 0, None, fake, 1, big, None) == RANGE
    assert lib.q4_gemm_f4(fake, half, fake, 1, fake, half, fake, 1, 0, None, None, fake, 0, 1, 1, 1, big, None) == RANGE
    assert lib.q4_gemm_f4(fake, 1, fake, 1, fake, 1, fake, big, 0, None, None, fake, 0, big, 1, big, 1, None) == RANGE
    assert lib.q4_expert_layer_f4(fake, big, 1, 1, big, 1, fake, None, 1, 1, 0, fake, half, fake, 1, None, fake, 1, fake, big, None, fake, big,
                                  256, 2 ** 60, None) == RANGE


def test_the_binding_refuses_what_does_not_fit():
    import torch
    from paper_2009_06488_b200 import binding as q4
    x, c, s = torch.zeros(4, 128), torch.zeros(4, 64, dtype=torch.uint8), torch.zeros(1, 4, dtype=torch.int32)
    with pytest.raises(ValueError):                                   # host tensors
        q4.q4_f4_quantize(x, c, s)
    with pytest.raises(ValueError):
        q4.q4_f4_dequantize(c, s, x)
    with pytest.raises(ValueError):
        q4.q4_gemm_f4(c, s, c, s, x, 4, 4, 128)
    with pytest.raises(ValueError):
        q4.q4_expert_layer_f4(x, s.view(4, 1), None, c, s, c, s, x, 1, 2, c)
