"""e4m3 quantizer and products on the GPU against the 64-bit oracle.

Codes and scales have to be equal to the last bit.  A product's bound: the terms of a block are exact in
binary32 (two 4-bit significands), so with one rounding per addition a block's sum of 128 terms, the two
products with scales and the sum over blocks are off by at most (128 + 2 + ceil(K / 128)) * 2^-24 times the
sum of the terms' magnitudes; the output's type adds half of its last place.
"""
import numpy as np
import pytest

from oracle import f8

pytestmark = pytest.mark.gpu

HALF_ULP = {"f32": 0.0, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}      # significands of 8 and 11 bits
HALF_SMALLEST = {"f32": 2.0 ** -150, "bf16": 2.0 ** -134, "f16": 2.0 ** -25}     # the last place of subnormal values


@pytest.fixture(scope="module")
def q4():
    from paper_2009_06488_b200 import binding
    binding.q4_set_variant(0)
    return binding


def types():
    import torch
    return {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def values(seed, rows, cols, t):
    """(values rounded to the type as float32, the same on the GPU)."""
    import torch
    r = np.random.default_rng(seed)
    x = (r.standard_normal((rows, cols)) * np.exp(r.standard_normal(cols))).astype(np.float32)
    if rows * cols:
        x[r.random((rows, cols)) < 0.01] = 0
    g = torch.from_numpy(x).cuda().to(types()[t])
    return g.float().cpu().numpy(), g


def placed(host, pitch=None, offset=0, dtype=None):
    """A 2-D array on the GPU with a row pitch and a base offset in elements; bytes around it are 0x55."""
    import torch
    rows, cols = host.shape
    pitch = pitch or max(cols, 1)
    t = torch.from_numpy(np.ascontiguousarray(host))
    buf = torch.full((offset + max(rows, 1) * pitch,), 0x55, dtype=t.dtype, device="cuda")
    view = buf[offset:].as_strided((rows, cols), (pitch, 1))
    view.copy_(t)
    return view


def up16(n):
    return (n + 15) // 16 * 16


# ------------------------------------------------------------------------------------------- quantizer
@pytest.mark.parametrize("t", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("blocks", [False, True])
@pytest.mark.parametrize("pow2", [False, True])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 128), (3, 129), (33, 100), (128, 128), (130, 257), (257, 385), (1000, 40)])
def test_quantize_matches_the_oracle(q4, t, blocks, pow2, rows, cols):
    import torch
    x, X = values(rows * 1000 + cols, rows, cols, t)
    q, s = f8.quantize(x, blocks, pow2)
    qt, st = f8.quantize(np.ascontiguousarray(x.T), blocks, pow2)
    for pad, straight, across in ((0, True, False), (5, True, True), (16, False, True)):
        new = lambda r, c: torch.full((r, up16(c) + pad), 0x5A, dtype=torch.uint8, device="cuda")
        sc = lambda a: torch.full((a.shape[0], a.shape[1] + pad), -1.0, device="cuda")
        Q, Qt, S, St = new(rows, cols), new(cols, rows), sc(s), sc(st)
        q4.q4_f8_quantize(X, Q[:, :cols] if straight else None, S if straight else None,
                          Qt[:, :rows] if across else None, St if across else None, blocks=blocks, pow2=pow2)
        if straight:
            assert (Q[:, :cols].cpu().numpy() == q).all() and (S[:, :s.shape[1]].cpu().numpy() == s).all()
            assert (Q[:, cols:] == 0x5A).all() and (S[:, s.shape[1]:] == -1).all()
        if across:
            assert (Qt[:, :rows].cpu().numpy() == qt).all() and (St[:, :st.shape[1]].cpu().numpy() == st).all()
            assert (Qt[:, rows:] == 0x5A).all() and (St[:, st.shape[1]:] == -1).all()


@pytest.mark.parametrize("t", ["f32", "bf16"])
@pytest.mark.parametrize("topk", [1, 3])
def test_quantize_of_picked_rows(q4, t, topk):
    import torch
    x, X = values(7, 37, 200, t)
    r = np.random.default_rng(8)
    source = r.integers(-2, 39 * topk, 150).astype(np.int32)          # some absent, some past the end
    rows = np.where((source >= 0) & (source // topk < 37), source // topk, -1)
    want = np.where(rows[:, None] >= 0, x[rows], np.float32(0))
    q, s = f8.quantize(want)
    qt, st = f8.quantize(np.ascontiguousarray(want.T))
    Q, S = torch.empty(150, 208, dtype=torch.uint8, device="cuda"), torch.empty(2, 150, device="cuda")
    Qt, St = torch.empty(200, 160, dtype=torch.float8_e4m3fn, device="cuda"), torch.empty(2, 200, device="cuda")
    q4.q4_f8_quantize(X, Q[:, :200], S, Qt, St, source=torch.from_numpy(source).cuda(), topk=topk)
    assert (Q[:, :200].cpu().numpy() == q).all() and (S.cpu().numpy() == s).all()
    assert (Qt.view(torch.uint8)[:, :150].cpu().numpy() == qt).all() and (St.cpu().numpy() == st).all()
    Q2, S2 = torch.empty_like(Q), torch.empty_like(S)
    q4.q4_f8_quantize(X, Q2[:, :200], S2, source=torch.from_numpy(source).cuda(), topk=topk)
    assert (Q2[:, :200].cpu().numpy() == q).all() and (S2.cpu().numpy() == s).all()


@pytest.mark.parametrize("blocks", [False, True])
@pytest.mark.parametrize("pow2", [False, True])
def test_quantize_of_extreme_values(q4, blocks, pow2):
    import torch
    x = np.zeros((140, 300), dtype=np.float32)
    x[0, :4] = [3.4e38, -3.4e38, 1e30, 1.0]
    x[1, :4] = [1e-45, -1e-40, 1e-38, 0.0]
    x[2, 130:134] = [2.0 ** -60, -2.0 ** -70, 2.0 ** -61, -0.0]
    x[3, :] = -0.0
    x[130, :300] = 448 * 2.0 ** np.arange(-20, 20).repeat(8)[:300]
    q, s = f8.quantize(x, blocks, pow2)
    qt, st = f8.quantize(np.ascontiguousarray(x.T), blocks, pow2)
    X = torch.from_numpy(x).cuda()
    Q, S = torch.empty(140, 304, dtype=torch.uint8, device="cuda"), torch.empty(*s.shape, device="cuda")
    Qt, St = torch.empty(300, 144, dtype=torch.uint8, device="cuda"), torch.empty(*st.shape, device="cuda")
    q4.q4_f8_quantize(X, Q, S, Qt, St, blocks=blocks, pow2=pow2)
    assert (Q[:, :300].cpu().numpy() == q).all() and (S.cpu().numpy() == s).all()
    assert (Qt[:, :140].cpu().numpy() == qt).all() and (St.cpu().numpy() == st).all()


def test_what_is_not_finite_stays_in_its_group(q4):
    import torch
    X = torch.ones(5, 300, device="cuda")
    X[1, 7], X[2, 130], X[3, 299] = float("inf"), float("nan"), float("-inf")
    Q, S = torch.empty(5, 304, dtype=torch.float8_e4m3fn, device="cuda"), torch.empty(3, 5, device="cuda")
    q4.q4_f8_quantize(X, Q, S)
    fine = np.ones((3, 5), dtype=bool)
    fine[0, 1] = fine[1, 2] = fine[2, 3] = False
    assert (np.isfinite(S.cpu().numpy()) == fine).all()
    W, SW = torch.full((16, 304), 0x38, dtype=torch.uint8, device="cuda"), torch.ones(1, 3, device="cuda")
    C = torch.empty(5, 16, device="cuda")
    q4.q4_gemm_f8(Q, S, W, SW, C, 5, 16, 300)
    c = C.cpu().numpy()
    assert np.isnan(c[1:4]).all() and np.allclose(c[[0, 4]], 300, rtol=1e-5)


# -------------------------------------------------------------------------------------------- products
def operands(seed, rows, cols, blocks):
    r = np.random.default_rng(seed)
    x = (r.standard_normal((rows, cols)) * np.exp(0.5 * r.standard_normal(cols))).astype(np.float32)
    return f8.quantize(x, blocks)


def check(got, want, mag, K, out):
    got = got.float().cpu().numpy().astype(np.float64)
    bound = (130 + f8.blocks_of(K)) * 2.0 ** -24 * mag
    bound = bound + (np.abs(want) + bound) * HALF_ULP[out] + HALF_SMALLEST[out] + 1e-30
    assert np.isfinite(got).all()
    worst = (np.abs(got - want) / bound).max() if got.size else 0
    assert worst <= 1, f"off by {worst:.3g} times the bound"


SHAPES = [(1, 1, 1), (1, 64, 128), (1, 200, 1000), (2, 129, 257), (8, 384, 512), (16, 100, 640), (17, 130, 384), (33, 256, 100),
          (64, 512, 2048), (100, 300, 129), (128, 128, 128), (129, 257, 255), (255, 255, 1024), (256, 256, 256), (257, 300, 400),
          (300, 1000, 640), (515, 130, 1500), (700, 777, 333)]


@pytest.mark.parametrize("M,N,K", SHAPES)
@pytest.mark.parametrize("b_rows", [False, True])
@pytest.mark.parametrize("out", ["f32", "bf16", "f16"])
def test_product_matches_the_oracle(q4, M, N, K, b_rows, out):
    import torch
    (a, sa), (b, sb) = operands(M + K, M, K, False), operands(N + K + 1, N, K, not b_rows)
    want, mag = f8.product(a, sa, b, sb, b_rows)
    A, B = placed(a, up16(K) + 16), placed(b, up16(K))
    SA, SB = placed(sa, sa.shape[1] + 3), placed(sb)
    C = torch.full((M + 1, up16(N) + 8), 7.0, dtype=types()[out], device="cuda")
    q4.q4_gemm_f8(A, SA, B, SB, C, M, N, K, b_rows=b_rows)
    check(C[:M, :N], want, mag, K, out)
    assert (C[M:] == 7).all() and (C[:, N:] == 7).all()
    # rows of C that do not begin on 16 bytes
    D = torch.full((M, N + 3), 7.0, dtype=types()[out], device="cuda")
    q4.q4_gemm_f8(A, SA, B, SB, D[:, 1:], M, N, K, b_rows=b_rows)
    assert torch.equal(D[:, 1:N + 1], C[:M, :N]) and (D[:, 0] == 7).all() and (D[:, N + 1:] == 7).all()
    assert q4.q4_last_device_status() == q4.Q4_OK


@pytest.mark.parametrize("M,N,K", [(130, 200, 6150), (300, 1000, 6300), (520, 1200, 6200), (40, 300, 8200), (700, 1200, 6200)])
@pytest.mark.parametrize("b_rows", [False, True])
@pytest.mark.parametrize("out", ["f32", "bf16"])
def test_long_products_of_few_tiles(q4, M, N, K, b_rows, out):
    """Few tiles and a long depth, which may be shared by several CTA pairs (2, 16, 30, 3 and 30 tiles)."""
    import torch
    (a, sa), (b, sb) = operands(M + K, M, K, False), operands(N + K + 1, N, K, not b_rows)
    want, mag = f8.product(a, sa, b, sb, b_rows)
    A, B, SA, SB = placed(a, up16(K)), placed(b, up16(K) + 32), placed(sa), placed(sb)
    for pad in (8, 3):
        C = torch.full((M + 1, N + pad), 7.0, dtype=types()[out], device="cuda")
        q4.q4_gemm_f8(A, SA, B, SB, C, M, N, K, b_rows=b_rows)
        check(C[:M, :N], want, mag, K, out)
        assert (C[M:] == 7).all() and (C[:, N:] == 7).all()
    assert q4.q4_last_device_status() == q4.Q4_OK


@pytest.mark.parametrize("off,pitch", [(3, 0), (0, 5)])
@pytest.mark.parametrize("M,N,K", [(1, 70, 300), (130, 70, 300)])
def test_product_of_unaligned_operands(q4, M, N, K, off, pitch):
    import torch
    (a, sa), (b, sb) = operands(1, M, K, False), operands(2, N, K, True)
    want, mag = f8.product(a, sa, b, sb)
    C = torch.empty(M, N, device="cuda")
    q4.q4_gemm_f8(placed(a, up16(K) + pitch, off), placed(sa), placed(b, up16(K) + pitch, off), placed(sb), C, M, N, K)
    check(C, want, mag, K, "f32")


def test_bytes_behind_the_depth_are_not_read(q4):
    """Codes of NaN in the padding of both operands."""
    import torch
    M, N, K = 40, 72, 200
    (a, sa), (b, sb) = operands(1, M, K, False), operands(2, N, K, True)
    want, mag = f8.product(a, sa, b, sb)
    wide = lambda x: np.concatenate([x, np.full((x.shape[0], 56), 0x7F, dtype=np.uint8)], 1)
    for m in (M, 3, 1):
        C = torch.empty(m, N, device="cuda")
        A = torch.from_numpy(wide(a)).cuda()
        q4.q4_gemm_f8(A, placed(sa), torch.from_numpy(wide(b)).cuda(), placed(sb), C, m, N, K)
        check(C, want[:m], mag[:m], K, "f32")


def test_large_product_and_repeated_calls_agree(q4):
    """Many tiles per CTA pair, ragged in every dimension; three calls in a row give the same bits."""
    import torch
    M, N, K = 4111, 5001, 1111
    (a, sa), (b, sb) = operands(1, M, K, False), operands(2, N, K, True)
    A, B, SA, SB = placed(a, up16(K)), placed(b, up16(K)), placed(sa), placed(sb)
    want, mag = f8.product(a, sa, b, sb)
    outs = [torch.empty(M, up16(N), dtype=torch.float32, device="cuda") for _ in range(3)]
    for C in outs:
        q4.q4_gemm_f8(A, SA, B, SB, C, M, N, K)
    check(outs[0][:, :N], want, mag, K, "f32")
    assert torch.equal(outs[0][:, :N], outs[1][:, :N]) and torch.equal(outs[0][:, :N], outs[2][:, :N])


def test_gradients_of_the_product(q4):
    """dX = G W and dW = G^T X from the transposed codes, against the formula in 64 bits and differences of the loss."""
    import torch
    T, N, K = 200, 150, 270
    r = np.random.default_rng(4)
    x, w, g = (r.standard_normal(s).astype(np.float32) for s in ((T, K), (N, K), (T, N)))
    new = lambda rows, cols: torch.empty(rows, up16(cols), dtype=torch.uint8, device="cuda")
    sc = lambda a, b: torch.empty(a, b, device="cuda")
    Wq, Sw, Wt, Swt = new(N, K), sc(2, 3), new(K, N), sc(3, 2)
    q4.q4_f8_quantize(torch.from_numpy(w).cuda(), Wq[:, :K], Sw, Wt[:, :N], Swt, blocks=True)
    Gq, Sg, Gt, Sgt = new(T, N), sc(2, T), new(N, T), sc(2, N)
    q4.q4_f8_quantize(torch.from_numpy(g).cuda(), Gq, Sg, Gt, Sgt)
    Xt, Sxt = new(K, T), sc(2, K)
    q4.q4_f8_quantize(torch.from_numpy(x).cuda(), Qt=Xt, St=Sxt)
    dX, dW = torch.empty(T, K, device="cuda"), torch.empty(N, K, device="cuda")
    q4.q4_gemm_f8(Gq, Sg, Wt, Swt, dX, T, K, N)
    q4.q4_gemm_f8(Gt, Sgt, Xt, Sxt, dW, N, K, T, b_rows=True)
    n = lambda t, c: t[:, :c].cpu().numpy()
    vw = f8.values(n(Wq, K), Sw.cpu().numpy(), blocks=True)
    vg, vgt = f8.values(n(Gq, N), Sg.cpu().numpy()), f8.values(n(Gt, T), Sgt.cpu().numpy())
    vx = f8.values(n(Xt, T), Sxt.cpu().numpy()).T
    check(dX, vg @ vw, np.abs(vg) @ np.abs(vw), N, "f32")
    check(dW, vgt @ vx, np.abs(vgt) @ np.abs(vx), T, "f32")
    h = 1e-3
    for i, j in ((0, 0), (7, 200), (149, 269)):
        d = np.zeros_like(vw); d[i, j] = h
        # the loss is linear in W: its difference is exact up to the rounding of 64 bits
        diff = ((vx @ (vw + d).T * vgt.T).sum() - (vx @ (vw - d).T * vgt.T).sum()) / (2 * h)
        assert abs(dW[i, j].item() - diff) <= 132 * 2.0 ** -24 * (np.abs(vgt[i]) @ np.abs(vx[:, j])) + 1e-6
    for i, j in ((0, 0), (100, 33), (199, 269)):
        d = np.zeros_like(vx); d[i, j] = h
        diff = (((vx + d) @ vw.T * vg).sum() - ((vx - d) @ vw.T * vg).sum()) / (2 * h)
        assert abs(dX[i, j].item() - diff) <= 132 * 2.0 ** -24 * (np.abs(vg[i]) @ np.abs(vw[:, j])) + 1e-6


def test_products_on_another_stream_and_in_a_graph(q4):
    import torch
    M, N, K = 300, 520, 700
    (a, sa), (b, sb) = operands(1, M, K, False), operands(2, N, K, True)
    want, mag = f8.product(a, sa, b, sb)
    side = torch.cuda.Stream()
    A, B, SA, SB = placed(a, up16(K)), placed(b, up16(K)), placed(sa), placed(sb)
    C = torch.empty(M, N, device="cuda")
    q4.q4_gemm_f8(A, SA, B, SB, C, M, N, K)
    C.zero_()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        q4.q4_gemm_f8(A, SA, B, SB, C, M, N, K)
    graph.replay()
    torch.cuda.synchronize()
    check(C, want, mag, K, "f32")
    C.zero_()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        q4.q4_gemm_f8(A, SA, B, SB, C, M, N, K)
    torch.cuda.current_stream().wait_stream(side)
    check(C, want, mag, K, "f32")


# --------------------------------------------------------------------------------- products by experts
def segments(counts, align=1):
    at = [0]
    for c in counts:
        at.append(at[-1] + -(-c // align) * align)
    return np.array(at, dtype=np.int32)


@pytest.mark.parametrize("counts", [[0, 0, 0], [1, 0, 3], [5, 17, 0, 1, 40], [128, 130, 0, 257], [0, 300, 2, 2, 2, 31, 33, 64, 0],
                                    [600, 1, 129]])
@pytest.mark.parametrize("N,K", [(64, 128), (200, 300), (384, 640), (777, 1000)])
@pytest.mark.parametrize("out", ["f32", "bf16"])
def test_experts_match_the_oracle(q4, counts, N, K, out):
    import torch
    starts = segments(counts)
    E, M = len(counts), int(starts[-1]) + 5                        # five rows behind the last segment
    a, sa = operands(sum(counts) + N, M, K, False)
    parts = [operands(100 + e, N, K, True) for e in range(E)]
    b, sb = np.concatenate([p[0] for p in parts]), np.concatenate([p[1] for p in parts])
    want, mag = f8.experts(a, sa, b, sb, starts, N)
    C = torch.full((M, up16(N)), 7.0, dtype=types()[out], device="cuda")
    q4.q4_gemm_f8_experts(placed(a, up16(K)), placed(sa), placed(b, up16(K)), placed(sb),
                          torch.from_numpy(starts).cuda(), C, M, N, K)
    live = int(starts[-1])
    check(C[:live, :N], want[:live], mag[:live], K, out)
    assert (C[live:] == 7).all() and (C[:, N:] == 7).all()
    D = torch.full((M, N + 1), 7.0, dtype=types()[out], device="cuda")
    q4.q4_gemm_f8_experts(placed(a, up16(K) + 3), placed(sa), placed(b, up16(K) + 3), placed(sb),
                          torch.from_numpy(starts).cuda(), D[:, 1:], M, N, K)
    check(D[:live, 1:], want[:live], mag[:live], K, out)
    assert (D[live:] == 7).all() and (D[:, 0] == 7).all()
    assert q4.q4_last_device_status() == q4.Q4_OK


def test_starts_out_of_range_touch_nothing(q4):
    """Starts that fall, are negative or pass the end are cut to 0 .. M and to rising order."""
    import torch
    M, N, K, E = 50, 64, 256, 4
    a, sa = operands(1, M, K, False)
    parts = [operands(100 + e, N, K, True) for e in range(E)]
    b, sb = np.concatenate([p[0] for p in parts]), np.concatenate([p[1] for p in parts])
    C = torch.full((M + 4, N), 7.0, device="cuda")
    starts = np.array([-5, 20, 10, 30, 1000], dtype=np.int32)       # segments 0..20, none, 10..30, 30..50
    q4.q4_gemm_f8_experts(placed(a), placed(sa), placed(b), placed(sb), torch.from_numpy(starts).cuda(), C, M, N, K)
    assert (C[M:] == 7).all()
    for e, (lo, hi) in ((0, (0, 10)), (2, (20, 30)), (3, (30, 50))):
        va, vb = f8.values(a, sa)[lo:hi], f8.values(*parts[e], blocks=True)
        check(C[lo:hi], va @ vb.T, np.abs(va) @ np.abs(vb).T, K, "f32")


@pytest.mark.parametrize("counts", [[0, 0], [1, 0, 200], [128, 256, 5], [700, 0, 0, 3, 130]])
@pytest.mark.parametrize("M,N", [(64, 64), (200, 136), (300, 520)])
@pytest.mark.parametrize("out", ["f32", "bf16"])
def test_experts_weight_gradient_matches_the_oracle(q4, counts, M, N, out):
    import torch
    starts = segments(counts, 128)
    E, K = len(counts), int(starts[-1]) + 128
    a, sa = operands(M + K, M, K, False)
    b, sb = operands(N + K + 1, N, K, False)
    want, mag = f8.experts_wgrad(a, sa, b, sb, starts)
    C = torch.full((E * M + 1, N + 8), 7.0, dtype=types()[out], device="cuda")
    q4.q4_gemm_f8_experts_wgrad(placed(a), placed(sa), placed(b), placed(sb), torch.from_numpy(starts).cuda(), C, M, N, K)
    check(C[:E * M, :N], want, mag, K, out)
    assert (C[E * M:] == 7).all() and (C[:, N:] == 7).all()
    assert q4.q4_last_device_status() == q4.Q4_OK
