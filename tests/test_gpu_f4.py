"""4-bit float quantizer, read-back and products on the GPU against the 64-bit oracle.

Codes and scales have to be equal to the last bit, and what is read back within half a last place of its type.  A
product's bound: every term is exact in binary32 (significands of 2, 2, 4 and 4 bits); an addition is off by one last
place at most (2^-23: the tensor cores may cut instead of round) of the terms' magnitudes, K of them and those of a
depth split, the two factors' products three more; the output's type adds half of its last place.
"""
import numpy as np
import pytest

from oracle import f4

pytestmark = pytest.mark.gpu

HALF_ULP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
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


def placed(host, pitch=None, offset=0, fill=0x55):
    """A 2-D array on the GPU with a row pitch and a base offset in elements; what is around it holds `fill`."""
    import torch
    rows, cols = host.shape
    pitch = pitch or max(cols, 1)
    t = torch.from_numpy(np.ascontiguousarray(host))
    buf = torch.full((offset + max(rows, 1) * pitch,), fill, dtype=t.dtype, device="cuda")
    view = buf[offset:].as_strided((rows, cols), (pitch, 1))
    view.copy_(t)
    return view


def up16(n):
    return (n + 15) // 16 * 16


def word_tensor(words, pad=0):
    """Words of scales on the GPU; words between the rows are 0x55..."""
    return placed(words.view(np.int32), words.shape[1] + pad, pad, 0x55555555)


# ------------------------------------------------------------------------------------------- quantizer
@pytest.mark.parametrize("t", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("by16", [False, True])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 4096), (3, 129), (33, 100), (128, 128), (130, 257), (257, 385), (1000, 40),
                                       (2048, 1024)])
def test_quantize_matches_the_oracle(q4, t, by16, rows, cols):
    import torch
    x, X = values(rows * 1000 + cols, rows, cols, t)
    factor = np.float32(np.abs(x).max() / 2688) if by16 else None
    F = torch.tensor([factor], device="cuda") if by16 else None
    q, s = f4.quantize(x, by16, factor)
    qt, st = f4.quantize(np.ascontiguousarray(x.T), by16, factor)
    for pad, straight, across in ((0, True, False), (5, True, True), (16, False, True)):
        new = lambda c: torch.full((c.shape[0], up16(c.shape[1]) + pad), 0x5A, dtype=torch.uint8, device="cuda")
        sc = lambda a: torch.full((a.shape[0], a.shape[1] + pad), -7, dtype=torch.int32, device="cuda")
        Q, Qt, S, St = new(q), new(qt), sc(s), sc(st)
        q4.q4_f4_quantize(X, Q if straight else None, S if straight else None, Qt if across else None, St if across else None,
                          by16=by16, factor=F)
        for on, D, W, d, w in ((straight, Q, S, q, s), (across, Qt, St, qt, st)):
            if on:
                assert (W[:, :w.shape[1]].cpu().numpy().view(np.uint32) == w).all() and (W[:, w.shape[1]:] == -7).all()
                assert (D[:, :d.shape[1]].cpu().numpy() == d).all() and (D[:, d.shape[1]:] == 0x5A).all()


@pytest.mark.parametrize("t", ["f32", "bf16"])
@pytest.mark.parametrize("pitch,offset", [(203, 0), (208, 3), (201, 1)])
def test_quantize_of_unaligned_rows(q4, t, pitch, offset):
    import torch
    x, X = values(5, 150, 200, t)
    buf = torch.full((offset + 150 * pitch,), float("nan"), device="cuda", dtype=types()[t])
    X2 = buf[offset:].as_strided((150, 200), (pitch, 1))
    X2.copy_(X)
    for by16 in (False, True):
        (q, s), (qt, st) = f4.quantize(x, by16), f4.quantize(np.ascontiguousarray(x.T), by16)
        Q, S = torch.empty(150, 101, dtype=torch.uint8, device="cuda"), torch.empty(*s.shape, dtype=torch.int32, device="cuda")
        Qt, St = torch.empty(200, 77, dtype=torch.uint8, device="cuda"), torch.empty(*st.shape, dtype=torch.int32, device="cuda")
        q4.q4_f4_quantize(X2, Q, S, Qt, St, by16=by16)
        assert (Q[:, :100].cpu().numpy() == q).all() and (S.cpu().numpy().view(np.uint32) == s).all()
        assert (Qt[:, :75].cpu().numpy() == qt).all() and (St.cpu().numpy().view(np.uint32) == st).all()


@pytest.mark.parametrize("topk", [1, 3])
def test_quantize_of_picked_rows(q4, topk):
    import torch
    x, X = values(7, 37, 200, "bf16")
    r = np.random.default_rng(8)
    source = r.integers(-2, 39 * topk, 150).astype(np.int32)          # some absent, some past the end
    rows = np.where((source >= 0) & (source // topk < 37), source // topk, -1)
    want = np.where(rows[:, None] >= 0, x[rows], np.float32(0))
    (q, s), (qt, st) = f4.quantize(want), f4.quantize(np.ascontiguousarray(want.T))
    Q, S = torch.empty(150, 112, dtype=torch.uint8, device="cuda"), torch.empty(2, 150, dtype=torch.int32, device="cuda")
    Qt, St = torch.empty(200, 80, dtype=torch.uint8, device="cuda"), torch.empty(2, 200, dtype=torch.int32, device="cuda")
    q4.q4_f4_quantize(X, Q, S, Qt, St, source=torch.from_numpy(source).cuda(), topk=topk)
    assert (Q[:, :100].cpu().numpy() == q).all() and (S.cpu().numpy().view(np.uint32) == s).all()
    assert (Qt[:, :75].cpu().numpy() == qt).all() and (St.cpu().numpy().view(np.uint32) == st).all()


@pytest.mark.parametrize("by16", [False, True])
def test_quantize_of_extreme_values_and_ties(q4, by16):
    import torch
    x = np.zeros((140, 300), dtype=np.float32)
    x[0, :4] = [3.4e38, -3.4e38, 1e30, 1.0]
    x[1, :4] = [1e-45, -1e-40, 1e-38, 0.0]
    x[2, 130:134] = [2.0 ** -60, -2.0 ** -70, 2.0 ** -61, -0.0]
    x[3, :] = -0.0
    x[4, ::2] = 6                                                     # the scale is 1: every tie between two codes
    x[4, 1::2] = np.resize(np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, -0.25, -0.75, -1.25, -1.75, -2.5, -3.5, -5]), 150)
    x[5, ::2] = np.nextafter(np.float32(6), np.float32(7))
    x[130, :300] = 6 * 2.0 ** np.arange(-20, 20).repeat(8)[:300]
    (q, s), (qt, st) = f4.quantize(x, by16), f4.quantize(np.ascontiguousarray(x.T), by16)
    X = torch.from_numpy(x).cuda()
    new = lambda a: torch.empty(*a.shape, dtype=torch.uint8 if a.dtype == np.uint8 else torch.int32, device="cuda")
    Q, S, Qt, St = new(q), new(s), new(qt), new(st)
    q4.q4_f4_quantize(X, Q, S, Qt, St, by16=by16)
    assert (S.cpu().numpy().view(np.uint32) == s).all() and (Q.cpu().numpy() == q).all()
    assert (St.cpu().numpy().view(np.uint32) == st).all() and (Qt.cpu().numpy() == qt).all()


@pytest.mark.parametrize("by16", [False, True])
def test_what_is_not_finite_stays_in_its_group(q4, by16):
    import torch
    X = torch.ones(5, 300, device="cuda")
    X[1, 7], X[2, 130], X[3, 299] = float("inf"), float("nan"), float("-inf")
    Q, S = torch.empty(5, 160, dtype=torch.uint8, device="cuda"), torch.empty(f4.words_of(300, by16), 5, dtype=torch.int32, device="cuda")
    q4.q4_f4_quantize(X, Q, S, by16=by16)
    Y = q4.q4_f4_dequantize(Q, S, torch.empty(5, 300, device="cuda"), by16=by16).cpu().numpy()
    g = f4.group_of(by16)
    fine = np.ones((5, 300), dtype=bool)
    for r, c in ((1, 7), (2, 130), (3, 299)):
        fine[r, c // g * g:c // g * g + g] = False
    assert (np.isfinite(Y) == fine).all() and (np.abs(Y[fine] - 1) <= 0.25).all()
    W, SW = torch.full((16, 160), 0x22, dtype=torch.uint8, device="cuda"), torch.empty(f4.words_of(300, by16), 16, dtype=torch.int32, device="cuda")
    SW[:] = 0x38383838 if by16 else 0x7F7F7F7F
    C = q4.q4_gemm_f4(Q, S, W, SW, torch.empty(5, 16, device="cuda"), 5, 16, 300, by16=by16).cpu().numpy()
    assert np.isnan(C[1:4]).all() and np.allclose(C[[0, 4]], Y[[0]].sum(), rtol=1e-5)


@pytest.mark.parametrize("t", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("by16", [False, True])
@pytest.mark.parametrize("rows,cols,pad", [(1, 1, 0), (65, 129, 3), (200, 256, 0), (7, 4096, 8)])
def test_read_back(q4, t, by16, rows, cols, pad):
    import torch
    x, _ = values(rows + cols, rows, cols, "f32")
    factor = np.float32(0.37) if by16 else None
    q, s = f4.quantize(x, by16, factor)
    want = f4.values(q, s, cols, by16, factor)
    Y = torch.full((rows, cols + pad), 7.0, dtype=types()[t], device="cuda")
    q4.q4_f4_dequantize(placed(q, q.shape[1] + pad), word_tensor(s, pad), Y[:, :cols], by16=by16,
                        factor=torch.tensor([factor], device="cuda") if by16 else None)
    got = Y[:, :cols].double().cpu().numpy()
    bound = np.abs(want) * (HALF_ULP[t] + (2.0 ** -24 if by16 else 0)) * 1.001 + HALF_SMALLEST[t]
    assert (np.abs(got - want) <= bound).all() and (Y[:, cols:] == 7).all()


# -------------------------------------------------------------------------------------------- products
def operand(seed, rows, cols, by16):
    """(packed codes, words, values) with every code and a wide range of scales."""
    r = np.random.default_rng(seed)
    codes = r.integers(0, 16, (rows, cols)).astype(np.uint8)
    n = -(-cols // f4.group_of(by16))
    byte = r.integers(8, 100, (rows, n)).astype(np.uint8) if by16 else r.integers(117, 137, (rows, n)).astype(np.uint8)
    q, s = f4.pack(codes), f4.to_words(byte)
    return q, s, f4.values(q, s, cols, by16)


def spoil_absent(words, cols, by16):
    """Bytes of groups behind the last column, which have to be ignored, set to NaN's."""
    n = -(-cols // f4.group_of(by16)) % 4
    out = words.copy()
    if n:
        out[-1] |= np.uint32((0xFFFFFFFF << (8 * n)) & 0xFFFFFFFF)
    return out


def check(C, want, mag, K, t, extra=0):
    """C (GPU) against the 64-bit product."""
    got = C.double().cpu().numpy()
    bound = mag * (K + 8 + extra) * 2.0 ** -23 + (np.abs(want) + mag * K * 2.0 ** -23) * HALF_ULP[t] + HALF_SMALLEST[t]
    bad = ~(np.abs(got - want) <= bound)
    assert not bad.any(), f"{bad.sum()} of {bad.size}, first at {np.argwhere(bad)[0]}: {got[bad][0]} for {want[bad][0]}"


SHAPES = [(1, 1, 1), (1, 64, 4096), (3, 130, 257), (16, 2048, 320), (17, 256, 1000), (33, 100, 63), (64, 64, 64), (65, 129, 191),
          (100, 512, 2048), (128, 128, 256), (129, 257, 511), (200, 1000, 1024), (257, 300, 300), (512, 768, 640), (1000, 520, 130)]


@pytest.mark.parametrize("by16", [False, True])
@pytest.mark.parametrize("M,N,K", SHAPES)
def test_product(q4, by16, M, N, K):
    import torch
    a, sa, va = operand(M * 7 + K, M, K, by16)
    b, sb, vb = operand(N * 5 + K + 1, N, K, by16)
    fa, fb = (np.float32(0.3), np.float32(1.7)) if (M + N) % 2 else (None, None)
    F = lambda f: None if f is None else torch.tensor([f], device="cuda")
    want, mag = f4.product(va * (1 if fa is None else np.float64(fa) * np.float64(fb)), vb)
    w = a.shape[1]
    for t, pitch, offset, pad in (("f32", up16(w), 0, 0), ("bf16", up16(w) + 16, 32, 5), ("f16", w + 1, 1, 3)):
        A, B = placed(a, pitch, offset), placed(b, pitch, offset)
        buf = torch.full((M + 1, N + pad), 9.0, dtype=types()[t], device="cuda")
        q4.q4_gemm_f4(A, word_tensor(spoil_absent(sa, K, by16), pad), B, word_tensor(spoil_absent(sb, K, by16), pad), buf[:M, :N], M, N, K,
                      by16=by16, FA=F(fa), FB=F(fb))
        if t == "f16":                                   # the values pass its range
            buf, w2 = buf.float(), np.where(np.abs(want) < 60000, want, np.nan)
            got = buf[:M, :N].double().cpu().numpy()
            keep = ~np.isnan(w2)
            bound = mag * (K + 8) * 2.0 ** -23 + (np.abs(want) + mag * K * 2.0 ** -23) * HALF_ULP[t] + HALF_SMALLEST[t]
            assert (np.abs(got - want)[keep] <= bound[keep]).all()
        else:
            check(buf[:M, :N], want, mag, K, t)
        assert (buf[M:] == 9).all() and (buf[:, N:] == 9).all()


@pytest.mark.parametrize("by16", [False, True])
@pytest.mark.parametrize("M,N,K", [(2304, 2310, 320), (2500, 2048, 1030), (130, 40, 4096), (300, 9500, 256)])
def test_product_on_wide_tiles(q4, by16, M, N, K):
    a, sa, va = operand(M + K, M, K, by16)
    b, sb, vb = operand(N + K + 1, N, K, by16)
    want, mag = f4.product(va, vb)
    import torch
    for t, pad in (("bf16", 2), ("f32", 0)):
        buf = torch.full((M, N + pad), 9.0, dtype=types()[t], device="cuda")
        q4.q4_gemm_f4(placed(a, up16(a.shape[1])), word_tensor(sa), placed(b, up16(b.shape[1])), word_tensor(sb, 1), buf[:, :N], M, N, K, by16=by16)
        check(buf[:, :N], want, mag, K, t)
        assert (buf[:, N:] == 9).all()


@pytest.mark.parametrize("by16", [False, True])
@pytest.mark.parametrize("M", [1, 5, 16, 17, 40, 64, 90, 128])
@pytest.mark.parametrize("N,K", [(300, 2048), (64, 700), (1536, 1100), (20000, 512)])
def test_few_rows(q4, by16, M, N, K):
    """Depth in one, two and four parts; every width of the tile; columns that end inside one."""
    import torch
    a, sa, va = operand(M + K, M, K, by16)
    b, sb, vb = operand(N + K + 1, N, K, by16)
    want, mag = f4.product(va, vb)
    for t, pad in (("bf16", 3), ("f32", 0)):
        buf = torch.full((M + 1, N + pad), 9.0, dtype=types()[t], device="cuda")
        q4.q4_gemm_f4(placed(a, up16(a.shape[1])), word_tensor(sa, 2), placed(b, up16(b.shape[1])), word_tensor(sb), buf[:M, :N], M, N, K, by16=by16)
        check(buf[:M, :N], want, mag, K, t, extra=4)
        assert (buf[M:] == 9).all() and (buf[:, N:] == 9).all()


@pytest.mark.parametrize("variant", [1, 2])
def test_every_kernel_gives_the_same_product(q4, variant):
    """The general kernel and the CTA-pair kernel on rows that the few-rows kernel takes."""
    import torch
    for by16 in (False, True):
        a, sa, va = operand(3, 20, 600, by16)
        b, sb, vb = operand(4, 3 * 200, 600, by16)
        starts = np.array([0, 7, 7, 20], dtype=np.int32)
        want, mag = f4.experts(va, vb, starts, 200)
        try:
            q4.q4_set_variant(variant)
            C = torch.zeros(20, 200, device="cuda")
            q4.q4_gemm_f4_experts(placed(a, 304), word_tensor(sa), placed(b, 304), word_tensor(sb), torch.from_numpy(starts).cuda(), C, 20, 200,
                                  600, by16=by16)
            check(C, want, mag, 600, "f32")
        finally:
            q4.q4_set_variant(0)


@pytest.mark.parametrize("by16", [False, True])
@pytest.mark.parametrize("counts,N,K", [([0, 5, 0, 1, 40, 0], 130, 300), ([128, 0, 129, 300], 256, 512), ([2] * 16, 200, 1024),
                                        ([0, 0, 0], 64, 64), ([700], 96, 192), ([1, 0, 0, 0, 0, 0, 0, 0, 1], 640, 257)])
def test_product_by_experts(q4, by16, counts, N, K):
    import torch
    E, first, behind = len(counts), 3, 4
    starts = (first + np.concatenate([[0], np.cumsum(counts)])).astype(np.int32)
    M = int(starts[-1]) + behind
    a, sa, va = operand(M + K, M, K, by16)
    b, sb, vb = operand(N + E, E * N, K, by16)
    fb = np.linspace(0.5, 2, E).astype(np.float32)
    want, mag = f4.experts(va, vb * np.repeat(fb.astype(np.float64), N)[:, None], starts, N)
    S = torch.from_numpy(starts).cuda()
    for t, pitch in (("f32", up16(a.shape[1])), ("bf16", up16(a.shape[1])), ("f32", a.shape[1] + 1)):
        C = torch.full((M, N), 9.0, dtype=types()[t], device="cuda")
        q4.q4_gemm_f4_experts(placed(a, pitch), word_tensor(sa, 1), placed(b, pitch), word_tensor(sb), S, C, M, N, K, by16=by16,
                              FB=torch.from_numpy(fb).cuda())
        assert (C[:first] == 9).all() and (C[M - behind:] == 9).all()
        if starts[-1] > first:
            rows = slice(first, int(starts[-1]))
            check(C[rows], want[rows], mag[rows], K, t)


def test_segments_out_of_range_are_cut(q4):
    import torch
    a, sa, va = operand(1, 40, 128, False)
    b, sb, vb = operand(2, 4 * 64, 128, False)
    starts = np.array([-5, 10, 8, 30, 99], dtype=np.int32)            # 0 .. 10, nothing, 8 .. 30, 30 .. 40
    C = torch.full((40, 64), 9.0, device="cuda")
    q4.q4_gemm_f4_experts(placed(a), word_tensor(sa), placed(b), word_tensor(sb), torch.from_numpy(starts).cuda(), C, 40, 64, 128)
    for e, lo, hi in ((0, 0, 8), (2, 10, 30), (3, 30, 40)):
        want, mag = f4.product(va[lo:hi], vb[e * 64:(e + 1) * 64])
        check(C[lo:hi], want, mag, 128, "f32")
