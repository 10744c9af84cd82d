"""Rows that begin at any element: the quantizer, the products' outputs and the expert layer's rows.

Inputs lie in buffers whose other values are NaN, outputs in buffers whose other values have to stay.  Bounds:
codes and scales equal; a product of K terms off by at most (128 + 2 + ceil(K / 128)) * 2^-24 of the terms'
magnitudes, a sum of n products by (n + 1) * 2^-24, plus half of the output's last place.
"""
import numpy as np
import pytest

from oracle import f8

pytestmark = pytest.mark.gpu

HALF_ULP = {"f32": 0.0, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
HALF_SMALLEST = {"f32": 2.0 ** -150, "bf16": 2.0 ** -134, "f16": 2.0 ** -25}
WIDTHS = [1, 3, 7, 8, 9, 15, 16, 17, 31, 100, 121, 255, 257, 513, 2051]
PLACES = [(0, 0), (1, 1), (3, 0), (5, 8), (7, 3), (8, 5)]              # elements before the first row, behind each row


@pytest.fixture(scope="module")
def q4():
    from paper_2009_06488_b200 import binding
    binding.q4_set_variant(0)
    return binding


def types():
    import torch
    return {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def view(rows, cols, t, place, fill):
    """(buffer, matrix in it): the buffer ends with the matrix's last value."""
    import torch
    off, pad = place
    buf = torch.full((off + (rows - 1) * (cols + pad) + cols,), fill, dtype=types()[t], device="cuda")
    return buf, buf[off:].as_strided((rows, cols), (cols + pad, 1))


def random(seed, rows, cols, t, place):
    import torch
    x = torch.from_numpy(np.random.default_rng(seed).standard_normal((rows, cols)).astype(np.float32)).to(types()[t])
    _, X = view(rows, cols, t, place, float("nan"))
    X.copy_(x)
    return x.float().numpy(), X


def untouched(buf, X, fill):
    X.fill_(fill)
    return bool((buf == fill).all())


def near(got, want, bound, t):
    got = got.float().cpu().numpy().astype(np.float64)
    bound = bound + (np.abs(want) + bound) * HALF_ULP[t] + HALF_SMALLEST[t] + 1e-30
    assert (np.abs(got - want) <= bound).all()


@pytest.mark.parametrize("t", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("place", PLACES)
def test_quantize(q4, t, place):
    import torch
    for n, cols in enumerate(WIDTHS):
        for rows in (1, 5, 130):
            x, X = random(n, rows, cols, t, place)
            q, s = f8.quantize(x)
            qt, st = f8.quantize(np.ascontiguousarray(x.T))
            Q, S = torch.empty(rows, cols, dtype=torch.uint8, device="cuda"), torch.empty(*s.shape, device="cuda")
            Qt, St = torch.empty(cols, rows, dtype=torch.uint8, device="cuda"), torch.empty(*st.shape, device="cuda")
            q4.q4_f8_quantize(X, Q, S, Qt, St)
            assert (Q.cpu().numpy() == q).all() and (S.cpu().numpy() == s).all()
            assert (Qt.cpu().numpy() == qt).all() and (St.cpu().numpy() == st).all()
            source = np.array([rows - 1, -1, 0], dtype=np.int32)
            q, s = f8.quantize(np.where(source[:, None] >= 0, x[source], np.float32(0)))
            Q, S = torch.empty(3, cols, dtype=torch.uint8, device="cuda"), torch.empty(*s.shape, device="cuda")
            q4.q4_f8_quantize(X, Q, S, source=torch.from_numpy(source).cuda())
            assert (Q.cpu().numpy() == q).all() and (S.cpu().numpy() == s).all()


@pytest.mark.parametrize("t", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("place", PLACES)
@pytest.mark.parametrize("weighted", [False, True])
def test_rows_of_the_expert_layer(q4, t, place, weighted):
    import torch
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()
    other = PLACES[(PLACES.index(place) + 2) % len(PLACES)]
    for n, D in enumerate(WIDTHS):
        tokens, topk, E = (1, 1, 2) if n % 3 == 0 else (19, 3, 5) if n % 3 == 1 else (6, 9, 4)
        r = np.random.default_rng(n)
        ids = r.integers(-1, E, (tokens, topk)).astype(np.int32)
        rows = f8.sort_rows(ids.size, E, 16)
        starts, source, slot = f8.sort(ids, E, 16, rows)
        w = r.standard_normal((tokens, topk)).astype(np.float32) if weighted else None
        W, u = None if w is None else dev(w), None if w is None else np.abs(w)
        x, X = random(n + 100, tokens, D, t, place)
        y, Y = random(n + 200, rows, D, t, other)
        xs, Xs = view(rows, D, t, other, 7.0)
        out, Out = view(tokens, D, t, other, 7.0)
        dy, dY = view(rows, D, t, place, 7.0)
        dw = torch.full((tokens, topk), 7.0, device="cuda")
        q4.q4_expert_gather(X, dev(source), topk, Xs, W)
        want = f8.gather(x, source, topk, w)
        near(Xs, want, 2.0 ** -24 * np.abs(want), t)
        q4.q4_expert_combine(Y, dev(slot), W, Out)
        near(Out, f8.combine(y, slot, w), (topk + 1) * 2.0 ** -24 * f8.combine(np.abs(y), slot, u), t)
        q4.q4_expert_combine_grad(X, Y, dev(slot), W, dev(source), dY, dw)
        wy, ww = f8.combine_grad(x, y, slot, w)
        near(dY, wy, 2.0 ** -24 * np.abs(wy), t)
        near(dw, ww, (D + 1) * 2.0 ** -24 * f8.combine_grad(np.abs(x), np.abs(y), slot, w)[1], "f32")
        assert untouched(xs, Xs, 7.0) and untouched(out, Out, 7.0) and untouched(dy, dY, 7.0)


@pytest.mark.parametrize("t", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("place", PLACES)
@pytest.mark.parametrize("b_rows", [False, True])
def test_outputs_of_products(q4, t, place, b_rows):
    import torch
    for n, (M, N, K) in enumerate([(1, 9, 130), (40, 1, 200), (130, 67, 260), (300, 130, 100), (257, 255, 300), (97, 513, 384), (70, 200, 3000)]):
        r = np.random.default_rng(n)
        q = lambda rows, blocks: f8.quantize(r.standard_normal((rows, K)).astype(np.float32), blocks)
        (a, sa), (b, sb) = q(M, False), q(N, not b_rows)
        pad = lambda m: torch.from_numpy(np.pad(m, ((0, 0), (0, -K % 16)))).cuda()
        buf, C = view(M, N, t, place, 7.0)
        q4.q4_gemm_f8(pad(a), torch.from_numpy(sa).cuda(), pad(b), torch.from_numpy(sb).cuda(), C, M, N, K, b_rows=b_rows)
        want, mag = f8.product(a, sa, b, sb, b_rows)
        near(C, want, (130 + f8.blocks_of(K)) * 2.0 ** -24 * mag, t)
        assert untouched(buf, C, 7.0)
    assert q4.q4_last_device_status() == q4.Q4_OK
