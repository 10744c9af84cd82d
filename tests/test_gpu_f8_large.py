"""Matrices of more than 2^31 values: the e4m3 quantizer, its products and the expert layer's rows, at their ends.

Bounds as for the small sizes: codes and scales equal; a product of K terms off by at most
(128 + 2 + ceil(K / 128)) * 2^-24 of the terms' magnitudes, a combination of topk rows by (topk + 1) * 2^-24,
plus half of the output's last place (2^-8 of a bfloat16).
"""
import numpy as np
import pytest

from oracle import f8

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def q4():
    import torch
    from paper_2009_06488_b200 import binding
    yield binding
    torch.cuda.empty_cache()


def codes(seed, rows, cols):
    """Random e4m3 codes without NaN, on the GPU."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    c = torch.randint(0, 256, (rows, cols), dtype=torch.uint8, device="cuda", generator=g)
    return c.masked_fill_((c & 0x7F) == 0x7F, 0x3A)


def near(got, want, mag, K, half_ulp):
    got = got.double().cpu().numpy()
    bound = (128 + 2 + -(-K // 128)) * 2.0 ** -24 * mag
    assert (np.abs(got - want) <= bound + (np.abs(want) + bound) * half_ulp + 1e-30).all()


def test_product_and_quantizer_past_two_to_the_31(q4):
    import torch
    M, N, K = 66000, 33000, 130
    r = np.random.default_rng(1)
    A, B = codes(1, M, 144), codes(2, N, 144)
    sa, sb = (r.uniform(0.01, 1, s).astype(np.float32) for s in ((2, M), (-(-N // 128), 2)))
    SA, SB = torch.from_numpy(sa).cuda(), torch.from_numpy(sb).cuda()
    C = torch.empty(M, N, dtype=torch.bfloat16, device="cuda")
    q4.q4_gemm_f8(A, SA, B, SB, C, M, N, K)
    rows = np.array([0, M // 2, M - 257, M - 2, M - 1])
    want, mag = f8.product(A[rows, :K].cpu().numpy(), sa[:, rows], B[:, :K].cpu().numpy(), sb)
    near(C[rows], want, mag, K, 2.0 ** -8)
    # quantized both ways: whole rows of the last row block, whole columns at the end
    Q, S = torch.empty(M, N, dtype=torch.uint8, device="cuda"), torch.empty(-(-N // 128), M, device="cuda")
    Qt, St = torch.empty(N, M, dtype=torch.uint8, device="cuda"), torch.empty(-(-M // 128), N, device="cuda")
    q4.q4_f8_quantize(C, Q, S, Qt, St)
    q, s = f8.quantize(C[rows].float().cpu().numpy())
    assert (Q[rows].cpu().numpy() == q).all() and (S[:, rows].cpu().numpy() == s).all()
    cols = np.array([0, N - 300, N - 1])
    q, s = f8.quantize(np.ascontiguousarray(C[:, cols].float().cpu().numpy().T))
    assert (Qt[cols].cpu().numpy() == q).all() and (St[:, cols].cpu().numpy() == s).all()
    assert q4.q4_last_device_status() == q4.Q4_OK


@pytest.mark.parametrize("variant", [0, 1, 2])
def test_weights_of_experts_past_two_to_the_31(q4, variant):
    import torch
    E, N, K, M = 64, 16500, 2064, 100
    counts = np.zeros(E, dtype=int)
    counts[[0, 31, 62, 63]] = 3, 50, 17, 30
    starts = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
    r = np.random.default_rng(3)
    A, B = codes(3, M, K), codes(4, E * N, K)
    nkb, nnb = -(-K // 128), -(-N // 128)
    sa, sb = (r.uniform(0.01, 1, s).astype(np.float32) for s in ((nkb, M), (E * nnb, nkb)))
    C = torch.empty(M, N, device="cuda")
    try:
        q4.q4_set_variant(variant)
        q4.q4_gemm_f8_experts(A, torch.from_numpy(sa).cuda(), B, torch.from_numpy(sb).cuda(), torch.from_numpy(starts).cuda(),
                              C, M, N, K)
    finally:
        q4.q4_set_variant(0)
    for e in (0, 31, 62, 63):
        m = [int(starts[e]), int(starts[e + 1]) - 1]
        a, b = A[m].cpu().numpy(), B[e * N:(e + 1) * N].cpu().numpy()
        want, mag = f8.product(a, sa[:, m], b, sb[e * nnb:(e + 1) * nnb])
        near(C[m], want, mag, K, 0.0)
    assert q4.q4_last_device_status() == q4.Q4_OK


def test_rows_of_the_expert_layer_past_two_to_the_31(q4):
    import torch
    tokens, topk, D = 131700, 8, 2048
    pairs = tokens * topk
    assert pairs * D > 2 ** 31
    g = torch.Generator(device="cuda").manual_seed(5)
    source = torch.randperm(pairs, device="cuda", generator=g).to(torch.int32)
    slot = torch.empty(pairs, dtype=torch.int32, device="cuda")
    slot[source.long()] = torch.arange(pairs, dtype=torch.int32, device="cuda")
    slot = slot.view(tokens, topk)
    w = torch.randn(tokens, topk, device="cuda", generator=g)
    X = torch.randn(tokens, D, device="cuda", generator=g).to(torch.bfloat16)
    Y, dY = (torch.empty(pairs, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    q4.q4_expert_gather(X, source, topk, Y)
    last = torch.arange(pairs - 300, pairs, device="cuda")
    assert (Y[last] == X[source[last].long() // topk]).all()

    out = torch.empty(tokens, D, dtype=torch.bfloat16, device="cuda")
    q4.q4_expert_combine(Y, slot, w, out)
    some = torch.cat([torch.arange(50, device="cuda"), torch.arange(tokens - 50, tokens, device="cuda"),
                      source[last].long() // topk])
    terms = Y[slot[some].long()].double() * w[some].double()[:, :, None]
    want, mag = terms.sum(1), terms.abs().sum(1)
    bound = (topk + 1) * 2.0 ** -24 * mag
    assert ((out[some].double() - want).abs() <= bound + (want.abs() + bound) * 2.0 ** -8 + 1e-30).all()

    dw = torch.empty(tokens, topk, device="cuda")
    q4.q4_expert_combine_grad(X, Y, slot, w, source, dY, dw)
    want = w.view(-1)[source[last].long()].double()[:, None] * X[source[last].long() // topk].double()
    assert ((dY[last].double() - want).abs() <= (want.abs() * (2.0 ** -8 + 2.0 ** -24)) + 1e-30).all()
    terms = X[some].double()[:, None, :] * Y[slot[some].long()].double()
    assert ((dw[some].double() - terms.sum(2)).abs() <= (D + 1) * 2.0 ** -24 * terms.abs().sum(2)).all()
