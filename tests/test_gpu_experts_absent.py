"""Pairs and rows that are absent, in the expert layer's gradient and in gathers from no tokens at all.

dw of an absent pair is 0 and a row of no pair gets zeros, whatever the other operands hold.  A product of two
binary32 values is off by 2^-24 of itself, a sum of D of them by (D + 1) * 2^-24 of their magnitudes; the output's
type adds half of its last place.
"""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

HALF_ULP = {"f32": 0.0, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}


@pytest.fixture(scope="module")
def q4():
    from paper_2009_06488_b200 import binding
    return binding


def types():
    import torch
    return {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def dev(a):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


@pytest.mark.parametrize("t", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("D", [8, 40, 41, 100, 129, 264, 2048, 2051])
def test_rows_whose_pair_lies_past_the_end_get_zeros(q4, t, D):
    import torch
    tokens, topk = 4, 3
    pairs = tokens * topk
    # rows 0, 4 and 5 hold pairs; all others are absent, in one way or another
    source = np.array([3, pairs, -1, 2 ** 31 - 1, 11, 0, pairs + 1, -2 ** 31] + [pairs] * 40 + [-1], dtype=np.int32)
    slot = np.full((tokens, topk), -1, dtype=np.int32)
    slot[1, 0], slot[3, 2], slot[0, 0] = 0, 4, 5
    slot[2, 1], slot[0, 2] = source.size, 2 ** 31 - 1
    r = np.random.default_rng(D)
    w = r.standard_normal((tokens, topk)).astype(np.float32)
    G, Y = (dev(r.standard_normal((n, D)).astype(np.float32)).to(types()[t]) for n in (tokens, source.size))
    for weights in (w, None):
        dY = torch.full((source.size, D), float("nan"), dtype=types()[t], device="cuda")
        dw = torch.full((tokens, topk), float("nan"), device="cuda")
        q4.q4_expert_combine_grad(G, Y, dev(slot), None if weights is None else dev(weights), dev(source), dY, dw)
        want, ww = np.zeros((source.size, D)), np.zeros((tokens, topk))
        mag = np.zeros((tokens, topk))
        g, y = G.double().cpu().numpy(), Y.double().cpu().numpy()
        for row, tok, j in ((0, 1, 0), (4, 3, 2), (5, 0, 0)):
            want[row] = g[tok] * (1.0 if weights is None else float(weights[tok, j]))
            ww[tok, j], mag[tok, j] = (g[tok] * y[row]).sum(), np.abs(g[tok] * y[row]).sum()
        off = np.abs(dY.double().cpu().numpy() - want)
        assert (off <= np.abs(want) * (2.0 ** -24 + HALF_ULP[t] * (1 + 2.0 ** -24)) + 2.0 ** -25 * (t == "f16")).all()
        assert (np.abs(dw.double().cpu().numpy() - ww) <= (D + 1) * 2.0 ** -24 * mag).all()


@pytest.mark.parametrize("t", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("D", [1, 8, 13, 64, 65, 100, 121, 128, 200, 2048, 2051])
def test_weight_gradient_of_an_absent_pair_is_zero_beside_infinities(q4, t, D):
    import torch
    tokens, topk, rows = 9, 3, 20
    r = np.random.default_rng(D)
    # tokens in turn: all pairs absent, none, the first only present, the last only
    slot = np.full((tokens, topk), -1, dtype=np.int32)
    at = 0
    for i in range(tokens):
        for j in range(topk):
            if i % 4 == 1 or (i % 4 == 2 and j == 0) or (i % 4 == 3 and j == topk - 1):
                slot[i, j], at = at, at + 1
    assert at <= rows
    source = np.full(rows, -1, dtype=np.int32)
    source[slot[slot >= 0]] = np.flatnonzero(slot.reshape(-1) >= 0)
    G = dev(r.standard_normal((tokens, D)).astype(np.float32)).to(types()[t])
    G[0::4, 0], G[2::4, D - 1], G[3::4, D // 2] = float("inf"), float("nan"), float("-inf")
    Y = dev(r.standard_normal((rows, D)).astype(np.float32)).to(types()[t])
    w = dev(np.full((tokens, topk), np.nan, dtype=np.float32))
    w[dev(slot) >= 0] = 1.0
    dY, dw = torch.full_like(Y, 7.0), torch.full((tokens, topk), 7.0, device="cuda")
    q4.q4_expert_combine_grad(G, Y, dev(slot), w, dev(source), dY, dw)
    dw, dY = dw.cpu().numpy(), dY.cpu()
    assert (dw[slot < 0] == 0).all()
    assert np.isfinite(dw[1::4]).all() and not np.isfinite(dw[2::4, 0]).any() and not np.isfinite(dw[3::4, -1]).any()
    assert (dY[torch.from_numpy(source < 0)] == 0).all()
    rows_of = slot[slot >= 0]
    assert torch.equal(dY[torch.from_numpy(rows_of)].nan_to_num(5.0),
                       G.cpu()[torch.from_numpy(np.flatnonzero(slot.reshape(-1) >= 0) // topk)].nan_to_num(5.0))


@pytest.mark.parametrize("blocks", [False, True])
def test_rows_picked_from_no_tokens_are_zeros(q4, blocks):
    """Every entry of source is past the end of an empty matrix: absent, as with any other."""
    import torch
    X = torch.empty(0, 200, dtype=torch.bfloat16, device="cuda")
    source = torch.tensor([-1, 0, 5], dtype=torch.int32, device="cuda")
    Q, Qt = torch.full((3, 200), 9, dtype=torch.uint8, device="cuda"), torch.full((200, 3), 9, dtype=torch.uint8, device="cuda")
    S = torch.full((1, 2) if blocks else (2, 3), -1.0, device="cuda")
    St = torch.full((2, 1) if blocks else (1, 200), -1.0, device="cuda")
    q4.q4_f8_quantize(X, Q, S, Qt, St, blocks=blocks, source=source)
    least = np.float32(2.0 ** -60) / np.float32(448)
    assert (Q == 0).all() and (Qt == 0).all()
    assert (S.cpu().numpy() == least).all() and (St.cpu().numpy() == least).all()
    Xs = torch.full((3, 200), 7.0, dtype=torch.bfloat16, device="cuda")
    q4.q4_expert_gather(X, source, 1, Xs)
    assert (Xs == 0).all()
    # a matrix that has rows has to be given
    assert q4._lib.q4_f8_quantize(None, q4.Q4_BF16, 200, 3, 200, source.data_ptr(), 1, 1, int(blocks), Q.data_ptr(), 200,
                                  S.data_ptr(), S.shape[1], None, 0, None, 0, None) == q4.Q4_ERR_INVALID_ARG


@pytest.mark.parametrize("t", ["f32", "bf16"])
@pytest.mark.parametrize("D", [0, 40, 41])
def test_gradient_without_tokens_rows_or_values(q4, t, D):
    import torch
    new = lambda n: torch.full((n, D), 7.0, dtype=types()[t], device="cuda")
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
    dY, none = new(5), torch.empty(0, 2, device="cuda")
    q4.q4_expert_combine_grad(new(0), new(5), none.int(), None, i32([-1, 0, 3, 9, -5]), dY, none)
    assert (dY == 0).all()
    dw = torch.full((3, 2), 7.0, device="cuda")
    q4.q4_expert_combine_grad(new(3), new(0), i32([[0, -1], [3, 4], [-1, 7]]), None, i32([]), new(0), dw)
    assert (dw == 0).all()
    dw.fill_(7.0)
    dY = new(2)
    q4.q4_expert_combine_grad(new(3), new(2), i32([[0, -1], [-1, 1], [-1, -1]]), None, i32([0, 3]), dY, dw)
    assert (dY == 7).all()
    want = torch.zeros(3, 2)
    want[0, 0] = want[1, 1] = 49.0 * D
    assert torch.equal(dw.cpu(), want)
