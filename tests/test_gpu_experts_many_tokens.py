"""The expert layer's gradient of combining for more tokens than the blocks take in one round, against 64 bits on the GPU.

dY is a product of two binary32 values, rounded once (2^-24 of itself, plus half of the output's last place); dw a sum of
D products, off by at most (D + 1) * 2^-24 of their magnitudes.
"""
import pytest

pytestmark = pytest.mark.gpu

HALF_ULP = {"f32": 0.0, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
HALF_SMALLEST = {"f32": 2.0 ** -150, "bf16": 2.0 ** -134, "f16": 2.0 ** -25}


@pytest.fixture(scope="module")
def q4():
    import torch
    from paper_2009_06488_b200 import binding
    yield binding
    torch.cuda.empty_cache()


# (tokens, topk, D): rows that begin anywhere, 1 to 32 tokens in a block, up to five rounds and beyond; aligned rows
CASES = [(2219, 3, 2047), (2220, 3, 2047), (2500, 5, 2051), (4441, 3, 971), (35521, 3, 121), (71041, 3, 61), (71100, 3, 13),
         (71041, 1, 7), (2300, 9, 1030), (1000, 3, 2048), (900, 9, 520), (30000, 3, 64)]


@pytest.mark.parametrize("tokens,topk,D", CASES)
@pytest.mark.parametrize("t", ["f32", "bf16", "f16"])
def test_gradient_of_many_tokens(q4, tokens, topk, D, t):
    import torch
    kind = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}[t]
    g = torch.Generator(device="cuda").manual_seed(tokens + D)
    randn = lambda *s: torch.randn(*s, generator=g, device="cuda")
    pairs, rows = tokens * topk, tokens * topk + 37
    # every pair has a row of its own but one in eight, which are absent; rows in any order, some of no pair
    perm = torch.randperm(rows, generator=g, device="cuda")[:pairs].to(torch.int32)
    absent = torch.rand(pairs, generator=g, device="cuda") < 0.125
    slot = torch.where(absent, torch.full_like(perm, -1), perm)
    source = torch.full((rows,), -1, dtype=torch.int32, device="cuda")
    pair = torch.arange(pairs, dtype=torch.int32, device="cuda")
    source[slot[~absent].long()] = pair[~absent]
    slot = slot.view(tokens, topk)

    def matrix(n, values):
        m = torch.full((n, D + 3 if D % 8 else D), 7.0, dtype=kind, device="cuda")[:, :D]
        if values is not None:
            m.copy_(values)
        return m
    G, Y, w = matrix(tokens, randn(tokens, D)), matrix(rows, randn(rows, D)), randn(tokens, topk)
    dY, dw = matrix(rows, None), torch.full((tokens, topk), 7.0, device="cuda")
    q4.q4_expert_combine_grad(G, Y, slot, w, source, dY, dw)
    at = source.clamp(min=0).long()
    want = torch.where((source >= 0)[:, None], w.view(-1)[at].double()[:, None] * G[at // topk].double(), 0.0)
    bound = want.abs() * (2.0 ** -24 + HALF_ULP[t] * (1 + 2.0 ** -24)) + HALF_SMALLEST[t]
    assert ((dY.double() - want).abs() <= bound).all()
    for j in range(topk):
        has, terms = slot[:, j] >= 0, G.double() * Y[slot[:, j].clamp(min=0).long()].double()
        want = torch.where(has, terms.sum(1), 0.0)
        bound = torch.where(has, (D + 1) * 2.0 ** -24 * terms.abs().sum(1), 0.0)
        assert ((dw[:, j].double() - want).abs() <= bound).all()
    if D % 8:
        spare = dY.as_strided((rows, 3), (D + 3, 1), D)
        assert (spare == 7.0).all()
