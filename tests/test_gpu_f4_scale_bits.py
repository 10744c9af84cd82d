"""Bit 7 of a scale by 16 has no meaning: products and the layer give the same bits with it and without, in every kernel."""
import numpy as np
import pytest

from test_gpu_f4 import check, operand, placed, up16, word_tensor
from test_gpu_f4_layer import Case

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def q4():
    from paper_2009_06488_b200 import binding
    binding.q4_set_variant(0)
    return binding


def marked(words, seed):
    """Bit 7 of about half the bytes set."""
    import torch
    r = np.random.default_rng(seed)
    bits = (r.integers(0, 2, (*words.shape, 4)) << np.array([7, 15, 23, 31])).sum(axis=2).astype(np.uint32)
    return words | torch.from_numpy(bits.view(np.int32)).cuda()


@pytest.mark.parametrize("M,N,K", [(5, 300, 400), (5, 300, 4096), (20, 20000, 512), (300, 520, 700), (2500, 2048, 300)])
def test_products(q4, M, N, K):
    """Few rows, few rows with the depth in parts, many tiles of them, pairs on narrow and wide tiles; the general kernel."""
    import torch
    (a, sa, va), (b, sb, vb) = operand(M, M, K, True), operand(N + 1, N, K, True)
    want = (va @ vb.T, np.abs(va) @ np.abs(vb).T)
    for pitch in (up16, lambda w: up16(w) + 1):
        A, B, SA, SB = placed(a, pitch(a.shape[1])), placed(b, pitch(b.shape[1])), word_tensor(sa), word_tensor(sb)
        plain, C = torch.full((M, N), 9.0, device="cuda"), torch.full((M, N), 8.0, device="cuda")
        q4.q4_gemm_f4(A, SA, B, SB, plain, M, N, K, by16=True)
        q4.q4_gemm_f4(A, marked(SA, 1), B, marked(SB, 2), C, M, N, K, by16=True)
        check(plain, *want, K, "f32", extra=4)
        assert torch.equal(C, plain)


@pytest.mark.parametrize("D", [256, 203])
def test_read_back_and_layer(q4, D):
    import torch
    c = Case(91, 5, 2, 4, D, 96, True, True, "bf16")
    c.run(q4).check()
    plain = c.Out.clone()
    assert torch.equal(q4.q4_f4_dequantize(c.W1, marked(c.S1, 3), torch.empty(c.W1.shape[0], D, device="cuda"), by16=True),
                       q4.q4_f4_dequantize(c.W1, c.S1, torch.empty(c.W1.shape[0], D, device="cuda"), by16=True))
    c.S1, c.S2 = marked(c.S1, 4), marked(c.S2, 5)
    c.run(q4)
    assert torch.equal(c.Out, plain)
