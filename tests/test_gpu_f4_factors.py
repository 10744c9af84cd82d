"""Scales by 16 under factors at the ends of binary32's range: a matrix of zeros, whose factor is 0 by max |X| / 2688, and
matrices so small that the factor, or its inverse, leaves the normal range.  Codes and scales have to be the oracle's."""
import numpy as np
import pytest

from oracle import f4

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def q4():
    from paper_2009_06488_b200 import binding
    binding.q4_set_variant(0)
    return binding


def both_ways(q4, x, factor):
    """(codes, words, transposed codes, transposed words) of the GPU, checked against the oracle, and the factor there."""
    import torch
    X, F = torch.from_numpy(x).cuda(), torch.tensor([factor], device="cuda")
    want = (*f4.quantize(x, True, factor), *f4.quantize(np.ascontiguousarray(x.T), True, factor))
    got = [torch.empty(*a.shape, dtype=torch.uint8 if a.dtype == np.uint8 else torch.int32, device="cuda") for a in want]
    q4.q4_f4_quantize(X, *got, by16=True, factor=F)
    for g, w in zip(got, want):
        assert (g.cpu().numpy().view(w.dtype) == w).all()
    return (*got, F)


@pytest.mark.parametrize("rows,cols", [(1, 16), (130, 203), (256, 512)])
def test_zeros_are_zeros(q4, rows, cols):
    import torch
    x = np.zeros((rows, cols), dtype=np.float32)
    x[::3, ::2] = -0.0
    for factor in (np.float32(0), np.float32(1e-42), np.float32(1)):
        q, s, qt, st, F = both_ways(q4, x, factor)
        assert (q4.q4_f4_dequantize(q, s, torch.full((rows, cols), 9.0, device="cuda"), by16=True, factor=F) == 0).all()
        assert (q4.q4_f4_dequantize(qt, st, torch.full((cols, rows), 9.0, device="cuda"), by16=True, factor=F) == 0).all()
        b, sb = f4.quantize(np.ones((8, cols), dtype=np.float32), True)
        B, SB = torch.zeros(8, q.shape[1], dtype=torch.uint8, device="cuda"), torch.from_numpy(sb.view(np.int32)).cuda()
        B.copy_(torch.from_numpy(b))
        C = torch.full((rows, 8), 9.0, device="cuda")
        assert (q4.q4_gemm_f4(q, s, B, SB, C, rows, 8, cols, by16=True, FA=F) == 0).all()


@pytest.mark.parametrize("size", [1e-30, 1e-36, 2.0 ** -126, 2.0 ** -133, 2.0 ** -140, 2.0 ** -149])
def test_small_matrices_are_finite(q4, size):
    """max |X| / 2688 from a normal number down to 0, groups of zeros among them."""
    import torch
    r = np.random.default_rng(3)
    x = (r.standard_normal((140, 300)) * size).astype(np.float32)
    x[:16, :160] = 0
    factor = np.float32(np.abs(x).max() / np.float32(2688))
    q, s, qt, st, F = both_ways(q4, x, factor)
    y = q4.q4_f4_dequantize(q, s, torch.empty(140, 300, device="cuda"), by16=True, factor=F).cpu().numpy()
    assert np.isfinite(y).all() and (y[:16, :160] == 0).all()
    if size >= 1e-30:
        # half a step of e2m1 is a quarter of the value at most, or of the group's smallest code; scales round by 2^-4
        assert np.abs(y - x).max() <= 0.3 * np.abs(x).max()
