"""Products on tiles of 256 columns and products by experts' depth whose depth several CTA pairs share.

Which tiles a call gets is decided by estimated clocks: with 74 pairs, wide ones where they go round once and narrow
ones (128 columns) twice, as in every shape of the first three tests; a depth is shared where few narrow tiles have
six blocks of 128 or more each, as in the last.  Bound: (128 + 2 + ceil(K / 128)) * 2^-24 of the terms' magnitudes,
plus half of the output's last place.
"""
import numpy as np
import pytest

from oracle import f8

pytestmark = pytest.mark.gpu

HALF_ULP = {"f32": 0.0, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
HALF_SMALLEST = {"f32": 2.0 ** -150, "bf16": 2.0 ** -134, "f16": 2.0 ** -25}
PLACES = [(0, 0), (0, 3), (1, 0), (3, 5)]              # elements before the first row; behind each row, beside an aligned pitch


@pytest.fixture(scope="module")
def q4():
    from paper_2009_06488_b200 import binding
    binding.q4_set_variant(0)
    return binding


def types():
    import torch
    return {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def operand(seed, rows, cols, blocks=False):
    """Codes and scales, on the host and on the GPU (rows on multiples of 16 bytes)."""
    import torch
    q, s = f8.quantize(np.random.default_rng(seed).standard_normal((rows, cols)).astype(np.float32), blocks)
    return q, s, torch.from_numpy(np.pad(q, ((0, 0), (0, -cols % 16)))).cuda(), torch.from_numpy(s).cuda()


def output(rows, N, t, place):
    import torch
    off, pad = place
    pitch = (N + 7) // 8 * 8 + pad
    buf = torch.full((off + rows * pitch,), 7.0, dtype=types()[t], device="cuda")
    return buf, buf[off:].as_strided((rows, N), (pitch, 1))


def check(buf, C, want, mag, K, t):
    got = C.float().cpu().numpy().astype(np.float64)
    bound = (130 + f8.blocks_of(K)) * 2.0 ** -24 * mag
    bound = bound + (np.abs(want) + bound) * HALF_ULP[t] + HALF_SMALLEST[t]
    assert (np.abs(got - want) <= bound).all()
    C.fill_(7.0)
    assert (buf == 7.0).all()


@pytest.mark.parametrize("M,N,K", [(1990, 2301, 333), (2048, 2300, 128), (1793, 2177, 700)])
@pytest.mark.parametrize("b_rows", [False, True])
def test_dense(q4, M, N, K, b_rows):
    a, sa, A, SA = operand(M, M, K)
    b, sb, B, SB = operand(N + 1, N, K, not b_rows)
    want, mag = f8.product(a, sa, b, sb, b_rows)
    for t in ("f32", "bf16", "f16"):
        for place in PLACES:
            buf, C = output(M, N, t, place)
            q4.q4_gemm_f8(A, SA, B, SB, C, M, N, K, b_rows=b_rows)
            check(buf, C, want, mag, K, t)
    assert q4.q4_last_device_status() == q4.Q4_OK


@pytest.mark.parametrize("counts", [[1300, 0, 1700], [0, 2999, 1]])
def test_rows_of_experts(q4, counts):
    import torch
    N, K = 1290, 333
    starts = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
    E, M = len(counts), int(starts[-1])
    a, sa, A, SA = operand(1, M, K)
    parts = [f8.quantize(np.random.default_rng(e + 5).standard_normal((N, K)).astype(np.float32), True) for e in range(E)]
    b, sb = np.concatenate([p[0] for p in parts]), np.concatenate([p[1] for p in parts])
    B, SB = torch.from_numpy(np.pad(b, ((0, 0), (0, -K % 16)))).cuda(), torch.from_numpy(sb).cuda()
    want, mag = f8.experts(a, sa, b, sb, starts, N)
    for t in ("f32", "bf16", "f16"):
        for place in PLACES:
            buf, C = output(M, N, t, place)
            q4.q4_gemm_f8_experts(A, SA, B, SB, torch.from_numpy(starts).cuda(), C, M, N, K)
            check(buf, C, want, mag, K, t)
    assert q4.q4_last_device_status() == q4.Q4_OK


def by_depth(q4, M, N, K, starts):
    import torch
    a, sa, A, SA = operand(M, M, K)
    b, sb, B, SB = operand(N + 1, N, K)
    at = np.where(np.array(starts) == K, K, np.array(starts) // 128 * 128)
    E = len(starts) - 1
    want, mag = f8.experts_wgrad(a, sa, b, sb, at)
    for t in ("f32", "bf16", "f16"):
        for place in PLACES:
            buf, C = output(E * M, N, t, place)
            q4.q4_gemm_f8_experts_wgrad(A, SA, B, SB, torch.tensor(starts, dtype=torch.int32, device="cuda"), C, M, N, K)
            check(buf, C, want, mag, K, t)
    assert q4.q4_last_device_status() == q4.Q4_OK


@pytest.mark.parametrize("starts,K", [([0, 256, 256, 700], 700), ([128, 384, 512, 512], 640), ([0, 200, 300, 641], 641)])
def test_depths_of_experts(q4, starts, K):
    by_depth(q4, 700, 1100, K, starts)


@pytest.mark.parametrize("M,N", [(86, 209), (40, 72), (130, 128), (256, 300)])
@pytest.mark.parametrize("starts,K", [([0, 384, 384, 2900, 3050], 3050), ([0, 5, 2944], 2944), ([128, 128, 256, 3000], 3200),
                                      ([0, 128, 384, 768, 4000, 4100], 4100)])
def test_shared_depths_of_experts(q4, M, N, starts, K):
    by_depth(q4, M, N, K, starts)
