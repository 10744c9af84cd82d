"""The experts' weight gradient where segments end: at a depth that is no multiple of 128, on starts that have to be
rounded down, and for experts without rows behind the last one that has some.

A segment is starts[e] .. starts[e + 1], cut to 0 .. K and to rising order; a value that is no multiple of 128 is
rounded down, K itself is not.  Bound: (128 + 2 + ceil(K / 128)) * 2^-24 of the terms' magnitudes, plus half of the
output's last place.
"""
import numpy as np
import pytest

from oracle import f8

pytestmark = pytest.mark.gpu

HALF_ULP = {"f32": 0.0, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
HALF_SMALLEST = {"f32": 2.0 ** -150, "bf16": 2.0 ** -134, "f16": 2.0 ** -25}


@pytest.fixture(scope="module")
def q4():
    from paper_2009_06488_b200 import binding
    yield binding
    binding.q4_set_variant(0)


def types():
    import torch
    return {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def whole_blocks(starts, K):
    """The segments' ends as the call understands them."""
    at = np.maximum.accumulate(np.clip(starts, 0, K))
    return np.where(at == K, K, at // 128 * 128)


@pytest.mark.parametrize("K,starts", [(200, [0, 200, 200]), (200, [0, 200, 200, 200, 200]), (200, [0, 0, 200, 200]),
                                      (200, [0, 300, 300, 1000]), (200, [0, 128, 200, 500, 200]), (200, [200, 200, 200]),
                                      (200, [0, 130, 200]), (700, [0, 255, 300, 513, 699]), (700, [5, 384, 384, 700, 700]),
                                      (65, [0, 64, 65, 65]), (1, [0, 0, 1, 1]), (1300, [0, 1300, 1300]), (256, [0, 256, 256])])
@pytest.mark.parametrize("M,N", [(40, 72), (200, 130), (300, 520)])
@pytest.mark.parametrize("variant", [0, 1, 2])
def test_segments_at_the_end_of_the_depth(q4, K, starts, M, N, variant):
    import torch
    r = np.random.default_rng(K + M)
    (a, sa), (b, sb) = (f8.quantize(r.standard_normal((n, K)).astype(np.float32)) for n in (M, N))
    pad = lambda m: torch.from_numpy(np.pad(m, ((0, 0), (0, -K % 16)))).cuda()
    E, starts = len(starts) - 1, np.array(starts, dtype=np.int32)
    want, mag = f8.experts_wgrad(a, sa, b, sb, whole_blocks(starts, K))
    t = ("f32", "bf16", "f16")[variant]
    C = torch.full((E * M + 1, N + 5), 7.0, dtype=types()[t], device="cuda")
    q4.q4_set_variant(variant)
    q4.q4_gemm_f8_experts_wgrad(pad(a), torch.from_numpy(sa).cuda(), pad(b), torch.from_numpy(sb).cuda(),
                                torch.from_numpy(starts).cuda(), C, M, N, K)
    got = C[:E * M, :N].float().cpu().numpy().astype(np.float64)
    bound = (130 + f8.blocks_of(K)) * 2.0 ** -24 * mag
    bound = bound + (np.abs(want) + bound) * HALF_ULP[t] + HALF_SMALLEST[t]
    assert (np.abs(got - want) <= bound).all()
    assert (C[E * M:] == 7).all() and (C[:, N:] == 7).all()
    assert q4.q4_last_device_status() == q4.Q4_OK
