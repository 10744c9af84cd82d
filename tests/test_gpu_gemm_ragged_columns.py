"""int32 products whose width is no multiple of four values while their rows begin on multiples of 16 bytes: what lies
between the rows, inside of the pitch, stays as it was.  Results bit for bit."""
import numpy as np
import pytest

import oracle
from paper_2009_06488_b200 import workloads as wl

pytestmark = pytest.mark.gpu
FILL = -1515870811


@pytest.fixture(scope="module")
def q4():
    from paper_2009_06488_b200 import binding
    yield binding
    binding.q4_set_variant(0)


def dev(a):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def columns(M, N):
    """A buffer whose first N columns are the product's; four spare rows behind it."""
    import torch
    return torch.full((M + 4, (N + 3) // 4 * 4 + 4), FILL, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("width", [5, 6])                  # tiles of 192 and of 256 columns
@pytest.mark.parametrize("N", [1, 2, 3, 5, 33, 191, 193, 255, 257, 385, 450, 513, 767])
@pytest.mark.parametrize("M", [70, 300, 513])
def test_four_bit_product(q4, width, M, N):
    K = 300
    c = wl.gemm_case("ragged", M, N, K, seed=M + N, lda=160, ldb=160)
    buf = columns(M, N)
    q4.q4_set_variant(width)
    q4.q4_gemm(dev(c.A), dev(c.Bt), buf[:M, :N], M, N, K, c.za, c.zb)
    assert q4.q4_last_device_status() == q4.Q4_OK
    out = buf.cpu().numpy()
    assert (out[:M, :N] == oracle.gemm(c.A, c.Bt, M, N, K, c.za, c.zb)).all()
    assert (out[M:] == FILL).all() and (out[:, N:] == FILL).all()


@pytest.mark.parametrize("N", [2341, 2342, 2343, 2344])
def test_four_bit_product_of_many_tiles(q4, N):
    M, K = 5000, 200
    c = wl.gemm_case("ragged", M, N, K, seed=N, lda=112, ldb=112)
    buf = columns(M, N)
    for width in (5, 6):
        buf.fill_(FILL)
        q4.q4_set_variant(width)
        q4.q4_gemm(dev(c.A), dev(c.Bt), buf[:M, :N], M, N, K, c.za, c.zb)
        out = buf.cpu().numpy()
        assert (out[:M, :N] == oracle.gemm(c.A, c.Bt, M, N, K, c.za, c.zb)).all()
        assert (out[M:] == FILL).all() and (out[:, N:] == FILL).all()


@pytest.mark.parametrize("N", [1289, 1290, 1291, 2333])
def test_eight_bit_product(q4, N):
    import torch
    M, K = 4100, 96
    A, Bt = wl.rand_bytes(N, 1, M * K).reshape(M, K), wl.rand_bytes(N, 2, N * K).reshape(N, K)
    buf = columns(M, N)
    ws = torch.empty(q4.q4_gemm_u8_workspace_bytes(M, N), dtype=torch.uint8, device="cuda")
    q4.q4_set_variant(0)
    q4.q4_gemm_u8(dev(A), dev(Bt), buf[:M, :N], M, N, K, 3, 200, None, None, ws)
    assert q4.q4_last_device_status() == q4.Q4_OK
    out = buf.cpu().numpy()
    assert (out[:M, :N] == oracle.gemm_u8(A, Bt, 3, 200)).all()
    assert (out[M:] == FILL).all() and (out[:, N:] == FILL).all()
