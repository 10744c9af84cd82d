"""Products behind a kernel that lets its successors start early and then runs on for longer than the products' bounded
waits last (about 2 s): a start beside its end may not count its running time, so nothing runs out and the results are
right.  The long kernel ends by itself: a limit on the clocks and one on its rounds.
"""
import ctypes
import os
import subprocess

import numpy as np
import pytest

from oracle import f8

pytestmark = pytest.mark.gpu
CLOCKS = 4_600_000_000               # the waits give up after 4e9

SOURCE = r"""
__global__ void run_on(long long clocks)
{
    asm volatile("griddepcontrol.launch_dependents;");
    const long long from = clock64();
    for (int i = 0; i < 6000000 && clock64() - from < clocks; ++i) __nanosleep(1000);
}
extern "C" int run_on_launch(long long clocks, void* stream)
{
    run_on<<<1, 1, 0, static_cast<cudaStream_t>(stream)>>>(clocks);
    return (int)cudaGetLastError();
}
"""


@pytest.fixture(scope="module")
def long_kernel(tmp_path_factory):
    d = tmp_path_factory.mktemp("long")
    (d / "run_on.cu").write_text(SOURCE)
    subprocess.check_call([os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc"), "-gencode", "arch=compute_100a,code=sm_100a", "-Xcompiler",
                           "-fPIC", "-shared", "-o", str(d / "run_on.so"), str(d / "run_on.cu")])
    call = ctypes.CDLL(str(d / "run_on.so")).run_on_launch
    call.argtypes = [ctypes.c_longlong, ctypes.c_void_p]
    return call


# a shared depth, one tile and six of a CTA pair, the kernel for few rows
@pytest.mark.parametrize("M,N,K", [(200, 250, 1024), (300, 520, 700), (4111, 5001, 300), (5, 300, 400)])
def test_product(long_kernel, M, N, K):
    import torch
    from paper_2009_06488_b200 import binding as q4
    r = np.random.default_rng(M)
    (a, sa), (b, sb) = (f8.quantize(r.standard_normal((n, K)).astype(np.float32), bl) for n, bl in ((M, False), (N, True)))
    put = lambda m: torch.from_numpy(np.pad(m, ((0, 0), (0, -m.shape[1] % 16)))).cuda()
    A, B, SA, SB = put(a), put(b), torch.from_numpy(sa).cuda(), torch.from_numpy(sb).cuda()
    C = torch.full((M, N), 7.0, device="cuda")
    q4.q4_gemm_f8(A, SA, B, SB, C, M, N, K)                       # the kernel is loaded
    C.fill_(7.0)
    torch.cuda.synchronize()
    assert q4.q4_last_device_status() == q4.Q4_OK
    assert long_kernel(CLOCKS, torch.cuda.current_stream().cuda_stream) == 0
    q4.q4_gemm_f8(A, SA, B, SB, C, M, N, K)
    torch.cuda.synchronize()
    assert q4.q4_last_device_status() == q4.Q4_OK
    want, mag = f8.product(a, sa, b, sb)
    assert (np.abs(C.double().cpu().numpy() - want) <= (130 + f8.blocks_of(K)) * 2.0 ** -24 * mag).all()
