"""The deepest product by experts: a depth whose end would outlast the kernels' bounded waits is refused before any launch."""
from test_abi_f4 import RANGE, fake, lib      # noqa: F401 (a fixture)


def test_experts_products_past_two_to_the_30(lib):      # noqa: F811
    def f(K, M=1):
        return lib.q4_gemm_f4_experts(fake, K, fake, 1, fake, K, fake, 1, 0, None, None, fake, 1, fake, 0, 1, M, 1, K, None)
    assert f(2 ** 30 + 1) == RANGE and f(2 ** 31 - 1000) == RANGE
    assert f(2 ** 30, M=0) == 0 and f(2 ** 31 - 1000, M=0) == 0
