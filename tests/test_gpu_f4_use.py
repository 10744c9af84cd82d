"""4-bit float operators as programs use them: in captured graphs, on several streams at once, right behind the kernels that
make their inputs, far into large buffers, and at the limits of the expert layer."""
import numpy as np
import pytest

from oracle import f4
from test_gpu_f4 import check, operand, placed, up16, word_tensor
from test_gpu_f4_layer import Case
from test_gpu_f8_behind_a_long_kernel import CLOCKS, long_kernel      # noqa: F401 (a fixture)

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def q4():
    from paper_2009_06488_b200 import binding
    binding.q4_set_variant(0)
    return binding


def empty_codes(rows, cols, by16):
    import torch
    return (torch.empty(rows, up16(-(-cols // 2)), dtype=torch.uint8, device="cuda"),
            torch.empty(f4.words_of(cols, by16), rows, dtype=torch.int32, device="cuda"))


def chain(q4, M, N, K, by16, seed):
    """x and w to codes, their product, and both gradients' products from the transposed codes; returns (call, results)."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    x, w, dy = (torch.randn(s, generator=g, device="cuda").bfloat16() for s in ((M, K), (N, K), (M, N)))
    x4, xt, w4, wt, d4, dt = (empty_codes(r, c, by16) for r, c in ((M, K), (K, M), (N, K), (K, N), (M, N), (N, M)))
    y, dx, dw = (torch.empty(s, device="cuda") for s in ((M, N), (M, K), (N, K)))

    def call():
        q4.q4_f4_quantize(x, *x4, *xt, by16=by16)
        q4.q4_f4_quantize(w, *w4, *wt, by16=by16)
        q4.q4_f4_quantize(dy, *d4, *dt, by16=by16)
        q4.q4_gemm_f4(x4[0], x4[1], w4[0], w4[1], y, M, N, K, by16=by16)
        q4.q4_gemm_f4(d4[0], d4[1], wt[0], wt[1], dx, M, K, N, by16=by16)
        q4.q4_gemm_f4(dt[0], dt[1], xt[0], xt[1], dw, N, K, M, by16=by16)
    return call, (x, w, dy), (y, dx, dw)


def host(m, by16):
    """What the quantizer makes of a matrix, in 64 bits."""
    q, s = f4.quantize(m.float().cpu().numpy(), by16)
    return f4.values(q, s, m.shape[1], by16)


@pytest.mark.parametrize("by16", [False, True])
@pytest.mark.parametrize("M,N,K", [(1, 200, 1000), (130, 257, 391), (640, 512, 777)])
def test_forward_and_both_gradients(q4, by16, M, N, K):
    call, (x, w, dy), (y, dx, dw) = chain(q4, M, N, K, by16, M)
    call()
    for got, a, b, depth in ((y, x, w, K), (dx, dy, w.t().contiguous(), N), (dw, dy.t().contiguous(), x.t().contiguous(), M)):
        want, mag = f4.product(host(a, by16), host(b, by16))
        check(got, want, mag, depth, "f32", extra=8)


def test_a_captured_chain_follows_its_inputs(q4):
    """One graph of the six calls, replayed on new inputs behind the copies that bring them; a second graph of the same
    buffers between the replays."""
    import torch
    call, ins, outs = chain(q4, 300, 500, 2048, True, 1)
    side = torch.cuda.Stream()
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    with torch.cuda.stream(side):
        call()
    side.synchronize()
    for gr in graphs:
        with torch.cuda.graph(gr):
            call()
    for k in range(4):
        new = [torch.randn(t.shape, generator=torch.Generator(device="cuda").manual_seed(10 + k), device="cuda").bfloat16() for t in ins]
        for t, n in zip(ins, new):
            t.copy_(n)
        graphs[k & 1].replay()
        replayed = [t.clone() for t in outs]
        for t in outs:
            t.fill_(7)
        call()
        assert all(torch.equal(a, b) for a, b in zip(replayed, outs))


def test_streams_at_once_and_behind_long_kernels(q4):
    """Chains on two streams, each behind work that has not finished when the calls are made, give what they give alone."""
    import torch
    chains = [chain(q4, *s, b, 3) for s, b in (((64, 4096, 2048), True), ((900, 1100, 640), False))]
    want = []
    for call, _, outs in chains:
        call()
        want.append([t.clone() for t in outs])
    big = torch.randn(4096, 4096, device="cuda")
    streams = [torch.cuda.Stream() for _ in chains]
    torch.cuda.synchronize()
    for _ in range(5):
        for st, (call, ins, outs) in zip(streams, chains):
            with torch.cuda.stream(st):
                keep = [t.clone() for t in ins]
                for t in (*ins, *outs):
                    t.zero_()
                big @ big
                for t, k in zip(ins, keep):
                    t.copy_(k)
                call()
    torch.cuda.synchronize()
    for (_, _, outs), ref in zip(chains, want):
        assert all(torch.equal(a, b) for a, b in zip(outs, ref))


def far(rows, cols, pitch, dtype):
    import torch
    return torch.empty((rows - 1) * pitch + cols, dtype=dtype, device="cuda").as_strided((rows, cols), (pitch, 1))


def test_offsets_past_32_bits(q4):
    """Rows a gigabyte apart, in what is read and in what is written."""
    import torch
    P = 2 ** 30 + 16
    x = far(4, 200, P, torch.bfloat16)
    x.copy_(torch.randn(4, 200, device="cuda"))
    q = far(4, 100, P, torch.uint8)
    s = torch.empty(f4.words_of(200, False), 4, dtype=torch.int32, device="cuda")
    q4.q4_f4_quantize(x, q, s)
    wq, ws = f4.quantize(x.float().cpu().numpy())
    assert (q.cpu().numpy() == wq).all() and (s.cpu().numpy().view(np.uint32) == ws).all()
    y = far(4, 200, P, torch.bfloat16)
    q4.q4_f4_dequantize(q, s, y)
    v = f4.values(wq, ws, 200)
    assert (y.double().cpu().numpy() == v).all()             # 2 bits times a power of two: exact
    del x, y
    b, sb, vb = operand(5, 130, 200, False)
    B, SB = placed(b, up16(100)), word_tensor(sb)
    c = far(4, 130, P, torch.bfloat16)
    want, mag = f4.product(v, vb)
    q4.q4_gemm_f4(q, s, B, SB, c, 4, 130, 200)
    check(c, want, mag, 200, "bf16")
    wide = far(130, 4, 2 ** 25, torch.float32)                # the long rows as weights
    q4.q4_gemm_f4(B, SB, q, s, wide, 130, 4, 200)
    check(wide, want.T, mag.T, 200, "f32")
    try:
        q4.q4_set_variant(1)
        c.zero_()
        q4.q4_gemm_f4(q, s, B, SB, c, 4, 130, 200)
        check(c, want, mag, 200, "bf16")
    finally:
        q4.q4_set_variant(0)


def test_weights_of_experts_past_32_bits(q4):
    """2.5 GiB of weights' rows: the last experts' begin behind 2^31 bytes."""
    import torch
    E, N, K, P = 20, 128, 96, 2 ** 20
    b, sb, vb = operand(7, E * N, K, True)
    B = far(E * N, K // 2, P, torch.uint8)
    B.copy_(torch.from_numpy(b))
    a, sa, va = operand(8, 2 * E, K, True)
    starts = (2 * np.arange(E + 1)).astype(np.int32)
    want, mag = f4.experts(va, vb, starts, N)
    C = torch.empty(2 * E, N, device="cuda")
    q4.q4_gemm_f4_experts(placed(a, 48), word_tensor(sa), B, word_tensor(sb), torch.from_numpy(starts).cuda(), C, 2 * E, N, K, by16=True)
    check(C, want, mag, K, "f32")


@pytest.mark.parametrize("counts", [[1] * 1024, [0] * 1023 + [300], [70] * 3 + [0] * 1000 + [5]])
def test_as_many_experts_as_there_may_be(q4, counts):
    import torch
    E, N, K = len(counts), 40, 64
    starts = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
    M = int(starts[-1])
    a, sa, va = operand(9, M, K, False)
    b, sb, vb = operand(10, E * N, K, False)
    want, mag = f4.experts(va, vb, starts, N)
    C = torch.empty(M, N, device="cuda")
    q4.q4_gemm_f4_experts(placed(a), word_tensor(sa), placed(b), word_tensor(sb), torch.from_numpy(starts).cuda(), C, M, N, K)
    check(C, want, mag, K, "f32")


@pytest.mark.parametrize("T,topk", [(1024, 1), (1025, 1), (32, 32), (1, 1024), (103, 10)])
def test_layer_at_its_largest_lists(q4, T, topk):
    """1024 pairs are the most that the streaming kernels sort; a token may name the same expert again and again."""
    Case(T + topk, T, topk, 5, 64, 48, True, topk > 1, "bf16").run(q4).check()


@pytest.mark.parametrize("D,H,by16", [(8704, 200, False), (7168, 256, True), (300, 8704, False), (4608, 130, False), (7169, 130, True), (5000, 6401, True)])
def test_layer_of_the_widest_tokens(q4, D, H, by16):
    """Depths at which one unit's activations fill shared memory, and the first that do not fit."""
    Case(D, 5, 2, 3, D, H, True, by16, "bf16").run(q4).check()


def test_layer_of_as_many_experts_as_there_may_be(q4):
    Case(51, 7, 4, 1024, 64, 32, True, True, "f16").run(q4).check()


def test_layers_in_turn_share_a_workspace(q4):
    """Calls one behind the other on a stream, of different sizes, in one workspace; each reads what the one before wrote."""
    import torch
    cases = [Case(60 + i, T, 2, 4, D, H, i & 1 == 1, False, "bf16") for i, (T, D, H) in enumerate(((16, 256, 128), (2, 640, 64), (9, 96, 320)))]
    ws = max((c.ws(q4) for c in cases), key=lambda t: t.numel())
    for _ in range(3):
        for c in cases:
            c.run(q4, ws=ws)
    for c in cases:
        c.check()
    # a layer on the last one's result, without a wait between
    c = Case(70, 16, 2, 4, 256, 256, True, True, "bf16")
    ids, w = torch.from_numpy(c.ids).cuda(), torch.from_numpy(c.w).cuda()

    def layers(sync):
        h = c.X.clone()
        for _ in range(4):
            out = torch.full_like(h, 5)
            q4.q4_expert_layer_f4(h, ids, w, c.W1, c.S1, c.W2, c.S2, out, c.E, c.H, c.ws(q4), gated=True, by16=True, F1=c.F1, F2=c.F2)
            if sync:
                torch.cuda.synchronize()
            h = out
        return h
    assert torch.equal(layers(False), layers(True))


def test_behind_a_kernel_that_outlasts_the_waits(q4, long_kernel):      # noqa: F811
    """The bounded waits inside the kernels begin when their inputs are there, not when an early start lets them in."""
    import torch

    def behind(call, out):
        call()
        out.fill_(7)
        torch.cuda.synchronize()
        assert q4.q4_last_device_status() == q4.Q4_OK
        assert long_kernel(CLOCKS, torch.cuda.current_stream().cuda_stream) == 0
        call()
        torch.cuda.synchronize()
        assert q4.q4_last_device_status() == q4.Q4_OK
    for M, N, K in ((5, 300, 400), (5, 300, 4096), (300, 520, 700), (2500, 2048, 300)):      # few rows, depth in parts, pairs: narrow and wide
        a, sa, va = operand(M, M, K, False)
        b, sb, vb = operand(N, N, K, False)
        A, SA, B, SB = placed(a, up16(a.shape[1])), word_tensor(sa), placed(b, up16(b.shape[1])), word_tensor(sb)
        C = torch.empty(M, N, device="cuda")
        behind(lambda: q4.q4_gemm_f4(A, SA, B, SB, C, M, N, K), C)
        want, mag = f4.product(va, vb)
        check(C, want, mag, K, "f32", extra=4)
    c = Case(71, 16, 4, 8, 512, 256, True, True, "bf16")
    ids, w, ws = torch.from_numpy(c.ids).cuda(), torch.from_numpy(c.w).cuda(), c.ws(q4)
    behind(lambda: q4.q4_expert_layer_f4(c.X, ids, w, c.W1, c.S1, c.W2, c.S2, c.Out, c.E, c.H, ws, gated=True, by16=True, F1=c.F1, F2=c.F2), c.Out)
    c.check()
