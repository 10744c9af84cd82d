"""The expert layer for a few tokens on 4-bit weights, on the GPU against the 64-bit oracle.

The bound is the oracle's count of roundings (oracle/f4.py: layer) and half a last place of the output's type."""
import numpy as np
import pytest

from oracle import f4
from test_gpu_f4 import HALF_SMALLEST, HALF_ULP, placed, types, up16, word_tensor

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def q4():
    from paper_2009_06488_b200 import binding
    binding.q4_set_variant(0)
    return binding


class Case:
    """Inputs on both sides.  Weights carry scales of their own per group and a factor per expert."""

    def __init__(self, seed, T, topk, E, D, H, gated, by16, t, pad=0, pitch=up16, spread=1.0):
        import torch
        r = np.random.default_rng(seed)
        self.a = (T, topk, E, D, H, gated, by16, t)
        up = (2 if gated else 1) * H
        self.E, self.D, self.H, self.gated, self.by16 = E, D, H, gated, by16
        f1, f2 = (r.uniform(0.5, 2, E).astype(np.float32) for _ in range(2))
        x = (r.standard_normal((T, D)) * spread ** r.standard_normal((T, D))).astype(np.float32)
        self.X = placed(x, D + pad, pad).to(types()[t]) if pad == 0 else None
        if pad:
            buf = torch.full((pad + T * (D + pad),), float("nan"), device="cuda", dtype=types()[t])
            self.X = buf[pad:].as_strided((T, D), (D + pad, 1))
            self.X.copy_(torch.from_numpy(x))
        self.x = self.X.double().cpu().numpy()
        self.ids = np.stack([r.permutation(E)[:topk] if topk <= E else r.integers(0, E, topk) for _ in range(T)]).astype(np.int32) if T else \
            np.zeros((0, topk), dtype=np.int32)
        self.w = r.uniform(0, 1, (T, topk)).astype(np.float32)
        (q1, s1), (q2, s2) = (f4.quantize((r.standard_normal((E * n, k)) * k ** -0.5 * np.exp(0.5 * r.standard_normal((E * n, 1)))), by16)
                              for n, k in ((up, D), (D, H)))
        self.w1 = f4.values(q1, s1, D, by16).reshape(E, up, D) * f1[:, None, None].astype(np.float64)
        self.w2 = f4.values(q2, s2, H, by16).reshape(E, D, H) * f2[:, None, None].astype(np.float64)
        self.W1, self.W2 = (placed(q, pitch(q.shape[1]), 16 if pitch is up16 else 1) for q in (q1, q2))
        self.S1, self.S2 = word_tensor(s1, 1), word_tensor(s2)
        self.F1, self.F2 = torch.from_numpy(f1).cuda(), torch.from_numpy(f2).cuda()
        self.Out = torch.full((T, D + pad), 9.0, dtype=types()[t], device="cuda")

    def ws(self, q4):
        import torch
        T, topk = self.ids.shape
        return torch.full((max(256, q4.q4_expert_layer_f4_workspace_bytes(T, topk, self.D, self.H)),), 0xFF, dtype=torch.uint8, device="cuda")

    def run(self, q4, ids=None, w="own", ws=None):
        import torch
        T, topk = self.ids.shape
        self.ids = self.ids if ids is None else ids
        self.w = None if w is None else self.w
        q4.q4_expert_layer_f4(self.X, torch.from_numpy(self.ids).cuda(), None if w is None else torch.from_numpy(self.w).cuda(), self.W1,
                              self.S1, self.W2, self.S2, self.Out[:, :self.D], self.E, self.H, self.ws(q4) if ws is None else ws,
                              gated=self.gated, by16=self.by16, F1=self.F1, F2=self.F2)
        return self

    def check(self):
        want, off = f4.layer(self.x, self.ids, self.w, self.w1, self.w2, self.gated)
        t = self.a[-1]
        got = self.Out[:, :self.D].double().cpu().numpy()
        bound = off + (np.abs(want) + off) * HALF_ULP[t] + HALF_SMALLEST[t]
        bad = ~(np.abs(got - want) <= bound)
        assert not bad.any(), f"{bad.sum()} of {bad.size}, first at {np.argwhere(bad)[0]}: {got[bad][0]} for {want[bad][0]} +- {bound[bad][0]}"
        assert (self.Out[:, self.D:] == 9).all()


@pytest.mark.parametrize("by16", [False, True])
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("T,topk,E,D,H,t", [
    (1, 1, 1, 1, 1, "bf16"), (1, 2, 4, 64, 32, "f16"), (1, 8, 16, 1024, 256, "bf16"), (3, 2, 8, 100, 33, "bf16"), (16, 4, 8, 512, 384, "bf16"),
    (5, 1, 3, 1362, 719, "f16"), (40, 2, 4, 256, 200, "bf16"), (17, 3, 5, 320, 130, "f32"), (9, 2, 2, 2048, 96, "bf16"), (2, 3, 2, 96, 64, "f16")])
def test_layer(q4, by16, gated, T, topk, E, D, H, t):
    Case(T + D, T, topk, E, D, H, gated, by16, t).run(q4).check()


def test_layer_wide_and_many_tokens(q4):
    Case(1, 3, 2, 3, 7168, 2048, True, True, "bf16").run(q4).check()
    Case(2, 2, 2, 2, 640, 5000, False, False, "bf16").run(q4).check()
    Case(3, 2, 2, 2, 20000, 40, True, False, "bf16").run(q4).check()
    Case(4, 200, 4, 6, 160, 96, True, True, "bf16").run(q4).check()


@pytest.mark.parametrize("by16", [False, True])
def test_rows_anywhere(q4, by16):
    Case(6, 5, 2, 4, 203, 77, True, by16, "bf16", pad=3).run(q4).check()
    Case(7, 5, 2, 4, 203, 77, True, by16, "f16", pad=5, pitch=lambda w: w + 1).run(q4).check()
    Case(8, 5, 2, 4, 256, 128, True, by16, "bf16", pad=3, pitch=lambda w: w + 16).run(q4).check()


def test_dropped_and_repeated_pairs(q4):
    c = Case(11, 6, 3, 4, 192, 96, True, True, "bf16")
    ids = np.array([[0, 0, 0], [-1, -1, -1], [4, -7, 2 ** 31 - 1], [3, 3, 1], [2, -1, 2], [1, 2, 3]], dtype=np.int32)
    c.run(q4, ids).check()
    assert (c.Out[1:3] == 0).all()
    c = Case(12, 6, 3, 4, 192, 96, True, False, "bf16")
    c.run(q4, np.full((6, 3), -1, dtype=np.int32)).check()
    assert (c.Out == 0).all()
    Case(13, 6, 3, 4, 192, 96, True, False, "bf16").run(q4, w=None).check()


def test_values_of_any_size(q4):
    """Rows whose values span many powers of two keep the oracle's bound."""
    for t, spread in (("bf16", 30.0), ("f16", 4.0), ("f32", 30.0)):
        c = Case(21, 8, 2, 4, 512, 128, False, False, t, spread=spread)
        c.run(q4).check()


def test_an_infinity_or_a_nan_stays_in_its_token(q4):
    import torch
    c = Case(22, 5, 2, 4, 256, 64, True, True, "bf16")
    c.run(q4)
    clean = c.Out.clone()
    c.X[1, 17], c.X[3, 200] = float("inf"), float("nan")
    c.run(q4)
    assert torch.equal(c.Out[[0, 2, 4]], clean[[0, 2, 4]])
    assert not torch.isfinite(c.Out[1]).any() and not torch.isfinite(c.Out[3]).any()


def test_same_bits_every_time_on_any_stream_and_in_a_graph(q4):
    import torch
    c = Case(31, 16, 4, 8, 1024, 512, True, True, "bf16")
    ws = c.ws(q4)
    c.run(q4, ws=ws).check()
    first = c.Out.clone()
    ids, w = torch.from_numpy(c.ids).cuda(), torch.from_numpy(c.w).cuda()

    def call(out, ws):
        q4.q4_expert_layer_f4(c.X, ids, w, c.W1, c.S1, c.W2, c.S2, out, c.E, c.H, ws, gated=True, by16=True, F1=c.F1, F2=c.F2)
    for _ in range(20):
        c.Out.fill_(3)
        call(c.Out, ws)
        assert torch.equal(c.Out, first)
    # two streams with workspaces of their own, and a graph replayed on new inputs
    outs, wss, streams = [torch.empty_like(first) for _ in range(2)], [c.ws(q4) for _ in range(2)], [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(10):
        for o, s, st in zip(outs, wss, streams):
            with torch.cuda.stream(st):
                call(o, s)
    torch.cuda.synchronize()
    assert torch.equal(outs[0], first) and torch.equal(outs[1], first)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(c.Out, ws)
    for k in range(3):
        ids.copy_(torch.from_numpy(np.roll(c.ids, 3 * k, axis=0)))
        graph.replay()
        eager = torch.empty_like(first)
        call(eager, c.ws(q4))
        torch.cuda.synchronize()
        assert torch.equal(c.Out, eager)


def test_refusals(q4):
    import torch
    c = Case(41, 2, 2, 4, 64, 32, True, False, "bf16")
    ids, w, ws = torch.from_numpy(c.ids).cuda(), torch.from_numpy(c.w).cuda(), c.ws(q4)

    def call(X=c.X, ids=ids, w=w, W1=c.W1, S1=c.S1, W2=c.W2, S2=c.S2, Out=c.Out, E=4, H=32, ws=ws, gated=True, F1=None):
        q4.q4_expert_layer_f4(X, ids, w, W1, S1, W2, S2, Out, E, H, ws, gated=gated, F1=F1)
    call()
    for bad in (dict(ids=ids[:1]), dict(w=w[:1]), dict(W1=c.W1[:-1]), dict(S1=c.S1[:, :-2]), dict(Out=c.Out.float()), dict(E=5), dict(H=33),
                dict(F1=c.F1[:3]), dict(ids=ids.view(-1))):
        with pytest.raises(ValueError):
            call(**bad)
    for bad in (dict(ids=ids.long()), dict(w=w.double()), dict(W1=c.W1.view(torch.int8)), dict(S2=c.S2.float())):
        with pytest.raises(TypeError):
            call(**bad)
    for bad in (dict(ws=ws[:64]), dict(ws=ws[1:])):
        with pytest.raises(q4.Q4Error):
            call(**bad)
    torch.cuda.synchronize()


def test_quantized_weights_serve_both_ways(q4):
    """Weights through the quantizer; a batch through sort, pick + quantize, product by experts, activation, quantize,
    product, combine; the same tokens through the layer: the two differ by the activations' rounding to 4 bits only, and
    the batch's products are what the oracle says of the codes that the quantizer wrote."""
    import torch
    T, topk, E, D, H = 24, 2, 4, 256, 128
    g = torch.Generator(device="cuda").manual_seed(3)
    w1 = torch.randn(E, 2 * H, D, generator=g, device="cuda") * D ** -0.5
    w2 = torch.randn(E, D, H, generator=g, device="cuda") * H ** -0.5
    x = torch.randn(T, D, generator=g, device="cuda").bfloat16()
    p, ids = torch.topk(torch.softmax(torch.randn(T, E, generator=g, device="cuda"), 1), topk, dim=1)
    ids = ids.to(torch.int32).contiguous()
    p = p.contiguous()
    for by16 in (False, True):
        def codes(m, factor=None, source=None, k=1):
            rows = m.shape[0] if source is None else source.numel()
            q = torch.empty(rows, m.shape[1] // 2, dtype=torch.uint8, device="cuda")
            s = torch.empty(f4.words_of(m.shape[1], by16), rows, dtype=torch.int32, device="cuda")
            q4.q4_f4_quantize(m, q, s, by16=by16, factor=factor, source=source, topk=k)
            return q, s

        def host(q, s, cols):
            return f4.values(q.cpu().numpy(), s.cpu().numpy().view(np.uint32), cols, by16)
        (q1, s1), (q2, s2) = codes(w1.view(-1, D)), codes(w2.view(-1, H))
        n = ids.numel()
        starts, source, slot = (torch.empty(k, dtype=torch.int32, device="cuda") for k in (E + 1, n, n))
        slot = slot.view(T, topk)
        q4.q4_expert_sort(ids, E, 1, starts, source, slot)
        a, sa = codes(x, source=source, k=topk)
        up = q4.q4_gemm_f4_experts(a, sa, q1, s1, starts, torch.zeros(n, 2 * H, device="cuda"), n, 2 * H, D, by16=by16)
        want, mag = f4.experts(host(a, sa, D), host(q1, s1, D), starts.cpu().numpy(), 2 * H)
        assert (np.abs(up.double().cpu().numpy() - want) <= mag * (D + 8) * 2.0 ** -23).all()
        h = torch.nn.functional.silu(up[:, :H]) * up[:, H:]
        b, sb = codes(h.bfloat16())
        y = q4.q4_gemm_f4_experts(b, sb, q2, s2, starts, torch.zeros(n, D, device="cuda"), n, D, H, by16=by16)
        batch = q4.q4_expert_combine(y, slot, p, torch.empty(T, D, device="cuda"))
        ws = torch.empty(q4.q4_expert_layer_f4_workspace_bytes(T, topk, D, H), dtype=torch.uint8, device="cuda")
        out = q4.q4_expert_layer_f4(x, ids, p, q1, s1, q2, s2, torch.empty_like(x), E, H, ws, gated=True, by16=by16)
        want, off = f4.layer(x.double().cpu().numpy(), ids.cpu().numpy(), p.cpu().numpy(), host(q1, s1, D).reshape(E, 2 * H, D),
                             host(q2, s2, H).reshape(E, D, H), True)
        got = out.double().cpu().numpy()
        assert (np.abs(got - want) <= off + (np.abs(want) + off) * 2.0 ** -8).all()
        # an e2m1 rounding is off by a quarter of the value at most, a third of that typically: two layers of them
        assert np.linalg.norm(batch.double().cpu().numpy() - want) < 0.5 * np.linalg.norm(want)


def test_scales_that_binary16_does_not_hold(q4):
    """Powers of two far below and above: some groups, some rows, and 2^-127 itself."""
    import torch
    T, topk, E, D, H = 3, 1, 2, 320, 64
    r = np.random.default_rng(5)
    for gated in (False, True):
        up = (2 if gated else 1) * H
        mats, dev = [], []
        for n, k, spread in ((E * up, D, 1), (E * D, H, 3)):
            byte = r.integers(120, 128, (n, -(-k // 32))).astype(np.uint8)
            byte[::3, 0] = 127 - 40 * spread
            byte[1::5, -1] = 0
            byte[2::7, 1] = 127 + 5 * spread
            q, s = f4.pack(r.integers(0, 16, (n, k)).astype(np.uint8)), f4.to_words(byte)
            mats.append(f4.values(q, s, k))
            dev += [placed(q, up16(q.shape[1])), word_tensor(s)]
        # the second matrix gets rows of tiny values only: nothing else of these rows is in the result
        x = torch.from_numpy(r.standard_normal((T, D)).astype(np.float32) * 0.01).cuda().half()
        ids = np.array([[0], [1], [0]], dtype=np.int32)
        out = torch.empty_like(x)
        ws = torch.empty(q4.q4_expert_layer_f4_workspace_bytes(T, topk, D, H), dtype=torch.uint8, device="cuda")
        q4.q4_expert_layer_f4(x, torch.from_numpy(ids).cuda(), None, *dev, out, E, H, ws, gated=gated)
        want, off = f4.layer(x.double().cpu().numpy(), ids, None, mats[0].reshape(E, up, D), mats[1].reshape(E, D, H), gated)
        got = out.double().cpu().numpy()
        fine = np.abs(want) < 60000
        assert fine.any() and (np.abs(got - want) <= off + (np.abs(want) + off) * HALF_ULP["f16"] + HALF_SMALLEST["f16"])[fine].all()
