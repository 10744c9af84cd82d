"""A mixture-of-experts feed-forward layer in e4m3, forward and backward, through the library's public calls.

    python examples/expert_layer.py [--tokens 4096 --topk 4 --experts 16 --width 1024 --hidden 1024]

Routing weights and the activation are plain torch; everything between is the library's:

    sort        q4_expert_sort          tokens by expert, segments on multiples of 128 rows
    dispatch    q4_f8_quantize          picked rows to codes, straight (forward) and transposed (gradient) from one read
    experts     q4_gemm_f8_experts      up and down products; with the transposed weights, the gradients of their inputs
                q4_gemm_f8_experts_wgrad  gradients of the weights
    combine     q4_expert_combine       weighted sum back to token order; without weights, the dispatch's gradient
                q4_expert_combine_grad  gradients of the experts' rows and of the routing weights

The program compares outputs and gradients with float32 torch on the same weights and prints the distance (the
rounding to e4m3) and the time of a step; a layer of one token runs with segments on single rows and keeps nothing
for a gradient.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2009_06488_b200 import binding as q4  # noqa: E402

F8, BF16 = torch.float8_e4m3fn, torch.bfloat16


def blocks(n):
    return (n + 127) // 128


class Weights:
    """Experts' matrices [E, N, K] held as codes by 128 x 128 block, straight and (for gradients) transposed."""

    def __init__(self, w):
        self.E, self.N, self.K = w.shape
        new = lambda n, k: torch.empty(self.E, n, k, dtype=F8, device=w.device)
        sc = lambda n, k: torch.empty(self.E, blocks(n), blocks(k), device=w.device)
        self.q, self.s = new(self.N, self.K), sc(self.N, self.K)
        self.qt, self.st = new(self.K, self.N), sc(self.K, self.N)
        for e in range(self.E):
            q4.q4_f8_quantize(w[e], self.q[e], self.s[e], self.qt[e], self.st[e], blocks=True)

    def rows(self, x, sx, starts, rows):
        """x W^T by expert."""
        out = torch.zeros(rows, self.N, dtype=BF16, device=x.device)
        return q4.q4_gemm_f8_experts(x, sx, self.q.view(-1, self.K), self.s.view(-1, blocks(self.K)), starts, out,
                                     rows, self.N, self.K)

    def rows_back(self, g, sg, starts, rows):
        """g W by expert: the gradient of `rows`' input."""
        out = torch.zeros(rows, self.K, dtype=BF16, device=g.device)
        return q4.q4_gemm_f8_experts(g, sg, self.qt.view(-1, self.N), self.st.view(-1, blocks(self.N)), starts, out,
                                     rows, self.K, self.N)


def codes(x, across=False, source=None, topk=1):
    """Codes of x's rows by group and, with across, of its columns; rows picked by source."""
    rows, cols = (x.shape[0] if source is None else source.numel()), x.shape[1]
    q, s = torch.empty(rows, cols, dtype=F8, device=x.device), torch.empty(blocks(cols), rows, device=x.device)
    qt = torch.empty(cols, rows, dtype=F8, device=x.device) if across else None
    st = torch.empty(blocks(rows), cols, device=x.device) if across else None
    q4.q4_f8_quantize(x, q, s, qt, st, source=source, topk=topk)
    return q, s, qt, st


class ExpertLayer:
    """y = sum_j p_j W2_e(silu(W1_e x)) over a token's topk experts e with routing weights p."""

    def __init__(self, w1, w2):
        self.w1, self.w2 = Weights(w1), Weights(w2)

    def forward(self, x, ids, p, train):
        E, (tokens, topk) = self.w1.E, ids.shape
        align = 128 if train else 1
        rows = q4.q4_expert_sort_rows(ids.numel(), E, align)
        i32 = lambda n: torch.empty(n, dtype=torch.int32, device=x.device)
        starts, source, slot = i32(E + 1), i32(rows), i32(ids.numel()).view(ids.shape)
        ws = torch.empty(max(16, q4.q4_expert_sort_workspace_bytes(ids.numel(), E)), dtype=torch.uint8, device=x.device)
        q4.q4_expert_sort(ids, E, align, starts, source, slot, ws)
        xq, xs, xt, xts = codes(x, across=train, source=source, topk=topk)
        up = self.w1.rows(xq, xs, starts, rows)
        h = torch.nn.functional.silu(up)
        hq, hs, ht, hts = codes(h, across=train)
        y = self.w2.rows(hq, hs, starts, rows)
        out = q4.q4_expert_combine(y, slot, p, torch.empty(tokens, y.shape[1], dtype=BF16, device=x.device))
        if train:
            self.kept = (p, slot, source, starts, rows, y, up, xt, xts, ht, hts)
        return out

    def backward(self, dout):
        """(dx, dp, dW1, dW2) of the last forward pass."""
        p, slot, source, starts, rows, y, up, xt, xts, ht, hts = self.kept
        dy, dp = torch.empty_like(y), torch.empty_like(p)
        q4.q4_expert_combine_grad(dout, y, slot, p, source, dy, dp)
        gq, gs, gt, gts = codes(dy, across=True)
        f32 = lambda w: torch.empty(w.E * w.N, w.K, device=dout.device)
        dw2 = q4.q4_gemm_f8_experts_wgrad(gt, gts, ht, hts, starts, f32(self.w2), self.w2.N, self.w2.K, rows)
        dup = torch.ops.aten.silu_backward(self.w2.rows_back(gq, gs, starts, rows), up)
        uq, us, ut, uts = codes(dup, across=True)
        dw1 = q4.q4_gemm_f8_experts_wgrad(ut, uts, xt, xts, starts, f32(self.w1), self.w1.N, self.w1.K, rows)
        dxs = self.w1.rows_back(uq, us, starts, rows)
        dx = q4.q4_expert_combine(dxs, slot, None, torch.empty(slot.shape[0], dxs.shape[1], dtype=BF16, device=dout.device))
        return dx, dp, dw1.view(self.w1.E, self.w1.N, -1), dw2.view(self.w2.E, self.w2.N, -1)


def reference(x, ids, p, w1, w2, dout):
    """The same in float32 torch: (y, dx, dp, dW1, dW2)."""
    leaves = [t.float().detach().requires_grad_() for t in (x, p, w1, w2)]
    x, p, w1, w2 = leaves
    y = torch.zeros(x.shape[0], w2.shape[1], device=x.device)
    for e in range(w1.shape[0]):
        t, j = torch.nonzero(ids == e, as_tuple=True)
        y = y.index_add(0, t, p[t, j, None] * (torch.nn.functional.silu(x[t] @ w1[e].t()) @ w2[e].t()))
    y.backward(dout.float())
    return (y.detach(),) + tuple(t.grad for t in leaves)


def run(tokens=4096, topk=4, experts=16, width=1024, hidden=1024, seed=0):
    """A training step and a one-token step; the distance of every result from float32, by name."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    rand = lambda *s: torch.randn(*s, generator=g, device="cuda")
    w1, w2 = rand(experts, hidden, width) * width ** -0.5, rand(experts, width, hidden) * hidden ** -0.5
    x, dout = rand(tokens, width).to(BF16), rand(tokens, width).to(BF16)
    p, ids = torch.topk(torch.softmax(rand(tokens, experts), 1), topk, dim=1)
    ids = ids.to(torch.int32).contiguous()
    p = (p / p.sum(1, keepdim=True)).contiguous()
    layer = ExpertLayer(w1.to(BF16), w2.to(BF16))
    got = (layer.forward(x, ids, p, train=True),) + layer.backward(dout)
    want = reference(x, ids, p, w1.to(BF16), w2.to(BF16), dout)
    off = {n: float((a.float() - b).norm() / b.norm()) for n, a, b in zip(("y", "dx", "dp", "dW1", "dW2"), got, want)}
    one = layer.forward(x[:1], ids[:1], p[:1], train=False)
    off["y of one token"] = float((one.float() - want[0][:1]).norm() / want[0][:1].norm())
    return off, layer, (x, ids, p, dout)


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, value in (("tokens", 4096), ("topk", 4), ("experts", 16), ("width", 1024), ("hidden", 1024)):
        ap.add_argument("--" + name, type=int, default=value)
    a = ap.parse_args()
    off, layer, (x, ids, p, dout) = run(**vars(a))
    for name, v in off.items():
        print(f"{name:16s} distance from float32 {v:.4f}")

    def step():
        layer.forward(x, ids, p, train=True)
        layer.backward(dout)
    for what, call in (("training step", step), ("one token", lambda: layer.forward(x[:1], ids[:1], p[:1], train=False))):
        for _ in range(3):
            call()
        begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        begin.record()
        for _ in range(20):
            call()
        end.record()
        end.synchronize()
        print(f"{what:16s} {begin.elapsed_time(end) / 20 * 1e3:.0f} us")


if __name__ == "__main__":
    main()
