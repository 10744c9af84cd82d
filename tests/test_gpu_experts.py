"""Sort by expert, gather, combine and its gradient on the GPU against the 64-bit oracle.

Whole numbers have to be equal.  Sums of topk (or D) products in binary32 are off by at most (terms + 1) *
2^-24 times the sum of the terms' magnitudes; the output's type adds half of its last place.
"""
import numpy as np
import pytest

from oracle import f8

pytestmark = pytest.mark.gpu

HALF_ULP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}      # significands of 24, 8 and 11 bits
HALF_SMALLEST = {"f32": 2.0 ** -150, "bf16": 2.0 ** -134, "f16": 2.0 ** -25}     # the last place of subnormal values


@pytest.fixture(scope="module")
def q4():
    from paper_2009_06488_b200 import binding
    return binding


def types():
    import torch
    return {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def dev(a):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def route(seed, tokens, topk, E):
    r = np.random.default_rng(seed)
    p = r.dirichlet(np.full(E, 0.3))
    ids = r.choice(E, size=(tokens, topk), p=p).astype(np.int32)
    ids[r.random((tokens, topk)) < 0.05] = r.choice([-1, E, 2 ** 31 - 1, -2 ** 31])
    return ids


def run_sort(q4, ids, E, align, extra=0):
    import torch
    rows = q4.q4_expert_sort_rows(ids.size, E, align) + extra
    starts, source = (torch.full((k,), 77, dtype=torch.int32, device="cuda") for k in (E + 1, rows))
    slot = torch.full(ids.shape, 77, dtype=torch.int32, device="cuda")
    ws = torch.empty(max(1, q4.q4_expert_sort_workspace_bytes(ids.size, E)), dtype=torch.uint8, device="cuda")
    q4.q4_expert_sort(dev(ids), E, align, starts, source, slot, ws)
    return starts, source, slot


@pytest.mark.parametrize("tokens,topk,E", [(0, 1, 4), (1, 1, 1), (1, 8, 64), (5, 3, 7), (64, 8, 64), (333, 2, 1024), (500, 8, 61),
                                           (513, 8, 5), (5000, 4, 128), (70001, 8, 256), (200000, 3, 1000)])
@pytest.mark.parametrize("align", [1, 16, 128])
def test_sort_matches_the_oracle(q4, tokens, topk, E, align):
    ids = route(tokens + E, tokens, topk, E)
    for extra in (0, 5):
        got = run_sort(q4, ids, E, align, extra)
        want = f8.sort(ids, E, align, f8.sort_rows(ids.size, E, align) + extra)
        for g, w in zip(got, want):
            assert (g.cpu().numpy() == w).all()


def test_sort_of_one_expert_and_of_dropped_pairs_only(q4):
    for fill in (3, -1):
        ids = np.full((3000, 4), fill, dtype=np.int32)
        for g, w in zip(run_sort(q4, ids, 9, 128), f8.sort(ids, 9, 128, f8.sort_rows(12000, 9, 128))):
            assert (g.cpu().numpy() == w).all()


def layer(seed, tokens, topk, E, D, t, align):
    """Random rows on both sides of a routing, rounded to the type, on the host and the GPU."""
    import torch
    r = np.random.default_rng(seed)
    ids = route(seed, tokens, topk, E)
    rows = f8.sort_rows(ids.size, E, align)
    starts, source, slot = f8.sort(ids, E, align, rows)
    pair = lambda *s: (lambda g: (g.float().cpu().numpy(), g))(dev(r.standard_normal(s).astype(np.float32)).to(types()[t]))
    w = r.standard_normal((tokens, topk)).astype(np.float32)
    return source, slot, rows, w, pair(tokens, D), pair(rows, D)


def check(got, want, mag, terms, t):
    got = got.float().cpu().numpy().astype(np.float64)
    bound = (terms + 1) * 2.0 ** -24 * mag
    bound = bound + (np.abs(want) + bound) * HALF_ULP[t] + HALF_SMALLEST[t] + 1e-30
    if got.size:
        assert (np.abs(got - want) / bound).max() <= 1


CASES = [(1, 1, 1, 8, 1), (1, 8, 16, 64, 1), (3, 2, 5, 7, 16), (40, 8, 8, 100, 1), (65, 3, 17, 256, 128), (70, 9, 40, 264, 16),
         (129, 4, 8, 1000, 1), (33, 8, 64, 2048, 128), (20, 17, 32, 4100, 1)]


@pytest.mark.parametrize("tokens,topk,E,D,align", CASES)
@pytest.mark.parametrize("t", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("weighted", [False, True])
def test_rows_there_and_back(q4, tokens, topk, E, D, align, t, weighted):
    import torch
    source, slot, rows, w, (x, X), (y, Y) = layer(tokens + D, tokens, topk, E, D, t, align)
    w = w if weighted else None
    W, src, sl = dev(w) if weighted else None, dev(source), dev(slot)

    def strided(n, pad):
        return torch.full((n + 1, D + pad), 7.0, dtype=types()[t], device="cuda")
    for pad in (0, 8, 3):
        Xs, Out, dY = strided(rows, pad), strided(tokens, pad), strided(rows, pad)
        dw = torch.full((tokens, topk), 7.0, device="cuda")
        q4.q4_expert_gather(X, src, topk, Xs[:, :D], W)
        want = f8.gather(x, source, topk, w)
        check(Xs[:rows, :D], want, np.abs(want), 0, t)
        q4.q4_expert_combine(Y, sl, W, Out[:, :D])
        check(Out[:tokens, :D], f8.combine(y, slot, w), f8.combine(np.abs(y), slot, None if w is None else np.abs(w)), topk, t)
        q4.q4_expert_combine_grad(X, Y, sl, W, src, dY[:, :D], dw)
        wy, ww = f8.combine_grad(x, y, slot, w)
        check(dY[:rows, :D], wy, np.abs(wy), 0, t)
        check(dw, ww, f8.combine_grad(np.abs(x), np.abs(y), slot, w)[1], D, "f32")
        for buf, n in ((Xs, rows), (Out, tokens), (dY, rows)):
            assert (buf[n:] == 7).all() and (buf[:, D:] == 7).all()


def test_gradient_against_differences(q4):
    """The loss <G, combine(Y, w)> is linear in Y and in w: central differences in 64 bits are exact."""
    import torch
    source, slot, rows, w, (x, X), (y, Y) = layer(11, 30, 4, 9, 136, "f32", 16)
    dY, dw = torch.empty(rows, 136, device="cuda"), torch.empty(30, 4, device="cuda")
    q4.q4_expert_combine_grad(X, Y, dev(slot), dev(w), dev(source), dY, dw)
    loss = lambda y, w: (f8.combine(y, slot, w) * x.astype(np.float64)).sum()
    y, w, h = y.astype(np.float64), w.astype(np.float64), 1e-2
    for at in [(0, 0), (7, 3), (29, 2)]:
        d = np.zeros_like(w); d[at] = h
        assert dw[at].item() == pytest.approx((loss(y, w + d) - loss(y, w - d)) / (2 * h), rel=1e-5, abs=1e-4)
    for at in [(0, 0), (5, 77), (rows - 1, 135)]:
        d = np.zeros_like(y); d[at] = h
        assert dY[at].item() == pytest.approx((loss(y + d, w) - loss(y - d, w)) / (2 * h), rel=1e-5, abs=1e-6)


def test_entries_out_of_range_are_absent(q4):
    """Rows and pairs outside their ranges count as dropped; NaN and infinity in rows nobody asked for stay out."""
    import torch
    D, rows, tokens, topk = 40, 12, 4, 3
    r = np.random.default_rng(2)
    y = r.standard_normal((rows, D)).astype(np.float32)
    y[5], y[6] = np.nan, np.inf
    slot = np.array([[0, 12, -1], [2 ** 31 - 1, 1, -2 ** 31], [-1, -1, -1], [3, 4, 7]], dtype=np.int32)
    cut = np.where((slot < 0) | (slot >= rows), -1, slot)
    w = r.standard_normal((tokens, topk)).astype(np.float32)
    w[0, 1] = np.nan
    Out = torch.empty(tokens, D, device="cuda")
    q4.q4_expert_combine(dev(y), dev(slot), dev(w), Out)
    w0 = np.where(cut < 0, 0, w)
    check(Out, f8.combine(y, cut, w0), f8.combine(np.abs(y), cut, np.abs(w0)), topk, "f32")
    source = np.array([0, tokens * topk, -1, 2 ** 31 - 1, 11], dtype=np.int32)
    x = r.standard_normal((tokens, D)).astype(np.float32)
    Xs = torch.full((5, D), 7.0, device="cuda")
    q4.q4_expert_gather(dev(x), dev(source), topk, Xs)
    want = np.zeros((5, D), dtype=np.float32)
    want[0], want[4] = x[0], x[3]
    assert (Xs.cpu().numpy() == want).all()
