"""Measured cases of the 8-bit float product with block scales and of the expert layer around it.

Five operators: the quantizer to e4m3 codes with a scale per 128 values (`quantize`), the product of such
operands (`product`), the product of each expert's rows or depth segment (`experts`, `experts_wgrad`), the sort of
tokens by expert (`sort`), and the weighted sum back to token order with its gradient (`combine`, `combine_grad`).
`run` computes them in plain torch operations in 32 bits, or, with `own` set, through the framework's calls.
"""
import torch

own = False

BLOCK = 128
FLOOR = 2.0 ** -60          # smallest block maximum the scale is taken from
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}


def _blocks(n):
    return (n + BLOCK - 1) // BLOCK


# ------------------------------------------------------------------------------------------------- cases
def listed():
    return [
        # one token's activations in front of a serving product: latency
        dict(name="quantize_one_token", op="quantize", rows=1, cols=4096, type="bf16", blocks=False, pow2=False,
             both=False, topk=0),
        # a training batch, straight for the forward product and transposed for the weight gradient
        dict(name="quantize_training_batch", op="quantize", rows=8192, cols=4096, type="bf16", blocks=False,
             pow2=True, both=True, topk=0),
        # one token through a square layer: the weights are read once
        dict(name="product_one_token", op="product", M=1, N=4096, K=4096, out="bf16", b_rows=False),
        # weight gradient of a 2304 -> 256 layer over a ragged batch of 4097 rows: both operands scaled by row
        dict(name="product_weight_gradient", op="product", M=2304, N=256, K=4097, out="f32", b_rows=True),
        # a prompt batch through a wide layer
        dict(name="product_prompt", op="product", M=8192, N=8192, K=8192, out="bf16", b_rows=False),
        # a few tokens being decoded: two rows per expert, the experts' weights are read once
        dict(name="experts_few_tokens", op="experts", tokens=16, topk=8, E=64, N=2048, K=1024, align=1, out="bf16"),
        # a prompt through the experts
        dict(name="experts_prompt", op="experts", tokens=4096, topk=8, E=64, N=2048, K=2048, align=1, out="bf16"),
        # the experts' weight gradients over a training batch
        dict(name="experts_weight_gradient", op="experts_wgrad", tokens=4096, topk=4, E=32, M=1024, N=1024, out="f32"),
        # routing of a decoding batch: latency
        dict(name="sort_few_tokens", op="sort", tokens=64, topk=8, E=64, align=1),
        # routing of a training batch, segments on multiples of 128 rows
        dict(name="sort_training_batch", op="sort", tokens=65536, topk=8, E=128, align=128),
        # experts' outputs back to token order, a prompt
        dict(name="combine_prompt", op="combine", tokens=4096, topk=8, D=2048, E=64, type="bf16"),
        # its gradient: rows for the experts and the routing weights' gradient
        dict(name="combine_gradient", op="combine_grad", tokens=4096, topk=8, D=2048, E=64, type="bf16"),
    ]


def _log(rng, lo, hi):
    """A whole number, uniform in the logarithm."""
    return int(min(hi, max(lo, round(lo * (hi / lo) ** rng.random()))))


def draw(rng):
    op = rng.choice(["quantize", "product", "experts", "experts_wgrad", "sort", "combine", "combine_grad"])
    if op == "quantize":
        blocks = rng.random() < 0.3
        return dict(op=op, rows=_log(rng, 1, 8192), cols=_log(rng, 64, 8192), type=rng.choice(["f32", "bf16", "f16"]),
                    blocks=blocks, pow2=rng.random() < 0.5, both=rng.random() < 0.5,
                    topk=0 if blocks else rng.choice([0, 0, 1, 2, 4]))
    if op == "product":
        return dict(op=op, M=_log(rng, 1, 8192), N=_log(rng, 64, 8192), K=_log(rng, 64, 8192),
                    out=rng.choice(["bf16", "f32", "f16"]), b_rows=rng.random() < 0.3)
    E, topk = rng.choice([8, 16, 32, 64]), rng.choice([1, 2, 4, 8])
    if op == "experts":
        return dict(op=op, tokens=_log(rng, 1, 4096), topk=topk, E=E, N=_log(rng, 64, 2048), K=_log(rng, 64, 2048),
                    align=rng.choice([1, 1, 128]), out=rng.choice(["bf16", "f32", "f16"]))
    if op == "experts_wgrad":
        return dict(op=op, tokens=_log(rng, 16, 4096), topk=min(topk, 4), E=min(E, 32), M=_log(rng, 64, 1024),
                    N=_log(rng, 64, 1024), out=rng.choice(["bf16", "f32"]))
    if op == "sort":
        return dict(op=op, tokens=_log(rng, 1, 65536), topk=topk, E=rng.choice([8, 61, 128, 256]),
                    align=rng.choice([1, 16, 128]))
    return dict(op=op, tokens=_log(rng, 1, 4096), topk=topk, D=_log(rng, 64, 4096), E=E,
                type=rng.choice(["bf16", "f32", "f16"]))


# ------------------------------------------------------------------------------------------------ inputs
def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _activations(g, rows, cols):
    """Bell-shaped values whose columns differ in size and of which one in a few hundred is an outlier."""
    x = torch.randn(rows, cols, generator=g, device="cuda")
    x *= torch.exp(0.5 * torch.randn(cols, generator=g, device="cuda"))
    return torch.where(torch.rand(rows, cols, generator=g, device="cuda") < 0.003, 12 * x, x)


def _rows16(codes):
    """The codes with rows that begin on multiples of 16 bytes, as the product wants them."""
    rows, cols = codes.shape
    held = torch.zeros(rows, (cols + 15) // 16 * 16, dtype=torch.uint8, device="cuda")
    held[:, :cols] = codes.view(torch.uint8)
    return held.view(torch.float8_e4m3fn)[:, :cols]


def _empty16(rows, cols):
    return torch.empty(rows, (cols + 15) // 16 * 16, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)[:, :cols]


def _route(g, tokens, topk, E):
    """[tokens, topk] different expert numbers of each token, the experts of uneven popularity; a few are dropped (-1)."""
    pull = 0.7 * torch.randn(E, generator=g, device="cuda")
    noise = -torch.log(-torch.log(torch.rand(tokens, E, generator=g, device="cuda").clamp(1e-7, 1 - 1e-6)))
    ids = torch.topk(pull + noise, topk, dim=1).indices.to(torch.int32)
    return torch.where(torch.rand(tokens, topk, generator=g, device="cuda") < 0.01, torch.full_like(ids, -1), ids)


def _sorted_rows(n, E, align):
    """Rows that the sorted order of n pairs may take."""
    return n if align == 1 else (n + min(n, E) * (align - 1)) // align * align


def prepare(case, seed):
    g, op = _gen(seed), case["op"]
    st = dict(case)
    if op == "quantize":
        rows, cols = case["rows"], case["cols"]
        st["X"] = _activations(g, rows, cols).to(TYPES[case["type"]])
        n = rows
        st["source"] = None
        if case["topk"]:
            # rows as a sort by expert leaves them: each pair once, some rows with no pair
            n = min(4 * 8192, rows * case["topk"])
            at = torch.randperm(rows * case["topk"], generator=g, device="cuda")[:n].to(torch.int32)
            st["source"] = torch.where(torch.rand(n, generator=g, device="cuda") < 0.05, torch.full_like(at, -1), at)
        st["Q"] = _empty16(n, cols)
        rb, cb = _blocks(n), _blocks(cols)
        st["S"] = torch.empty((rb, cb) if case["blocks"] else (cb, n), device="cuda")
        st["Qt"] = _empty16(cols, n) if case["both"] else None
        st["St"] = torch.empty((cb, rb) if case["blocks"] else (rb, cols), device="cuda") if case["both"] else None
        return st
    if op == "product":
        M, N, K = case["M"], case["N"], case["K"]
        q, st["SA"] = _codes(_activations(g, M, K), False, False)
        st["A"] = _rows16(q)
        q, st["SB"] = _codes(0.02 * torch.randn(N, K, generator=g, device="cuda"), not case["b_rows"], False)
        st["B"] = _rows16(q)
        st["C"] = torch.empty(M, N, dtype=TYPES[case["out"]], device="cuda")
        return st
    ids = _route(g, case["tokens"], case["topk"], case["E"])
    st["ids"] = ids
    align = case.get("align", 128 if op == "experts_wgrad" else 1)
    rows = _sorted_rows(ids.numel(), case["E"], align)
    st["starts"], st["source"], st["slot"] = _sort(ids, case["E"], align, rows)
    if op == "experts":
        E, N, K = case["E"], case["N"], case["K"]
        q, st["SA"] = _codes(_activations(g, rows, K), False, False)
        st["A"] = _rows16(q)
        w = 0.02 * torch.randn(E, _blocks(N) * BLOCK, K, generator=g, device="cuda")
        w[:, N:] = 0
        q, st["SB"] = _codes(w.view(-1, K), True, False)
        st["B"] = _rows16(q.view(E, -1, K)[:, :N].reshape(E * N, K))
        st["C"] = torch.zeros(rows, N, dtype=TYPES[case["out"]], device="cuda")
    elif op == "experts_wgrad":
        used = (st["source"] >= 0)[:, None]
        for side, width in (("A", case["M"]), ("B", case["N"])):
            x = _activations(g, rows, width) * used
            q, st["S" + side] = _codes(x.t(), False, False)
            st[side] = _rows16(q)
        st["C"] = torch.empty(case["E"] * case["M"], case["N"], dtype=TYPES[case["out"]], device="cuda")
    elif op == "sort":
        st["starts"], st["source"], st["slot"] = (torch.empty_like(st[k]) for k in ("starts", "source", "slot"))
        st["ws"] = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
    else:
        D, t = case["D"], TYPES[case["type"]]
        st["w"] = torch.softmax(torch.randn(case["tokens"], case["topk"], generator=g, device="cuda"), 1)
        st["Y"] = _activations(g, rows, D).to(t)
        if op == "combine":
            st["out"] = torch.empty(case["tokens"], D, dtype=t, device="cuda")
        else:
            st["dout"] = torch.randn(case["tokens"], D, generator=g, device="cuda").to(t)
            st["dY"], st["dw"] = torch.empty_like(st["Y"]), torch.empty_like(st["w"])
    return st


def work(case):
    op = case["op"]
    if op == "quantize":
        rows, cols = case["rows"], case["cols"]
        n = min(4 * 8192, rows * case["topk"]) if case["topk"] else rows
        ways = 2 if case["both"] else 1
        scales = _blocks(n) * _blocks(cols) if case["blocks"] else n * _blocks(cols) + (ways - 1) * cols * _blocks(n)
        return dict(bytes=rows * cols * SIZE[case["type"]] + ways * n * cols + 4 * scales + (4 * n if case["topk"] else 0),
                    flops=2 * n * cols)
    if op == "product":
        M, N, K = case["M"], case["N"], case["K"]
        return dict(bytes=M * K + N * K + 4 * _blocks(K) * (M + (N if case["b_rows"] else _blocks(N))) + M * N * SIZE[case["out"]],
                    flops=2 * M * N * K)
    n, E = case["tokens"] * case["topk"], case["E"]
    if op == "experts":
        N, K = case["N"], case["K"]
        used = E * (1 - (1 - case["topk"] / E) ** case["tokens"])       # experts that a token reaches, on average
        return dict(bytes=n * K + 4 * n * _blocks(K) + used * (N * K + 4 * _blocks(N) * _blocks(K)) + n * N * SIZE[case["out"]],
                    flops=2 * n * N * K)
    if op == "experts_wgrad":
        M, N = case["M"], case["N"]
        return dict(bytes=n * (M + N) + 4 * _blocks(n) * (M + N) + E * M * N * SIZE[case["out"]], flops=2 * n * M * N)
    if op == "sort":
        return dict(bytes=4 * (2 * n + _sorted_rows(n, E, case["align"]) + E), flops=4 * n)
    each = case["D"] * SIZE[case["type"]]
    if op == "combine":
        return dict(bytes=(n + case["tokens"]) * each + 8 * n, flops=2 * n * case["D"])
    return dict(bytes=(2 * n + case["tokens"]) * each + 16 * n, flops=3 * n * case["D"])


# ------------------------------------------------------------------------------------------- plain forms
def _scale_of(a, pow2):
    """(scale, its inverse) of block maxima a."""
    a = torch.maximum(a, torch.full_like(a, FLOOR))
    top = torch.full_like(a, 448.0)
    s = a / top
    if not pow2:
        return s, top / a
    s = ((s.view(torch.int32) + 0x7FFFFF) & ~0x7FFFFF).view(torch.float32)
    return s, torch.ones_like(s) / s


def _codes(x, blocks, pow2):
    """e4m3 codes of a matrix and its scales: [block of columns][row], or [block of rows][block of columns]."""
    rows, cols = x.shape
    rb, cb = _blocks(rows), _blocks(cols)
    x = torch.nn.functional.pad(x.float(), (0, cb * BLOCK - cols, 0, rb * BLOCK - rows if blocks else 0))
    v = x.view(rb, BLOCK, cb, BLOCK) if blocks else x.view(rows, 1, cb, BLOCK)
    s, inv = _scale_of(v.abs().amax((1, 3), keepdim=True), pow2)
    q = (v * inv).to(torch.float8_e4m3fn).view(-1, cb * BLOCK)[:rows, :cols]
    s = s.view(-1, cb)
    return q, s if blocks else s.t().contiguous()


def _values(codes, scales):
    """Values of codes whose scales are [block of columns][row]."""
    return codes.float() * scales.t().repeat_interleave(BLOCK, 1)[:, :codes.shape[1]]


def _weights(codes, scales, rows):
    """Values of matrices of `rows` rows each, a scale per 128 x 128 block."""
    cols = codes.shape[1]
    s = scales.view(-1, _blocks(rows), _blocks(cols)).repeat_interleave(BLOCK, 1)[:, :rows].repeat_interleave(BLOCK, 2)
    return codes.view(-1, rows, cols).float() * s[:, :, :cols]


def _sort(ids, E, align, rows):
    n = ids.numel()
    key = ids.reshape(-1).long()
    key = torch.where((key < 0) | (key >= E), E, key)
    sorted_key, order = torch.sort(key, stable=True)
    counts = torch.zeros(E + 1, dtype=torch.int64, device=ids.device).index_add_(0, key, torch.ones_like(key))
    first = torch.cumsum(counts, 0) - counts
    taken = (counts[:E] + align - 1) // align * align
    starts = torch.cat([torch.zeros_like(taken[:1]), torch.cumsum(taken, 0)])
    at = torch.arange(n, device=ids.device) - first[sorted_key] + starts[sorted_key]
    at = torch.where(sorted_key == E, rows, at)
    source = torch.full((rows + 1,), -1, dtype=torch.int32, device=ids.device)
    source[at] = order.to(torch.int32)
    slot = torch.empty(n, dtype=torch.int32, device=ids.device)
    slot[order] = torch.where(sorted_key == E, -1, at).to(torch.int32)
    return starts.to(torch.int32), source[:rows].contiguous(), slot.view(ids.shape)


def _segments(starts, rows):
    """Blocks of 128 rows that no expert shares with another: each row's place in them, and each block's expert."""
    E = starts.numel() - 1
    starts = starts.long()
    count = starts[1:] - starts[:-1]
    ends = torch.cumsum((count + BLOCK - 1) // BLOCK, 0)
    blocks = _blocks(rows) + E
    row = torch.arange(rows, device=starts.device)
    expert = torch.searchsorted(starts[1:].contiguous(), row, right=True).clamp(max=E - 1)
    place = (ends - (count + BLOCK - 1) // BLOCK)[expert] * BLOCK + row - starts[expert]
    place = torch.where(row < starts[-1], place, blocks * BLOCK)
    of = torch.searchsorted(ends, torch.arange(blocks, device=starts.device), right=True).clamp(max=E - 1)
    return place, of, blocks


def _plain(st):
    op = st["op"]
    if op == "quantize":
        x = st["X"].float()
        if st["source"] is not None:
            src = st["source"].long()
            x = torch.where((src >= 0)[:, None], x[src.clamp(min=0) // st["topk"]], torch.zeros_like(x[:1]))
        q, s = _codes(x, st["blocks"], st["pow2"])
        if not st["both"]:
            return q, s
        return (q, s) + _codes(x.t(), st["blocks"], st["pow2"])
    if op == "product":
        b = _values(st["B"], st["SB"]) if st["b_rows"] else _weights(st["B"], st["SB"], st["N"])[0]
        return (_values(st["A"], st["SA"]) @ b.t()).to(st["C"].dtype)
    if op == "experts":
        rows = st["A"].shape[0]
        place, of, blocks = _segments(st["starts"], rows)
        a = torch.zeros(blocks * BLOCK + 1, st["K"], device="cuda")
        a[place] = _values(st["A"], st["SA"])
        w = _weights(st["B"], st["SB"], st["N"])
        c = torch.bmm(a[:-1].view(blocks, BLOCK, -1), w[of].transpose(1, 2)).view(-1, st["N"])
        c = torch.cat([c, torch.zeros_like(c[:1])])
        return c[place].to(st["C"].dtype)
    if op == "experts_wgrad":
        a, b = _values(st["A"], st["SA"]), _values(st["B"], st["SB"])
        row = torch.arange(0, a.shape[1], BLOCK, device="cuda")
        of = torch.searchsorted(st["starts"][1:].long().contiguous(), row, right=True)
        p = torch.bmm(a.view(st["M"], -1, BLOCK).transpose(0, 1), b.view(st["N"], -1, BLOCK).permute(1, 2, 0))
        c = torch.zeros(st["E"] + 1, st["M"], st["N"], device="cuda").index_add_(0, of.clamp(max=st["E"]), p)
        return c[:-1].view(-1, st["N"]).to(st["C"].dtype)
    if op == "sort":
        return _sort(st["ids"], st["E"], st["align"], st["source"].numel())
    slot = st["slot"].long()
    has = (slot >= 0)[:, :, None]
    if op == "combine":
        y = st["Y"].float()[slot.clamp(min=0)]
        return torch.where(has, y * st["w"][:, :, None], torch.zeros_like(y[:1])).sum(1).to(st["out"].dtype)
    dout, src = st["dout"].float(), st["source"].long()
    pair = src.clamp(min=0)
    d = dout[pair // st["topk"]] * st["w"].reshape(-1)[pair][:, None]
    d = torch.where((src >= 0)[:, None], d, torch.zeros_like(d[:1])).to(st["Y"].dtype)
    y = st["Y"].float()[slot.clamp(min=0)]
    return d, torch.where(has[:, :, 0], (y * dout[:, None, :]).sum(2), torch.zeros_like(st["w"]))


def run(st):
    if not own:
        return _plain(st)
    from paper_2009_06488_b200 import binding as q4
    op = st["op"]
    if op == "quantize":
        q4.q4_f8_quantize(st["X"], st["Q"], st["S"], st["Qt"], st["St"], blocks=st["blocks"], pow2=st["pow2"],
                          source=st["source"], topk=max(1, st["topk"]))
        return (st["Q"], st["S"]) if not st["both"] else (st["Q"], st["S"], st["Qt"], st["St"])
    if op == "product":
        return q4.q4_gemm_f8(st["A"], st["SA"], st["B"], st["SB"], st["C"], st["M"], st["N"], st["K"], b_rows=st["b_rows"])
    if op == "experts":
        return q4.q4_gemm_f8_experts(st["A"], st["SA"], st["B"], st["SB"], st["starts"], st["C"], st["A"].shape[0],
                                     st["N"], st["K"])
    if op == "experts_wgrad":
        return q4.q4_gemm_f8_experts_wgrad(st["A"], st["SA"], st["B"], st["SB"], st["starts"], st["C"], st["M"],
                                           st["N"], st["A"].shape[1])
    if op == "sort":
        q4.q4_expert_sort(st["ids"], st["E"], st["align"], st["starts"], st["source"], st["slot"], st["ws"])
        return st["starts"], st["source"], st["slot"]
    if op == "combine":
        return q4.q4_expert_combine(st["Y"], st["slot"], st["w"], st["out"])
    q4.q4_expert_combine_grad(st["dout"], st["Y"], st["slot"], st["w"], st["source"], st["dY"], st["dw"])
    return st["dY"], st["dw"]


# ---------------------------------------------------------------------------------------- in 64 bits
def _e4m3_64(y):
    """Nearest e4m3 value (ties to even) of 64-bit values within +-448."""
    _, e = torch.frexp(y)
    step = torch.ldexp(torch.ones_like(y), (e - 4).clamp(min=-9))
    return torch.round(y / step) * step


def _quantized_64(x, blocks, pow2):
    rows, cols = x.shape
    q, high = torch.empty_like(x), BLOCK if blocks else rows
    s = torch.empty(_blocks(cols), _blocks(rows) if blocks else rows, dtype=torch.float64, device="cuda")
    for c in range(0, cols, BLOCK):
        for r in range(0, rows, high):
            part = x[r:r + high, c:c + BLOCK]
            a = part.abs().max() if blocks else part.abs().max(1).values
            scale = a.clamp(min=FLOOR) / 448
            if pow2:
                m, e = torch.frexp(scale)
                scale = torch.ldexp(torch.ones_like(scale), torch.where(m == 0.5, e - 1, e))
            if blocks:
                s[c // BLOCK, r // BLOCK] = scale
            else:
                s[c // BLOCK, r:r + high] = scale
            q[r:r + high, c:c + BLOCK] = _e4m3_64(part / (scale if blocks else scale[:, None]))
    return q, s.t().contiguous() if blocks else s


def _stretch(s, cols):
    return s[torch.arange(cols, device="cuda") // BLOCK]


def exact(case, seed):
    op = case["op"]
    if op == "sort":
        return None             # whole numbers
    st = prepare(case, seed)
    if op == "quantize":
        x = st["X"].double()
        if st["source"] is not None:
            x = x[(st["source"] // case["topk"]).clamp(min=0).long()]
            x[st["source"] < 0] = 0
        out = _quantized_64(x, case["blocks"], case["pow2"])
        return out + _quantized_64(x.t().contiguous(), case["blocks"], case["pow2"]) if case["both"] else out
    if op == "product":
        a = st["A"].double() * _stretch(st["SA"].double(), case["K"]).t()
        if case["b_rows"]:
            return a @ (st["B"].double().t() * _stretch(st["SB"].double(), case["K"]))
        return a @ (st["B"].double() * _stretch(_stretch(st["SB"].double(), case["N"]).t(), case["K"]).t()).t()
    at = st["starts"].tolist()
    if op == "experts":
        N, K = case["N"], case["K"]
        a = st["A"].double() * _stretch(st["SA"].double(), K).t()
        c = torch.zeros(a.shape[0], N, dtype=torch.float64, device="cuda")
        for e in range(case["E"]):
            s = st["SB"][e * _blocks(N):(e + 1) * _blocks(N)].double()
            w = st["B"][e * N:(e + 1) * N].double() * _stretch(_stretch(s, N).t(), K).t()
            c[at[e]:at[e + 1]] = a[at[e]:at[e + 1]] @ w.t()
        return c
    if op == "experts_wgrad":
        rows = st["A"].shape[1]
        a = st["A"].double().t() * _stretch(st["SA"].double(), rows)
        b = st["B"].double().t() * _stretch(st["SB"].double(), rows)
        return torch.cat([a[at[e]:at[e + 1]].t() @ b[at[e]:at[e + 1]] for e in range(case["E"])])
    w, slot = st["w"].double(), st["slot"].long()
    tokens = torch.arange(case["tokens"], device="cuda")
    if op == "combine":
        out = torch.zeros(case["tokens"], case["D"], dtype=torch.float64, device="cuda")
        for j in range(case["topk"]):
            got = slot[:, j] >= 0
            out[got] += w[got, j, None] * st["Y"][slot[got, j]].double()
        return out
    dY, dw = torch.zeros_like(st["Y"], dtype=torch.float64), torch.zeros_like(w)
    for j in range(case["topk"]):
        got = slot[:, j] >= 0
        d = st["dout"][tokens[got]].double()
        dY[slot[got, j]] = w[got, j, None] * d
        dw[got, j] = (d * st["Y"][slot[got, j]].double()).sum(1)
    return dY, dw
