"""Measured cases of the 4-bit float (e2m1) operators with microscales and of the expert layer for a few tokens.

Four operators: the quantizer to e2m1 codes and its read-back (`quantize`), the product of such operands (`product`),
the product of each expert's rows (`experts`), and a whole expert layer on 4-bit weights for a few tokens (`layer`).
`run` computes them in plain torch operations in 32 bits, or, with `own` set, through the framework's calls.

Codes are e2m1, two per byte (low half: the even column).  A scale belongs to 32 columns and is a power of two (a byte,
exponent + 127), or to 16 columns and is an e4m3 number, times one float32 factor of the matrix.  The scales of four
neighbouring groups of a row make a 32-bit word; words are stored [word of columns][row].
"""
import torch

own = False

FLOOR = 2.0 ** -60          # smallest group maximum that a power-of-two scale is taken from
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}


def _up(n, to):
    return (n + to - 1) // to * to


def _group(by16):
    return 16 if by16 else 32


def _words(cols, by16):
    """Words of scales per row."""
    return _up(cols, 4 * _group(by16)) // (4 * _group(by16))


# ------------------------------------------------------------------------------------------------- cases
def listed():
    return [
        # one token's activations in front of a serving product, and read back: latency
        dict(name="quantize_one_token", op="quantize", rows=1, cols=4096, type="bf16", by16=True, both=False),
        # a training batch, straight for the forward product and transposed for the weight gradient, both read back
        dict(name="quantize_training_batch", op="quantize", rows=8192, cols=4096, type="bf16", by16=False, both=True),
        # a weight matrix out of an optimizer's master copy, odd sizes
        dict(name="quantize_weights_odd", op="quantize", rows=2047, cols=1363, type="f32", by16=True, both=False),
        # one token through a square layer: the weights are read once
        dict(name="product_one_token", op="product", M=1, N=4096, K=4096, out="bf16", by16=True),
        # weight gradient of a 2304 -> 256 layer over a ragged batch of 4097 rows
        dict(name="product_weight_gradient", op="product", M=2304, N=256, K=4097, out="f32", by16=False),
        # a prompt batch through a wide layer, both kinds of scales
        dict(name="product_prompt", op="product", M=8192, N=8192, K=8192, out="bf16", by16=True),
        dict(name="product_batch", op="product", M=1024, N=4096, K=4096, out="bf16", by16=False),
        # a few tokens being decoded: two rows per expert, the experts' weights are read once
        dict(name="experts_few_tokens", op="experts", tokens=16, topk=8, E=64, N=2048, K=1024, align=1, out="bf16", by16=True),
        # a prompt through the experts
        dict(name="experts_prompt", op="experts", tokens=4096, topk=8, E=64, N=2048, K=2048, align=1, out="bf16", by16=False),
        # a decoding step of an expert layer: one token, and sixteen
        dict(name="layer_one_token", op="layer", tokens=1, topk=8, E=64, D=2048, H=1024, gated=True, type="bf16", by16=True),
        dict(name="layer_few_tokens", op="layer", tokens=16, topk=8, E=64, D=2048, H=1024, gated=True, type="bf16", by16=False),
        # few experts of odd widths, each hit by several tokens
        dict(name="layer_odd_widths", op="layer", tokens=21, topk=2, E=8, D=1362, H=719, gated=False, type="f16", by16=True),
    ]


def _log(rng, lo, hi):
    """A whole number, uniform in the logarithm."""
    return int(min(hi, max(lo, round(lo * (hi / lo) ** rng.random()))))


def draw(rng):
    op, by16 = rng.choice(["quantize", "product", "experts", "layer"]), rng.random() < 0.5
    if op == "quantize":
        return dict(op=op, rows=_log(rng, 1, 8192), cols=_log(rng, 64, 4096), type=rng.choice(["f32", "bf16", "f16"]),
                    by16=by16, both=rng.random() < 0.5)
    if op == "product":
        return dict(op=op, M=_log(rng, 1, 8192), N=_log(rng, 64, 8192), K=_log(rng, 64, 8192),
                    out=rng.choice(["bf16", "f32", "f16"]), by16=by16)
    E, topk = rng.choice([8, 16, 32, 64]), rng.choice([1, 2, 4, 8])
    if op == "experts":
        return dict(op=op, tokens=_log(rng, 1, 4096), topk=topk, E=E, N=_log(rng, 64, 2048), K=_log(rng, 64, 2048),
                    align=rng.choice([1, 1, 128]), out=rng.choice(["bf16", "f32", "f16"]), by16=by16)
    return dict(op=op, tokens=_log(rng, 1, 32), topk=topk, E=E, D=_log(rng, 256, 2048), H=_log(rng, 128, 1024),
                gated=rng.random() < 0.7, type=rng.choice(["bf16", "bf16", "f16"]), by16=by16)


# ------------------------------------------------------------------------------------------------ inputs
def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _activations(g, rows, cols):
    """Bell-shaped values whose columns differ in size and of which one in a few hundred is an outlier."""
    x = torch.randn(rows, cols, generator=g, device="cuda")
    x *= torch.exp(0.5 * torch.randn(cols, generator=g, device="cuda"))
    return torch.where(torch.rand(rows, cols, generator=g, device="cuda") < 0.003, 12 * x, x)


def _rows16(codes):
    """The codes with rows that begin on multiples of 16 bytes, as the fast products want them."""
    rows, width = codes.shape
    held = torch.zeros(rows, _up(width, 16), dtype=torch.uint8, device="cuda")
    held[:, :width] = codes
    return held[:, :width]


def _empty(rows, cols, by16):
    """Room for a matrix's codes (rows on multiples of 16 bytes) and scales."""
    return (torch.empty(rows, _up((cols + 1) // 2, 16), dtype=torch.uint8, device="cuda")[:, :(cols + 1) // 2],
            torch.empty(_words(cols, by16), rows, dtype=torch.int32, device="cuda"))


def _factor(x, by16):
    """The factor that puts the largest group's scale at e4m3's largest value."""
    return (x.abs().amax() / (6 * 448)).float().reshape(1) if by16 else None


def _route(g, tokens, topk, E):
    """[tokens, topk] different expert numbers of each token, the experts of uneven popularity; a few are dropped (-1)."""
    pull = 0.7 * torch.randn(E, generator=g, device="cuda")
    noise = -torch.log(-torch.log(torch.rand(tokens, E, generator=g, device="cuda").clamp(1e-7, 1 - 1e-6)))
    ids = torch.topk(pull + noise, topk, dim=1).indices.to(torch.int32)
    return torch.where(torch.rand(tokens, topk, generator=g, device="cuda") < 0.01, torch.full_like(ids, -1), ids)


def _weights_in(st, g, at, E, N, K):
    """Codes, scales and factors (one per expert) of E matrices [N x K] under the names that end in `at`."""
    by16 = st["by16"]
    w = torch.randn(E, N, K, generator=g, device="cuda") * K ** -0.5
    f = w.abs().amax((1, 2)) / (6 * 448) if by16 else None
    q, st["S" + at] = _codes(w.view(E * N, K), by16, f.repeat_interleave(N)[:, None] if by16 else None)
    st["W" + at], st["F" + at] = _rows16(q), f


def prepare(case, seed):
    g, op, by16 = _gen(seed), case["op"], case["by16"]
    st = dict(case)
    if op == "quantize":
        rows, cols, t = case["rows"], case["cols"], TYPES[case["type"]]
        back = torch.bfloat16 if t == torch.float32 else t
        st["X"] = _activations(g, rows, cols).to(t)
        st["F"] = _factor(st["X"].float(), by16)
        st["Q"], st["S"] = _empty(rows, cols, by16)
        st["Y"] = torch.empty(rows, cols, dtype=back, device="cuda")
        st["Qt"], st["St"] = _empty(cols, rows, by16) if case["both"] else (None, None)
        st["Yt"] = torch.empty(cols, rows, dtype=back, device="cuda") if case["both"] else None
        return st
    if op == "product":
        for at, rows, x in (("A", case["M"], _activations(g, case["M"], case["K"])),
                            ("B", case["N"], 0.02 * torch.randn(case["N"], case["K"], generator=g, device="cuda"))):
            st["F" + at] = _factor(x, by16)
            q, st["S" + at] = _codes(x, by16, st["F" + at])
            st[at] = _rows16(q)
        st["C"] = torch.empty(case["M"], case["N"], dtype=TYPES[case["out"]], device="cuda")
        return st
    ids = _route(g, case["tokens"], case["topk"], case["E"])
    if op == "experts":
        E, N, K, align = case["E"], case["N"], case["K"], case["align"]
        n = ids.numel()
        rows = n if align == 1 else (n + min(n, E) * (align - 1)) // align * align
        key = ids.reshape(-1).long()
        counts = torch.zeros(E, dtype=torch.int64, device="cuda").index_add_(0, key.clamp(min=0), (key >= 0).long())
        st["starts"] = torch.cat([counts.new_zeros(1), torch.cumsum((counts + align - 1) // align * align, 0)]).to(torch.int32)
        x = _activations(g, rows, K)
        st["FA"] = _factor(x, by16)
        q, st["SA"] = _codes(x, by16, st["FA"])
        st["A"] = _rows16(q)
        _weights_in(st, g, "", E, N, K)
        st["C"] = torch.zeros(rows, N, dtype=TYPES[case["out"]], device="cuda")
        return st
    E, D, H, T, t = case["E"], case["D"], case["H"], case["tokens"], TYPES[case["type"]]
    st["ids"] = ids
    st["w"] = torch.softmax(torch.randn(T, case["topk"], generator=g, device="cuda"), 1)
    st["X"] = torch.randn(T, D, generator=g, device="cuda").to(t)
    _weights_in(st, g, "1", E, (2 if case["gated"] else 1) * H, D)
    _weights_in(st, g, "2", E, D, H)
    st["out"] = torch.empty(T, D, dtype=t, device="cuda")
    # 12 bytes per pair and value of either width, and counters, are what the layer asks for at most
    st["ws"] = torch.empty(12 * ids.numel() * (H + D) + (1 << 16), dtype=torch.uint8, device="cuda")
    return st


def _held(rows, cols, by16):
    """Bytes of codes and scales."""
    return rows * ((cols + 1) // 2) + rows * (-(-cols // _group(by16)))


def work(case):
    op, by16 = case["op"], case["by16"]
    if op == "quantize":
        # read, codes and scales written, read back, values written
        rows, cols = case["rows"], case["cols"]
        held = _held(rows, cols, by16) + (_held(cols, rows, by16) if case["both"] else 0)
        return dict(bytes=rows * cols * (SIZE[case["type"]] + 2 * (2 if case["both"] else 1)) + 2 * held, flops=4 * rows * cols)
    if op == "product":
        M, N, K = case["M"], case["N"], case["K"]
        return dict(bytes=_held(M, K, by16) + _held(N, K, by16) + M * N * SIZE[case["out"]], flops=2 * M * N * K)
    n, E = case["tokens"] * case["topk"], case["E"]
    used = E * (1 - (1 - case["topk"] / E) ** case["tokens"])       # experts that a token reaches, on average
    if op == "experts":
        N, K = case["N"], case["K"]
        return dict(bytes=_held(n, K, by16) + used * _held(N, K, by16) + n * N * SIZE[case["out"]], flops=2 * n * N * K)
    D, H, up = case["D"], case["H"], 2 if case["gated"] else 1
    return dict(bytes=used * (_held(up * H, D, by16) + _held(D, H, by16)) + 2 * case["tokens"] * D * 2 + 8 * n,
                flops=2 * n * D * H * (up + 1))


# ------------------------------------------------------------------------------------------- plain forms
def _codes(x, by16, factor):
    """Codes [rows, bytes] and words of scales [word of columns][row] of a float32 matrix."""
    rows, cols = x.shape
    grp = _group(by16)
    v = torch.nn.functional.pad(x.float(), (0, _up(cols, 4 * grp) - cols)).view(rows, -1, grp)
    a = v.abs().amax(2)
    if by16:
        r = torch.ones_like(factor) / factor
        s = (a * (r / torch.full_like(r, 6.0))).clamp(max=448).to(torch.float8_e4m3fn).float().clamp(min=2.0 ** -9)
        inv, byte = r / s, s.to(torch.float8_e4m3fn).view(torch.uint8)
    else:
        s = a.clamp(min=FLOOR) / torch.full_like(a, 6.0)
        byte = ((s.view(torch.int32) + 0x7FFFFF) >> 23)
        inv = ((254 - byte) << 23).view(torch.float32)
        byte = byte.to(torch.uint8)
    byte = torch.where(torch.arange(byte.shape[1], device=x.device) * grp < cols, byte, torch.zeros_like(byte))
    y = (v * inv[:, :, None]).view(rows, -1)
    m = y.abs()
    c = (m > 0.25).to(torch.uint8) + (m >= 0.75) + (m > 1.25) + (m >= 1.75) + (m > 2.5) + (m >= 3.5) + (m > 5)
    c = c + 8 * torch.signbit(y)
    c = (c[:, 0::2] + 16 * c[:, 1::2])[:, :(cols + 1) // 2].contiguous()
    return c, byte.view(torch.int32).t().contiguous()


def _values(codes, words, cols, by16):
    """What codes and scales stand for (without the factor), float32."""
    table = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6, -0., -.5, -1, -1.5, -2, -3, -4, -6], device=codes.device)
    c = torch.stack([codes & 15, codes >> 4], 2).view(codes.shape[0], -1)[:, :cols]
    byte = words.t().contiguous().view(torch.uint8)
    s = byte.view(torch.float8_e4m3fn).float() if by16 else torch.exp2(byte.float() - 127)
    return table[c.int()] * s.repeat_interleave(_group(by16), 1)[:, :cols]


def _read(codes, words, cols, by16, factor, t):
    v = _values(codes, words, cols, by16)
    return (v if factor is None else v * factor).to(t)


def _experts_of(st, at, N, K):
    """Experts' matrices [E, N, K]."""
    w = _values(st["W" + at], st["S" + at], K, st["by16"]).view(-1, N, K)
    return w if st["F" + at] is None else w * st["F" + at][:, None, None]


def _plain(st):
    op, by16 = st["op"], st["by16"]
    if op == "quantize":
        x = st["X"].float()
        q, s = _codes(x, by16, st["F"])
        y = _read(q, s, st["cols"], by16, st["F"], st["Y"].dtype)
        if not st["both"]:
            return y
        q, s = _codes(x.t(), by16, st["F"])
        return y, _read(q, s, st["rows"], by16, st["F"], st["Y"].dtype)
    if op == "product":
        c = _values(st["A"], st["SA"], st["K"], by16) @ _values(st["B"], st["SB"], st["K"], by16).t()
        return (c * (st["FA"] * st["FB"]) if by16 else c).to(st["C"].dtype)
    if op == "experts":
        # blocks of 64 rows that no expert shares with another
        B, rows, E, starts = 64, st["A"].shape[0], st["E"], st["starts"].long()
        each = (starts[1:] - starts[:-1] + B - 1) // B
        ends, blocks = torch.cumsum(each, 0), _up(rows, B) // B + E
        row = torch.arange(rows, device="cuda")
        e = torch.searchsorted(starts[1:].contiguous(), row, right=True).clamp(max=E - 1)
        place = torch.where(row < starts[-1], (ends - each)[e] * B + row - starts[e], blocks * B)
        of = torch.searchsorted(ends, torch.arange(blocks, device="cuda"), right=True).clamp(max=E - 1)
        a = torch.zeros(blocks * B + 1, st["K"], device="cuda")
        a[place] = _read(st["A"], st["SA"], st["K"], by16, st["FA"], torch.float32)
        c = torch.bmm(a[:-1].view(blocks, B, -1), _experts_of(st, "", st["N"], st["K"])[of].transpose(1, 2)).view(-1, st["N"])
        return torch.cat([c, torch.zeros_like(c[:1])])[place].to(st["C"].dtype)
    E, D, H, T = st["E"], st["D"], st["H"], st["tokens"]
    up = torch.matmul(st["X"].float(), _experts_of(st, "1", (2 if st["gated"] else 1) * H, D).transpose(1, 2))
    h = up[:, :, :H] / (1 + torch.exp(-up[:, :, :H]))
    h = h * up[:, :, H:] if st["gated"] else h
    y = torch.bmm(h, _experts_of(st, "2", D, H).transpose(1, 2))
    ids = st["ids"].long()
    p = torch.zeros(T, E + 1, device="cuda").scatter_add_(1, torch.where(ids < 0, E, ids), st["w"])[:, :E]
    return (y * p.t()[:, :, None]).sum(0).to(st["out"].dtype)


def run(st):
    if not own:
        return _plain(st)
    from paper_2009_06488_b200 import binding as q4
    op, by16 = st["op"], st["by16"]
    if op == "quantize":
        q4.q4_f4_quantize(st["X"], st["Q"], st["S"], st["Qt"], st["St"], by16=by16, factor=st["F"])
        y = q4.q4_f4_dequantize(st["Q"], st["S"], st["Y"], by16=by16, factor=st["F"])
        return (y, q4.q4_f4_dequantize(st["Qt"], st["St"], st["Yt"], by16=by16, factor=st["F"])) if st["both"] else y
    if op == "product":
        return q4.q4_gemm_f4(st["A"], st["SA"], st["B"], st["SB"], st["C"], st["M"], st["N"], st["K"], by16=by16,
                             FA=st["FA"], FB=st["FB"])
    if op == "experts":
        return q4.q4_gemm_f4_experts(st["A"], st["SA"], st["W"], st["S"], st["starts"], st["C"], st["A"].shape[0], st["N"],
                                     st["K"], by16=by16, FA=st["FA"], FB=st["F"])
    return q4.q4_expert_layer_f4(st["X"], st["ids"], st["w"], st["W1"], st["S1"], st["W2"], st["S2"], st["out"], st["E"],
                                 st["H"], st["ws"], gated=st["gated"], by16=by16, F1=st["F1"], F2=st["F2"])


# ---------------------------------------------------------------------------------------- in 64 bits
def _e2m1_64(y):
    """Nearest e2m1 value (steps of a half below 2, of one below 4, else of two), ties to the even code."""
    m = y.abs().clamp(max=6)
    step = torch.where(m < 2, 0.5, torch.where(m < 4, 1.0, 2.0)).double()
    return torch.round(m / step) * step * torch.sign(y)


def _e4m3_64(y):
    _, e = torch.frexp(y)
    step = torch.ldexp(torch.ones_like(y), (e - 4).clamp(min=-9))
    return (torch.round(y / step) * step).clamp(2.0 ** -9, 448)


def _f32(x):
    """A step whose result is a binary32 number by definition."""
    return x.float().double()


def _round_trip_64(x, by16, factor):
    """Values of x's codes; the scales and quotients that the codes are decided by are binary32 numbers."""
    y = torch.empty_like(x)
    grp = _group(by16)
    for c in range(0, x.shape[1], grp):
        part = x[:, c:c + grp]
        a = part.abs().amax(1, keepdim=True)
        if by16:
            r = _f32(1 / factor.double())
            s = _e4m3_64(_f32(a * _f32(r / 6)))
            y[:, c:c + grp] = _e2m1_64(_f32(part * _f32(r / s))) * s * factor.double()
        else:
            m, e = torch.frexp(_f32(a.clamp(min=FLOOR) / 6))
            s = torch.ldexp(torch.ones_like(a), torch.where(m == 0.5, e - 1, e))
            y[:, c:c + grp] = _e2m1_64(_f32(part / s)) * s
    return y


def _decoded_64(codes, words, cols, by16):
    out = torch.empty(codes.shape[0], codes.shape[1] * 2, dtype=torch.float64, device="cuda")
    for half in (0, 1):
        c = (codes >> (4 * half)) & 15
        e, m = ((c >> 1) & 3).double(), (c & 1).double()
        mag = torch.where(e == 0, 0.5 * m, (1 + 0.5 * m) * 2.0 ** (e - 1))
        out[:, half::2] = torch.where(c >= 8, -mag, mag)
    out = out[:, :cols]
    grp = _group(by16)
    for k in range(0, cols, grp):
        word = words[k // (4 * grp)].long()
        byte = (word >> (8 * (k // grp % 4))) & 255
        if by16:
            e, m = ((byte >> 3) & 15).double(), (byte & 7).double()
            s = torch.where(e == 0, m / 8 * 2.0 ** -6, (1 + m / 8) * 2.0 ** (e - 7))
        else:
            s = 2.0 ** (byte.double() - 127)
        out[:, k:k + grp] *= s[:, None]
    return out


def exact(case, seed):
    op, by16 = case["op"], case["by16"]
    st = prepare(case, seed)
    if op == "quantize":
        x = st["X"].double()
        y = _round_trip_64(x, by16, st["F"])
        return (y, _round_trip_64(x.t().contiguous(), by16, st["F"])) if case["both"] else y
    if op == "product":
        a, b = (_decoded_64(st[k], st["S" + k], case["K"], by16) for k in ("A", "B"))
        return a @ b.t() * (st["FA"].double() * st["FB"].double() if by16 else 1)
    one = lambda at, e, N, K: _decoded_64(st["W" + at][e * N:(e + 1) * N], st["S" + at][:, e * N:(e + 1) * N], K, by16) * (
        st["F" + at][e].double() if by16 else 1)
    if op == "experts":
        N, K, at = case["N"], case["K"], st["starts"].tolist()
        a = _decoded_64(st["A"], st["SA"], K, by16) * (st["FA"].double() if by16 else 1)
        c = torch.zeros(a.shape[0], N, dtype=torch.float64, device="cuda")
        for e in range(case["E"]):
            if at[e] < at[e + 1]:
                c[at[e]:at[e + 1]] = a[at[e]:at[e + 1]] @ one("", e, N, K).t()
        return c
    D, H = case["D"], case["H"]
    out = torch.zeros(case["tokens"], D, dtype=torch.float64, device="cuda")
    for e in range(case["E"]):
        t, j = torch.nonzero(st["ids"] == e, as_tuple=True)
        if t.numel():
            up = st["X"][t].double() @ one("1", e, (2 if case["gated"] else 1) * H, D).t()
            h = torch.nn.functional.silu(up[:, :H]) * (up[:, H:] if case["gated"] else 1)
            out.index_add_(0, t, st["w"][t, j, None].double() * (h @ one("2", e, D, H).t()))
    return out
