"""The expert layer's bound on the activations that enter its products: seven base-8 digits below a power of two keep it, six
do not, and the cases below (run on the GPU by test_gpu_f4_layer_digits.py) tell the two apart.

An activation is rounded to whole steps of 2^-18 under a power of two 2^a of its group, a = floor(log2 of the largest) - 1; by 16
a is 18 powers below the row's own at most.  What is rounded is split in digits of -4 .. 3 and a first one of -4 .. 4."""
import numpy as np
import pytest

from oracle import f4


def as_parts(v, by16, parts=7):
    """Rows of values as the sum of their first `parts` parts."""
    g = f4.group_of(by16)
    rows, cols = v.shape
    m = np.zeros((rows, -(-cols // g) * g))
    m[:, :cols] = np.abs(v)
    m = m.reshape(rows, -1, g).max(axis=2)
    a = np.floor(np.log2(np.maximum(m, 2.0 ** -125))) - 1
    if by16:
        a = np.maximum(a, np.maximum(np.floor(np.log2(np.maximum(m.max(axis=1, keepdims=True), 2.0 ** -149))), -107) - 18)
    step = np.repeat(2.0 ** (a - 18), g, axis=1)[:, :cols]
    n = np.round(v / step)                       # ties to even
    assert (np.abs(n) <= 2.0 ** 20).all()
    for q in range(6, parts - 1, -1):            # the last parts off
        unit = 8.0 ** (6 - q)
        n -= (np.mod(n / unit + 4, 8) - 4) * unit
    return n * step


def layer_of(x, ids, w1, w2, by16, parts_x=7, parts_h=7):
    """The layer (without gate) on activations of so many parts, otherwise in 64 bits."""
    out = np.zeros_like(x)
    x = as_parts(x, by16, parts_x)
    for t, e in enumerate(ids[:, 0]):
        h = w1[e] @ x[t]
        h = h / (1 + np.exp(-h))
        out[t] = w2[e] @ as_parts(h[None], by16, parts_h)[0]
    return out


class Digits:
    """16 tokens, 2 experts, one group wide.  where == "x": a token's first value is 2^12 times its second, and only the second
    meets weights that are not 0.  where == "h": the first hidden value is 2^12 times the others, and the weights behind it
    are 0.  w2 picks one hidden value for each output, so no error is averaged."""

    def __init__(self, where, by16):
        r = np.random.default_rng(17 + by16)
        g = self.G = f4.group_of(by16)
        self.by16, self.where = by16, where
        x = np.zeros((16, g))
        c1, c2 = np.zeros((2, g, g), dtype=np.uint8), np.zeros((2, g, g), dtype=np.uint8)
        s1 = np.full((2, g, 1), 0x38 if by16 else 127, dtype=np.uint8)        # 1
        if where == "x":
            x[:, 0], x[:, 1] = 4096 * r.uniform(1, 2, 16), r.uniform(1, 2, 16)
            c1[:, :, 1] = r.integers(1, 8, (2, g))
            first = 0
        else:
            x[:] = r.uniform(0.5, 1, (16, g))
            c1[:] = r.integers(1, 4, (2, g, g))
            s1[:, 0], s1[:, 1:] = (0x7E, 0x20) if by16 else (127 + 9, 127 - 3)    # 448 and 1/8; 2^9 and 1/8
            first = 1
        for d in range(g):
            c2[:, d, max(d, first)] = 2                                        # 1
        self.x = x.astype(np.float16).astype(np.float64)
        self.ids = r.integers(0, 2, (16, 1)).astype(np.int32)
        one = np.full((2 * g, 1), 0x38 if by16 else 127, dtype=np.uint8)
        self.q1, self.s1 = f4.pack(c1.reshape(-1, g)), f4.to_words(s1.reshape(-1, 1))
        self.q2, self.s2 = f4.pack(c2.reshape(-1, g)), f4.to_words(one)
        self.w1, self.w2 = (f4.values(q, s, g, by16).reshape(2, g, g) for q, s in ((self.q1, self.s1), (self.q2, self.s2)))

    def outside(self, got):
        """How many outputs, rounded to binary16, are further off than the layer may be."""
        want, off = f4.layer(self.x, self.ids, None, self.w1, self.w2, False, self.by16)
        return (np.abs(got - want) > off + (np.abs(want) + off) * 2.0 ** -11 + 2.0 ** -25).sum()


def far_below(by16):
    """(x, w1, w2): tokens whose first group holds 1 and meets weights that are 0, and whose second one holds values 2^-d."""
    g = f4.group_of(by16)
    r = np.random.default_rng(23)
    x = np.zeros((40, 2 * g))
    x[:, 0] = 1
    x[:, g:] = r.uniform(1, 2, (40, g)) * 2.0 ** -np.arange(1.0, 41)[:, None]
    x = (x * 2.0 ** 60).astype(np.float32).view(np.uint32) & 0xFFFF0000                       # to bfloat16, towards 0
    x = x.view(np.float32).astype(np.float64) * 2.0 ** -60
    c = np.zeros((g, 2 * g), dtype=np.uint8)
    c[np.arange(g), g + np.arange(g)] = r.integers(1, 8, g)
    one = np.full((g, 2), 0x38 if by16 else 127, dtype=np.uint8)
    q1, s1 = f4.pack(c), f4.to_words(one)
    q2, s2 = f4.pack(np.concatenate([2 * np.eye(g), 2 * np.eye(g)]).astype(np.uint8)), f4.to_words(np.full((2 * g, 1), one[0, 0], dtype=np.uint8))
    return x, q1, s1, q2, s2


@pytest.mark.parametrize("by16", [False, True])
def test_seven_parts_keep_the_bound(by16):
    r = np.random.default_rng(5)
    v = r.standard_normal((50, 200)) * 2.0 ** (r.uniform(-40, 40, (50, 200)) * r.integers(0, 2, (50, 1)))
    off = np.abs(as_parts(v, by16) - v)
    assert all((o <= f4.entered(x, by16)).all() for o, x in zip(off, v))
    assert any((o > f4.entered(x, by16)).any() for o, x in zip(np.abs(as_parts(v, by16, 6) - v), v))


@pytest.mark.parametrize("by16", [False, True])
@pytest.mark.parametrize("where", ["x", "h"])
def test_the_cases_see_every_part(where, by16):
    c = Digits(where, by16)
    rounded = lambda **k: layer_of(c.x, c.ids, c.w1, c.w2, by16, **k).astype(np.float16).astype(np.float64)
    assert c.outside(rounded()) == 0
    for parts in range(1, 7):
        assert c.outside(rounded(**{"parts_" + where: parts})) > 10


def test_by_16_a_small_group_has_the_rows_steps():
    """2^-20 of a group's largest is not kept where it is 2^-17 of the row's largest: 2^-37 of that is."""
    x, q1, s1, q2, s2 = far_below(True)
    off = np.abs(as_parts(x, True) - x)[:, 16:]
    assert (off[30:] > x[30:, 16:].max(axis=1, keepdims=True) * 2.0 ** -20).any()
    assert all((np.abs(as_parts(r[None], True)[0] - r) <= f4.entered(r, True)).all() for r in x)
