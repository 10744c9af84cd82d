"""Pins of the e4m3 / expert-layer oracle: hand-computed codes, closed forms, and the gradients of its
formulas against differences."""
import numpy as np
import pytest

from oracle import f8


def test_e4m3_values_by_hand():
    t = f8.decode_table()
    assert t[0x00] == 0 and t[0x01] == 2.0 ** -9 and t[0x07] == 7 * 2.0 ** -9 and t[0x08] == 2.0 ** -6
    assert t[0x38] == 1.0 and t[0x39] == 1.125 and t[0x7E] == 448.0 and np.isnan(t[0x7F]) and np.isnan(t[0xFF])
    assert t[0xB8] == -1.0 and t[0x40] == 2.0
    assert (np.diff(t[:127]) > 0).all()


def test_encoding_rounds_to_nearest_with_ties_to_even():
    t = f8.decode_table()
    assert (f8.encode(t[:127]) == np.arange(127)).all() and (f8.encode(-t[1:127]) == np.arange(1, 127) + 128).all()
    mid = (t[:126] + t[1:127]) / 2
    even = np.where(np.arange(126) % 2 == 0, np.arange(126), np.arange(126) + 1)
    assert (f8.encode(mid) == even).all()
    assert (f8.encode(np.nextafter(mid, 1e9)) == np.arange(1, 127)).all()
    assert (f8.encode(np.nextafter(mid, 0)) == np.arange(126)).all()
    assert f8.encode(np.array([1e9, np.nan, -0.0])).tolist() == [0x7E, 0x7F, 0x80]


def test_scales_by_hand():
    x = np.zeros((2, 256), dtype=np.float32)
    x[0, 3], x[0, 200], x[1, 0] = 448.0, -7.0, 3.5
    q, s = f8.quantize(x)
    assert s.shape == (2, 2) and s[0, 0] == 1.0 and s[1, 0] == np.float32(7) / np.float32(448)
    assert q[0, 3] == 0x7E and q[0, 200] == 0xFE and q[1, 0] == 0x7E and q[1, 1] == 0
    assert s[1, 1] == f8.FLOOR / np.float32(448)
    _, s = f8.quantize(x, pow2=True)
    assert s[0, 0] == 1.0 and s[1, 0] == 2.0 ** -6 and s[0, 1] == 2.0 ** -7
    x[0, 3] = 449.0
    assert f8.quantize(x, pow2=True)[1][0, 0] == 2.0
    q, s = f8.quantize(x, blocks=True)
    assert s.shape == (1, 2) and s[0, 0] == np.float32(449) / np.float32(448) and q[1, 0] == f8.encode(3.5 * 448 / 449)


@pytest.mark.parametrize("blocks", [False, True])
@pytest.mark.parametrize("pow2", [False, True])
def test_quantized_values_are_near(blocks, pow2):
    r = np.random.default_rng(3)
    x = (r.standard_normal((200, 300)) * np.exp(r.standard_normal(300))).astype(np.float32)
    v = f8.values(*f8.quantize(x, blocks, pow2), blocks=blocks)
    # nearest of 3 mantissa bits: 2^-4 relative, or half the smallest step (2^-10) times the scale
    s = f8.quantize(x, blocks, pow2)[1].max()
    assert (np.abs(v - x) <= np.maximum(np.abs(x) * 2.0 ** -4 * (1 + 1e-6), s * 2.0 ** -10 * (1 + 1e-6))).all()


def test_not_finite_values_spoil_their_block_only():
    x = np.ones((3, 256), dtype=np.float32)
    x[0, 5], x[1, 130] = np.inf, np.nan
    q, s = f8.quantize(x)
    assert np.isinf(s[0, 0]) and np.isnan(s[1, 1]) and np.isfinite(s[[1, 0], [0, 1]]).all()
    with np.errstate(all="ignore"):
        c, _ = f8.product(q, s, q, s, b_rows=True)
    assert np.isnan(c[:2]).all() and np.isnan(c[2, :2]).all() and c[2, 2] == pytest.approx(256, rel=1e-6)


def test_sort_by_hand():
    ids = np.array([[2, 0], [0, -1], [2, 5]], dtype=np.int32)
    starts, source, slot = f8.sort(ids, 4, 1, 6)
    assert starts.tolist() == [0, 2, 2, 4, 4] and source.tolist() == [1, 2, 0, 4, -1, -1]
    assert slot.tolist() == [[2, 0], [1, -1], [3, -1]]
    starts, source, slot = f8.sort(ids, 4, 4, f8.sort_rows(6, 4, 4))
    assert starts.tolist() == [0, 4, 4, 8, 8] and source.tolist()[:8] == [1, 2, -1, -1, 0, 4, -1, -1]
    assert f8.sort_rows(6, 4, 4) == 16


def test_gradients_against_differences():
    r = np.random.default_rng(5)
    T, k, D, E = 7, 3, 11, 5
    ids = np.stack([r.permutation(E)[:k] for _ in range(T)]).astype(np.int32)
    ids[2, 1] = -1
    starts, source, slot = f8.sort(ids, E, 4, f8.sort_rows(T * k, E, 4))
    y, w, g = r.standard_normal((source.size, D)), r.standard_normal((T, k)), r.standard_normal((T, D))
    loss = lambda y, w: (f8.combine(y, slot, w) * g).sum()
    dy, dw = f8.combine_grad(g, y, slot, w)
    h = 1e-6
    for at in [(0, 0), (3, 2), (2, 1), (6, 1)]:
        d = np.zeros_like(w); d[at] = h
        assert dw[at] == pytest.approx((loss(y, w + d) - loss(y, w - d)) / (2 * h), abs=1e-8)
    for at in [(0, 0), (1, 4), (source.size - 1, 3)]:
        d = np.zeros_like(y); d[at] = h
        assert dy[at] == pytest.approx((loss(y + d, w) - loss(y - d, w)) / (2 * h), abs=1e-8)
    # the gather's gradient is the unweighted combine
    x, gx = r.standard_normal((T, D)), r.standard_normal((source.size, D))
    dx = f8.combine(gx, slot)
    for at in [(0, 0), (2, 5), (6, 10)]:
        d = np.zeros_like(x); d[at] = h
        diff = ((f8.gather(x + d, source, k) - f8.gather(x - d, source, k)) * gx).sum() / (2 * h)
        assert dx[at] == pytest.approx(diff, abs=1e-8)
