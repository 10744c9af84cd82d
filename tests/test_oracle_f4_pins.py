"""The 4-bit float oracle against values written by hand from the formats' definitions."""
import numpy as np

from oracle import f4


def test_codes_round_to_the_nearest_value_and_ties_to_the_even_code():
    pairs = [(0, 0), (0.25, 0), (0.26, 1), (0.5, 1), (0.74, 1), (0.75, 2), (1.25, 2), (1.26, 3), (1.5, 3), (1.75, 4), (2.5, 4),
             (2.51, 5), (3.49, 5), (3.5, 6), (5.0, 6), (5.01, 7), (6, 7), (1e9, 7), (-0.5, 9), (-7, 15), (-0.0, 8), (-0.1, 8)]
    y, c = zip(*pairs)
    assert f4.encode(np.array(y)).tolist() == list(c)


def test_codes_are_packed_low_half_first():
    assert f4.pack(np.array([[1, 2, 3]], dtype=np.uint8)).tolist() == [[0x21, 0x03]]
    assert f4.unpack(np.array([[0x21, 0x03]], dtype=np.uint8), 3).tolist() == [[1, 2, 3]]


def test_a_scale_is_the_next_power_of_two():
    x = np.zeros((5, 40), dtype=np.float32)
    x[0, :2] = [6, -3]                       # 6 fits 1
    x[1, 0] = np.nextafter(np.float32(6), np.float32(7))       # needs 2
    x[2, 0], x[2, 35] = 0.75, 48             # 2^-3, 8
    x[3, 3] = np.nan
    q, s = f4.quantize(x)
    assert s.shape == (1, 5) and q.shape == (5, 20)
    byte = f4.from_words(s, 5)
    assert byte[:, 0].tolist()[:4] == [127, 128, 124, 255] and byte[2, 1] == 130 and (byte[:, 2:] == 0).all()
    assert byte[4, 0] == 127 - 62            # the floor: 2^-60 / 6 is above 2^-63
    assert f4.unpack(q, 2)[0].tolist() == [7, 13]


def test_scales_by_16_are_e4m3_times_the_factor():
    x = np.zeros((1, 33), dtype=np.float32)
    x[0, 0], x[0, 16], x[0, 32] = 6 * 448, -6 * 0.5, 6 * 2.0 ** -9
    q, s = f4.quantize(x, by16=True)
    assert f4.from_words(s, 1)[0].tolist() == [0x7E, 0x30, 1, 0]
    assert f4.values(q, s, 33, True)[0, [0, 16, 32]].tolist() == [2688, -3, 6 * 2.0 ** -9]
    q, s = f4.quantize(x / 4, by16=True, factor=0.25)
    assert f4.from_words(s, 1)[0].tolist() == [0x7E, 0x30, 1, 0]
    assert f4.values(q, s, 33, True, 0.25)[0, 0] == 672
    q, s = f4.quantize(np.zeros((1, 16), dtype=np.float32), by16=True)
    assert f4.from_words(s, 1)[0, 0] == 1 and not q.any()


def test_the_layer_by_hand():
    x = np.array([[1.0, 2.0], [0.5, 0.0]])
    w1 = np.array([[[1.0, 0.0], [0.0, 3.0]], [[2.0, 0.0], [4.0, 0.0]]])        # two experts, H = 1, gated
    w2 = np.array([[[1.0], [2.0]], [[-1.0], [0.5]]])
    silu = lambda v: v / (1 + np.exp(-v))
    ids, w = np.array([[0, 1], [1, -1]]), np.array([[0.5, 0.25], [2.0, 9.0]])
    h0, h1, h2 = silu(1.0) * 6, silu(2.0) * 4, silu(1.0) * 2
    want = np.array([[0.5 * h0 - 0.25 * h1, h0 + 0.125 * h1], [-2 * h2, h2]])
    assert np.allclose(f4.layer(x, ids, w, w1, w2, True)[0], want, rtol=1e-14)


def test_a_factor_of_zero_stands_for_a_matrix_of_zeros():
    """1 / factor and its quotient by the scale end at binary32's largest value: zeros times it are zeros."""
    x = np.zeros((2, 40), dtype=np.float32)
    x[1] = -0.0
    for factor in (np.float32(0), np.float32(1e-45), np.float32(1)):
        q, s = f4.quantize(x, by16=True, factor=factor)
        assert f4.from_words(s, 2).tolist() == [[1, 1, 1, 0]] * 2
        assert f4.unpack(q, 40).tolist() == [[0] * 40, [8] * 40]
        assert (f4.values(q, s, 40, True, factor) == 0).all()
    x[0, :3] = [2.0 ** -140, -2.0 ** -149, 0]                 # a factor that is 0 in binary32: nothing but saturated quotients
    q, s = f4.quantize(x, by16=True, factor=np.float32(0))
    assert f4.from_words(s, 2)[0].tolist() == [1, 1, 1, 0] and f4.unpack(q, 3)[0].tolist() == [0, 8, 0]
    x[0, 0] = 1
    q, s = f4.quantize(x, by16=True, factor=np.float32(0))
    assert f4.from_words(s, 2)[0].tolist() == [0x7E, 1, 1, 0] and f4.unpack(q, 3)[0].tolist() == [7, 8, 0]
