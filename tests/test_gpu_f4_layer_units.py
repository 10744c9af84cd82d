"""Expert layer for a few tokens where each thread block walks several units (up to four or eight pairs of one expert): the
buffers of their parts, the rows' factors and the accumulators go from hand to hand.

Tokens differ by powers of two, so that a factor or a part of another unit's row would show."""
import numpy as np
import pytest

from test_gpu_f4_layer import Case

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def q4():
    from paper_2009_06488_b200 import binding
    binding.q4_set_variant(0)
    return binding


def most_units(ids, E, per, rows):
    """Units of one block at most, where a unit is up to `per` pairs of an expert and `rows` of its tiles' rows are 128."""
    import torch
    units = sum(-(-int((ids == e).sum()) // per) for e in range(E))
    each, blocks = -(-rows // 128), torch.cuda.get_device_properties(0).multi_processor_count
    ends = [units * each * b // blocks for b in range(blocks + 1)]
    return max((hi - 1) // each - lo // each + 1 for lo, hi in zip(ends, ends[1:]) if hi > lo)


def scaled(c, seed):
    """The case with tokens of sizes 2^-9 to 2^9."""
    import torch
    r = np.random.default_rng(seed)
    c.X.mul_(torch.from_numpy(2.0 ** r.integers(-9, 10, c.X.shape[0])).to(c.X.dtype).cuda()[:, None])
    c.x = c.X.double().cpu().numpy()
    return c


@pytest.mark.parametrize("gated,H", [(True, 64), (False, 128), (True, 17)])
def test_five_units_and_more_of_one_tile_each(q4, gated, H):
    """By 16 a unit's rows have factors in one of four slots."""
    c = scaled(Case(81, 128, 8, 1024, 64, H, gated, True, "bf16"), 82)
    c.ids = np.random.default_rng(83).permutation(1024).reshape(128, 8).astype(np.int32)
    assert most_units(c.ids, 1024, 4, H * (2 if gated else 1)) >= 6 and most_units(c.ids, 1024, 4, 64) >= 6
    c.run(q4).check()
