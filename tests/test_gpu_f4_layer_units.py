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


# ------------------------------------------------------------------------------- buffers from unit to unit
# T, topk, E, D, H, gated, by16, pairs per unit, units of a block in the first and the second kernel at least
CHAINS = [(128, 8, 256, 64, 160, True, False, 8, 3, 2), (128, 8, 1024, 64, 100, True, False, 4, 6, 6), (128, 8, 1024, 300, 200, False, True, 4, 6, 6),
          (50, 6, 300, 2880, 16, True, True, 4, 2, 2),         # four pairs' parts of the first kernel fill one buffer
          (50, 6, 300, 24, 2880, False, True, 4, 2, 2),        # ... of the second
          (128, 8, 100, 2048, 64, True, False, 8, 2, 2),       # eight pairs' of the first
          (128, 8, 100, 100, 2048, False, False, 8, 2, 2)]


@pytest.mark.parametrize("T,topk,E,D,H,gated,by16,per,up,down", CHAINS)
def test_parts_of_one_unit_after_another(q4, T, topk, E, D, H, gated, by16, per, up, down):
    """A unit's parts are written where an earlier unit's were read, with two buffers and with one."""
    c = scaled(Case(T + E + D, T, topk, E, D, H, gated, by16, "bf16"), E)
    assert (T * topk > 3 * E) == (per == 8)
    if T * topk <= E:                            # every expert once
        c.ids = np.random.default_rng(D).permutation(E)[:T * topk].reshape(T, topk).astype(np.int32)
    assert most_units(c.ids, E, per, H * (2 if gated else 1)) >= up and most_units(c.ids, E, per, D) >= down
    c.run(q4).check()
    first = c.Out.clone()
    c.Out.fill_(9)
    c.run(q4)
    assert (c.Out == first).all()
