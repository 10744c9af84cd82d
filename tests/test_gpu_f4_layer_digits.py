"""Expert layer for a few tokens where the low digits of activations decide the result, on the GPU: large values beside small
ones, in X and in the hidden values (the cases of test_oracle_f4_parts.py, which shows that they see every digit)."""
import numpy as np
import pytest

from oracle import f4
from test_gpu_f4 import HALF_SMALLEST, HALF_ULP, placed, up16, word_tensor
from test_gpu_f4_layer import Case
from test_oracle_f4_parts import Digits, far_below

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def q4():
    from paper_2009_06488_b200 import binding
    binding.q4_set_variant(0)
    return binding


def layer(q4, x, ids, q1, s1, q2, s2, E, H, by16):
    import torch
    out = torch.full_like(x, 9)
    ws = torch.empty(q4.q4_expert_layer_f4_workspace_bytes(*ids.shape, x.shape[1], H), dtype=torch.uint8, device="cuda")
    q4.q4_expert_layer_f4(x, torch.from_numpy(ids).cuda(), None, placed(q1, up16(q1.shape[1])), word_tensor(s1), placed(q2, up16(q2.shape[1])),
                          word_tensor(s2), out, E, H, ws, gated=False, by16=by16)
    return out.double().cpu().numpy()


@pytest.mark.parametrize("by16", [False, True])
@pytest.mark.parametrize("where", ["x", "h"])
def test_every_digit_counts(q4, where, by16):
    import torch
    c = Digits(where, by16)
    x = torch.from_numpy(c.x).cuda().half()
    assert c.outside(layer(q4, x, c.ids, c.q1, c.s1, c.q2, c.s2, 2, c.G, by16)) == 0


@pytest.mark.parametrize("by16", [False, True])
def test_groups_far_below_their_row(q4, by16):
    import torch
    x, q1, s1, q2, s2 = far_below(by16)
    g = f4.group_of(by16)
    X = torch.from_numpy(x).cuda().bfloat16()
    assert (X.double().cpu().numpy() == x).all()
    ids = np.zeros((40, 1), dtype=np.int32)
    got = layer(q4, X, ids, q1, s1, q2, s2, 1, g, by16)
    want, off = f4.layer(x, ids, None, f4.values(q1, s1, 2 * g, by16)[None], f4.values(q2, s2, g, by16)[None], False, by16)
    assert (np.abs(got - want) <= off + (np.abs(want) + off) * HALF_ULP["bf16"] + HALF_SMALLEST["bf16"]).all()


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("t,spread", [("bf16", 30.0), ("f16", 4.0)])
def test_values_of_any_size_by_16(q4, t, spread, gated):
    Case(21, 8, 2, 4, 512, 128, gated, True, t, spread=spread).run(q4).check()
