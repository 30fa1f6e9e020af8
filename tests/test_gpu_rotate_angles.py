"""Cosines and sines of rotary positions alone, to the last bits."""
import numpy as np
import pytest
import torch

from oracle import cache8 as C
from paper_2412_14838_b200 import binding as B
from paper_2412_14838_b200 import build

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    build.build()
    B.load()


@pytest.mark.parametrize("layout,rot", [("half", 128), ("pairs", 128), ("half", 10)])
@pytest.mark.parametrize("first", [0, 5000, 100000, -20000])
def test_cosines_and_sines_to_two_and_a_half_steps(layout, rot, first):
    """Pairs (1, 0) and (0, 1) in fp32 turn into (cos, sin) and (-sin, cos) exactly.  sincospif is good to two steps of its result,
    the rounding of its argument is added back, to first order: of that sum the rounding, half a step, is left.  A step is at most 2^-23
    of the result, so 2.5 * 2^-23 of it.  Then what 64 bits lose: an angle of t radians is off by 2^-53 t in each of the power, the division
    and the product on both sides, 8 * 2^-53 t in all, and the correction by 2^-23 of the argument's rounding, pi 2^-25 * 2^-23, and
    by its square, 2^-47.  Without the correction results near 0 would be off by up to pi 2^-25 = 9e-8, more than is allowed for all that are
    below 0.3."""
    T = 4000
    f, _ = C.frequencies(rot, 10000.0)
    r = B.dkv_rotary_init(128, rot, B.DKV_ROTARY_HALF if layout == "half" else B.DKV_ROTARY_PAIRS, 10000.0)
    pos = torch.arange(first, first + T, dtype=torch.int32, device="cuda")[None].contiguous()
    a, b = (slice(0, rot // 2), slice(rot // 2, rot)) if layout == "half" else (slice(0, rot, 2), slice(1, rot, 2))
    x = torch.zeros(1, 2, T, 128, device="cuda")
    x[:, 0, :, a], x[:, 1, :, b] = 1.0, 1.0
    out = torch.empty_like(x)
    B.dkv_rotate(r, pos, x, out)
    t = pos[0].double().cpu().numpy()[:, None] * np.array(f)
    got, small = out[0].double().cpu().numpy(), 0
    for value, want in ((got[0][:, a], np.cos(t)), (got[0][:, b], np.sin(t)), (got[1][:, a], -np.sin(t)), (got[1][:, b], np.cos(t))):
        allowed = 2.5 * 2.0 ** -23 * np.abs(want) + 8 * 2.0 ** -53 * np.abs(t) + 2.0 ** -46
        off = np.abs(value - want)
        assert (off <= allowed).all(), (off / allowed).max()
        small += (allowed < 2.0 ** -26).sum()
    assert small > 1000                                                      # results that tell the correction
