"""The cache in 8 bits at the ends of its range, against the oracle: values near the largest and smallest numbers, long sums,
more sequences than one pass of the planner takes, and calls that only documents allow."""
import numpy as np
import pytest
import torch

from oracle import cache8 as C
from paper_2412_14838_b200 import binding as B
from paper_2412_14838_b200 import build
from tests.test_gpu_cache8 import Both

pytestmark = pytest.mark.gpu
BIG = float(torch.finfo(torch.bfloat16).max)


@pytest.fixture(scope="module", autouse=True)
def _lib():
    build.build()
    B.load()


def put(c, first, n, k, v):
    """Rows k, v [n, Hkv, rows, D] behind those of sequences first, first + 1, .. on both sides."""
    rows = k.shape[2]
    B.dkv_cache8_reserve(c.h, first, n, 1, None, rows)
    c.o.reserve(range(first, first + n), [rows] * n)
    B.dkv_cache8_append(c.h, first, n, 1, k, v)
    for i in range(n):
        c.o.append(first + i, k[i].double().cpu().numpy(), v[i].double().cpu().numpy())


def signs(n, Hkv, rows, D, size):
    """+size and -size by turns, with ones between them: averages stay far below `size`."""
    x = torch.full((n, Hkv, rows, D), size, device="cuda")
    x[:, :, 1::2] *= -1.0
    x[..., 1::2] = 1.0
    return x.to(torch.bfloat16)


@pytest.mark.parametrize("kind", ["e4m3", "int8"])
@pytest.mark.parametrize("held,more", [(5, 20), (20, 9), (3, 2)])            # rounded again by append8_kernel; by nobody
def test_the_largest_numbers_stay_what_they_are_behind_other_rows(kind, held, more):
    """Such a number is 256 * 2^120 as an e4m3 value and 64 * 2^122 as an int8 one: more than any fp32 number."""
    with Both(kind=kind, n_seqs=2) as c:
        x = signs(2, 2, held, 64, BIG)
        put(c, 0, 2, x, x)
        y = torch.ones(2, 2, more, 64, device="cuda").to(torch.bfloat16)
        put(c, 0, 2, y, y)
        c.check()
        c.attend(0, 2, 1, 1, False, scale=0.0)                               # q = 0: the average of all rows
