"""The cache in 8 bits at the ends of its range, against the oracle: values near the largest and smallest numbers, long sums,
more sequences than one pass of the planner takes, and calls that only documents allow."""
import ctypes

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


@pytest.mark.parametrize("kind", ["e4m3", "int8"])
def test_the_largest_numbers_stay_what_they_are_in_a_compaction(kind):
    with Both(kind=kind, n_seqs=2, D=128) as c:
        x = signs(2, 2, 40, 128, BIG)
        x[1, :, 7:30] = 2.0 ** -100                                          # a page whose values are far apart
        put(c, 0, 2, x, -x)
        idx = [np.stack([np.arange(39, 2, -1), np.arange(37)]) for _ in range(2)]
        B.dkv_cache8_compact(c.h, 0, 2, 1, torch.tensor(np.stack(idx), dtype=torch.int32, device="cuda"))
        c.o.compact([0, 1], [i.tolist() for i in idx])
        c.check()
        c.attend(0, 2, 1, 1, False, scale=0.0)


@pytest.mark.parametrize("size", [2.0 ** -121, 2.0 ** -127, 2.0 ** -133])
def test_the_smallest_numbers_in_a_compaction(size):
    with Both(n_seqs=1) as c:
        x = (torch.randint(-64, 65, (1, 2, 50, 64), device="cuda") * (size / 64 if size > 2.0 ** -127 else size)).to(torch.bfloat16)
        put(c, 0, 1, x, x.flip(2))
        idx = np.stack([np.arange(49, 9, -1), np.arange(40)])
        B.dkv_cache8_compact(c.h, 0, 1, 1, torch.tensor(idx[None], dtype=torch.int32, device="cuda"))
        c.o.compact([0], [idx.tolist()])
        c.check()


@pytest.mark.parametrize("kind", ["e4m3", "int8"])
@pytest.mark.parametrize("rows", [4, 20])
def test_infinities_are_the_largest_code_of_a_page_of_the_largest_numbers(kind, rows):
    """448 * 2^120 or 127 * 2^122: seen by attention, whose average of one such row among many is an fp32 number."""
    with Both(kind=kind, n_seqs=1) as c:
        y = torch.ones(1, 2, 28, 64, device="cuda").to(torch.bfloat16)
        put(c, 0, 1, y, y)
        x = signs(1, 2, rows, 64, BIG)
        x[0, 0, 0, 0], x[0, 1, 2, 6], x[0, 0, 1, 3] = float("inf"), float("-inf"), float("nan")
        put(c, 0, 1, x, x)
        c.attend(0, 1, 1, 1, False, scale=0.0)
        put(c, 0, 1, y[:, :, :9], y[:, :, :9])                               # rounded again
        c.attend(0, 1, 1, 1, False, scale=0.0)
        idx = np.stack([np.arange(c.o.len[0])] * 2)
        B.dkv_cache8_compact(c.h, 0, 1, 1, torch.tensor(idx[None], dtype=torch.int32, device="cuda"))
        c.o.compact([0], [idx.tolist()])
        c.attend(0, 1, 1, 1, False, scale=0.0)


@pytest.mark.parametrize("layout,rot", [("half", 64), ("pairs", 32), ("half", 10)])
@pytest.mark.parametrize("T", [5, 20])
@pytest.mark.parametrize("kind", ["e4m3", "int8"])
def test_a_negative_amplitude_turns_keys_into_the_negatives_of_a_positive_one_s(layout, rot, T, kind):
    """dkv_rotary is plain data of the caller's: near the largest numbers the products pass fp32's range, with either sign."""
    r = [B.dkv_rotary_init(64, rot, B.DKV_ROTARY_HALF if layout == "half" else B.DKV_ROTARY_PAIRS, 10000.0) for _ in range(2)]
    r[0].amplitude, r[1].amplitude = 3.0, -3.0
    with Both(n_seqs=2, oracle=False, kind=kind) as c:
        k = torch.randn(1, 2, T, 64, device="cuda")
        k[:, 0, T // 2:] *= 1e38
        k[:, 1, 0, 3] = 3e38
        k = k.to(torch.bfloat16)
        k[..., rot:] = 0.0
        pos0 = torch.tensor([100], dtype=torch.int32, device="cuda")
        B.dkv_cache8_reserve(c.h, 0, 2, 1, None, T)
        found = []
        for s in range(2):
            B.dkv_cache8_append(c.h, s, 1, 1, k, torch.zeros_like(k), None, r[s], pos0)
            found.append(B.dkv_cache8_status(c.h)[1][0])
        got = c.read(0, 2, 1, T)[0]
        assert np.isfinite(got).all() and (got[0] == -got[1]).all()
        assert found[0] == found[1]
        q, out = torch.randn(2, 4, 1, 64, device="cuda").to(torch.bfloat16) * 0, torch.zeros(2, 4, 1, 64, device="cuda")
        B.dkv_cache8_attend(c.h, 0, 2, 1, q, out)
        assert (out == 0).all()                                              # logits of 0 * key: NaN were a key NaN or infinite


@pytest.mark.parametrize("n_pages", [3150, 2200])                            # pages for everybody; too few
def test_forks_among_more_sequences_than_the_planner_takes_at_a_time(n_pages):
    """Who copies a shared page, and which pages are free, goes by what the call finds, for all its sequences."""
    n = 2100
    with Both(n_pages=n_pages, n_seqs=n, max_pages=2, Hkv=1, G=1) as c:
        c.add(0, n // 2, 1, [i % 3 + 30 for i in range(n // 2)], 3, cap=32)  # 32: full pages, which are not copied
        B.dkv_cache8_fork(c.h, 0, n // 2, n // 2, 1)
        c.o.fork([(i, i + n // 2) for i in range(n // 2)])
        none, full = c.o.reserve(range(n), [1] * n)
        B.dkv_cache8_reserve(c.h, 0, n, 1, None, 1)
        c.check()
        words = B.dkv_cache8_status(c.h)[1]
        assert bool(words[0] & B.DKV_C8_NO_PAGES) == bool(none) and not full and words[2] == sum(r == 0 for r in c.o.refs())
        assert bool(none) == (n_pages < 3150)
        B.dkv_cache8_reserve(c.h, 0, n, 1, None, 1)                          # what was given back is found again
        c.o.reserve(range(n), [1] * n)
        c.check()


@pytest.mark.parametrize("n", [1, 80])                                       # slices of blocks, of warps
@pytest.mark.parametrize("rows", [20, 700])
def test_an_infinite_query_whose_logits_are_all_minus_infinity_gives_nan(n, rows):
    with Both(n_pages=n * 24, n_seqs=n, max_pages=24) as c:
        k = torch.randn(n, 2, rows, 64, device="cuda").abs().to(torch.bfloat16) + 0.5
        put(c, 0, n, k, k)
        q = torch.randn(n, 4, 2, 64, device="cuda").to(torch.bfloat16)
        q[0, 1, 1, 5] = float("-inf")
        out, lse = torch.zeros(q.shape, device="cuda"), torch.zeros(q.shape[:3], device="cuda")
        B.dkv_cache8_attend(c.h, 0, n, 1, q, out, lse)
        odd = torch.zeros(n, 4, 2, dtype=torch.bool, device="cuda")
        odd[0, 1, 1] = True
        assert torch.isnan(out[odd]).all() and torch.isnan(lse[odd]).all()
        assert torch.isfinite(out[~odd]).all() and torch.isfinite(lse[~odd]).all()


@pytest.mark.parametrize("size", [2.0 ** -120, 1e-35, 1e-33, 1e-30])
@pytest.mark.parametrize("n,Hkv,rows", [(1, 2, 3000), (1, 1, 40), (60, 3, 100)])      # slices of blocks, one slice, slices of warps
def test_attention_over_values_near_the_smallest(size, n, Hkv, rows):
    with Both(n_pages=n * (rows // 32 + 1) + 4, n_seqs=n, max_pages=rows // 32 + 1, Hkv=Hkv) as c:
        k = torch.randn(n, Hkv, rows, 64, device="cuda").to(torch.bfloat16)
        v = (torch.randn(n, Hkv, rows, 64, device="cuda") * size).to(torch.bfloat16)
        put(c, 0, n, k, v)
        c.attend(0, n, 1, 2, False)


@pytest.mark.parametrize("G,nq", [(2, 1), (5, 3), (8, 4)])                   # 8 query rows a pass, 16, two teams
def test_attention_over_pages_whose_values_are_far_apart(G, nq):
    """Small values first and large ones behind them, and the other way round, in one warp's rows and in several blocks'."""
    with Both(n_pages=300, n_seqs=2, max_pages=150, G=G) as c:
        k = torch.randn(2, 2, 4000, 64, device="cuda").to(torch.bfloat16)
        size = 2.0 ** torch.linspace(-110, 100, 4000, device="cuda")
        v = torch.randn(2, 2, 4000, 64, device="cuda") * torch.stack([size, size.flip(0)])[:, None, :, None]
        put(c, 0, 2, k, v.to(torch.bfloat16))
        c.attend(0, 2, 1, nq, True)


@pytest.mark.parametrize("size", [1.0, 1e-6, 1e-13, 1e-22])
@pytest.mark.parametrize("n", [1, 80])                                       # slices of blocks, of warps
def test_a_page_of_the_largest_numbers_leaves_other_dims_as_they_are(size, n):
    """Half of the dims of one page are near the largest numbers, the others 0: what the other pages add there keeps its own precision."""
    with Both(n_pages=10 * n, n_seqs=n, max_pages=10) as c:
        v = torch.randn(n, 2, 320, 64, device="cuda") * size
        for i in range(n):
            page = 32 * (i % 10)
            v[i, :, page:page + 32, ::2], v[i, :, page:page + 32, 1::2] = 3e38, 0.0
        v = v.to(torch.bfloat16)
        put(c, 0, n, torch.zeros_like(v), v)
        q, out = torch.zeros(n, 4, 1, 64, dtype=torch.bfloat16, device="cuda"), torch.zeros(n, 4, 1, 64, device="cuda")
        B.dkv_cache8_attend(c.h, 0, n, 1, q, out)
        for i in range(n):
            rows = c.o.rows(i, 1)
            off = np.abs(out[i, ::2, 0].double().cpu().numpy() - rows.mean(1))
            assert (off <= 2.0 ** -18 * np.abs(rows).max(1)).all(), i        # of the dim's own largest value: weights all alike


def test_many_large_values_whose_logits_pass_the_reference():
    """The first rows of every warp have logits of 0, the others of 6.5 (log2): weights of 2^14.5, of which each warp adds up 960 times
    values near the largest."""
    blocks = torch.cuda.get_device_properties(0).multi_processor_count
    with Both(n_pages=200, R=64, n_seqs=blocks, max_pages=200, Hkv=1, G=1) as c:
        rows = 12000
        k = torch.zeros(1, 1, rows, 64, device="cuda")
        k[:, :, 12 * 32:, 0] = 36.0
        v = torch.full((1, 1, rows, 64), 3e38, device="cuda")
        put(c, 0, 1, k.to(torch.bfloat16), v.to(torch.bfloat16))
        for s in range(1, blocks):                                           # a head a block: no slice shares one
            B.dkv_cache8_fork(c.h, 0, s, 1, 1)
        q = torch.zeros(blocks, 1, 1, 64, device="cuda")
        q[..., 0] = 1.0
        out, lse = torch.zeros(blocks, 1, 1, 64, device="cuda"), torch.zeros(blocks, 1, 1, device="cuda")
        B.dkv_cache8_attend(c.h, 0, blocks, 1, q.to(torch.bfloat16), out, lse)
        want, want_lse = c.o.attend(0, q[0].double().cpu().numpy(), False)
        assert np.abs(out.double().cpu().numpy() / want[None] - 1).max() < 2.0 ** -19
        assert np.abs(lse.double().cpu().numpy() - want_lse).max() < 1e-5


def test_many_large_values_with_equal_logits():
    """Weights of 2^8 each: a block adds up 90000 times 2^8 times values near the largest."""
    blocks = torch.cuda.get_device_properties(0).multi_processor_count
    with Both(n_pages=720, R=128, n_seqs=blocks, max_pages=720, Hkv=1, G=1) as c:
        k = torch.zeros(1, 1, 90000, 64, device="cuda").to(torch.bfloat16)
        put(c, 0, 1, k, torch.full_like(k, 3.2e38))
        for s in range(1, blocks):                                           # a head a block: no slice shares one
            B.dkv_cache8_fork(c.h, 0, s, 1, 1)
        out = torch.zeros(blocks, 1, 1, 64, device="cuda")
        B.dkv_cache8_attend(c.h, 0, blocks, 1, torch.zeros(blocks, 1, 1, 64, dtype=torch.bfloat16, device="cuda"), out)
        assert np.abs(out.double().cpu().numpy() / c.o.rows(0, 1).max() - 1).max() < 2.0 ** -19


def test_every_call_wants_the_cache_s_own_device():
    """The device that a cache remembers, behind its configuration, is put to another number than the current one's."""
    with Both(n_seqs=2) as c:
        c.add(0, 2, 1, [10, 20], 1)
        k = torch.zeros(2, 2, 1, 64, dtype=torch.bfloat16, device="cuda")
        q, out = torch.zeros(2, 4, 1, 64, dtype=torch.bfloat16, device="cuda"), torch.zeros(2, 4, 1, 64, device="cuda")
        device = ctypes.c_int32.from_address(c.h + ctypes.sizeof(B.DkvCache8Config))
        assert device.value == torch.cuda.current_device()
        calls = [lambda: B.dkv_cache8_reserve(c.h, 0, 2, 1, None, 1), lambda: B.dkv_cache8_append(c.h, 0, 2, 1, k, k),
                 lambda: B.dkv_cache8_read(c.h, 0, 2, 1, k, k), lambda: B.dkv_cache8_attend(c.h, 0, 2, 1, q, out),
                 lambda: B.dkv_cache8_fork(c.h, 0, 1, 1, 1), lambda: B.dkv_cache8_compact(c.h, 0, 2, 1, torch.zeros(2, 2, 0, dtype=torch.int32, device="cuda")),
                 lambda: B.dkv_cache8_trim(c.h, 0, 2, 1, None, 1)]
        torch.cuda.synchronize()
        device.value += 1
        try:
            for call in calls:
                with pytest.raises(B.DkvError) as e:
                    call()
                assert e.value.code == B.DKV_ERR_INVALID_ARG
            assert B.dkv_cache8_status(c.h)[0] == B.DKV_ERR_INVALID_ARG
        finally:
            device.value -= 1
        assert B.dkv_cache8_status(c.h)[0] == B.DKV_OK
        c.check()


@pytest.mark.parametrize("n,Hkv", [(1, 2), (60, 3)])                        # a slice a block, a slice a warp
def test_the_shortest_limit_of_waits_leaves_nothing_behind(n, Hkv):
    """1000 clock ticks are fewer than a copy takes: warps stop at their first chunk, wait for the copies that they have started, and
    the next call with a usual limit finds the cache, and its scratch, as ever."""
    with Both(n_pages=4000, n_seqs=n, max_pages=4000 // n, Hkv=Hkv, D=128, oracle=False) as c:
        rows = 60000 if n == 1 else 2000
        k, v = (torch.randn(n, Hkv, rows, 128, device="cuda").to(torch.bfloat16) for _ in range(2))
        B.dkv_cache8_reserve(c.h, 0, n, 1, None, rows)
        B.dkv_cache8_append(c.h, 0, n, 1, k, v)
        q = torch.randn(n, Hkv * 2, 4, 128, device="cuda").to(torch.bfloat16)
        good, out = torch.zeros(q.shape, device="cuda"), torch.zeros(q.shape, device="cuda")
        B.dkv_cache8_attend(c.h, 0, n, 1, q, good)
        for _ in range(3):
            B.dkv_cache8_set_wait_limit(c.h, 1000)
            for _ in range(5):
                B.dkv_cache8_attend(c.h, 0, n, 1, q, out)
            code, words = B.dkv_cache8_status(c.h)
            assert code == (B.DKV_ERR_TIMEOUT if words[0] else B.DKV_OK) and words[0] in (0, B.DKV_C8_TIMEOUT)
            B.dkv_cache8_set_wait_limit(c.h, 4_000_000_000)
            B.dkv_cache8_attend(c.h, 0, n, 1, q, out)
            assert torch.equal(out, good) and B.dkv_cache8_status(c.h)[0] == B.DKV_OK
