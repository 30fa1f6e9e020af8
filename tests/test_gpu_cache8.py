"""The cache in 8 bits against the oracle: rows in and out bit by bit, attention, pages, and a prompt's way from its compressed
buffers through decoding steps.  Codes are compared as the values they stand for: every one is a 16-bit number."""
import numpy as np
import pytest
import torch

from oracle import cache8 as C
from paper_2412_14838_b200 import binding as B
from paper_2412_14838_b200 import build, synth

pytestmark = pytest.mark.gpu
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16}


@pytest.fixture(scope="module", autouse=True)
def _lib():
    build.build()
    B.load()


class View:
    def __init__(self, address, shape):
        self.__cuda_array_interface__ = {"data": (address, False), "shape": shape, "typestr": "<i4", "version": 3}


class Both:
    """A cache of the library beside the oracle's."""

    def __init__(self, n_pages=40, R=32, n_seqs=4, max_pages=12, Hkv=2, D=64, kind="e4m3", io="bf16", G=2, oracle=True):
        self.Hkv, self.D, self.G, self.io, self.n_seqs, self.n_pages, self.max_pages, self.R = Hkv, D, G, TYPES[io], n_seqs, n_pages, max_pages, R
        self.kind = kind
        self.h = B.dkv_cache8_create(B.make_cache8_config(n_pages, R, n_seqs, max_pages, Hkv * G, Hkv, D,
                                                          B.DKV_E4M3 if kind == "e4m3" else B.DKV_INT8, B.DKV_BF16 if io == "bf16" else B.DKV_F16))
        self.o = C.Cache(n_pages, R, n_seqs, max_pages, Hkv, D, kind) if oracle else None

    def __enter__(self):
        return self

    def __exit__(self, *_):
        B.dkv_cache8_destroy(self.h)

    def views(self):
        at = B.dkv_cache8_views(self.h)
        shapes = dict(len=(self.n_seqs,), held=(self.n_seqs,), table=(self.n_seqs, self.max_pages), refs=(self.n_pages,))
        return {n: torch.as_tensor(View(at[n], shapes[n]), device="cuda").cpu().numpy().copy() for n in at}

    def add(self, first, n, step, rows, seed=0, scale=1.0, cap=None, reserve=True):
        """rows[i] normal rows for every sequence, on both sides."""
        g = torch.Generator(device="cuda").manual_seed(seed)
        cap = max(rows) if cap is None else cap
        k, v = (scale * torch.randn(n, self.Hkv, cap, self.D, generator=g, device="cuda") for _ in range(2))
        k, v = k.to(self.io), v.to(self.io)
        counts = torch.tensor(rows, dtype=torch.int32, device="cuda")
        if reserve:
            B.dkv_cache8_reserve(self.h, first, n, step, counts)
            self.o.reserve([first + i * step for i in range(n)], rows)
        B.dkv_cache8_append(self.h, first, n, step, k, v, counts)
        for i in range(n):
            self.o.append(first + i * step, k[i, :, :rows[i]].double().cpu().numpy(), v[i, :, :rows[i]].double().cpu().numpy())
        return k, v

    def read(self, first, n, step, cap):
        out = [torch.full((n, self.Hkv, cap, self.D), 77.0, dtype=self.io, device="cuda") for _ in range(2)]
        B.dkv_cache8_read(self.h, first, n, step, *out)
        return [o.double().cpu().numpy() for o in out]

    def check(self):
        """Rows, lengths, tables and holders are the oracle's."""
        got = self.views()
        assert got["len"].tolist() == self.o.len and got["refs"].tolist() == self.o.refs()
        assert got["held"].tolist() == [len(t) for t in self.o.table]
        for s, t in enumerate(self.o.table):
            assert got["table"][s, :len(t)].tolist() == t
        cap = max(1, max(self.o.len))
        big = float(torch.finfo(self.io).max)
        for w, rows in enumerate(self.read(0, self.n_seqs, 1, cap)):
            for s in range(self.n_seqs):
                n = self.o.len[s]
                assert (rows[s, :, :n] == np.clip(self.o.rows(s, w), -big, big)).all(), f"sequence {s}, tensor {w}"
                assert (rows[s, :, n:] == 77.0).all()

    def attend(self, first, n, step, nq, causal, seed=1, scale=1.0, q=None):
        """Against the oracle.  Logits: fp32 sums of D exact products, each rounding 2^-24 of the running sum (at most
        sum |q k|), so the error stays below 2^-24 D sum |q k| / sqrt(D), and the weights' relative error is that of twice the largest
        logit's plus 2^-21 for ex2, the split into fp16 parts and their sums: weights, and with them the result relative to the
        largest value, are off by at most twice that."""
        g = torch.Generator(device="cuda").manual_seed(seed)
        if q is None:
            q = (scale * torch.randn(n, self.Hkv * self.G, nq, self.D, generator=g, device="cuda")).to(self.io)
        out = torch.full(q.shape, 55.0, device="cuda")
        lse = torch.full(q.shape[:3], 55.0, device="cuda")
        B.dkv_cache8_attend(self.h, first, n, step, q, out, lse, causal)
        for i in range(n):
            s = first + i * step
            want, want_lse = self.o.attend(s, q[i].double().cpu().numpy(), causal)
            k, v = self.o.rows(s, 0), self.o.rows(s, 1)
            for hq in range(q.shape[1]):
                size = np.abs(k[hq // self.G]) @ np.abs(q[i, hq].double().cpu().numpy()).T if self.o.len[s] else np.zeros((1, nq))
                z = 2.0 ** -24 * self.D ** 0.5 * size.max(0)
                bound = 4 * (z + 2.0 ** -21) * np.abs(v[hq // self.G]).max(initial=0.0)
                assert (np.abs(out[i, hq].double().cpu().numpy() - want[hq]) <= bound[:, None]).all(), (i, hq)
                a, b = lse[i, hq].double().cpu().numpy(), want_lse[hq]
                assert (np.isneginf(a) == np.isneginf(b)).all()
                there = ~np.isneginf(b)
                assert (np.abs(a[there] - b[there]) <= (z + 2.0 ** -20 + 2.0 ** -22 * np.abs(b))[there]).all()
        return out, lse


KINDS = [("e4m3", "bf16"), ("int8", "f16"), ("e4m3", "f16"), ("int8", "bf16")]


@pytest.mark.parametrize("kind,io", KINDS)
@pytest.mark.parametrize("D,R", [(64, 32), (128, 32), (64, 64), (128, 64), (64, 128), (128, 128)])
def test_rows_come_back_as_the_oracle_rounds_them(kind, io, D, R):
    with Both(R=R, D=D, kind=kind, io=io, n_pages=64, max_pages=16) as c:
        c.add(0, 4, 1, [0, 1, R, 3 * R + 5], 1)
        c.check()
        c.add(0, 4, 1, [R - 1, R - 1, 1, 2], 2, 3.0)                         # page ends inside, at and after the rows; scales grow
        c.check()
        c.add(1, 2, 2, [1, 1], 3, 40.0)
        c.check()
        c.add(0, 4, 1, [1, 0, 70, 2 * R], 4, 0.01)                           # scales stay
        c.check()
        assert B.dkv_cache8_status(c.h)[0] == B.DKV_OK


@pytest.mark.parametrize("kind,io", KINDS)
def test_one_token_after_the_other(kind, io):
    with Both(kind=kind, io=io, D=128) as c:
        for i in range(70):
            c.add(0, 2, 2, [1, 1], 100 + i, 1.0 + (i % 13 == 5) * i)
        c.check()
        c.attend(0, 2, 2, 1, False)


@pytest.mark.parametrize("kind", ["e4m3", "int8"])
def test_numbers_at_the_ends_of_their_types(kind):
    big, tiny = torch.finfo(torch.bfloat16).max, 2.0 ** -133
    rows = [[0.0, -0.0, 1.0, 1.0], [big, -big, 1.0, 2.0 ** -120], [tiny, -tiny, 3 * tiny, 2.0 ** -126], [448.0, 449.0, 17.0, 19.0],
            [127.0, 127.5, 0.5, -2.5], [float("inf"), 2.0, -1.0, 1.0], [float("nan"), 2.0, -1.0, 1.0], [float("-inf"), float("nan"), 0.0, 0.0]]
    for j, row in enumerate(rows):
        with Both(kind=kind, n_seqs=1, Hkv=1) as c:
            x = torch.tensor(row, device="cuda").to(torch.bfloat16).repeat(16).view(1, 1, 1, 64)
            B.dkv_cache8_reserve(c.h, 0, 1, 1, None, 3)
            c.o.reserve([0], [3])
            for y in (x, torch.ones_like(x), x):
                B.dkv_cache8_append(c.h, 0, 1, 1, y, y)
                c.o.append(0, y[0].double().cpu().numpy(), y[0].double().cpu().numpy())
            c.check()
            code, words = B.dkv_cache8_status(c.h)
            assert code == B.DKV_OK and words[0] == (B.DKV_C8_NOT_FINITE if j >= 5 else 0) and words[1] == (0 if j >= 5 else -1)


def test_rows_in_other_orders_and_parts_of_larger_tensors():
    with Both(n_pages=30) as c:
        T = 50
        big = torch.randn(4, T + 3, 3, 2, 128, device="cuda").to(torch.bfloat16)      # [n, tokens, what, heads, 2 D]
        k, v = big[:, 1:T + 1, 0, :, :64].transpose(1, 2), big[:, 1:T + 1, 2, :, 64:].transpose(1, 2)
        counts = torch.tensor([50, 0, 33, 7], dtype=torch.int32, device="cuda")
        B.dkv_cache8_reserve(c.h, 0, 4, 1, counts)
        B.dkv_cache8_append(c.h, 0, 4, 1, k.view(torch.int16), v, counts)             # 16-bit patterns are as good
        c.o.reserve(range(4), counts.tolist())
        for s in range(4):
            c.o.append(s, *(x[s, :, :counts[s]].double().cpu().numpy() for x in (k, v)))
        c.check()
        out = torch.full_like(big, 9.0)
        B.dkv_cache8_read(c.h, 0, 4, 1, out[:, 1:T + 1, 0, :, :64].transpose(1, 2), out[:, 1:T + 1, 2, :, 64:].transpose(1, 2))
        for s in range(4):
            got = out[s, 1:T + 1, 0, :, :64].transpose(0, 1)[:, :counts[s]].double().cpu().numpy()
            assert (got == c.o.rows(s, 0)).all()
            out[s, 1:1 + counts[s], 0, :, :64] = out[s, 1:1 + counts[s], 2, :, 64:] = 9.0
        assert (out == 9.0).all()                                            # nothing beside the rows was written
        short = c.read(0, 4, 1, 20)                                          # fewer rows than there are
        assert (short[0][0] == c.o.rows(0, 0)[:, :20]).all()


@pytest.mark.parametrize("layout,rot,D", [("half", 64, 64), ("pairs", 64, 64), ("half", 32, 128), ("pairs", 10, 64), ("half", 10, 64), ("half", 128, 128)])
@pytest.mark.parametrize("kind", ["e4m3", "int8"])
def test_keys_turned_on_the_way_in(layout, rot, D, kind):
    """A stored value is half a code step from what it rounds; that, in 32 bits, is off the exact turn by what test_gpu_rotate.py
    derives, 8e-7 of |a| + |b| <= 2 max|x|."""
    freq, amp = C.frequencies(rot, 10000.0, "ramp", 4.0, 1.0, 32.0, 8192.0)
    r = B.dkv_rotary_init(D, rot, B.DKV_ROTARY_HALF if layout == "half" else B.DKV_ROTARY_PAIRS, 10000.0, B.DKV_SCALING_RAMP, 4.0, 1.0, 32.0, 8192.0)
    with Both(n_seqs=2, D=D, kind=kind) as c:
        n, T = 2, 45
        k, v = (torch.randn(n, 2, T, D, device="cuda").to(torch.bfloat16) for _ in range(2))
        pos0 = torch.tensor([0, 123456], dtype=torch.int32, device="cuda")
        counts = torch.tensor([45, 40], dtype=torch.int32, device="cuda")
        B.dkv_cache8_reserve(c.h, 0, n, 1, counts)
        B.dkv_cache8_append(c.h, 0, n, 1, k, v, counts, r, pos0)
        c.o.reserve([0, 1], counts.tolist())
        got = c.read(0, n, 1, T)
        for s in range(n):
            m = int(counts[s])
            x = k[s, :, :m].double().cpu().numpy()
            want = C.rotate(x, int(pos0[s]) + np.arange(m), freq, amp, layout)
            c.o.append(s, want, v[s, :, :m].double().cpu().numpy())
            off = np.abs(got[0][s, :, :m] - want)
            step = C.step_at(want, c.o.scales(s, 0)[..., None] + 0 * want, kind)
            assert (off <= step / 2 + 2 * np.abs(x).max() * amp * 8e-7).all()
            assert (got[1][s, :, :m] == c.o.rows(s, 1)).all()


@pytest.mark.parametrize("layout,rot", [("half", 64), ("pairs", 32), ("half", 10), ("pairs", 6)])
@pytest.mark.parametrize("T", [1, 5, 8, 9])                                  # a block a sequence up to eight rows, then a block a page
def test_turned_keys_behind_others_and_numbers_that_are_not_finite(layout, rot, T):
    """As above, behind 30 rows (pages end inside the new ones), with an infinity and a NaN in one new row: what they turn into is NaN
    or infinite in 64 bits too, and stored as 0 or the largest code."""
    D = 64
    freq, amp = C.frequencies(rot, 10000.0)
    r = B.dkv_rotary_init(D, rot, B.DKV_ROTARY_HALF if layout == "half" else B.DKV_ROTARY_PAIRS, 10000.0)
    with Both(n_seqs=2, D=D, n_pages=20) as c:
        c.add(0, 2, 1, [30, 3], 5)
        k, v = (torch.randn(2, 2, T, D, device="cuda").to(torch.bfloat16) for _ in range(2))
        k[0, 1, T - 1, 1] = float("nan")
        k[0, 0, 0, 2] = float("inf")
        v[1, 0, 0, 3] = float("-inf")
        v[1, 1, T - 1, 63] = float("nan")
        pos0 = torch.tensor([77, 0], dtype=torch.int32, device="cuda")
        B.dkv_cache8_reserve(c.h, 0, 2, 1, None, T)
        B.dkv_cache8_append(c.h, 0, 2, 1, k, v, None, r, pos0)
        c.o.reserve([0, 1], [T, T])
        wants = []
        for s in range(2):
            x = k[s].double().cpu().numpy()
            with np.errstate(invalid="ignore"):
                wants.append(C.rotate(x, int(pos0[s]) + np.arange(T), freq, amp, layout))
            c.o.append(s, wants[s], v[s].double().cpu().numpy())
        got = c.read(0, 2, 1, 30 + T)
        for s, before in enumerate((30, 3)):
            assert (got[1][s, :, :before + T] == c.o.rows(s, 1)).all()
            new, fine = got[0][s, :, before:before + T], np.isfinite(wants[s])
            scale = c.o.scales(s, 0)[:, before:, None] + 0 * new
            step = C.step_at(np.where(fine, wants[s], 0), scale, "e4m3")
            assert (np.abs(new - wants[s])[fine] <= (step / 2 + 2 * 5 * amp * 8e-7)[fine]).all()
            assert (new[~fine] == c.o.rows(s, 0)[:, before:][~fine]).all()
            assert (got[0][s, :, :before] == c.o.rows(s, 0)[:, :before]).all()
        assert B.dkv_cache8_status(c.h)[1][:2] == [B.DKV_C8_NOT_FINITE, 0]


@pytest.mark.parametrize("kind", ["e4m3", "int8"])
def test_many_rows_with_numbers_that_are_not_finite(kind):
    with Both(n_seqs=2, n_pages=20, kind=kind, D=128) as c:
        c.add(0, 2, 1, [5, 0], 5)
        x = torch.randn(2, 2, 70, 128, device="cuda").to(torch.bfloat16)
        x[0, 0, 3, 7], x[0, 1, 40, 100], x[1, 0, 69, 127], x[1, 1, :, :] = float("nan"), float("-inf"), float("inf"), float("nan")
        B.dkv_cache8_reserve(c.h, 0, 2, 1, None, 70)
        B.dkv_cache8_append(c.h, 0, 2, 1, x, x.flip(2))
        c.o.reserve([0, 1], [70, 70])
        for s in range(2):
            c.o.append(s, x[s].double().cpu().numpy(), x[s].flip(1).double().cpu().numpy())
        c.check()
        c.attend(0, 2, 1, 1, False)
        assert B.dkv_cache8_status(c.h)[1][0] == B.DKV_C8_NOT_FINITE


def test_two_caches_on_two_streams():
    with Both(n_pages=60, n_seqs=4, D=128, G=4) as a, Both(n_pages=60, n_seqs=4, D=64, kind="int8", G=2) as b:
        torch.cuda.synchronize()
        streams = [torch.cuda.Stream() for _ in range(2)]
        for turn in range(20):
            for c, s in zip((a, b), streams):
                with torch.cuda.stream(s):
                    c.add(0, 4, 1, [turn % 7, 1, 13, 0], turn)
        torch.cuda.synchronize()
        for c in (a, b):
            c.check()
            c.attend(0, 4, 1, 2, True)


def test_forks_between_one_another_s_sequences():
    with Both(n_pages=30, n_seqs=6) as c:
        c.add(0, 3, 2, [40, 33, 64], 1)                                      # sequences 0, 2, 4
        c.add(1, 3, 2, [70, 1, 0], 2)
        B.dkv_cache8_fork(c.h, 0, 1, 3, 2)                                   # onto 1, 3, 5, whose own pages go back
        c.o.fork([(0, 1), (2, 3), (4, 5)])
        c.check()
        B.dkv_cache8_fork(c.h, 1, 0, 3, 2)                                   # and back: every page is held by both
        c.o.fork([(1, 0), (3, 2), (5, 4)])
        c.check()
        c.add(0, 6, 1, [1, 2, 3, 4, 5, 6], 3, 7.0)
        c.check()


@pytest.mark.parametrize("kind,io", KINDS)
@pytest.mark.parametrize("G,nq,causal", [(1, 1, False), (4, 1, True), (2, 4, True), (3, 3, False), (4, 4, True), (7, 5, True), (8, 8, True), (17, 1, False)])
@pytest.mark.parametrize("D", [64, 128])
def test_attention_matches_the_oracle(kind, io, G, nq, causal, D):
    with Both(n_pages=120, n_seqs=7, max_pages=40, D=D, kind=kind, io=io, G=G, Hkv=3 if G < 8 else 1) as c:
        c.add(0, 7, 1, [0, 1, 31, 32, 33, 300, 1201], G)
        c.attend(0, 7, 1, nq, causal)
        c.attend(1, 3, 2, nq, causal, 5, 4.0)


@pytest.mark.parametrize("R", [64, 128])
@pytest.mark.parametrize("kind", ["e4m3", "int8"])
def test_attention_over_larger_pages(R, kind):
    with Both(n_pages=60, R=R, n_seqs=3, max_pages=30, kind=kind, D=128) as c:
        c.add(0, 3, 1, [R + 1, 1500, R - 32], 8)
        c.attend(0, 3, 1, 2, True)


@pytest.mark.parametrize("kind,io", KINDS)
@pytest.mark.parametrize("G,nq", [(4, 1), (5, 3), (6, 3)])                  # one pass of 8, one of 16, two: another division of the work
@pytest.mark.parametrize("D", [64, 128])
def test_attention_of_many_heads(kind, io, G, nq, D):
    lens = [0, 1, 32, 33, 500] + [(i * 97) % 400 for i in range(55)]
    with Both(n_pages=600, n_seqs=60, max_pages=20, D=D, kind=kind, io=io, G=G, Hkv=3) as c:
        c.add(0, 60, 1, lens, G)
        c.attend(0, 60, 1, nq, True)
        c.attend(0, 40, 1, nq, True)                                         # fewer heads than blocks


def test_a_long_sequence_lies_in_every_block():
    with Both(n_pages=700, n_seqs=1, max_pages=700, D=64, Hkv=1, G=4, R=128) as c:
        c.add(0, 1, 1, [65000], 1)                                           # 170 groups of twelve chunks: a slice of one or two each
        c.attend(0, 1, 1, 1, False)
        c.attend(0, 1, 1, 16, True)


@pytest.mark.parametrize("size", [3e38, 1e-25])
def test_values_at_the_ends_of_bf16(size):
    with Both(n_pages=30, n_seqs=1, max_pages=30) as c:
        k = torch.randn(1, 2, 300, 64, device="cuda").to(torch.bfloat16)
        v = (torch.rand(1, 2, 300, 64, device="cuda") * size).to(torch.bfloat16)
        B.dkv_cache8_reserve(c.h, 0, 1, 1, None, 300)
        B.dkv_cache8_append(c.h, 0, 1, 1, k, v)
        c.o.reserve([0], [300])
        c.o.append(0, k[0].double().cpu().numpy(), v[0].double().cpu().numpy())
        c.attend(0, 1, 1, 2, False)


@pytest.mark.parametrize("n,Hkv", [(1, 2), (60, 3)])                        # a slice a block, a slice a warp
@pytest.mark.parametrize("chunk", [0, 1])
def test_a_wait_that_runs_out_is_reported_and_leaves_the_cache_usable(n, Hkv, chunk):
    with Both(n_pages=4000, n_seqs=n, max_pages=900 // n * 4 + 20, Hkv=Hkv) as c:
        rows = 60000 if n == 1 else 2000                                     # so many that the first warp has two chunks
        c.add(0, n, 1, [rows] * n, 1)
        q = torch.randn(n, Hkv * 2, 1, 64, device="cuda").to(torch.bfloat16)
        out = torch.zeros(n, Hkv * 2, 1, 64, device="cuda")
        B.dkv_cache8_attend(c.h, 0, n, 1, q, out)
        good = out.clone()
        B.dkv_cache8_set_wait_limit(c.h, 2_000_000)                          # about a millisecond
        B.dkv_cache8_debug_withhold(c.h, chunk)
        B.dkv_cache8_attend(c.h, 0, n, 1, q, out)
        code, words = B.dkv_cache8_status(c.h)
        assert code == B.DKV_ERR_TIMEOUT and words[0] == B.DKV_C8_TIMEOUT and words[1] == 0
        B.dkv_cache8_debug_withhold(c.h, -1)
        B.dkv_cache8_attend(c.h, 0, n, 1, q, out)
        assert torch.equal(out, good) and B.dkv_cache8_status(c.h)[0] == B.DKV_OK
        with pytest.raises(B.DkvError):
            B.dkv_cache8_set_wait_limit(c.h, 10)


def test_values_of_very_different_sizes_and_large_logits():
    with Both(n_pages=60, n_seqs=2, max_pages=30, D=128) as c:
        for i, scale in enumerate([1e-3, 1.0, 1e4, 1e-6, 30.0]):             # pages whose scales differ by 2^33
            c.add(0, 2, 1, [64, 32], i, scale)
        c.attend(0, 2, 1, 2, False, 1, 1e-3)
        c.attend(0, 2, 1, 2, True, 2, 1.0)                                   # logits of some 1e4: one row takes all
        c.attend(0, 2, 1, 1, False, 3, 0.0)                                  # all weights alike


def test_rows_that_no_query_sees_have_no_part():
    with Both(n_seqs=2, n_pages=20) as c:
        c.add(0, 2, 1, [40, 1], 1)
        bad = torch.full((2, 2, 1, 64), float("nan"), dtype=torch.bfloat16, device="cuda")
        bad[:, :, :, ::2] = float("inf")
        huge = torch.full((2, 2, 1, 64), 3e38, dtype=torch.bfloat16, device="cuda")
        want = c.attend(0, 2, 1, 1, False)[0]
        for x in (bad, huge):
            B.dkv_cache8_reserve(c.h, 0, 2, 1, None, 2)
            B.dkv_cache8_append(c.h, 0, 2, 1, x, bad)
            B.dkv_cache8_append(c.h, 0, 2, 1, bad, x)
            B.dkv_cache8_trim(c.h, 0, 2, 1, None, 2)
        q = torch.randn(2, 4, 3, 64, device="cuda").to(torch.bfloat16)
        q[0, 1, 1] = float("nan")
        q[1, 2, 0, 5] = float("inf")
        out = torch.zeros(q.shape, device="cuda")
        lse = torch.zeros(q.shape[:3], device="cuda")
        B.dkv_cache8_attend(c.h, 0, 2, 1, q, out, lse, True)
        odd = torch.zeros(2, 4, 3, dtype=torch.bool, device="cuda")
        odd[0, 1, 1] = True                                                  # the other bad query sees no row: limits -1, 0, 1
        assert torch.isnan(out[odd]).all() and torch.isnan(lse[odd]).all() and torch.isfinite(out[~odd]).all()
        assert (out[1, :, :2] == 0).all() and torch.isneginf(lse[1, :, :2]).all() and want.isfinite().all()


def test_results_do_not_change_from_call_to_call_and_strides_do_not_matter():
    with Both(n_pages=200, n_seqs=3, max_pages=100, G=4, D=128, oracle=False) as c:
        rows = torch.tensor([3000, 17, 900], dtype=torch.int32, device="cuda")
        k, v = (torch.randn(3, 2, 3000, 128, device="cuda").to(torch.bfloat16) for _ in range(2))
        B.dkv_cache8_reserve(c.h, 0, 3, 1, rows)
        B.dkv_cache8_append(c.h, 0, 3, 1, k, v, rows)
        q = torch.randn(3, 2, 8, 128, device="cuda").to(torch.bfloat16).transpose(1, 2)       # [n, heads, tokens, D] of token-major rows
        a, b = torch.zeros(3, 8, 2, 128, device="cuda"), torch.zeros(3, 2, 8, 128, device="cuda").transpose(1, 2)
        B.dkv_cache8_attend(c.h, 0, 3, 1, q, a, None, True)
        for _ in range(20):
            B.dkv_cache8_attend(c.h, 0, 3, 1, q, b, None, True)
        assert torch.equal(a, b)
        B.dkv_cache8_attend(c.h, 0, 3, 1, q.contiguous(), b, None, True)
        assert torch.equal(a, b)
        one = torch.zeros(1, 8, 2, 128, device="cuda")
        B.dkv_cache8_attend(c.h, 1, 1, 1, q[1:2], one, None, True)           # another cut of the work
        assert torch.allclose(one, a[1:2], rtol=1e-5, atol=1e-6)


def test_more_sequences_than_a_launch_takes():
    n = 2100
    with Both(n_pages=n + 10, n_seqs=n, max_pages=2, Hkv=1, G=1) as c:
        rows = [i % 3 for i in range(n)]
        c.add(0, n, 1, rows, 3, cap=2)
        c.check()
        c.attend(0, n, 1, 1, False)


@pytest.mark.parametrize("n_pages,max_pages,bits_seen", [(37, 9, 0), (11, 4, 7)])       # pages for everything; too few
def test_page_operations_follow_the_oracle(n_pages, max_pages, bits_seen):
    rng = np.random.default_rng(7)
    for kind in ("e4m3", "int8"):
        with Both(n_pages=n_pages, n_seqs=6, max_pages=max_pages, kind=kind) as c:
            bits = 0
            for turn in range(60):
                first, step = int(rng.integers(0, 3)), int(rng.integers(1, 3))
                n = int(rng.integers(1, (5 - first) // step + 2))
                seqs = [first + i * step for i in range(n)]
                what = rng.choice(["add", "add", "fork", "trim", "compact"])
                if what == "add":
                    rows = [int(x) for x in rng.integers(0, 60, n)]
                    none, full = c.o.reserve(seqs, rows)
                    B.dkv_cache8_reserve(c.h, first, n, step, torch.tensor(rows, dtype=torch.int32, device="cuda"))
                    bits |= (1 if none else 0) | (2 if full else 0)
                    room = [c.o.len[s] + r <= len(c.o.table[s]) * c.R and not (r and c.o.len[s] % c.R and
                            c.o.refs()[c.o.table[s][c.o.len[s] // c.R]] != 1) for s, r in zip(seqs, rows)]
                    bits |= 0 if all(room) else 4
                    c.add(first, n, step, rows, turn, float(rng.choice([0.1, 1.0, 20.0])), reserve=False, cap=max(1, max(rows)))
                elif what == "fork":
                    src, dst = (0, 3) if rng.random() < 0.5 else (3, 0)
                    B.dkv_cache8_fork(c.h, src, dst, 3, 1)
                    c.o.fork([(src + i, dst + i) for i in range(3)])
                elif what == "trim":
                    keep = [int(x) for x in rng.integers(0, 200, n)]
                    B.dkv_cache8_trim(c.h, first, n, step, torch.tensor(keep, dtype=torch.int32, device="cuda"))
                    for s, x in zip(seqs, keep):
                        c.o.trim(s, x)
                else:
                    counts = [int(rng.integers(0, 50)) if c.o.len[s] else 0 for s in seqs]
                    idx = [rng.integers(0, max(1, c.o.len[s]), (2, 50)) for s in seqs]
                    B.dkv_cache8_compact(c.h, first, n, step, torch.tensor(np.stack(idx), dtype=torch.int32, device="cuda"),
                                         torch.tensor(counts, dtype=torch.int32, device="cuda"))
                    bits |= 1 if c.o.compact(seqs, [x[:, :m].tolist() for x, m in zip(idx, counts)]) else 0
                c.check()
            code, words = B.dkv_cache8_status(c.h)
            assert words[0] == bits == bits_seen and words[2] == sum(r == 0 for r in c.o.refs())
            assert code == (B.DKV_ERR_NOMEM if bits else B.DKV_OK) and B.dkv_cache8_status(c.h)[1][:2] == [0, -1]
            c.attend(0, 6, 1, 2, True)


def test_a_fork_and_its_source_part_where_either_is_written():
    with Both(n_pages=20, n_seqs=3, Hkv=2) as c:
        c.add(0, 1, 1, [45], 1)
        B.dkv_cache8_fork(c.h, 0, 1, 1, 1)
        B.dkv_cache8_fork(c.h, 0, 2, 1, 1)
        c.o.fork([(0, 1)])
        c.o.fork([(0, 2)])
        c.check()
        k = torch.ones(1, 2, 1, 64, dtype=torch.bfloat16, device="cuda")
        B.dkv_cache8_append(c.h, 1, 1, 1, k, k)                              # no room of its own yet
        c.check()
        code, words = B.dkv_cache8_status(c.h)
        assert (code, words[0], words[1]) == (B.DKV_ERR_STATE, B.DKV_C8_NO_ROOM, 1)
        c.add(0, 3, 1, [1, 30, 2], 2, 5.0)                                   # all three take a copy in one call
        c.check()
        assert c.views()["refs"].max() == 3
        c.attend(0, 3, 1, 1, False)


def test_a_sequence_cut_into_a_shared_page_does_not_write_there():
    with Both(n_pages=20, n_seqs=2) as c:
        c.add(0, 1, 1, [64], 1)
        B.dkv_cache8_fork(c.h, 0, 1, 1, 1)
        c.o.fork([(0, 1)])
        B.dkv_cache8_trim(c.h, 0, 1, 1, None, 10)
        c.o.trim(0, 54)
        c.add(0, 1, 1, [3], 2, 9.0)
        c.check()
        assert c.views()["refs"][:3].tolist() == [2, 1, 1]


@pytest.mark.parametrize("kind", ["e4m3", "int8"])
def test_compaction_by_head(kind):
    rng = np.random.default_rng(3)
    with Both(n_pages=60, n_seqs=3, max_pages=20, D=128, kind=kind) as c:
        c.add(0, 3, 1, [500, 33, 1], 1)
        c.add(0, 1, 1, [5], 2, 100.0)
        counts = [100, 33, 1]
        idx = [np.stack([rng.permutation(c.o.len[s])[:m] for _ in range(2)]) for s, m in enumerate(counts)]
        padded = np.full((3, 2, 128), -5)
        for s in range(3):
            padded[s, :, :counts[s]] = idx[s]
        B.dkv_cache8_compact(c.h, 0, 3, 1, torch.tensor(padded, dtype=torch.int32, device="cuda"),
                             torch.tensor(counts, dtype=torch.int32, device="cuda"))
        assert c.o.compact([0, 1, 2], [x.tolist() for x in idx]) == []
        c.check()
        assert B.dkv_cache8_status(c.h)[0] == B.DKV_OK
        # a row number outside: reported, a row of zeros
        B.dkv_cache8_compact(c.h, 1, 1, 1, torch.tensor([[[0, 33], [-1, 2]]], dtype=torch.int32, device="cuda"))
        code, words = B.dkv_cache8_status(c.h)
        assert (code, words[0], words[1]) == (B.DKV_ERR_INVALID_ARG, B.DKV_C8_BAD_ARGUMENT, 1)
        got = c.read(1, 1, 1, 2)
        assert (got[0][0, 0, 1] == 0).all() and (got[0][0, 1, 0] == 0).all() and (got[0][0, 0, 0] != 0).any()


def test_counts_out_of_range_change_nothing():
    with Both(n_seqs=2) as c:
        c.add(0, 2, 1, [10, 20], 1)
        x = torch.ones(2, 2, 4, 64, dtype=torch.bfloat16, device="cuda")
        for counts in ([-1, -2**31], [5, 2**31 - 1]):
            counts = torch.tensor(counts, dtype=torch.int32, device="cuda")
            B.dkv_cache8_append(c.h, 0, 2, 1, x, x, counts)
            assert B.dkv_cache8_status(c.h)[1][:2] == [B.DKV_C8_BAD_ARGUMENT, 0]
            B.dkv_cache8_compact(c.h, 0, 2, 1, torch.zeros((2, 2, 4), dtype=torch.int32, device="cuda"), counts)
            assert B.dkv_cache8_status(c.h)[1][0] == B.DKV_C8_BAD_ARGUMENT
            c.check()
        B.dkv_cache8_reserve(c.h, 0, 2, 1, torch.tensor([-3, 2**31 - 1], dtype=torch.int32, device="cuda"))
        code, words = B.dkv_cache8_status(c.h)
        assert code == B.DKV_ERR_NOMEM and words[:2] == [B.DKV_C8_BAD_ARGUMENT | B.DKV_C8_TABLE_FULL, 0]
        c.check()
        B.dkv_cache8_trim(c.h, 0, 1, 1, torch.tensor([-4], dtype=torch.int32, device="cuda"))
        assert B.dkv_cache8_status(c.h)[1][0] == B.DKV_C8_BAD_ARGUMENT and c.views()["len"].tolist() == [0, 20]


def test_pages_behind_the_first_four_gigabytes():
    Hkv, D, R, n_pages = 8, 128, 32, 70000                                   # pages of 64 KB
    with Both(n_pages=n_pages, R=R, n_seqs=2, max_pages=n_pages, Hkv=Hkv, D=D, G=1, oracle=False) as c:
        B.dkv_cache8_reserve(c.h, 0, 1, 1, None, (n_pages - 3) * R)          # takes all but the last three pages
        k, v = (torch.randn(1, Hkv, 80, D, device="cuda").to(torch.bfloat16) for _ in range(2))
        B.dkv_cache8_reserve(c.h, 1, 1, 1, None, 80)
        B.dkv_cache8_append(c.h, 1, 1, 1, k, v)
        at = B.dkv_cache8_views(c.h)
        assert torch.as_tensor(View(at["table"], (2, n_pages)), device="cuda")[1, :3].tolist() == [n_pages - 3, n_pages - 2, n_pages - 1]
        o = C.Cache(3, R, 1, 3, Hkv, D, "e4m3")
        o.reserve([0], [80])
        o.append(0, k[0].double().cpu().numpy(), v[0].double().cpu().numpy())
        got = c.read(1, 1, 1, 80)
        assert (got[0][0] == o.rows(0, 0)).all() and (got[1][0] == o.rows(0, 1)).all()
        q, out = torch.randn(1, Hkv, 1, D, device="cuda").to(torch.bfloat16), torch.zeros(1, Hkv, 1, D, device="cuda")
        B.dkv_cache8_attend(c.h, 1, 1, 1, q, out)
        want = o.attend(0, q[0].double().cpu().numpy(), False)[0]
        assert np.abs(out[0].cpu().numpy() - want).max() < 1e-4
        assert B.dkv_cache8_status(c.h)[1][:3] == [0, -1, 0]
        B.dkv_cache8_trim(c.h, 0, 1, 1, None, 2**31 - 1)
        assert B.dkv_cache8_status(c.h)[1][2] == n_pages - 3


def test_a_step_as_a_graph_on_another_stream():
    with Both(n_pages=40, n_seqs=4, D=128, G=4) as c:
        c.add(0, 4, 1, [50, 3, 0, 31], 1)
        k, v = (torch.zeros(4, 2, 1, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        q, out = torch.zeros(4, 8, 1, 128, dtype=torch.bfloat16, device="cuda"), torch.zeros(4, 8, 1, 128, device="cuda")
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            B.dkv_cache8_reserve(c.h, 0, 4, 1, None, 1)
            B.dkv_cache8_append(c.h, 0, 4, 1, k, v)
            B.dkv_cache8_attend(c.h, 0, 4, 1, q, out, causal=True)
        c.check()                                                            # nothing ran yet
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            for i in range(40):
                if i == 20:                                                  # forks made after the capture are parted too
                    B.dkv_cache8_fork(c.h, 0, 2, 2, 1)
                    c.o.fork([(0, 2), (1, 3)])
                for x in (k, v, q):
                    x.copy_(torch.randn(x.shape, device="cuda"))
                graph.replay()
                c.o.reserve(range(4), [1] * 4)
                for s in range(4):
                    c.o.append(s, k[s].double().cpu().numpy(), v[s].double().cpu().numpy())
        torch.cuda.current_stream().wait_stream(side)
        c.check()
        for s in range(4):
            want = c.o.attend(s, q[s].double().cpu().numpy(), True)[0]
            assert np.abs(out[s].double().cpu().numpy() - want).max() < 1e-4


def test_calls_are_checked():
    with Both() as c:
        k = torch.zeros(2, 2, 4, 64, dtype=torch.bfloat16, device="cuda")
        q, out = torch.zeros(2, 4, 1, 64, dtype=torch.bfloat16, device="cuda"), torch.zeros(2, 4, 1, 64, device="cuda")
        ints = torch.zeros(2, dtype=torch.int32, device="cuda")
        odd = torch.zeros(2 * 2 * 4 * 64 + 1, dtype=torch.bfloat16, device="cuda")[1:].view(2, 2, 4, 64)
        r = B.dkv_rotary_init(64, 64, 0, 1e4)
        other = B.dkv_rotary_init(128, 64, 0, 1e4)
        h = c.h
        bad = [lambda: B.dkv_cache8_reserve(h, -1, 1, 1, None, 1), lambda: B.dkv_cache8_reserve(h, 0, 5, 1, None, 1),
               lambda: B.dkv_cache8_reserve(h, 1, 3, 2, None, 1), lambda: B.dkv_cache8_reserve(h, 0, 2, 0, None, 1),
               lambda: B.dkv_cache8_reserve(h, 0, -1, 1, None, 1), lambda: B.dkv_cache8_reserve(h, 0, 2, 1, None, -1),
               lambda: B.dkv_cache8_reserve(h, 0, 2, 1, ints[:1]), lambda: B.dkv_cache8_reserve(h, 0, 2, 1, ints.long()),
               lambda: B.dkv_cache8_reserve(h, 0, 2, 1, ints.cpu()), lambda: B.dkv_cache8_reserve(h, 0, 2, 2**30, None, 1),
               lambda: B.dkv_cache8_append(h, 0, 3, 1, k, k), lambda: B.dkv_cache8_append(h, 0, 2, 1, k, k[:, :, :3]),
               lambda: B.dkv_cache8_append(h, 0, 2, 1, k, k.half()), lambda: B.dkv_cache8_append(h, 0, 2, 1, k.float(), k.float()),
               lambda: B.dkv_cache8_append(h, 0, 2, 1, k[:, :1], k[:, :1]), lambda: B.dkv_cache8_append(h, 0, 2, 1, odd, k),
               lambda: B.dkv_cache8_append(h, 0, 2, 1, k[..., :32], k[..., :32]), lambda: B.dkv_cache8_append(h, 0, 2, 1, k, None),
               lambda: B.dkv_cache8_append(h, 0, 2, 1, k, k, None, r, None), lambda: B.dkv_cache8_append(h, 0, 2, 1, k, k, None, None, ints),
               lambda: B.dkv_cache8_append(h, 0, 2, 1, k, k, None, other, ints), lambda: B.dkv_cache8_append(h, 0, 2, 1, k.cpu(), k.cpu()),
               lambda: B.dkv_cache8_append(h, 0, 2, 1, k.transpose(2, 3), k.transpose(2, 3)),
               lambda: B.dkv_cache8_read(h, 0, 2, 1, k, k[:, :, :3]), lambda: B.dkv_cache8_read(h, 0, 2, 1, k, odd), lambda: B.dkv_cache8_read(h, 0, 1, 1, k, k),
               lambda: B.dkv_cache8_attend(h, 0, 2, 1, q, out.half()), lambda: B.dkv_cache8_attend(h, 0, 2, 1, q, out[:1]),
               lambda: B.dkv_cache8_attend(h, 0, 2, 1, q[:, :2], out[:, :2]), lambda: B.dkv_cache8_attend(h, 0, 2, 1, q, out, out[:1, :, :, 0].contiguous()),
               lambda: B.dkv_cache8_attend(h, 0, 2, 1, q.expand(2, 4, 33, 64), torch.zeros(2, 4, 33, 64, device="cuda")),
               lambda: B.dkv_cache8_fork(h, 0, 1, 2, 1), lambda: B.dkv_cache8_fork(h, 0, 0, 1, 1), lambda: B.dkv_cache8_fork(h, 0, 3, 2, 1),
               lambda: B.dkv_cache8_fork(h, 2, 0, 2, 2), lambda: B.dkv_cache8_compact(h, 0, 2, 1, ints), lambda: B.dkv_cache8_compact(h, 0, 2, 1, ints.view(2, 1, 1)),
               lambda: B.dkv_cache8_compact(h, 0, 1, 1, torch.zeros(2, 2, 1, dtype=torch.int32, device="cuda")),
               lambda: B.dkv_cache8_trim(h, 0, 2, 1, None, -1), lambda: B.dkv_cache8_trim(h, 0, 2, 1, ints[::2]), lambda: B.dkv_cache8_trim(h, 3, 2, 1, None, 1)]
        for i, call in enumerate(bad):
            with pytest.raises(B.DkvError) as e:
                call()
            assert e.value.code == B.DKV_ERR_INVALID_ARG, i
        # nothing to do
        none = k[:0]
        B.dkv_cache8_reserve(h, 0, 0, 1, None, 1)
        B.dkv_cache8_append(h, 0, 0, 1, none, none)
        B.dkv_cache8_append(h, 0, 2, 1, k[:, :, :0], k[:, :, :0])
        B.dkv_cache8_read(h, 0, 2, 1, k[:, :, :0], k[:, :, :0])
        B.dkv_cache8_attend(h, 0, 2, 1, q[:, :, :0], out[:, :, :0])
        B.dkv_cache8_fork(h, 0, 0, 0, 1)
        B.dkv_cache8_compact(h, 0, 2, 1, torch.zeros(2, 2, 0, dtype=torch.int32, device="cuda"))
        B.dkv_cache8_trim(h, 0, 0, 1)
        assert B.dkv_cache8_status(h)[0] == B.DKV_OK and B.dkv_cache8_last_cuda_error(h) == 0
        c.check()


@pytest.mark.parametrize("kind", ["e4m3", "int8"])
def test_a_prompt_s_way_into_pages_and_through_decoding(kind):
    """Compression, its buffers into pages, and three decoded tokens in every layer: rotated, added, attended to, the last of them
    rejected again; then a sample's memory is given back."""
    w = synth.Workload("gen", 95, L=4, Hq=8, Hkv=2, D=64, Bt=2, S=1024, ws=16, pool=5, N=64, Bl=128, m=2, recipe="sink")
    host = [synth.layer_inputs(w, l) for l in range(w.L)]
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a).view(np.int16)).cuda()
    q, k, v = ([dev(t[n]) for t in host] for n in ("q", "k", "v"))
    rows = w.Blc + w.ws
    kb, vb = ([torch.zeros((w.Bt, w.Hkv, rows, w.D), dtype=torch.int16, device="cuda") for _ in range(w.L)] for _ in range(2))
    ctx = B.dkv_create(B.config_of(w))
    try:
        B.dkv_run_prefill_pass(ctx, q, k, v, kb, vb)
        counts = np.zeros((w.Bt, w.L), dtype=np.int32)
        B.dkv_get_counts(ctx, counts)
    finally:
        B.dkv_destroy(ctx)
    n = w.L * w.Bt
    lens = torch.from_numpy(np.ascontiguousarray(counts.T + w.ws)).cuda().view(-1)       # sequence = layer * Bt + sample
    with Both(n_pages=60, n_seqs=n, max_pages=8, Hkv=w.Hkv, D=w.D, G=w.Hq // w.Hkv, kind=kind) as c:
        B.dkv_cache8_reserve(c.h, 0, n, 1, lens)
        c.o.reserve(range(n), lens.tolist())
        for l in range(w.L):
            B.dkv_cache8_append(c.h, l * w.Bt, w.Bt, 1, kb[l], vb[l], lens[l * w.Bt:(l + 1) * w.Bt])
            for b in range(w.Bt):
                m = int(lens[l * w.Bt + b])
                c.o.append(l * w.Bt + b, *(x[l][b, :, :m].view(torch.bfloat16).double().cpu().numpy() for x in (kb, vb)))
        c.check()
        r = B.dkv_rotary_init(w.D, w.D, B.DKV_ROTARY_HALF, 10000.0)
        g = torch.Generator(device="cuda").manual_seed(4)
        for t in range(3):
            B.dkv_cache8_reserve(c.h, 0, n, 1, None, 1)
            c.o.reserve(range(n), [1] * n)
            pos = torch.full((w.Bt, 1), w.S + t, dtype=torch.int32, device="cuda")
            for l in range(w.L):
                fused = torch.randn((w.Bt, 1, w.Hq + 2 * w.Hkv, w.D), generator=g, device="cuda").to(torch.bfloat16).transpose(1, 2)
                qn, kn, vn = fused[:, :w.Hq], fused[:, w.Hq:w.Hq + w.Hkv], fused[:, w.Hq + w.Hkv:]
                B.dkv_rotate(r, pos, qn, qn, kn, kn)
                B.dkv_cache8_append(c.h, l * w.Bt, w.Bt, 1, kn, vn)
                for b in range(w.Bt):
                    c.o.append(l * w.Bt + b, kn[b].double().cpu().numpy(), vn[b].double().cpu().numpy())
                c.attend(l * w.Bt, w.Bt, 1, 1, True, q=qn)
        B.dkv_cache8_trim(c.h, 0, n, 1, None, 1)
        for s in range(n):
            c.o.trim(s, c.o.len[s] - 1)
        c.check()
        B.dkv_cache8_trim(c.h, 1, w.L, w.Bt, None, 2**31 - 1)                # sample 1, all layers
        for l in range(w.L):
            c.o.trim(l * w.Bt + 1, 0)
        c.check()
        assert B.dkv_cache8_status(c.h)[1][:3] == [0, -1, sum(x == 0 for x in c.o.refs())]


def test_a_cache_that_does_not_fit_is_refused_and_nothing_is_kept():
    free = torch.cuda.mem_get_info()[0]
    with pytest.raises(B.DkvError) as e:
        B.dkv_cache8_create(B.make_cache8_config(2**26, 128, 1, 1, 8, 8, 128))       # 17 TB
    assert e.value.code == B.DKV_ERR_NOMEM and torch.cuda.mem_get_info()[0] == free
    with Both() as c:                                                        # the failure is not taken for a later call's
        c.add(0, 2, 1, [3, 40], 1)
        c.check()
