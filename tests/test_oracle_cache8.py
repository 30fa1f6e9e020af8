"""The oracle of the cache in 8 bits and of rotary positions, pinned without the library; and what the library refuses before it
touches a GPU."""
import ctypes
import math
import os
import re
import subprocess
import sys

import numpy as np
import pytest
import torch

from oracle import cache8 as C
from paper_2412_14838_b200 import binding as B
from paper_2412_14838_b200 import build


@pytest.fixture(scope="module", autouse=True)
def _lib():
    build.build()
    B.load()


def test_e4m3_codes_are_those_of_the_format():
    every = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).to(torch.float64).numpy()
    every = np.unique(every[np.isfinite(every)])
    assert every.max() == 448 and (C.nearest(every, "e4m3") == every).all()
    x = np.concatenate([np.random.default_rng(1).normal(size=5000) * 10.0 ** np.random.default_rng(2).integers(-4, 3, 5000),
                        (every[1:] + every[:-1]) / 2])       # the last: ties
    x = np.clip(x, -448, 448)
    near = every[np.abs(x[:, None] - every).argmin(1)]
    got = C.nearest(x, "e4m3")
    assert (np.abs(got - x) <= np.abs(near - x)).all() and np.isin(got, every).all()
    torch_codes = torch.tensor(x, dtype=torch.float64).to(torch.float32).to(torch.float8_e4m3fn).double().numpy()
    exact32 = x.astype(np.float32).astype(np.float64) == x
    assert (torch_codes[exact32] == got[exact32]).all() and exact32[5000:].all()


@pytest.mark.parametrize("kind,most,scale", [("e4m3", 448.0, 1.0), ("e4m3", 448.0001, 2.0), ("e4m3", 3.5, 2.0 ** -7), ("int8", 127.0, 1.0),
                                             ("int8", 127.5, 2.0), ("int8", 1.0, 2.0 ** -6), ("int8", 0.0, 2.0 ** -126), ("e4m3", 1e-40, 2.0 ** -126)])
def test_scales_by_hand(kind, most, scale):
    assert C.scale_for([-most, most / 3, np.inf, np.nan], kind) == scale


def test_ties_infinities_and_nan():
    assert C.nearest([0.5, 1.5, -2.5, 200.0, np.inf, -np.inf, np.nan], "int8").tolist() == [0, 2, -2, 127, 127, -127, 0]
    # around 16 the step of e4m3 is 2
    assert C.nearest([17.0, 19.0, 1e9, -np.inf, np.nan, 2.0 ** -10], "e4m3").tolist() == [16, 20, 448, -448, 0, 0]


def test_a_growing_scale_rounds_old_codes_again():
    c = C.Cache(2, 32, 1, 2, 1, 64, "int8")
    assert not c.append(0, np.ones((1, 1, 64)), np.ones((1, 1, 64)))          # no room yet
    c.reserve([0], [3])
    one = np.zeros((1, 1, 64))
    one[0, 0, :2] = 127.0, 3.0
    c.append(0, one, one)
    c.append(0, one * 2, one)
    assert c.scales(0, 0).tolist() == [[2, 2]] and c.scales(0, 1).tolist() == [[1, 1]]
    assert c.rows(0, 0)[0, :, :2].tolist() == [[128, 4], [254, 6]]            # 63.5 and 1.5 steps of 2: to even
    assert c.rows(0, 1)[0, :, :2].tolist() == [[127, 3], [127, 3]]


def test_pages_by_hand():
    c = C.Cache(6, 32, 4, 3, 1, 64, "e4m3")
    x = np.random.default_rng(0).normal(size=(1, 40, 64))
    assert c.reserve([0, 1], [40, 1]) == ([], []) and c.table[:2] == [[0, 1], [2]]
    c.append(0, x, x)
    c.fork([(0, 2)])
    assert c.refs() == [2, 2, 1, 0, 0, 0] and not c.append(2, x[:, :1], x[:, :1])
    assert c.reserve([2], [1]) == ([], []) and c.table[2] == [0, 3] and c.refs() == [2, 1, 1, 1, 0, 0]
    source = c.rows(0, 0)
    c.append(2, x[:, :1] * 1000, x[:, :1])
    assert (c.rows(0, 0) == source).all() and c.scales(0, 0)[0, 33] < c.scales(2, 0)[0, 33]
    assert c.reserve([3, 1], [90, 1]) == ([3], []) and c.len == [40, 0, 41, 0]   # 3 pages wanted, 2 free; 1 has room
    assert c.reserve([1], [97]) == ([], [1])
    before = c.rows(2, 1)
    assert c.compact([2], [[[40, 0, 0]]]) == [] and c.table[2] == [4] and (c.rows(2, 1) == before[:, [40, 0, 0]]).all()
    c.trim(0, 32)
    assert c.table[0] == [0] and c.refs() == [1, 0, 1, 0, 1, 0]


def test_attention_by_hand():
    k = np.zeros((1, 3, 64))
    v = np.arange(3.0)[None, :, None] + np.zeros((1, 3, 64))
    k[0, 1, 0] = 8 * math.log(2)                                              # weights 1 : 2 : 1
    q = np.zeros((2, 2, 64))
    q[0, :, 0] = 1.0
    out, lse = C.attention(q, k, v, True)
    assert np.allclose(out[0, 1], 1.0) and np.allclose(out[0, 0], 2 / 3) and np.allclose(out[1], [[0.5] * 64, [1.0] * 64])
    assert np.allclose(lse, np.log([[3, 4], [2, 3]]))
    out, lse = C.attention(q, k[:, :1], v[:, :1], True)                       # the first query sees no row
    assert (out[:, 0] == 0).all() and (lse[:, 0] == -np.inf).all() and np.allclose(lse[:, 1], 0)


@pytest.mark.parametrize("layout", ["half", "pairs"])
def test_rotations_keep_lengths_and_add_up(layout):
    rng = np.random.default_rng(5)
    x, g = rng.normal(size=(2, 7, 12)), rng.normal(size=(2, 7, 12))
    pos, (f, a) = rng.integers(-50, 1000, size=(2, 7)), C.frequencies(8, 10000.0)
    y = C.rotate(x, pos, f, a, layout)
    assert np.allclose((y ** 2).sum(-1), (x ** 2).sum(-1)) and (y[..., 8:] == x[..., 8:]).all()
    assert np.allclose(C.rotate(y, 3 - pos, f, a, layout), C.rotate(x, np.full((2, 7), 3), f, a, layout))
    assert np.isclose((g * y).sum(), (C.rotate(g, pos, f, a, layout, True) * x).sum())
    a, b = (0, 4) if layout == "half" else (0, 1)
    assert np.allclose(y[0, 0, a], x[0, 0, a] * math.cos(pos[0, 0]) - x[0, 0, b] * math.sin(pos[0, 0]))


@pytest.mark.parametrize("scaling", ["none", "linear", "base", "wavelength", "ramp"])
@pytest.mark.parametrize("rot", [4, 10, 64, 128, 256])
def test_the_library_has_the_oracle_s_frequencies(scaling, rot):
    code = ["none", "linear", "base", "wavelength", "ramp"].index(scaling)
    high = 32.0 if scaling == "ramp" else 4.0
    r = B.dkv_rotary_init(256, rot, B.DKV_ROTARY_HALF, 500000.0, code, 8.0, 1.0, high, 8192.0)
    f, a = C.frequencies(rot, 500000.0, scaling, 8.0, 1.0, high, 8192.0)
    # 64 bits on both sides: a few roundings of relative 2^-53, and pow's own error of an ulp or two
    assert np.allclose(np.array(r.turns[:rot // 2]) * 2 * math.pi, f, rtol=1e-14, atol=0) and abs(r.amplitude - a) < 1e-7


def test_the_slowest_pair_of_an_extended_base_turns_slower_by_the_factor():
    f, g = C.frequencies(64, 1e4)[0], C.frequencies(64, 1e4, "base", 4.0)[0]
    assert math.isclose(f[-1] / g[-1], 4.0) and f[0] == g[0] == 1.0


GOOD = dict(head_dim=64, rot_dim=64, layout=0, theta=1e4, scaling=0, factor=1.0, low=1.0, high=4.0, trained_len=100.0)


@pytest.mark.parametrize("kw", [dict(head_dim=63), dict(head_dim=258), dict(rot_dim=66), dict(rot_dim=0), dict(rot_dim=7), dict(layout=2),
                                dict(theta=0.0), dict(theta=math.nan), dict(scaling=5), dict(scaling=-1), dict(scaling=1, factor=0.5),
                                dict(scaling=2, rot_dim=2, factor=2.0), dict(scaling=3, low=4.0), dict(scaling=3, trained_len=0.0),
                                dict(scaling=4, theta=1.0), dict(scaling=3, high=math.inf), dict(scaling=1, factor=math.inf)])
def test_bad_rotary_configurations_are_refused(kw):
    B.dkv_rotary_init(**GOOD)
    with pytest.raises(B.DkvError) as e:
        B.dkv_rotary_init(**{**GOOD, **kw})
    assert e.value.code == B.DKV_ERR_INVALID_ARG


def test_rotations_are_checked_on_the_host():
    r = B.dkv_rotary_init(**GOOD)
    x, pos = torch.zeros(1, 2, 3, 64), torch.zeros(1, 3, dtype=torch.int32)
    # (addresses that the library would refuse before it uses them)
    rows = lambda **kw: B.DkvRows(**{**dict(data=4096, type=B.DKV_F32, batch=1, heads=2, tokens=3, head_dim=64, batch_stride=384,
                                            head_stride=192, token_stride=64), **kw})
    good = rows()
    bad = [lambda: B.dkv_rotate(r, pos, x, x, stream=0),                                         # not on a GPU
           lambda: B.dkv_rotate(None, 4096, good, good, stream=0), lambda: B.dkv_rotate(r, None, good, good, stream=0),
           lambda: B.dkv_rotate(r, 4096, None, good, stream=0), lambda: B.dkv_rotate(r, 4098, good, good, stream=0),
           lambda: B.dkv_rotate(r, 4096, good, good, good, None, stream=0), lambda: B.dkv_rotate(B.DkvRotary(), 4096, good, good, stream=0)]
    for kw in (dict(data=None), dict(data=4097), dict(type=3), dict(type=-1), dict(heads=-1), dict(head_dim=128), dict(token_stride=-64), dict(tokens=4)):
        bad += [lambda kw=kw: B.dkv_rotate(r, 4096, rows(**kw), good, stream=0), lambda kw=kw: B.dkv_rotate(r, 4096, good, rows(**kw), stream=0),
                lambda kw=kw: B.dkv_rotate(r, 4096, good, good, rows(**kw), rows(**kw), stream=0)] if kw != dict(tokens=4) else [
                lambda: B.dkv_rotate(r, 4096, rows(tokens=4), good, stream=0)]
    bad.append(lambda: B.dkv_rotate(r, 4096, good, rows(token_stride=128), stream=0))            # in place, other strides
    for call in bad:
        with pytest.raises(B.DkvError) as e:
            call()
        assert e.value.code == B.DKV_ERR_INVALID_ARG
    for kw in (dict(batch=0), dict(heads=0), dict(tokens=0)):                                    # nothing to do
        B.dkv_rotate(r, None, rows(data=None, **kw), rows(data=None, **kw), stream=0)


CONFIG = dict(n_pages=8, page_rows=32, n_seqs=4, max_pages=4, n_q_heads=4, n_kv_heads=2, head_dim=64)


@pytest.mark.parametrize("kw,code", [(dict(n_pages=0), -1), (dict(n_seqs=0), -1), (dict(max_pages=0), -1), (dict(n_q_heads=3), -1),
                                     (dict(n_kv_heads=0), -1), (dict(page_rows=16), -5), (dict(head_dim=96), -5), (dict(kind=2), -5),
                                     (dict(io=2), -5), (dict(n_pages=2**26 + 1), -5), (dict(n_seqs=65536), -5), (dict(max_pages=2**20), -5)])
def test_bad_caches_are_refused(kw, code):
    with pytest.raises(B.DkvError) as e:
        B.dkv_cache8_create(B.make_cache8_config(**{**CONFIG, **kw}))
    assert e.value.code == code


def test_calls_without_a_cache_are_refused():
    lib, rows, out = B.load(), B.DkvRows(), (ctypes.c_int32 * 8)()
    assert lib.dkv_cache8_create(None, None) == lib.dkv_cache8_destroy(None) == lib.dkv_cache8_status(None, out) == B.DKV_ERR_INVALID_ARG
    assert lib.dkv_cache8_views(None, None, None, None, None) == B.DKV_ERR_INVALID_ARG and lib.dkv_cache8_last_cuda_error(None) == 0
    for call in (lambda: B.dkv_cache8_reserve(0, 0, 1, 1, None, 1, 0), lambda: B.dkv_cache8_append(0, 0, 1, 1, rows, rows, stream=0),
                 lambda: B.dkv_cache8_read(0, 0, 1, 1, rows, rows, 0), lambda: B.dkv_cache8_attend(0, 0, 1, 1, rows, rows, stream=0),
                 lambda: B.dkv_cache8_fork(0, 0, 1, 1, 1, 0), lambda: B.dkv_cache8_compact(0, 0, 1, 1, 4096, stream=0),
                 lambda: B.dkv_cache8_trim(0, 0, 1, 1, None, 1, 0)):
        with pytest.raises(B.DkvError) as e:
            call()
        assert e.value.code == B.DKV_ERR_INVALID_ARG
    with pytest.raises(TypeError):
        B.dkv_cache8_read(0, 0, 1, 1, "x", rows, 0)


def test_a_program_without_torch_makes_the_same_calls():
    code = """
import sys
sys.modules["torch"] = None                                   # "import torch" fails
from paper_2412_14838_b200 import binding as B
def refused(call):
    try: call()
    except B.DkvError as e: return e.code == B.DKV_ERR_INVALID_ARG
r = B.dkv_rotary_init(64, 64, B.DKV_ROTARY_PAIRS, 1e4)
rows = lambda n: B.DkvRows(None, B.DKV_F32, 1, 2, n, 64, 128, 64, 64)
B.dkv_rotate(r, 0, rows(0), rows(0), stream=0)                # nothing to do
assert refused(lambda: B.dkv_rotate(r, 4096, rows(3), rows(3), transpose=True, stream=0))      # no data
assert refused(lambda: B.dkv_cache8_append(0, 0, 1, 1, rows(1), rows(1), None, r, 4096, 0))
assert refused(lambda: B.dkv_cache8_compact(0, 0, 1, 1, 4096, None, 0, heads=2, cols=3))
assert refused(lambda: B.dkv_cache8_attend(0, 0, 1, 1, rows(1), rows(1), None, True, 0))
"""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    subprocess.run([sys.executable, "-c", code], cwd=root, check=True)


@pytest.mark.parametrize("field,value", [("amplitude", math.nan), ("amplitude", math.inf), ("turns", math.nan), ("turns", math.inf)])
def test_frequencies_that_are_not_finite_are_refused(field, value):
    r = B.dkv_rotary_init(**GOOD)
    if field == "turns":
        r.turns[31] = value
    else:
        r.amplitude = value
    rows = B.DkvRows(4096, B.DKV_F32, 1, 2, 3, 64, 384, 192, 64)
    with pytest.raises(B.DkvError) as e:
        B.dkv_rotate(r, 4096, rows, rows, stream=0)
    assert e.value.code == B.DKV_ERR_INVALID_ARG


@pytest.mark.parametrize("header", ["cache8.cuh", "attend8.cuh", "rotary.cuh"])
def test_every_kernel_waits_for_the_one_before_it_before_it_does_or_skips_anything(header):
    """All are launched while their predecessor may still run, and each counts on every kernel before it being complete: that
    holds if no block of any of them ends without its own wait."""
    from tests.test_launch_overlap import _functions, _source
    kernels = {n: b for n, _, b in _functions(_source(header)) if n.endswith("_kernel")}
    assert kernels
    for name, body in kernels.items():
        wait = body.index("pdl_wait();")
        assert body.index("pdl_launch();") < wait, name
        assert "return" not in body[:wait], name
        head = body[:wait]
        assert head.count("{") - head.count("}") == 1, f"{name}: the wait holds for every thread"
        assert not re.search(r"\bc\.(len|held|table|refs|free|hint|scales|pages)\s*\[", head), f"{name} reads ahead of its wait"
