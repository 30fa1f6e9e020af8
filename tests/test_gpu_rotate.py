"""Rotary positions against the oracle in 64 bits: types, layouts, parts of a head, strides, far positions, gradients."""
import numpy as np
import pytest
import torch

from oracle import cache8 as C
from paper_2412_14838_b200 import binding as B
from paper_2412_14838_b200 import build

pytestmark = pytest.mark.gpu
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


@pytest.fixture(scope="module", autouse=True)
def _lib():
    build.build()
    B.load()


def spec(D, rot, layout, scaling="none", factor=1.0, theta=10000.0):
    high = 32.0 if scaling == "ramp" else 4.0
    r = B.dkv_rotary_init(D, rot, B.DKV_ROTARY_HALF if layout == "half" else B.DKV_ROTARY_PAIRS, theta,
                          ["none", "linear", "base", "wavelength", "ramp"].index(scaling), factor, 1.0, high, 8192.0)
    return r, C.frequencies(rot, theta, scaling, factor, 1.0, high, 8192.0)


def check(got, x, pos, freq, amplitude, layout, transpose):
    """got against the oracle for x [B, H, T, D].  Half a step of the type, and the 32-bit arithmetic before it: the argument of
    sincospif is rounded (2^-24 of at most pi), it is good to two ulp (2^-23 of at most 1), amplitude, product and sum round three times
    more (2^-24 each): less than 8e-7 of |a| + |b| times the amplitude."""
    rot, t = 2 * len(freq), got.dtype
    want = C.rotate(x.double().cpu().numpy(), pos.cpu().numpy()[:, None], freq, amplitude, layout, transpose)
    size = np.abs(x.double().cpu().numpy())
    pair = np.zeros_like(size)
    a, b = (slice(0, rot // 2), slice(rot // 2, rot)) if layout == "half" else (slice(0, rot, 2), slice(1, rot, 2))
    pair[..., a] = pair[..., b] = size[..., a] + size[..., b]
    info = torch.finfo(t)
    bound = np.abs(want) * info.eps / 2 + info.smallest_normal * info.eps / 2 + pair * amplitude * 8e-7 * (1 + info.eps)
    off = np.abs(got.double().cpu().numpy() - want)
    assert (off <= bound).all(), f"off by {(off - bound).max():.3g} more than allowed"
    assert torch.equal(got[..., rot:], x[..., rot:])


@pytest.mark.parametrize("io", list(TYPES))
@pytest.mark.parametrize("layout", ["half", "pairs"])
@pytest.mark.parametrize("D,rot", [(64, 64), (64, 32), (128, 128), (128, 10), (80, 80), (80, 48), (256, 256), (6, 4), (2, 2)])
@pytest.mark.parametrize("transpose", [False, True])
def test_rotation_matches_the_oracle(io, layout, D, rot, transpose):
    g = torch.Generator(device="cuda").manual_seed(D + rot)
    Bt, T, Hq, Hk = 2, 5, 3, 2
    x, y = (torch.randn(Bt, h, T, D, generator=g, device="cuda").to(TYPES[io]) for h in (Hq, Hk))
    pos = torch.randint(-10, 100000, (Bt, T), generator=g, device="cuda", dtype=torch.int32)
    r, (f, a) = spec(D, rot, layout)
    xo, yo = torch.full_like(x, 7.0), torch.full_like(y, 7.0)
    B.dkv_rotate(r, pos, x, xo, y, yo, transpose)
    check(xo, x, pos, f, a, layout, transpose)
    check(yo, y, pos, f, a, layout, transpose)
    alone = torch.full_like(x, 7.0)
    B.dkv_rotate(r, pos, x, alone, transpose=transpose)
    B.dkv_rotate(r, pos, x, x, transpose=transpose)                           # in place
    assert torch.equal(alone, xo) and torch.equal(x, xo)


@pytest.mark.parametrize("scaling", ["linear", "base", "wavelength", "ramp"])
@pytest.mark.parametrize("first", [0, 1 << 20, 2**31 - 40, -(2**31)])
def test_scalings_and_far_positions(scaling, first):
    """The position times its turns is off by 2^-53 of itself, a turn of 2^31 / (2 pi) positions by 4e-8: 2.4e-7 radians at the
    farthest, and the oracle's own product the same: their sum is a part of the bound's 8e-7."""
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn(1, 4, 33, 64, generator=g, device="cuda")
    pos = (first + torch.arange(33, device="cuda", dtype=torch.int64)).to(torch.int32)[None].contiguous()
    r, (f, a) = spec(64, 64, "half", scaling, 8.0, 500000.0)
    out = torch.empty_like(x)
    B.dkv_rotate(r, pos, x, out)
    check(out, x, pos, f, a, "half", False)


@pytest.mark.parametrize("io", ["bf16", "f32"])
def test_token_major_projections_and_their_gradient(io):
    g = torch.Generator(device="cuda").manual_seed(2)
    Bt, T, Hq, Hk, D = 3, 37, 6, 2, 64
    fused = torch.randn(Bt, T, Hq + 2 * Hk, D, generator=g, device="cuda").to(TYPES[io])
    q, k = fused.transpose(1, 2)[:, :Hq], fused.transpose(1, 2)[:, Hq:Hq + Hk]
    pos = torch.randint(0, 5000, (Bt, T), generator=g, device="cuda", dtype=torch.int32)
    r, (f, a) = spec(D, D, "half")
    qo, ko = torch.empty(Bt, Hq, T, D, device="cuda", dtype=fused.dtype), torch.empty(Bt, Hk, T, D, device="cuda", dtype=fused.dtype)
    B.dkv_rotate(r, pos, q, qo, k, ko)
    check(qo, q, pos, f, a, "half", False)
    check(ko, k, pos, f, a, "half", False)
    grad = torch.full_like(fused, 3.0)
    gq, gk = grad.transpose(1, 2)[:, :Hq], grad.transpose(1, 2)[:, Hq:Hq + Hk]
    B.dkv_rotate(r, pos, qo, gq, ko, gk, transpose=True)
    check(gq, qo, pos, f, a, "half", True)
    assert (grad[:, :, Hq + Hk:] == 3.0).all()                                # the values' part is not touched


def test_the_gradient_is_that_of_differences():
    """The map is linear, so a difference quotient is exact but for rounding: with step 1 it is the map itself of one unit vector."""
    r, _ = spec(8, 6, "pairs", "ramp", 4.0)
    pos = torch.tensor([[5, 900]], dtype=torch.int32, device="cuda")
    w = torch.arange(16.0, device="cuda").view(1, 1, 2, 8) / 8 - 1            # loss = sum(w * rotate(x))
    grad, x = torch.empty_like(w), torch.randn(1, 1, 2, 8, device="cuda")
    B.dkv_rotate(r, pos, w, grad, transpose=True)

    def loss(x):
        out = torch.empty_like(x)
        B.dkv_rotate(r, pos, x, out)
        return (w * out).double().sum().item()

    for t in range(2):
        for d in range(8):
            e = torch.zeros_like(x)
            e[0, 0, t, d] = 1.0
            # four values below 4 are rounded to 2^-22 or finer on either side, times weights below 1
            assert abs(loss(x + e) - loss(x) - grad[0, 0, t, d].item()) < 1e-5


def test_unaligned_rows_other_streams_and_graphs():
    r, (f, a) = spec(64, 64, "half")
    raw = torch.randn(2 * 3 * 5 * 64 + 1, device="cuda").to(torch.bfloat16)
    x = raw[1:].view(2, 3, 5, 64)                                             # rows on odd 2-byte places
    pos = torch.arange(10, dtype=torch.int32, device="cuda").view(2, 5)
    out = torch.zeros_like(x)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    B.dkv_rotate(r, pos, x, out, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    check(out, x, pos, f, a, "half", False)
    graph, again = torch.cuda.CUDAGraph(), torch.zeros_like(x)
    with torch.cuda.graph(graph):
        B.dkv_rotate(r, pos, x, again)
    raw.copy_(torch.randn_like(raw))
    pos.add_(77)
    graph.replay()
    B.dkv_rotate(r, pos, x, out)
    assert torch.equal(again, out)
    check(again, x, pos, f, a, "half", False)


def test_many_tokens_and_heads_take_every_share_of_heads():
    r, (f, a) = spec(64, 64, "half")
    for T, H in [(1, 40), (700, 40), (5000, 40), (4096, 1), (1, 1000)]:       # one head a thread up to sixteen
        x = torch.randn(1, H, T, 64, device="cuda").to(torch.bfloat16)
        pos = torch.arange(T, dtype=torch.int32, device="cuda")[None].contiguous()
        out, one = torch.zeros_like(x), torch.zeros_like(x)
        B.dkv_rotate(r, pos, x[:, :H // 2], out[:, :H // 2], x[:, H // 2:], out[:, H // 2:])
        for h in range(0, H, max(1, H // 7)):                                 # heads on their own: another share
            B.dkv_rotate(r, pos, x[:, h:h + 1], one[:, h:h + 1])
            assert torch.equal(one[:, h], out[:, h])
        check(out[:, -1:, -3:], x[:, -1:, -3:], pos[:, -3:], f, a, "half", False)


def test_rotations_refuse_what_does_not_fit():
    r, _ = spec(64, 64, "half")
    x, pos = torch.zeros(1, 2, 3, 64, device="cuda"), torch.zeros(1, 3, dtype=torch.int32, device="cuda")
    bad = [lambda: B.dkv_rotate(r, pos, x, x.double()), lambda: B.dkv_rotate(r, pos, x, x.half()), lambda: B.dkv_rotate(r, pos[:, :2].contiguous(), x, x),
           lambda: B.dkv_rotate(r, pos.long(), x, x), lambda: B.dkv_rotate(r, pos.cpu(), x, x), lambda: B.dkv_rotate(r, pos, x.cpu(), x),
           lambda: B.dkv_rotate(r, pos, x[0], x[0]), lambda: B.dkv_rotate(r, pos, x[..., :32], x[..., :32]),
           lambda: B.dkv_rotate(r, pos, x.transpose(2, 3), x.transpose(2, 3)), lambda: B.dkv_rotate(r, pos, x, x, x[:, :, :2], x[:, :, :2]),
           lambda: B.dkv_rotate(r, pos, x.short(), x.short())]
    for call in bad:
        with pytest.raises(B.DkvError) as e:
            call()
        assert e.value.code == B.DKV_ERR_INVALID_ARG
    B.dkv_rotate(r, pos[:, :0].contiguous(), x[:, :, :0], x[:, :, :0])        # nothing to do
