"""Rotary positions and norms of heads on the GPU against the plain definition in 64 bits."""

import math

import numpy as np
import pytest
import torch

from oracle import pages_oracle as orc
from tests._util import f64

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F16, BF16, F32 = torch.float16, torch.bfloat16, torch.float32
HALF = {F32: 2.0 ** -24, F16: 2.0 ** -11, BF16: 2.0 ** -8}   # most that a rounding is off, relative
TINY = {F32: 2.0 ** -150, F16: 2.0 ** -25, BF16: 2.0 ** -134}   # or in all, among the smallest numbers


def _rand(shape, dtype, seed, std=1.0):
    g = torch.Generator(device="cpu")
    g.manual_seed(seed)
    return (torch.randn(*shape, generator=g) * std).to(dtype).to(DEV)


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def assert_turned(got, want, x, scale, norm, dtype):
    """Half a unit of the result, and of fp32: an angle within 2 2^-24 (an eighth of a turn at most, two roundings), its sine and
    cosine within 4 2^-24 with the series' own roundings and `scale`, two products and a sum, 3 2^-24, of both channels' size; with a
    norm 2^-24 for each of the 16 + 6 additions of a lane and between lanes, halved by the root, and 5 for mean, eps, root,
    quotient and products: 16."""
    size = np.abs(x).max(-1, keepdims=True) * math.sqrt(2.0)   # of a pair, after the norm
    bound = HALF[dtype] * np.abs(want) + TINY[dtype] + 2.0 ** -24 * (9.0 * max(scale, 1.0) + (16.0 * max(scale, 1.0) if norm else 0.0)) * size
    err = np.abs(f64(got) - want)
    assert np.all(err <= bound), float((err / bound).max())


def _check(lib, T, H, D, rot, dtype, style="half", norm=False, backward=False, scaling=None, pos=None, view=lambda t: t, into=None,
           seed=0, eps=1e-6):
    kw = scaling or {}
    angles = lib.rope_angles(rot, style=style, device=DEV, **kw) if rot else None
    x = view(_rand((T, H, D), dtype, seed, 2.0))
    w = (1.0 + _rand((D,), F32, seed + 1, 0.3)).to(dtype) if norm else None
    pos = np.random.default_rng(seed).integers(0, 1 << 20, T) if pos is None else np.asarray(pos)
    out = None if into is None else into(torch.full((T, H, D), 7.0, dtype=dtype, device=DEV))
    y = lib.rope(x, _ints(pos.tolist()) if rot else None, angles, norm=w, eps=eps, backward=backward, out=out)
    f = orc.frequencies(rot, **{k: v for k, v in kw.items() if k != "scale"}) if rot else ()
    scale = angles.scale if rot else 1.0
    normed = orc.rope(f64(x), pos, norm=f64(w) if norm else None, eps=eps)
    want = orc.rope(f64(x), pos, f, style, scale, f64(w) if norm else None, eps, backward)
    assert_turned(y, want, normed, scale, norm, dtype)
    return x, y


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("style", ["half", "interleaved"])
@pytest.mark.parametrize("D,rot", [(128, 128), (128, 64), (64, 64), (64, 16), (96, 96), (80, 32), (256, 64), (512, 512), (2, 2), (6, 4),
                                   (127, 126), (100, 50), (128, 36), (64, 0), (1, 0)])
def test_every_shape(lib, D, rot, style, dtype):
    for T, H, norm in ((1, 3, False), (5, 40, True), (2, 1, True)):
        _check(lib, T, H, D, rot, dtype, style, norm, seed=D + rot + T)


@pytest.mark.parametrize("T,H", [(1, 1), (1, 33), (1023, 3), (1024, 5), (1030, 72), (4097, 2)])
@pytest.mark.parametrize("style", ["half", "interleaved"])
@pytest.mark.parametrize("norm", [False, True])
def test_many_tokens_and_heads(lib, T, H, style, norm):
    _check(lib, T, H, 128, 128, BF16, style, norm, seed=T)
    _check(lib, T, H, 64, 32, F32, style, norm, backward=not norm, seed=T + 1)


@pytest.mark.parametrize("kw", [dict(scaling="linear", factor=4.0), dict(scaling="base", factor=8.0), dict(base=500000.0),
                                dict(scaling="parts", factor=4.0, original=4096.0), dict(scale=0.5)])
def test_scaled_frequencies(lib, kw):
    _check(lib, 33, 4, 128, 128, F32, scaling=kw)
    _check(lib, 33, 4, 128, 64, F16, "interleaved", True, scaling=kw)


def test_far_and_negative_positions_are_exact(lib):
    """At 2^31 - 1 an angle in fp32 would be off by 64 radians."""
    pos = [0, 1, -1, 2 ** 31 - 1, -2 ** 31, 10 ** 9 + 7, -12345, 65536]
    for style in ("half", "interleaved"):
        # the frequencies' own rounding, 2^-53 of them, is 2^-22 at these positions: taken from the host's turns instead
        x = torch.ones((len(pos), 1, 128), dtype=F32, device=DEV)
        angles = lib.rope_angles(128, style=style, device=DEV)
        y = f64(lib.rope(x, _ints(pos), angles))[:, 0]
        turns = [int(v) & (2 ** 64 - 1) for v in angles.turns.tolist()]
        for i, p in enumerate(pos):
            for j, t in enumerate(turns):
                a = 2 * math.pi * (t * p % 2 ** 64) / 2 ** 64
                u, v = (j, j + 64) if style == "half" else (2 * j, 2 * j + 1)
                assert abs(y[i, u] - (math.cos(a) - math.sin(a))) <= 2.0 ** -24 * 14 and \
                    abs(y[i, v] - (math.cos(a) + math.sin(a))) <= 2.0 ** -24 * 14, (p, j)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_strided_and_misaligned_rows(lib, dtype):
    T, H, D = 7, 3, 64
    for norm in (False, True):
        for odd in (0, 1, 8):
            def slice_of_fused(t):
                wide = torch.full((T, 5 * D * H + odd), 9.0, dtype=dtype, device=DEV)
                part = wide[:, D * H + odd:2 * D * H + odd].unflatten(-1, (H, D))
                part.copy_(t)
                return part
            _check(lib, T, H, D, 32, dtype, norm=norm, view=slice_of_fused)
            _check(lib, T, H, D, 32, dtype, norm=norm, into=slice_of_fused)
            # heads of one token apart from one another: [H, T, D] memory
            _check(lib, T, H, D, 32, dtype, norm=norm, view=lambda t: t.transpose(0, 1).contiguous().transpose(0, 1))


def test_what_lies_between_strided_rows_stays(lib):
    T, H, D = 1027, 3, 64
    wide = torch.full((T, 4 * H, D), 9.0, dtype=F16, device=DEV)
    out = wide[:, H:2 * H]
    x = _rand((T, H, D), F16, 3)
    pos = _ints(list(range(T)))
    angles = lib.rope_angles(64, device=DEV)
    lib.rope(x, pos, angles, out=out)
    assert torch.equal(out, lib.rope(x, pos, angles))
    assert bool((wide[:, :H] == 9.0).all()) and bool((wide[:, 2 * H:] == 9.0).all())


@pytest.mark.parametrize("T,D,rot", [(5, 128, 128), (5, 128, 36), (1500, 64, 32)])
@pytest.mark.parametrize("norm", [False, True])
def test_in_place(lib, T, D, rot, norm):
    x = _rand((T, 9, D), BF16, 1)
    w = _rand((D,), BF16, 2) if norm else None
    pos = _ints(list(range(100, 100 + T)))
    angles = lib.rope_angles(rot, device=DEV)
    want = lib.rope(x, pos, angles, norm=w)
    got = lib.rope(x, pos, angles, norm=w, out=x)
    assert got is x and torch.equal(x, want)


@pytest.mark.parametrize("style", ["half", "interleaved"])
@pytest.mark.parametrize("rot", [64, 36])
def test_backward_is_the_gradient(lib, style, rot):
    """Against differences of the plain definition (a linear map: their error is rounding), and <y, J x> = <J^T y, x>."""
    T, H, D = 4, 2, 64
    pos = np.array([0, 3, 1000, 77])
    angles = lib.rope_angles(rot, style=style, scale=1.25, device=DEV)
    x, dy = _rand((T, H, D), F32, 1), _rand((T, H, D), F32, 2)
    dx = f64(lib.rope(dy, _ints(pos.tolist()), angles, backward=True))
    f = orc.frequencies(rot)
    loss = lambda v: float((orc.rope(v, pos, f, style, 1.25) * f64(dy)).sum())  # noqa: E731
    rng = np.random.default_rng(0)
    for _ in range(20):
        at = tuple(rng.integers(0, n) for n in (T, H, D))
        step = np.zeros((T, H, D))
        step[at] = 0.5
        assert abs(loss(f64(x) + step) - loss(f64(x) - step) - dx[at]) <= 2.0 ** -24 * 16 * np.abs(f64(dy)).max()
    y = f64(lib.rope(x, _ints(pos.tolist()), angles))
    assert abs((y * f64(dy)).sum() - (f64(x) * dx).sum()) <= 2.0 ** -20 * np.abs(y * f64(dy)).sum()


def test_turned_and_turned_back(lib):
    x = _rand((50, 4, 128), F32, 5)
    pos = _ints([i * 7919 for i in range(50)])
    angles = lib.rope_angles(128, device=DEV)
    back = lib.rope(lib.rope(x, pos, angles), pos, angles, backward=True)
    assert float((back - x).abs().max()) <= 2.0 ** -24 * 24 * math.sqrt(2.0) * float(x.abs().max())


def test_infinities_stay_in_their_head(lib):
    x = _rand((3, 4, 128), F32, 6)
    x[1, 2, 5] = math.inf
    x[2, 0, 127] = math.nan
    pos, angles, w = _ints([4, 5, 6]), lib.rope_angles(64, device=DEV), torch.ones(128, device=DEV)
    for norm in (None, w):
        y = lib.rope(x, pos, angles, norm=norm)
        bad = ~torch.isfinite(y).all(-1)
        assert bad.tolist() == [[False] * 4, [False, False, True, False], [True, False, False, False]]
    # without a norm only the pair: channels 5 and 37
    y = lib.rope(x, pos, angles)
    assert (~torch.isfinite(y[1, 2])).nonzero().flatten().tolist() == [5, 37]


def test_a_zero_head_with_a_norm(lib):
    x = torch.zeros((2, 3, 64), dtype=F16, device=DEV)
    y = lib.rope(x, None, None, norm=torch.ones(64, dtype=F16, device=DEV), eps=1e-6)
    assert bool((y == 0).all())


def test_captured_with_positions_that_move(lib):
    x, angles, pos = _rand((3, 8, 128), BF16, 1), lib.rope_angles(128, device=DEV), _ints([0, 0, 0])
    out = torch.empty_like(x)
    lib.rope(x, pos, angles, out=out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        lib.rope(x, pos, angles, out=out)
    for i in range(4):
        pos.copy_(_ints([i, 10 * i, 1000 * i]))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, lib.rope(x, pos, angles))


def test_on_a_stream_of_its_own(lib):
    x, angles, pos = _rand((300, 8, 128), BF16, 1), lib.rope_angles(128, device=DEV), _ints(list(range(300)))
    want = lib.rope(x, pos, angles)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = lib.rope(x, pos, angles)
    side.synchronize()
    assert torch.equal(got, want)
