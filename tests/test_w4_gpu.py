"""4-bit weights on the GPU against the plain definitions: packing exactly, products within the rounding of their sums."""

import numpy as np
import pytest
import torch

from oracle import q4_oracle as orc
from tests._util import f64

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F16, BF16, F32 = torch.float16, torch.bfloat16, torch.float32
HALF_ULP = {F32: 2.0 ** -24, F16: 2.0 ** -11, BF16: 2.0 ** -8}   # of a result's magnitude (bf16: a whole one)
OFFSET = {F32: 0.0, F16: 64.0, BF16: 128.0}                      # what the operands carry beside a code


def _rand(shape, dtype, seed, std=1.0, device=DEV):
    g = torch.Generator(device="cpu")
    g.manual_seed(seed)
    return (torch.randn(*shape, generator=g) * std).to(dtype).to(device)


def _sum_bound(x, w, group, offset):
    """Error of a sum of C rounded products and additions: each rounds 2^-24 of a partial sum, which is as large as the
    root of the terms' squares; the roundings add up like their root, and eight times that is not passed."""
    codes, steps, lows = orc.hold(w, group)
    size = steps * (offset + 15.0) + np.abs(lows)
    scale = np.sqrt((np.asarray(x, dtype=np.float64) ** 2) @ (size ** 2).T)
    return 8.0 * np.sqrt(w.shape[1] + 32) * 2.0 ** -24 * scale


def _matvec_bound(x, w, gate, bias, act, group, x_dtype, y_dtype, want):
    err = _sum_bound(x, w, group, OFFSET[x_dtype])
    if act == "swiglu":
        hw, hg = orc.held_values(w, group), orc.held_values(gate, group)
        u, g = x @ hw.T, x @ hg.T
        # SiLU's slope is below 1.1, its fp32 error a few 2^-22 of it
        err = np.abs(u) * (1.1 * _sum_bound(x, gate, group, OFFSET[x_dtype]) + 2.0 ** -20 * np.abs(orc.silu(g))) + np.abs(orc.silu(g)) * err
    floor = 2.0 ** -24 if y_dtype == F16 else 0.0   # below fp16's normal numbers
    return 1.01 * err + HALF_ULP[y_dtype] * (np.abs(want) + err) + floor + 1e-30


def _check(lib, M, R, C, group, act, x_dtype, w_dtype=None, y_dtype=None, bias=True, seed=0, x=None):
    w_dtype, y_dtype = w_dtype or x_dtype, y_dtype or x_dtype
    w = _rand((R, C), w_dtype, seed + 1, 0.02)
    gate = _rand((R, C), w_dtype, seed + 2, 0.02) if act == "swiglu" else None
    b = _rand((R,), w_dtype, seed + 3, 0.1) if bias and act != "swiglu" else None
    x = _rand((M, C), x_dtype, seed + 4) if x is None else x
    pw, pg = lib.w4_quantize(w, group), None if gate is None else lib.w4_quantize(gate, group)
    y = lib.w4_matvec(x, pw, gate=pg, bias=b, act=act, out_dtype=y_dtype)
    assert y.dtype == y_dtype and y.shape == (M, R)
    xw, ww, gw = f64(x), f64(w), f64(gate)
    want = orc.matvec(xw, orc.held_values(ww, group), None if gate is None else orc.held_values(gw, group), f64(b), act)
    bound = _matvec_bound(xw, ww, gw, b, act, group, x_dtype, y_dtype, want)
    err = np.abs(f64(y) - want)
    assert (err <= bound).all(), (err.max(), bound.flat[err.argmax()], want.flat[err.argmax()])


@pytest.mark.parametrize("R,C", [(1, 1), (16, 128), (17, 129), (5, 31), (40, 200), (33, 1000)])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("dtype", [F32, F16, BF16])
def test_packing_is_exact(lib, R, C, group, dtype):
    w = _rand((R, C), dtype, R + C + group, 0.3)
    w[0, 0] = 7.0                      # a range far from the others'
    w[R // 2] = 0.5                    # a row of equal elements: step 0
    got = lib.w4_read(lib.w4_quantize(w, group), F32)
    want = orc.held_values(f64(w), group).astype(np.float32)
    assert np.array_equal(got.cpu().numpy(), want)
    again = lib.w4_read(lib.w4_quantize(w, group), dtype)
    assert torch.equal(again, torch.from_numpy(want).to(dtype).to(DEV))


def test_packing_of_strided_rows_and_reuse_of_a_buffer(lib):
    base = _rand((70, 301), F16, 3)
    w = base[1::2, 5:206]              # odd offset, row stride 602 elements
    packed = torch.empty(lib.w4_size(*w.shape, 64), dtype=torch.uint8, device=DEV).fill_(0xa5)
    got = lib.w4_read(lib.w4_quantize(w, 64, packed), F32)
    assert np.array_equal(got.cpu().numpy(), orc.held_values(f64(w), 64).astype(np.float32))
    out = torch.full((35, 250), 3.0, dtype=F16, device=DEV)
    lib.w4_read(lib.w4_quantize(w, 64, packed), F16, out=out[:, 20:221])
    assert (out[:, :20] == 3.0).all() and (out[:, 221:] == 3.0).all()
    assert torch.equal(out[:, 20:221], got.to(F16))


def test_values_that_fp16_does_not_hold(lib):
    w = torch.zeros(5, 64, dtype=F32, device=DEV)
    w[0, 3], w[1, 5], w[2, 7] = 1e6, -1e6, float("nan")
    w[3, 1], w[3, 2] = float("inf"), -5.0
    w[4] = torch.linspace(0, 1e-9, 64)     # a step that fp16 rounds to zero
    got = lib.w4_read(lib.w4_quantize(w, 32), F32).cpu().numpy()
    want = orc.held_values(f64(w), 32).astype(np.float32)
    assert np.array_equal(got, want, equal_nan=True)
    assert np.isnan(got[2, :32]).all() and np.isfinite(got[2, 32:]).all() and np.isfinite(got[[0, 1, 3, 4]]).all()


@pytest.mark.parametrize("act", ["none", "relu", "swiglu"])
@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("group", [32, 64, 128])
def test_one_row(lib, group, dtype, act):
    for R, C in ((1, 1), (16, 128), (15, 127), (33, 129), (260, 1000), (1100, 640)):
        _check(lib, 1, R, C, group, act, dtype, seed=R + C)


@pytest.mark.parametrize("M", [2, 3, 8, 15, 16, 17, 31, 33, 48, 64])
@pytest.mark.parametrize("dtype,act,group", [(F16, "relu", 64), (BF16, "swiglu", 128), (F32, "none", 32)])
def test_several_rows(lib, M, dtype, act, group):
    _check(lib, M, 75, 333, group, act, dtype, seed=M)
    _check(lib, M, 130, 512, group, act, dtype, seed=M + 100)


@pytest.mark.parametrize("M,R,C,group,act,dtype", [
    (1, 16390, 520, 64, "none", F16), (1, 20000, 128, 32, "relu", BF16),      # two tiles of rows a workgroup
    (8, 64, 9216, 64, "relu", F16), (16, 40, 4104, 128, "swiglu", BF16),      # x does not fit beside two workgroups
    (1, 24, 36864, 64, "none", F16), (3, 48, 11008, 128, "none", F32),        # long rows
    (16, 14410, 2056, 64, "relu", BF16),                                       # fours of tiles beside rows in memory
    (1, 24, 70000, 128, "none", BF16), (64, 100, 2056, 32, "swiglu", F16)])
def test_the_ways_that_sizes_choose(lib, M, R, C, group, act, dtype):
    _check(lib, M, R, C, group, act, dtype, seed=7)


@pytest.mark.parametrize("x_dtype,y_dtype,w_dtype", [(BF16, F32, BF16), (F32, BF16, BF16), (F32, F16, F16), (F16, BF16, F32)])
def test_mixed_types(lib, x_dtype, y_dtype, w_dtype):
    for act in ("relu", "swiglu", "none"):
        _check(lib, 2, 70, 300, 64, act, x_dtype, w_dtype=w_dtype, y_dtype=y_dtype)


def test_strided_rows_of_x_and_y(lib):
    w = _rand((50, 203), F16, 1, 0.02)
    pw = lib.w4_quantize(w, 32)
    for M in (3, 20):
        base = _rand((M, 311), F16, 2)
        x = base[:, 1:204]                                    # unaligned rows
        out = torch.full((M, 71), 9.0, dtype=F16, device=DEV)
        lib.w4_matvec(x, pw, y=out[:, 3:53])
        whole = lib.w4_matvec(x.contiguous(), pw)
        assert torch.equal(out[:, 3:53], whole)
        assert (out[:, :3] == 9.0).all() and (out[:, 53:] == 9.0).all()
    one = lib.w4_matvec(x[0], pw)
    assert one.shape == (50,) and torch.equal(one, lib.w4_matvec(x[:1].contiguous(), pw)[0])


def test_rows_that_are_not_finite_stay_among_themselves(lib):
    pw = lib.w4_quantize(_rand((40, 300), BF16, 5, 0.02), 64)
    for M in (3, 40):
        x = _rand((M, 300), BF16, 6)
        good = lib.w4_matvec(x, pw)
        x[1, 7], x[2, 250] = float("inf"), float("nan")
        y = lib.w4_matvec(x, pw)
        assert torch.isnan(y[1]).all() and torch.isnan(y[2]).all()
        rest = [m for m in range(M) if m not in (1, 2)]
        assert torch.equal(y[rest], good[rest])


def test_products_repeat_to_the_bit_on_another_stream_and_in_a_graph(lib):
    pw = lib.w4_quantize(_rand((500, 1500), F16, 5, 0.02), 64)
    for M in (1, 40):
        x = _rand((M, 1500), F16, 6)
        y = lib.w4_matvec(x, pw)
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            other = lib.w4_matvec(x, pw)
        torch.cuda.current_stream().wait_stream(s)
        assert torch.equal(y, other)
        need = lib.w4_matvec_workspace_size(M, 1500, F16)
        ws, out = torch.empty(max(need, 16), dtype=torch.uint8, device=DEV), torch.empty_like(y)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            lib.w4_matvec(x, pw, y=out, ws=ws)
        for seed in (8, 9, 10):
            x.copy_(_rand((M, 1500), F16, seed))
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, lib.w4_matvec(x, pw))


def test_a_layer_of_deployed_core_neurons_in_4_bits(lib):
    """Compact buffers of both layouts, packed, and the FFN of one token as two products with fp32 hidden values."""
    d, N, K = 256, 1000, 301
    for act in ("relu", "swiglu"):
        w_up, w_down = _rand((N, d), F16, 1, 0.02), _rand((d, N), F16, 2, 0.02)
        w_gate = _rand((N, d), F16, 3, 0.02) if act == "swiglu" else None
        b_up = _rand((N,), F16, 4, 0.1) if act == "relu" else None
        idx = torch.arange(0, 3 * K, 3, dtype=torch.int32, device=DEV)
        c = lib.compact(w_up, w_gate, b_up, w_down, "out_major", act, idx, down_c_layout="out_major")
        up, down = lib.w4_quantize(c["w_up_c"], 64), lib.w4_quantize(c["w_down_c"][:, :K], 64)
        gate = None if w_gate is None else lib.w4_quantize(c["w_gate_c"], 64)
        x = _rand((2, d), F16, 9)
        h = lib.w4_matvec(x, up, gate=gate, bias=None if b_up is None else c["b_up_c"][:K].contiguous(), act=act, out_dtype=F32)
        y = lib.w4_matvec(h, down, out_dtype=F16)
        at = idx.cpu().numpy()
        rows = lambda m: None if m is None else orc.held_values(f64(m)[at], 64)  # noqa: E731
        hid = orc.matvec(f64(x), rows(w_up), rows(w_gate), None if b_up is None else f64(b_up)[at], act)
        want = hid @ orc.held_values(f64(w_down)[:, at], 64).T
        # hidden values 2^-14 off at most relative to their size, and the output's rounding
        rms = np.sqrt(np.mean(want ** 2))
        assert np.abs(f64(y) - want).max() <= 2e-3 * rms + 2.0 ** -11 * np.abs(want).max()


@pytest.mark.parametrize("M", [1, 8, 40])
@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("group", [32, 64, 128])
def test_fp32_results_of_16_bit_rows_keep_their_bits(lib, group, dtype, M):
    """The hidden values between two products.  16-bit rows multiply codes with an offset of 16, sums of about 24 instead of 9 where the same
    rows in fp32 multiply the codes: errors 2.7 times those, four times allowed, relative to the results' size."""
    R, C = 512, 4096
    w = _rand((R, C), dtype, 1, 0.02)
    x = _rand((M, C), dtype, 2)
    pw = lib.w4_quantize(w, group)
    want = f64(x) @ orc.held_values(f64(w), group).T
    rms = lambda t: np.sqrt(np.mean(t ** 2))  # noqa: E731
    narrow, wide = (rms(f64(lib.w4_matvec(t, pw, out_dtype=F32)) - want) / rms(want) for t in (x, x.float()))
    print(f"group {group} {dtype} M {M}: error {narrow:.2e}, of the same rows in fp32 {wide:.2e}")
    assert wide <= 2.0 ** -20 and narrow <= 4 * wide


@pytest.mark.parametrize("M,R,C,group,act,dtype", [
    (8, 64, 6554, 64, "relu", F16), (8, 40, 6554, 128, "swiglu", BF16),       # an even number of core neurons
    (16, 40, 4098, 128, "none", BF16), (9, 33, 4102, 32, "relu", F16), (16, 17, 2054, 64, "none", F16),
    (2, 24, 20006, 64, "none", BF16), (1, 24, 33002, 128, "none", F16), (16, 14410, 2050, 64, "relu", BF16)])
def test_rows_read_as_they_are_that_end_inside_a_piece(lib, M, R, C, group, act, dtype):
    """16-bit rows past the LDS whose length is no multiple of the eight elements of a load: what follows a row, another one or the
    end of them all, is no part of it, NaN or not; rows that are not even are laid out instead."""
    _check(lib, M, R, C, group, act, dtype, seed=11)
    _check(lib, M, R, C - 1, group, act, dtype, seed=12)
    for gap in (2, 6, 8, 130):
        base = torch.full((M, C + gap), float("nan"), dtype=dtype, device=DEV)
        for first in (0, 2):
            x = base[:, first:first + C]
            x.copy_(_rand((M, C), dtype, 13))
            _check(lib, M, R, C, group, act, dtype, seed=13, x=x)
            base.fill_(float("nan"))
