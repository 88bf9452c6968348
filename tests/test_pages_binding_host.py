"""What the Python calls of rotary positions and the cache in pages refuse by themselves, without a GPU.  No call here may reach a launch."""

import ctypes
import importlib.util
import math

import pytest
import torch

F16, F32, I32 = torch.float16, torch.float32, torch.int32


def _host(lib, T=4):
    cache = lib.kvp_cache(8, 3, 16, 64, F16, torch.zeros((2, 4), dtype=I32))
    x = torch.zeros((T, 3, 64), dtype=F16)
    return cache, x, torch.zeros(3, dtype=I32), torch.zeros(2, dtype=I32), torch.zeros(T, dtype=I32)


@pytest.mark.parametrize("T", [0, 4])
def test_calls_on_host_memory_are_refused(lib, T):
    """All of a call's tensors are in host memory: they agree, and a kernel would read the host's addresses."""
    cache, x, first, lens, pos = _host(lib, T)
    angles = lib.rope_angles(64, device="cpu")
    norm = torch.ones(64, dtype=F16)
    for call in (lambda: lib.rope(x, pos, angles), lambda: lib.rope(x, None, None, norm=norm), lambda: lib.rope(x, pos, angles, out=x),
                 lambda: lib.kvp_append(cache, x, x, first, lens), lambda: lib.kvp_append(cache, x, x, first, lens, angles, pos, norm, q=x, q_norm=norm),
                 lambda: lib.kvp_attend(x, cache, first, lens), lambda: lib.kvp_attend(x, cache, first, lens, lse=torch.zeros(T, 3))):
        with pytest.raises(AssertionError, match="host memory"):
            call()


def test_other_refusals_come_before_that_one(lib):
    cache, x, first, lens, pos = _host(lib)
    for bad in (lambda: lib.kvp_append(cache, x, x.float(), first, lens), lambda: lib.kvp_append(cache, x[:, :2], x[:, :2], first, lens),
                lambda: lib.kvp_append(cache, x, x, lens, lens), lambda: lib.kvp_append(cache, x, x, first, first),
                lambda: lib.kvp_append(cache, x, x, first.long(), lens), lambda: lib.kvp_append(cache, x, x, first, lens, q_norm=x[0, 0]),
                lambda: lib.kvp_append(cache, x, x, first, lens, k_norm=x[0]), lambda: lib.kvp_append(cache, x, x, first, lens, pos=first),
                lambda: lib.kvp_attend(x.float(), cache, first, lens), lambda: lib.kvp_attend(x, cache, first, lens, out=x[:3]),
                lambda: lib.kvp_attend(x, cache, first, lens, lse=x), lambda: lib.rope(x, first, None),
                lambda: lib.rope(x, None, None, norm=x[0, 0].float()), lambda: lib.rope(x.transpose(1, 2), None, None)):
        with pytest.raises(AssertionError) as e:
            bad()
        assert "host memory" not in str(e.value)


def test_angles_of_another_size_or_type_are_refused(lib):
    """A kernel reads rot / 2 of them."""
    turns = lib.rope_turns(64)
    lib.RopeAngles(turns, 1.0, 64, "half")
    lib.RopeAngles(turns[:0], 1.0, 0, "half")
    for bad, rot in ((turns[:31], 64), (turns, 66), (turns, 62), (turns.int(), 64), (turns.double(), 64), (turns.reshape(1, 32), 64),
                     (lib.rope_turns(128)[::2], 64), (turns, 65), (turns[:0], -2), (turns[:1].expand(32), 64)):
        with pytest.raises(AssertionError):
            lib.RopeAngles(bad, 1.0, rot, "half")


def test_tensors_whose_addresses_calls_go_by_are_not_replaced(lib):
    cache, angles = _host(lib)[0], lib.rope_angles(64, device="cpu")
    for owner, name in ((cache, "k"), (cache, "v"), (cache, "table"), (angles, "turns")):
        was = getattr(owner, name)
        with pytest.raises(AttributeError):
            setattr(owner, name, was.clone())
        assert getattr(owner, name) is was
        was.zero_()      # written to they may be


@pytest.mark.parametrize("stride", [(384, 128), (128, 512), (1024, 128)])
def test_results_over_the_rows_that_they_come_from_are_refused(lib, stride):
    """Addresses that no call may touch: each is refused for the overlap alone, which other distances show (on the GPU, where they run)."""
    F, T, H, D = 1 << 20, 4, 3, 128
    strides = (ctypes.c_int64 * 2)(*stride)
    last = (T - 1) * stride[0] + (H - 1) * stride[1] + D      # elements
    size = T * H * D
    cache = ctypes.byref(lib.ci_kvp(F, F, F, 8, 4, 2, 3, 16, D, 1))
    rope = ctypes.byref(lib.ci_rope(F, 1.0, 64, 0))
    block = (ctypes.c_int64 * 2)(H * D, D)
    for away in (0, 8, -8, D, last - 8, 8 - size):      # out from q on; 16-byte aligned
        q = 4 * F
        out = q + 2 * away
        assert lib.raw.coreinfer_kvp_attend(cache, q, H, strides, T, F, F, 4, 64, 0, 0, 1.0, out, None, F, 1 << 40, None) == lib.CI_ERR_BAD_LAYOUT
        assert lib.raw.coreinfer_kvp_append(cache, F, F, block, T, F, F, None, None, None, 0.0, q, H, strides, None, out, None) == lib.CI_ERR_BAD_LAYOUT
        if away or stride[0] < stride[1]:      # in place it may be, with the same strides
            assert lib.raw.coreinfer_rope(q, strides, T, H, D, 1, None, 0.0, rope, F, 0, out, block, None) == lib.CI_ERR_BAD_LAYOUT
            assert lib.raw.coreinfer_rope(out, block, T, H, D, 1, None, 0.0, rope, F, 0, q, strides, None) == lib.CI_ERR_BAD_LAYOUT
    for away in (1, -1, 127, stride[0] - 127, stride[0] + stride[1] + 5, last - 1, 1 - last):
        assert lib.raw.coreinfer_rope(4 * F, strides, T, H, D, 1, None, 0.0, rope, F, 0, 4 * F + 2 * away, strides, None) == lib.CI_ERR_BAD_LAYOUT


@pytest.mark.parametrize("factor,scale", [(4.0, 0.1 * math.log(4.0) + 1.0), (1.0, 1.0), (0.5, 1.0), (1e-6, 1.0)])
def test_the_scale_of_parts_is_that_of_longer_contexts(lib, factor, scale):
    """A factor of 1e-6 would make it -0.38, and turn the heads over."""
    kw = dict(scaling="parts", factor=factor, original=4096.0, device="cpu")
    assert lib.rope_angles(64, **kw).scale == scale
    assert lib.rope_angles(64, scale=0.75, **kw).scale == 0.75


def test_a_workspace_with_fewer_bytes_than_elements_is_refused(lib):
    """An expanded tensor has one element's memory."""
    cache, x, first, lens, _ = _host(lib)
    for ws in (torch.empty(1, dtype=torch.uint8).expand(1 << 20), torch.empty(1 << 21, dtype=torch.uint8)[::2]):
        with pytest.raises(AssertionError) as e:
            lib.kvp_attend(x, cache, first, lens, ws=ws)
        assert "host memory" not in str(e.value)


@pytest.fixture(scope="module")
def plain(lib):
    """The module as it is where the C module was not built."""
    from paper_2410_18311_amd import build
    was, build.BINDING_PATH = build.BINDING_PATH, "/nonexistent"
    try:
        spec = importlib.util.spec_from_file_location("paper_2410_18311_amd.coreinfer_plain", lib.__file__)
        module = importlib.util.module_from_spec(spec)
        spec.loader.exec_module(module)
    finally:
        build.BINDING_PATH = was
    assert module._binding is None
    return module


def test_calls_through_ctypes_say_the_same(lib, plain):
    """Every argument in its place: no rows are nothing to do, and each refusal is the C module's."""
    F = 1 << 20
    angles, cache = lib.ci_rope(F, 1.0, 64, 0), lib.ci_kvp(F, F, F, 8, 1024, 2, 3, 16, 128, 1)
    r, c = ctypes.addressof(angles), ctypes.addressof(cache)
    rope = [F, 384, 128, 4, 3, 128, 1, None, 1e-6, r, F, 0, 4 * F, 384, 128, None]
    append = [c, F, F, 384, 128, 4, F, F, None, r, None, 1e-6, F, 3, 384, 128, None, 4 * F, None]
    attend = [c, F, 6, 768, 128, 4, F, F, 4, 16384, 0, 0, 1.0, 4 * F, None, F, 1 << 40, None]
    ok, size, layout = lib.CI_OK, lib.CI_ERR_INVALID_ARG, lib.CI_ERR_BAD_LAYOUT
    for name, args, T, changes in (
            ("_rope_call", rope, 3, {0: (F + 1, layout), 1: (-1, layout), 2: (-1, layout), 4: (0, size), 5: (0, size), 6: (7, lib.CI_ERR_BAD_DTYPE),
                                     7: (F + 1, layout), 9: (ctypes.addressof(lib.ci_rope(F, 1.0, 63, 0)), size), 10: (None, size), 12: (F + 2, layout),
                                     13: (0, layout), 14: (0, layout)}),
            ("_kvp_append_call", append, 5, {0: (None, size), 1: (F + 1, layout), 2: (None, size), 3: (-1, layout), 4: (-1, layout), 6: (None, size),
                                             7: (F + 1, layout), 8: (F + 1, layout), 10: (F + 1, layout), 12: (None, size), 13: (-1, size),
                                             14: (-1, layout), 15: (-1, layout), 16: (F + 1, layout), 17: (F, layout)}),
            ("_kvp_attend_call", attend, 5, {0: (None, size), 1: (F + 1, layout), 2: (5, size), 3: (-1, layout), 4: (-1, layout), 6: (F + 1, layout),
                                             7: (None, size), 8: (0, size), 9: (0, size), 10: (-1, size), 11: (-1, size), 12: (math.nan, size),
                                             13: (F, layout), 14: (F + 1, layout), 15: (None, lib.CI_ERR_WORKSPACE),
                                             16: (0, lib.CI_ERR_WORKSPACE)})):
        for at, (value, status) in {**changes, T: (0, ok)}.items():
            call = args[:at] + [value] + args[at + 1:]
            assert getattr(lib, name)(*call) == getattr(plain, name)(*call) == status, (name, at)
