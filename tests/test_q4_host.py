"""Host-side checks of the 4-bit operators' C ABI (no GPU): sizes and refusals, before any HIP call."""

import ctypes

import pytest

F = 0x10000      # an address that no call may touch


def _size(fn, *args):
    b = ctypes.c_size_t(0)
    return fn(*args, ctypes.byref(b)), b.value


def test_w4_sizes(lib):
    r = lib.raw
    # whole blocks of 16 rows and 128 columns, 1 KB of codes and 64 bytes a group
    assert _size(r.coreinfer_w4_size, 16, 128, 128) == (0, 1024 + 64)
    assert _size(r.coreinfer_w4_size, 17, 129, 32) == (0, 4 * (1024 + 256))
    for bad in ((0, 1, 32), (1, 0, 32), (1048577, 1, 32), (1, 1048577, 32)):
        assert _size(r.coreinfer_w4_size, *bad)[0] == lib.CI_ERR_INVALID_ARG
    assert _size(r.coreinfer_w4_size, 16, 16, 16)[0] == lib.CI_ERR_UNSUPPORTED
    assert r.coreinfer_w4_size(1, 1, 32, None) == lib.CI_ERR_INVALID_ARG
    assert _size(r.coreinfer_w4_matvec_workspace_size, 1, 9216, lib.CI_F16) == (0, 0)
    assert _size(r.coreinfer_w4_matvec_workspace_size, 64, 256, lib.CI_F32) == (0, 64 * 256 * 6)
    assert _size(r.coreinfer_w4_matvec_workspace_size, 65, 256, lib.CI_F32)[0] == lib.CI_ERR_INVALID_ARG
    assert _size(r.coreinfer_w4_matvec_workspace_size, 1, 256, 7)[0] == lib.CI_ERR_BAD_DTYPE


def test_w4_quantize_and_read_refuse(lib):
    r = lib.raw
    for fn, args in ((r.coreinfer_w4_quantize, lambda w=F, R=4, C=8, ld=8, dt=1, g=32, p=F: (w, R, C, ld, dt, g, p, None)),
                     (r.coreinfer_w4_read, lambda w=F, R=4, C=8, ld=8, dt=1, g=32, p=F: (p, R, C, g, w, ld, dt, None))):
        assert fn(*args(dt=3)) == lib.CI_ERR_BAD_DTYPE
        assert fn(*args(w=None)) == fn(*args(p=None)) == fn(*args(R=0)) == fn(*args(C=1 << 21)) == lib.CI_ERR_INVALID_ARG
        assert fn(*args(g=48)) == lib.CI_ERR_UNSUPPORTED
        assert fn(*args(ld=7)) == fn(*args(w=F + 1)) == fn(*args(p=F + 8)) == fn(*args(ld=1 << 41)) == lib.CI_ERR_BAD_LAYOUT


def _matvec(lib, x=F, M=1, ldx=64, xd=1, w=F, gate=None, bias=None, bd=1, act=2, R=32, C=64, g=32, y=F, ldy=32, yd=1, ws=F, wb=1 << 30):
    return lib.raw.coreinfer_w4_matvec(x, M, ldx, xd, w, gate, bias, bd, act, R, C, g, y, ldy, yd, ws, wb, None)


def test_w4_matvec_refuses(lib):
    for kw in (dict(xd=5), dict(yd=-1), dict(bias=F, bd=3), dict(act=3), dict(act=-1)):
        assert _matvec(lib, **kw) == lib.CI_ERR_BAD_DTYPE, kw
    for kw in (dict(x=None), dict(w=None), dict(y=None), dict(M=0), dict(M=65), dict(R=0), dict(C=0), dict(act=1), dict(gate=F),
               dict(act=0, gate=F), dict(act=1, gate=F, bias=F)):
        assert _matvec(lib, **kw) == lib.CI_ERR_INVALID_ARG, kw
    assert _matvec(lib, g=256) == lib.CI_ERR_UNSUPPORTED
    for kw in (dict(ldx=63), dict(ldy=31), dict(x=F + 1), dict(y=F + 1), dict(w=F + 8), dict(act=1, gate=F + 4), dict(bias=F + 1),
               dict(M=64, ws=F + 8)):
        assert _matvec(lib, **kw) == lib.CI_ERR_BAD_LAYOUT, kw
    for kw in (dict(M=64, ws=None), dict(M=64, wb=64 * 128 * 2 - 1), dict(M=8, C=9216, ldx=9216, ws=None)):
        assert _matvec(lib, **kw) == lib.CI_ERR_WORKSPACE, kw


def test_which_rows_need_a_workspace(lib):
    """None while the operands of up to 16 rows, filled up to 128 columns, fit 64 KB; one row of hidden values may be too long for that."""
    size = lambda M, C, dt: _size(lib.raw.coreinfer_w4_matvec_workspace_size, M, C, dt)  # noqa: E731
    for dt, e in ((lib.CI_F16, 2), (lib.CI_BF16, 2), (lib.CI_F32, 6)):
        for M in (1, 2, 3, 8, 16):
            most = 65536 // (e * M) // 128 * 128
            assert size(M, most, dt) == (0, 0)
            assert size(M, most + 1, dt) == (0, 16 * (most + 128) * e)
        assert size(17, 1, dt) == (0, 32 * 128 * e) and size(33, 129, dt) == (0, 64 * 256 * e)
    assert size(1, 10880, lib.CI_F32) == size(1, 32768, lib.CI_F16) == (0, 0)
    for kw in (dict(C=10881, xd=0), dict(C=32769, xd=1), dict(C=32769, xd=2)):
        assert _matvec(lib, ldx=kw["C"], ws=None, wb=0, **kw) == lib.CI_ERR_WORKSPACE, kw


def _cache(lib, **kw):
    f = dict(k=F, v=F, k_scale=F, v_scale=F, weight=F, pos=F, B=2, H=3, cap=64, D=128, group=64)
    f.update(kw)
    return ctypes.byref(lib.ci_kv4(*f.values()))


STRIDE = (ctypes.c_int64 * 3)(1024, 512, 128)


def _calls(lib):
    r = lib.raw
    return {
        "append": lambda c, S=1, k=F, v=F, st=STRIDE, dt=1, lens=F, start=None, nxt=None: r.coreinfer_kv4_append(
            c, k, v, S, st, dt, start, lens, nxt, None),
        "read": lambda c, lens=F, first=0, count=1, k=F, v=F, dt=1: r.coreinfer_kv4_read(c, lens, first, count, k, v, dt, None),
        "attend": lambda c, q=F, S=1, Hq=3, st=STRIDE, dt=1, scale=1.0, lens=F, max_len=64, out=F, lse=None, w=None, ws=F,
        wb=1 << 40: r.coreinfer_kv4_attend(c, q, S, Hq, st, dt, scale, lens, max_len, out, lse, w, ws, wb, None),
        "evict": lambda c, lens=F, nxt=F, max_len=64, budget=8, recent=2, w=F, p=F, lo=None, ws=F, wb=1 << 40:
        r.coreinfer_kv4_evict(c, lens, nxt, max_len, budget, recent, w, p, lo, ws, wb, None)}


@pytest.mark.parametrize("name", ["append", "read", "attend", "evict"])
def test_every_call_refuses_a_bad_cache(lib, name):
    call = _calls(lib)[name]
    assert call(None) == lib.CI_ERR_INVALID_ARG
    for kw in (dict(k=None), dict(v=None), dict(k_scale=None), dict(v_scale=None), dict(B=0), dict(H=0), dict(cap=0),
               dict(B=300, H=300), dict(cap=1 << 25)):
        assert call(_cache(lib, **kw)) == lib.CI_ERR_INVALID_ARG, kw
    for kw in (dict(cap=63), dict(k=F + 8), dict(v=F + 4), dict(k_scale=F + 4), dict(v_scale=F + 8), dict(weight=F + 2),
               dict(pos=F + 1)):
        assert call(_cache(lib, **kw)) == lib.CI_ERR_BAD_LAYOUT, kw
    for kw in (dict(D=96), dict(D=256), dict(group=16), dict(D=64, group=128)):
        assert call(_cache(lib, **kw)) == lib.CI_ERR_UNSUPPORTED, kw


def test_cache_calls_refuse_their_arguments(lib):
    c, call = _cache(lib), _calls(lib)
    bad_stride = (ctypes.c_int64 * 3)(-1, 512, 128)
    cases = {
        "append": [(dict(dt=9), "DTYPE"), (dict(k=None), "INVALID"), (dict(v=None), "INVALID"), (dict(lens=None), "INVALID"),
                   (dict(S=0), "INVALID"), (dict(S=(1 << 19) + 1), "INVALID"),
                   (dict(st=None), "INVALID"), (dict(st=bad_stride), "LAYOUT"), (dict(k=F + 1), "LAYOUT"),
                   (dict(start=F + 2), "LAYOUT"), (dict(nxt=F + 1), "LAYOUT"), (dict(lens=F + 1), "LAYOUT")],
        "read": [(dict(dt=-1), "DTYPE"), (dict(lens=None), "INVALID"), (dict(first=-1), "INVALID"), (dict(count=0), "INVALID"),
                 (dict(first=60, count=5), "INVALID"), (dict(count=65), "INVALID"), (dict(k=None), "INVALID"),
                 (dict(v=F + 8), "LAYOUT"), (dict(lens=F + 3), "LAYOUT")],
        "attend": [(dict(dt=3), "DTYPE"), (dict(q=None), "INVALID"), (dict(out=None), "INVALID"), (dict(lens=None), "INVALID"),
                   (dict(S=0), "INVALID"), (dict(Hq=2), "INVALID"), (dict(Hq=4), "INVALID"), (dict(max_len=0), "INVALID"),
                   (dict(max_len=65), "INVALID"), (dict(scale=0.0), "INVALID"), (dict(scale=-1.0), "INVALID"),
                   (dict(scale=float("nan")), "INVALID"), (dict(scale=float("inf")), "INVALID"), (dict(S=1 << 19, Hq=9), "INVALID"),
                   (dict(st=bad_stride), "LAYOUT"), (dict(out=F + 8), "LAYOUT"), (dict(lse=F + 2), "LAYOUT"), (dict(w=F + 2), "LAYOUT"),
                   (dict(ws=F + 8), "LAYOUT"), (dict(ws=None), "WORKSPACE"), (dict(wb=255), "WORKSPACE")],
        "evict": [(dict(lens=None), "INVALID"), (dict(nxt=None), "INVALID"), (dict(w=None), "INVALID"), (dict(p=None), "INVALID"),
                  (dict(max_len=0), "INVALID"), (dict(max_len=65), "INVALID"), (dict(budget=0), "INVALID"),
                  (dict(recent=9), "INVALID"), (dict(recent=-1), "INVALID"), (dict(lo=F + 1), "LAYOUT"), (dict(p=F + 2), "LAYOUT"),
                  (dict(ws=F + 4), "LAYOUT"), (dict(ws=None), "WORKSPACE"), (dict(wb=100), "WORKSPACE")]}
    status = {"DTYPE": lib.CI_ERR_BAD_DTYPE, "INVALID": lib.CI_ERR_INVALID_ARG, "LAYOUT": lib.CI_ERR_BAD_LAYOUT,
              "WORKSPACE": lib.CI_ERR_WORKSPACE}
    for name, todo in cases.items():
        for kw, want in todo:
            assert call[name](c, **kw) == status[want], (name, kw)
    bare = _cache(lib, weight=None)
    assert call["attend"](bare, w=F) == call["evict"](bare) == lib.CI_ERR_INVALID_ARG
    assert call["evict"](_cache(lib, pos=None)) == lib.CI_ERR_INVALID_ARG


def test_cache_sizes(lib):
    r = lib.raw
    a, b = ctypes.c_size_t(0), ctypes.c_size_t(0)
    assert r.coreinfer_kv4_sizes(2, 3, 64, 128, 32, ctypes.byref(a), ctypes.byref(b)) == 0
    assert (a.value, b.value) == (2 * 3 * 64 * 64, 2 * 3 * 64 * 4 * 4)
    assert r.coreinfer_kv4_sizes(2, 3, 65535, 128, 32, ctypes.byref(a), ctypes.byref(b)) == lib.CI_ERR_BAD_LAYOUT
    assert r.coreinfer_kv4_sizes(2, 3, 64, 128, 32, None, ctypes.byref(b)) == lib.CI_ERR_INVALID_ARG
    # one slot over the budget: a list of one move a head
    assert _size(r.coreinfer_kv4_evict_workspace_size, 1, 4, 1025, 1024) == (0, 3 * 256)
    assert _size(r.coreinfer_kv4_evict_workspace_size, 1, 4, 0, 8)[0] == lib.CI_ERR_INVALID_ARG
    for heads in (1, 8, 320):
        for S, G in ((1, 1), (1, 8), (16, 1), (17, 1), (512, 1), (100, 4)):
            last = 0
            for T in (1, 32, 33, 1000, 4096, 65536):
                for w in (0, 1):
                    rc, n = _size(r.coreinfer_kv4_attend_workspace_size, 1, heads, 128, S, heads * G, T, w)
                    assert rc == 0 and n >= 256
                    if w and S * G <= 16:
                        assert n >= heads * S * G * T * 4      # the logits
                    last = max(last, n)
            assert last < 1 << 34


def test_python_binding_refuses_what_the_kernels_would_misread(lib):
    import torch
    cache = lib.kv4_cache(1, 2, 32, 64, 32, device="cpu")
    k = torch.zeros(1, 3, 2, 64, dtype=torch.float16)
    n = torch.zeros(1, dtype=torch.int32)
    for bad in (dict(k=k[..., :32], v=k), dict(k=k, v=k.float()), dict(k=k, v=k, lens=n.long()),
                dict(k=k.transpose(2, 3), v=k.transpose(2, 3)), dict(k=k.expand(2, 3, 2, 64), v=k.expand(2, 3, 2, 64))):
        with pytest.raises(AssertionError):
            lib.kv4_append(cache, **{"lens": n, **bad})
    with pytest.raises(AssertionError):
        lib.kv4_attend(torch.zeros(1, 1, 2, 128, dtype=torch.float16), cache, n)
    with pytest.raises(AssertionError):
        lib.kv4_attend(k, cache, n, out=torch.zeros(1, 3, 2, 64))
    w = lib.W4(torch.zeros(lib.w4_size(16, 128, 64), dtype=torch.uint8), 16, 128, 64)
    with pytest.raises(AssertionError):
        lib.w4_matvec(torch.zeros(1, 127), w)
    with pytest.raises(AssertionError):
        lib.w4_matvec(torch.zeros(2, 128), w, y=torch.zeros(2, 15))
    with pytest.raises(AssertionError):
        lib.w4_quantize(torch.zeros(16, 128), 64, packed=torch.zeros(8, dtype=torch.uint8))
    with pytest.raises(lib.CoreInferError):
        lib.kv4_cache(1, 2, 33, 64, 32, device="cpu")


def test_the_per_token_calls_take_no_float_or_nothing_for_a_number(lib):
    """The bits of a float, or 0 for None, are none of the sizes and addresses: refused before the library is called, with the C module
    and through ctypes alike.  Every other argument is one that the library refuses by itself."""
    calls = [   # p an address or None, i an integer, f a float
        (lib._w4_matvec_call, "piiipppiiiiipiipip"), (lib._kv4_append_call, "pppiiiiipppp"), (lib._kv4_read_call, "ppiippip"),
        (lib._kv4_attend_call, "ppiiiiiifpippppip"), (lib._kv4_evict_call, "pppiiippppip")]
    for call, kinds in calls:
        good = [{"p": None, "i": 0, "f": 1.0}[k] for k in kinds]
        assert call(*good) == lib.CI_ERR_INVALID_ARG
        for i, kind in enumerate(kinds):
            for bad in {"p": (0.0, 1.5), "i": (0.0, 1.5, "1", None), "f": ("1", None)}[kind]:
                with pytest.raises((TypeError, ctypes.ArgumentError)):
                    call(*good[:i], bad, *good[i + 1:])
        with pytest.raises(TypeError):
            call(*good[:-1])


def test_no_kernel_is_built_that_no_call_launches(lib):
    """Four tiles of weights a workgroup go with rows of x in memory and with nothing else; rows move in the launch that plans them only with the
    keys in the LDS."""
    import re
    from paper_2410_18311_amd import build
    with open(build.LIB_PATH, "rb") as f:
        data = f.read()
    rows = set(re.findall(rb"gemm_q4_rows_kernelINS_\d\w+?ELi\d+ELi(\d)ELi(\d)ELb(\d)ELi(\d)ELi(\d+)ELi(\d)EE", data))
    assert {(t, x) for t, _, _, x, _, _ in rows} == {(b"1", b"0"), (b"2", b"0"), (b"4", b"0"), (b"1", b"1"), (b"2", b"1"), (b"2", b"2")}
    assert not {dual for t, _, dual, x, _, _ in rows if (t, x) == (b"2", b"0")} & {b"0"}      # pairs there are pairs of up and gate
    plans = set(re.findall(rb"kv4_plan_kernelILi(\d+)ELb(\d)ELi\d+ELi\d+ELb(\d)ELb(\d)EE", data))
    assert plans == {(b"256", b"1", b"1", b"1"), (b"1024", b"1", b"1", b"1"), (b"256", b"1", b"1", b"0"), (b"1024", b"1", b"1", b"0"),
                     (b"256", b"1", b"0", b"0"), (b"1024", b"1", b"0", b"0"), (b"1024", b"0", b"0", b"0")}


def test_attention_refuses_a_scale_that_overflows_in_base_2(lib):
    """Times log2(e), which is what multiplies the logits, it would be infinite, and a logit of 0 a NaN."""
    call, c = _calls(lib)["attend"], _cache(lib)
    for scale in (2.4e38, 3.4e38):
        assert call(c, scale=scale) == lib.CI_ERR_INVALID_ARG
    assert call(c, scale=2.3e38, ws=None) == lib.CI_ERR_WORKSPACE   # which is looked at after the scale
