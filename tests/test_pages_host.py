"""Host-side checks of rotary positions and of the cache in pages (no GPU): frequencies, sizes and refusals, before any HIP call."""

import ctypes
import math

import numpy as np
import pytest

from oracle import pages_oracle as orc

F = 0x10000      # an address that no call may touch
STRIDE = (ctypes.c_int64 * 2)(1024, 128)


# -------------------------------------------------------------------------------------------------- frequencies

def _turns(lib, rot, **kw):
    return lib.rope_turns(rot, **kw).numpy().view(np.uint64)


@pytest.mark.parametrize("rot", [2, 6, 16, 128, 512])
@pytest.mark.parametrize("kw", [dict(), dict(base=500000.0), dict(scaling="linear", factor=8.0), dict(scaling="base", factor=4.0),
                                dict(scaling="parts", factor=4.0, original=4096.0),
                                dict(scaling="parts", factor=8.0, original=8192.0, fast=4.0, slow=1.0), dict(base=0.5)])
def test_turns_are_the_frequencies(lib, rot, kw):
    want = orc.frequencies(rot, **kw) / (2 * math.pi)
    got = _turns(lib, rot, **kw).astype(np.float64) / 2.0 ** 64
    # pow, two products or quotients and the division by 2 pi: eight roundings of 2^-53 at most on either side
    assert np.all(np.abs(got - (want - np.floor(want))) <= 16 * 2.0 ** -53 * np.maximum(want, 2.0 ** -11))


def test_turns_refuse(lib):
    fn = lib.raw.coreinfer_rope_turns
    out = (ctypes.c_uint64 * 256)()
    call = lambda rot=8, base=1e4, sc=0, fa=2.0, orig=4096.0, fast=32.0, slow=1.0, o=out: fn(rot, base, sc, fa, orig, fast, slow, o)  # noqa: E731
    assert call() == call(sc=1) == call(sc=2) == call(sc=3) == call(fa=0.0) == lib.CI_OK
    assert call(sc=4) == call(sc=-1) == lib.CI_ERR_BAD_DTYPE
    nan, inf = math.nan, math.inf
    for kw in (dict(rot=0), dict(rot=7), dict(rot=514), dict(base=0.0), dict(base=nan), dict(base=inf), dict(base=-1.0), dict(o=None),
               dict(sc=1, fa=0.0), dict(sc=2, fa=nan), dict(sc=1, fa=inf), dict(sc=3, orig=0.0), dict(sc=3, orig=nan),
               dict(sc=3, fast=1.0), dict(sc=3, slow=nan), dict(sc=3, fast=inf), dict(sc=1, fa=1e-320)):
        assert call(**kw) == lib.CI_ERR_INVALID_ARG, kw


# ----------------------------------------------------------------------------------------------------- refusals

def _rope(lib, **kw):
    f = dict(turns=F, scale=1.0, rot=32, style=0)
    f.update(kw)
    return ctypes.byref(lib.ci_rope(*f.values()))


def _cache(lib, **kw):
    f = dict(k=F, v=F, table=F, pages=8, most=4, B=2, H=3, page=16, D=128, dtype=1)
    f.update(kw)
    return ctypes.byref(lib.ci_kvp(*f.values()))


def _strides(a, b):
    return (ctypes.c_int64 * 2)(a, b)


def _call_rope(lib, x=F, st=STRIDE, T=4, H=2, D=64, dt=1, norm=None, eps=1e-6, rope="one", pos=F, back=0, y=2 * F, yst=STRIDE):
    rope = _rope(lib) if rope == "one" else rope
    return lib.raw.coreinfer_rope(x, st, T, H, D, dt, norm, eps, rope, pos, back, y, yst, None)


def test_rope_refuses(lib):
    assert _call_rope(lib, dt=3) == _call_rope(lib, rope=_rope(lib, style=2)) == lib.CI_ERR_BAD_DTYPE
    for kw in (dict(x=None), dict(y=None), dict(st=None), dict(yst=None), dict(T=-1), dict(T=(1 << 20) + 1), dict(H=0), dict(H=65536),
               dict(D=0), dict(D=513), dict(pos=None), dict(rope=_rope(lib, rot=66)), dict(rope=_rope(lib, rot=-2)),
               dict(rope=_rope(lib, rot=31)), dict(rope=_rope(lib, scale=math.nan)), dict(rope=_rope(lib, scale=math.inf)),
               dict(rope=_rope(lib, turns=None)), dict(back=1, norm=F), dict(norm=F, eps=-1.0), dict(norm=F, eps=math.nan)):
        assert _call_rope(lib, **kw) == lib.CI_ERR_INVALID_ARG, kw
    for kw in (dict(x=F + 1), dict(y=F + 1), dict(norm=F + 1), dict(pos=F + 2), dict(st=_strides(-1, 64)), dict(yst=_strides(1 << 41, 64)),
               dict(rope=_rope(lib, turns=F + 4)), dict(y=F, yst=_strides(1024, 64))):
        assert _call_rope(lib, **kw) == lib.CI_ERR_BAD_LAYOUT, kw


def test_rope_refuses_results_that_overlap(lib):
    for T, H, yst in ((4, 2, (0, 64)), (4, 2, (128, 63)), (4, 2, (127, 64)), (4, 2, (64, 255)), (4, 1, (63, 0)), (1, 2, (0, 0))):
        assert _call_rope(lib, T=T, H=H, yst=_strides(*yst)) == lib.CI_ERR_BAD_LAYOUT, (T, H, yst)


def test_no_rows_is_nothing_to_do(lib):
    assert _call_rope(lib, T=0, x=None, y=None, pos=None) == lib.CI_OK
    assert _append(lib, T=0, k=None, v=None, first=None, lens=None) == lib.CI_OK
    assert _attend(lib, T=0, q=None, out=None, first=None, lens=None, ws=None) == lib.CI_OK
    assert _size(lib, T=0) == (lib.CI_OK, 0)


def _append(lib, cache="one", k=F, v=F, st=STRIDE, T=4, first=F, lens=F, pos=None, rope="one", kn=None, eps=1e-6, q=None, Hq=0, qst=None,
            qn=None, qo=None):
    cache = _cache(lib) if cache == "one" else cache
    rope = _rope(lib) if rope == "one" else rope
    return lib.raw.coreinfer_kvp_append(cache, k, v, st, T, first, lens, pos, rope, kn, eps, q, Hq, qst, qn, qo, None)


def _attend(lib, cache="one", q=F, Hq=6, st=STRIDE, T=4, first=F, lens=F, rows=4, max_len=64, window=0, sinks=0, scale=1.0, out=F,
            lse=None, ws=F, wb=1 << 40):
    cache = _cache(lib) if cache == "one" else cache
    return lib.raw.coreinfer_kvp_attend(cache, q, Hq, st, T, first, lens, rows, max_len, window, sinks, scale, out, lse, ws, wb, None)


def _size(lib, cache="one", T=4, Hq=6, rows=4, max_len=64, window=0, sinks=0, null=False):
    cache = _cache(lib) if cache == "one" else cache
    b = ctypes.c_size_t(0)
    return lib.raw.coreinfer_kvp_attend_workspace_size(cache, T, Hq, rows, max_len, window, sinks,
                                                       None if null else ctypes.byref(b)), b.value


@pytest.mark.parametrize("name", ["append", "attend", "size"])
def test_every_call_refuses_a_bad_cache(lib, name):
    call = {"append": lambda c: _append(lib, c), "attend": lambda c: _attend(lib, c), "size": lambda c: _size(lib, c)[0]}[name]
    assert call(None) == lib.CI_ERR_INVALID_ARG
    for kw in (dict(k=None), dict(v=None), dict(table=None), dict(pages=0), dict(pages=1 << 31), dict(most=0), dict(most=1 << 21),
               dict(B=0), dict(H=0), dict(B=300, H=300), dict(B=1 << 40)):
        assert call(_cache(lib, **kw)) == lib.CI_ERR_INVALID_ARG, kw
    assert call(_cache(lib, dtype=3)) == lib.CI_ERR_BAD_DTYPE
    for kw in (dict(D=96), dict(D=256), dict(page=8), dict(page=48), dict(page=512), dict(page=-16)):
        assert call(_cache(lib, **kw)) == lib.CI_ERR_UNSUPPORTED, kw
    if name != "size":
        for kw in (dict(k=F + 8), dict(v=F + 4), dict(table=F + 2)):
            assert call(_cache(lib, **kw)) == lib.CI_ERR_BAD_LAYOUT, kw


def test_workspaces_stay_small_however_many_sentences(lib):
    """Partial results are a few thousand tiles' at most: 128 MiB and some for B = 1, not that for each sentence."""
    for dtype in (lib.CI_F16, lib.CI_F32):
        for B in (1, 7, 100, 1000, 8000):
            for T, rows in ((B, 1), (B + 500, 500), (1 << 16, 1 << 16)):
                for most in (4, 1 << 12, 1 << 18):
                    cache = _cache(lib, B=B, H=8, D=128, page=64, most=most, dtype=dtype)
                    rc, n = _size(lib, cache, T, 16, min(rows, T), most * 64)
                    assert rc == 0 and n <= 300 << 20, (B, T, rows, most, n)


def test_append_refuses(lib):
    q = dict(q=F, Hq=2, qst=STRIDE, qo=2 * F)
    assert _append(lib, rope=_rope(lib, style=5)) == lib.CI_ERR_BAD_DTYPE
    for kw in (dict(k=None), dict(v=None), dict(st=None), dict(first=None), dict(lens=None), dict(T=-1), dict(T=1 << 21),
               dict(rope=_rope(lib, rot=130)), dict(kn=F, eps=-1.0), {**q, "qn": F, "eps": math.inf}, {**q, "Hq": 0}, {**q, "q": None},
               {**q, "qo": None}, {**q, "qst": None}, {**q, "Hq": -1}, {**q, "Hq": 65536}, dict(qn=F)):
        assert _append(lib, **kw) == lib.CI_ERR_INVALID_ARG, kw
    for kw in (dict(k=F + 1), dict(v=F + 1), dict(kn=F + 1), dict(first=F + 1), dict(lens=F + 2), dict(pos=F + 2), dict(st=_strides(8, -8)),
               {**q, "q": F + 1}, {**q, "qo": F + 8}, {**q, "qn": F + 1}, {**q, "qst": _strides(1 << 41, 0)}):
        assert _append(lib, **kw) == lib.CI_ERR_BAD_LAYOUT, kw


def test_attend_refuses(lib):
    for kw in (dict(q=None), dict(st=None), dict(first=None), dict(lens=None), dict(out=None), dict(Hq=4), dict(Hq=0), dict(Hq=3 * 4097),
               dict(T=1 << 21), dict(rows=0), dict(max_len=0), dict(max_len=65), dict(window=-1), dict(sinks=-1), dict(scale=0.0),
               dict(scale=-1.0), dict(scale=math.nan), dict(scale=3e38), dict(T=1 << 20, Hq=1026)):
        assert _attend(lib, **kw) == lib.CI_ERR_INVALID_ARG, kw
    for kw in (dict(q=F + 1), dict(out=F + 8), dict(first=F + 2), dict(lens=F + 1), dict(lse=F + 2), dict(st=_strides(-8, 8))):
        assert _attend(lib, **kw) == lib.CI_ERR_BAD_LAYOUT, kw
    long = dict(cache=_cache(lib, most=1024), max_len=16384)
    need = _size(lib, **long)[1]
    assert need > 0
    assert _attend(lib, ws=None, **long) == _attend(lib, wb=need - 1, **long) == lib.CI_ERR_WORKSPACE
    assert _attend(lib, ws=F + 8, **long) == lib.CI_ERR_BAD_LAYOUT
    assert _size(lib, null=True)[0] == lib.CI_ERR_INVALID_ARG


def test_binding_refuses_what_does_not_fit(lib):
    import torch
    table = torch.zeros((2, 4), dtype=torch.int32)
    cache = lib.kvp_cache(8, 3, 16, 64, torch.float16, table)
    first, lens = torch.zeros(3, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    x = torch.zeros((4, 3, 64), dtype=torch.float16)
    for bad in (lambda: lib.kvp_append(cache, x, x.float(), first, lens), lambda: lib.kvp_append(cache, x[:, :2], x[:, :2], first, lens),
                lambda: lib.kvp_append(cache, x, x, lens, lens), lambda: lib.kvp_append(cache, x, x, first, first),
                lambda: lib.kvp_append(cache, x, x, first.long(), lens), lambda: lib.kvp_append(cache, x, x, first, lens, q_norm=x[0, 0]),
                lambda: lib.kvp_append(cache, x, x, first, lens, k_norm=x[0]), lambda: lib.kvp_append(cache, x, x, first, lens, pos=first),
                lambda: lib.kvp_attend(x.float(), cache, first, lens), lambda: lib.kvp_attend(x, cache, first, lens, out=x[:3]),
                lambda: lib.kvp_attend(x, cache, first, lens, lse=x), lambda: lib.rope(x, first, None),
                lambda: lib.rope(x, None, None, norm=x[0, 0].float()), lambda: lib.rope(x.transpose(1, 2), None, None),
                lambda: lib.KvpCache(cache.k, cache.v[:4], table), lambda: lib.KvpCache(cache.k, cache.v, table.long())):
        with pytest.raises(AssertionError):
            bad()
