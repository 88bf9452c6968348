"""The cache in pages on the GPU against the plain definitions in 64 bits: writes exactly (but for the rotation's rounding),
attention within the rounding of its sums."""

import math

import numpy as np
import pytest
import torch

from oracle import pages_oracle as orc
from tests._util import f64

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F16, BF16, F32 = torch.float16, torch.bfloat16, torch.float32
HALF = {F32: 2.0 ** -24, F16: 2.0 ** -11, BF16: 2.0 ** -8}
TINY = {F32: 2.0 ** -150, F16: 2.0 ** -25, BF16: 2.0 ** -134}
FEW = 64   # rows of a head of the cache up to which probabilities enter in two pieces (16 where contexts are long)


def _rand(shape, dtype, seed, std=1.0):
    g = torch.Generator(device="cpu")
    g.manual_seed(seed)
    return (torch.randn(*shape, generator=g) * std).to(dtype).to(DEV)


def _ints(*v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def _first(rows):
    return [sum(rows[:i]) for i in range(len(rows) + 1)]


def _cache(lib, H, page, D, dtype, lens, seed=0, spare=3, ahead=1):
    """A cache whose pages are given out in no order, NaN wherever no sentence has a slot in use."""
    have = [-(-max(n, 0) // page) for n in lens]
    most, pages = max(have) + ahead, sum(have) + spare
    order = np.random.default_rng(seed).permutation(pages)
    table = np.full((len(lens), most), -1, dtype=np.int32)
    at = 0
    for b, n in enumerate(have):
        table[b, :n] = order[at:at + n]
        at += n
    cache = lib.kvp_cache(pages, H, page, D, dtype, torch.from_numpy(table).to(DEV))
    cache.k.fill_(math.nan)
    cache.v.fill_(math.nan)
    return cache, table


def _fill(cache, table, lens, seed):
    """Random keys and values in the slots in use, keys with a few larger channels."""
    page = cache.page
    for b, n in enumerate(lens):
        k, v = (_rand((max(n, 0), cache.H, cache.D), cache.dtype, seed + 2 * b + i) for i in (0, 1))
        if n > 0:
            k[..., 3] *= 3.0
        for i in range(-(-max(n, 0) // page)):
            g, t = table[b][i], min(page, n - i * page)
            cache.k[g, :, :t] = k[i * page:i * page + t].transpose(0, 1)
            cache.v[g, :, :t] = v[i * page:i * page + t].transpose(0, 1)


# -------------------------------------------------------------------------------------------------------- writing

def _append(lib, lens, rows, H, G, D, page, dtype, rot=0, style="half", norm=False, pos=None, seed=0, odd=0, tail=0, table_edit=None):
    """Appends and compares with the definition: queries, what is in the pages, and that nothing else changed."""
    cache, table = _cache(lib, H, page, D, dtype, lens, seed)
    if table_edit:
        table_edit(table)
        cache.table.copy_(torch.from_numpy(table))
    _fill(cache, table, [n - m for n, m in zip(lens, rows)], seed + 100)
    cache.k.nan_to_num_(nan=3.0)      # what lies there otherwise is compared too
    cache.v.nan_to_num_(nan=-3.0)
    before = [f64(cache.k).copy(), f64(cache.v).copy()]
    first = _first(rows)
    T = first[-1] + tail
    fused = _rand((T, (G + 2) * H * D + odd), dtype, seed + 7)
    q, k, v = (fused[:, odd + a * H * D:odd + b * H * D].unflatten(-1, (-1, D)) for a, b in ((0, G), (G, G + 1), (G + 1, G + 2)))
    wq, wk = ((1.0 + _rand((D,), F32, seed + i, 0.3)).to(dtype) if norm else None for i in (11, 12))
    angles = lib.rope_angles(rot, style=style, device=DEV) if rot else None
    q_out = torch.full((T, G * H, D), 5.0, dtype=dtype, device=DEV)
    got = lib.kvp_append(cache, k, v, _ints(*first), _ints(*lens), angles, None if pos is None else _ints(*pos), k_norm=wk, q=q, q_norm=wq,
                         q_out=q_out)
    assert got is q_out
    where = list(orc.slots(first, lens))
    at = np.zeros(T) if pos is None else np.asarray(pos, dtype=np.float64)
    if pos is None:
        for r, _, t in where:
            at[r] = t
    f = orc.frequencies(rot) if rot else ()
    turned = {}
    for name, x, w in (("q", q, wq), ("k", k, wk)):
        n = orc.rope(f64(x), at, norm=None if w is None else f64(w), eps=1e-6)
        turned[name] = (orc.rope(f64(x), at, f, style, 1.0, None if w is None else f64(w), 1e-6),
                        np.abs(n).max(-1, keepdims=True) * math.sqrt(2.0) * 2.0 ** -24 * (25.0 if norm else 9.0) * (1.0 if rot or norm else 0.0))
    want_q, slack_q = turned["q"]
    want_k, slack_k = before[0].copy(), np.zeros(before[0].shape)
    want_v = before[1].copy()
    for r, b, t in where:
        if 0 <= t < table.shape[1] * page and 0 <= table[b][t // page] < cache.pages:
            g, i = table[b][t // page], t % page
            want_k[g, :, i], want_v[g, :, i] = turned["k"][0][r], f64(v[r])
            slack_k[g, :, i] = turned["k"][1][r]
    for have, want, slack in ((cache.k, want_k, slack_k), (cache.v, want_v, 0.0)):
        h = f64(have)
        assert np.all(np.abs(h - want) <= (slack > 0) * (HALF[dtype] * np.abs(want) + TINY[dtype]) + slack)
    mine = np.array([r for r, _, _ in where], dtype=int)
    h = f64(q_out)
    assert np.all(np.abs(h - want_q)[mine] <= (slack_q > 0)[mine] * (HALF[dtype] * np.abs(want_q) + TINY[dtype])[mine] + slack_q[mine])
    rest = np.setdiff1d(np.arange(T), mine)
    assert np.all(h[rest] == 5.0)
    return cache


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("D,rot,style,norm", [(128, 128, "half", False), (64, 32, "interleaved", True), (128, 0, "half", True),
                                              (64, 64, "half", False), (128, 12, "interleaved", True), (64, 0, "half", False)])
@pytest.mark.parametrize("page", [16, 64, 256])
def test_append_of_ragged_sentences(lib, page, D, rot, style, norm, dtype):
    _append(lib, [33, 5, 0, 300, 1], [3, 5, 0, 40, 1], 3, 2, D, page, dtype, rot, style, norm, seed=page + D, tail=2)


@pytest.mark.parametrize("B", [1, 63, 64, 65, 130, 4100])
def test_append_one_token_each(lib, B):
    lens = [1 + (7 * b) % 40 for b in range(B)]
    _append(lib, lens, [0 if b % 5 == 2 else 1 for b in range(B)], 1, 1, 64, 16, F16, 64, seed=B)


def test_append_of_many_tokens(lib):
    for page in (16, 128):
        _append(lib, [700, 1, 900], [650, 1, 901 - 1], 5, 3, 64, page, BF16, 64, norm=True, seed=3, tail=5)


def test_append_positions_of_its_own(lib):
    _append(lib, [20, 8], [4, 3], 2, 4, 128, 16, F32, 128, pos=[5, 900, -3, 1 << 20, 0, 7, 70000], seed=4)


def test_append_of_misaligned_slices(lib):
    for dtype, odd in ((F16, 1), (BF16, 8), (F32, 3)):
        _append(lib, [20, 33], [20, 2], 2, 2, 64, 32, dtype, 64, norm=True, seed=5, odd=odd)


def test_append_keeps_to_its_pages(lib):
    """Slots without a page, pages outside the pool, more new tokens than slots, lengths past the table and below zero."""
    def edit(table):
        table[0][1] = -1
        table[1][0] = 10 ** 6
        table[2][0] = -2 ** 31
    _append(lib, [40, 5, 3, 20], [30, 5, 3, 2], 2, 1, 64, 16, F16, 64, seed=6, table_edit=edit)
    cache, table = _cache(lib, 2, 16, 64, F16, [16, 16, 16], spare=2, ahead=0)
    cache.k.fill_(1.0)
    cache.v.fill_(2.0)
    x = _rand((12, 2, 64), F16, 1)
    # two of four tokens past the table; two ahead of slot 0; far outside on both sides
    lib.kvp_append(cache, x, x, _ints(0, 4, 8, 12), _ints(18, 2, 2 ** 31 - 1))
    k = cache.k.clone()
    for b, t, r in ((0, 14, 0), (0, 15, 1), (1, 0, 6), (1, 1, 7)):
        assert torch.equal(k[table[b][0], :, t], x[r])
        k[table[b][0], :, t] = 1.0
    assert bool((k == 1.0).all())
    before = cache.k.clone()
    lib.kvp_append(cache, x, x, _ints(0, 4, 8, 12), _ints(-2 ** 31, -5, 0))
    assert torch.equal(cache.k, before)


def test_append_takes_what_first_says_only(lib):
    """Beginnings that fall, lie outside the rows or are equal: rows of no sentence are not written, nothing else is touched."""
    for first in ([0, 9, 4, 12], [-5, 3, 3, 99], [6, 6, 6, 6], [12, 0, 0, 0], [2 ** 31 - 1, -2 ** 31, 5, 7]):
        cache, table = _cache(lib, 1, 16, 64, F16, [32, 32, 32])
        cache.k.fill_(1.0)
        x = _rand((12, 1, 64), F16, 2)
        lib.kvp_append(cache, x, x, _ints(*first), _ints(20, 20, 20))
        known = {tuple(r.tolist()) for r in x[:, 0].cpu()}
        rows = cache.k.reshape(-1, 64).cpu()
        assert all(tuple(r.tolist()) in known for r in rows[(rows != 1.0).any(-1)])


def test_append_without_queries_and_without_rotation_copies(lib):
    cache, table = _cache(lib, 2, 16, 128, BF16, [7])
    k, v = _rand((7, 2, 128), BF16, 1), _rand((7, 2, 128), BF16, 2)
    k[3, 1, 5], v[2, 0, 9], v[4, 1, 0] = math.nan, math.inf, math.nan
    assert lib.kvp_append(cache, k, v, _ints(0, 7), _ints(7)) is None
    for have, want in ((cache.k, k), (cache.v, v)):
        assert torch.equal(have[table[0][0], :, :7].transpose(0, 1).contiguous().view(torch.int16), want.view(torch.int16))


def test_append_of_one_token_whose_values_lie_elsewhere(lib):
    """Strides of lengths of one are not compared."""
    cache, table = _cache(lib, 2, 16, 64, F16, [5])
    k, v = _rand((1, 2, 64), F16, 1), _rand((1, 6, 64), F16, 2)[:, 4:]
    lib.kvp_append(cache, k, v, _ints(0, 1), _ints(5))
    assert torch.equal(cache.k[table[0][0], :, 4], k[0]) and torch.equal(cache.v[table[0][0], :, 4], v[0])
    with pytest.raises(AssertionError):
        lib.kvp_append(cache, k.expand(2, 2, 64), v.expand(2, 2, 64).contiguous(), _ints(0, 2), _ints(5))


def test_slots_far_into_a_large_pool(lib):
    """Offsets past 2^31 elements."""
    H, page, D = 8, 256, 128
    pages = (1 << 31) // (H * page * D) + 40
    table = _ints(pages - 1, 0, pages - 2, 5).reshape(2, 2)
    cache = lib.kvp_cache(pages, H, page, D, BF16, table)
    lens = [300, 270]
    for b, n in enumerate(lens):
        for i in range(2):
            cache.k[table[b, i]] = _rand((H, page, D), BF16, 10 * b + i)
            cache.v[table[b, i]] = _rand((H, page, D), BF16, 10 * b + i + 5)
    x = _rand((20, H, D), BF16, 3)
    rows = [15, 5]
    lib.kvp_append(cache, x, x, _ints(*_first(rows)), _ints(*lens))
    assert torch.equal(cache.k[0, :, 29:44].transpose(0, 1), x[:15]) and torch.equal(cache.k[5, :, 9:14].transpose(0, 1), x[15:])
    small = lib.kvp_cache(4, H, page, D, BF16, _ints(0, 1, 2, 3).reshape(2, 2))
    for i, g in enumerate(table.flatten().tolist()):
        small.k[i], small.v[i] = cache.k[g], cache.v[g]
    q = _rand((20, H * 2, D), BF16, 4)
    for rows in ([15, 5], [1, 1]):
        args = (_ints(*_first(rows)), _ints(*lens))
        assert torch.equal(lib.kvp_attend(q[:sum(rows)], cache, *args), lib.kvp_attend(q[:sum(rows)], small, *args))


# ------------------------------------------------------------------------------------------------------ attention

def _bound(dtype, want, size, reach, D, n, rows_share):
    """Half a unit of the result; of the sum of p |v|: a logit's D products and sums in fp32 (relative to the terms' size) and its scale, exponential and
    maximum, four roundings of a number up to 2^8 in the exponent; the probabilities' own form (two pieces, or one
    rounding in prompts: PIECE); sums of n / 4 terms and the join's."""
    piece = {F32: 0.0, F16: 2.0 ** -21, BF16: 2.0 ** -15}[dtype] if rows_share <= FEW else HALF[dtype]
    rel = 2.0 ** -24 * ((D + 8) * reach[..., None] + 16.0 + n / 4.0 + 80.0) + piece
    return HALF[dtype] * np.abs(want) + TINY[dtype] + 2.0 * rel * size





def _check_attend(lib, lens, rows, H, G, D, page, dtype, window=0, sinks=0, seed=0, qstd=1.0, max_rows=None, max_len=None, tail=0,
                  table_edit=None, edit=None, odd=0, scale=None, share=None, ahead=1):
    cache, table = _cache(lib, H, page, D, dtype, lens, seed, ahead=ahead)
    _fill(cache, table, lens, seed + 50)
    if table_edit:
        table_edit(table)
        cache.table.copy_(torch.from_numpy(table))
    if edit:
        edit(cache, table)
    first = _first(rows)
    T = first[-1] + tail
    q = _rand((T, G * H * D + odd), dtype, seed + 9, qstd)[:, odd:].unflatten(-1, (-1, D))
    out = torch.full((T, G * H, D), 5.0, dtype=dtype, device=DEV)
    lse = torch.full((T, G * H), 5.0, dtype=F32, device=DEV)
    args = dict(max_rows=max_rows or max(max(rows), 1), max_len=max_len or max(max(lens), 1), window=window, sinks=sinks, scale=scale)
    lib.kvp_attend(q, cache, _ints(*first), _ints(*lens), out=out, lse=lse, **args)
    seen = [min(max(n, 0), args["max_len"]) for n in lens]
    k, v = f64(cache.k), f64(cache.v)
    want, want_lse, size, reach = orc.attend(f64(q), k, v, table, first, seen, window, sinks, D ** -0.5 if scale is None else scale)
    got, got_lse = f64(out), f64(lse)
    mine = ~np.isnan(want_lse)
    assert np.all(got[~mine] == 5.0) and np.all(got_lse[~mine] == 5.0)
    share = share or max(rows) * G
    ok = np.abs(got - want)[mine] <= _bound(dtype, want, size, reach, D, max(seen), share)[mine]
    assert ok.all(), (np.abs(got - want)[mine] / _bound(dtype, want, size, reach, D, max(seen), share)[mine]).max()
    none = mine & np.isneginf(want_lse)
    assert np.all(got[none] == 0.0) and np.all(np.isneginf(got_lse[none]))
    some = mine & np.isfinite(want_lse)
    err = np.abs(got_lse[some] - want_lse[some])
    assert np.all(err <= 2.0 ** -24 * ((D + 8) * reach[some] + 32.0 + max(seen) / 4.0 + np.abs(want_lse[some]) * 4.0))
    return cache, table, q, out, args


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("D,page", [(64, 16), (64, 64), (128, 16), (128, 32), (128, 256)])
@pytest.mark.parametrize("n", [1, 2, 15, 16, 17, 31, 32, 33, 77, 300])
def test_one_token(lib, n, D, page, dtype):
    _check_attend(lib, [n], [1], 3, 1, D, page, dtype, seed=n)


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("G", [1, 3, 8, 16, 40])
def test_heads_that_share(lib, G, dtype):
    _check_attend(lib, [70, 33], [1, 1], 2, G, 128, 16, dtype, seed=G)
    _check_attend(lib, [70, 33], [5, 2], 2, G, 64, 32, dtype, seed=G + 1)


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("D", [64, 128])
def test_chunks_of_ragged_sentences(lib, D, dtype):
    _check_attend(lib, [200, 1, 0, 64, 130, 97], [40, 1, 0, 64, 3, 97], 2, 2, D, 16, dtype, seed=D, tail=3)
    _check_attend(lib, [300, 160], [290, 160], 1, 1, D, 64, dtype, seed=D + 1)


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
@pytest.mark.parametrize("rows", [63, 64, 65, 127, 128, 129, 257])
def test_prompts_around_the_tiles(lib, rows, dtype):
    _check_attend(lib, [rows], [rows], 2, 1, 128, 16, dtype, seed=rows)
    _check_attend(lib, [rows + 40], [rows], 1, 3, 64, 32, dtype, seed=rows + 1)


@pytest.mark.parametrize("dtype", [F16, F32])
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (7, 0), (16, 4), (33, 40), (64, 100), (100, 0), (5000, 3)])
def test_windows_and_sinks(lib, window, sinks, dtype):
    _check_attend(lib, [300, 1, 150, 12], [1, 1, 1, 1], 2, 2, 64, 16, dtype, window, sinks, seed=window)
    _check_attend(lib, [300, 3, 150], [130, 3, 70], 1, 2, 128, 64, dtype, window, sinks, seed=window + 1)


@pytest.mark.parametrize("dtype", [F16, F32])
@pytest.mark.parametrize("B", [1, 2, 64, 65, 200])
def test_slots_shared_out_over_the_chip(lib, B, dtype):
    rng = np.random.default_rng(B)
    lens = [int(n) for n in rng.integers(0, 600 if B > 2 else 3000, B)]
    lens[0] = 2999 if B <= 2 else 777
    _check_attend(lib, lens, [min(n, 1) for n in lens], 1, 4, 128, 32, dtype, seed=B)
    _check_attend(lib, lens, [min(n, 1) for n in lens], 2, 1, 64, 16, dtype, 200, 5, seed=B + 1)


@pytest.mark.parametrize("dtype", [F16, F32])
@pytest.mark.parametrize("B", [65, 200])
def test_one_long_sentence_among_many(lib, B, dtype):
    """Pieces whose sentence is looked for in several rounds."""
    rng = np.random.default_rng(B)
    lens = [int(n) for n in rng.integers(0, 90, B)]
    lens[B - 3], lens[3] = 5000, 1500
    rows = [min(n, 1 + b % 2) for b, n in enumerate(lens)]
    _check_attend(lib, lens, rows, 1, 2, 64, 32, dtype, seed=B + 30)
    _check_attend(lib, lens, rows, 1, 1, 128, 16, dtype, 4500, 5, seed=B + 31)


def test_a_long_context(lib):
    for dtype in (F16, BF16):
        _check_attend(lib, [16000, 3000], [1, 2], 1, 2, 128, 64, dtype, seed=1, qstd=2.0)


def test_some_rows_over_a_long_context(lib):
    """Few rows that go in tiles all the same, whose probabilities are rounded once."""
    for dtype in (F16, BF16, F32):
        _check_attend(lib, [4200, 50], [48, 17], 8, 1, 64, 16, dtype, seed=21, share=FEW + 1)
        _check_attend(lib, [2100, 700, 9], [5, 5, 0], 4, 8, 128, 64, dtype, 600, 70, seed=22, share=FEW + 1, max_len=6000, ahead=61)
        _check_attend(lib, [1000, 90], [17, 1], 2, 1, 64, 16, dtype, seed=23, share=FEW + 1, max_len=1 << 17, ahead=1 << 13)


def test_a_mixed_batch(lib):
    for dtype in (F16, BF16, F32):
        _check_attend(lib, [150, 900, 40, 0, 333], [150, 1, 1, 0, 2], 2, 2, 128, 16, dtype, seed=2, tail=1)
        _check_attend(lib, [350, 900, 40, 5, 333], [300, 1, 1, 1, 2], 2, 1, 64, 16, dtype, 100, 4, seed=3)


def test_many_sentences_beside_one_of_many_rows(lib):
    """More rows than there are workgroups for in a launch of many sentences' pieces."""
    lens, rows = [230] + [5] * 250 + [90], [200] + [1] * 250 + [33]
    for dtype in (F32, F16):
        _check_attend(lib, lens, rows, 8, 1, 64, 16, dtype, seed=24)


def test_rows_ahead_of_the_first_slot_see_nothing(lib):
    for dtype in (F16, F32):
        _check_attend(lib, [3, 0, 80], [5, 4, 100], 2, 2, 64, 16, dtype, seed=4)


def test_lengths_and_rows_past_their_limits(lib):
    """lens beyond 0 .. max_len are taken as its ends; rows from max_rows on are left."""
    cache, table = _cache(lib, 2, 16, 64, F16, [64, 64])
    _fill(cache, table, [64, 64], 1)
    q = _rand((20, 2, 64), F16, 2)
    first = _ints(0, 12, 20)
    a = lib.kvp_attend(q, cache, first, _ints(2 ** 31 - 1, -7), max_rows=12, max_len=50)
    b = lib.kvp_attend(q, cache, first, _ints(50, 0), max_rows=12, max_len=50)
    assert torch.equal(a, b) and bool((a[12:] == 0).all())
    out = torch.full_like(q, 5.0)
    lib.kvp_attend(q, cache, first, _ints(50, 30), max_rows=5, max_len=50, out=out)
    full = lib.kvp_attend(q, cache, first, _ints(50, 30), max_rows=12, max_len=50)
    for at, n in ((0, 12), (12, 8)):
        assert torch.allclose(out[at:at + 5].float(), full[at:at + 5].float(), rtol=2.0 ** -9, atol=2.0 ** -9)
        assert bool((out[at + 5:at + n] == 5.0).all())


def test_beginnings_that_do_not_ascend_touch_no_other_rows(lib):
    cache, table = _cache(lib, 2, 16, 64, F16, [64, 64, 64])
    _fill(cache, table, [64, 64, 64], 1)
    q = _rand((12, 2, 64), F16, 2)
    buf = torch.full((14, 2, 64), 5.0, dtype=F16, device=DEV)
    for first in ([0, 9, 4, 12], [-5, 3, 3, 99], [6, 6, 6, 6], [12, 0, 0, 0], [2 ** 31 - 1, -2 ** 31, 5, 7]):
        buf.fill_(5.0)
        lib.kvp_attend(q, cache, _ints(*first), _ints(64, 20, 64), out=buf[1:13])
        assert bool((buf[0] == 5.0).all()) and bool((buf[13] == 5.0).all())


def test_pages_that_are_none_are_not_seen(lib):
    def edit(table):
        table[0][1] = -1
        table[0][3] = 10 ** 6
        table[1][0] = -2 ** 31
    for dtype in (F16, F32):
        _check_attend(lib, [100, 10], [1, 1], 2, 2, 64, 16, dtype, seed=5, table_edit=edit)
        _check_attend(lib, [100, 10], [90, 10], 2, 2, 64, 16, dtype, seed=6, table_edit=edit)


def test_a_page_of_several_sentences(lib):
    def edit(table):
        table[1][:2] = table[0][:2]
    for rows in ([1, 1], [80, 40]):
        _check_attend(lib, [100, 60], rows, 2, 2, 128, 32, BF16, seed=7, table_edit=edit)


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
@pytest.mark.parametrize("rows,G", [(1, 1), (4, 2), (100, 2)])
def test_what_a_row_does_not_see_does_not_touch_it(lib, rows, G, dtype):
    """Infinities and NaN in later tokens' keys and values, and behind a window: the rows that do not see them stay as they
    are to the bit of what finite values there give, or within a rounding of it; those that see them are not finite."""
    lens, D, page = [130, 70], 64, 16
    for window, sinks, slot in ((0, 0, 128), (40, 3, 50)):
        cache, table = _cache(lib, 1, page, D, dtype, lens, 3)
        _fill(cache, table, lens, 4)
        first = _first([rows, rows])
        q = _rand((2 * rows, G, D), dtype, 5)
        args = (q, cache, _ints(*first), _ints(*lens))
        kw = dict(max_rows=rows, max_len=130, window=window, sinks=sinks)
        clean = f64(lib.kvp_attend(*args, **kw))
        v = cache.v.clone()
        for bad in (math.inf, -math.inf, math.nan):
            cache.v.copy_(v)
            cache.v[table[0][slot // page], 0, slot % page, 7] = bad
            cache.v[table[0][slot // page], 0, slot % page, 40] = -bad
            got = f64(lib.kvp_attend(*args, **kw))
            for r in range(2 * rows):
                p = lens[0] - rows + r
                if r < rows and slot in orc.seen(p, lens[0], window, sinks):
                    assert not np.isfinite(got[r, :, [7, 40]]).any()
                    assert math.isnan(bad) or (np.all(got[r, :, 7] == bad) and np.all(got[r, :, 40] == -bad))
                    others = np.delete(np.arange(D), [7, 40])
                    assert np.isfinite(got[r][:, others]).all()
                else:
                    assert np.all(np.abs(got[r] - clean[r]) <= 2 * HALF[dtype] * (np.abs(clean[r]) + 1.0) + 2.0 ** -18)
        cache.v.copy_(v)
        cache.k[table[0][slot // page], 0, slot % page, 7] = math.nan
        got = f64(lib.kvp_attend(*args, **kw))
        for r in range(2 * rows):
            p = lens[0] - rows + r
            hit = r < rows and slot in orc.seen(p, lens[0], window, sinks)
            assert np.isnan(got[r]).all() if hit else np.array_equal(got[r], clean[r]), r


def test_large_logits_and_one_slot_that_takes_all(lib):
    for dtype in (F16, BF16, F32):
        _check_attend(lib, [200, 64], [1, 1], 2, 2, 64, 16, dtype, seed=8, qstd=30.0)
        _check_attend(lib, [200, 164], [150, 140], 2, 1, 64, 16, dtype, seed=9, qstd=30.0)


def test_maxima_that_rise_all_the_way(lib):
    """Keys whose logits grow by more than the running maximum allows at every step."""
    def edit(cache, table):
        for t in range(300):
            cache.k[table[0][t // 16], :, t % 16] = 0.0
            cache.k[table[0][t // 16], :, t % 16, 0] = t * 0.5
    for rows in (1, 100):
        for dtype in (F16, F32):
            _check_attend(lib, [300], [rows], 1, 1, 64, 16, dtype, seed=10, edit=edit, scale=1.0)


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
@pytest.mark.parametrize("rows", [1, 65])
def test_very_many_slots_of_next_to_no_weight(lib, rows, dtype):
    """2^18 slots of 2^-25.2 of the first one's weight are 0.7 % of the sum together."""
    n, D, page = 1 << 18, 64, 256
    cache = lib.kvp_cache(n // page, 1, page, D, dtype, torch.arange(n // page, dtype=torch.int32, device=DEV).reshape(1, -1))
    cache.k.zero_()
    cache.v.fill_(1.0)
    cache.k[0, 0, 0, 0] = 17.5     # logits 17.5 and 0; 17.5 log2(e) = 25.25
    cache.v[0, 0, 0] = -1.0
    q = torch.zeros((rows, 1, D), dtype=dtype, device=DEV)
    q[..., 0] = 1.0
    got = f64(lib.kvp_attend(q, cache, _ints(0, rows), _ints(n), scale=1.0))
    small = np.exp(-17.5) * (n - rows + np.arange(rows, dtype=np.float64))
    want = ((small - 1.0) / (small + 1.0))[:, None, None]
    # the result's rounding; a weight's own, of the small ones' sum; fp32 sums of n / 4 terms at most, of the small ones' sum too, and exponentials of
    # 25 within 2^-24 of it
    rel = HALF[dtype] + 2.0 ** -24 * (n / 4.0 + 100.0)
    assert np.all(np.abs(got - want) <= HALF[dtype] + 2.0 * rel * small[:, None, None] + 2.0 ** -20)


def test_strided_and_misaligned_queries(lib):
    for odd in (1, 8):
        _check_attend(lib, [40, 70], [3, 1], 2, 2, 64, 16, F16, seed=11, odd=odd)
        _check_attend(lib, [240, 170], [140, 3], 2, 2, 128, 16, BF16, seed=12, odd=odd)


def test_the_same_bits_twice(lib):
    cache, table, q, out, args = _check_attend(lib, [900, 4, 333], [200, 1, 7], 2, 2, 128, 16, BF16, seed=13)
    first, lens = _ints(*_first([200, 1, 7])), _ints(900, 4, 333)
    for _ in range(3):
        assert torch.equal(lib.kvp_attend(q, cache, first, lens, **args), out)


def test_defaults_take_the_whole_table(lib):
    cache, table, q, out, args = _check_attend(lib, [90, 33], [20, 1], 2, 2, 64, 16, F16, seed=14)
    got = lib.kvp_attend(q, cache, _ints(0, 20, 21), _ints(90, 33))
    assert torch.allclose(got.float(), out.float(), rtol=2.0 ** -9, atol=2.0 ** -9)


def test_workspaces_hold_what_they_are_asked_for(lib):
    """Nothing is written behind the size that the query states."""
    for rows, lens, G in (([1, 1], [3000, 90], 2), ([300, 1], [2000, 90], 4), ([600, 5], [5000, 400], 1)):
        cache, table = _cache(lib, 2, 16, 64, F16, lens)
        _fill(cache, table, lens, 3)
        q = _rand((sum(rows), 2 * G, 64), F16, 4)
        n = lib.kvp_attend_workspace_size(cache, sum(rows), 2 * G, max(rows), max(lens))
        ws = torch.full((n + 4096,), 0x5a, dtype=torch.uint8, device=DEV)
        kw = dict(max_rows=max(rows), max_len=max(lens))
        a = lib.kvp_attend(q, cache, _ints(*_first(rows)), _ints(*lens), ws=ws[:n], **kw)
        assert bool((ws[n:] == 0x5a).all())
        assert torch.equal(a, lib.kvp_attend(q, cache, _ints(*_first(rows)), _ints(*lens), **kw))


def test_captured_steps_while_sentences_grow(lib):
    """Append and attend captured once, replayed with lengths, tables and rows that change on the device."""
    H, G, D, page, B = 2, 2, 64, 16, 3
    table = torch.full((B, 8), -1, dtype=torch.int32, device=DEV)
    angles = lib.rope_angles(D, device=DEV)
    caches = [lib.kvp_cache(24, H, page, D, BF16, table) for _ in range(2)]
    for c in caches:
        c.k.fill_(math.nan)
        c.v.fill_(math.nan)
    fused = torch.zeros((B, (G + 2) * H, D), dtype=BF16, device=DEV)
    q, k, v = fused[:, :G * H], fused[:, G * H:G * H + H], fused[:, G * H + H:]
    first, lens = _ints(0, 1, 2, 3), _ints(0, 0, 0)
    outs = [torch.empty((B, G * H, D), dtype=BF16, device=DEV) for _ in range(2)]
    turned = [torch.empty((B, G * H, D), dtype=BF16, device=DEV) for _ in range(2)]
    ws = torch.empty(max(1, lib.kvp_attend_workspace_size(caches[0], B, G * H, 1, 128)), dtype=torch.uint8, device=DEV)

    def step(i):
        lib.kvp_append(caches[i], k, v, first, lens, angles, q=q, q_out=turned[i])
        lib.kvp_attend(turned[i], caches[i], first, lens, max_rows=1, max_len=128, out=outs[i], ws=ws)

    step(0)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(0)
    used = [0] * B
    for i in range(40):
        fused.copy_(_rand(tuple(fused.shape), BF16, 60 + i))
        grows = [1, int(i % 3 > 0), int(i > 20)]
        for b in range(B):
            if grows[b] and used[b] % page == 0:
                table[b, used[b] // page] = 8 * b + used[b] // page
            used[b] += grows[b]
        lens.copy_(_ints(*used))
        first.copy_(_ints(*_first(grows)))
        graph.replay()
        torch.cuda.synchronize()
        step(1)
        n = sum(grows)
        assert torch.equal(outs[0][:n], outs[1][:n]) and torch.equal(turned[0][:n], turned[1][:n])
        assert bool(torch.isfinite(outs[0][:n]).all())


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
def test_a_prompt_in_chunks_and_token_by_token_is_the_prompt_at_once(lib, dtype):
    """Norm, rotation, append and attention together: 150 tokens at once, in chunks beside another sentence's tokens, and
    at the end one by one, against the definition over all of them."""
    H, G, D, page, n = 2, 2, 64, 16, 150
    fused = _rand((n, (G + 2) * H, D), dtype, 1)
    other = _rand((n, (G + 2) * H, D), dtype, 2)
    wq, wk = ((1.0 + _rand((D,), F32, 3 + i, 0.2)).to(dtype) for i in range(2))
    angles = lib.rope_angles(32, style="interleaved", scaling="parts", factor=4.0, original=128.0, device=DEV)
    most = -(-n // page)
    cache = lib.kvp_cache(2 * most, H, page, D, dtype, torch.arange(2 * most, dtype=torch.int32, device=DEV).flip(0).reshape(2, most).contiguous())
    f = orc.frequencies(32, scaling="parts", factor=4.0, original=128.0)
    got = torch.empty((n, G * H, D), dtype=dtype, device=DEV)
    done = extra = 0
    for m in [64, 1, 50, 7] + [1] * 28:
        e = min(3, n - extra)
        x = torch.cat([other[extra:extra + e], fused[done:done + m]])      # the other sentence's tokens go first
        q, k, v = x[:, :G * H], x[:, G * H:G * H + H], x[:, G * H + H:]
        first, lens = _ints(0, e, e + m), _ints(extra + e, done + m)
        q = lib.kvp_append(cache, k, v, first, lens, angles, k_norm=wk, q=q, q_norm=wq)
        y = lib.kvp_attend(q, cache, first, lens, max_rows=max(e, m), max_len=n, window=100, sinks=4)
        got[done:done + m] = y[e:]
        done, extra = done + m, extra + e
    assert done == n
    pos = np.arange(n)
    rounded = lambda t: f64(torch.from_numpy(t).to(dtype))  # noqa: E731
    q = rounded(orc.rope(f64(fused[:, :G * H]), pos, f, "interleaved", angles.scale, f64(wq), 1e-6))
    k = rounded(orc.rope(f64(fused[:, G * H:G * H + H]), pos, f, "interleaved", angles.scale, f64(wk), 1e-6))
    v = f64(fused[:, G * H + H:])
    want, _, size, reach = orc.attend(q, k.transpose(1, 0, 2)[None], v.transpose(1, 0, 2)[None], [[0]], [0, n], [n], 100, 4, D ** -0.5)
    # keys and queries may be rounded to the neighbour of what the definition's are rounded to: two units of each, which are 4 half units of a
    # logit's terms, and a probability is off by twice that
    slack = 2.0 * 8.0 * HALF[dtype] * reach[..., None] * size
    err = np.abs(f64(got) - want)
    assert np.all(err <= _bound(dtype, want, size, reach, D, n, n * G) + slack)


def test_tensors_of_another_device_are_refused(lib):
    """Host tensors among the device's would be read by the kernels at the host's addresses."""
    cache, table = _cache(lib, 2, 16, 64, F16, [5])
    x, first, lens = _rand((1, 2, 64), F16, 1), _ints(0, 1), _ints(5)
    angles, host = lib.rope_angles(64, device=DEV), lib.rope_angles(64, device="cpu")
    norm, pos = torch.ones(64, dtype=F16), torch.zeros(1, dtype=torch.int32)
    for kw in (dict(k=x.cpu()), dict(v=x.cpu()), dict(first=first.cpu()), dict(lens=lens.cpu()), dict(angles=host), dict(pos=pos),
               dict(k_norm=norm), dict(q=x.cpu()), dict(q=x, q_norm=norm), dict(q=x, q_out=torch.empty(1, 2, 64, dtype=F16))):
        with pytest.raises(AssertionError):
            lib.kvp_append(**{**dict(cache=cache, k=x, v=x, first=first, lens=lens), **kw})
    for kw in (dict(q=x.cpu()), dict(first=first.cpu()), dict(lens=lens.cpu()), dict(out=torch.empty(1, 2, 64, dtype=F16)),
               dict(lse=torch.empty(1, 2)), dict(ws=torch.empty(1 << 20, dtype=torch.uint8))):
        with pytest.raises(AssertionError):
            lib.kvp_attend(**{**dict(q=x, cache=cache, first=first, lens=lens), **kw})
    for kw in (dict(pos=pos), dict(angles=host), dict(norm=norm), dict(out=torch.empty(1, 2, 64, dtype=F16))):
        with pytest.raises(AssertionError):
            lib.rope(**{**dict(x=x, pos=_ints(0), angles=angles), **kw})
    with pytest.raises(AssertionError):
        lib.kvp_cache(1, 2, 16, 64, F16, torch.zeros(1, 1, dtype=torch.int32)).__class__(cache.k, cache.v, torch.zeros(1, 1, dtype=torch.int32))
