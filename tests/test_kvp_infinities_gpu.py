"""Attention over pages where what a row sees is infinite or NaN: what the definition in 64 bits gives, however the call is split."""

import math

import numpy as np
import pytest
import torch

from oracle import pages_oracle as orc
from tests._util import f64
from tests.test_kvp_gpu import BF16, DEV, F16, F32, _bound, _cache, _fill, _first, _ints, _rand

pytestmark = pytest.mark.gpu


def _run(lib, cache, q, lens, rows, window=0, sinks=0, scale=None):
    lse = torch.full(q.shape[:2], 5.0, dtype=F32, device=DEV)
    out = lib.kvp_attend(q, cache, _ints(*_first(rows)), _ints(*lens), max_rows=max(rows), max_len=max(lens), window=window, sinks=sinks,
                         scale=scale, lse=lse)
    return f64(out), f64(lse)


def _check(lib, cache, table, q, lens, rows, window=0, sinks=0):
    """Against the definition: NaN where it is NaN, the same infinities, and the other results within the usual bounds, whose logits' size is
    that of the finite factors.  Slots outside the sentences are NaN in the cache and not seen."""
    got, got_lse = _run(lib, cache, q, lens, rows, window, sinks)
    first, D, scale = _first(rows), cache.D, cache.D ** -0.5
    qq, k, v = f64(q), f64(cache.k), f64(cache.v)
    cut = lambda x: np.where(np.isfinite(x), x, 0.0)  # noqa: E731
    with np.errstate(all="ignore"):
        want, want_lse, _, _ = orc.attend(qq, k, v, table, first, lens, window, sinks, scale)
        _, _, size, reach = orc.attend(cut(qq), cut(k), cut(v), table, first, lens, window, sinks, scale)
    assert np.array_equal(np.isnan(got), np.isnan(want)) and np.array_equal(np.isnan(got_lse), np.isnan(want_lse))
    ok = np.isfinite(want)
    assert np.array_equal(np.where(ok | np.isnan(want), 0.0, got), np.where(ok | np.isnan(want), 0.0, want))   # infinities
    size = np.maximum(size, np.abs(cut(v)).max())      # weights are not those of the cut logits
    bound = _bound(cache.dtype, cut(want), size, reach, D, max(lens), max(rows) * (q.shape[1] // cache.H))
    assert np.all(np.abs(got[ok] - want[ok]) <= bound[ok])
    return want, want_lse


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("n,rows", [(60, 1), (256, 1), (300, 1), (513, 1), (3000, 1), (60, 60), (200, 130), (300, 300), (1500, 70)])
@pytest.mark.parametrize("what", ["first", "last", "query"])
def test_an_infinite_key_or_query(lib, n, rows, what, dtype):
    """Products of both signs: a logit of +infinity makes its row NaN, one of -infinity takes its slot's weight only."""
    H, G, D, page = 1, 2, 64, 16
    cache, table = _cache(lib, H, page, D, dtype, [n], 1)
    _fill(cache, table, [n], 2)
    q = _rand((rows, G, D), dtype, 3)
    q[:, 0, 3], q[:, 1, 3] = 1.0, -1.0
    if what == "query":
        q[rows // 2, 0, 5] = math.inf
        q[rows - 1, 1, 5] = -math.inf
    else:
        slot = 1 if what == "first" else n - 1
        cache.k[table[0][slot // page], 0, slot % page, 3] = math.inf
    want, _ = _check(lib, cache, table, q, [n], [rows])
    assert np.isnan(want).any() and (what == "query" and rows == 1 or np.isfinite(want).any())


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("n,rows", [(4000, 1), (4000, 100), (300, 1), (300, 100), (700, 66)])
@pytest.mark.parametrize("low_first", [True, False])
def test_an_infinite_value_of_next_to_no_weight(lib, n, rows, low_first, dtype):
    """Seen at 2^-216 of the largest weight, in another piece of its row, in another round, or in the same one: it is not finite all the same."""
    D, page, low = 64, 16, -150.0
    cache, table = _cache(lib, 1, page, D, dtype, [n], 1)
    _fill(cache, table, [n], 2)
    half, slot = n // 2 - 60, 10
    for t in range(n):
        cache.k[table[0][t // page], 0, t % page] = 0.0
        cache.k[table[0][t // page], 0, t % page, 0] = low if (t < half) == low_first else 0.0
    if not low_first:
        slot = n - rows - 5
    q = torch.zeros((rows, 1, D), dtype=dtype, device=DEV)
    q[..., 0] = 1.0
    clean, clean_lse = _run(lib, cache, q, [n], [rows], scale=1.0)
    at = cache.v[table[0][slot // page], 0, slot % page]
    for channel, x in ((7, math.inf), (9, -math.inf), (11, math.nan)):
        at[channel] = x
    got, got_lse = _run(lib, cache, q, [n], [rows], scale=1.0)
    assert np.all(got[..., 7] == math.inf) and np.all(got[..., 9] == -math.inf) and np.isnan(got[..., 11]).all()
    rest = np.delete(np.arange(D), [7, 9, 11])
    # both ways have the bounds of a clean call: every logit is 0 or `low`, so a row is off by its weights' rounding (half a unit of the largest value
    # each, and none of `low` counts) and fp32 sums, and by the result's rounding
    bound = _bound(dtype, clean[..., rest], np.full(clean[..., rest].shape, np.abs(f64(cache.v)[np.isfinite(f64(cache.v))]).max()),
                   np.zeros((rows, 1)), D, n, rows)
    assert np.all(np.abs(got[..., rest] - clean[..., rest]) <= 2.0 * bound)
    assert np.all(np.abs(got_lse - clean_lse) <= 2.0 ** -24 * (32.0 + n / 4.0 + 4.0 * np.abs(clean_lse)))


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("n,rows", [(1, 1), (60, 1), (300, 1), (4000, 1), (60, 60), (300, 300), (4000, 80)])
def test_rows_whose_logits_are_all_minus_infinity(lib, n, rows, dtype):
    """0 / 0, and not the zeros of a row that sees nothing; the logarithm of their sum is that of 0."""
    D, page = 64, 16
    lens = [n, rows - 1]
    cache, table = _cache(lib, 1, page, D, dtype, lens, 1)
    _fill(cache, table, lens, 2)
    cache.k[..., 3] = math.inf
    q = _rand((2 * rows, 1, D), dtype, 3)
    q[..., 3] = -1.0
    if rows > 1:
        q[1, 0, 3] = 1.0       # this one has logits of +infinity
    got, got_lse = _run(lib, cache, q, lens, [rows, rows])
    assert np.isnan(got[:rows]).all()
    assert np.isneginf(np.delete(got_lse[:rows], 1 if rows > 1 else [])).all() and (rows == 1 or math.isnan(got_lse[1, 0]))
    # the second sentence's first row is ahead of its first slot
    assert np.all(got[rows] == 0.0) and math.isinf(got_lse[rows, 0]) and np.isnan(got[rows + 1:]).all()
    # a page that is none is not seen, whatever its number would have held
    cache.table.fill_(-1)
    got, got_lse = _run(lib, cache, q, lens, [rows, rows])
    assert np.all(got == 0.0) and np.isneginf(got_lse).all()


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("n,rows", [(60, 1), (300, 1), (4000, 1), (60, 60), (300, 300)])
def test_an_infinite_value_behind_a_logit_of_minus_infinity(lib, n, rows, dtype):
    """0 times infinity."""
    D, page = 64, 16
    cache, table = _cache(lib, 1, page, D, dtype, [n], 1)
    _fill(cache, table, [n], 2)
    cache.k[table[0][0], 0, 5, 3] = math.inf
    cache.v[table[0][0], 0, 5, 8] = math.inf
    q = _rand((rows, 1, D), dtype, 3)
    q[..., 3] = -1.0
    _check(lib, cache, table, q, [n], [rows])


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("D,window", [(64, 0), (128, 0), (128, 70)])
@pytest.mark.parametrize("n,rows", [(90, 1), (90, 17), (300, 16), (3000, 3), (200, 130), (2500, 66), (2500, 300)])
def test_every_place_of_infinite_values(lib, n, rows, D, window, dtype):
    """Values of every kind at random: rows see them or not, several of a kind and of both signs in a channel, whole slots."""
    H, G, page = 2, 2, 16
    rng = np.random.default_rng(n + rows)
    lens, counts = [n, 40], [rows, 2]
    cache, table = _cache(lib, H, page, D, dtype, lens, 1)
    _fill(cache, table, lens, 2)
    for i in range(40):
        b = int(i % 8 == 0)
        t = int(rng.integers(0, lens[b])) if i % 2 else max(0, lens[b] - 1 - int(rng.integers(0, 2 * counts[b])))
        where = table[b][t // page], int(rng.integers(0, H)), t % page, int(rng.integers(0, D))
        cache.v[where] = (math.inf, -math.inf, math.nan)[i % 3]
    cache.v[table[0][(n - 1) // page], 1, (n - 1) % page] = math.inf      # the last row's slot
    q = _rand((sum(counts), H * G, D), dtype, 3)
    want, _ = _check(lib, cache, table, q, lens, counts, window, 3 if window else 0)
    assert np.isinf(want).any() and np.isfinite(want).any()


@pytest.mark.parametrize("dtype", [F16, F32])
def test_a_prompt_with_an_infinite_value_ends_in_good_time(lib, dtype):
    """Rows that see one are done again, sixteen at a time: within 60 times what finite values take, for any of them; row by row it was
    more than 1000 times, and grew with the context."""
    n, H, D, page = 4096, 8, 128, 16
    table = torch.arange(n // page, dtype=torch.int32, device=DEV).reshape(1, -1)
    cache = lib.kvp_cache(n // page, H, page, D, dtype, table)
    cache.k.copy_(_rand(tuple(cache.k.shape), dtype, 1))
    cache.v.copy_(_rand(tuple(cache.v.shape), dtype, 2))
    q, first, lens = _rand((n, H, D), dtype, 3), _ints(0, n), _ints(n)
    out = torch.empty_like(q)

    def took():
        times = []
        for _ in range(3):
            start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            start.record()
            lib.kvp_attend(q, cache, first, lens, max_rows=n, max_len=n, out=out)
            end.record()
            end.synchronize()
            times.append(start.elapsed_time(end))
        return min(times)

    clean = took()
    cache.v[0, :, 10, 7] = math.inf
    assert took() <= 60.0 * clean
    assert bool((out[10:, :, 7] == math.inf).all()) and bool(torch.isfinite(out[:10]).all()) and bool(torch.isfinite(out[:, :, :7]).all())
    cache.v.fill_(math.nan)
    assert took() <= 60.0 * clean
    assert bool(torch.isnan(out).all())
