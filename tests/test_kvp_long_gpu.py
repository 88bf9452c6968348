"""Attention of long prompts over pages against float64, by torch on the GPU: tiles that see many steps, whole and in pieces, and both ways of calling."""

import math

import pytest
import torch

from tests.test_kvp_gpu import BF16, DEV, F16, F32, HALF, TINY, _cache, _fill, _first, _ints, _rand
from tests.test_pages_binding_host import plain  # noqa: F401

pytestmark = pytest.mark.gpu


def _definition(cache, table, q, b, row, rows, length, window, sinks):
    """One sentence's rows in 64 bits: results, lse, the weights' sum of |v|, and the largest sum |q| |k| of a row."""
    D, H = cache.D, cache.H
    pages = torch.tensor(table[b][:-(-length // cache.page)], device=DEV, dtype=torch.long)
    k, v = (t[pages].transpose(0, 1).reshape(H, -1, D)[:, :length].to(torch.float64) for t in (cache.k, cache.v))
    G = q.shape[1] // H
    x = q[row:row + rows].to(torch.float64)
    p = torch.arange(length - rows, length, device=DEV)[:, None]
    t = torch.arange(length, device=DEV)[None]
    seen = t <= p
    if window:
        seen &= (t > p - window) | (t < sinks)
    out, lse, size, reach = [], [], [], []
    for i in range(q.shape[1]):
        kt = k[i // G].t().contiguous()
        z = (x[:, i] @ kt) / math.sqrt(D)
        z = z.masked_fill(~seen, -math.inf)
        w = torch.softmax(z, -1)
        out.append(w @ v[i // G])
        lse.append(torch.logsumexp(z, -1))
        size.append(w @ v[i // G].abs())
        reach.append((x[:, i].abs() @ kt.abs()).amax(-1) / math.sqrt(D))
    return (torch.stack(a, 1) for a in (out, lse, size, reach))


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
@pytest.mark.parametrize("lens,rows,H,G,D,page,window,sinks", [
    ([2100], [2100], 2, 1, 128, 16, 0, 0),            # whole tiles of up to 33 steps
    ([1999], [1999], 2, 2, 64, 64, 0, 0),
    ([5000], [300], 2, 2, 128, 32, 0, 0),             # pieces
    ([5000], [777], 1, 1, 64, 256, 1500, 70),
    ([2600, 1300, 4000], [2600, 1, 2], 2, 2, 64, 16, 0, 0),      # beside single tokens
    ([1500, 1500, 1500, 900], [1024, 1500, 700, 900], 4, 4, 128, 16, 0, 0),      # many tiles: none in pieces
])
def test_long_prompts(lib, lens, rows, H, G, D, page, window, sinks, dtype):
    """Half a unit of the result; of the sum of p |v|: a logit's D products and sums in fp32 relative to the terms' size, its scale, exponential and
    maximum, 2^-24 (D + 8) |q||k| + 16; the weights' one rounding in tiles, none in fp32; fp32 sums of n / 4 terms at most and the join's."""
    cache, table = _cache(lib, H, page, D, dtype, lens, 1)
    _fill(cache, table, lens, 2)
    first = _first(rows)
    q = _rand((first[-1], G * H, D), dtype, 3)
    lse = torch.empty(first[-1], G * H, device=DEV)
    out = lib.kvp_attend(q, cache, _ints(*first), _ints(*lens), max_rows=max(rows), max_len=max(lens), window=window, sinks=sinks, lse=lse)
    for b, (n, m) in enumerate(zip(lens, rows)):
        want, want_lse, size, reach = _definition(cache, table, q, b, first[b], m, n, window, sinks)
        part = slice(first[b], first[b] + m)
        rel = 2.0 ** -24 * ((D + 8) * reach[..., None] + 16.0 + n / 4.0 + 80.0) + (0.0 if dtype is F32 else HALF[dtype])
        bound = HALF[dtype] * want.abs() + TINY[dtype] + 2.0 * rel * size
        err = (out[part].to(torch.float64) - want).abs()
        assert bool((err <= bound).all()), float((err / bound).max())
        bound = 2.0 ** -24 * ((D + 8) * reach + 32.0 + n / 4.0 + want_lse.abs() * 4.0)
        assert bool(((lse[part].to(torch.float64) - want_lse).abs() <= bound).all())


def test_calls_through_ctypes_give_the_same(lib, plain):  # noqa: F811
    results = []
    for module in (lib, plain):
        cache, table = _cache(module, 2, 16, 64, F16, [90, 33])
        _fill(cache, table, [90, 33], 2)
        fused = _rand((9, 8, 64), F16, 3)
        first, lens, angles, norm = _ints(0, 7, 9), _ints(90, 33), module.rope_angles(64, device=DEV), torch.ones(64, dtype=F16, device=DEV)
        turned = module.rope(fused[:, :4], _ints(*range(9)), angles, norm=norm, backward=False)
        q = module.kvp_append(cache, fused[:, 4:6], fused[:, 6:], first, lens, angles, k_norm=norm, q=turned, q_norm=norm)
        lse = torch.empty(9, 4, device=DEV)
        out = module.kvp_attend(q, cache, first, lens, max_rows=7, max_len=90, window=40, sinks=3, lse=lse)
        results.append((turned, q, torch.nan_to_num(cache.k), torch.nan_to_num(cache.v), out, lse))
    assert all(torch.equal(a, b) for a, b in zip(*results))
