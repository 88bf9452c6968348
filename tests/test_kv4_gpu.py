"""The 4-bit cache on the GPU against the plain definitions: writes, reads and evictions exactly, attention within the rounding of
its sums."""

import ctypes

import numpy as np
import pytest
import torch

from oracle import q4_oracle as orc
from tests._util import f64

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F16, BF16, F32 = torch.float16, torch.bfloat16, torch.float32
HALF_ULP = {F32: 2.0 ** -24, F16: 2.0 ** -11, BF16: 2.0 ** -8}
OFFSET = {F32: 0.0, F16: 64.0, BF16: 128.0}
PIECES = {F32: 2.0 ** -23, F16: 2.0 ** -16, BF16: 2.0 ** -16}   # of a probability
SHAPES = [(64, 32), (64, 64), (128, 32), (128, 64), (128, 128)]


def _rand(shape, dtype, seed, std=1.0):
    g = torch.Generator(device="cpu")
    g.manual_seed(seed)
    return (torch.randn(*shape, generator=g) * std).to(dtype).to(DEV)


def _ints(*v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def _dirty(cache):
    """What lies in the buffers before anything is written: codes of all ones, NaN steps."""
    for t in (cache.k, cache.v, cache.k_scale, cache.v_scale):
        t.fill_(0xff)
    return cache


def _filled(lib, B, H, T, D, group, dtype, seed, cap=None):
    """A cache whose sentences all have T tokens, with the held values [B, H, T, D]."""
    cap = cap or -(-T // 32) * 32
    cache = _dirty(lib.kv4_cache(B, H, cap, D, group, device=DEV))
    k, v = _rand((B, T, H, D), dtype, seed), _rand((B, T, H, D), dtype, seed + 1)
    k[..., 3] *= 5.0
    lib.kv4_append(cache, k, v, _ints(*[T] * B))
    hold = lambda t: orc.held_values(f64(t), group).transpose(0, 2, 1, 3)  # noqa: E731
    return cache, hold(k), hold(v)


# ------------------------------------------------------------------------------------------ writing and reading

@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("D,group", SHAPES)
@pytest.mark.parametrize("T", [1, 2, 5, 16, 33, 100])
def test_written_slots_read_back_as_the_values_they_stand_for(lib, T, D, group, dtype):
    cache, k, v = _filled(lib, 2, 3, T, D, group, dtype, T)
    lens = _ints(T, T)
    for got, want in zip(lib.kv4_read(cache, lens, 0, T, F32), (k, v)):
        assert np.array_equal(got.cpu().numpy(), want.astype(np.float32))
    for got, want in zip(lib.kv4_read(cache, _ints(T, T // 2), T // 2, T - T // 2, dtype), (k, v)):
        part = torch.from_numpy(want[:, :, T // 2:].astype(np.float32)).to(dtype)
        part[1] = 0.0                     # from the second sentence's length on
        assert torch.equal(got.cpu(), part)


@pytest.mark.parametrize("D,group", SHAPES)
def test_tokens_one_by_one_and_in_ragged_chunks_are_the_tokens_at_once(lib, D, group):
    B, H, T, cap = 3, 2, 45, 64
    k, v = _rand((B, T, H, D), F16, 1), _rand((B, T, H, D), F16, 2)
    whole, grown = (_dirty(lib.kv4_cache(B, H, cap, D, group, device=DEV)) for _ in range(2))
    lib.kv4_append(whole, k, v, _ints(T, T, T))
    have = [0, 0, 0]
    for i, new in enumerate([(1, 1, 1), (0, 3, 7), (7, 0, 2), (13, 20, 1)] + [(1, 1, 1)] * 40):
        new = [min(n, T - h) for n, h in zip(new, have)]
        S = max(max(new), 1)
        ck, cv = torch.full((B, S, H, D), 77.0, dtype=F16, device=DEV), torch.full((B, S, H, D), 77.0, dtype=F16, device=DEV)
        for b in range(B):
            if new[b]:
                ck[b, S - new[b]:], cv[b, S - new[b]:] = k[b, have[b]:have[b] + new[b]], v[b, have[b]:have[b] + new[b]]
        lens = [h + n for h, n in zip(have, new)]
        lib.kv4_append(grown, ck, cv, _ints(*lens), start=_ints(*have))
        have = lens
    assert have == [T] * 3
    lens = _ints(T, T, T)
    for a, b in zip(lib.kv4_read(whole, lens, 0, cap, F32), lib.kv4_read(grown, lens, 0, cap, F32)):
        assert torch.equal(a, b)
    assert torch.equal(whole.pos, grown.pos)


def test_append_keeps_to_its_slots(lib):
    B, H, D, group, cap = 4, 2, 128, 64, 64
    cache, k, v = _filled(lib, B, H, cap, D, group, BF16, 5)
    before = [t.clone() for t in lib.kv4_read(cache, _ints(*[cap] * B), 0, cap, F32)]
    cache.weight.fill_(3.0)
    pos = cache.pos.clone()
    nk, nv = _rand((B, 6, H, D), BF16, 8), _rand((B, 6, H, D), BF16, 9)
    # two tokens past the capacity; an empty sentence; fewer new tokens than the chunk; a length far past everything
    lib.kv4_append(cache, nk, nv, _ints(cap + 2, 0, 33, 2 ** 31 - 1), start=_ints(0, 0, 31, 0), next_pos=_ints(500, 0, 900, 0))
    after = lib.kv4_read(cache, _ints(*[cap] * B), 0, cap, F32)
    for got, old, new in zip(after, before, (nk, nv)):
        want = old.cpu().numpy().copy()
        held = orc.held_values(f64(new), group).transpose(0, 2, 1, 3).astype(np.float32)
        want[0, :, cap - 4:] = held[0, :, :4]
        want[2, :, 31:33] = held[2, :, 4:]
        assert np.array_equal(got.cpu().numpy(), want)
    w = torch.full_like(cache.weight, 3.0)
    w[0, :, cap - 4:] = 0.0
    w[2, :, 31:33] = 0.0
    assert torch.equal(cache.weight, w)
    pos[0, :, cap - 4:] = torch.arange(494, 498, device=DEV)
    pos[2, :, 31:33] = torch.arange(898, 900, device=DEV)
    assert torch.equal(cache.pos, pos)


def test_append_takes_slices_of_a_fused_projection(lib):
    B, S, H, D = 2, 7, 3, 64
    for odd in (0, 1):                                                  # rows aligned to 16 bytes, and not
        fused = _rand((B, S, 3 * H * D + odd), F16, 4)
        k, v = (fused[..., odd + i * H * D:odd + (i + 1) * H * D].unflatten(-1, (H, D)) for i in (1, 2))
        a, b = (_dirty(lib.kv4_cache(B, H, 32, D, 32, device=DEV)) for _ in range(2))
        lib.kv4_append(a, k, v, _ints(S, S))
        lib.kv4_append(b, k.contiguous(), v.contiguous(), _ints(S, S))
        for x, y in zip(lib.kv4_read(a, _ints(S, S), 0, S, F32), lib.kv4_read(b, _ints(S, S), 0, S, F32)):
            assert torch.equal(x, y)


def test_a_cache_without_weights_and_positions(lib):
    cache = lib.kv4_cache(1, 2, 32, 64, 32, weights=False, device=DEV)
    k = _rand((1, 9, 2, 64), F16, 1)
    lib.kv4_append(cache, k, k, _ints(9))
    got, _ = lib.kv4_read(cache, _ints(9), 0, 9, F32)
    assert np.array_equal(got.cpu().numpy(), orc.held_values(f64(k), 32).transpose(0, 2, 1, 3).astype(np.float32))
    assert lib.kv4_attend(k[:, -1:], cache, _ints(9)).isfinite().all()


# ---------------------------------------------------------------------------------------------------- attention

def _check_attend(lib, B, H, G, T, S, D, group, dtype, lens=None, seed=0, weights=True, max_len=None, qstd=1.0, cap=None):
    cache, k, v = _filled(lib, B, H, T, D, group, dtype, seed + 10, cap=cap)
    lens = [T] * B if lens is None else lens
    q = _rand((B, S, H * G, D), dtype, seed + 20, qstd)
    used = _rand((B, H, cache.cap), F32, seed + 30).abs()
    cache.weight.copy_(used)
    out = torch.full_like(q, 5.0)
    lse = torch.full((B, S, H * G), 5.0, dtype=F32, device=DEV)
    wout = torch.full_like(used, 7.0) if weights else None
    lib.kv4_attend(q, cache, _ints(*lens), max_len=max_len or T, out=out, lse=lse, weight_out=wout)
    scale = D ** -0.5
    seen = [min(max(n, 0), max_len or T) for n in lens]
    want, want_lse, add = orc.attend(f64(q), k, v, seen, scale)
    # logits: D rounded products with the offset that the operands carry; a probability is off by as much, relatively, and by its
    # pieces' rounding; sums over the slots round 2^-24 of sums that carry an offset as well
    steps = (np.abs(k).max() * 2 / 15)
    logit = scale * 8 * np.sqrt(D + 32) * 2.0 ** -24 * np.sqrt((f64(q) ** 2).sum(-1)) * (steps * (OFFSET[dtype] + 15) + np.abs(k).max())
    logit = logit + 2.0 ** -22 * np.abs(np.where(np.isfinite(want_lse), want_lse, 0.0)) + 2.0 ** -20
    vmax = np.abs(v).max()
    offset_v = 0.0 if dtype == F32 else 128.0
    sums = 8 * np.sqrt(T + 32) * 2.0 ** -24 * (1 + 2 * (offset_v + 15) / 15)
    err = np.abs(f64(out) - want)
    bound = vmax * (2 * logit[..., None] + 2 * PIECES[dtype] + sums) * 1.01
    bound = bound + HALF_ULP[dtype] * (np.abs(want) + bound) + (2.0 ** -24 if dtype == F16 else 0.0)
    assert (err <= bound).all(), (err.max(), bound.flat[err.argmax()])
    fin = np.isfinite(want_lse)
    got_lse = f64(lse)
    assert np.array_equal(fin, np.isfinite(got_lse)) and (got_lse[~fin] == -np.inf).all()
    assert (np.abs(got_lse - want_lse)[fin] <= (logit + sums)[fin]).all()
    if weights:
        w, u = f64(wout), f64(used)
        for b in range(B):
            n = seen[b]
            total = u[b, :, :n] + add[b, :, :n]
            slack = add[b, :, :n] * (2 * logit[b].max() + 2 * sums) + 2.0 ** -22 * total + 2.0 ** -30 * S * G
            assert (np.abs(w[b, :, :n] - total) <= slack).all()
            assert (w[b, :, n:] == 7.0).all()       # slots that are not in use are left as they are
    return cache, q, out


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("D,group", SHAPES)
@pytest.mark.parametrize("G", [1, 4])
def test_one_token(lib, G, D, group, dtype):
    for T in (1, 2, 31, 32, 33, 100):
        _check_attend(lib, 2, 2, G, T, 1, D, group, dtype, seed=T)


@pytest.mark.parametrize("T", [255, 1000, 3001])
@pytest.mark.parametrize("G,dtype,D,group", [(1, F16, 128, 64), (8, BF16, 128, 128), (16, F16, 64, 32), (5, F32, 128, 32)])
def test_one_token_over_splits_of_the_cache(lib, T, G, dtype, D, group):
    _check_attend(lib, 1, 2, G, T, 1, D, group, dtype, seed=T)
    _check_attend(lib, 1, 2, G, T, 1, D, group, dtype, seed=T, weights=False)


@pytest.mark.parametrize("S,G", [(2, 1), (7, 1), (16, 1), (17, 1), (5, 4), (33, 2), (64, 1), (70, 2), (130, 1)])
@pytest.mark.parametrize("dtype,D,group", [(F16, 128, 64), (BF16, 64, 32), (F32, 64, 64), (BF16, 128, 128)])
def test_chunks_see_what_came_before_them(lib, S, G, dtype, D, group):
    for T in (S, S + 1, S + 100, S + 700):
        _check_attend(lib, 1, 2, G, T, S, D, group, dtype, seed=S + T)


@pytest.mark.parametrize("D,group", SHAPES)
@pytest.mark.parametrize("S,G", [(1, 1), (1, 8), (9, 1), (40, 2)])
def test_ragged_sentences_and_rows_that_see_nothing(lib, S, G, D, group):
    lens = [150, 0, 1, S - 1, 37, -3, 1000]            # the last: more than max_len
    _check_attend(lib, 7, 2, G, 150, S, D, group, F16, lens=lens, seed=S)
    _check_attend(lib, 7, 2, G, 150, S, D, group, BF16, lens=lens, seed=S, weights=False)


@pytest.mark.parametrize("S", [1, 20])
def test_max_len_below_the_capacity_and_lengths_beyond_it(lib, S):
    _check_attend(lib, 3, 2, 1, 300, S, 128, 64, F16, lens=[300, 200, 65], max_len=129)
    _check_attend(lib, 2, 2, 1, 300, S, 128, 64, F16, lens=[300, 200], cap=1024)


def test_logits_far_apart(lib):
    """A maximum that rises along the cache by much more than a sum's range, and falls."""
    for dtype in (F16, BF16, F32):
        for S in (1, 40):
            B, H, T, D, group = 1, 2, 500, 64, 64
            cache = _dirty(lib.kv4_cache(B, H, 512, D, group, device=DEV))
            ramp = torch.cat([torch.linspace(-3, 3, 300), torch.linspace(3, -3, 200)])
            k = ramp[None, :, None, None].to(DEV) * torch.ones(1, T, H, D, device=DEV)
            k = (k + 0.01 * _rand((1, T, H, D), F32, 1)).to(dtype)
            v = _rand((1, T, H, D), dtype, 2)
            lib.kv4_append(cache, k, v, _ints(T))
            q = torch.full((1, S, H, D), 4.0, dtype=dtype, device=DEV)
            out = lib.kv4_attend(q, cache, _ints(T), max_len=T)
            hold = lambda t: orc.held_values(f64(t), group).transpose(0, 2, 1, 3)  # noqa: E731
            want, _, _ = orc.attend(f64(q), hold(k), hold(v), [T], D ** -0.5)
            # logits up to 96: off by 2^-20 of that and the offset's share, and the probabilities by as much
            tol = 96 * 2.0 ** -16 + 2 * HALF_ULP[dtype]
            assert np.abs(f64(out) - want).max() <= tol * np.abs(f64(v)).max()


def test_a_nan_key_or_value_reaches_only_what_sees_it(lib):
    B, H, T, D, group = 2, 2, 80, 128, 64
    cache = _dirty(lib.kv4_cache(B, H, 96, D, group, device=DEV))
    k, v = _rand((B, T, H, D), F16, 1), _rand((B, T, H, D), F16, 2)
    lib.kv4_append(cache, k, v, _ints(T, T))
    q = _rand((B, 3, H, D), F16, 3)
    good = lib.kv4_attend(q, cache, _ints(T, T), max_len=T)
    k[0, T - 1, 0, 5], v[1, T - 2, 1, 70] = float("nan"), float("nan")
    lib.kv4_append(cache, k, v, _ints(T, T))
    out = lib.kv4_attend(q, cache, _ints(T, T), max_len=T)
    assert out[0, 2, 0].isnan().all() and torch.equal(out[0, :2], good[0, :2]) and torch.equal(out[0, 2, 1], good[0, 2, 1])
    assert out[1, 1:, 1, 64:].isnan().all() and torch.equal(out[1, :, 0], good[1, :, 0])
    assert torch.equal(out[1, 1:, 1, :64], good[1, 1:, 1, :64]) and torch.equal(out[1, 0], good[1, 0])
    # ... and nothing that ends before it
    short = lib.kv4_attend(q, cache, _ints(T - 1, T - 2), max_len=T)
    assert short.isfinite().all()


def test_a_strided_query_and_a_scale(lib):
    B, S, H, G, D = 2, 4, 2, 3, 64
    cache, k, v = _filled(lib, B, H, 90, D, 32, F16, 3)
    for odd in (0, 1):
        fused = _rand((B, S, 2 * H * G * D + odd), F16, 4)
        q = fused[..., odd:odd + H * G * D].unflatten(-1, (H * G, D))
        a = lib.kv4_attend(q, cache, _ints(90, 50), scale=0.3)
        assert torch.equal(a, lib.kv4_attend(q.contiguous(), cache, _ints(90, 50), scale=0.3))
        want, _, _ = orc.attend(f64(q), k, v, [90, 50], 0.3)
        assert np.abs(f64(a) - want).max() <= 2e-3 * np.abs(v).max()


def test_offsets_past_32_bits(lib):
    """The last head of a cache of more than 4 GiB of keys."""
    B, H, cap, D, group = 2, 2, 16777216, 128, 128
    cache = lib.kv4_cache(B, H, cap, D, group, weights=False, device=DEV)
    assert cache.k.numel() == 1 << 32
    k, v = _rand((B, 70, H, D), F16, 1), _rand((B, 70, H, D), F16, 2)
    lens = _ints(70, cap)
    lib.kv4_append(cache, k, v, lens)
    got, _ = lib.kv4_read(cache, lens, cap - 70, 70, F32)
    assert np.array_equal(got[1].cpu().numpy(), orc.held_values(f64(k), group).transpose(0, 2, 1, 3)[1].astype(np.float32))
    lens = _ints(70, 70)
    lib.kv4_append(cache, k, v, lens)
    q = _rand((B, 1, H, D), F16, 3)
    small = lib.kv4_cache(B, H, 96, D, group, weights=False, device=DEV)
    lib.kv4_append(small, k, v, lens)
    assert torch.equal(lib.kv4_attend(q, cache, lens, max_len=70), lib.kv4_attend(q, small, lens, max_len=70))


def test_attention_repeats_to_the_bit_on_another_stream_and_in_a_graph(lib):
    for S, T in ((1, 900), (40, 900), (1, 50)):
        cache, k, v = _filled(lib, 2, 3, T, 128, 64, BF16, 3, cap=1024)
        q = _rand((2, S, 3, 128), BF16, 4)
        lens = _ints(T, T - 7)
        first = lib.kv4_attend(q, cache, lens, weight_out=cache.weight.clone())
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            other = lib.kv4_attend(q, cache, lens, weight_out=cache.weight.clone())
        torch.cuda.current_stream().wait_stream(s)
        assert torch.equal(first, other)
        # a captured step: append, attend with the weights in place, evict; replayed while the sentences grow
        def step(c, kk, vv, n, nxt, out, ws, ws2):
            lib.kv4_append(c, kk, vv, n, next_pos=nxt)
            lib.kv4_attend(q, c, n, out=out, weight_out=c.weight, ws=ws)
            lib.kv4_evict(c, n, nxt, T + 3, 16, ws=ws2)
        caches, outs, counts = [], [], []
        for _ in range(2):
            c, _, _ = _filled(lib, 2, 3, T, 128, 64, BF16, 3, cap=1024)
            caches.append(c)
            outs.append(torch.zeros_like(q))
            counts.append((lens.clone(), lens.clone()))
        ws = torch.zeros(lib.kv4_attend_workspace_size(cache, S, 3, 1024, True), dtype=torch.uint8, device=DEV)
        ws2 = torch.zeros(lib.kv4_evict_workspace_size(cache, 1024, T + 3), dtype=torch.uint8, device=DEV)
        kk, vv = _rand((2, 1, 3, 128), BF16, 5), _rand((2, 1, 3, 128), BF16, 6)
        graph = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph):
            for n in counts[1]:
                n.add_(1)
            step(caches[1], kk, vv, *counts[1], outs[1], ws, ws2)
        for i in range(6):
            kk.copy_(_rand((2, 1, 3, 128), BF16, 50 + i))
            for n in counts[0]:
                n.add_(1)
            step(caches[0], kk, vv, *counts[0], outs[0], None, None)
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(outs[0], outs[1]) and torch.equal(caches[0].weight, caches[1].weight)
            assert torch.equal(caches[0].pos, caches[1].pos) and torch.equal(counts[0][0], counts[1][0])


def test_one_workspace_serves_calls_of_other_sizes(lib):
    """Whatever the last call left in it."""
    calls = []
    for B, H, G, T, S, D, group, dtype in ((1, 2, 1, 900, 1, 64, 64, F16), (3, 40, 1, 700, 1, 128, 64, BF16),
                                           (1, 1, 8, 3000, 1, 128, 128, F16), (1, 3, 1, 800, 40, 128, 32, F16),
                                           (2, 2, 2, 1500, 100, 64, 32, BF16), (1, 2, 1, 20, 1, 64, 64, F32)):
        cache, _, _ = _filled(lib, B, H, T, D, group, dtype, T)
        calls.append((cache, _rand((B, S, H * G, D), dtype, S), _ints(*[T - 5 * b for b in range(B)])))
    alone = [lib.kv4_attend(q, c, n, weight_out=torch.empty_like(c.weight)) for c, q, n in calls]
    need = max(lib.kv4_attend_workspace_size(c, q.shape[1], q.shape[2], c.cap, True) for c, q, _ in calls)
    ws = torch.full((need,), 0xff, dtype=torch.uint8, device=DEV)
    for i in (0, 1, 2, 3, 4, 5, 2, 1, 0, 4, 3, 1, 5):
        c, q, n = calls[i]
        assert torch.equal(lib.kv4_attend(q, c, n, weight_out=torch.empty_like(c.weight), ws=ws), alone[i]), i
        assert torch.equal(lib.kv4_attend(q, c, n, ws=ws), alone[i]), i


def test_many_sentences_of_very_different_lengths(lib):
    """Pieces of the slots are found by length: one long sentence among short ones, and more sentences than lanes."""
    g = torch.Generator().manual_seed(3)
    lens = torch.randint(0, 40, (70,), generator=g).tolist()
    lens[33], lens[69], lens[5] = 2000, 700, 0
    _check_attend(lib, 70, 1, 1, 2000, 1, 64, 64, F16, lens=lens)
    _check_attend(lib, 4, 3, 4, 2500, 1, 128, 64, BF16, lens=[3, 2500, 0, 90])
    _check_attend(lib, 3, 1, 2, 1500, 40, 64, 32, F16, lens=[1500, 20, 333])


@pytest.mark.parametrize("qstd", [0.2, 1.5])
@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("H,S", [(32, 520), (390, 1)])
def test_sums_over_a_long_context_that_is_not_split(lib, H, S, dtype, qstd):
    """Results shrink as slots average out, and what the codes' offsets add up to does not: errors against the results' own size, at
    calls of so many workgroups that one wave (prompts), or four (single tokens), sum a row's whole context.

    16-bit results: rounding the exact ones is an error r, and the sums may add a quarter of that, independent of it: sqrt(1 + 1/16) r.
    fp32: the codes' 7.5 on average and the lowest values below them cancel, which 4 steps of 32 slots hold until they are put
    together; there they are up to 30 times what the slots' values come to at random, in four roundings of 2^-24 / 2: 3.6e-6, twice that
    allowed, and 2^-20 for logits and probabilities."""
    T, D, group = 16384, 64, 64
    g = torch.Generator(device=DEV)
    g.manual_seed(H + S)
    rand = lambda *shape: torch.randn(*shape, generator=g, device=DEV).to(dtype)  # noqa: E731
    cache = _dirty(lib.kv4_cache(1, H, T, D, group, weights=False, device=DEV))
    k, v = rand(1, T, H, D), rand(1, T, H, D)
    lib.kv4_append(cache, k, v, _ints(T))
    q = (qstd * torch.randn(1, S, H, D, generator=g, device=DEV)).to(dtype)
    out = lib.kv4_attend(q, cache, _ints(T))
    got, want = [], []
    for h in np.linspace(0, H - 1, 2 if S > 1 else 8).astype(int):
        hk, hv = (orc.held_values(f64(t[0, :, h]), group) for t in (k, v))
        for s in sorted({0, 1, S // 3, S // 2, S - 9, S - 1} & set(range(S))):
            n = T - S + s + 1
            z = D ** -0.5 * (hk[:n] @ f64(q[0, s, h]))
            p = np.exp(z - z.max())
            want.append(p @ hv[:n] / p.sum())
            got.append(f64(out[0, s, h]))
    got, want = np.array(got), np.array(want)
    rms = lambda t: np.sqrt(np.mean(t ** 2))  # noqa: E731
    rounding = rms(f64(torch.from_numpy(want).to(dtype)) - want)
    allowed = (7.2e-6 + 2.0 ** -20) * rms(want) if dtype == F32 else np.sqrt(1 + 1 / 16) * rounding
    print(f"H {H} S {S} {dtype} qstd {qstd}: error {rms(got - want) / rms(want):.2e}, allowed {allowed / rms(want):.2e}, rounding {rounding / rms(want):.2e}")
    assert rms(got - want) <= allowed


@pytest.mark.parametrize("D,group", [(128, 64), (128, 128), (64, 32)])
@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("S", [1, 40])
def test_weights_of_16_bit_queries_keep_their_bits(lib, S, dtype, D, group):
    """The fp32 weights that the slots get.  Logits of 16-bit queries multiply codes with an offset of 16, sums of about 24 instead of 9 where
    the same queries in fp32 multiply the codes, and that is one part of a probability's error: at most 24 / 9 of it."""
    T, H = 2048, 4
    cache, k, v = _filled(lib, 1, H, T, D, group, dtype, 7)
    q = _rand((1, S, H, D), dtype, 9)
    _, _, want = orc.attend(f64(q), k, v, [T], D ** -0.5)
    err = []
    for x in (q, q.float()):
        cache.weight.zero_()
        lib.kv4_attend(x, cache, _ints(T), weight_out=cache.weight)
        err.append(np.sqrt(np.mean(((f64(cache.weight) - want) / want) ** 2)))
    print(f"S {S} {dtype} {D} {group}: error {err[0]:.2e}, of the same queries in fp32 {err[1]:.2e}")
    assert err[1] <= 2.0 ** -20 and err[0] <= 24 / 9 * err[1]


def test_weights_of_many_rows_of_more_than_2_to_the_31_slots(lib):
    """A workgroup has 128 slots of a head: more threads than 32 bits count.  All slots are alike, so each row gives every one that it sees
    the same weight."""
    H, cap, D, group, S = 129, 16777216, 64, 64, 20
    if torch.cuda.mem_get_info()[0] < 190 << 30:
        pytest.skip("180 GB of device memory are not free")
    cache = lib.kv4_cache(1, H, cap, D, group, device=DEV)
    for t in (cache.k, cache.v, cache.k_scale, cache.v_scale):
        t.zero_()
    lib.kv4_attend(_rand((1, S, H, D), F16, 3), cache, _ints(cap), weight_out=cache.weight)
    rows = torch.full((cap,), float(S), device=DEV)
    rows[cap - S:] = torch.arange(S, 0, -1, device=DEV)
    off = max((cache.weight[0, h] * cap - rows).abs().max().item() for h in range(H))
    del cache
    torch.cuda.empty_cache()
    assert off <= S * 2.0 ** -16      # log-sums of 24: 2^-20 of each of S weights, and rows that see up to 20 slots fewer


# ----------------------------------------------------------------------------------------------------- eviction

def _check_evict(lib, B, H, T, D, group, budget, recent, lens=None, weight=None, pos=None, nxt=None, alias=True, max_len=None,
                 seed=0):
    cache, k, v = _filled(lib, B, H, T, D, group, F16, seed)
    lens = [T] * B if lens is None else lens
    g = torch.Generator(device="cpu")
    g.manual_seed(seed)
    if weight is None:
        weight = torch.rand(B, H, T, generator=g) ** 4
        weight[torch.rand(B, H, T, generator=g) < 0.4] = 0.0
    pos = torch.arange(T, dtype=torch.int32).expand(B, H, T) if pos is None else pos
    nxt = lens if nxt is None else nxt
    cache.weight[:, :, :T] = weight.to(DEV)
    cache.pos[:, :, :T] = pos.to(DEV)
    w_in, p_in = cache.weight.cpu().numpy().copy(), cache.pos.cpu().numpy().copy()
    max_len = max_len or T
    n, nx = _ints(*lens), _ints(*nxt)
    if alias:
        wo, po, lo = cache.weight, cache.pos, n
        lib.kv4_evict(cache, n, nx, budget, recent, max_len=max_len)
    else:
        wo, po, lo = torch.full_like(cache.weight, 9.0), torch.full_like(cache.pos, 9), torch.full_like(n, 9)
        lib.kv4_evict(cache, n, nx, budget, recent, max_len=max_len, weight_out=wo, pos_out=po, lens_out=lo)
        assert np.array_equal(cache.weight.cpu().numpy(), w_in, equal_nan=True) and np.array_equal(cache.pos.cpu().numpy(), p_in)
    used = [min(max(x, 0), max_len) for x in lens]
    left = [min(x, budget) for x in used]
    assert lo.tolist() == left
    gk, gv = (t.cpu().numpy() for t in lib.kv4_read(cache, _ints(*left), 0, min(budget, cache.cap), F32))
    want_w, want_p = (w_in.copy(), p_in.copy()) if alias else (np.full_like(w_in, 9.0), np.full_like(p_in, 9))
    for b in range(B):
        for h in range(H):
            src = orc.evict_head(w_in[b, h], p_in[b, h], used[b], nx[b].item(), budget, recent)
            assert len(src) == left[b]
            want_w[b, h, :used[b]], want_p[b, h, :used[b]] = 0.0, -1
            want_w[b, h, :left[b]], want_p[b, h, :left[b]] = w_in[b, h, src], p_in[b, h, src]
            assert np.array_equal(gk[b, h, :left[b]], k[b, h, src].astype(np.float32))
            assert np.array_equal(gv[b, h, :left[b]], v[b, h, src].astype(np.float32))
    assert np.array_equal(wo.cpu().numpy(), want_w, equal_nan=True) and np.array_equal(po.cpu().numpy(), want_p)


@pytest.mark.parametrize("alias", [True, False])
@pytest.mark.parametrize("D,group", SHAPES)
def test_eviction(lib, D, group, alias):
    for T, budget, recent in ((2, 1, 0), (33, 32, 8), (100, 99, 99), (100, 30, 10), (100, 1, 1), (300, 150, 0), (90, 90, 3), (90, 200, 5)):
        _check_evict(lib, 2, 3, T, D, group, budget, recent, alias=alias, seed=T)


def test_eviction_of_ragged_sentences(lib):
    _check_evict(lib, 6, 2, 500, 64, 32, 100, 20, lens=[500, 0, 100, 101, 57, -4])
    _check_evict(lib, 3, 2, 500, 64, 32, 100, 20, lens=[500, 300, 900], max_len=400, nxt=[500, 300, 900])


def test_eviction_of_equal_negative_infinite_and_nan_weights(lib):
    T = 200
    w = torch.zeros(4, 2, T)
    w[1] = 0.25
    w[2] = torch.randn(2, T, generator=torch.Generator().manual_seed(3))
    w[2, 0, ::7], w[2, 1, 50:90] = float("nan"), float("inf")
    w[2, 1, 3:9], w[2, 1, 100:120] = float("-inf"), -0.0
    w[3, :, ::3] = float("nan")
    for budget in (1, 7, 100, 199):
        _check_evict(lib, 4, 2, T, 64, 64, budget, 0, weight=w)
        _check_evict(lib, 4, 2, T, 64, 64, budget, min(budget, 40), weight=w)


def test_eviction_goes_by_positions_where_slots_are_out_of_order(lib):
    g = torch.Generator().manual_seed(5)
    T = 257
    pos = torch.stack([torch.stack([torch.randperm(1000, generator=g)[:T] for _ in range(2)]) for _ in range(2)]).to(torch.int32)
    _check_evict(lib, 2, 2, T, 64, 32, 120, 60, pos=pos, nxt=[1000, 990])
    _check_evict(lib, 2, 2, T, 64, 32, 20, 20, pos=pos, nxt=[1000, 990])     # more recent ones than the budget
    _check_evict(lib, 2, 2, T, 64, 32, 120, 60, pos=pos, nxt=[5000, 0])      # none and all


@pytest.mark.parametrize("T", [5, 70, 1000, 2049, 3000])
def test_eviction_of_few_slots(lib, T):
    """One to five slots more than the budget, with the lowest among the last slots, equal, recent, NaN or zero."""
    for gone in (1, 2, 3, 4, 5):
        budget = T - gone
        if budget < 1:
            continue
        w = torch.rand(4, 2, T, generator=torch.Generator().manual_seed(T + gone))
        w[1] = 0.5                                   # all equal: the last slots leave
        w[2, :, budget:] = 0.0                       # the last slots leave
        w[3, 0, ::2], w[3, 1, : T // 2] = float("nan"), 0.0
        for recent in (0, 1, budget // 2, budget):
            for alias in (True, False):
                _check_evict(lib, 4, 2, T, 64, 64, budget, recent, weight=w, alias=alias, lens=[T, T, T - 1 if gone > 1 else T, T])


def test_eviction_writes_lengths_over_what_it_reads(lib):
    """lens_out over lens or over the positions, with few and with many moves: every head goes by what was there before."""
    B, H, T = 2, 70, 300
    for budget in (299, 20):
        got = []
        for over in ("apart", "lens", "next"):
            cache, _, _ = _filled(lib, B, H, T, 64, 64, F16, 1)
            cache.weight[:, :, :T] = _rand((B, H, T), F32, 2).abs()
            n, nx, left = _ints(T, T - 1), _ints(T, T), _ints(0, 0)
            out = {"apart": left, "lens": n, "next": nx}[over]
            lib.kv4_evict(cache, n, nx, budget, 10, max_len=T, lens_out=out)
            assert out.tolist() == [min(T, budget), min(T - 1, budget)]
            got.append((cache.pos.clone(), cache.weight.clone()))
        for pos, weight in got[1:]:
            assert torch.equal(pos, got[0][0]) and torch.equal(weight, got[0][1])


@pytest.mark.parametrize("T", [9000, 33000])
def test_eviction_of_long_caches(lib, T):
    """From 40960 bytes of keys on the launch asks for its LDS, beyond 32768 slots the keys are formed again."""
    w = (torch.rand(1, 2, T, generator=torch.Generator().manual_seed(1)) * 500).floor() / 500    # many equal
    for budget in (2048, T - 1):
        _check_evict(lib, 1, 2, T, 64, 64, budget, 64, weight=w)


@pytest.mark.parametrize("D,group", [(64, 64), (128, 32)])
@pytest.mark.parametrize("T,budget", [(32768, 32767), (32769, 32768), (33000, 32999), (33000, 32990), (33000, 256), (33000, 100)])
def test_eviction_of_few_slots_of_long_caches_into_other_lengths(lib, T, budget, D, group):
    """Few moves, and lengths apart from what is read, on both sides of the 32768 slots whose keys fit the LDS."""
    w = (torch.rand(1, 2, T, generator=torch.Generator().manual_seed(T + budget)) * 500).floor() / 500    # many equal
    _check_evict(lib, 1, 2, T, D, group, budget, 64, weight=w, alias=False)


def test_eviction_without_lengths(lib):
    """lens_out NULL, which is apart from everything: the same slots stay as where the lengths are written."""
    for T, budget in ((300, 299), (300, 50), (3000, 700), (33000, 32999), (33000, 200)):
        got = []
        for written in (True, False):
            cache, _, _ = _filled(lib, 1, 2, T, 64, 32, F16, 4)
            cache.weight[:, :, :T] = _rand((1, 2, T), F32, 5).abs()
            n, out = _ints(T), _ints(0)
            wo, po = torch.full_like(cache.weight, 9.0), torch.full_like(cache.pos, 9)
            ws = torch.full((lib.kv4_evict_workspace_size(cache, T, budget),), 0xff, dtype=torch.uint8, device=DEV)
            status = lib.raw.coreinfer_kv4_evict(ctypes.byref(cache.desc), n.data_ptr(), n.data_ptr(), T, budget, 9, wo.data_ptr(), po.data_ptr(),
                                                 out.data_ptr() if written else None, ws.data_ptr(), ws.numel(),
                                                 torch.cuda.current_stream().cuda_stream)
            assert status == lib.CI_OK and out.item() == (budget if written else 0)
            got.append((wo, po, *lib.kv4_read(cache, _ints(budget), 0, budget, F32)))
        for a, b in zip(*got):
            assert torch.equal(a, b)
