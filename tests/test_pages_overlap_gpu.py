"""Results beside, between and over the rows that they come from: refused where they share an element, right where they do not."""

import random

import pytest
import torch

from tests.test_kvp_gpu import DEV, F16, _cache, _fill, _ints, _rand

pytestmark = pytest.mark.gpu


def _at(at, strides, T, H, D):
    return {at + i * strides[0] + j * strides[1] + d for i in range(T) for j in range(H) for d in range(D)}


def _views(rng, D, step):
    """Rows within one buffer, and others of a kind of their own: a block, the same strides, or others."""
    T, H = rng.choice([1, 1, 2, 5]), rng.choice([1, 2, 4])
    inner = D + step * rng.choice([0, 0, 1, 9, 40])
    strides = (H * inner + step * rng.choice([0, 0, 3, 50]), inner)
    if rng.random() < 0.3:
        strides = (inner, T * inner + step * rng.choice([0, 2, 60]))
    reach = (T - 1) * strides[0] + (H - 1) * strides[1] + D
    return T, H, strides, reach


def test_rotations_within_one_buffer(lib):
    D, N = 16, 6000
    rng, angles = random.Random(1), lib.rope_angles(D, device=DEV)
    refused = passed = between = 0
    for _ in range(600):
        T, H, strides, reach = _views(rng, D, 1)
        block = (H * D, D)
        ys = strides if rng.random() < 0.5 else block
        x_at = rng.randrange(2000, 3000)
        y_at = x_at + (0 if rng.random() < 0.1 else rng.randrange(-reach - 40, reach + 40))
        buf = _rand((N,), F16, 3)
        x, y = buf.as_strided((T, H, D), (*strides, 1), x_at), buf.as_strided((T, H, D), (*ys, 1), y_at)
        a, b = _at(x_at, strides, T, H, D), _at(y_at, ys, T, H, D)
        same = x_at == y_at and all(n == 1 or s == t for n, s, t in zip((T, H), strides, ys))
        pos = _ints(*range(5, 5 + T))
        want, before = lib.rope(x.clone(), pos, angles), buf.clone()
        if a & b and not same:
            refused += 1
            with pytest.raises(lib.CoreInferError) as e:
                lib.rope(x, pos, angles, out=y)
            assert e.value.status == lib.CI_ERR_BAD_LAYOUT and torch.equal(buf, before)
        else:
            passed += 1
            between += min(b) < max(a) and min(a) < max(b)
            assert torch.equal(lib.rope(x, pos, angles, out=y), want)
            kept = torch.ones(N, dtype=torch.bool)
            kept[list(b)] = False
            assert torch.equal(buf.cpu()[kept], before.cpu()[kept])
    assert refused > 100 and passed > 100 and between > 20


def test_attention_and_appends_within_one_buffer(lib):
    D, N = 64, 20000
    rng = random.Random(2)
    refused = passed = between = 0
    for _ in range(300):
        T, H, strides, reach = _views(rng, D, 8)
        at = 8 * rng.randrange(800, 900)
        out_at = at + 8 * rng.randrange(-(T * H * D) // 8 - 8, reach // 8 + 8)
        buf = _rand((N,), F16, 4)
        q, out = buf.as_strided((T, H, D), (*strides, 1), at), buf.as_strided((T, H, D), (H * D, D, 1), out_at)
        a, b = _at(at, strides, T, H, D), set(range(out_at, out_at + T * H * D))
        cache, table = _cache(lib, H, 16, D, F16, [20], 1)
        _fill(cache, table, [20], 2)
        first, lens = _ints(0, T), _ints(20)
        k, v = _rand((T, H, D), F16, 5), _rand((T, H, D), F16, 6)
        before = buf.clone()
        for call in (lambda q, out: lib.kvp_attend(q, cache, first, lens, out=out), lambda q, out: lib.kvp_append(cache, k, v, first, lens, q=q, q_out=out)):
            buf.copy_(before)
            if a & b:
                refused += 1
                with pytest.raises(lib.CoreInferError) as e:
                    call(q, out)
                assert e.value.status == lib.CI_ERR_BAD_LAYOUT and torch.equal(buf, before)
            else:
                passed += 1
                between += min(b) < max(a) and min(a) < max(b)
                want = call(q.clone(), torch.empty((T, H, D), dtype=F16, device=DEV))
                assert torch.equal(call(q, out), want)
    assert refused > 50 and passed > 50 and between > 5
