"""The 4-bit operators together: decode steps of one layer, replayed from a graph, against the plain definitions."""

import numpy as np
import pytest
import torch

from oracle import q4_oracle as orc
from tests._util import f64

pytestmark = pytest.mark.gpu


def test_steps_of_a_layer_follow_the_definitions(lib):
    """Every replayed step, from the cache and the lengths it found: attention over what the cache holds, the slots that stay, and the FFN over
    the packed core neurons.  Rounding to bf16 between the steps is the path's own, so each product is compared from its own inputs."""
    from examples import decode_4bit as ex
    B, T, heads, D, N, group, budget, recent = 3, 40, 2, 64, 256, 32, 36, 8
    layer = ex.Layer(heads, D, N, torch.bfloat16, group)
    dec = ex.Decoder(layer, B, 64, budget, recent)
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    out, core = dec.prompt(torch.randn(B, T, layer.d, generator=g, device="cuda").to(torch.bfloat16), 0.2, 0.4)
    assert core.numel() == lib.keep_count(0.4, N) and dec.lens.tolist() == [budget] * B and dec.positions.tolist() == [T] * B
    c, x = dec.cache, out[:, -1].clone()
    w = {n: f64(lib.w4_read(getattr(layer, n), torch.float32)) for n in ("qkv", "out", "core_up", "core_gate", "core_down")}
    for step in range(6):
        old_k, old_v = (f64(t) for t in lib.kv4_read(c, dec.lens, 0, budget, torch.float32))
        old_weight, old_pos = f64(c.weight), c.pos.cpu().numpy()
        y = f64(dec.token(x).clone())
        assert dec.lens.tolist() == [budget] * B and dec.positions.tolist() == [T + 1 + step] * B
        # the same step in float64, from rows rounded where the path rounds them
        bf = lambda t: f64(torch.from_numpy(t).to(torch.bfloat16))  # noqa: E731
        nx = f64(ex.norm(x))
        qkv = bf(nx @ w["qkv"].T).reshape(B, 3, heads, D)
        k, v = (np.concatenate([old, orc.held_values(qkv[:, i], group)[:, :, None]], 2) for i, old in ((1, old_k), (2, old_v)))
        o, _, add = orc.attend(qkv[:, None, 0], k, v, [budget + 1] * B, D ** -0.5)
        a = bf(f64(x) + bf(bf(o[:, 0]).reshape(B, layer.d) @ w["out"].T))
        n = bf(a / np.sqrt((a ** 2).mean(-1, keepdims=True) + 1e-5))
        hidden = orc.matvec(n, w["core_up"], w["core_gate"], None, "swiglu")
        want = a + bf(hidden @ w["core_down"].T)
        # eight roundings to bf16 in a row, 2^-9 of values of the size of the largest; a rounding that falls the other way moves a code
        assert np.abs(y - want).max() <= 8 * 2.0 ** -9 * max(1.0, np.abs(want).max())
        # what stays: the weights and positions of the evicted cache are a subset of those before, the smallest weight gone
        new_weight, new_pos = f64(c.weight), c.pos.cpu().numpy()
        for b in range(B):
            for h in range(heads):
                before = np.append(old_weight[b, h, :budget] + add[b, h, :budget], add[b, h, budget])
                pos = np.append(old_pos[b, h, :budget], T + step)
                src = orc.evict_head(before, pos, budget + 1, T + 1 + step, budget, recent)
                gone = set(pos.tolist()) - set(new_pos[b, h, :budget].tolist())
                assert len(gone) == 1
                lost = before[pos.tolist().index(gone.pop())]
                expected = before[list(set(range(budget + 1)) - set(src))[0]]
                assert abs(lost - expected) <= 0.02 * max(expected, 0.01)      # another slot only where the two are as good as equal
                assert abs(new_weight[b, h, :budget].sum() - (before.sum() - lost)) <= 0.02
        x = torch.from_numpy(y).to(torch.bfloat16).to("cuda")
