"""Decode steps of one gated decoder layer with everything a token reads in 4 bits: projections, key-value cache and deployed
core neurons.

    python examples/decode_4bit.py [--sentences B] [--prompt T] [--tokens N] [--budget S] [--recent R]

The prompt goes through the projections and fills the cache, its attention adds up what weight every slot gets, the dense FFN's
hidden values choose the core neurons, and those are deployed and packed.  Every token then takes one pass: q, k and v from
4-bit weights, the cache's append, attention, eviction of the slot with the least weight where the cache is over its budget, the output
projection, and the FFN over the core neurons as two products with fp32 hidden values between them.  The step is captured in a HIP
graph once and replayed; lengths live on the device.  Inputs and weights are random, of the shape of a layer of Llama-2-7B by default.
"""

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2410_18311_amd import coreinfer as ci  # noqa: E402


class Layer:
    """Random weights of a layer: d = heads x D, N neurons; packed in 4 bits, the FFN's dense ones kept for the prompt."""

    def __init__(self, heads, D, N, dtype, group, seed=0):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        d = heads * D
        rand = lambda r, c: (torch.randn(r, c, generator=g, device="cuda") * 0.02).to(dtype)  # noqa: E731
        self.heads, self.D, self.d, self.N, self.dtype, self.group = heads, D, d, N, dtype, group
        self.qkv, self.out = ci.w4_quantize(rand(3 * d, d), group), ci.w4_quantize(rand(d, d), group)
        self.up, self.gate, self.down = rand(N, d), rand(N, d), rand(d, N)

    def deploy(self, hidden, alpha, beta):
        """Core neurons of a prompt from its hidden values [M, N]: selected, gathered and packed."""
        core, _ = ci.select_hidden(hidden, "swiglu", alpha, beta)
        c = ci.compact(self.up, self.gate, None, self.down, "out_major", "swiglu", core, down_c_layout="out_major")
        self.core_up, self.core_gate = ci.w4_quantize(c["w_up_c"], self.group), ci.w4_quantize(c["w_gate_c"], self.group)
        self.core_down = ci.w4_quantize(c["w_down_c"][:, :core.numel()], self.group)
        return core


def norm(x):
    return (x.float() * torch.rsqrt(x.float().pow(2).mean(-1, keepdim=True) + 1e-5)).to(x.dtype)


class Decoder:
    """Buffers of B sentences and the captured step."""

    def __init__(self, layer, B, capacity, budget, recent):
        self.layer, self.budget, self.recent = layer, budget, recent
        kw = dict(dtype=torch.int32, device="cuda")
        self.cache = ci.kv4_cache(B, layer.heads, capacity, layer.D, layer.group)
        self.lens, self.positions, self.left = torch.zeros(B, **kw), torch.zeros(B, **kw), torch.zeros(B, **kw)
        self.x = torch.zeros(B, layer.d, dtype=layer.dtype, device="cuda")
        self.y = torch.zeros_like(self.x)
        self.graph = None

    def attend(self, x):
        """x [B, S, d], the sentences' next S tokens, through the attention; the cache grows by S."""
        L, (B, S, _) = self.layer, x.shape
        rows = norm(x).reshape(B * S, L.d)
        # as many rows at a time as the products take
        qkv = torch.cat([ci.w4_matvec(rows[i:i + 64], L.qkv) for i in range(0, B * S, 64)])
        q, k, v = qkv.view(B, S, 3, L.heads, L.D).unbind(2)
        self.lens.add_(S)
        self.positions.add_(S)
        ci.kv4_append(self.cache, k, v, self.lens, next_pos=self.positions)
        o = ci.kv4_attend(q, self.cache, self.lens, weight_out=self.cache.weight).view(B * S, L.d)
        out = torch.cat([ci.w4_matvec(o[i:i + 64], L.out) for i in range(0, B * S, 64)])
        return x + out.view(B, S, L.d)

    def evict(self):
        ci.kv4_evict(self.cache, self.lens, self.positions, self.budget, self.recent, lens_out=self.left)
        self.lens.copy_(self.left)

    def step(self):
        L = self.layer
        x = self.attend(self.x[:, None])[:, 0]
        self.evict()
        h = ci.w4_matvec(norm(x), L.core_up, gate=L.core_gate, act="swiglu", out_dtype=torch.float32)
        self.y.copy_(x + ci.w4_matvec(h, L.core_down, out_dtype=L.dtype))

    def prompt(self, x, alpha, beta):
        """x [B, T, d]: attention, dense FFN, core neurons of the first sentence's prompt for all."""
        L, (B, T, _) = self.layer, x.shape
        a = self.attend(x)
        Y, H = ci.ffn_dense_hidden(norm(a).reshape(B * T, L.d), L.up, L.gate, None, L.down, None, "out_major", "swiglu")
        core = L.deploy(H[:T], alpha, beta)
        self.evict()
        return a + Y.view(B, T, L.d), core

    def token(self, x):
        self.x.copy_(x)
        if self.graph is None:
            state = [t.clone() for t in (self.lens, self.positions)]
            side = torch.cuda.Stream()
            side.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(side):   # what a first call allocates
                keep = [t.clone() for t in (self.cache.k, self.cache.v, self.cache.k_scale, self.cache.v_scale, self.cache.weight,
                                            self.cache.pos)]
                self.step()
                for t, old in zip((self.cache.k, self.cache.v, self.cache.k_scale, self.cache.v_scale, self.cache.weight,
                                   self.cache.pos), keep):
                    t.copy_(old)
                self.lens.copy_(state[0])
                self.positions.copy_(state[1])
            torch.cuda.current_stream().wait_stream(side)
            self.graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(self.graph):
                self.step()
        self.graph.replay()
        return self.y


def main(argv=None):
    p = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, value in (("sentences", 4), ("prompt", 512), ("tokens", 64), ("budget", 384), ("recent", 96), ("heads", 32), ("channels", 128),
                        ("neurons", 11008), ("group", 64)):
        p.add_argument("--" + name, type=int, default=value)
    a = p.parse_args(argv)
    layer = Layer(a.heads, a.channels, a.neurons, torch.bfloat16, a.group)
    dec = Decoder(layer, a.sentences, -(-(max(a.prompt, a.budget) + 1) // 32) * 32, a.budget, a.recent)
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    out, core = dec.prompt(torch.randn(a.sentences, a.prompt, layer.d, generator=g, device="cuda").to(torch.bfloat16), 0.2, 0.4)
    y = dec.token(out[:, -1])
    start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    start.record()
    for _ in range(a.tokens - 1):
        y = dec.token(y)
    end.record()
    torch.cuda.synchronize()
    us = start.elapsed_time(end) * 1e3 / max(a.tokens - 1, 1)
    print(f"{a.sentences} sentences, prompt {a.prompt}, {core.numel()} of {a.neurons} neurons deployed, slots in use {dec.lens.tolist()}, "
          f"tokens so far {dec.positions.tolist()}: {us:.1f} us a step of one layer")
    return y, dec


if __name__ == "__main__":
    main()
