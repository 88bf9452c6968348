"""The operators of a 16-bit (or fp32) cache in pages that their performance is judged by: sizes, inputs, plain forms and 64-bit results.

A decoder layer that serves several sentences at once takes their new tokens packed one behind the other, a prompt's chunk beside other
sentences' single tokens.  Queries and keys are normed by head and turned by their positions, keys and values go to the pages that
a sentence has been given, and every new token attends over its sentence's pages, to all of it or to a sliding window and the
first few tokens.  The plain forms do that with elementary torch operations in 32 bits, angles in 64.
"""

import math

import torch

own = False

DEV = "cuda:0"
DTYPE = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
ELEM = {"f32": 4, "f16": 2, "bf16": 2}
BASE = 10000.0
EPS = 1e-6
# context that the frequencies were made for, and by how much it is stretched, where they are scaled
ORIGINAL, FACTOR, FAST, SLOW = 4096, 4.0, 32.0, 1.0


def _ci():
    from paper_2410_18311_amd import coreinfer
    return coreinfer


def listed():
    return [
        # queries of one token: the smallest call, latency is all of it
        dict(name="rope_token", kind="rope", dtype="f16", T=1, H=32, D=128, rot=128, style="half", scaling="none", norm=False,
             backward=False, far=4096),
        # queries of a prompt with head norms, frequencies scaled for a longer context
        dict(name="rope_prompt_4096", kind="rope", dtype="bf16", T=4096, H=40, D=128, rot=128, style="half", scaling="parts", norm=True,
             backward=False, far=16384),
        # gradient of half of each head's channels, pairs of neighbours, fp32, far positions
        dict(name="rope_part_f32_back", kind="rope", dtype="f32", T=777, H=72, D=128, rot=64, style="interleaved", scaling="linear",
             norm=False, backward=True, far=1 << 20),
        # one token each of eight sentences: queries, keys and values of a layer's fused projection, keys and values to the pages
        dict(name="append_step_llama13b", kind="append", dtype="bf16", B=8, H=40, G=1, D=128, S=1, T=777, page=16, rot=128,
             style="half", scaling="none", norm=False, rows="each"),
        # the same with eight query heads to a head of the cache and head norms, 48 sentences
        dict(name="append_step_grouped", kind="append", dtype="f16", B=48, H=8, G=8, D=128, S=1, T=1025, page=64, rot=128,
             style="half", scaling="parts", norm=True, rows="each"),
        # chunks of prompts of four sentences, an idle one among them
        dict(name="append_prompts_2048", kind="append", dtype="f16", B=4, H=32, G=1, D=128, S=2048, T=2048, page=16, rot=128,
             style="half", scaling="none", norm=True, rows="ragged"),
        # one token after a short question
        dict(name="attend_step_77", kind="attend", dtype="f16", B=1, H=32, G=1, D=128, S=1, T=77, page=16, window=0, sinks=0,
             rows="each"),
        # one token after a long prompt
        dict(name="attend_step_4096", kind="attend", dtype="bf16", B=1, H=40, G=1, D=128, S=1, T=4096, page=64, window=0, sinks=0,
             rows="each"),
        # one token each of eight sentences of other lengths (an idle one among them), eight query heads to a head of the
        # cache, up to 65536 slots: the most bytes
        dict(name="attend_steps_65536", kind="attend", dtype="bf16", B=8, H=8, G=8, D=128, S=1, T=65536, page=256, window=0, sinks=0,
             rows="ragged"),
        # a whole prompt: the most operations
        dict(name="attend_prompt_4096", kind="attend", dtype="f16", B=1, H=32, G=1, D=128, S=4096, T=4096, page=16, window=0,
             sinks=0, rows="each"),
        # a chunk of a long prompt that sees the last 4096 tokens and the first four
        dict(name="attend_chunk_window", kind="attend", dtype="bf16", B=1, H=8, G=4, D=128, S=512, T=16384, page=64, window=4096,
             sinks=4, rows="each"),
        # a prompt's chunk beside single tokens of seven sentences, smaller heads, an odd number of rows
        dict(name="attend_mixed_8192", kind="attend", dtype="f16", B=8, H=16, G=2, D=64, S=777, T=8192, page=16, window=0, sinks=0,
             rows="mixed"),
    ]


def _log(rng, lo, hi, step=1):
    """A size between lo and hi, even over the logarithm, rounded to a multiple of step."""
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return max(lo, min(hi, int(round(v / step)) * step))


def draw(rng):
    """One more case, of no more bytes and no more operations than the largest listed ones."""
    most = {n: max(work(c)[n] for c in listed()) for n in ("bytes", "flops")}
    while True:
        c = _draw(rng)
        if all(work(c)[n] <= most[n] for n in most):
            return c


def _draw(rng):
    kind = rng.choice(["rope", "rope", "append", "append", "attend", "attend", "attend", "attend"])
    dtype = rng.choice(["f16", "f16", "bf16", "bf16", "f32"])
    D = rng.choice([64, 128, 128])
    turn = dict(rot=rng.choice([D, D, D // 2, D // 4]), style=rng.choice(["half", "half", "interleaved"]),
                scaling=rng.choice(["none", "none", "linear", "base", "parts"]))
    norm = rng.random() < 0.4
    if kind == "rope":
        return dict(kind=kind, dtype=dtype, T=_log(rng, 1, 8192), H=rng.choice([4, 8, 32, 40, 72]), D=D, **turn, norm=norm,
                    backward=not norm and rng.random() < 0.3, far=_log(rng, 1 << 13, 1 << 20))
    B = rng.choice([1, 1, 2, 4, 8])
    H = rng.choice([4, 8, 32, 40])
    G = rng.choice([1, 4, 8]) if H <= 8 else 1
    page = rng.choice([16, 16, 32, 64, 128, 256])
    rows = rng.choice(["each", "ragged", "mixed"]) if B > 1 else "each"
    if kind == "append":
        S = rng.choice([1, _log(rng, 2, 2048)])
        return dict(kind=kind, dtype=dtype, B=B, H=H, G=G, D=D, S=S, T=S + _log(rng, 1, 1024), page=page, **turn, norm=norm, rows=rows)
    S = rng.choice([1, 1, 1, _log(rng, 2, 4096)])
    T = _log(rng, S, 65536 if S <= 8 else 16384)
    window = rng.choice([0, 0, _log(rng, 16, 8192)])
    return dict(kind=kind, dtype=dtype, B=B, H=H, G=G, D=D, S=S, T=T, page=page, window=window,
                sinks=rng.choice([0, 4, _log(rng, 1, 128)]) if window else 0, rows=rows)


# ---------------------------------------------------------------------------------------------- inputs

class _Draws:
    """Tensors from one seeded generator, in the order they are asked for."""

    def __init__(self, seed):
        self.g = torch.Generator(device=DEV)
        self.g.manual_seed(int(seed))

    def randn(self, *shape, std=1.0, dtype=torch.float32):
        t = torch.randn(shape, generator=self.g, device=DEV, dtype=torch.float32)
        return (t.mul_(std) if std != 1.0 else t).to(dtype)

    def leaning(self, *shape, dtype):
        """Queries or keys: a few channels of each head are larger than the others, as projections have them."""
        big = 1.0 + 3.0 * (torch.rand(shape[-2:], generator=self.g, device=DEV) > 0.97)
        return self.randn(*shape).mul_(big).to(dtype)

    def norm(self, D, dtype):
        return (1.0 + 0.2 * torch.randn(D, generator=self.g, device=DEV)).to(dtype)

    def positions(self, c):
        """Positions of a chunk that ends before `far`, and of other sentences' tokens."""
        start = int(torch.randint(0, max(1, c["far"] - c["T"]), (1,), generator=self.g, device=DEV).item())
        p = torch.arange(start, start + c["T"], device=DEV, dtype=torch.int32)
        other = torch.randint(0, c["far"], (c["T"],), generator=self.g, device=DEV, dtype=torch.int32)
        return torch.where(torch.rand(c["T"], generator=self.g, device=DEV) < 0.25, other, p)

    def pages(self, c):
        """Which page of the pool holds which slots of which sentence, in no order; -1 where a sentence has none."""
        most, have = _table_shape(c)
        order = torch.randperm(_pool(c), generator=self.g, device=DEV, dtype=torch.int32)
        table = torch.full((c["B"], most), -1, dtype=torch.int32, device=DEV)
        at = 0
        for b, n in enumerate(have):
            table[b, :n] = order[at:at + n]
            at += n
        return table


def _lens(c):
    """Slots in use per sentence, the new tokens included: all of them, or, ragged or mixed, the full length, none, and lengths between."""
    T, B = c["T"], c["B"]
    if c["rows"] == "each":
        return [T] * B
    return [T if b == 0 else 0 if b == 1 and B >= 4 else max(1, T * (B - b) // B) for b in range(B)]


def _rows(c):
    """New tokens per sentence: S, or in a mixed batch one for all but the first."""
    return [min(n, 1 if c["rows"] == "mixed" and b else c["S"]) for b, n in enumerate(_lens(c))]


def _first(c):
    first = [0]
    for n in _rows(c):
        first.append(first[-1] + n)
    return first


def _table_shape(c):
    have = [-(-n // c["page"]) for n in _lens(c)]
    return max(have) + 1, have


def _pool(c):
    return sum(_table_shape(c)[1]) + 3


def _frequencies(c):
    """Radians a position of each pair, 64 bits, on the GPU."""
    i = torch.arange(c["rot"] // 2, dtype=torch.float64, device=DEV)
    base = BASE * FACTOR ** (c["rot"] / (c["rot"] - 2.0)) if c["scaling"] == "base" else BASE
    f = torch.pow(torch.tensor(base, dtype=torch.float64, device=DEV), -2.0 * i / c["rot"])
    if c["scaling"] == "linear":
        f = f / FACTOR
    if c["scaling"] == "parts":
        keep = ((ORIGINAL * f / (2.0 * math.pi) - SLOW) / (FAST - SLOW)).clamp(0.0, 1.0)
        f = f * keep + f / FACTOR * (1.0 - keep)
    return f


def _magnitude(c):
    return 0.1 * math.log(FACTOR) + 1.0 if c["scaling"] == "parts" else 1.0


def prepare(case, seed):
    c, r = case, _Draws(seed)
    s = {"case": c}
    dt = DTYPE[c["dtype"]]
    if c["kind"] != "attend":
        if own:
            s["angles"] = _ci().rope_angles(c["rot"], base=BASE, style=c["style"], scaling=c["scaling"], factor=FACTOR,
                                            original=ORIGINAL, fast=FAST, slow=SLOW, device=DEV)
        else:
            s["freq"] = _frequencies(c)
    if c["kind"] == "rope":
        # the queries of a fused projection whose keys and values lie behind them
        fused = torch.zeros((c["T"], c["H"] + 4, c["D"]), dtype=dt, device=DEV)
        s["x"] = fused[:, :c["H"]]
        s["x"].copy_(r.leaning(c["T"], c["H"], c["D"], dtype=dt))
        s["norm"] = r.norm(c["D"], dt) if c["norm"] else None
        s["pos"] = r.positions(c)
        if own:
            s["out"] = torch.empty((c["T"], c["H"], c["D"]), dtype=dt, device=DEV)
        return s
    H, G, D, n = c["H"], c["G"], c["D"], _first(c)[-1]
    s["table"] = r.pages(c)
    s["lens"] = torch.tensor(_lens(c), dtype=torch.int32, device=DEV)
    s["first"] = torch.tensor(_first(c), dtype=torch.int32, device=DEV)
    pages = [r.leaning(_pool(c), H, c["page"], D, dtype=dt) for _ in range(2)]
    if own:
        s["cache"] = cache = _ci().kvp_cache(_pool(c), H, c["page"], D, dt, s["table"])
        cache.k.copy_(pages[0])
        cache.v.copy_(pages[1])
    else:
        s["k_pages"], s["v_pages"] = pages
    if c["kind"] == "append":
        fused = r.leaning(n, (G + 2) * H, D, dtype=dt)
        s["q"], s["k"], s["v"] = fused[:, :G * H], fused[:, G * H:(G + 1) * H], fused[:, (G + 1) * H:]
        s["q_norm"], s["k_norm"] = (r.norm(D, dt) if c["norm"] else None for _ in range(2))
        if own:
            s["q_out"] = torch.empty((n, G * H, D), dtype=dt, device=DEV)
        else:
            s["where"] = _where(c)
        return s
    s["q"] = r.leaning(n, G * H, D, dtype=dt)
    if own:
        s["out"] = torch.empty_like(s["q"])
        s["ws"] = torch.zeros(_ci().kvp_attend_workspace_size(s["cache"], n, G * H, max(_rows(c)), c["T"], c["window"], c["sinks"]),
                              dtype=torch.uint8, device=DEV)
    return s


# -------------------------------------------------------------------------------------- the plain forms

def _where(c):
    """Sentence and slot of every packed row."""
    b = [b for b, n in enumerate(_rows(c)) for _ in range(n)]
    t = [m - n + i for m, n in zip(_lens(c), _rows(c)) for i in range(n)]
    return torch.tensor(b, device=DEV), torch.tensor(t, device=DEV)


def _turned(c, x, norm, pos, freq, sign=1.0):
    """x [T, H, D] in 32 bits: normed by head, turned by its positions."""
    x = x.to(torch.float32)
    if norm is not None:
        x = x * (1.0 / torch.sqrt((x * x).mean(-1, keepdim=True) + EPS)) * norm.to(torch.float32)
    angle = pos.to(torch.float64)[:, None] * freq
    cos = (torch.cos(angle) * _magnitude(c)).to(torch.float32)[:, None]
    sin = (torch.sin(angle) * (sign * _magnitude(c))).to(torch.float32)[:, None]
    rot = c["rot"]
    if c["style"] == "half":
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
    else:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
    a, b = a * cos - b * sin, b * cos + a * sin
    out = torch.cat([a, b], -1) if c["style"] == "half" else torch.stack([a, b], -1).flatten(-2)
    return torch.cat([out, x[..., rot:]], -1)


def _append(s):
    c = s["case"]
    dt = s["k"].dtype
    b, t = s["where"]
    page = s["table"][b, t // c["page"]].long()
    s["k_pages"][page, :, t % c["page"]] = _turned(c, s["k"], s["k_norm"], t, s["freq"]).to(dt)
    s["v_pages"][page, :, t % c["page"]] = s["v"]
    return {"q": _turned(c, s["q"], s["q_norm"], t, s["freq"]).to(dt), "k": s["k_pages"], "v": s["v_pages"]}


def _attend(s):
    c = s["case"]
    H, G, D = c["H"], c["G"], c["D"]
    out = torch.zeros_like(s["q"])
    for b, (n, m) in enumerate(zip(_lens(c), _rows(c))):
        if m == 0 or n == 0:
            continue
        row = _first(c)[b]
        page = s["table"][b, :-(-n // c["page"])].long()
        k, v = (s[x][page].transpose(0, 1).reshape(H, -1, D)[:, :n].to(torch.float32) for x in ("k_pages", "v_pages"))
        q = s["q"][row:row + m].to(torch.float32).reshape(m, H, G, D).permute(1, 2, 0, 3).reshape(H, G * m, D)
        logits = torch.matmul(q, k.transpose(1, 2).contiguous()) * (1.0 / math.sqrt(D))
        at = torch.arange(n - m, n, device=DEV)[:, None]
        t = torch.arange(n, device=DEV)[None]
        seen = t <= at
        if c["window"]:
            seen = seen & ((t > at - c["window"]) | (t < c["sinks"]))
        logits = torch.where(seen, logits.reshape(H, G, m, n), torch.full((), -math.inf, device=DEV))
        p = torch.exp(logits - logits.amax(-1, keepdim=True))
        p = (p / p.sum(-1, keepdim=True)).reshape(H, G * m, n)
        y = torch.matmul(p, v.contiguous()).reshape(H, G, m, D).permute(2, 0, 1, 3)
        out[row:row + m] = y.reshape(m, H * G, D).to(out.dtype)
    return {"out": out}


def _plain(s):
    c = s["case"]
    if c["kind"] == "rope":
        return {"y": _turned(c, s["x"], s["norm"], s["pos"], s["freq"], -1.0 if c["backward"] else 1.0).to(s["x"].dtype)}
    return _append(s) if c["kind"] == "append" else _attend(s)


# ------------------------------------------------------------------------------------------------- run

def run(s):
    if not own:
        return _plain(s)
    ci, c = _ci(), s["case"]
    if c["kind"] == "rope":
        return {"y": ci.rope(s["x"], s["pos"], s["angles"], norm=s["norm"], eps=EPS, backward=c["backward"], out=s["out"])}
    cache = s["cache"]
    if c["kind"] == "append":
        ci.kvp_append(cache, s["k"], s["v"], s["first"], s["lens"], angles=s["angles"], k_norm=s["k_norm"], eps=EPS, q=s["q"],
                      q_norm=s["q_norm"], q_out=s["q_out"])
        return {"q": s["q_out"], "k": cache.k, "v": cache.v}
    ci.kvp_attend(s["q"], cache, s["first"], s["lens"], max_rows=max(_rows(c)), max_len=c["T"], window=c["window"],
                  sinks=c["sinks"], out=s["out"], ws=s["ws"])
    return {"out": s["out"]}


# ------------------------------------------------------------------------------------------------ work

def _pairs(n, m, window, sinks):
    """Slots that the last m of n tokens see, summed over them."""
    if not window:
        return m * n - m * (m - 1) // 2
    return sum(min(p + 1, window) + min(sinks, max(0, p + 1 - window)) for p in range(n - m, n))


def work(case):
    """Bytes that have to move (every input read once, every output written once) and operations."""
    c, e = case, ELEM[case["dtype"]]
    D = c["D"]
    if c["kind"] == "rope":
        n = c["T"] * c["H"]
        return {"bytes": 2 * n * D * e + 4 * c["T"] + (D * e if c["norm"] else 0), "flops": n * (3 * c["rot"] + (4 * D if c["norm"] else 0))}
    H, Hq, total = c["H"], c["H"] * c["G"], sum(_rows(c))
    if c["kind"] == "append":
        return {"bytes": 2 * total * (Hq + 2 * H) * D * e + (2 * D * e if c["norm"] else 0),
                "flops": total * (Hq + H) * (3 * c["rot"] + (4 * D if c["norm"] else 0))}
    slots = pairs = 0
    for n, m in zip(_lens(c), _rows(c)):
        if m == 0 or n == 0:
            continue
        low = max(0, n - m + 1 - c["window"]) if c["window"] else 0   # the first slot of the first row's window
        slots += n - low + min(low, c["sinks"])
        pairs += _pairs(n, m, c["window"], c["sinks"])
    return {"bytes": slots * H * 2 * D * e + 2 * total * Hq * D * e, "flops": 4 * D * Hq * pairs}


# ----------------------------------------------------------------------------------- 64-bit references

def _rotated64(c, x, w, pos, back=False):
    """Each pair of channels as a complex number times magnitude e^(i position frequency)."""
    x = x.to(torch.float64)
    if w is not None:
        x = x / torch.sqrt(x.square().sum(-1, keepdim=True) / c["D"] + EPS) * w.to(torch.float64)
    rot = c["rot"]
    base = BASE * math.pow(FACTOR, rot / (rot - 2.0)) if c["scaling"] == "base" else BASE
    f = [math.exp(-math.log(base) * (2 * i) / rot) for i in range(rot // 2)]
    if c["scaling"] == "linear":
        f = [v / FACTOR for v in f]
    if c["scaling"] == "parts":
        share = [min(1.0, max(0.0, (ORIGINAL / (2 * math.pi / v) - SLOW) / (FAST - SLOW))) for v in f]
        f = [v * (g + (1 - g) / FACTOR) for v, g in zip(f, share)]
    angle = pos.to(torch.float64)[:, None] * torch.tensor(f, dtype=torch.float64, device=DEV)
    turn = torch.polar(torch.full_like(angle, _magnitude(c)), -angle if back else angle)[:, None]
    y = x.clone()
    if c["style"] == "half":
        z = torch.complex(x[..., :rot // 2].contiguous(), x[..., rot // 2:rot].contiguous()) * turn
        y[..., :rot // 2], y[..., rot // 2:rot] = z.real, z.imag
    else:
        z = torch.view_as_complex(x[..., :rot].unflatten(-1, (-1, 2)).contiguous()) * turn
        y[..., :rot] = torch.view_as_real(z).flatten(-2)
    return y


def exact(case, seed):
    c, r = case, _Draws(seed)
    dt, D = DTYPE[c["dtype"]], c["D"]
    if c["kind"] == "rope":
        x = r.leaning(c["T"], c["H"], D, dtype=dt)
        w = r.norm(D, dt) if c["norm"] else None
        return {"y": _rotated64(c, x, w, r.positions(c), c["backward"])}
    H, G, page, n = c["H"], c["G"], c["page"], _first(c)[-1]
    table = r.pages(c).tolist()
    k_pages, v_pages = (r.leaning(_pool(c), H, page, D, dtype=dt).to(torch.float64) for _ in range(2))
    lens, rows = _lens(c), _rows(c)
    if c["kind"] == "append":
        fused = r.leaning(n, (G + 2) * H, D, dtype=dt)
        wq, wk = (r.norm(D, dt) if c["norm"] else None for _ in range(2))
        pos = torch.cat([torch.arange(m - i, m) for m, i in zip(lens, rows)]).to(DEV)
        q, k = _rotated64(c, fused[:, :G * H], wq, pos), _rotated64(c, fused[:, G * H:G * H + H], wk, pos)
        v = fused[:, G * H + H:].to(torch.float64)
        at = 0
        for b in range(c["B"]):
            slot = lens[b] - rows[b]
            while slot < lens[b]:                       # as far as the page goes
                count = min(page - slot % page, lens[b] - slot)
                to = (table[b][slot // page], slice(None), slice(slot % page, slot % page + count))
                k_pages[to], v_pages[to] = k[at:at + count].transpose(0, 1), v[at:at + count].transpose(0, 1)
                slot, at = slot + count, at + count
        return {"q": q, "k": k_pages, "v": v_pages}
    q = r.leaning(n, G * H, D, dtype=dt).to(torch.float64)
    out = torch.zeros_like(q)
    at = 0
    for b in range(c["B"]):
        m, i = lens[b], rows[b]
        if i:
            p = torch.arange(m - i, m, device=DEV).unsqueeze(1) - torch.arange(m, device=DEV)   # how far back a slot is
            hide = p < 0
            if c["window"]:
                hide |= (p >= c["window"]) & (torch.arange(m, device=DEV) >= c["sinks"])
            pages = table[b][:-(-m // page)]
            for h in range(H):
                kk, vv = (torch.cat([t[g, h] for g in pages])[:m] for t in (k_pages, v_pages))
                kt = kk.t().contiguous()
                for j in range(h * G, h * G + G):
                    z = (q[at:at + i, j] @ kt) / math.sqrt(D)
                    out[at:at + i, j] = torch.softmax(z.masked_fill_(hide, -math.inf), -1) @ vv
        at += i
    return {"out": out}
