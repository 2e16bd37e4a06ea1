"""Operators of a training step on long sequences, images and video, as timed cases.

``rotary``    rotary positions of one to three axes (a token's place; frame, row and column) on the queries and keys of the
              attention's qkv blocks, and the gradient of it.
``selected``  attention in which every query sees its own block of keys and those blocks that a cheap score, its product with
              each block's mean key, ranks highest: the choice and the forward pass, or the backward pass.
``norm``      the norm of all gradients of a layer or a stack, the factor that clips them, and the clipped gradients, the parts of a
              vector's added up, beside the gradients themselves (which the next micro-batch adds to).

A case is a dict of plain values; ``listed()`` names twelve, ``draw()`` gives more of the same ranges.  ``run()`` computes a
case in plain torch operations, or with ``own`` through the entry points of ``paper_2104_05343_amd``; ``exact()`` computes it in
64 bits from the definitions.
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

DEV = "cuda:0"


# ------------------------------------------------------------------------------------------------ the cases
def _rotary(name, direction, b, s, h, n, q, i, j, pairs, order="sections", shared=False, interleaved=False, dtype="bf16", start=0,
            in_place=False):
    c = {"kind": "rotary", "direction": direction, "b": b, "s": s, "h": h, "n": n, "q": q, "i": i, "j": j,
         "pairs": "+".join(map(str, pairs)), "order": order, "shared": shared, "interleaved": interleaved, "dtype": dtype,
         "start": start, "in_place": in_place}
    return {"name": name, **c} if name else c


def _selected(name, direction, b, s, h, n, q, i, j, block, count, causal=True, lengths=False):
    c = {"kind": "selected", "direction": direction, "b": b, "s": s, "h": h, "n": n, "q": q, "i": i, "j": j, "block": block,
         "count": count, "causal": causal, "lengths": lengths}
    return {"name": name, **c} if name else c


def _norm(name, h, q, layers, dtype="fp32", extra=0):
    c = {"kind": "norm", "h": h, "q": q, "layers": layers, "dtype": dtype, "extra": extra}
    return {"name": name, **c} if name else c


def listed():
    return [
        # the next token of eight sequences, far into each: latency
        _rotary("rotary_token", "fwd", 8, 1, 1024, 16, 1, 0, 0, (32,), start=1000000),
        # one device of the 4096-wide layer of the benchmark: text, one axis, where the projection left it
        _rotary("rotary_text", "fwd", 8, 1024, 4096, 32, 4, 1, 2, (64,), in_place=True),
        # the gradient on every device of a 2048-wide layer on video, three axes of unequal shares
        _rotary("rotary_video_bwd", "bwd", 8, 4096, 2048, 16, 2, -1, -1, (16, 24, 24), interleaved=True),
        # fp32, odd shares of the axes taken in turn, some pairs of a head left as they are
        _rotary("rotary_ragged_fp32", "fwd", 4, 777, 1280, 20, 2, 1, 0, (8, 9, 9), order="turn", shared=True, dtype="fp32"),
        # a unit test's or a debugging run's sequences: launches and latency
        _selected("selected_fwd_short", "fwd", 2, 70, 256, 4, 2, -1, -1, 64, 2),
        # one device of the 4096-wide causal layer of the benchmark on sequences of 4096
        _selected("selected_fwd", "fwd", 8, 4096, 4096, 32, 4, 1, 2, 128, 8),
        _selected("selected_bwd", "bwd", 8, 4096, 4096, 32, 4, 1, 2, 128, 8),
        # a long document on one device: one sixteenth of the blocks
        _selected("selected_fwd_long", "fwd", 1, 32768, 1024, 8, 1, 0, 0, 128, 16),
        # sequences of different lengths, short of a multiple of the block, narrow heads
        _selected("selected_bwd_ragged", "bwd", 4, 10000, 1280, 20, 2, 1, 0, 64, 12, lengths=True),
        # the gradients of a small layer (latency), of a 2048-wide one with its vectors in parts, of four 4096-wide layers in bf16
        # with a table of odd width
        _norm("norm_small", 256, 2, 1),
        _norm("norm_h2048", 2048, 4, 1),
        _norm("norm_stack_bf16", 4096, 4, 4, dtype="bf16", extra=1000003),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the ranges the listed ones stand for."""
    kind = rng.choice(["rotary", "rotary", "selected", "selected", "selected", "norm"])
    most = {k: max(work(c)["flops" if kind == "selected" else "bytes"] for c in listed() if c["kind"] == kind)
            for k in ("selected", "rotary", "norm") if k == kind}[kind]
    while True:
        q = rng.choice([1, 1, 2, 4])
        i, j = (-1, -1) if rng.random() < 0.2 else (rng.randrange(q), rng.randrange(q))
        if kind == "norm":
            h = q * rng.choice([8, 16, 64]) * _log_int(rng, 4, 64)
            extra = rng.choice([0, _log_int(rng, 1, 50000000)])
            c = _norm("", min(h, 4096), q, _log_int(rng, 1, 24), rng.choice(["fp32", "bf16"]), extra=extra)
            if work(c)["bytes"] <= most:
                return c
            continue
        nh, b = rng.choice([1, 2, 3, 4, 5, 8, 16]), q * _log_int(rng, 1, 8)
        if kind == "rotary":
            d = rng.choice([16, 40, 64, 64, 80, 128, 128, 256])
            axes, left = rng.choice([1, 1, 2, 3]), d // 2
            pairs = [d // 2] if axes == 1 and rng.random() < 0.6 else []
            while len(pairs) < axes:
                pairs.append(rng.randint(1, max(1, left - (axes - len(pairs) - 1))))
                left -= pairs[-1]
            c = _rotary("", rng.choice(["fwd", "bwd"]), b, _log_int(rng, 1, 16384), q * nh * d, q * nh, q, i, j, pairs,
                        order=rng.choice(["sections", "turn"]), shared=rng.random() < 0.5, interleaved=rng.random() < 0.5,
                        dtype=rng.choice(["bf16", "bf16", "fp32"]), start=rng.choice([0, 0, _log_int(rng, 1, 4000000)]),
                        in_place=rng.random() < 0.5)
            if work(c)["bytes"] <= most and b * c["s"] * c["h"] <= 1 << 29:   # all devices' blocks are in memory
                return c
            continue
        d, s, block = rng.choice([64, 128]), _log_int(rng, 1, 32768), rng.choice([64, 128, 128, 256, 512])
        causal = rng.random() < 0.8
        if not causal:   # whole blocks, so that every choice has the same work
            s = -(-s // block) * block
        c = _selected("", rng.choice(["fwd", "bwd"]), b, s, q * nh * d, q * nh, q, i, j, block, _log_int(rng, 1, 24), causal=causal,
                      lengths=causal and rng.random() < 0.3)
        visited = len(_devices(c)) * (b // q) * nh * s * s   # by the plain form: all pairs
        if work(c)["flops"] <= most and b * s * c["h"] <= 1 << 29 and visited <= 1.8e10:
            return c


# ------------------------------------------------------------------------------------------------ what a case is made of
def _devices(c):
    q = c["q"]
    return list(range(q * q)) if c["i"] < 0 else [c["i"] * q + c["j"]]


def _dtype(c):
    return {"bf16": torch.bfloat16, "fp32": torch.float32}[c["dtype"]]


def _pairs_of(c):
    return [int(x) for x in c["pairs"].split("+")]


def _positions(c):
    """int32 [axes, b * s].  One axis: places from `start` on.  More: a text of a tenth of the sequence, whose axes run together, then
    frames of rows of up to 24 tokens."""
    b, s, axes = c["b"], c["s"], len(_pairs_of(c))
    t = np.arange(s)
    if axes == 1:
        rows = [t]
    else:
        head = s // 10
        u = np.maximum(t - head, 0)
        col, row, frame = u % 24, u // 24 % 24, u // 576
        rows = [np.where(t < head, t, head + x) for x in ([frame, row, col] if axes == 3 else [row + 24 * frame, col])]
    all_of = np.tile(np.stack(rows)[:, None, :], (1, b, 1)) + c["start"] + 17 * np.arange(b)[None, :, None]
    return all_of.reshape(axes, b * s).astype(np.int32)


def _lengths(c):
    r = random.Random(c["s"] * 31 + c["b"])
    return np.array([r.randint(c["s"] // 2, c["s"]) if c["lengths"] else c["s"] for _ in range(c["b"])], dtype=np.int32)


def _gradients(c):
    """(elements, parts) of every gradient: a layer's matrices, and its vectors as the partial sums of the q devices of a column."""
    h = c["h"]
    layer = [(n, 1) for n in (3 * h * h, h * h, 4 * h * h, 4 * h * h)] + [(n, c["q"]) for n in (3 * h, h, 4 * h, h, h, h, h, h)]
    return layer * c["layers"] + ([(c["extra"], 1)] if c["extra"] else [])


def _score_pairs(c):
    """(pairs of a query and a key that the attention has, pairs of a query and a block that the choice scores), all matrices."""
    s, B, k, q = c["s"], c["block"], c["count"], c["q"]
    pairs = scored = 0
    rows = {}
    for dev in _devices(c):
        rows[dev // q] = rows.get(dev // q, 0) + 1
    lengths = _lengths(c)
    for i, times in rows.items():
        for n in lengths[i * (c["b"] // q):(i + 1) * (c["b"] // q)]:
            t = np.arange(int(n), dtype=np.int64)
            if c["causal"]:
                own_block = t // B
                chosen = np.minimum(own_block, k - 1)
                pairs += times * int((t % B + 1 + chosen * B).sum())
                scored += times * int(own_block[own_block > k - 1].sum())
            else:
                blocks = s // B
                pairs += times * len(t) * min(blocks, k) * B
                scored += times * len(t) * (blocks - 1 if blocks > k else 0)
    return pairs * (c["n"] // q), scored * (c["n"] // q)


def work(case):
    c = case
    if c["kind"] == "norm":
        size = 2 if c["dtype"] == "bf16" else 4
        total = sum(n * (p * 4 + 4 if p > 1 else 2 * size) for n, p in _gradients(c))
        return {"bytes": total, "flops": sum(n * (p + 2) for n, p in _gradients(c))}
    q, d = c["q"], c["h"] // c["n"]
    rows = len(_devices(c)) * (c["b"] // q) * c["s"]
    heads = c["n"] // q
    if c["kind"] == "rotary":
        size = 2 if c["dtype"] == "bf16" else 4
        turned = 2 * 2 * sum(_pairs_of(c))                    # elements of a head's query and key that change
        moved = turned if c["in_place"] else 3 * d            # elsewhere, the whole head is written
        return {"bytes": rows * (heads * moved * size * 2 + 4 * len(_pairs_of(c))), "flops": rows * heads * turned * 3}
    pairs, scored = _score_pairs(c)
    wide = heads * d
    if c["direction"] == "fwd":
        return {"bytes": rows * (wide * 2 * 4 + heads * 4 * (1 + c["count"])), "flops": 4 * d * pairs + 2 * d * scored}
    return {"bytes": rows * (wide * 2 * 8 + heads * 4 * (1 + c["count"])), "flops": 10 * d * pairs}


def _normal(gen, n, scale, dtype):
    """n draws of a normal distribution, made in pieces."""
    out = torch.empty(n, dtype=dtype, device=DEV)
    for at in range(0, n, 1 << 26):
        m = min(1 << 26, n - at)
        out[at:at + m] = torch.randn(m, generator=gen, device=DEV) * scale
    return out


def prepare(case, seed):
    c = case
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    if c["kind"] == "norm":
        st = {"case": c, "max_norm": 1.0, "tensors": []}
        for n, parts in _gradients(c):
            g = _normal(gen, n * parts, 1e-3, torch.float32)
            for at in range(0, g.numel(), 1 << 26):   # rows that differ in size, as those of a trained layer do
                piece = g[at:at + (1 << 26)]
                piece *= torch.exp(1.5 * torch.sin(torch.arange(at, at + piece.numel(), device=DEV) * 0.37))
            st["tensors"].append((g if parts > 1 or c["dtype"] == "fp32" else g.to(torch.bfloat16), n, parts))
        # what is clipped, in one buffer a type
        sizes = {t: sum(n for g, n, _ in st["tensors"] if g.dtype == t) for t in {g.dtype for g, _, _ in st["tensors"]}}
        st["buffers"] = {t: torch.zeros(k, dtype=t, device=DEV) for t, k in sizes.items()}
        at, st["clipped"] = dict.fromkeys(sizes, 0), []
        for g, n, _ in st["tensors"]:
            st["clipped"].append(st["buffers"][g.dtype][at[g.dtype]:at[g.dtype] + n])
            at[g.dtype] += n
        return st
    b, s, h, n, q = c["b"], c["s"], c["h"], c["n"], c["q"]
    M, d = b * s, h // n
    if c["kind"] == "rotary":
        st = {"case": c, "x": _normal(gen, 3 * M * h, 1.0, _dtype(c)), "positions": torch.from_numpy(_positions(c)).to(DEV)}
        st["y"] = st["x"] if c["in_place"] else torch.zeros_like(st["x"])
        return st
    # keys of a block have something in common, and a query looks for what a block in front of it has
    x = _normal(gen, 3 * M * h, 1.0, torch.bfloat16).view(q * q, b // q, s, n // q, 3, d)
    blocks = -(-s // c["block"])
    of = torch.arange(s, device=DEV) // c["block"]
    sought = (torch.rand(s, generator=gen, device=DEV) * (of + 1)).long()
    for dev in range(q * q):
        topics = torch.randn(b // q, blocks, n // q, d, generator=gen, device=DEV)
        for k in range(b // q):
            x[dev, k, :, :, 1] += 0.5 * topics[k][of]
            x[dev, k, :, :, 0] += 0.3 * topics[k][sought]
    st = {"case": c, "qkv": x.view(-1), "lengths": torch.from_numpy(_lengths(c)).to(DEV) if c["lengths"] else None}
    heads = q * q * (b // q) * (n // q)
    st["attn"] = torch.zeros(M * h, dtype=torch.bfloat16, device=DEV)
    st["lse"] = torch.zeros(heads * s, dtype=torch.float32, device=DEV)
    st["selected"] = torch.full((heads * s * c["count"],), -1, dtype=torch.int32, device=DEV)
    if c["direction"] == "bwd":   # what the forward pass left
        out, devs = _plain_selected_forward(st), _devices(c)
        for name in ("selected", "attn", "lse"):
            st[name].view(q * q, -1)[devs] = out[name].reshape(len(devs), -1)
        st["d_attn"] = _normal(gen, M * h, 1.0, torch.bfloat16)
        st["d_qkv"] = torch.zeros(3 * M * h, dtype=torch.bfloat16, device=DEV)
    return st


def run(state):
    kind = state["case"]["kind"]
    if kind == "norm":
        return _own_norm(state) if own else _plain_norm(state)
    if kind == "rotary":
        return _own_rotary(state) if own else _plain_rotary(state)
    if own:
        return _own_selected(state)
    return _plain_selected_forward(state) if state["case"]["direction"] == "fwd" else _plain_selected_backward(state)


# ------------------------------------------------------------------------------------------------ the framework's calls
def _own_rotary(st):
    import paper_2104_05343_amd as opt
    c = st["case"]
    b, s, h, n, q, i, j = (c[k] for k in ("b", "s", "h", "n", "q", "i", "j"))
    if "rotary" not in st:   # what a program keeps: the description of the axes
        st["rotary"] = opt.make_rotary(st["positions"], _pairs_of(c), in_turn=c["order"] == "turn", shared=c["shared"],
                                       interleaved=c["interleaved"])
    call = opt.rotary if c["direction"] == "fwd" else opt.rotary_bwd
    call(st["x"], st["y"], b, s, h, n, q, i, j, opt.BF16 if c["dtype"] == "bf16" else opt.FP32, st["rotary"])
    return _blocks_of(c, st["y"].view(q * q, b // q, s, n // q, 3, h // n))


def _own_selected(st):
    import paper_2104_05343_amd as opt
    c = st["case"]
    b, s, h, n, q, i, j = (c[k] for k in ("b", "s", "h", "n", "q", "i", "j"))
    if "selection" not in st:   # what a program keeps over its steps
        st["selection"] = opt.make_selection(c["block"], c["count"], st["lengths"])
        st["ws"] = torch.empty(opt.attention_selected_workspace_bytes(b, s, h, n, q, i, j, st["selection"]), dtype=torch.uint8, device=DEV)
    at = (b, s, h, n, q, i, j, c["causal"], opt.BF16, st["selection"], st["ws"])
    if c["direction"] == "bwd":
        opt.attention_selected_bwd(st["qkv"], st["selected"], st["attn"], st["lse"], st["d_attn"], st["d_qkv"], *at)
        return _blocks_of(c, st["d_qkv"].view(q * q, b // q, s, n // q, 3, h // n))
    opt.attention_select(st["qkv"], st["selected"], *at)
    opt.attention_selected_fwd(st["qkv"], st["selected"], st["attn"], st["lse"], *at)
    return {"selected": _blocks_of(c, st["selected"].view(q * q, b // q, n // q, s, c["count"])),
            "attn": _blocks_of(c, st["attn"].view(q * q, b // q, s, n // q, h // n)),
            "lse": _blocks_of(c, st["lse"].view(q * q, b // q, n // q, s))}


def _own_norm(st):
    import paper_2104_05343_amd as opt
    if "list" not in st:   # a program lists its gradients once
        st["list"] = opt.make_gradients([dict(grad=g, n=n, parts=p, clipped=y) for (g, n, p), y in zip(st["tensors"], st["clipped"])])
        st["ws"] = torch.empty(opt.gradient_norm_workspace_bytes(st["list"]), dtype=torch.uint8, device=DEV)
        st["norm"], st["scale"], st["norms"] = (torch.zeros(k, dtype=torch.float32, device=DEV) for k in (1, 1, len(st["tensors"])))
    opt.gradient_norm(st["list"], st["max_norm"], st["norm"], st["scale"], st["norms"], st["ws"])
    opt.gradient_clip(st["list"], st["scale"])
    return {"norm": st["norm"], "scale": st["scale"], "norms": st["norms"], **_buffers_of(st)}


def _buffers_of(st):
    return {"clipped_" + str(t)[6:]: x for t, x in st["buffers"].items()}


def _blocks_of(c, x):
    """The blocks of the case's devices of x [q * q, ...]."""
    return x if c["i"] < 0 else x[_devices(c)[0]:_devices(c)[0] + 1]


# ------------------------------------------------------------------------------------------------ plain forms: rotary positions
def _ladder(c):
    """(axis, frequency) of every pair that turns, frequencies in 64 bits."""
    pairs = _pairs_of(c)
    order = [a for a, k in enumerate(pairs) for _ in range(k)]
    if c["order"] == "turn":
        left, order = list(pairs), []
        while any(left):
            for a in range(len(pairs)):
                if left[a]:
                    order.append(a)
                    left[a] -= 1
    seen = [0] * len(pairs)
    out = []
    for p, a in enumerate(order):
        out.append((a, 10000.0 ** (-(p / sum(pairs) if c["shared"] else seen[a] / pairs[a]))))
        seen[a] += 1
    return out


def _plain_rotary(st):
    c = st["case"]
    b, s, h, n, q = (c[k] for k in ("b", "s", "h", "n", "q"))
    d, P = h // n, sum(_pairs_of(c))
    devs = _devices(c)
    ladder = _ladder(c)
    axis = torch.tensor([a for a, _ in ladder], device=DEV)
    freq = torch.tensor([f for _, f in ladder], dtype=torch.float64, device=DEV)
    angle = st["positions"].double()[axis].T.contiguous() * freq                     # [b * s, P]
    angle = angle.view(q, b // q, s, 1, 1, P)[[dev // q for dev in devs]]
    cos, sin = torch.cos(angle).float(), torch.sin(angle).float()
    if c["direction"] == "bwd":
        sin = -sin
    X, Y = (st[k].view(q * q, b // q, s, n // q, 3, d) for k in ("x", "y"))
    x = X[devs][..., :2, :2 * P].float()
    first, second = (x[..., 0::2], x[..., 1::2]) if c["interleaved"] else (x[..., :P], x[..., P:])
    turned = (first * cos - second * sin, first * sin + second * cos)
    whole = torch.stack(turned, -1).flatten(-2) if c["interleaved"] else torch.cat(turned, -1)
    if not c["in_place"]:
        Y[devs] = X[devs]
    Y[devs, ..., :2, :2 * P] = whole.to(Y.dtype)
    return _blocks_of(c, Y)


# ------------------------------------------------------------------------------------------------ plain forms: selected attention
def _heads_of(c, x, width, parts=1):
    """x, rows of heads of `parts` things of `width`, as fp32 [part][matrix, s, width] of the case's devices."""
    q, s = c["q"], c["s"]
    y = x.view(q * q, c["b"] // q, s, c["n"] // q, parts, width)[_devices(c)]
    return [y[..., p, :].permute(0, 1, 3, 2, 4).reshape(-1, s, width).float() for p in range(parts)]


def _rows_of(c, x, width):
    """The other way: [matrix, s, width] as [device, sequence, s, head, width]."""
    return x.view(len(_devices(c)), c["b"] // c["q"], c["n"] // c["q"], c["s"], width).permute(0, 1, 3, 2, 4)


def _lengths_of(st):
    """Length of every matrix' sequence."""
    c = st["case"]
    nb, nh = c["b"] // c["q"], c["n"] // c["q"]
    all_of = st["lengths"].long() if c["lengths"] else torch.full((c["b"],), c["s"], device=DEV)
    return torch.cat([all_of[dev // c["q"] * nb:dev // c["q"] * nb + nb].repeat_interleave(nh) for dev in _devices(c)])


def _pieces(c, mats):
    """(matrices, rows) slices whose scores are at most 2^28."""
    s = c["s"]
    rows = max(1, min(s, (1 << 28) // s))
    group = max(1, (1 << 28) // (rows * s))
    for m in range(0, mats, group):
        for r in range(0, s, rows):
            yield slice(m, min(mats, m + group)), slice(r, min(s, r + rows))


def _plain_select(c, Q, K, lengths):
    """int32 [matrix, s, count]: the own block and the best ones by the product with the blocks' mean keys, ascending, -1 behind them.
    Scores in 64 bits, from means rounded to bf16: neighbours at the border are told apart."""
    mats, s, d = Q.shape
    B, count = c["block"], c["count"]
    blocks = -(-s // B)
    t = torch.arange(s, device=DEV)
    seen = t[None, :] < lengths[:, None]
    held = torch.nn.functional.pad(torch.where(seen[..., None], K, torch.zeros_like(K)), (0, 0, 0, blocks * B - s)).view(mats, blocks, B, d)
    keys = torch.nn.functional.pad(seen, (0, blocks * B - s)).view(mats, blocks, B).sum(-1)
    means = (held.double().sum(2) / keys.clamp_min(1)[..., None]).float().to(torch.bfloat16).double()
    scores = torch.matmul(Q.double(), means.transpose(1, 2).contiguous())
    j = torch.arange(blocks, device=DEV)
    mine = t // B
    can = (keys > 0)[:, None, :] & (j[None, None, :] != mine[None, :, None])
    if c["causal"]:
        can = can & (j[None, None, :] < mine[None, :, None])
    order = torch.argsort(torch.where(can, scores, -math.inf), dim=-1, descending=True, stable=True)[..., :count - 1]
    chosen = torch.where(torch.gather(can.expand(mats, s, blocks), 2, order), order, blocks)
    chosen = torch.sort(torch.cat([mine[None, :, None].expand(mats, s, 1), chosen], -1), -1).values
    chosen = torch.nn.functional.pad(chosen, (0, max(0, count - chosen.shape[-1])), value=blocks)[..., :count]
    return torch.where((chosen < blocks) & seen[..., None], chosen, -1).to(torch.int32)


def _left_out(c, selected, lengths, rows):
    """bool [matrix, rows, s]: pairs that the attention does not have."""
    s, B = c["s"], c["block"]
    blocks = -(-s // B)
    t = torch.arange(s, device=DEV)
    picked = torch.zeros(*selected.shape[:2], blocks + 1, dtype=torch.bool, device=DEV)
    picked.scatter_(2, torch.where(selected < 0, blocks, selected).long(), True)
    has = picked[..., t // B] & (t < lengths[:, None])[:, None, :] & (t[rows] < lengths[:, None])[..., None]
    return ~(has & (t[None, :] <= t[rows][:, None])) if c["causal"] else ~has


def _plain_selected_forward(st):
    c = st["case"]
    d = c["h"] // c["n"]
    Q, K, V = _heads_of(c, st["qkv"], d, 3)
    lengths = _lengths_of(st)
    selected = _plain_select(c, Q, K, lengths)
    O, L = torch.empty_like(Q), torch.empty(Q.shape[:2], device=DEV)
    for m, r in _pieces(c, len(Q)):
        S = torch.matmul(Q[m, r], K[m].transpose(1, 2).contiguous()) / math.sqrt(d)
        S = S.masked_fill_(_left_out(c, selected[m, r], lengths[m], r), -math.inf)
        top = S.amax(-1, keepdim=True)
        top = torch.where(top == -math.inf, torch.zeros_like(top), top)
        P = torch.exp(S - top)
        total = P.sum(-1, keepdim=True)
        O[m, r] = torch.matmul(P, V[m]) / torch.where(total == 0, torch.ones_like(total), total)
        L[m, r] = (top + torch.log(total)).squeeze(-1)
    devs, nb, nh = len(_devices(c)), c["b"] // c["q"], c["n"] // c["q"]
    return {"selected": selected.view(devs, nb, nh, c["s"], c["count"]), "attn": _rows_of(c, O, d).to(torch.bfloat16).contiguous(),
            "lse": L.view(devs, nb, nh, c["s"])}


def _plain_selected_backward(st):
    c = st["case"]
    q, d = c["q"], c["h"] // c["n"]
    Q, K, V = _heads_of(c, st["qkv"], d, 3)
    (G,), (O,) = _heads_of(c, st["d_attn"], d), _heads_of(c, st["attn"], d)
    lengths, devs = _lengths_of(st), _devices(c)
    selected = st["selected"].view(q * q, -1)[devs].view(len(Q), c["s"], c["count"])
    lse = st["lse"].view(q * q, -1)[devs].view(len(Q), c["s"], 1)
    dQ, dK, dV = torch.empty_like(Q), torch.zeros_like(Q), torch.zeros_like(Q)
    for m, r in _pieces(c, len(Q)):
        out = _left_out(c, selected[m, r], lengths[m], r)
        P = torch.exp(torch.matmul(Q[m, r], K[m].transpose(1, 2).contiguous()) / math.sqrt(d) - lse[m, r]).masked_fill_(out, 0)
        dV[m] += torch.matmul(P.transpose(1, 2).contiguous(), G[m, r])
        dS = P * (torch.matmul(G[m, r], V[m].transpose(1, 2).contiguous()) - (G[m, r] * O[m, r]).sum(-1, keepdim=True))
        dQ[m, r] = torch.matmul(dS, K[m]) / math.sqrt(d)
        dK[m] += torch.matmul(dS.transpose(1, 2).contiguous(), Q[m, r]) / math.sqrt(d)
    nothing = (torch.arange(c["s"], device=DEV) >= lengths[:, None])[..., None]
    return torch.stack([_rows_of(c, x.masked_fill(nothing, 0), d) for x in (dQ, dK, dV)], 4).to(torch.bfloat16)


# ------------------------------------------------------------------------------------------------ plain forms: the norm
def _plain_norm(st):
    squares = []
    for g, n, parts in st["tensors"]:
        x = g.view(parts, n)
        x = x[0].float() if parts == 1 else x.sum(0)
        squares.append(torch.stack([(x[at:at + (1 << 26)].double() ** 2).sum() for at in range(0, n, 1 << 26)]).sum())
    squares = torch.stack(squares)
    norm = torch.sqrt(squares.sum())
    scale = torch.where(norm > st["max_norm"], st["max_norm"] / norm, torch.ones_like(norm)).float()
    for (g, n, parts), y in zip(st["tensors"], st["clipped"]):
        x = g.view(parts, n)
        y.copy_((x[0].float() if parts == 1 else x.sum(0)) * scale)
    return {"norm": norm.float().view(1), "scale": scale.view(1), "norms": torch.sqrt(squares).float(), **_buffers_of(st)}


# ------------------------------------------------------------------------------------------------ 64 bits
def exact(case, seed):
    st = prepare(case, seed)
    return {"norm": _exact_norm, "rotary": _exact_rotary, "selected": _exact_selected}[case["kind"]](st)


def _exact_norm(st):
    each = []
    for g, n, parts in st["tensors"]:
        total = torch.zeros((), dtype=torch.float64, device=DEV)
        for at in range(0, n, 1 << 25):
            piece = sum(g[p * n + at:p * n + min(n, at + (1 << 25))].double() for p in range(parts))
            total += torch.dot(piece, piece)
        each.append(total)
    norm = sum(each).sqrt()
    scale = (st["max_norm"] / norm).clamp_max(1.0)
    out = {"norm": norm.view(1), "scale": scale.view(1), "norms": torch.stack(each).sqrt()}
    for t in st["buffers"]:
        out["clipped_" + str(t)[6:]] = torch.cat([sum(g[p * n:(p + 1) * n].double() for p in range(parts)) * scale
                                                  for g, n, parts in st["tensors"] if g.dtype == t])
    return out


def _exact_rotary(st):
    """Pairs as complex numbers, device by device."""
    c = st["case"]
    b, s, h, n, q = (c[k] for k in ("b", "s", "h", "n", "q"))
    d, P, sign = h // n, sum(_pairs_of(c)), 1 if c["direction"] == "fwd" else -1
    out = []
    for dev in _devices(c):
        x = st["x"].view(q * q, b // q, s, n // q, 3, d)[dev].double().clone()
        where = st["positions"].view(-1, q, b // q, s)[:, dev // q].double()
        for p, (axis, freq) in enumerate(_ladder(c)):
            e, f = (2 * p, 2 * p + 1) if c["interleaved"] else (p, p + P)
            turn = torch.polar(torch.ones_like(where[axis]), sign * freq * where[axis])[..., None, None]
            z = torch.complex(x[..., :2, e], x[..., :2, f]) * turn
            x[..., :2, e], x[..., :2, f] = z.real, z.imag
        out.append(x)
    return torch.stack(out)


def _exact_choice(c, Q, K, length):
    """int32 [s, count] of one matrix: a block is chosen if fewer than count - 1 are better (ties: lower ones are)."""
    s, B, k = c["s"], c["block"], c["count"] - 1
    blocks = -(-s // B)
    out = torch.full((s, c["count"]), -1, dtype=torch.int32, device=DEV)
    have = -(-length // B)
    if have == 0:
        return out
    mean = torch.stack([K[v * B:min(length, (v + 1) * B)].sum(0) / (min(length, (v + 1) * B) - v * B) for v in range(have)])
    mean = mean.float().bfloat16().double()
    number = torch.arange(have, device=DEV)
    for at in range(0, length, 512):
        rows = torch.arange(at, min(length, at + 512), device=DEV)
        x = Q[rows] @ mean.T
        mine = (rows // B)[:, None]
        can = number[None] < mine if c["causal"] else number[None] != mine
        x = x.masked_fill(~can, -math.inf)
        better = (x[:, None, :] > x[:, :, None]) | ((x[:, None, :] == x[:, :, None]) & (number[None, None, :] < number[None, :, None]))
        chosen = (can & ((better & can[:, None, :]).sum(-1) < k)) | (number[None] == mine)
        place = chosen.cumsum(1) - 1
        r, v = chosen.nonzero(as_tuple=True)
        out[rows[r], place[r, v]] = v.to(torch.int32)
    return out


def _exact_selected(st):
    c = st["case"]
    s, q, nb, nh, d, B = c["s"], c["q"], c["b"] // c["q"], c["n"] // c["q"], c["h"] // c["n"], c["block"]
    bwd, f64 = c["direction"] == "bwd", torch.float64
    u = torch.arange(s, device=DEV)
    out = {"selected": [], "attn": [], "lse": []} if not bwd else {"d_qkv": []}
    for dev in _devices(c):
        block = st["qkv"].view(q * q, nb, s, nh, 3, d)[dev]
        for b in range(nb):
            length = int(st["lengths"][dev // q * nb + b]) if c["lengths"] else s
            for a in range(nh):
                Q, K, V = (block[b, :, a, k].to(f64) for k in range(3))
                if bwd:
                    choice = st["selected"].view(q * q, nb, nh, s, c["count"])[dev, b, a]
                    G = st["d_attn"].view(q * q, nb, s, nh, d)[dev, b, :, a].to(f64)
                    O = st["attn"].view(q * q, nb, s, nh, d)[dev, b, :, a].to(f64)
                    L = st["lse"].view(q * q, nb, nh, s)[dev, b, a].to(f64)
                    grad = torch.zeros(3, s, d, dtype=f64, device=DEV)
                else:
                    choice = _exact_choice(c, Q, K, length)
                    attn, lse = torch.zeros(s, d, dtype=f64, device=DEV), torch.full((s,), -math.inf, dtype=f64, device=DEV)
                step = max(1, (1 << 26) // s)
                for at in range(0, length, step):
                    r = slice(at, min(length, at + step))
                    see = (u[None, :] // B == choice[r][:, :1]) & (choice[r][:, :1] >= 0)
                    for e in range(1, c["count"]):
                        see |= (u[None, :] // B == choice[r][:, e:e + 1]) & (choice[r][:, e:e + 1] >= 0)
                    see &= u[None, :] < length
                    if c["causal"]:
                        see &= u[None, :] <= u[r][:, None]
                    x = ((Q[r] @ K.T) * d ** -0.5).masked_fill(~see, -math.inf)
                    if bwd:
                        P = torch.exp(x - L[r].view(-1, 1)).masked_fill(~see, 0)
                        D = P * (G[r] @ V.T - (G[r] * O[r]).sum(1, keepdim=True))
                        grad[0, r] = D @ K * d ** -0.5
                        grad[1] += D.T @ Q[r] * d ** -0.5
                        grad[2] += P.T @ G[r]
                    else:
                        lse[r] = torch.logsumexp(x, 1)
                        attn[r] = torch.exp(x - lse[r].view(-1, 1)).masked_fill(~see, 0) @ V
                if bwd:
                    out["d_qkv"].append(grad)
                else:
                    out["selected"].append(choice), out["attn"].append(attn), out["lse"].append(lse)
    devs = len(_devices(c))
    if bwd:
        return torch.stack(out["d_qkv"]).view(devs, nb, nh, 3, s, d).permute(0, 1, 4, 2, 3, 5)
    return {"selected": torch.stack(out["selected"]).view(devs, nb, nh, s, -1),
            "attn": torch.stack(out["attn"]).view(devs, nb, nh, s, d).permute(0, 1, 3, 2, 4),
            "lse": torch.stack(out["lse"]).view(devs, nb, nh, s)}
