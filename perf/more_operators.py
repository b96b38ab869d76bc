"""Operators of serving in less memory, their plain forms and their cases.

  append   kvg_int8_append: RMS norm of every query and key head, the rotation, and the append of packed sequences to a paged
           cache of 8-bit integers with a scale for each page and KV head; a page that grows beyond its scale is rescaled
  attn     kvg_int8_attn: causal attention of packed sequences over that cache (whole prompts, chunks over a restored
           block, single tokens)
  axes     kvg_rotate_axes and kvg_norm_append_axes: rotary positions with several axes (time, height, width), alone and
           with the norms and the append
  sample   kvg_sample: tokens from logits by temperature, top-k, top-p and min-p, from given random numbers

Shapes are those of the synthetic workloads (synth/workloads.py): the 12B-class geometry (16 query / 8 KV heads,
head_dim 256), the 31B-class one (32 / 16, 128), the 8-queries-per-KV-head one (16 / 2, 128) and a small one (4 / 2, 64);
4,096-token blocks, 32,768-token windows, suffixes of 35 to 1,024 tokens, a vocabulary of 262,144.  A model runs its
layers one after the other, so most cases are one layer's call.
"""

import math
import random

import numpy
import torch

own = False

PAGE = 16
GEOMETRY = {              # query heads, KV heads, head_dim
    "12b": (16, 8, 256),
    "31b": (32, 16, 128),
    "gqa8": (16, 2, 128),
    "small": (4, 2, 64),
}
BASE = 10000.0
EPS = 1e-6
# Frequencies for long contexts: original is the context they were made for, fast and slow are turns over it.
SCALING = {
    "plain": dict(scaling="plain", factor=1.0, original=0.0, fast=0.0, slow=0.0),
    "linear": dict(scaling="linear", factor=8.0, original=0.0, fast=0.0, slow=0.0),
    "rotations": dict(scaling="rotations", factor=8.0, original=8192.0, fast=4.0, slow=1.0),
}
# How a head's pairs go to the axes of a position: shares of the pairs (in 32nds), contiguous or in turn, with the whole
# rotary's frequencies or each axis with its own.
AXES = {
    "sections": dict(share=(8, 12, 12), order="sections", own=False, pairing="half"),
    "turns": dict(share=(12, 10, 10), order="turns", own=False, pairing="half"),
    "own": dict(share=(8, 12, 12), order="sections", own=True, pairing="interleaved"),
    "grid": dict(share=(16, 16), order="sections", own=True, pairing="half"),
}


def listed():
    return [
        # one layer's step of a serving batch: 16 conversations, a token each, into pages that are partly filled
        dict(name="append-12b-step", kind="append", geometry="12b", layers=1, batch=16, longest=1, ctx=200, mix=1, scaling="plain"),
        # one layer of 8 prompts of 1 to 4,096 tokens
        dict(name="append-31b-prompts", kind="append", geometry="31b", layers=1, batch=8, longest=4096, ctx=0, mix=2,
             scaling="rotations"),
        # one layer's step of one conversation over a 4,096-token block, its suffix and a few decoded tokens: latency
        dict(name="attn-12b-token", kind="attn", geometry="12b", layers=1, batch=1, longest=1, ctx=4613, mix=4, window=0),
        # one layer's step of a serving batch, each sequence over up to 8 store blocks
        dict(name="attn-12b-step-32k", kind="attn", geometry="12b", layers=1, batch=16, longest=1, ctx=33301, mix=5, window=0),
        # a mixed batch of a windowed and a global layer: a few chunks among single tokens
        dict(name="attn-gqa8-mixed-window", kind="attn", geometry="gqa8", layers=2, batch=12, longest=700, ctx=5000, mix=7,
             window=1024),
        # one layer of 8 prompts of 1 to 4,096 tokens with nothing cached: the largest call
        dict(name="attn-31b-prompts", kind="attn", geometry="31b", layers=1, batch=8, longest=4096, ctx=0, mix=2, window=0),
        # the query and key heads of one decoded token of a prompt with images: the smallest call
        dict(name="axes-12b-token", kind="axes", geometry="12b", dtype="bf16", tokens=1, heads=24, axes="sections",
             scaling="plain"),
        # the query and key heads of 4,096 tokens of images and text
        dict(name="axes-31b-images", kind="axes", geometry="31b", dtype="bf16", tokens=4096, heads=48, axes="turns",
             scaling="plain"),
        # one layer of 3 prompts with images, normed, rotated and appended to a bf16 cache
        dict(name="axes-12b-append", kind="axes_append", geometry="12b", layers=1, batch=3, longest=2312, ctx=0, mix=9, axes="own",
             scaling="linear"),
        # the next token of one conversation
        dict(name="sample-token", kind="sample", rows=1, vocab=262144, filters="p"),
        # the next tokens of a serving batch, every filter on
        dict(name="sample-batch16", kind="sample", rows=16, vocab=262144, filters="kpm"),
        # 64 requests, each with filters of its own
        dict(name="sample-batch64-mixed", kind="sample", rows=64, vocab=262144, filters="mixed"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same ranges, no dearer than the largest listed one of its kind."""
    kind = rng.choice(["append", "attn", "attn", "axes", "axes_append", "sample", "sample"])
    geometry = rng.choice(["12b", "31b", "gqa8", "small"])
    Hq, Hkv, D = GEOMETRY[geometry]
    scaling = rng.choice(sorted(SCALING))
    if kind == "sample":
        return dict(kind=kind, rows=_log_int(rng, 1, 64), vocab=_log_int(rng, 100, 262144),
                    filters=rng.choice(["none", "k", "p", "m", "kp", "kpm", "mixed"]))
    if kind == "axes":
        return dict(kind=kind, geometry=geometry, dtype=rng.choice(["bf16", "f32"]), tokens=_log_int(rng, 1, 4096),
                    heads=rng.choice([Hq, Hkv, Hq + Hkv]), axes=rng.choice(sorted(AXES)), scaling=scaling)
    layers = rng.choice([1, 1, 1, 2])
    batch = _log_int(rng, 1, 16)
    longest = rng.choice([1, _log_int(rng, 2, 64), _log_int(rng, 65, 4096)])
    mix = rng.randrange(1, 1000)
    if kind != "attn":
        more = dict(axes=rng.choice(sorted(AXES))) if kind == "axes_append" else {}
        while batch * longest * layers * Hkv * D > 8 * 4096 * 2048:
            batch = max(1, batch // 2)
        return dict(kind=kind, geometry=geometry, layers=layers, batch=batch, longest=longest,
                    ctx=rng.choice([0, _log_int(rng, 1, 600)]), mix=mix, scaling=scaling, **more)
    # single tokens read long contexts; the plain form's scores (batch x heads x rows x keys) bound the others
    ctx = rng.choice([0, _log_int(rng, 16, 32768)]) if longest > 1 else _log_int(rng, 16, 32768)
    while batch * layers * Hq * longest * (longest + ctx) > 2.4e9:
        batch, longest, ctx = max(1, batch // 2), max(2, longest * 2 // 3), ctx * 3 // 4
    return dict(kind=kind, geometry=geometry, layers=layers, batch=batch, longest=longest, ctx=ctx, mix=mix,
                window=rng.choice([0, 0, 200, 1024]))


# ---------------------------------------------------------------------------- what a case holds

def _sequences(case):
    """Tokens of the call and tokens cached before it, of every sequence.  The first one has the longest of each.  About
    a third of a mixed batch are single tokens, one in ten has none."""
    rng = random.Random(case["mix"])
    lens, ctxs = [case["longest"]], [case["ctx"]]
    for _ in range(case["batch"] - 1):
        u = rng.random()
        lens.append(1 if case["longest"] == 1 else 0 if u < 0.1 else 1 if u < 0.4 else rng.randint(1, case["longest"]))
        ctxs.append(rng.randint(case["ctx"] // 2, case["ctx"]))
    return lens, ctxs


def _windows(case):
    """Every second layer of a windowed case is global."""
    return [case["window"] if case["window"] and l % 2 == 0 else 0 for l in range(case["layers"])]


def _pages(case):
    lens, ctxs = _sequences(case)
    return -(-(max(c + n for c, n in zip(ctxs, lens)) + 1) // PAGE)


def work(case):
    if case["kind"] == "sample":
        n = case["rows"] * case["vocab"]
        return {"bytes": 4 * n, "flops": 4 * n}
    Hq, Hkv, D = GEOMETRY[case["geometry"]]
    if case["kind"] == "axes":
        values = case["tokens"] * case["heads"] * D
        return {"bytes": 2 * values * (2 if case["dtype"] == "bf16" else 4), "flops": 3 * values}
    lens, ctxs = _sequences(case)
    tokens = sum(lens) * case["layers"]
    if case["kind"] == "axes_append":
        return {"bytes": 4 * tokens * Hq * D + 8 * tokens * Hkv * D, "flops": 8 * tokens * (Hq + Hkv) * D}
    if case["kind"] == "append":
        # queries in and out, raw keys and values in; the cache is given back as the values it stands for
        pool = 2 * case["layers"] * case["batch"] * _pages(case) * PAGE * Hkv * D
        return {"bytes": 4 * tokens * Hq * D + 4 * tokens * Hkv * D + 3 * pool, "flops": 10 * tokens * (Hq + Hkv) * D}
    pairs = keys = 0
    for w in _windows(case):
        for n, c in zip(lens, ctxs):
            if n:
                pairs += sum(min(c + i + 1, w) if w else c + i + 1 for i in range(n))
                keys += min(c + n, w + n - 1) if w else c + n
    return {"bytes": 4 * tokens * Hq * D + 2 * keys * Hkv * D + keys * Hkv // 2, "flops": 4 * D * Hq * pairs}


# ---------------------------------------------------------------------------- inputs

def _normal(gen, shape, sigma, dtype):
    x = torch.empty(shape, dtype=torch.float32, device="cuda")
    return x.normal_(0.0, sigma, generator=gen).to(dtype)


def _int8(gen, shape):
    """Pages as an append leaves them: normal values over a scale that puts the largest of a page near 127."""
    return _normal(gen, shape, 34.0, torch.float32).round_().clamp_(-127, 127).to(torch.int8)


def _scale(gen, shape):
    return _normal(gen, shape, 0.4, torch.float32).exp_().mul_(1.0 / 34.0)


def _inputs(case, gen, storage):
    """Sequences over a paged cache: pages in random order, more tokens' room than any sequence takes."""
    Hq, Hkv, D = GEOMETRY[case["geometry"]]
    lens, ctxs = _sequences(case)
    B, L, pages = case["batch"], case["layers"], _pages(case)
    shape = (L, B * pages, Hkv, PAGE, D)
    cu = [0]
    for n in lens:
        cu.append(cu[-1] + n)
    i32 = dict(dtype=torch.int32, device="cuda")
    seq = [b for b, n in enumerate(lens) for _ in range(n)]
    off = [i for n in lens for i in range(n)]
    s = dict(
        case=case, lens=lens, ctxs=ctxs, tokens=cu[-1], longest=max(lens), max_ctx=max(ctxs),
        max_keys=max(c + n for c, n in zip(ctxs, lens)),
        table=torch.randperm(B * pages, generator=gen, device="cuda").to(torch.int32).view(B, pages),
        cu=torch.tensor(cu, **i32), ctx=torch.tensor(ctxs, **i32),
        start=torch.randint(0, 8192, (B,), generator=gen, device="cuda"),
        seq=torch.tensor(seq, device="cuda"), off=torch.tensor(off, device="cuda"))
    if storage == "int8":
        s.update(k_pool=_int8(gen, shape), v_pool=_int8(gen, shape), k_scale=_scale(gen, shape[:3]), v_scale=_scale(gen, shape[:3]))
    else:
        s.update(k_pool=_normal(gen, shape, 1.0, torch.bfloat16), v_pool=_normal(gen, shape, 1.0, torch.bfloat16))
    return s


def _positions(case, tokens, gen):
    """Positions of text and images in turn: 64 tokens of text, which have one position on every axis, then an image of 32 x
    32 patches, whose axes are time, height and width (the last two where there are two)."""
    n = len(AXES[case["axes"]]["share"])
    at = torch.arange(tokens, device="cuda")
    block, r = at // 1088, at % 1088
    base = block * 96 + torch.randint(0, 100000, (1,), generator=gen, device="cuda")
    text, patch = r < 64, (r - 64).clamp(min=0)
    time = base + r.clamp(max=64)
    return torch.stack([time, time + torch.where(text, 0, patch // 32), time + torch.where(text, 0, patch % 32)])[3 - n:].contiguous()


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    if case["kind"] == "sample":
        R, V = case["rows"], case["vocab"]
        # a broad base and a few dozen likely tokens a row, through a soft cap at 30
        z = _normal(gen, (R, V), 3.0, torch.float32)
        likely = torch.randint(0, V, (R, 48), generator=gen, device="cuda")
        z.scatter_add_(1, likely, torch.rand((R, 48), generator=gen, device="cuda") * 16.0)
        s = dict(case=case, logits=torch.tanh(z / 30.0) * 30.0, u=torch.rand((R,), dtype=torch.float64, generator=gen, device="cuda"))
        pick = lambda values, dtype: torch.tensor(values, dtype=dtype, device="cuda")[  # noqa: E731
            torch.randint(0, len(values), (R,), generator=gen, device="cuda")]
        f = case["filters"]
        mixed = f == "mixed"
        s["temperature"] = pick([0.0, 0.5, 0.8, 1.0, 1.4], torch.float32) if mixed else pick([0.7, 0.8, 1.0], torch.float32)
        s["top_k"] = pick([0, 1, 20, 50, 1000, V], torch.int32) if mixed else pick([20, 50, 64], torch.int32) if "k" in f else None
        s["top_p"] = pick([1.0, 0.95, 0.9, 0.5, 0.1], torch.float32) if mixed else pick([0.9, 0.95], torch.float32) if "p" in f else None
        s["min_p"] = pick([0.0, 0.01, 0.1], torch.float32) if mixed else pick([0.02, 0.05], torch.float32) if "m" in f else None
        s.update(token=torch.empty((R,), dtype=torch.int32, device="cuda"), logprob=torch.empty((R,), device="cuda"))
        return s
    Hq, Hkv, D = GEOMETRY[case["geometry"]]
    if case["kind"] == "axes":
        raw = torch.float32 if case["dtype"] == "f32" else torch.bfloat16
        # rows of a fused projection: the heads that are rotated, then as many value heads as there are KV heads
        fused = _normal(gen, (case["tokens"], case["heads"] + Hkv, D), 1.0, raw)
        return dict(case=case, x=fused[:, :case["heads"]], positions=_positions(case, case["tokens"], gen),
                    y=torch.empty((case["tokens"], case["heads"], D), dtype=raw, device="cuda"))
    s = _inputs(case, gen, "bf16" if case["kind"] == "axes_append" else "int8")
    L, T = case["layers"], s["tokens"]
    if case["kind"] == "attn":
        s["q"] = _normal(gen, (L, T, Hq, D), 2.0, torch.bfloat16)            # scores of std 2
    else:
        s["qkv"] = _normal(gen, (L, T, Hq + 2 * Hkv, D), 1.5, torch.bfloat16)    # the fused projection's rows
        s["q_weight"] = _normal(gen, (L, D), 0.2, torch.bfloat16)            # norm weights, stored less 1
        s["k_weight"] = _normal(gen, (L, D), 0.2, torch.bfloat16)
        if case["kind"] == "axes_append":
            s["positions"] = _positions(case, T, gen)
    s["out"] = torch.zeros((L, T, Hq, D), dtype=torch.bfloat16, device="cuda")
    return s


# ---------------------------------------------------------------------------- plain forms

def _theta(case, r, device):
    """Angular frequencies of a rotary over r components, in 64 bits."""
    p = SCALING[case["scaling"]]
    theta = torch.pow(torch.tensor(BASE, dtype=torch.float64, device=device),
                      -2.0 * torch.arange(r // 2, dtype=torch.float64, device=device) / r)
    if p["scaling"] == "linear":
        return theta / p["factor"]
    if p["scaling"] == "rotations":
        keep = ((p["original"] * theta / (2 * math.pi) - p["slow"]) / (p["fast"] - p["slow"])).clamp(0, 1)
        return theta * keep + theta / p["factor"] * (1 - keep)
    return theta


def _axis_pairs(case):
    """Pairs of each axis, and the axis of each pair of a head."""
    a = AXES[case["axes"]]
    n = GEOMETRY[case["geometry"]][2] // 2
    pairs = [n * x // 32 for x in a["share"]]
    if a["order"] == "sections":
        return pairs, [k for k, c in enumerate(pairs) for _ in range(c)]
    left, axis = list(pairs), []
    while len(axis) < n:
        for k in range(len(left)):
            if left[k]:
                left[k] -= 1
                axis.append(k)
    return pairs, axis


def _angles(case, positions):
    """Angle of every token and pair, in 64 bits."""
    D = GEOMETRY[case["geometry"]][2]
    if "axes" not in case:
        return positions.double()[:, None] * _theta(case, D, positions.device)
    pairs, axis = _axis_pairs(case)
    theta = torch.cat([_theta(case, 2 * c, positions.device) for c in pairs]) if AXES[case["axes"]]["own"] else _theta(case, D, positions.device)
    return positions[torch.tensor(axis, device=positions.device)].double().t() * theta


def _rotate_plain(case, x, positions):
    """x [..., tokens, heads, D] in 32 bits, angles in 64."""
    angle = _angles(case, positions)[:, None]
    cos, sin = angle.cos().float(), angle.sin().float()
    if "axes" not in case or AXES[case["axes"]]["pairing"] == "half":
        a, b = x.chunk(2, dim=-1)
        return torch.cat([a * cos - b * sin, a * sin + b * cos], dim=-1)
    a, b = x[..., 0::2], x[..., 1::2]
    return torch.stack([a * cos - b * sin, a * sin + b * cos], dim=-1).flatten(-2)


def _normed_plain(s, at, positions):
    """Queries, keys and values of the call's tokens, normed and rotated, in 32 bits."""
    case = s["case"]
    Hq, Hkv, D = GEOMETRY[case["geometry"]]
    x = s["qkv"].float()
    norm = lambda h, w: (h * torch.rsqrt(h.square().mean(-1, keepdim=True) + EPS) *  # noqa: E731
                         (1.0 + w.float()[:, None, None, :]))
    return (_rotate_plain(case, norm(x[:, :, :Hq], s["q_weight"]), positions),
            _rotate_plain(case, norm(x[:, :, Hq:Hq + Hkv], s["k_weight"]), positions), x[:, :, Hq + Hkv:])


def _values(pool, scale):
    """The values that pages of 8-bit integers stand for."""
    return torch.mul(pool, scale[..., None, None], out=torch.empty(pool.shape, dtype=torch.bfloat16, device=pool.device))


def _append_plain(s):
    at = s["ctx"][s["seq"]] + s["off"]
    q, k, v = _normed_plain(s, at, s["start"][s["seq"]] + at)
    s["out"].copy_(q)
    page, row = s["table"][s["seq"], at // PAGE].long(), at % PAGE
    P = s["k_pool"].shape[1]
    # rows that a page of the call held before it: those below the first new token in the page that it falls into
    held = torch.zeros(P, dtype=torch.long, device="cuda")
    held[page] = torch.where(at // PAGE == s["ctx"][s["seq"]] // PAGE, s["ctx"][s["seq"]] % PAGE, 0).long()
    touched = torch.zeros(P, dtype=torch.bool, device="cuda")
    touched[page] = True
    old = touched[:, None] & (torch.arange(PAGE, device="cuda") < held[:, None])             # [P][PAGE]
    for pool, scale, rows in ((s["k_pool"], s["k_scale"], k), (s["v_pool"], s["v_scale"], v)):
        most = torch.zeros_like(scale).index_reduce_(1, page, rows.abs().amax(-1), "amax")     # [L][P][Hkv]
        before = torch.where((held > 0)[:, None], scale, 0.0)
        after = torch.where(touched[:, None], torch.maximum(before, most / 127.0), scale)
        ratio = torch.where(after > 0, before / after, 0.0)
        pool.copy_(torch.where(old[None, :, None, :, None], (pool * ratio[..., None, None]).round().to(torch.int8), pool))
        per_token = after[:, page][..., None]
        new = torch.where(per_token > 0, rows / per_token, 0.0).round().clamp(-127, 127).to(torch.int8)
        pool.permute(1, 3, 0, 2, 4)[page, row] = new.transpose(0, 1)      # the indexed axes come first
        scale.copy_(after)
    return dict(q=s["out"], k=_values(s["k_pool"], s["k_scale"]), v=_values(s["v_pool"], s["v_scale"]), k_scale=s["k_scale"],
                v_scale=s["v_scale"])


def _axes_append_plain(s):
    at = s["ctx"][s["seq"]] + s["off"]
    q, k, v = _normed_plain(s, at, s["positions"])
    s["out"].copy_(q)
    page, row = s["table"][s["seq"], at // PAGE].long(), at % PAGE
    for pool, rows in ((s["k_pool"], k), (s["v_pool"], v)):
        pool.permute(1, 3, 0, 2, 4)[page, row] = rows.to(torch.bfloat16).transpose(0, 1)
    return dict(q=s["out"], k_pool=s["k_pool"], v_pool=s["v_pool"])


def _gathered(s, pool, scale, n):
    """Keys or values [0, n) of every sequence: [L][B][Hkv][n][D] in 32 bits."""
    pages = s["table"][:, :-(-n // PAGE)].long()
    x = pool[:, pages].float() * scale[:, pages][..., None, None]
    return x.permute(0, 1, 3, 2, 4, 5).flatten(3, 4)[:, :, :, :n].contiguous()


def _attn_plain(s):
    case = s["case"]
    Hq, Hkv, D = GEOMETRY[case["geometry"]]
    L, B, M, n = case["layers"], case["batch"], s["longest"], s["max_keys"]
    rows = (s["cu"][:-1, None] + torch.arange(M, device="cuda")).clamp(max=s["tokens"] - 1)
    q = s["q"][:, rows].float().view(L, B, M, Hkv, Hq // Hkv, D).permute(0, 1, 3, 2, 4, 5).flatten(3, 4).contiguous()
    k = _gathered(s, s["k_pool"], s["k_scale"], n)
    scores = torch.matmul(q, k.transpose(-1, -2)) * (1.0 / math.sqrt(D))
    at = s["ctx"][:, None] + torch.arange(M, device="cuda")                       # [B][M] index of each row
    key = torch.arange(n, device="cuda")
    window = torch.tensor([w or n + 1 for w in _windows(case)], device="cuda")[:, None, None, None]
    hidden = (key > at[..., None]) | (key <= at[..., None] - window)              # [L][B][M][n]
    scores = scores.view(L, B, Hkv, M, Hq // Hkv, n).masked_fill_(hidden[:, :, None, :, None], -math.inf)
    p = (scores - scores.amax(-1, keepdim=True)).exp_()
    o = torch.matmul((p / p.sum(-1, keepdim=True)).flatten(3, 4), _gathered(s, s["v_pool"], s["v_scale"], n))
    o = o.view(L, B, Hkv, M, Hq // Hkv, D).permute(0, 1, 3, 2, 4, 5).reshape(L, B, M, Hq, D)
    s["out"].copy_(o[:, s["seq"], s["off"]])
    return s["out"]


def _sample_plain(s):
    """In 64 bits: the borders between tokens lie as close as the smallest weights."""
    logits, V = s["logits"], s["case"]["vocab"]
    t = s["temperature"].double()[:, None]
    order = torch.sort(logits, dim=1, descending=True, stable=True).indices        # equal ones: the lowest index first
    y = (logits.double() - logits.gather(1, order[:, :1]).double()) / torch.where(t > 0, t, 1.0)
    e = y.exp()
    es = e.gather(1, order)
    rank = torch.arange(V, device="cuda")
    keep = torch.ones_like(es, dtype=torch.bool)
    if s["top_k"] is not None:
        keep &= rank < torch.where(s["top_k"] > 0, s["top_k"], V)[:, None]
    if s["top_p"] is not None:
        # the fewest of them, from the likeliest on, that reach top_p of their sum
        p = s["top_p"].double()[:, None]
        c = (es * keep).cumsum(1)
        keep &= (c - es < p * c[:, -1:]) | (p >= 1.0) | (rank == 0)
    if s["min_p"] is not None:
        keep &= es >= s["min_p"].double()[:, None]
    w = e * torch.zeros_like(keep).scatter_(1, order, keep)
    c = w.cumsum(1)
    token = (c <= s["u"][:, None] * c[:, -1:]).sum(1, keepdim=True).clamp(max=V - 1)
    logprob = y.gather(1, token) - c[:, -1:].log()
    s["token"].copy_(torch.where(t > 0, token, order[:, :1])[:, 0])
    s["logprob"].copy_(torch.where(t > 0, logprob, 0.0)[:, 0])
    return dict(token=s["token"], logprob=s["logprob"])


# ---------------------------------------------------------------------------- the framework's calls

def _handle(s):
    """What a serving program keeps beside the tensors: the cache, the batch, the rotary plan, the workspace."""
    from paper_2607_14431_amd import kvg
    case = s["case"]
    h = dict(kvg=kvg)
    if case["kind"] == "sample":
        h["ws"] = kvg.sample_workspace(case["rows"], case["vocab"], s["logits"].device)
        return h
    Hq, Hkv, D = GEOMETRY[case["geometry"]]
    if "axes" in case:
        a = AXES[case["axes"]]
        h["axes"] = kvg.Axes(s["positions"], tuple(_axis_pairs(case)[0]),
                             order={"sections": kvg.KVG_AXES_SECTIONS, "turns": kvg.KVG_AXES_TURNS}[a["order"]],
                             own_frequencies=a["own"])
    if case["kind"] != "attn":
        p = SCALING[case["scaling"]]
        pairing = AXES[case["axes"]]["pairing"] if "axes" in case else "half"
        h["rotary"] = kvg.rotary(BASE, pairing={"half": kvg.KVG_ROPE_HALF, "interleaved": kvg.KVG_ROPE_INTERLEAVED}[pairing],
                                 scaling=getattr(kvg, "KVG_ROTARY_" + p["scaling"].upper()), factor=p["factor"],
                                 original_len=p["original"], fast=p["fast"], slow=p["slow"])
    if case["kind"] == "axes":
        return h
    windows = tuple(_windows(case)) if case.get("window") else None
    if case["kind"] == "axes_append":
        h["cache"] = kvg.Cache(s["k_pool"], s["v_pool"], Hq, windows)
    else:
        h["cache"] = kvg.Int8Cache(s["k_pool"], s["v_pool"], s["k_scale"], s["v_scale"], Hq, windows)
    h["seqs"] = kvg.Seqs(s["table"], s["ctx"], s["start"], s["max_ctx"])
    h["packed"] = kvg.Packed(s["cu"], s["tokens"], s["longest"])
    if case["kind"] == "attn":
        h["ws"] = kvg.int8_attn_workspace(h["cache"], h["seqs"], h["packed"], case["layers"])
    else:
        h["norm"] = kvg.HeadNorm(s["q_weight"], s["k_weight"], EPS, 1.0)
    return h


def _own(s):
    case = s["case"]
    if "handle" not in s:
        s["handle"] = _handle(s)
    h = s["handle"]
    kvg = h["kvg"]
    if case["kind"] == "sample":
        kvg.kvg_sample(s["logits"], s["temperature"], s["u"], s["token"], h["ws"], top_k=s["top_k"], top_p=s["top_p"],
                       min_p=s["min_p"], logprobs=s["logprob"])
        return dict(token=s["token"], logprob=s["logprob"])
    if case["kind"] == "axes":
        kvg.kvg_rotate_axes(h["rotary"], h["axes"], s["x"], s["y"])
        return s["y"]
    Hq, Hkv, D = GEOMETRY[case["geometry"]]
    if case["kind"] == "attn":
        kvg.kvg_int8_attn(h["cache"], h["seqs"], h["packed"], 0, case["layers"], s["q"], 1.0 / math.sqrt(D), s["out"], h["ws"])
        return s["out"]
    x = s["qkv"]
    rows = x[:, :, :Hq], x[:, :, Hq:Hq + Hkv], x[:, :, Hq + Hkv:]
    if case["kind"] == "axes_append":
        kvg.kvg_norm_append_axes(h["cache"], h["seqs"], h["packed"], h["rotary"], h["axes"], h["norm"], 0, case["layers"], *rows, s["out"])
        return dict(q=s["out"], k_pool=s["k_pool"], v_pool=s["v_pool"])
    kvg.kvg_int8_append(h["cache"], h["seqs"], h["packed"], h["rotary"], h["norm"], 0, case["layers"], *rows, s["out"])
    return dict(q=s["out"], k=_values(s["k_pool"], s["k_scale"]), v=_values(s["v_pool"], s["v_scale"]), k_scale=s["k_scale"],
                v_scale=s["v_scale"])


def run(state):
    if own:
        return _own(state)
    kind = state["case"]["kind"]
    if kind == "axes":
        state["y"].copy_(_rotate_plain(state["case"], state["x"].float(), state["positions"]))
        return state["y"]
    return {"append": _append_plain, "axes_append": _axes_append_plain, "attn": _attn_plain, "sample": _sample_plain}[kind](state)


# ---------------------------------------------------------------------------- definitions in 64 bits

def _turned(case, x, positions):
    """x [..., tokens, heads, D] in 64 bits, each pair a complex number times e^(i position theta)."""
    D = x.shape[-1]
    p = SCALING[case["scaling"]]

    def frequency(j, r):
        t = math.exp(-2.0 * j / r * math.log(BASE))
        if p["scaling"] == "linear":
            return t / p["factor"]
        if p["scaling"] == "rotations":
            g = min(max((p["original"] * t / (2.0 * math.pi) - p["slow"]) / (p["fast"] - p["slow"]), 0.0), 1.0)
            return t * (g + (1.0 - g) / p["factor"])
        return t

    angles = []
    if "axes" in case:
        a = AXES[case["axes"]]
        counts, seen = [D // 2 * c // 32 for c in a["share"]], [0] * len(a["share"])
        k = 0
        for i in range(D // 2):
            while seen[k] == counts[k]:
                k = (k + 1) % len(counts)
            angles.append(positions[k].double() * (frequency(seen[k], 2 * counts[k]) if a["own"] else frequency(i, D)))
            seen[k] += 1
            if a["order"] == "turns":
                k = (k + 1) % len(counts)
        half = a["pairing"] == "half"
    else:
        angles, half = [positions.double() * frequency(i, D) for i in range(D // 2)], True
    angle = torch.stack(angles, dim=-1)
    unit = torch.polar(torch.ones_like(angle), angle)[:, None]
    if half:
        z = torch.complex(x[..., :D // 2].contiguous(), x[..., D // 2:].contiguous()) * unit
        return torch.cat([z.real, z.imag], dim=-1)
    return torch.view_as_real(torch.view_as_complex(x.reshape(*x.shape[:-1], D // 2, 2).contiguous()) * unit).flatten(-2)


def _sample_exact(s):
    tokens, logprobs = [], []
    param = {k: None if s[k] is None else s[k].tolist() for k in ("temperature", "top_k", "top_p", "min_p", "u")}
    for r, row in enumerate(s["logits"].cpu().numpy()):
        order = numpy.argsort(-row, kind="stable")
        t = param["temperature"][r]
        if t == 0:
            tokens.append(int(order[0]))
            logprobs.append(0.0)
            continue
        y = (row.astype(numpy.longdouble) - row[order[0]]) / numpy.longdouble(t)
        e = numpy.exp(y)
        n = len(row)
        if param["top_k"] is not None and param["top_k"][r] > 0:
            n = min(n, param["top_k"][r])
        if param["top_p"] is not None and param["top_p"][r] < 1:
            c = numpy.cumsum(e[order[:n]])
            n = max(1, int(numpy.searchsorted(c, param["top_p"][r] * c[-1], side="left")) + 1)
        if param["min_p"] is not None:
            n = min(n, int((e[order] >= param["min_p"][r]).sum()))
        kept = numpy.sort(order[:n])
        c = numpy.cumsum(e[kept])
        i = min(int(numpy.searchsorted(c, param["u"][r] * c[-1], side="right")), n - 1)
        tokens.append(int(kept[i]))
        logprobs.append(float(y[kept[i]] - numpy.log(c[-1])))
    return dict(token=torch.tensor(tokens, dtype=torch.int32), logprob=torch.tensor(logprobs, dtype=torch.float64))


def _normed_exact(s, b, positions):
    """Sequence b's queries, keys and values in 64 bits."""
    case = s["case"]
    Hq, Hkv, D = GEOMETRY[case["geometry"]]
    r0, n = sum(s["lens"][:b]), s["lens"][b]
    x = s["qkv"][:, r0:r0 + n].double()
    parts = []
    for h0, h1, w in ((0, Hq, s["q_weight"]), (Hq, Hq + Hkv, s["k_weight"])):
        h = x[:, :, h0:h1]
        rms = (torch.linalg.vector_norm(h, dim=-1, keepdim=True) ** 2 / D + EPS).sqrt()
        parts.append(_turned(case, h / rms * (w.double() + 1.0)[:, None, None, :], positions))
    return parts + [x[:, :, Hq + Hkv:]]


def _append_exact(s):
    case = s["case"]
    q = torch.empty(s["out"].shape, dtype=torch.float64, device="cuda")
    int8 = case["kind"] == "append"
    pools = [s["k_pool"].double(), s["v_pool"].double()]
    scales = [s["k_scale"].double(), s["v_scale"].double()] if int8 else None
    r0 = 0
    for b, (n, c) in enumerate(zip(s["lens"], s["ctxs"])):
        if not n:
            continue
        pos = s["positions"][:, r0:r0 + n] if "axes" in case else s["start"][b] + torch.arange(c, c + n, device="cuda")
        qn, *kv = _normed_exact(s, b, pos)
        q[:, r0:r0 + n] = qn
        for j in range(2):
            for t0 in range(c - c % PAGE, c + n, PAGE):
                lo, hi = max(t0, c), min(t0 + PAGE, c + n)
                page = int(s["table"][b, t0 // PAGE])
                new = kv[j][:, lo - c:hi - c].transpose(1, 2)             # [L][Hkv][rows][D]
                if int8:
                    most = new.abs().amax((2, 3)) / 127
                    if lo > t0:
                        was = scales[j][:, page]
                        now = torch.maximum(was, most)
                        held = pools[j][:, page, :, :lo - t0]
                        pools[j][:, page, :, :lo - t0] = torch.round(held * (was / now)[:, :, None, None])
                    else:
                        now = most
                    scales[j][:, page] = now
                    new = torch.round(new / now[:, :, None, None])
                pools[j][:, page, :, lo - t0:hi - t0] = new
        r0 += n
    if not int8:
        return dict(q=q, k_pool=pools[0], v_pool=pools[1])
    k, v = (x * y[..., None, None] for x, y in zip(pools, scales))
    return dict(q=q, k=k, v=v, k_scale=scales[0], v_scale=scales[1])


def _attn_exact(s):
    case = s["case"]
    Hq, Hkv, D = GEOMETRY[case["geometry"]]
    out = torch.empty(s["out"].shape, dtype=torch.float64, device="cuda")
    for l, w in enumerate(_windows(case)):
        r0 = 0
        for b, (n, c) in enumerate(zip(s["lens"], s["ctxs"])):
            if not n:
                continue
            pages = s["table"][b, :-(-(c + n) // PAGE)].long()
            k, v = ((pool[l].index_select(0, pages).double() * scale[l].index_select(0, pages).double()[:, :, None, None])
                    .transpose(0, 1).flatten(1, 2)[:, :c + n] for pool, scale in ((s["k_pool"], s["k_scale"]), (s["v_pool"], s["v_scale"])))
            for i0 in range(0, n, 1024):                       # rows a thousand at a time
                i1 = min(i0 + 1024, n)
                hi, lo = c + i1, max(0, c + i0 - w + 1) if w else 0
                q = s["q"][l, r0 + i0:r0 + i1].double().view(i1 - i0, Hkv, Hq // Hkv, D)
                e = torch.einsum("ihgd,hjd->hgij", q, k[:, lo:hi]) / math.sqrt(D)
                i, j = torch.arange(c + i0, c + i1, device="cuda")[:, None], torch.arange(lo, hi, device="cuda")
                seen = (j <= i) & (j > i - w) if w else j <= i
                weight = torch.softmax(e.masked_fill(~seen, -math.inf), dim=-1)
                out[l, r0 + i0:r0 + i1] = torch.einsum("hgij,hjd->ihgd", weight, v[:, lo:hi]).reshape(i1 - i0, Hq, D)
            r0 += n
    return out


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "sample":
        return _sample_exact(s)
    if case["kind"] == "axes":
        return _turned(case, s["x"].double(), s["positions"])
    return _attn_exact(s) if case["kind"] == "attn" else _append_exact(s)
