"""Timed cases of the 8-bit projections and the expert routing, in a plain form and through the library.

Three operators: the router (scores, bias, groups, the best experts and their
weights), a projection of bf16 activations by 8-bit weights (rows to codes, then
the integer product with a scale for each row and each channel), and the
feed-forward of routed experts in 8 bits.  The sizes are those of the decoders in
perf/cases.py: the Qwen3-8B- and Qwen3-30B-A3B-shaped ones and the small one,
with other expert counts and odd sizes beside them.
"""
import math
from types import SimpleNamespace

import torch

own = False
DEV = "cuda"
F64 = torch.float64

# Decoder projections (output channels, input channels, epilogue): 0 fp32 results,
# 1 bf16 results, 3 SwiGLU (gate and up rows interleaved in groups of 16).
PROJ = {
    "8b-qkv": (6144, 4096, 0), "8b-o": (4096, 4096, 1), "8b-gate-up": (24576, 4096, 3), "8b-down": (4096, 12288, 1),
    "moe-qkv": (5120, 2048, 0), "moe-o": (2048, 4096, 1),
    "small-qkv": (1536, 1024, 0), "small-gate-up": (8192, 1024, 3), "small-down": (1024, 4096, 1),
    "odd": (4112, 2064, 1), "odd-gate-up": (5664, 1456, 3), "odd-f32": (1552, 720, 0),
}
# Expert layers: d_model, experts, experts per row, expert hidden size.
LAYERS = {
    "moe": (2048, 128, 8, 768), "moe-small": (1024, 16, 4, 512), "moe-wide": (1024, 64, 6, 1408),
    "moe-odd": (1456, 60, 4, 720),
}


def listed():
    return [
        # the last live trajectory of a rollout: latency of one launch
        dict(name="route-1", kind="route", rows=1, experts=128, k=8, groups=1, top_groups=1, group_best=1,
             score="softmax", bias=False, dtype="f32"),
        # a decode step of a router with a balance bias and expert groups
        dict(name="route-976-groups", kind="route", rows=976, experts=256, k=8, groups=8, top_groups=4, group_best=2,
             score="sigmoid", bias=True, dtype="bf16"),
        # the prefill of 64 prompts of 512 tokens
        dict(name="route-32768", kind="route", rows=32768, experts=128, k=8, groups=1, top_groups=1, group_best=1,
             score="softmax", bias=False, dtype="f32"),
        # decoder projections: the last trajectory, the tail of a rollout, a full
        # decode batch, sizes that divide no tile, and the largest one of a prefill
        dict(name="linear-qkv-1", kind="linear", proj="8b-qkv", rows=1),
        dict(name="linear-down-45", kind="linear", proj="8b-down", rows=45),
        dict(name="linear-gate-up-389", kind="linear", proj="8b-gate-up", rows=389),
        dict(name="linear-odd-777", kind="linear", proj="odd", rows=777),
        dict(name="linear-prefill-gate-up", kind="linear", proj="8b-gate-up", rows=16384),
        # an expert layer: the last trajectory, the tail, a full decode batch, a prefill
        dict(name="experts-1", kind="experts", layer="moe", rows=1),
        dict(name="experts-61", kind="experts", layer="moe", rows=61),
        dict(name="experts-976", kind="experts", layer="moe", rows=976),
        dict(name="experts-prefill", kind="experts", layer="moe", rows=32768),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["route", "linear", "linear", "experts"])
    if kind == "route":
        experts = rng.choice([8, 16, 60, 64, 96, 128, 160, 256])
        groups = rng.choice([1, 1, 4, 8]) if experts % 8 == 0 else 1
        top = rng.randint(1, groups)
        k = min(rng.choice([1, 2, 4, 6, 8]), experts // groups * top)
        return dict(kind=kind, rows=_log(rng, 1, 32768), experts=experts, k=k, groups=groups, top_groups=top,
                    group_best=rng.choice([1, 2]), score=rng.choice(["softmax", "sigmoid"]),
                    bias=rng.random() < 0.5, dtype=rng.choice(["f32", "bf16"]))
    if kind == "linear":
        return dict(kind=kind, proj=rng.choice(sorted(PROJ)), rows=_log(rng, 1, 16384))
    return dict(kind=kind, layer=rng.choice(sorted(LAYERS)), rows=_log(rng, 1, 16384))


def _gen(seed, salt):
    return torch.Generator(device=DEV).manual_seed(int(seed) * 1000003 + salt)


# --------------------------------------------------------------------- router
def _route_inputs(case, seed):
    g = _gen(seed, 1)
    r, e = case["rows"], case["experts"]
    logits = torch.empty(r, e, device=DEV).normal_(0.0, 1.5, generator=g)
    # padding rows, as in a batch of prompts of several lengths, are masked out whole
    pad = torch.rand(r, 1, device=DEV, generator=g) < (0.02 if r > 16 else 0.0)
    logits = logits.masked_fill(pad, -math.inf)
    logits = logits.bfloat16() if case["dtype"] == "bf16" else logits
    bias = torch.empty(e, device=DEV).normal_(0.0, 0.05, generator=g) if case["bias"] else None
    return logits, bias


def _route_prepare(case, seed):
    logits, bias = _route_inputs(case, seed)
    shape = (case["rows"], case["k"])
    return SimpleNamespace(case=case, logits=logits, bias=bias, ids=torch.empty(shape, dtype=torch.int32, device=DEV),
                           weights=torch.empty(shape, device=DEV))


def _best(t, n):
    """The n largest values of each row and their places, the lower place first among equals."""
    v, i = torch.sort(t, dim=-1, descending=True, stable=True)
    return v[..., :n], i[..., :n]


def _route_plain(s):
    """Scores in 64 bits: which of two experts is taken hangs on their last digits."""
    c, x = s.case, s.logits.to(F64)
    r, e = x.shape
    bias = torch.zeros(e, dtype=F64, device=DEV) if s.bias is None else s.bias.to(F64)
    bad = (torch.isnan(x + bias) | (x + bias == math.inf)).any(1, keepdim=True)
    if c["score"] == "softmax":
        top = x.amax(1, keepdim=True)
        p = torch.exp(x - torch.where(top == -math.inf, torch.zeros_like(top), top))
        total = p.sum(1, keepdim=True)
        p = p / torch.where(total == 0, torch.ones_like(total), total)
    else:
        p = 1.0 / (1.0 + torch.exp(-x))
    t = torch.where((x > -math.inf) & (bias > -math.inf), p + bias, torch.full_like(p, -math.inf))
    n = c["groups"]
    two = _best(t.view(r, n, e // n), c["group_best"])[0]
    value = torch.where(two[..., 1:] == -math.inf, torch.zeros_like(two[..., 1:]), two[..., 1:]).sum(-1) + two[..., 0]
    chosen = _best(value, c["top_groups"])[1]
    keep = torch.zeros(r, n, dtype=torch.bool, device=DEV).scatter_(1, chosen, True)
    t = torch.where(keep.repeat_interleave(e // n, 1), t, torch.full_like(t, -math.inf))
    v, ids = _best(t, c["k"])
    some = (v > -math.inf) & ~bad
    w = torch.where(some, p.gather(1, ids), torch.zeros_like(v))
    total = w.sum(1, keepdim=True)
    w = w / torch.where(total == 0, torch.ones_like(total), total)
    w = torch.where(bad, torch.full_like(w, math.nan), w)
    return torch.where(some, ids, torch.full_like(ids, -1)).int(), w


def _route_run(s):
    if own:
        from paper_2605_30859_amd import binding as B
        c = s.case
        B.darts_moe_route(s.logits, B.DARTS_BF16 if c["dtype"] == "bf16" else B.DARTS_F32, s.ids, s.weights,
                          score=B.SCORE_SIGMOID if c["score"] == "sigmoid" else B.SCORE_SOFTMAX, bias=s.bias,
                          n_groups=c["groups"], top_groups=c["top_groups"], group_best=c["group_best"])
        return dict(ids=s.ids, weights=s.weights)
    ids, w = _route_plain(s)
    return dict(ids=ids, weights=w.float())


def _route_exact(case, seed):
    """By log-probabilities and one pick after the other, rather than by sorting."""
    logits, bias = _route_inputs(case, seed)
    x = logits.to(F64)
    r, e = x.shape
    n, per = case["groups"], e // case["groups"]
    real = (x > -math.inf).any(1, keepdim=True)
    if case["score"] == "softmax":
        p = torch.exp(x - torch.logsumexp(torch.where(real, x, torch.zeros_like(x)), 1, keepdim=True))
    else:
        p = torch.special.expit(x)
    t = p if bias is None else p + bias.to(F64)
    t = torch.where(x > -math.inf, t, torch.full_like(t, -math.inf))
    groups = t.view(r, n, per)
    value = groups.amax(2)
    if case["group_best"] == 2 and per > 1:
        value = value + torch.topk(groups, 2, dim=2).values[..., 1].clamp_min(-1e300)
    out = torch.zeros_like(value, dtype=torch.bool)
    rows = torch.arange(r, device=DEV)
    for _ in range(case["top_groups"]):
        g = torch.where(out, torch.full_like(value, -math.inf), value).argmax(1)
        out[rows, g] = True
    t = torch.where(out.unsqueeze(2).expand(r, n, per).reshape(r, e), t, torch.full_like(t, -math.inf))
    weights = torch.zeros(r, case["k"], dtype=F64, device=DEV)
    for j in range(case["k"]):
        best, i = t.max(1)
        weights[:, j] = torch.where(best > -math.inf, p[rows, i], torch.zeros_like(best))
        t[rows, i] = -math.inf
    total = weights.sum(1, keepdim=True)
    return dict(ids=None, weights=torch.where(total > 0, weights / total, torch.zeros_like(weights)))


def _route_work(case):
    r, e = case["rows"], case["experts"]
    return dict(bytes=r * e * (2.0 if case["dtype"] == "bf16" else 4.0) + 8.0 * r * case["k"], flops=20.0 * r * e)


# --------------------------------------------------------- 8-bit projections
def _codes(w):
    """Weight rows as codes and scales, the way weights are stored."""
    top = w.abs().amax(-1, keepdim=True)
    scale = torch.full_like(top, 1.0) * (top / 127.0)
    return torch.round(w / scale).clamp_(-127, 127).to(torch.int8), scale.squeeze(-1).contiguous()


def _linear_inputs(case, seed):
    n, k, _ = PROJ[case["proj"]]
    g = _gen(seed, 2)
    x = torch.empty(case["rows"], k, device=DEV).normal_(generator=g)
    # a few channels of activations are much larger than the rest
    x *= 1.0 + 15.0 * (torch.rand(k, device=DEV, generator=g) < 0.005)
    w, scale = _codes(torch.empty(n, k, device=DEV).normal_(0.0, 1.0 / math.sqrt(k), generator=g))
    return x.bfloat16(), w, scale


def _linear_prepare(case, seed):
    x, w, scale = _linear_inputs(case, seed)
    n, k, epi = PROJ[case["proj"]]
    m = case["rows"]
    return SimpleNamespace(x=x, w=w, w_scale=scale, m=m, n=n, k=k, epi=epi, ws=None,
                           q=torch.empty(m, k, dtype=torch.int8, device=DEV), q_scale=torch.empty(m, device=DEV),
                           c=torch.empty(m, n // 2 if epi == 3 else n, device=DEV,
                                         dtype=torch.float32 if epi == 0 else torch.bfloat16))


def _plain_rows(x):
    """Codes and scales of the rows of x: fp32 arithmetic, as the codes are defined."""
    x = x.float()
    top = x.abs().amax(-1, keepdim=True)
    up = torch.full_like(top, 127.0) / torch.where(top == 0, torch.ones_like(top), top)
    return torch.round(x * up).clamp(-127, 127), top / torch.full_like(top, 127.0)


def _swiglu(c):
    """silu(gate) * up of interleaved columns."""
    g = c.reshape(*c.shape[:-1], c.shape[-1] // 32, 2, 16)
    gate, up = g[..., 0, :], g[..., 1, :]
    return (gate / (1.0 + torch.exp(-gate)) * up).reshape(*c.shape[:-1], c.shape[-1] // 2)


def _linear_run(s):
    if own:
        from paper_2605_30859_amd import binding as B
        if s.ws is None:
            s.ws = torch.empty(B.darts_gemm_i8_workspace_bytes(s.m, s.n, s.k), dtype=torch.uint8, device=DEV)
        B.darts_quantize_rows(s.x, B.DARTS_BF16, s.q, s.q_scale)
        B.darts_gemm_i8(s.q, s.q_scale, s.w, s.w_scale, s.c, s.m, s.n, s.k, s.epi, s.ws)
        return s.c
    q, scale = _plain_rows(s.x)
    c = q @ s.w.float().t() * scale * s.w_scale
    if s.epi == 3:
        c = _swiglu(c)
    return c if s.epi == 0 else c.bfloat16()


def _exact_rows(x):
    """The codes by their definition (nearest to fl32(x fl32(127/max)), halves to
    even) and the scale fl32(max/127), both as 64-bit numbers."""
    top = x.float().abs().amax(-1, keepdim=True)
    up = (127.0 / top.to(F64)).float()
    return torch.round((x.to(F64) * up.to(F64)).float()).to(F64), (top.to(F64) / 127.0).float().to(F64)


def _exact_swiglu(c):
    cols = torch.arange(c.shape[-1] // 2, device=DEV)
    gate = cols // 16 * 32 + cols % 16
    g = c[..., gate]
    return g * torch.special.expit(g) * c[..., gate + 16]


def _linear_exact(case, seed):
    x, w, scale = _linear_inputs(case, seed)
    q, s = _exact_rows(x)
    c = torch.matmul(q, w.to(F64).t()) * (s * scale.to(F64))
    return _exact_swiglu(c) if PROJ[case["proj"]][2] == 3 else c


def _linear_work(case):
    n, k, epi = PROJ[case["proj"]]
    m = case["rows"]
    out = m * n * 4.0 if epi == 0 else m * n * 2.0 if epi == 1 else m * n * 1.0
    return dict(bytes=m * k * 2.0 + n * k * 1.0 + n * 4.0 + out, flops=2.0 * m * n * k)


# ------------------------------------------------------------ routed experts
def _experts_inputs(case, seed):
    d, e, k, f = LAYERS[case["layer"]]
    g = _gen(seed, 3)
    r = case["rows"]
    x = torch.empty(r, d, device=DEV).normal_(generator=g)
    x *= 1.0 + 15.0 * (torch.rand(d, device=DEV, generator=g) < 0.005)
    # some experts are called more often than others
    liking = torch.empty(e, device=DEV).normal_(0.0, 0.3, generator=g)
    score, ids = torch.topk(torch.empty(r, e, device=DEV).normal_(generator=g) + liking, k, dim=1)
    gu, s_gu = _codes(torch.empty(e, 2 * f, d, device=DEV).normal_(0.0, 1.0 / math.sqrt(d), generator=g))
    down, s_down = _codes(torch.empty(e, d, f, device=DEV).normal_(0.0, 1.0 / math.sqrt(f), generator=g))
    return x.bfloat16(), ids.int(), torch.softmax(score, 1), gu, s_gu, down, s_down


def _experts_prepare(case, seed):
    x, ids, weights, gu, s_gu, down, s_down = _experts_inputs(case, seed)
    return SimpleNamespace(layer=LAYERS[case["layer"]], x=x, ids=ids, weights=weights, gu=gu, s_gu=s_gu, down=down,
                           s_down=s_down, ws=None, out=torch.empty_like(x))


def _places(ids, experts):
    """For each (row, slot) pair a place in a table of [experts][the most that one expert has]."""
    flat = ids.reshape(-1).long()
    count = torch.bincount(flat, minlength=experts)
    most = int(count.max())
    order = torch.argsort(flat, stable=True)
    first = torch.cumsum(count, 0) - count
    nth = torch.empty_like(flat)
    nth[order] = torch.arange(flat.numel(), device=DEV) - first[flat[order]]
    return flat * most + nth, most


def _experts_run(s):
    d, e, k, f = s.layer
    if own:
        from paper_2605_30859_amd import binding as B
        if s.ws is None:
            s.ws = torch.empty(B.darts_moe_ffn_i8_workspace_bytes(s.x.shape[0], d, e, k, f), dtype=torch.uint8,
                               device=DEV)
        B.darts_moe_ffn_i8(s.x, s.ids, s.weights, e, f, s.gu, s.s_gu, s.down, s.s_down, s.out, 1, s.ws)
        return s.out
    r = s.x.shape[0]
    q, scale = _plain_rows(s.x)
    place, most = _places(s.ids, e)
    row = torch.arange(r, device=DEV).repeat_interleave(k)
    table = torch.zeros(e * most, d, device=DEV)
    table[place] = q[row]
    by_row = torch.zeros(e * most, 1, device=DEV)
    by_row[place] = scale[row]
    h = torch.bmm(table.view(e, most, d), s.gu.float().transpose(1, 2))
    h = _swiglu(h * by_row.view(e, most, 1) * s.s_gu.unsqueeze(1)).bfloat16()
    q, scale = _plain_rows(h)
    y = torch.bmm(q, s.down.float().transpose(1, 2)) * scale * s.s_down.unsqueeze(1)
    y = y.view(e * most, d)[place].view(r, k, d)
    return (y * s.weights.unsqueeze(2)).sum(1).bfloat16()


def _experts_exact(case, seed):
    """One expert after the other.  The hidden activations are bf16 and their codes
    those of bf16 rows: the operator's definition."""
    x, ids, weights, gu, s_gu, down, s_down = _experts_inputs(case, seed)
    out = torch.zeros(x.shape, dtype=F64, device=DEV)
    q, scale = _exact_rows(x)
    for e in range(gu.shape[0]):
        row, slot = torch.nonzero(ids == e, as_tuple=True)
        if not row.numel():
            continue
        c = torch.matmul(q[row], gu[e].to(F64).t()) * (scale[row] * s_gu[e].to(F64))
        h, s = _exact_rows(_exact_swiglu(c).float().bfloat16())
        y = torch.matmul(h, down[e].to(F64).t()) * (s * s_down[e].to(F64))
        out.index_add_(0, row, y * weights[row, slot].to(F64).unsqueeze(1))
    return out


def _experts_work(case):
    d, e, k, f = LAYERS[case["layer"]]
    r = case["rows"]
    touched = e * (1.0 - (1.0 - k / e) ** r)
    return dict(bytes=touched * (3.0 * d * f + 4.0 * (2 * f + d)) + 4.0 * r * d + 8.0 * r * k, flops=6.0 * r * k * d * f)


_OPS = {
    "route": (_route_prepare, _route_run, _route_exact, _route_work),
    "linear": (_linear_prepare, _linear_run, _linear_exact, _linear_work),
    "experts": (_experts_prepare, _experts_run, _experts_exact, _experts_work),
}


def prepare(case, seed):
    s = _OPS[case["kind"]][0](case, seed)
    s.run = _OPS[case["kind"]][1]
    return s


def run(state):
    return state.run(state)


def exact(case, seed):
    return _OPS[case["kind"]][2](case, seed)


def work(case):
    return _OPS[case["kind"]][3](case)
