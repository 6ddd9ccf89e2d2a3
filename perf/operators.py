"""Workloads of the language-model block operators: norms around a block, routing to experts, the fused matrix
product and the experts' products.

`run` computes an operator either in its plain form (elementary torch operations in 32 bits, rounded once at the
end) or, where `own` is true, through this framework's entry points.  Packed weights follow the framework's
sub-byte order: element e in byte e // (8 // bits), first element in the low bits, two's complement.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
SIZE = {"bf16": 2, "f16": 2, "f32": 4}


# ---------------------------------------------------------------- cases

def _norm(name, t, d, dtype="bf16", res="bf16", kind="rms", post=True, gates=1, pad=0):
    return dict(name=name, op="norm", t=t, d=d, dtype=dtype, res=res, kind=kind, post=post, gates=gates, pad=pad)


def _route(name, t, e, k, dtype="f32", score="softmax", groups=1, top_groups=1, masked=False):
    return dict(name=name, op="route", t=t, e=e, k=k, dtype=dtype, score=score, groups=groups, top_groups=top_groups,
                masked=masked)


def _matmul(name, t, k, m, bits, dtype="bf16", gated=False, act="none", bias=False, residual=False, pad=0):
    return dict(name=name, op="matmul", t=t, k=k, m=m, bits=bits, dtype=dtype, gated=gated, act=act, bias=bias,
                residual=residual, pad=pad)


def _experts(name, form, t, top, e, k, m, bits, dtype="bf16", gated=False, act="none", residual=False, dropped=False):
    return dict(name=name, op="experts", form=form, t=t, top=top, e=e, k=k, m=m, bits=bits, dtype=dtype, gated=gated,
                act=act, residual=residual, dropped=dropped)


def listed():
    return [
        # one decode step of a batch of 8: latency of the norm pair between two blocks
        _norm("norm decode", 8, 4096),
        # ragged rows of 4 sequences with a gate each, odd width, rows padded in memory, layer norm without a post norm
        _norm("norm ragged layer", 1004, 2049, dtype="f16", res="f16", kind="layer", post=False, gates=4, pad=15),
        # a long prompt with its residual stream kept in 32 bits
        _norm("norm prompt", 16384, 8192, res="f32"),
        # a decode batch through a small router
        _route("route decode", 64, 64, 4),
        # a long prompt through a router with a balance bias and limited groups, some tokens masked (padding)
        _route("route prompt groups", 32768, 256, 8, score="sigmoid", groups=16, top_groups=4, masked=True),
        # one token against INT-4 weights: the decode of a single user, all weight traffic
        _matmul("matmul one token int4", 1, 8192, 8192, 4, residual=True),
        # a decode batch against 16-bit weights with the gated activation of a feed-forward block
        _matmul("matmul batch16 gated", 16, 4096, 8192, 16, gated=True, act="silu"),
        # a chunk of prompt, odd everywhere, INT-2 weights, 16-bit floats of the other type, strided rows
        _matmul("matmul ragged int2", 333, 4104, 1001, 2, dtype="f16", act="relu", bias=True, residual=True, pad=24),
        # a prompt through a gated feed-forward projection with INT-8 weights
        _matmul("matmul prompt int8", 8192, 4096, 8192, 8, gated=True, act="silu"),
        # a decode batch through the experts' gated up projection, INT-4 weights
        _experts("experts dispatch decode", "dispatch", 16, 4, 64, 2048, 1024, 4, gated=True, act="silu"),
        # a prompt through the experts' gated up projection, 16-bit weights
        _experts("experts dispatch prompt", "dispatch", 8192, 4, 32, 2048, 1024, 16, gated=True, act="silu"),
        # a ragged prompt with dropped pairs through the down projection and the weighted sum, INT-8 weights
        _experts("experts combine prompt", "combine", 4099, 4, 32, 1024, 2048, 8, residual=True, dropped=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same ranges, no dearer than the largest listed one."""
    while True:
        c = _draw(rng)
        w = work(c)
        if w["flops"] <= 1.1e12 and w["bytes"] <= 1.6e9:
            c.pop("name")
            return c


def _draw(rng):
    op = rng.choice(["norm", "route", "matmul", "matmul", "experts", "experts"])
    dtype = rng.choice(["bf16", "bf16", "f16"])
    if op == "norm":
        gates = rng.choice([0, 1, 1, 3])
        t = _log(rng, 1, 16384)
        if gates > 1:
            t = -(-t // gates) * gates
        return _norm("", t, _log(rng, 64, 8192), dtype=dtype, res=rng.choice([dtype, "f32"]),
                     kind=rng.choice(["rms", "layer"]), post=rng.random() < 0.5, gates=gates, pad=rng.choice([0, 0, 7, 16]))
    if op == "route":
        groups = rng.choice([1, 1, 4, 8])
        e = groups * rng.randint(max(2, 8 // groups), 256 // groups)
        top_groups = groups if groups == 1 else rng.randint(2, groups)
        k = rng.randint(1, min(8, (e // groups) * top_groups))
        return _route("", _log(rng, 1, 32768), e, k, dtype=rng.choice(["f32", "bf16"]),
                      score=rng.choice(["softmax", "sigmoid"]), groups=groups, top_groups=top_groups,
                      masked=rng.random() < 0.5)
    bits = rng.choice([16, 8, 4, 2])
    gated = rng.random() < 0.4
    act = rng.choice(["silu", "gelu"]) if gated else rng.choice(["none", "relu", "gelu", "silu"])
    if op == "matmul":
        return _matmul("", _log(rng, 1, 8192), 4 * _log(rng, 16, 2048), _log(rng, 64, 8192), bits, dtype=dtype, gated=gated,
                       act=act, bias=rng.random() < 0.5, residual=rng.random() < 0.5, pad=rng.choice([0, 0, 5, 24]))
    e = rng.choice([8, 16, 32, 64])
    form = rng.choice(["dispatch", "combine"])
    if form == "combine":
        gated, act = False, "none"
    return _experts("", form, _log(rng, 1, 8192), rng.randint(1, 6), e, 8 * _log(rng, 16, 256), _log(rng, 64, 2048), bits,
                    dtype=dtype, gated=gated, act=act, residual=form == "combine" and rng.random() < 0.5,
                    dropped=rng.random() < 0.3)


def work(c):
    """Bytes and operations one pass cannot do without: inputs read once, outputs written once."""
    if c["op"] == "norm":
        n = c["t"] * c["d"]
        par = (c["gates"] + 1 + c["post"] + 2 * (c["kind"] == "layer")) * c["d"] * SIZE[c["dtype"]]
        return {"bytes": n * (2 * SIZE[c["dtype"]] + 2 * SIZE[c["res"]]) + par, "flops": n * 12}
    if c["op"] == "route":
        t, e, k = c["t"], c["e"], c["k"]
        return {"bytes": t * e * SIZE[c["dtype"]] + t * k * (4 + 4) + t * k * 8 + 4 * (e + 1), "flops": t * e * 4}
    rows = c["m"] * (2 if c["gated"] else 1)
    if c["op"] == "matmul":
        t = c["t"]
        b = rows * c["k"] * c["bits"] / 8 + rows * 4 * ((c["bits"] < 16) + c["bias"])
        b += t * c["k"] * 2 + t * c["m"] * 2 * (1 + c["residual"])
        return {"bytes": b, "flops": 2.0 * t * rows * c["k"]}
    pairs = c["t"] * c["top"]
    hit = c["e"] * (1 - (1 - 1 / c["e"]) ** pairs)  # experts that some token chose, on average
    b = hit * rows * (c["k"] * c["bits"] / 8 + 4 * (c["bits"] < 16)) + 4 * pairs
    if c["form"] == "dispatch":
        b += c["t"] * c["k"] * 2 + pairs * c["m"] * 2
    else:
        b += pairs * (c["k"] * 2 + 4) + c["t"] * c["m"] * 2 * (1 + c["residual"])
    live = 0.9 if c["dropped"] else 1.0
    return {"bytes": b, "flops": 2.0 * pairs * rows * c["k"] * live}


# ---------------------------------------------------------------- inputs

def _padded(v, pad):
    """The same values in rows `pad` elements further apart."""
    if not pad:
        return v.contiguous()
    buf = torch.zeros(v.shape[0], v.shape[1] + pad, dtype=v.dtype, device=v.device)
    buf[:, :v.shape[1]] = v
    return buf[:, :v.shape[1]]


def _weights(c, g, dev, experts):
    """Weight matrix (packed codes or 16-bit) and one scale a row, so that products come out near one."""
    rows = c["m"] * (2 if c["gated"] else 1)
    shape = ((experts,) if experts else ()) + (rows, c["k"])
    if c["bits"] == 16:
        w = torch.randn(shape, generator=g, device=dev, dtype=torch.float32) / math.sqrt(c["k"])
        return w.to(DTYPES[c["dtype"]]), None
    per = 8 // c["bits"]
    w = torch.randint(0, 256, shape[:-1] + (c["k"] // per,), generator=g, device=dev, dtype=torch.uint8)
    rms = math.sqrt((4.0 ** c["bits"] + 2) / 12)
    scale = (0.5 + torch.rand(shape[:-1], generator=g, device=dev)) / (rms * math.sqrt(c["k"]))
    return w, scale


def prepare(case, seed):
    c, dev = case, torch.device("cuda")
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    s = {"case": c}

    def normal(*shape, dtype="f32", mul=1.0):
        return (torch.randn(shape, generator=g, device=dev) * mul).to(DTYPES[dtype])

    if c["op"] == "norm":
        t, d, dt = c["t"], c["d"], c["dtype"]
        s["x"] = _padded(normal(t, d, dtype=dt) + 0.1, c["pad"])
        s["residual"] = _padded(normal(t, d, dtype=c["res"], mul=2.0), c["pad"])
        s["pre_weight"] = (1 + normal(d, mul=0.1)).to(DTYPES[dt])
        s["pre_bias"] = normal(d, dtype=dt, mul=0.1) if c["kind"] == "layer" else None
        s["post_weight"] = (1 + normal(d, mul=0.1)).to(DTYPES[dt]) if c["post"] else None
        s["gate"] = normal(c["gates"], d, dtype=dt) if c["gates"] else None
    elif c["op"] == "route":
        x = normal(c["t"], c["e"], mul=1.5) + normal(c["e"], mul=0.5)
        if c["masked"]:  # some experts closed, some tokens padding
            x[torch.rand(x.shape, generator=g, device=dev) < 0.05] = -math.inf
            x[torch.rand(c["t"], generator=g, device=dev) < 0.05] = -math.inf
        s["logits"] = x.to(DTYPES[c["dtype"]])
        s["bias"] = normal(c["e"], mul=0.1) if c["score"] == "sigmoid" else None
    elif c["op"] == "matmul":
        s["x"] = _padded(normal(c["t"], c["k"], dtype=c["dtype"]), c["pad"])
        s["w"], s["scale"] = _weights(c, g, dev, 0)
        s["bias"] = normal(c["m"] * (2 if c["gated"] else 1), mul=0.5) if c["bias"] else None
        s["residual"] = _padded(normal(c["t"], c["m"], dtype=c["dtype"]), c["pad"]) if c["residual"] else None
    else:
        t, top, e = c["t"], c["top"], c["e"]
        logits = normal(t, e) + normal(e, mul=0.5)
        s["weights"], ids = torch.softmax(logits, -1).topk(top)
        s["weights"] = s["weights"] / s["weights"].sum(-1, keepdim=True)
        if c["dropped"]:
            gone = torch.rand(ids.shape, generator=g, device=dev) < 0.1
            ids = ids.masked_fill(gone, -1)
            s["weights"] = s["weights"].masked_fill(gone, 0.0)
        s["ids"] = ids.to(torch.int32)
        s["x"] = normal(t if c["form"] == "dispatch" else t * top, c["k"], dtype=c["dtype"])
        s["w"], s["scale"] = _weights(c, g, dev, e)
        s["residual"] = normal(t, c["m"], dtype=c["dtype"]) if c["residual"] else None
    if own:
        from paper_1908_11263_gb300 import qnn
        s["qnn"] = qnn
        if c["op"] == "matmul":
            s["layer"] = qnn.PreparedMatmul(s["w"], scale=s["scale"], bias=s["bias"], bits=c["bits"],
                                            dtype=DTYPES[c["dtype"]], gated=c["gated"], act=c["act"])
        elif c["op"] == "experts":
            s["layer"] = qnn.PreparedExperts(s["w"], scale=s["scale"], bits=c["bits"], dtype=DTYPES[c["dtype"]],
                                             gated=c["gated"], act=c["act"])
    return s


# ---------------------------------------------------------------- one pass

def run(state):
    c = state["case"]
    if own:
        return _RUN_OWN[c["op"]](state, c, state["qnn"])
    return _RUN_PLAIN[c["op"]](state, c)


def _own_norm(s, c, qnn):
    return qnn.block_norm(s["x"], s["residual"], pre_weight=s["pre_weight"], pre_bias=s["pre_bias"], post_norm=c["post"],
                          post_weight=s["post_weight"], gate=s["gate"], scale=0.5, eps=1e-5, kind=c["kind"])


def _own_route(s, c, qnn):
    weights, ids = qnn.route_topk(s["logits"], c["k"], score=c["score"], bias=s["bias"], groups=c["groups"],
                                  top_groups=c["top_groups"], group_score="top2", renormalise=True, scale=2.5)
    plan = qnn.expert_plan(ids, c["e"])
    return weights, ids, plan.offsets, plan.order, plan.position


def _own_matmul(s, c, qnn):
    return s["layer"](s["x"], residual=s["residual"])


def _own_experts(s, c, qnn):
    plan = qnn.expert_plan(s["ids"], c["e"])
    if c["form"] == "dispatch":
        return s["layer"].dispatch(s["x"], plan)
    return s["layer"].combine(s["x"], plan, s["weights"], residual=s["residual"])


_RUN_OWN = {"norm": _own_norm, "route": _own_route, "matmul": _own_matmul, "experts": _own_experts}


def _normed(v, weight, bias, kind):
    if kind == "layer":
        v = v - v.mean(-1, keepdim=True)
    y = v * torch.rsqrt((v * v).mean(-1, keepdim=True) + 1e-5)
    y = y if weight is None else y * weight.float()
    return y if bias is None else y + bias.float()


def _plain_norm(s, c):
    u = s["x"].float()
    if c["post"]:
        u = _normed(u, s["post_weight"], None, c["kind"])
    if s["gate"] is not None:
        u = u * s["gate"].float().repeat_interleave(c["t"] // c["gates"], 0)
    r = s["residual"].float() + 0.5 * u
    h = _normed(r, s["pre_weight"], s["pre_bias"], c["kind"])
    return r.to(s["residual"].dtype), h.to(s["x"].dtype)


def _plan(ids, experts):
    """Slots (token * top + choice) sorted by expert, each expert's in order; dropped slots (-1) in none."""
    flat = ids.reshape(-1).long()
    key = torch.where(flat < 0, experts, flat)
    order = torch.sort(key, stable=True).indices
    counts = torch.bincount(key, minlength=experts + 1)[:experts]
    offsets = torch.cat([counts.new_zeros(1), counts.cumsum(0)])
    rank = torch.arange(flat.numel(), device=ids.device)
    position = torch.empty_like(flat)
    position[order] = rank
    position = torch.where(flat < 0, -1, position)
    order = torch.where(rank < offsets[-1], order, -1)
    return offsets.int(), order.int(), position.int().view(ids.shape)


def _plain_route(s, c):
    x = s["logits"].float()
    t, e, k = c["t"], c["e"], c["k"]
    dead = x == -math.inf
    if c["score"] == "softmax":
        top = x.amax(-1, keepdim=True)
        score = torch.exp(x - torch.where(top == -math.inf, torch.zeros_like(top), top))
        choose = x
    else:
        score = 1.0 / (1.0 + torch.exp(-x))
        choose = score + s["bias"]
    choose = choose.masked_fill(dead, -math.inf)
    if c["groups"] > 1:
        of = (score if s["bias"] is None else choose).masked_fill(dead, -math.inf).view(t, c["groups"], -1)
        two = of.sort(dim=-1, descending=True).values[..., :2]
        group = two[..., 0] + two[..., 1].masked_fill(two[..., 1] == -math.inf, 0.0)
        best = group.sort(dim=-1, descending=True, stable=True).indices[:, :c["top_groups"]]
        keep = torch.zeros(group.shape, dtype=torch.bool, device=x.device).scatter_(1, best, True)
        choose = choose.masked_fill(~keep.repeat_interleave(e // c["groups"], 1), -math.inf)
    by = torch.sort(choose, dim=-1, descending=True, stable=True)
    ids, none = by.indices[:, :k], by.values[:, :k] == -math.inf
    w = score.gather(1, ids).masked_fill(none, 0.0)
    total = w.sum(-1, keepdim=True)
    w = w / torch.where(total > 0, total, torch.ones_like(total)) * 2.5
    ids = ids.masked_fill(none, -1).int()
    return (w, ids) + _plan(ids, e)


def _unpacked(w, scale, bits):
    """Weights in 32 bits."""
    if bits == 16:
        return w.float()
    shifts = torch.arange(0, 8, bits, device=w.device, dtype=torch.uint8)
    v = (w.unsqueeze(-1) >> shifts) & ((1 << bits) - 1)
    v = v.float().flatten(-2)
    return torch.where(v >= (1 << (bits - 1)), v - (1 << bits), v) * scale.unsqueeze(-1)


def _act(v, act):
    if act == "relu":
        return v.clamp_min(0)
    if act == "silu":
        return v / (1 + torch.exp(-v))
    if act == "gelu":
        return 0.5 * v * (1 + torch.erf(v * math.sqrt(0.5)))
    return v


def _activated(v, c):
    if c["gated"]:
        return _act(v[..., :c["m"]], c["act"]) * v[..., c["m"]:]
    return _act(v, c["act"])


def _plain_matmul(s, c):
    v = s["x"].float() @ _unpacked(s["w"], s["scale"], c["bits"]).t()
    v = _activated(v if s["bias"] is None else v + s["bias"], c)
    return (v if s["residual"] is None else v + s["residual"].float()).to(s["x"].dtype)


def _plain_experts(s, c):
    offsets, order, position = _plan(s["ids"], c["e"])
    x, live = s["x"].float(), order >= 0
    if c["form"] == "dispatch":
        x = x[order.clamp_min(0).long() // c["top"]]
    # every expert's rows padded to the fullest expert's number
    most = max(1, int((offsets[1:] - offsets[:-1]).max()))
    at = offsets[:-1, None].long() + torch.arange(most, device=x.device)
    inside = at < offsets[1:, None]
    at = at.clamp_max(x.shape[0] - 1)
    v = torch.bmm(x[at], _unpacked(s["w"], s["scale"], c["bits"]).transpose(1, 2))
    v = _activated(v, c)
    out = torch.zeros(x.shape[0], c["m"], device=x.device)
    out[at[inside]] = v[inside]
    out = torch.where(live[:, None], out, torch.zeros_like(out))
    if c["form"] == "dispatch":
        return out.to(s["x"].dtype)
    w = s["weights"].masked_fill(position < 0, 0.0)
    y = (out[position.clamp_min(0).long()] * w[..., None]).sum(1)
    return (y if s["residual"] is None else y + s["residual"].float()).to(s["x"].dtype)


_RUN_PLAIN = {"norm": _plain_norm, "route": _plain_route, "matmul": _plain_matmul, "experts": _plain_experts}


# ---------------------------------------------------------------- 64 bits, from the definitions

def exact(case, seed):
    global own
    was, own = own, False
    s = prepare(case, seed)
    own = was
    return {"norm": _exact_norm, "route": _exact_route, "matmul": _exact_matmul, "experts": _exact_experts}[case["op"]](s, case)


def _exact_norm(s, c):
    def n(v, weight, bias):
        mean = v.mean(1, keepdim=True) if c["kind"] == "layer" else 0.0
        var = ((v - mean) ** 2).sum(1, keepdim=True) / c["d"]
        v = (v - mean) / torch.sqrt(var + 1e-5)
        v = v if weight is None else v * weight.double()
        return v if bias is None else v + bias.double()

    u = s["x"].double()
    u = n(u, s["post_weight"], None) if c["post"] else u
    if c["gates"]:
        u = (u.view(c["gates"], -1, c["d"]) * s["gate"].double()[:, None]).view(c["t"], c["d"])
    r = s["residual"].double() + u / 2
    return r, n(r, s["pre_weight"], s["pre_bias"])


def _exact_route(s, c):
    x = s["logits"].double()
    p = torch.sigmoid(x) if c["score"] == "sigmoid" else torch.softmax(x, 1).nan_to_num(0.0)
    pick = p + (s["bias"].double() if s["bias"] is not None else 0.0)
    pick[torch.isneginf(x)] = -math.inf
    if c["groups"] > 1:
        two = pick.view(c["t"], c["groups"], -1).topk(2, -1).values
        total = two[..., 0] + torch.where(torch.isneginf(two[..., 1]), 0.0, two[..., 1])
        out = total.sort(dim=1, descending=True, stable=True).indices[:, c["top_groups"]:]
        pick.view(c["t"], c["groups"], -1).scatter_(1, out[..., None].expand(-1, -1, c["e"] // c["groups"]), -math.inf)
    value, ids = pick.sort(dim=1, descending=True, stable=True)
    w = p.gather(1, ids[:, :c["k"]])
    w[torch.isneginf(value[:, :c["k"]])] = 0.0
    w = 2.5 * w / w.sum(1, keepdim=True)
    return w.nan_to_num(0.0), None, None, None, None


def _exact_codes(w, scale, bits):
    if bits == 16:
        return w.double()
    v = torch.stack([(w.to(torch.int32) // (1 << b)) % (1 << bits) for b in range(0, 8, bits)], -1).flatten(-2)
    return ((v + (1 << (bits - 1))) % (1 << bits) - (1 << (bits - 1))).double() * scale.double()[..., None]


def _exact_act(v, c):
    f = {"none": lambda a: a, "relu": lambda a: a.clamp(min=0.0), "silu": lambda a: a * torch.sigmoid(a),
         "gelu": lambda a: a * torch.special.ndtr(a)}[c["act"]]
    return f(v[:, :c["m"]]) * v[:, c["m"]:] if c["gated"] else f(v)


def _exact_matmul(s, c):
    v = torch.mm(s["x"].double(), _exact_codes(s["w"], s["scale"], c["bits"]).T)
    y = _exact_act(v + s["bias"].double() if c["bias"] else v, c)
    return y + s["residual"].double() if c["residual"] else y


def _exact_experts(s, c):
    flat = s["ids"].reshape(-1)
    dispatch = c["form"] == "dispatch"
    rows, y, done = [], torch.zeros(c["t"], c["m"], dtype=torch.float64, device=flat.device), 0
    for e in range(c["e"]):
        slots = (flat == e).nonzero()[:, 0]
        n = slots.numel()
        x = s["x"][slots // c["top"]] if dispatch else s["x"][done:done + n]
        done += n
        v = _exact_act(x.double() @ _exact_codes(s["w"][e], s["scale"][e] if s["scale"] is not None else None, c["bits"]).T, c)
        if dispatch:
            rows.append(v)
        else:
            y.index_add_(0, slots // c["top"], v * s["weights"].reshape(-1)[slots].double()[:, None])
    if dispatch:
        rows.append(torch.zeros(flat.numel() - done, c["m"], dtype=torch.float64, device=flat.device))
        return torch.cat(rows)
    return y + s["residual"].double() if c["residual"] else y
