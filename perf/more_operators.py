"""Workloads of the attention operators: rotary positions, appending to a paged cache with the rotation on the way,
attention over that cache (single tokens and prompts) and cross attention to an encoder's states.

`run` computes an operator either in its plain form (elementary torch operations in 32 bits, angles in 64, rounded once
at the end) or, where `own` is true, through this framework's entry points.  A cache is two tensors of pages
[pages, kv_heads, page_size, head_dim]; sequence s keeps token j in row j % page_size of page table[s][j // page_size].
"""
import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


# ---------------------------------------------------------------- cases

def _rope(name, t, heads, d, rotary, dtype="bf16", interleaved=False, scaling="none", far=0, pad=0):
    return dict(name=name, op="rope", t=t, heads=heads, d=d, rotary=rotary, dtype=dtype, interleaved=interleaved,
                scaling=scaling, far=far, pad=pad)


def _append(name, seqs, new, cached, heads, kv, d, page, dtype="bf16", interleaved=False, scaling="none", mix=1):
    return dict(name=name, op="append", seqs=seqs, new=new, cached=cached, heads=heads, kv=kv, d=d, page=page, dtype=dtype,
                interleaved=interleaved, scaling=scaling, mix=mix)


def _attend(name, seqs, new, cached, heads, kv, d, page, dtype="bf16", window=0, even=False, mix=1):
    return dict(name=name, op="attend", seqs=seqs, new=new, cached=cached, heads=heads, kv=kv, d=d, page=page, dtype=dtype,
                window=window, even=even, mix=mix)


def _cross(name, b, n, src, heads, kv, d, dtype="bf16", ragged=True, mix=1):
    return dict(name=name, op="cross", b=b, n=n, src=src, heads=heads, kv=kv, d=d, dtype=dtype, ragged=ragged, mix=mix)


def listed():
    return [
        # one decode step of a batch of 16: queries between the projection and the attention, far positions, scaled by parts
        _rope("rope decode", 16, 32, 128, 128, scaling="ramp", far=1000000, pad=2048),
        # a long prompt, neighbouring pairs, two thirds of the head rotated, odd number of tokens
        _rope("rope prompt partial", 20011, 20, 96, 64, dtype="f16", interleaved=True, scaling="linear"),
        # one decode step of 64 users: a token each into small pages
        _append("append decode", 64, 1, 500, 32, 8, 128, 16),
        # prompts of seven users, ragged, some onto a prefix that is there already
        _append("append prompt", 7, 4001, 1500, 32, 8, 128, 64, dtype="f16", interleaved=True, scaling="base"),
        # one user's next token over a long cache: latency, and one sequence over the whole GPU
        _attend("attend one user", 1, 1, 8190, 32, 8, 128, 64, even=True),
        # one decode step of 64 users with caches of very different lengths, some just begun: bandwidth
        _attend("attend decode batch", 64, 1, 24575, 32, 8, 128, 16),
        # a decode step of many short sequences, a key head for each query head, odd pages, a sliding window
        _attend("attend short window", 200, 1, 700, 16, 16, 64, 24, dtype="f16", window=256),
        # a long prompt attends to itself
        _attend("attend prompt", 1, 8192, 0, 32, 8, 128, 64, even=True),
        # a mixed step: some sequences have one new token, some a chunk of their prompt, all over a cache
        _attend("attend mixed chunks", 12, 600, 8000, 16, 2, 128, 32),
        # a decoder's forced tokens over the states of an encoder, padded batch
        _cross("cross prompt", 16, 448, 1500, 16, 16, 64, dtype="f16"),
        # the same decoder's next token
        _cross("cross one token", 32, 1, 1500, 20, 20, 64, ragged=False),
        # a small batch, odd everywhere
        _cross("cross ragged", 5, 77, 333, 10, 5, 80),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same ranges, no dearer than the largest listed ones."""
    while True:
        c = _draw(rng)
        w = work(c)
        if w["flops"] <= 5.4e11 and w["bytes"] <= 2.8e9 and _scores(c) <= 2.1e9:
            c.pop("name")
            return c


def _draw(rng):
    op = rng.choice(["rope", "append", "attend", "attend", "attend", "cross", "cross"])
    dtype = rng.choice(["bf16", "bf16", "f16"])
    scaling = rng.choice(["none", "linear", "base", "ramp"])
    d = rng.choice([64, 80, 96, 128, 128])
    kv = rng.choice([1, 2, 4, 5, 8])
    heads = kv * rng.choice([1, 2, 4, 5, 8])
    if op == "rope":
        return _rope("", _log(rng, 1, 20011), heads, d, rng.choice([d, d, d // 2]), dtype=dtype,
                     interleaved=rng.random() < 0.5, scaling=scaling, far=rng.choice([0, 0, 100000, 1000000]),
                     pad=rng.choice([0, 0, 2 * d, 40]))
    mix = rng.randint(1, 1 << 20)
    page = rng.choice([16, 16, 24, 32, 64, 128])
    if op == "append":
        return _append("", _log(rng, 1, 64), rng.choice([1, _log(rng, 2, 4000)]), _log(rng, 1, 2000), heads, kv, d, page,
                       dtype=dtype, interleaved=rng.random() < 0.5, scaling=scaling, mix=mix)
    if op == "attend":
        return _attend("", _log(rng, 1, 200), rng.choice([1, 1, _log(rng, 2, 8192)]), _log(rng, 1, 24575), heads, kv, d, page,
                       dtype=dtype, window=rng.choice([0, 0, 0, 256, 1000]), even=rng.random() < 0.2, mix=mix)
    return _cross("", _log(rng, 1, 32), rng.choice([1, _log(rng, 2, 600)]), _log(rng, 16, 4000), heads, kv, d, dtype=dtype,
                  ragged=rng.random() < 0.7, mix=mix)


def _counts(c):
    """New tokens and lengths (with the new tokens) of each sequence: from 1 and 0 cached to the case's, one at the most."""
    rng = random.Random(c["mix"])
    even = c.get("even", False)
    new = [c["new"] if even else rng.choice([1, rng.randint(1, c["new"])]) for _ in range(c["seqs"])]
    cached = [c["cached"] if even else rng.randint(0, c["cached"]) for _ in range(c["seqs"])]
    new[-1], cached[-1] = c["new"], c["cached"]
    return new, [a + b for a, b in zip(new, cached)]


def _sources(c):
    """Keys of each row of a batch for cross attention: none to all."""
    rng = random.Random(c["mix"])
    return [rng.randint(0, c["src"]) if c["ragged"] and i else c["src"] for i in range(c["b"])]


def _scores(c):
    """Scores of the plain form, which pads the sequences."""
    if c["op"] == "cross":
        return c["b"] * c["heads"] * c["n"] * c["src"]
    if c["op"] == "attend":
        return c["seqs"] * c["heads"] * c["new"] * (c["new"] + c["cached"])
    return 0


def work(c):
    """Bytes and operations one pass cannot do without: inputs read once, outputs written once."""
    if c["op"] == "rope":
        n = c["t"] * c["heads"] * c["d"]
        return {"bytes": 4 * n + 8 * c["t"], "flops": 3.0 * c["t"] * c["heads"] * c["rotary"]}
    if c["op"] == "append":
        t = sum(_counts(c)[0])
        return {"bytes": 4.0 * t * (c["heads"] + 2 * c["kv"]) * c["d"] + 8 * t, "flops": 3.0 * t * (c["heads"] + c["kv"]) * c["d"]}
    if c["op"] == "cross":
        keys = _sources(c)
        return {"bytes": 4.0 * sum(keys) * c["kv"] * c["d"] + 4.0 * c["b"] * c["n"] * c["heads"] * c["d"],
                "flops": 4.0 * c["heads"] * c["d"] * c["n"] * sum(keys)}
    pairs = keys = 0
    for n, length in zip(*_counts(c)):
        w = c["window"] or length
        first = max(0, length - n + 1 - w)  # the oldest key that a new token sees
        keys += length - first
        full = max(0, min(n, length - w))  # new tokens that see a whole window
        rest = n - full  # ... and those that see all before them, the first of them length - n + 1 keys
        pairs += full * w + rest * (length - n) + rest * (rest + 1) // 2
    t = sum(_counts(c)[0])
    return {"bytes": 4.0 * keys * c["kv"] * c["d"] + 4.0 * t * c["heads"] * c["d"] + 4 * keys / c["page"],
            "flops": 4.0 * c["heads"] * c["d"] * pairs}


# ---------------------------------------------------------------- inputs

BASE, FACTOR, CONTEXT, LOW, HIGH = 10000.0, 8.0, 8192, 1.0, 32.0


def _frequencies(dim, scaling):
    """Radians a position of each pair, in 64 bits."""
    base = BASE * FACTOR ** (dim / (dim - 2)) if scaling == "base" else BASE
    f = base ** (-torch.arange(0, dim, 2, dtype=torch.float64, device="cuda") / dim)
    if scaling == "linear":
        f = f / FACTOR
    if scaling == "ramp":
        keep = ((CONTEXT * f / (2 * math.pi) - LOW) / (HIGH - LOW)).clamp(0, 1)
        f = f * (keep + (1 - keep) / FACTOR)
    return f


def _amplitude(scaling):
    return 0.1 * math.log(FACTOR) + 1 if scaling == "ramp" else 1.0


def prepare(case, seed):
    c, dev = case, torch.device("cuda")
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    s = {"case": c}

    def normal(*shape, mul=1.0):
        return (torch.randn(shape, generator=g, device=dev) * mul).to(DTYPES[c["dtype"]])

    d, heads = c["d"], c["heads"]
    if c["op"] == "rope":
        s["x"] = normal(c["t"], heads * d + c["pad"])[:, :heads * d].unflatten(1, (heads, d))
        s["positions"] = torch.arange(c["t"], device=dev)
        if c["far"]:
            s["positions"] = torch.randint(0, c["far"], (c["t"],), generator=g, device=dev)
    elif c["op"] == "cross":
        kv = c["kv"]
        s["q"] = normal(c["b"], c["n"], heads, d, mul=2.0)
        both = normal(c["b"], c["src"], 2 * kv * d).unflatten(2, (2, kv, d))  # keys and values of one projection
        s["k"], s["v"] = both[:, :, 0], both[:, :, 1]
        s["lengths"] = torch.tensor(_sources(c), dtype=torch.int32, device=dev) if c["ragged"] else None
    else:
        kv, page = c["kv"], c["page"]
        new, lengths = _counts(c)
        width = -(-(c["new"] + c["cached"]) // page)
        used = [-(-n // page) for n in lengths]
        pages = sum(used) + 3
        s["k_pages"], s["v_pages"] = normal(pages, kv, page, d), normal(pages, kv, page, d)
        ids = torch.randperm(pages, generator=g, device=dev).int()
        at = torch.tensor([0] + used, device=dev).cumsum(0)
        column = torch.arange(width, device=dev)
        live = column < torch.tensor(used, device=dev)[:, None]
        s["table"] = torch.where(live, ids[(at[:-1, None] + column).clamp_max(pages - 1)], -1).int()
        s["lengths"] = torch.tensor(lengths, dtype=torch.int32, device=dev)
        t = sum(new)
        s["offsets"] = torch.tensor([0] + new, device=dev).cumsum(0).int() if t != c["seqs"] else None
        s["most"] = max(new)
        projected = normal(t, (heads + 2 * kv) * d)  # queries, keys and values of one projection
        if c["op"] == "attend":
            projected *= 2
        s["q"] = projected[:, :heads * d].unflatten(1, (heads, d))
        s["k"] = projected[:, heads * d:(heads + kv) * d].unflatten(1, (kv, d))
        s["v"] = projected[:, (heads + kv) * d:].unflatten(1, (kv, d))
    if c["op"] in ("rope", "append"):
        s["frequencies"] = _frequencies(c["rotary"] if c["op"] == "rope" else d, c["scaling"])
    if own:
        from paper_1908_11263_gb300 import qnn
        s["qnn"] = qnn
        if c["op"] in ("rope", "append"):
            s["rotary"] = qnn.Rotary(c["rotary"] if c["op"] == "rope" else d, base=BASE, interleaved=c["interleaved"],
                                     scaling=c["scaling"], factor=FACTOR, context=CONTEXT, low=LOW, high=HIGH,
                                     amplitude=_amplitude(c["scaling"]))
        if c["op"] in ("append", "attend"):
            s["cache"] = qnn.PagedCache(s["k_pages"], s["v_pages"])
    return s


# ---------------------------------------------------------------- one pass

def run(state):
    c = state["case"]
    if own:
        return _RUN_OWN[c["op"]](state, c, state["qnn"])
    return _RUN_PLAIN[c["op"]](state, c)


def _own_rope(s, c, qnn):
    return qnn.rope(s["x"], s["positions"], s["rotary"])


def _own_append(s, c, qnn):
    q = s["cache"].append(s["k"], s["v"], s["table"], s["lengths"], s["offsets"], rotary=s["rotary"], q=s["q"])
    return q, s["k_pages"], s["v_pages"]


def _own_attend(s, c, qnn):
    return s["cache"].attend(s["q"], s["table"], s["lengths"], s["offsets"], window=c["window"] or None)


def _own_cross(s, c, qnn):
    return qnn.cross_attention(s["q"], s["k"], s["v"], s["lengths"])


_RUN_OWN = {"rope": _own_rope, "append": _own_append, "attend": _own_attend, "cross": _own_cross}


def _rotated(x, positions, frequencies, interleaved, amplitude):
    angle = positions.double()[:, None] * frequencies
    cos, sin = (amplitude * torch.cos(angle)).float()[:, None], (amplitude * torch.sin(angle)).float()[:, None]
    half = frequencies.numel()
    v, rest = x.float()[..., :2 * half], x.float()[..., 2 * half:]
    a, b = (v[..., 0::2], v[..., 1::2]) if interleaved else (v[..., :half], v[..., half:])
    a, b = a * cos - b * sin, a * sin + b * cos
    v = torch.stack([a, b], -1).flatten(-2) if interleaved else torch.cat([a, b], -1)
    return torch.cat([v, rest], -1).to(x.dtype)


def _plain_rope(s, c):
    return _rotated(s["x"], s["positions"], s["frequencies"], c["interleaved"], _amplitude(c["scaling"]))


def _places(s, c, tokens):
    """Sequence and position of each new token."""
    token = torch.arange(tokens, device="cuda")
    if s["offsets"] is None:
        return token, s["lengths"].long() - 1
    sequence = torch.searchsorted(s["offsets"], token, right=True) - 1
    return sequence, s["lengths"][sequence].long() - s["offsets"][sequence + 1].long() + token


def _plain_append(s, c):
    sequence, position = _places(s, c, s["q"].shape[0])
    q, k = (_rotated(x, position, s["frequencies"], c["interleaved"], _amplitude(c["scaling"])) for x in (s["q"], s["k"]))
    page, row = s["table"][sequence, position // c["page"]].long(), position % c["page"]
    s["k_pages"][page, :, row] = k
    s["v_pages"][page, :, row] = s["v"]
    return q, s["k_pages"], s["v_pages"]


def _softmax_sum(scores, allowed, v):
    """sum_j softmax_j(scores) v_j over the allowed j; zero where there is none."""
    scores = scores.masked_fill(~allowed, -math.inf)
    top = scores.amax(-1, keepdim=True)
    p = torch.exp(scores - top.masked_fill(top == -math.inf, 0.0))
    total = p.sum(-1, keepdim=True)
    return (p @ v) / total.masked_fill(total == 0, 1.0)


def _plain_attend(s, c):
    q, most, group, seqs = s["q"].float(), s["most"], c["heads"] // c["kv"], c["seqs"]
    sequence, position = _places(s, c, q.shape[0])
    first = sequence * 0 if s["offsets"] is None else s["offsets"][sequence].long()
    slot = sequence * most + (torch.arange(q.shape[0], device=q.device) - first if s["offsets"] is not None else 0)
    # queries padded to the longest sequence's: [seqs, kv, group * most, d]
    padded = q.new_zeros(seqs * most, c["heads"], c["d"])
    padded[slot] = q
    padded = padded.view(seqs, most, c["kv"], group, c["d"]).permute(0, 2, 3, 1, 4).flatten(2, 3)
    last = torch.full((seqs * most,), -1, device=q.device)
    last[slot] = position
    last = last.view(seqs, 1, 1, most, 1).expand(-1, -1, group, -1, -1).flatten(2, 3)
    table = s["table"].clamp_min(0).long()
    k, v = (s[n][table].transpose(1, 2).flatten(2, 3).float() for n in ("k_pages", "v_pages"))
    j = torch.arange(k.shape[2], device=q.device)
    allowed = j <= last
    if c["window"]:
        allowed = allowed & (j > last - c["window"])
    o = _softmax_sum(padded @ k.transpose(2, 3) / math.sqrt(c["d"]), allowed, v)
    o = o.view(seqs, c["kv"], group, most, c["d"]).permute(0, 3, 1, 2, 4).reshape(seqs * most, c["heads"], c["d"])
    return o[slot].to(s["q"].dtype)


def _plain_cross(s, c):
    group = c["heads"] // c["kv"]
    q = s["q"].float().unflatten(2, (c["kv"], group)).permute(0, 2, 3, 1, 4).flatten(2, 3)
    k, v = s["k"].float().transpose(1, 2), s["v"].float().transpose(1, 2)
    allowed = torch.arange(c["src"], device=q.device).expand(c["b"], 1, 1, -1)
    allowed = allowed < (c["src"] if s["lengths"] is None else s["lengths"].view(-1, 1, 1, 1))
    o = _softmax_sum(q @ k.transpose(2, 3) / math.sqrt(c["d"]), allowed, v)
    o = o.view(c["b"], c["kv"], group, c["n"], c["d"]).permute(0, 3, 1, 2, 4)
    return o.reshape(s["q"].shape).to(s["q"].dtype)


_RUN_PLAIN = {"rope": _plain_rope, "append": _plain_append, "attend": _plain_attend, "cross": _plain_cross}


# ---------------------------------------------------------------- 64 bits, from the definitions

def exact(case, seed):
    global own
    was, own = own, False
    s = prepare(case, seed)
    own = was
    return {"rope": _exact_rope, "append": _exact_append, "attend": _exact_attend, "cross": _exact_cross}[case["op"]](s, case)


def _turned(x, positions, frequencies, interleaved, scaling):
    """The pairs as complex numbers, turned."""
    x, half = x.double(), frequencies.numel()
    a = x[..., :2 * half]
    z = torch.complex(a[..., ::2].contiguous(), a[..., 1::2].contiguous()) if interleaved else \
        torch.complex(a[..., :half].contiguous(), a[..., half:].contiguous())
    turn = torch.polar(torch.full_like(frequencies, _amplitude(scaling)).expand(x.shape[0], -1), torch.outer(positions.double(), frequencies))
    z = torch.view_as_real(z * turn[:, None])
    y = x.clone()
    y[..., :2 * half] = z.flatten(-2) if interleaved else z.transpose(-1, -2).flatten(-2)
    return y


def _exact_rope(s, c):
    return _turned(s["x"], s["positions"], s["frequencies"], c["interleaved"], c["scaling"])


def _spans(c):
    at = 0
    for i, (n, length) in enumerate(zip(*_counts(c))):
        yield i, at, n, length
        at += n


def _exact_append(s, c):
    positions = torch.cat([torch.arange(length - n, length) for _, _, n, length in _spans(c)]).cuda()
    q, k = (_turned(s[x], positions, s["frequencies"], c["interleaved"], c["scaling"]) for x in "qk")
    pools = s["k_pages"].double(), s["v_pages"].double()
    for i, at, n, length in _spans(c):
        p = positions[at:at + n]
        page = s["table"][i, torch.div(p, c["page"], rounding_mode="floor")].long()
        for pool, x in zip(pools, (k, s["v"].double())):
            pool[page, :, torch.remainder(p, c["page"])] = x[at:at + n]
    return (q,) + pools


def _attention64(q, k, v, ahead, window):
    """q [n, heads, d] over k, v [keys, kv, d]; query i sees keys up to ahead + i (all where ahead is None)."""
    n, heads, d = q.shape
    out = torch.zeros(n, heads, d, dtype=torch.float64, device=q.device)
    if k.shape[0] == 0:
        return out
    group = heads // k.shape[1]
    for h in range(heads):
        kh, vh = k[:, h // group].double(), v[:, h // group].double()
        for lo in range(0, n, 2048):
            hi = min(n, lo + 2048)
            keys = k.shape[0] if ahead is None else min(k.shape[0], ahead + hi)
            z = torch.mm(q[lo:hi, h].double(), kh[:keys].T) * d ** -0.5
            if ahead is not None:
                back = (ahead + torch.arange(lo, hi, device=q.device))[:, None] - torch.arange(keys, device=q.device)
                z[back < 0] = -math.inf
                if window:
                    z[back >= window] = -math.inf
            out[lo:hi, h] = torch.softmax(z, 1) @ vh[:keys]
    return out


def _exact_attend(s, c):
    rows = []
    for i, at, n, length in _spans(c):
        pages = s["table"][i, :-(-length // c["page"])].long()
        k, v = (s[x][pages].permute(0, 2, 1, 3).flatten(0, 1)[:length] for x in ("k_pages", "v_pages"))
        rows.append(_attention64(s["q"][at:at + n], k, v, length - n, c["window"]))
    return torch.cat(rows)


def _exact_cross(s, c):
    return torch.stack([_attention64(s["q"][i], s["k"][i, :n], s["v"][i, :n], None, 0) for i, n in enumerate(_sources(c))])
