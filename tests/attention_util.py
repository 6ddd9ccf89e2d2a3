"""Plain 64-bit forms of the attention operators, with bounds on how far a 32-bit evaluation may be from them.

Rotation: a pair's phase is kept to 2^-32 of a turn and rounded to 24 bits (half a turn at most), sine and cosine are off by
two steps of 2^-24, their products with the amplitude and the pair by another: under 2^-21 (|a| + |b|) in all.

Attention: a score, a sum of D exact products in 32 bits in any order, is off by (D / 16 + 36) 2^-23 of the sum of magnitudes
(an MMA adds 16 at a time), its scaling included; z = scale q k then moves a weight 2^(z - max) by as much relatively, and
the sum of weights by the largest of these.  The maximum itself cancels.  A weight is off by 2^-21 more from 2^x and from the
factors that raise the maximum, and is rounded to the element type (U relative; float16 below 2^-14 of a row's largest
weight: 2^-25 of that weight) before it multiplies a value.  Sums over N keys in 32 bits: (N / 16 + 64) 2^-22.
With w the weights, normalised, that is  |error| <= sum_j w_j |v_j| (U + 2 Ez + 2^-20 + (N / 16 + 64) 2^-22) (+ 2^-25 sum |v_j| for
float16), and the result is rounded once."""
import math

import torch

U = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}
TINY = {torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25, torch.float32: 2.0 ** -150}  # half a step of the smallest numbers


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def randn(g, *shape, dtype=torch.bfloat16, mul=1.0):
    return (torch.randn(shape, generator=g, device="cuda") * mul).to(dtype)


def strided_heads(g, t, heads, d, dtype, pad, mul=1.0):
    """[t, heads, d] as a part of wider rows that hold NaN elsewhere."""
    buf = torch.full((t, heads * d + pad), math.nan, dtype=dtype, device="cuda")
    x = buf[:, pad // 2:pad // 2 + heads * d].unflatten(1, (heads, d))
    x.copy_(randn(g, t, heads, d, dtype=dtype, mul=mul))
    return x


# ---------------------------------------------------------------- rotation

def frequencies(dim, base=10000.0, scaling="none", factor=1.0, context=0, low=1.0, high=32.0):
    """Radians a position, from the formulas, as Python floats."""
    out = []
    if scaling == "base":
        base = base * factor ** (dim / (dim - 2))
    for i in range(dim // 2):
        f = base ** (-2.0 * i / dim)
        if scaling == "linear":
            f /= factor
        if scaling == "ramp":
            g = min(1.0, max(0.0, (context * f / (2 * math.pi) - low) / (high - low)))
            f *= g + (1 - g) / factor
        out.append(f)
    return out


def rotate64(x, positions, turns, interleaved, amplitude):
    """(rotated, bound on the 32-bit error); positions and turns (64-bit fractions) as Python integers."""
    half = len(turns)
    phase = torch.tensor([[(p * f) % (1 << 64) / 2.0 ** 64 for f in turns] for p in positions], dtype=torch.float64,
                         device=x.device).reshape(len(positions), half)
    cos, sin = (amplitude * t[:, None] for t in (torch.cos(2 * math.pi * phase), torch.sin(2 * math.pi * phase)))
    x = x.double()
    y, err = x.clone(), torch.zeros_like(x)
    if half:
        ia = torch.arange(half, device=x.device) * (2 if interleaved else 1)
        ib = ia + (1 if interleaved else half)
        a, b = x[..., ia], x[..., ib]
        y[..., ia], y[..., ib] = a * cos - b * sin, a * sin + b * cos
        err[..., ia] = err[..., ib] = (a.abs() + b.abs()) * abs(amplitude) * 2.0 ** -21
    return y, err


def check(got, want, err, name=""):
    tol = U[got.dtype] * (want.abs() + err) + err + TINY[got.dtype]
    d = (got.double() - want).abs()
    bad = ~(d <= tol)
    assert not bad.any(), f"{name}: {int(bad.sum())} of {d.numel()} off, worst {float((d / tol).nan_to_num(math.inf).max()):.2f} " \
                          f"of the tolerance at {tuple(int(i) for i in bad.nonzero()[0])}"


# ---------------------------------------------------------------- attention

def attention64(q, k, v, seen, scale):
    """q [n, heads, d], k, v [keys, kv, d] as they are stored, seen [n, keys]: (out, bound, lse, bound on lse); rows that see
    nothing are zero with lse -inf."""
    n, heads, d = q.shape
    keys, kv = k.shape[0], k.shape[1]
    u = U[q.dtype]
    out = torch.zeros(n, heads, d, dtype=torch.float64, device=q.device)
    err, lse = torch.zeros_like(out), torch.full((n, heads), -math.inf, dtype=torch.float64, device=q.device)
    lse_err = torch.zeros_like(lse)
    if keys == 0 or n == 0:
        return out, err, lse, lse_err
    some = seen.any(1)
    for h in range(heads):
        qh, kh, vh = q[:, h].double(), k[:, h // (heads // kv)].double(), v[:, h // (heads // kv)].double()
        z = (qh @ kh.T * scale).masked_fill(~seen, -math.inf)
        size = (qh.abs() @ kh.abs().T * scale).masked_fill(~seen, 0.0)
        ez = (d / 16 + 36) * 2.0 ** -23 * size.amax(1)
        w = torch.softmax(z.masked_fill(~some[:, None], 0.0), 1).masked_fill(~some[:, None], 0.0)
        rel = u + 2 * ez + 2.0 ** -20 + (keys / 16 + 64) * 2.0 ** -22
        out[:, h] = w @ vh
        err[:, h] = w @ vh.abs() * rel[:, None]
        if q.dtype is torch.float16:
            err[:, h] += 2.0 ** -25 * (seen.double() @ vh.abs())
        lse[:, h] = torch.logsumexp(z, 1)
        lse_err[:, h] = ez + 2.0 ** -20 + (keys / 16 + 64) * 2.0 ** -22 + 2.0 ** -22 * lse[:, h].abs().nan_to_num(0.0, 0.0, 0.0)
    return out, err, lse, lse_err


def check_lse(got, want, err, name=""):
    bad = ~((got.double() - want).abs() <= err + 2.0 ** -23 * want.abs()) & (got.double() != want)
    assert not bad.any(), f"{name}: lse {int(bad.sum())} off, first at {bad.nonzero()[0].tolist()}"


def check_cache_attention(got, lse, q, k_pages, v_pages, table, lengths, offsets, *, causal=True, window=None, scale=None, name="",
                          skip=()):
    """Compares attend()'s outputs for every sequence not in `skip`; arguments as the call's, pages as [pages, heads, rows, d]."""
    tokens, heads, d = q.shape
    scale = 1 / math.sqrt(d) if scale is None else scale
    pages, page = k_pages.shape[0], k_pages.shape[2]
    seqs, width = table.shape
    starts = offsets.tolist() if offsets is not None else [i * (tokens // seqs) for i in range(seqs + 1)]
    for s, length in enumerate(lengths.tolist()):
        lo, hi = starts[s], starts[s + 1]
        if s in skip or hi <= lo:
            continue
        room = max(0, min(length, width * page))
        row = table[s].long()
        there = (row >= 0) & (row < pages)
        safe = torch.where(there, row, 0)[:-(-room // page)]
        kk, vv = (t[safe].permute(0, 2, 1, 3).reshape(-1, t.shape[1], d)[:room] for t in (k_pages, v_pages))
        j = torch.arange(room, device=q.device)
        p = length - (hi - lo) + torch.arange(hi - lo, device=q.device)[:, None]
        seen = there[j // page].expand(hi - lo, -1)
        if causal:
            seen = seen & (j <= p)
        if window:
            seen = seen & (j > p - window)
        any_row = seen.any(0)  # what nobody sees may be NaN
        kk, vv = (torch.where(any_row[:, None, None], t, 0) for t in (kk, vv))
        want, err, wl, le = attention64(q[lo:hi], kk, vv, seen, scale)
        check(got[lo:hi], want, err, f"{name} sequence {s}")
        if lse is not None:
            check_lse(lse[lo:hi], wl, le, f"{name} sequence {s}")
