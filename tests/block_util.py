"""Plain 64-bit forms of the matrix products, with a bound on how far a 32-bit evaluation may be from them.

The bound: a product of two 16-bit values is exact in 32 bits; a sum of K of them in any order, each partial sum rounded
or truncated to 24 bits, is off by at most (terms + 32) * 2^-23 of the sum of magnitudes, where an MMA adds 16 columns
at a time (terms = K / 16).  Scale, bias, activation (slope below 1.13, 16 roundings of its own), gate and residual each
add their own roundings; the result is rounded once to its type (unit roundoff U)."""
import math

import torch

U = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}
E = 2.0 ** -23


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def weights(rows, k, bits, dtype, g, experts=None):
    """(packed or 16-bit weights, scale or None, weights in 64 bits without the scale)."""
    shape = ((experts,) if experts else ()) + (rows, k)
    if bits == 16:
        w = (torch.randn(shape, generator=g, device="cuda") / math.sqrt(k)).to(dtype)
        return w, None, w.double()
    lo = -(1 << (bits - 1))
    codes = torch.randint(lo, -lo, shape, generator=g, device="cuda", dtype=torch.int32)
    scale = (0.5 + torch.rand(shape[:-1], generator=g, device="cuda")) / (2.0 ** (bits - 2) * math.sqrt(k))
    return pack(codes, bits), scale, codes.double()


def pack(codes, bits):
    """Packed bytes of signed codes: element e in byte e // (8 // bits), the first in the low bits."""
    per = 8 // bits
    u = (codes.to(torch.int64) % (1 << bits)).unflatten(-1, (-1, per))
    shifts = torch.arange(per, device=codes.device) * bits
    return (u << shifts).sum(-1).to(torch.uint8)


def act64(v, act):
    if act == "relu":
        return v.clamp_min(0)
    if act == "silu":
        return v * torch.sigmoid(v)
    if act == "gelu":
        return v * 0.5 * (1 + torch.erf(v / math.sqrt(2)))
    if act == "gelu_tanh":
        return 0.5 * v * (1 + torch.tanh(math.sqrt(2 / math.pi) * (v + 0.044715 * v ** 3)))
    return v


def product64(x, w, scale, bias, m, gated, act):
    """(value, bound on the 32-bit error) of act(scale * x w^T + bias), gated or not."""
    x = x.double()
    s = 1.0 if scale is None else scale.double()
    b = 0.0 if bias is None else bias.double()
    v = x @ w.t() * s + b
    err = E * (x.shape[1] / 16 + 32) * (x.abs() @ w.abs().t() * s) + 2 * E * (v.abs() + abs(b))

    def activated(v, err):
        y = act64(v, act)
        return y, (err if act == "none" else 1.13 * err + 16 * E * (y.abs() + (v.abs() if act != "relu" else 0)))

    if not gated:
        return activated(v, err)
    a, ea = activated(v[:, :m], err[:, :m])
    u, eu = v[:, m:], err[:, m:]
    return a * u, ea * u.abs() + a.abs() * eu + ea * eu + E * (a * u).abs()


def check(got, want, err, name=""):
    tol = U[got.dtype] * (want.abs() + err) + err + 2.0 ** -25
    d = (got.double() - want).abs()
    bad = ~(d <= tol)
    assert not bad.any(), f"{name}: {int(bad.sum())} of {d.numel()} off, worst {float((d / tol).nan_to_num(math.inf).max()):.2f} " \
                          f"of the tolerance at {tuple(int(i) for i in bad.nonzero()[0])}"


def strided(t, pad):
    """The same values in rows `pad` elements further apart, with NaN between them."""
    if not pad:
        return t
    buf = torch.full((t.shape[0], t.shape[1] + pad), math.nan, dtype=t.dtype, device=t.device)
    buf[:, :t.shape[1]] = t
    return buf[:, :t.shape[1]]
