"""Rotary(frequencies=...): what it keeps of frequencies of one's own, of either sign."""
import contextlib
import math
from fractions import Fraction

import pytest
import torch

from attention_util import check, gen, randn
from paper_1908_11263_gb300 import qnn

TAU = Fraction(2 * 31415926535897932384626433832795028841971693993751, 10 ** 49)  # 2 pi to 50 digits
OWN = [0.5, -0.25, 1e-6, -1e-6, -3.0, 700.25, -700.25, 1e-15, -1e-15, 2.0 ** -80, -2.0 ** -80, 0.0, -0.0, -2.0 * math.pi]


@pytest.fixture
def on_host(monkeypatch):
    """Rotations laid out in host memory."""
    monkeypatch.setattr(qnn, "_empty", lambda shape, dtype, device, stream: torch.empty(shape, dtype=dtype))
    monkeypatch.setattr(qnn, "_current_device", lambda: 0)
    monkeypatch.setattr(qnn, "_on_current", lambda device, name: None)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda: None)
    monkeypatch.setattr(torch.cuda, "stream", lambda s: contextlib.nullcontext())


def turns_of(rotary):
    return [v % (1 << 64) for v in rotary.turns.tolist()]


def test_negative_frequencies_are_the_others_turned_back(on_host):
    there = turns_of(qnn.Rotary(2 * len(OWN), frequencies=OWN))
    back = turns_of(qnn.Rotary(2 * len(OWN), frequencies=[-f for f in OWN]))
    assert [-t % (1 << 64) for t in there] == back


def test_fractions_of_either_sign(on_host):
    """The quotient f / 2 pi is rounded to 53 bits and 2 pi itself is, 2^-52 relative in all; the fraction is cut at 2^-64."""
    for f, t in zip(OWN, turns_of(qnn.Rotary(2 * len(OWN), frequencies=OWN))):
        want = Fraction(f) / TAU
        off = (Fraction(t, 1 << 64) - want) % 1
        assert min(off, 1 - off) <= abs(want) / (1 << 52) + Fraction(1, 1 << 64), f


@pytest.mark.gpu
@pytest.mark.parametrize("interleaved", [False, True])
def test_far_positions_with_negative_frequencies(interleaved):
    """Phases computed from the frequencies themselves, not from what the rotation keeps of them."""
    f = [-0.25, 0.25, -1e-6, 1e-6, -3.0, 3.0, -1e-4, 1.0]
    positions = [0, 1, -1, 10 ** 6, -(10 ** 6), 2 ** 31 - 1, 2 ** 40 + 12345, -(2 ** 40)]
    x = randn(gen(8), len(positions), 3, 24, dtype=torch.float32)
    rotary = qnn.Rotary(16, frequencies=f, interleaved=interleaved)
    got = qnn.rope(x, torch.tensor(positions, device="cuda"), rotary)
    phase = [[float(Fraction(p) * Fraction(v) / TAU % 1) for v in f] for p in positions]
    angle = 2 * math.pi * torch.tensor(phase, dtype=torch.float64, device="cuda")
    ia = torch.arange(8, device="cuda") * (2 if interleaved else 1)
    ib = ia + (1 if interleaved else 8)
    want, err = x.double(), torch.zeros(x.shape, dtype=torch.float64, device="cuda")
    a, b = want[..., ia], want[..., ib]
    cos, sin = torch.cos(angle)[:, None], torch.sin(angle)[:, None]
    want[..., ia], want[..., ib] = a * cos - b * sin, a * sin + b * cos
    # radians: the fraction's error (above) a position, and the 2^-21 of an evaluation in 32 bits
    lost = [[float(2 * math.pi * abs(p) * (abs(v) / math.tau * 2.0 ** -52 + 2.0 ** -64)) for v in f] for p in positions]
    size = (a.abs() + b.abs()) * (torch.tensor(lost, dtype=torch.float64, device="cuda")[:, None] + 2.0 ** -21)
    err[..., ia] = err[..., ib] = size
    check(got, want, err)
    back = qnn.rope(x, -torch.tensor(positions, device="cuda"), qnn.Rotary(16, frequencies=[-v for v in f], interleaved=interleaved))
    assert torch.equal(got, back)
