"""Angles of far positions: the table's steps against frequencies in 50 digits, and rotated rows up to position 2^38."""
import math
from decimal import Decimal, localcontext

import pytest
import torch

import _paged as P
from paper_2606_26344_b200 import build as B
from paper_2606_26344_b200 import gmlp

TURN = 2 * Decimal("3.14159265358979323846264338327950288419716939937510582097494459")
KINDS = [None, ("linear", 4.0), ("bands", 8.0, 1.0, 4.0, 8192), ("ramp", 16.0, 32.0, 1.0, 4096)]


def turns_per_position(rot, base, scaling):
    """[rot / 2] Decimals, from the documented formulas."""
    with localcontext() as c:
        c.prec = 50
        f = [(Decimal(base).ln() * -2 * i / rot).exp() / TURN for i in range(rot // 2)]
        if scaling is None:
            return f
        factor, rest = Decimal(scaling[1]), [Decimal(x) for x in scaling[2:]]
        if scaling[0] == "linear":
            keep = [Decimal(0)] * len(f)
        elif scaling[0] == "bands":
            low, high, original = rest
            keep = [(original * v - low) / (high - low) for v in f]
        else:
            high, low, original = rest
            at = lambda n: rot * (original / (n * TURN)).ln() / (2 * Decimal(base).ln())
            a, b = max(math.floor(at(high)), 0), min(math.ceil(at(low)), rot - 1)
            keep = [1 - Decimal(i - a) / max(Decimal(b - a), Decimal("0.001")) for i in range(len(f))]
        keep = [min(Decimal(1), max(Decimal(0), w)) for w in keep]
        return [v * w + v / factor * (1 - w) for v, w in zip(f, keep)]


@pytest.mark.parametrize("rot,base", [(4, 1e4), (20, 1e4), (64, 1e4), (128, 5e5), (256, 1e6), (1024, 1e9)])
@pytest.mark.parametrize("scaling", KINDS)
def test_steps_are_good_to_their_last_place(rot, base, scaling):
    """Half a unit of 2^-64 for the rounding; in 80 bits (2^-64 of a value for each rounding) some ten roundings of values of a sixth of a turn or
    less and the exponent's, e^-y y <= 0.37 of it: another unit at most."""
    B.build_libgmlp()
    steps, _ = gmlp.rope_steps(rot, base, scaling)
    for s, v in zip(steps, turns_per_position(rot, base, scaling)):
        assert abs(Decimal(s) - v * 2 ** 64) <= Decimal("1.5")


@pytest.mark.gpu
@pytest.mark.parametrize("scaling", KINDS)
@pytest.mark.parametrize("inter", [False, True])
def test_rows_at_far_positions(scaling, inter):
    """An entry 1.5 units of 2^-64 off makes position p's angle p * 1.5 * 2^-64 turns wrong: at 2^38 less than 2^-22 radians, about what the
    rotation's fp32 arithmetic takes anyway."""
    dev, rot, base = torch.device("cuda"), 128, 5e5
    rope = gmlp.Rope(rot, base=base, interleaved=inter, scaling=scaling)
    at = [0, 1, 131072, (1 << 31) + 7, -(1 << 31) - 7, (1 << 36) + 12345, 1 << 38, -(1 << 38) + 1]
    x = torch.randn(len(at), 2 * 128, generator=torch.Generator(device=dev).manual_seed(1), device=dev).to(torch.bfloat16)
    y = gmlp.rope_apply(x, torch.tensor(at, device=dev), rope, 2, checked=True).view(-1, 2, 128)
    f = turns_per_position(rot, base, scaling)
    for i, p in enumerate(at):
        with localcontext() as c:
            c.prec = 50
            angles = [float((p * v) % 1 * TURN) for v in f]
        row = x[i:i + 1].view(1, 2, 128)
        want = P.rotate(row, torch.ones(1, dtype=torch.int64, device=dev), angles, rope.amplitude, rot, inter)
        j = torch.arange(rot // 2, device=dev)
        a, b = (2 * j, 2 * j + 1) if inter else (j, j + rot // 2)
        size = torch.zeros_like(want)
        size[..., a] = size[..., b] = row.double()[..., a].abs() + row.double()[..., b].abs()
        bound = P.rotate_bound(row, want, rope.amplitude, rot, inter) + abs(p) * 1.5 * 2.0 ** -64 * 2 * math.pi * abs(rope.amplitude) * size
        assert bool(((y[i:i + 1].double() - want).abs() <= bound).all()), p
