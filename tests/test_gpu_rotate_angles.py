"""Angles of rotate_heads over the whole range of frequencies and positions, against whole-number arithmetic (needs a GB300).

Heads of pairs (1, 0) turn to (cos t, sin t) exactly, but for the output's rounding.  Tolerance, before any run: that rounding (u = 2^-8 of
bf16, relative), sine and cosine of the rest of at most pi / 4 as the library gives them (2 units of their last place: 2^-22
relative) with the rest rounded to fp32 (2^-24 relative; of a sine relative to itself, of a cosine at most 2^-24), and the fraction of a
turn off by |pos| 2^-64: 2 pi 2^-33 = 7.4e-10 at most.  In all (2^-8 + 2^-21) |y| + 8e-10.
"""
import math
import random
from fractions import Fraction

import pytest

from test_gpu_rotate import sv  # noqa: F401

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
PI = Fraction(314159265358979323846264338327950288419716939937510582097494459230781640628620899862803483, 10 ** 89)


def turned(freq, pos):
    """(cos, sin) of pos freq: the fraction of a turn in whole numbers, the nearest quarter off, the rest (small numbers keep their digits) in 64 bits."""
    turns = pos * Fraction(freq) / (2 * PI)
    quarter = math.floor(4 * turns + Fraction(1, 2))
    t = float((turns - Fraction(quarter, 4)) * 2 * PI)
    c, s = math.cos(t), math.sin(t)
    return [(c, s), (-s, c), (-c, -s), (s, -c)][quarter % 4]


def nearest_positions(freq, most):
    """Positions up to `most` whose angle is next to a quarter turn's multiple: the denominators of the continued fraction of 4 turns."""
    x = 4 * Fraction(freq) / (2 * PI) % 1
    found, p, q = [], 0, 1
    for _ in range(60):
        if x == 0:
            break
        a = int(1 / x)
        x = 1 / x - a
        p, q = q, p + a * q
        if q > most:
            break
        found.append(q)
    return found


def check(sv, freqs, positions, neighbours):  # noqa: F811
    n = len(freqs)
    head = torch.zeros(len(positions), 1, 2 * n, device="cuda", dtype=torch.bfloat16)
    a, b = (slice(0, None, 2), slice(1, None, 2)) if neighbours else (slice(0, n), slice(n, None))
    head[..., a] = 1
    pos = torch.tensor(positions, dtype=torch.int32, device="cuda")
    got = sv.rotate_heads(head, head.clone(), pos, torch.tensor(freqs, dtype=torch.float64, device="cuda"), neighbours=neighbours)
    assert torch.equal(got[0], got[1])
    want = torch.tensor([[turned(f, p) for f in freqs] for p in positions], dtype=torch.float64, device="cuda")
    for y, w in ((got[0][:, 0, a], want[..., 0]), (got[0][:, 0, b], want[..., 1])):
        err = (y.double() - w).abs()
        bound = (2.0 ** -8 + 2.0 ** -21) * w.abs() + 8e-10
        worst = (err / bound).max().item()
        assert (err <= bound).all(), (worst, freqs[int((err / bound).amax(0).argmax())])


@pytest.mark.parametrize("neighbours", [False, True])
@pytest.mark.parametrize("hd", [64, 128])
def test_far_positions_of_any_frequency(sv, hd, neighbours):  # noqa: F811
    """Angles next to a multiple of a quarter turn, where a sine (or cosine) shows the angle to its last bits."""
    rng = random.Random(hd)
    ends = [5e-324, 2.0 ** -1022, 1e-300, 2.0 ** -64, 1.0, 2 * math.pi, 1e4, 1e6, 1e8, 4e9, math.nextafter(2.0 ** 32, 0), 2.0 ** 31]
    freqs = (ends + [2.0 ** rng.uniform(-40, 32) for _ in range(64)])[: hd // 2]
    freqs = [f if i % 3 else -f for i, f in enumerate(freqs)]
    positions = [0, 1, -1, 2 ** 31 - 1, -2 ** 31, 1000003]
    for f in freqs:
        near = nearest_positions(abs(f), 2 ** 31 - 1)[-3:]
        positions += near + [-x for x in near[-1:]]
    check(sv, freqs, positions, neighbours)


def test_gradient_turns_back(sv):  # noqa: F811
    """The gradient's angles are the same: there and back is the head, within two roundings."""
    freqs = torch.tensor([2.0 ** (i - 32) for i in range(64)], dtype=torch.float64, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(1)
    q = torch.randn(40, 2, 128, generator=g, device="cuda").half()
    pos = torch.randint(-2 ** 31, 2 ** 31, (40,), generator=g, device="cuda", dtype=torch.int64).int()
    there = sv.rotate_heads(q, q, pos, freqs)[0]
    back = sv.rotate_heads_grad(there, there, q, q, pos, freqs)["q"]
    size = q.double()[..., :64].abs() + q.double()[..., 64:].abs()
    # 2^-11 of each rounded element there, which the turn back adds in pairs, and 2^-11 of the result
    assert ((back.double() - q.double()).abs() <= 4 * 2.0 ** -11 * torch.cat([size, size], -1)).all()
