"""The intermediate of the microscaled 4-bit experts is silu(a) u to 32 bits, over the sigmoid's whole range and in every shape's epilogue.

One feature in a block: what comes back is silu(a) u to 2 bits, and those say on which side of a border the kernel's number was: 1.25 and 2 times a power of
two (between codes 4 and 6, and between 6 and the next power's 4).  a stands on both sides of the border, as near as fp32 numbers and 16 steps of 2^-24 of
silu(a) allow: silu_times is off by 8.5 at most.  Every digit of a is a block of its own with one number, so a is exact, and so is u, a power of
two in another block.
"""
import math

import numpy as np
import pytest
import torch

from oracle import mx4_oracle as Q
from paper_2603_19172_amd import binding as B
from paper_2603_19172_amd.layer import Mx4Experts
from gpu_helpers import DEV
from test_mx4_rule import experts, rule  # noqa: F401  (fixtures)

DIGITS, STEP = 24, 2.0 ** -24
H = 32 * (DIGITS + 1)


def silu(a):
    return a / (1.0 + np.exp(-a))


def root(lo, hi, y):
    """silu's argument for y on a piece where it only rises or only falls."""
    up = silu(hi) > silu(lo)
    for _ in range(200):
        mid = (lo + hi) / 2
        if (silu(mid) < y) == up:
            lo = mid
        else:
            hi = mid
    return (lo + hi) / 2


def arguments():
    """fp32 numbers on both sides of every border."""
    least = -1.2784645427610738                                   # where silu turns
    pieces = [(-87.2, least, -1, range(-119, -1)), (least, -2.0 ** -24, -1, range(-22, -1)), (2.0 ** -24, 100.0, 1, range(-22, 7))]
    out = []
    for lo, hi, sign, powers in pieces:
        for m in powers:
            for c in (1.0, 1.25):
                y = sign * c * 2.0 ** m
                if not min(silu(lo), silu(hi)) < y < max(silu(lo), silu(hi)):
                    continue
                a = root(lo, hi, y)
                for way in (-math.inf, math.inf):
                    v = np.float32(a)
                    while abs(silu(np.float64(v)) / y - 1) < 16 * STEP or (v > a) != (way > 0):
                        v = np.nextafter(v, np.float32(way))
                    out.append(float(v))
    return np.array(out)


def rows():
    """x [n, H], the values silu(a) u converted [n]."""
    a = arguments()
    # (a power of two that brings the product back from 2^-120, and others for the rest)
    u = np.where(a < -40, 2.0 ** 70, 2.0 ** (np.arange(len(a)) % 13 - 6.0))
    # the ends: 0 below -87.34, where e^-a passes 2^126, and a itself from 18 on
    far = np.array([-87.4, -88.0, -100.0, -127.5, -129.0, -1000.0, -2.0 ** 100, 87.5, 90.0, 127.0, 128.5, 1000.0, 2.0 ** 100])
    a = np.concatenate([a, far.astype(np.float32).astype(np.float64)])
    u = np.concatenate([u, np.ones(len(far))])
    with np.errstate(over="ignore"):
        h = np.where(a < -87.34, 0.0, silu(a)) * u
    block = np.zeros((len(a), 32))
    block[:, 0] = h
    want = Q.values(*Q.quantize(block))[:, 0]
    x = np.zeros((len(a), H))
    for i, v in enumerate(a):
        m, e = math.frexp(v)
        whole = int(abs(m) * (1 << DIGITS))
        for b in range(DIGITS):
            x[i, 32 * b] = math.copysign(math.ldexp((whole >> b) & 1, b - DIGITS + e), v)
        assert x[i].sum() == v
    x[:, 32 * DIGITS] = u
    return torch.from_numpy(x).float(), want


def one_expert(F):
    """Feature 32 j is silu(a) u, output j its converted value."""
    w1, w3, w2 = torch.zeros((F, H)), torch.zeros((F, H)), torch.zeros((H, F))
    w1[::32, 0:32 * DIGITS:32] = 1.0
    w3[::32, 32 * DIGITS] = 1.0
    w2[torch.arange(F // 32), 32 * torch.arange(F // 32)] = 1.0
    return [w1, w3, w2]


# name, rows at once, F, E, waves of the up projection
SHAPES = [("thin", 2, 64, 8, 0), ("thin", 32, 32, 128, 0), ("small", 700, 32, 128, 4), ("small", 700, 256, 128, 2), ("small", 700, 480, 128, 1),
          ("tall", 700, 32, 1, 0), ("tall", 700, 320, 1, 0)]


def test_the_rows_say_something(experts):  # noqa: F811
    x, want = rows()
    a = x[:, :32 * DIGITS].double().sum(1).numpy()
    assert len(a) > 500 and (want != 0).mean() > 0.95 and a[want != 0].min() < -86.9 and len(set(want.tolist())) > 100
    # an error of 200 steps of 2^-24 would show in nine rows of ten, up or down
    moved = 0
    for d in (1 + 200 * STEP, 1 - 200 * STEP):
        block = np.zeros((len(a), 32))
        block[:, 0] = silu(np.clip(a, -87.34, 1e30)) * x[:, 32 * DIGITS].double().numpy() * d
        moved += (Q.values(*Q.quantize(block))[:, 0] != want)[:-13].mean()
    assert moved > 0.9
    for name, T, F, E, up in SHAPES:
        assert experts(min(T, len(a)), H, F, E, 1)[:2] == (name, up), (name, T, F, E)


@pytest.mark.gpu
@pytest.mark.parametrize("name,T,F,E,up", SHAPES)
def test_intermediate_is_silu_to_32_bits(name, T, F, E, up):
    ctx = B.Context(0)
    x, want = rows()
    ex = Mx4Experts(ctx, [[t.to(DEV) for t in one_expert(F)]] + [None] * (E - 1), DEV)
    T = min(T, len(x))
    for i in range(0, len(x), T):
        part = x[max(0, min(i, len(x) - T)):][:T].to(DEV)
        y = ctx.moe_ffn_mx4(part, torch.zeros((T, 1), dtype=torch.int32, device=DEV), torch.ones((T, 1), device=DEV), ex.table, F, out_dtype=B.OUT_F32)
        ref = torch.from_numpy(want[max(0, min(i, len(x) - T)):][:T]).float().to(DEV)
        assert torch.equal(y[:, :F // 32], ref[:, None].expand(-1, F // 32)), i
        assert (y[:, F // 32:] == 0).all()
    assert ctx.device_flags() == 0
    ctx.close()
