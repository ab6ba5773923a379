"""Sines of small angles, value by value relative to themselves, and of all others.

Tolerance.  The angle's conversion, its factor and the product with it are 2^-24 of it each, the sine's last sum, the amplitude and
the product with a value of 1 as much again, what the Taylor sums leave 2^-28 at an eighth of a turn: below 2^-21 of the sine.
Further on sine and cosine may be small where the angle is not: below 2^-20 of the amplitude.
"""
import numpy as np
import pytest

from paper_2605_15890_amd import api

TWO_PI = 2 * np.longdouble("3.14159265358979323846264338327950288")


@pytest.mark.gpu
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("inverse", [False, True])
@pytest.mark.parametrize("rot,base,scaling,factor", [(128, 1e6, "linear", 32.0), (64, 10000.0, "none", 1.0), (256, 5e8, "parts", 64.0)])
def test_slow_pairs_near_the_first_positions(rot, base, scaling, factor, layout, inverse):
    import torch
    turns, amplitude = api.agc_rotary_frequencies(rot, base, scaling, factor, 4096.0)
    positions = np.array([0, 1, 2, 3, 7, 1000, -1, -5, -4097], dtype=np.int64)
    # the phase as the table defines it, a signed share of a turn
    phase = np.array([[(int(p) * int(t) + 2 ** 63) % 2 ** 64 - 2 ** 63 for t in turns.view(np.uint64)] for p in positions], dtype=object)
    angle = phase.astype(np.longdouble) * (TWO_PI / np.longdouble(2) ** 64) * (-1 if inverse else 1)
    a, b = (np.arange(rot // 2) * 2 + i for i in (0, 1)) if layout == "interleaved" else (np.arange(rot // 2) + i * (rot // 2) for i in (0, 1))
    x = torch.zeros(len(positions), rot, device="cuda")
    x[:, b] = 1.0
    out = torch.empty_like(x)
    api.agc_rotary_apply(x, 1, torch.from_numpy(positions).cuda(), torch.from_numpy(turns).cuda(), layout, out, amplitude, inverse)
    got = out.double().cpu().numpy()
    near = np.abs(angle) <= TWO_PI / 8
    assert near.sum() > near.size // 2 and np.abs(angle[1]).min() < 1e-3
    for at, want in ((a, -np.sin(angle) * amplitude), (b, np.cos(angle) * amplitude)):
        off = np.abs(got[:, at] - want)
        assert np.all(off[near] <= 2.0 ** -21 * np.abs(want[near])), np.max(off[near] / np.maximum(np.abs(want[near]), 1e-30))
        assert np.all(off <= 2.0 ** -20 * amplitude)
