"""The gate's activations far from zero, one value at a time: a and u are single bfloat16 weights (x is 1), so that they
are exact, and h, G are what the activation makes of them.
"""
import math

import numpy as np
import pytest

from paper_2605_15890_amd import api

U = 2.0 ** -24


def block(tokens, gates, ups, d_in=64):
    """x and weights with a[t, f] = sum of the columns of gates[f], u[t, f] = ups[f]."""
    import torch
    gates = np.asarray(gates, dtype=np.float32).reshape(len(ups), -1)
    x = torch.zeros(tokens, d_in, dtype=torch.bfloat16, device="cuda")
    wg, wu = (torch.zeros(len(ups), d_in, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    n = gates.shape[1]
    x[:, :n + 1] = 1.0
    wg[:, :n] = torch.from_numpy(gates).cuda()
    wu[:, n] = torch.tensor(ups, device="cuda")
    return x, wg, wu


def forward(tokens, gates, ups, act):
    import torch
    x, wg, wu = block(tokens, gates, ups)
    h = torch.empty(tokens, len(ups), dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(api.agc_gated_workspace_bytes(tokens, 64, len(ups)), dtype=torch.uint8, device="cuda")
    api.agc_gated_forward(x, wg, wu, act, h, ws)
    assert torch.equal(h, h[:1].expand(tokens, len(ups))) or torch.isnan(h).any()
    return h[0].double().cpu().numpy()


def gradient(gates, ups, act, dh_value):
    """da and du, read off G: one token, x is 1."""
    import torch
    x, wg, wu = block(1, gates, ups)
    n = len(ups)
    dh = torch.full((1, n), dh_value, dtype=torch.bfloat16, device="cuda")
    G = torch.empty(1, 2 * n * 64, device="cuda")
    ws = torch.empty(api.agc_gated_workspace_bytes(1, 64, n, 1), dtype=torch.uint8, device="cuda")
    api.agc_gated_partial_gradients(x, wg, wu, act, dh, [1], None, G[:, :n * 64], G[:, n * 64:], ws)
    G = G.double().cpu().numpy().reshape(2, n, 64)
    return G[0, :, 0], G[1, :, 0], float(dh[0, 0])


@pytest.mark.gpu
@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("tokens", [3, 100])
def test_gates_near_the_largest_binary32_and_beyond(act, tokens):
    """act(a) = a, also where a log2(e) or the sum of finite products itself is infinite; 0 far below zero.  Half of a
    bfloat16 value is exact."""
    gates = [[1e38, 0], [2.3e38, 0], [2.4e38, 0], [3e38, 0], [3e38, 3e38], [-3e38, 0], [1e30, 0]]
    got = forward(tokens, gates, [0.5] * len(gates), act)
    import torch
    want = torch.tensor([1e38, 2.3e38, 2.4e38, 3e38, float("inf"), 0.0, 1e30]).bfloat16().double().numpy() / 2
    assert np.array_equal(got, want)


@pytest.mark.gpu
def test_gradients_of_gates_near_the_largest_binary32():
    """da = dh u, du = dh a: two roundings at most."""
    gates = [[1e38], [2.4e38], [3e38], [-3e38]]
    da, du, dh = gradient(gates, [0.5] * 4, "silu", 1e-9)
    import torch
    a = torch.tensor(gates).bfloat16().double().numpy()[:, 0]
    on = a > 0
    assert np.all(np.abs(da - dh * 0.5 * on) <= 2 * U * dh)
    assert np.all(np.abs(du - dh * a * on) <= 2 * U * np.abs(dh * a * on))


def gelu(a):
    """Value, derivative and the bound of a binary32 derivative's error: the arguments of erfc and exp are rounded (2 and 1
    roundings: a^2 of their relative error each time 2, and a^2 / 2), erfc is within 16 ulp, exp within 3, and 4 operations."""
    a = np.asarray(a)
    cdf = np.array([0.5 * math.erfc(-v / math.sqrt(2.0)) for v in a])
    bell = a * np.exp(-0.5 * a * a) / math.sqrt(2.0 * math.pi)
    return a * cdf, cdf + bell, (2 * a * a + 36) * U * cdf + (2 * a * a + 10) * U * np.abs(bell)


TAILS = [-12.0, -10.0, -9.0, -8.0, -7.0, -6.0, -5.75, -5.5, -5.25, -5.0, -4.5, -4.0, -3.0, -2.0, -1.0, -0.5, -0.01, 0.01, 1.0, 5.0, 12.0]


@pytest.mark.gpu
@pytest.mark.parametrize("tokens", [3, 100])
def test_gelu_below_zero(tokens):
    """h is activation and one rounding to bfloat16, however small it is."""
    import torch
    got = forward(tokens, [[v] for v in TAILS], [1.0] * len(TAILS), "gelu")
    a = torch.tensor(TAILS).bfloat16().double().numpy()
    want, _, _ = gelu(a)
    assert np.all(np.abs(got - want) <= (2.0 ** -8 + (2 * a * a + 36) * U) * np.abs(want))


@pytest.mark.gpu
def test_gradients_of_gelu_below_zero():
    import torch
    da, du, dh = gradient([[v] for v in TAILS], [1.0] * len(TAILS), "gelu", 1.0)
    a = torch.tensor(TAILS).bfloat16().double().numpy()
    value, slope, bound = gelu(a)
    assert np.all(np.abs(da - slope) <= bound)
    assert np.all(np.abs(du - value) <= (2 * a * a + 36) * U * np.abs(value))
