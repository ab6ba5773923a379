"""Gated block on the GPU against the formulas in 64 bits on the host.

Tolerances, of the 2-norm of the difference over that of the result or, for the sums dx and G whose terms may cancel
(all of them where a single value is summed), over that of the sums of the terms' magnitudes.  bfloat16 has 8 bits, so rounding to it is off by at
most 2^-8 of a value (1 + 2^-8 lies between two of them).  h: one such rounding, and binary32 sums of up to 1100
products, far below 1e-5.  dx: its own rounding and that of da and du: 2 * 2^-8.  G: da and du as pairs of bfloat16,
2^-16 = 1.53e-5 at most, and binary32 sums: 1.7e-5.
"""
import math

import numpy as np
import pytest

from paper_2605_15890_amd import api

TOL_H, TOL_DX, TOL_G = 2.0 ** -8 + 1e-5, 2.0 ** -7, 1.7e-5


def act_and_slope(a, act):
    if act == "silu":
        s = 1.0 / (1.0 + np.exp(-a))
        return a * s, s * (1.0 + a * (1.0 - s))
    cdf = 0.5 * (1.0 + np.vectorize(math.erf)(a / math.sqrt(2.0)))
    return a * cdf, cdf + a * np.exp(-0.5 * a * a) / math.sqrt(2.0 * math.pi)


def host_forward(x, wg, wu, act):
    return act_and_slope(x @ wg.T, act)[0] * (x @ wu.T)


def host_gradients(x, wg, wu, act, dh, ends):
    a, u = x @ wg.T, x @ wu.T
    value, slope = act_and_slope(a, act)
    da, du = dh * u * slope, dh * value
    def sums(da, du, x, wg, wu):
        G, start = [], 0
        for end in ends:
            G.append(np.concatenate([(da[start:end].T @ x[start:end]).ravel(), (du[start:end].T @ x[start:end]).ravel()]))
            start = end
        return da @ wg + du @ wu, np.array(G)

    return sums(da, du, x, wg, wu) + sums(*(np.abs(v) for v in (da, du, x, wg, wu)))


def normal(rng, rows, cols, std, pad=0, shift=0):
    """bfloat16 rows on the GPU, `pad` elements apart and `shift` elements off the allocation, and their values."""
    import torch
    whole = torch.full((rows * (cols + pad) + shift + 8,), float("nan"), dtype=torch.bfloat16, device="cuda")
    view = whole[shift:shift + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
    view.copy_(torch.from_numpy((std * rng.standard_normal((rows, cols))).astype(np.float32)).bfloat16())
    return view, view.double().cpu().numpy()


def off_by(got, want, size=None):
    return np.linalg.norm(got - want) / np.linalg.norm(want if size is None else size)


def problem(tokens, d_in, d_ff, pad=0, shift=0, seed=0):
    rng = np.random.default_rng(seed)
    x, xh = normal(rng, tokens, d_in, 1.0, pad, shift)
    wg, wgh = normal(rng, d_ff, d_in, d_in ** -0.5, pad, shift)
    wu, wuh = normal(rng, d_ff, d_in, d_in ** -0.5, pad, shift)
    return rng, (x, wg, wu), (xh, wgh, wuh)


def forward(tokens, d_in, d_ff, act, pad=0, shift=0, seed=0):
    import torch
    _, (x, wg, wu), host = problem(tokens, d_in, d_ff, pad, shift, seed)
    whole = torch.full((tokens, d_ff + pad), 3.0, dtype=torch.bfloat16, device="cuda")
    ws = torch.full((api.agc_gated_workspace_bytes(tokens, d_in, d_ff),), 0xFF, dtype=torch.uint8, device="cuda")
    api.agc_gated_forward(x, wg, wu, act, whole[:, :d_ff], ws)
    got = whole.double().cpu().numpy()
    assert np.all(got[:, d_ff:] == 3.0)
    return got[:, :d_ff], host_forward(*host, act)


@pytest.mark.gpu
@pytest.mark.parametrize("tokens", [1, 2, 16, 17, 33, 64, 65, 129, 300])
@pytest.mark.parametrize("d_in,d_ff", [(1, 1), (8, 15), (64, 16), (130, 70), (256, 513), (1100, 200)])
def test_forward(tokens, d_in, d_ff):
    got, want = forward(tokens, d_in, d_ff, "silu", seed=tokens + d_in)
    assert off_by(got, want) < TOL_H


@pytest.mark.gpu
@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("tokens", [5, 200])
@pytest.mark.parametrize("pad,shift", [(0, 1), (8, 0), (8, 8), (3, 0), (64, 4)])
def test_forward_strides_and_alignment(act, tokens, pad, shift):
    got, want = forward(tokens, 128, 96, act, pad, shift, seed=pad + shift)
    assert off_by(got, want) < TOL_H


@pytest.mark.gpu
def test_forward_large_tiles():
    got, want = forward(4100, 192, 4160, "silu")
    assert off_by(got, want) < TOL_H


@pytest.mark.gpu
@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("tokens", [3, 100])
def test_forward_far_arguments(act, tokens):
    """Gates of +-300: exp overflows on one side, the activation ends at a or at 0."""
    import torch
    x = torch.ones(tokens, 64, dtype=torch.bfloat16, device="cuda")
    wg = torch.zeros(4, 64, dtype=torch.bfloat16, device="cuda")
    wg[:, 0] = torch.tensor([300.0, -300.0, 90.0, -90.0])
    wu = torch.full((4, 64), 1 / 64, dtype=torch.bfloat16, device="cuda")
    h = torch.empty(tokens, 4, dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(api.agc_gated_workspace_bytes(tokens, 64, 4), dtype=torch.uint8, device="cuda")
    api.agc_gated_forward(x, wg, wu, act, h, ws)
    want = torch.tensor([300.0, 0.0, 90.0, 0.0])
    assert torch.allclose(h.float().cpu(), want.expand(tokens, 4), rtol=2.0 ** -8, atol=1e-30)


def gradients(tokens, d_in, d_ff, act, ends, pad=0, shift=0, seed=0, with_dx=True):
    import torch
    rng, (x, wg, wu), host = problem(tokens, d_in, d_ff, pad, shift, seed)
    dh, dhh = normal(rng, tokens, d_ff, 1e-3, pad, shift)
    k, half = len(ends), d_in * d_ff
    row = (shift + 2 * half + 5 + 3) // 4 * 4
    G = torch.full((k, row), 7.0, device="cuda")
    dx = torch.full((tokens, d_in + pad), 3.0, dtype=torch.bfloat16, device="cuda")
    ws = torch.full((api.agc_gated_workspace_bytes(tokens, d_in, d_ff, k),), 0xFF, dtype=torch.uint8, device="cuda")
    api.agc_gated_partial_gradients(x, wg, wu, act, dh, ends, dx[:, :d_in] if with_dx else None, G[:, shift:shift + half],
                                    G[:, shift + half:shift + 2 * half], ws)
    got_dx, got_G = dx.double().cpu().numpy(), G.double().cpu().numpy()
    assert np.all(got_G[:, :shift] == 7.0) and np.all(got_G[:, shift + 2 * half:] == 7.0)
    assert np.all(got_dx[:, d_in:] == 3.0) and (with_dx or np.all(got_dx == 3.0))
    want_dx, want_G, size_dx, size_G = host_gradients(*host, act, dhh, ends)
    got_G = got_G[:, shift:shift + 2 * half]
    if with_dx:
        assert off_by(got_dx[:, :d_in], want_dx, size_dx) < TOL_DX
    start = 0
    for p, end in enumerate(ends):
        if end == start:
            assert np.all(got_G[p] == 0.0)
        else:
            assert off_by(got_G[p], want_G[p], size_G[p]) < TOL_G, p
        start = end
    return got_G, host, dhh


@pytest.mark.gpu
@pytest.mark.parametrize("tokens,ends", [(1, [1]), (1, [0, 1, 1]), (31, [5, 31]), (32, [32]), (33, [0, 33]),
                                         (200, [64, 128, 200]), (261, [1, 1, 97, 260, 261])])
@pytest.mark.parametrize("d_in,d_ff,act", [(1, 1, "silu"), (9, 31, "gelu"), (64, 64, "silu"), (130, 70, "gelu"), (300, 210, "silu")])
def test_gradients(tokens, ends, d_in, d_ff, act):
    gradients(tokens, d_in, d_ff, act, ends, seed=tokens + d_in)


@pytest.mark.gpu
@pytest.mark.parametrize("pad,shift", [(0, 1), (8, 0), (8, 8), (3, 0)])
def test_gradients_strides_and_alignment(pad, shift):
    gradients(100, 128, 96, "silu", [40, 100], pad, shift)


@pytest.mark.gpu
def test_gradients_without_dx_and_of_large_tiles():
    gradients(4100, 256, 2100, "silu", [2000, 4100], with_dx=False)
    gradients(4100, 2100, 256, "silu", [2000, 4100])


@pytest.mark.gpu
@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_gradients_against_differences(act):
    """Slope of sum(dh * h) along a random direction of each weight, by central differences in 64 bits: their error is
    about eps^2 = 1e-8 of the slope."""
    tokens, d_in, d_ff, ends = 50, 40, 33, [20, 50]
    G, (x, wg, wu), dh = gradients(tokens, d_in, d_ff, act, ends, seed=5)
    rng, eps = np.random.default_rng(6), 1e-4
    for which, w in ((0, wg), (1, wu)):
        v = rng.standard_normal(w.shape)
        start = 0
        for p, end in enumerate(ends):
            def loss(t):
                ws = [wg, wu]
                ws[which] = w + t * v
                return np.sum(dh[start:end] * host_forward(x[start:end], ws[0], ws[1], act))
            slope = (loss(eps) - loss(-eps)) / (2 * eps)
            row = G[p].reshape(2, d_ff, d_in)[which]
            assert abs(np.sum(row * v) - slope) < 2e-5 * np.linalg.norm(row) * np.linalg.norm(v)
            start = end


@pytest.mark.gpu
@pytest.mark.parametrize("x_std,w_std,dh_std", [(1e-12, 1.0, 1e-3), (1.0, 1e-9, 1e-30), (1e6, 1e-6, 1e12), (1.0, 1.0, 1e-34)])
def test_gradients_far_from_one(x_std, w_std, dh_std):
    """Magnitudes that binary16 does not reach: the partitions' powers of two bring them there and back."""
    import torch
    tokens, d_in, d_ff, ends = 96, 72, 40, [32, 96]
    rng = np.random.default_rng(11)
    x, xh = normal(rng, tokens, d_in, x_std)
    wg, wgh = normal(rng, d_ff, d_in, w_std)
    wu, wuh = normal(rng, d_ff, d_in, w_std)
    dh, dhh = normal(rng, tokens, d_ff, dh_std)
    half = d_in * d_ff
    G = torch.empty(2, 2 * half, device="cuda")
    ws = torch.empty(api.agc_gated_workspace_bytes(tokens, d_in, d_ff, 2), dtype=torch.uint8, device="cuda")
    api.agc_gated_partial_gradients(x, wg, wu, "silu", dh, ends, None, G[:, :half], G[:, half:], ws)
    _, want, _, size = host_gradients(xh, wgh, wuh, "silu", dhh, ends)
    got = G.double().cpu().numpy()
    for p in range(2):
        for part in (slice(0, half), slice(half, 2 * half)):
            # binary32 holds nothing below 2^-149
            assert np.linalg.norm(got[p, part] - want[p, part]) < TOL_G * np.linalg.norm(size[p, part]) + half ** 0.5 * 2.0 ** -149


@pytest.mark.gpu
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_what_is_not_finite_stays_in_its_partition(bad):
    import torch
    tokens, d_in, d_ff, ends = 100, 40, 24, [30, 60, 100]
    rng, (x, wg, wu), _ = problem(tokens, d_in, d_ff, seed=3)
    dh, _ = normal(rng, tokens, d_ff, 1e-3)
    half = d_in * d_ff
    ws = torch.empty(api.agc_gated_workspace_bytes(tokens, d_in, d_ff, 3), dtype=torch.uint8, device="cuda")

    def call():
        G = torch.empty(3, 2 * half, device="cuda")
        dx = torch.empty(tokens, d_in, dtype=torch.bfloat16, device="cuda")
        api.agc_gated_partial_gradients(x, wg, wu, "silu", dh, ends, dx, G[:, :half], G[:, half:], ws)
        return G, dx

    G, dx = call()
    x[45, 7] = bad
    dh[50, 3] = bad
    H, dy = call()
    assert torch.equal(G[0], H[0]) and torch.equal(G[2], H[2]) and not torch.isfinite(H[1]).all()
    others = torch.ones(tokens, dtype=torch.bool, device="cuda")
    others[[45, 50]] = False
    assert torch.equal(dx[others], dy[others]) and not torch.isfinite(dy[45].float()).all()


@pytest.mark.gpu
def test_zero_tokens():
    import torch
    bf16 = torch.bfloat16
    x, w = torch.empty(0, 24, dtype=bf16, device="cuda"), torch.randn(16, 24, device="cuda").to(bf16)
    h, ws = torch.empty(0, 16, dtype=bf16, device="cuda"), torch.empty(1 << 16, dtype=torch.uint8, device="cuda")
    api.agc_gated_forward(x, w, w, "silu", h, ws)
    G = torch.full((3, 2 * 16 * 24), 7.0, device="cuda")
    api.agc_gated_partial_gradients(x, w, w, "silu", h, [0, 0, 0], None, G[:, :384], G[:, 384:], ws)
    assert torch.all(G == 0)


@pytest.mark.gpu
def test_same_result_twice_on_another_stream_and_in_a_graph():
    import torch
    tokens, d_in, d_ff, ends = 150, 72, 100, [50, 150]
    rng, (x, wg, wu), _ = problem(tokens, d_in, d_ff)
    dh, _ = normal(rng, tokens, d_ff, 1e-3)
    ws = torch.empty(api.agc_gated_workspace_bytes(tokens, d_in, d_ff, 2), dtype=torch.uint8, device="cuda")
    half = d_in * d_ff

    def make():
        return (torch.zeros(tokens, d_ff, dtype=torch.bfloat16, device="cuda"),
                torch.zeros(tokens, d_in, dtype=torch.bfloat16, device="cuda"), torch.zeros(2, 2 * half, device="cuda"))

    def call(h, dx, G):
        api.agc_gated_forward(x, wg, wu, "silu", h, ws)
        api.agc_gated_partial_gradients(x, wg, wu, "silu", dh, ends, dx, G[:, :half], G[:, half:], ws)

    first, second, third = make(), make(), make()
    call(*first)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call(*second)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, second))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(*third)
    for _ in range(3):
        for t in third:
            t.fill_(9.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(first, third))


def test_refusals():
    """Arguments that are refused before anything reaches the GPU (addresses are never followed)."""
    L = api.load()

    def fwd(x=4096, ldx=16, wg=8192, wu=12288, ldw=16, tokens=4, d_in=16, d_ff=8, act=0, h=16384, ldh=8, ws=20480):
        return L.agc_gated_forward(x, ldx, wg, wu, ldw, tokens, d_in, d_ff, act, h, ldh, ws, None)

    for kw in (dict(x=None), dict(wg=None), dict(wu=None), dict(h=None), dict(ws=None), dict(act=2), dict(act=-1)):
        assert fwd(**kw) == api.AGC_EINVAL, kw
    for kw in (dict(ldx=15), dict(ldw=15), dict(ldh=7), dict(tokens=-1), dict(tokens=(1 << 26) + 1), dict(d_in=0),
               dict(d_ff=65537)):
        assert fwd(**kw) == api.AGC_ESHAPE, kw
    for kw in (dict(x=4097), dict(wg=8193), dict(wu=12289), dict(h=16385), dict(ws=20480 + 16)):
        assert fwd(**kw) == api.AGC_EALIGN, kw

    def grad(x=4096, dh=8192, lddh=8, ends=(2, 4), k=2, dx=12288, lddx=16, gg=16384, gu=20480, ldg=256, act=0, ws=24576):
        packed = None if ends is None else np.array(ends, dtype=np.int64).tobytes()
        return L.agc_gated_partial_gradients(x, 16, 4096, 4096, 16, dh, lddh, 4, packed, k, 16, 8, act, dx, lddx, gg, gu, ldg,
                                             ws, None)

    for kw in (dict(x=None), dict(dh=None), dict(ends=None), dict(gg=None), dict(gu=None), dict(act=3), dict(ws=None)):
        assert grad(**kw) == api.AGC_EINVAL, kw
    for kw in (dict(lddh=7), dict(lddx=15), dict(ldg=127), dict(ends=(3, 2)), dict(ends=(-1, 4)), dict(ends=(2, 3)), dict(k=0),
               dict(k=257)):
        assert grad(**kw) == api.AGC_ESHAPE, kw
    for kw in (dict(dh=8193), dict(dx=12289), dict(gg=16386), dict(gu=20481), dict(ws=24577)):
        assert grad(**kw) == api.AGC_EALIGN, kw
    assert b"agc_gated_partial_gradients" in L.agc_last_error(None)
    assert api.agc_gated_workspace_bytes(-1, 4, 4) == 0 and api.agc_gated_workspace_bytes(4, 0, 4) == 0
    assert api.agc_gated_workspace_bytes(4, 4, 4, 257) == 0 and api.agc_gated_workspace_bytes(4, 4, 4) > 0
