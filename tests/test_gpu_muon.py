"""Orthogonalised update on the GPU against the same formulas in 64 bits on the host.

Tolerance of X (read off beta with beta = 0, rate 1): operands of 22 bits and binary32 sums give each of the three
products of a step a relative error of about 2^-22 in the 2-norm; a step multiplies what is there in directions of
small singular values by at most 3.4445, as it does X itself, so against |X| the error of a matrix whose singular values
are alike grows with the number of products alone: 15 * 2^-22 = 4e-6, taken as 1e-5.  Matrices of low rank are held to
the amplification of binary32 rounding instead, 3.4445^5 * 2^-24 * 4 = 1.2e-4.
"""
import numpy as np
import pytest

from paper_2605_15890_amd import api

A, B, C = 3.4445, -4.7750, 2.0315


def host_update(beta, m1, g, rows, cols, lr, mu, nesterov, decay, scale, steps):
    m1 = mu * m1 + g
    u = (g + mu * m1 if nesterov else m1).reshape(rows, cols)
    x = u / (np.linalg.norm(u) + 1e-7)
    x = x.T if rows > cols else x
    for _ in range(steps):
        gram = x @ x.T
        x = A * x + (B * gram + C * (gram @ gram)) @ x
    x = x.T if rows > cols else x
    return (1 - lr * decay) * beta - lr * scale * x.reshape(-1), m1


def run(rows, cols, mats=1, lr=1.0, mu=0.0, nesterov=False, decay=0.0, scale=1.0, steps=5, lead=0, gap=0, rank=0,
        copy=False, beta_std=0.0, seed=0):
    import torch
    rng = np.random.default_rng(seed)
    size = rows * cols
    offsets = [lead + i * (size + gap) for i in range(mats)]
    length = lead + mats * (size + gap) + 3
    beta = (beta_std * rng.standard_normal(length)).astype(np.float32)
    m1, g = (rng.standard_normal(length).astype(np.float32) for _ in range(2))
    if rank:
        for off in offsets:
            g[off:off + size] = (rng.standard_normal((rows, rank)) @ rng.standard_normal((rank, cols))).reshape(-1)
        m1[:] = 0
    dev = [torch.from_numpy(v.copy()).cuda() for v in (beta, m1, g)]
    half = torch.full((length,), 7.0, dtype=torch.bfloat16, device="cuda") if copy else None
    ws = torch.full((api.agc_muon_workspace_bytes(rows, cols, mats),), 0xFF, dtype=torch.uint8, device="cuda")
    api.agc_muon_update(dev[0], dev[1], dev[2], offsets, rows, cols, lr, mu, nesterov, decay, scale, steps, ws,
                        beta_bf16=half)
    torch.cuda.synchronize()
    got_beta, got_m1 = dev[0].cpu().numpy(), dev[1].cpu().numpy()
    assert np.array_equal(dev[2].cpu().numpy(), g)
    inside = np.zeros(length, bool)
    want_beta, want_m1 = beta.astype(np.float64), m1.astype(np.float64)
    for off in offsets:
        here = slice(off, off + size)
        inside[here] = True
        want_beta[here], want_m1[here] = host_update(want_beta[here], want_m1[here], g[here].astype(np.float64), rows, cols,
                                                     lr, mu, nesterov, decay, scale, steps)
    # nothing beside the matrices is written
    assert np.array_equal(got_beta[~inside], beta[~inside]) and np.array_equal(got_m1[~inside], m1[~inside])
    if copy:
        h = half.float().cpu().numpy()
        assert np.all(h[~inside] == 7.0)
        assert np.array_equal(h[inside], torch.from_numpy(got_beta).bfloat16().float().numpy()[inside])
    return got_beta, want_beta, got_m1, want_m1, [slice(o, o + size) for o in offsets]


def off_by(got, want):
    return np.linalg.norm(got - want) / np.linalg.norm(want)


@pytest.mark.gpu
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 7), (5, 1), (31, 33), (64, 64), (96, 64), (127, 129), (128, 256),
                                       (130, 700), (257, 255), (515, 301), (640, 1025)])
@pytest.mark.parametrize("mats", [1, 3])
def test_orthogonal_factor(rows, cols, mats):
    got, want, m1, want_m1, at = run(rows, cols, mats, lead=1, gap=5, seed=rows * 1000 + cols)
    for here in at:
        assert off_by(got[here], want[here]) < 1e-5
        assert np.array_equal(m1[here], want_m1[here].astype(np.float32))


@pytest.mark.gpu
@pytest.mark.parametrize("rows,cols", [(96, 100), (33, 255), (570, 20), (65, 110), (97, 97), (1, 600), (1030, 3)])
def test_orthogonal_factor_round_the_limits_of_one_launch(rows, cols):
    got, want, m1, want_m1, at = run(rows, cols, 2, gap=1, seed=rows + cols)
    for here in at:
        assert off_by(got[here], want[here]) < 1e-5
        assert np.array_equal(m1[here], want_m1[here].astype(np.float32))


@pytest.mark.gpu
@pytest.mark.parametrize("rows,cols", [(96, 190), (1, 1900), (2000, 33), (64, 700), (95, 1000), (97, 1000), (700, 96)])
@pytest.mark.parametrize("steps", [4, 5])
def test_orthogonal_factor_of_long_matrices(rows, cols, steps):
    """Two steps at once, and a short side of up to 96 between the long products."""
    got, want, _, _, at = run(rows, cols, 2, gap=1, steps=steps, seed=rows + cols)
    for here in at:
        assert off_by(got[here], want[here]) < 1e-5


@pytest.mark.gpu
@pytest.mark.parametrize("rows,cols,mats", [(1300, 1290, 2), (1025, 3001, 5), (4097, 2050, 4), (1111, 1200, 12)])
def test_orthogonal_factor_of_large_matrices(rows, cols, mats):
    """Every tile size and its edges; the 64-bit products are taken on the GPU."""
    import torch
    size = rows * cols
    g = torch.randn(mats * size, device="cuda", generator=torch.Generator("cuda").manual_seed(rows))
    beta, m1 = torch.zeros_like(g), torch.zeros_like(g)
    ws = torch.full((api.agc_muon_workspace_bytes(rows, cols, mats),), 0xFF, dtype=torch.uint8, device="cuda")
    api.agc_muon_update(beta, m1, g, [i * size for i in range(mats)], rows, cols, 1.0, 0.0, False, 0.0, 1.0, 5, ws)
    for i in (0, mats - 1):
        u = g[i * size:(i + 1) * size].double().view(rows, cols)
        x = u.t() if rows > cols else u
        x = (x / (x.norm() + 1e-7)).contiguous()
        for _ in range(5):
            gram = x @ x.t()
            x = A * x + (B * gram + C * (gram @ gram)) @ x
        x = (x.t() if rows > cols else x).reshape(-1)
        assert float((beta[i * size:(i + 1) * size].double() + x).norm() / x.norm()) < 1e-5


@pytest.mark.gpu
@pytest.mark.parametrize("rows,cols", [(70, 200), (200, 70), (300, 300)])
@pytest.mark.parametrize("nesterov,decay,copy,lead", [(True, 0.1, True, 0), (False, 0.0, True, 2), (True, 0.0, False, 4)])
def test_whole_update(rows, cols, nesterov, decay, copy, lead):
    got, want, m1, want_m1, at = run(rows, cols, 2, lr=0.05, mu=0.9, nesterov=nesterov, decay=decay, scale=1.7, lead=lead,
                                     gap=64, copy=copy, beta_std=0.02, seed=rows + cols)
    for here in at:
        assert off_by(got[here], want[here]) < 1e-5
        assert off_by(m1[here], want_m1[here]) < 2e-7


@pytest.mark.gpu
@pytest.mark.parametrize("rows,cols,rank", [(128, 128, 1), (300, 200, 4), (64, 900, 16)])
def test_low_rank(rows, cols, rank):
    got, want, _, _, at = run(rows, cols, rank=rank, seed=rank)
    assert off_by(got[at[0]], want[at[0]]) < 1.2e-4


@pytest.mark.gpu
@pytest.mark.parametrize("steps", [1, 2, 6])
def test_number_of_steps(steps):
    got, want, _, _, at = run(100, 60, steps=steps, seed=steps)
    assert off_by(got[at[0]], want[at[0]]) < 1e-5


@pytest.mark.gpu
@pytest.mark.parametrize("size", [1e-20, 1e18])
def test_norms_outside_the_range_of_squares(size):
    """Squares of the gradient leave binary32; its norm is 64-bit.  Below eps the factor fades out."""
    import torch
    rows, cols = 40, 50
    g = np.random.default_rng(3).standard_normal(rows * cols).astype(np.float32) * np.float32(size)
    beta, m1, gd = torch.zeros(rows * cols, device="cuda"), torch.zeros(rows * cols, device="cuda"), torch.from_numpy(g).cuda()
    ws = torch.empty(api.agc_muon_workspace_bytes(rows, cols, 1), dtype=torch.uint8, device="cuda")
    api.agc_muon_update(beta, m1, gd, [0], rows, cols, 1.0, 0.0, False, 0.0, 1.0, 5, ws)
    want, _ = host_update(np.zeros(rows * cols), np.zeros(rows * cols), g.astype(np.float64), rows, cols, 1.0, 0.0, False,
                          0.0, 1.0, 5)
    got = beta.cpu().numpy()
    if size > 1:
        assert off_by(got, want) < 1e-5
    else:   # |U| = 1e-18 of eps = 1e-7: X = 5e-10 after five steps, below the unit that X is held in
        assert np.abs(got - want).max() < 2.0 ** -25 / 16384 * 485


@pytest.mark.gpu
def test_zero_gradient_and_a_matrix_that_is_not_finite():
    import torch
    rows, cols = 33, 65
    size = rows * cols
    g = torch.randn(3 * size, device="cuda")
    g[:size] = 0.0
    g[size + 5] = float("nan")
    beta, m1 = torch.zeros(3 * size, device="cuda"), torch.zeros(3 * size, device="cuda")
    ws = torch.empty(api.agc_muon_workspace_bytes(rows, cols, 3), dtype=torch.uint8, device="cuda")
    api.agc_muon_update(beta, m1, g, [0, size, 2 * size], rows, cols, 1.0, 0.9, True, 0.0, 1.0, 5, ws)
    assert torch.all(beta[:size] == 0)
    assert torch.isnan(beta[size:2 * size]).any()
    assert torch.isfinite(beta[2 * size:]).all() and beta[2 * size:].abs().sum() > 0


@pytest.mark.gpu
def test_same_result_twice_on_another_stream_and_in_a_graph():
    import torch
    rows, cols, mats = 200, 333, 2
    size = rows * cols
    g, m0 = torch.randn(mats * size, device="cuda"), torch.randn(mats * size, device="cuda")
    ws = torch.empty(api.agc_muon_workspace_bytes(rows, cols, mats), dtype=torch.uint8, device="cuda")

    def update(beta, m1):
        api.agc_muon_update(beta, m1, g, [0, size], rows, cols, 0.1, 0.9, True, 0.01, 1.0, 5, ws)

    beta, m1 = torch.ones_like(g), m0.clone()
    update(beta, m1)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    beta2, m2 = torch.ones_like(g), m0.clone()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        update(beta2, m2)
    torch.cuda.synchronize()
    assert torch.equal(beta, beta2) and torch.equal(m1, m2)
    beta3, m3 = torch.ones_like(g), m0.clone()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        update(beta3, m3)
    for _ in range(3):
        beta3.fill_(1.0)
        m3.copy_(m0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(beta, beta3) and torch.equal(m1, m3)


def test_refusals():
    """Arguments that are refused before anything reaches the GPU (addresses are never followed)."""
    L = api.load()
    off = np.array([0, 4096], dtype=np.int64).tobytes()

    def call(beta=4096, m1=8192, g=12288, offsets=off, n=2, rows=8, cols=16, steps=5, half=None, ws=16384):
        return L.agc_muon_update(beta, m1, g, offsets, n, rows, cols, 0.1, 0.9, 1, 0.0, 1.0, steps, half, ws, None)

    for kw in (dict(beta=None), dict(m1=None), dict(g=None), dict(offsets=None), dict(ws=None), dict(steps=0), dict(steps=33)):
        assert call(**kw) == api.AGC_EINVAL, kw
    for kw in (dict(rows=0), dict(cols=-1), dict(rows=32769), dict(n=0), dict(n=257),
               dict(offsets=np.array([0, 127], dtype=np.int64).tobytes()),
               dict(offsets=np.array([-1, 4096], dtype=np.int64).tobytes())):
        assert call(**kw) == api.AGC_ESHAPE, kw
    for kw in (dict(beta=4098), dict(m1=8193), dict(g=12290), dict(half=4097), dict(ws=16384 + 128)):
        assert call(**kw) == api.AGC_EALIGN, kw
    assert b"agc_muon_update" in L.agc_last_error(None)
    assert api.agc_muon_workspace_bytes(0, 4, 1) == 0 and api.agc_muon_workspace_bytes(4, 32769, 1) == 0
    assert api.agc_muon_workspace_bytes(4, 4, 257) == 0 and api.agc_muon_workspace_bytes(4, 4, 1) > 0
