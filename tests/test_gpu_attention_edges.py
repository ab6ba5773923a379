"""Differential attention at the ends of its ranges, against the formulas in 64 bits; tolerances are those of
test_gpu_attention.py, whose oracle and operands these tests use."""
import numpy as np
import pytest

from paper_2605_15890_amd import api
from test_gpu_attention import Case, raw


# ------------------------------------------------------------------ the scale of the scores
SCALE_LENS = [(90, 130), (33, 33), (1, 700), (40, 7), (0, 5), (64, 64)]


@pytest.mark.gpu
@pytest.mark.parametrize("scale", [0.0, 2.0 ** -149, 2.0 ** -40])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("heads,kv_heads,d,e", [(2, 2, 32, 64), (4, 2, 64, 128), (2, 1, 128, 256), (3, 1, 20, 33), (2, 1, 40, 72)])
def test_scales_that_make_the_maps_uniform(scale, causal, heads, kv_heads, d, e):
    """Every key in sight counts alike, those out of sight not at all."""
    c = Case(SCALE_LENS, heads, kv_heads, d, e, causal)
    c.scale = float(np.float32(scale))
    c.head = (*c.head[:8], c.scale, causal)
    c.check_forward(c.forward())
    parts = [50, c.nq]
    c.check_gradients(*c.gradients(parts), parts)


@pytest.mark.gpu
def test_scale_zero_with_scores_of_any_size():
    """Scores of up to 2^126 are still all alike."""
    c = Case([(70, 70), (5, 300)], 2, 1, 64, 128, True)
    for t in (c.q, c.k):
        t.mul_(2.0 ** 60)
    c.qh, c.kh, c.scale = c.q.double().cpu().numpy(), c.k.double().cpu().numpy(), 0.0
    c.head = (*c.head[:8], 0.0, True)
    c.check_forward(c.forward())
    c.q.mul_(2.0 ** -60)     # the products of dk stay finite
    c.qh = c.q.double().cpu().numpy()
    c.check_gradients(*c.gradients([c.nq]), [c.nq])


@pytest.mark.gpu
def test_scale_zero_in_large_workgroups():
    """Under the causal mask query i of as many keys gets the mean of the first i + 1 values times 1 - lambda: a map's value
    and the result are rounded, 2^-8 each."""
    import torch
    n, heads, seqs = 1300, 8, 8
    c = Case([(n, n)] * seqs, heads, heads, 64, 128, True)
    c.head = (*c.head[:8], 0.0, True)
    out = c.forward()[:, :heads * 128].double().view(seqs, n, heads, 128)
    v = c.v.double().view(seqs, n, heads, 128)
    count = torch.arange(1, n + 1, device="cuda").double()[:, None, None]
    lam = c.lam.double()[:, None]
    want = v.cumsum(1) / count * (1 - lam)
    tol = 2.0 ** -8 * want.abs() + (2.0 ** -8 + c.full({"A": 0.0})) * v.abs().cumsum(1) / count * (1 + lam.abs())
    assert bool(((out - want).abs() <= tol).all())
    lse = c.lse.double().view(heads, 2, seqs, n)
    assert float((lse - torch.log2(count[:, 0, 0])).abs().max()) <= 2.0 ** -20
    dq, dk, dv, G = c.gradients([c.nq])
    assert not dq.any() and not dk.any()
    # every key's dv: the sum over the queries from it on of (1 - lambda) dout / (i + 1)
    part = (c.dout.double().view(seqs, n, heads, 128) / count).flip(1).cumsum(1).flip(1)
    size = (c.dout.double().view(seqs, n, heads, 128).abs() / count).flip(1).cumsum(1).flip(1)
    dv = dv.double().view(seqs, n, heads, 128)
    tol = 2.0 ** -8 * (part * (1 - lam)).abs() + 2.0 ** -16 * size * (1 - lam).abs() + c.full({"A": 0.0}) * size * (1 + lam.abs())
    assert bool(((dv - part * (1 - lam)).abs() <= tol).all())


@pytest.mark.gpu
@pytest.mark.parametrize("d,e", [(32, 64), (64, 128), (128, 256)])
def test_scores_of_two_to_the_29th(d, e):
    """Products that are exact, 2^21 and more apart: each query takes the one key of its largest score in each map, whose power is
    within 2^32 of 1 and rounded with the map, and the result: 2^-8 each, and 2^-22 for the division."""
    import torch
    c = Case([(40, 250), (70, 70)], 2, 1, d, e, True)
    g = torch.Generator(device="cuda").manual_seed(d)
    level = torch.stack([torch.cat([torch.randperm(n, generator=g, device="cuda") for n in c.lk]) for _ in range(2)], 1) + 1     # of a key and map
    c.q.fill_(2.0 ** 14)
    c.k.view(-1, 2, d).copy_((level.float() * (2.0 ** 7 / d))[:, :, None])
    c.head = (*c.head[:8], 1.0, True)
    out = c.forward()[:, :2 * e].double().view(-1, 2, e)
    lam, v, i, j = c.lam.double()[:, None], c.v.double(), 0, 0
    for lq, lk in c.lens:
        for t in range(lq):
            seen = t + lk - lq + 1
            first, second = (v[j + int(level[j:j + seen, m].argmax())] for m in range(2))
            want, size = first - lam * second, first.abs() + lam.abs() * second.abs()
            assert bool(((out[i + t] - want).abs() <= 2.0 ** -8 * want.abs() + (2.0 ** -8 + 2.0 ** -21) * size).all())
        i, j = i + lq, j + lk


# ------------------------------------------------------------------ rows far apart
@pytest.mark.gpu
@pytest.mark.parametrize("d,e,far", [(32, 64, "v"), (64, 128, "v"), (64, 128, "k"), (24, 40, "v"), (64, 128, "q"), (64, 128, "dout")])
def test_partial_tiles_of_rows_at_the_largest_stride(d, e, far):
    """The large keys' pass has 256 values a workgroup, and 200 of them span 2^32 bytes at a stride of 2^24: the same results, bit
    for bit, as from rows side by side."""
    import torch
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("needs 40 GB")
    heads = 96
    c = Case([(90, 712)] if far in "kv" else [(712, 712)], heads, heads, d, e, False)
    want, got = [], []
    for which in (want, got):
        out = c.forward()
        dq, dk, dv, G = c.gradients([c.nq])
        which.extend((out, c.lse.clone(), dq, dk, dv, torch.from_numpy(G)))
        if which is want:
            near = getattr(c, far)
            wide = torch.empty(len(near), 1 << 24, dtype=torch.bfloat16, device="cuda")
            moved = wide[:, 4096:4096 + near.shape[1]]
            moved.copy_(near)
            setattr(c, far, moved)
            c.head = (c.q, c.k, c.v, *c.head[3:])
    assert all(torch.equal(a, b) for a, b in zip(got, want))


# ------------------------------------------------------------------ the most sequences
@pytest.mark.gpu
def test_a_million_sequences_of_many_rows():
    """2^20 sequences of 64 queries, four heads on one, and a key each, which the last query alone sees: its map is 1."""
    import torch
    if torch.cuda.mem_get_info()[0] < 48 << 30:
        pytest.skip("needs 48 GB")
    n, heads, d, e = 1 << 20, 4, 8, 8
    g = torch.Generator(device="cuda").manual_seed(0)
    bf16 = torch.bfloat16
    q = torch.randn(64 * n, heads * 2 * d, generator=g, device="cuda").to(bf16)
    k, v = (torch.randn(n, w, generator=g, device="cuda").to(bf16) for w in (2 * d, e))
    lam = torch.tensor([0.25, -0.5, 1.0, 0.75], device="cuda")
    q_end = (torch.arange(1, n + 1, device="cuda") * 64).to(torch.int32)
    k_end = torch.arange(1, n + 1, device="cuda", dtype=torch.int32)
    out = torch.full((64 * n, heads * e), 3.0, dtype=bf16, device="cuda")
    ws = torch.empty(api.agc_diff_attn_workspace_bytes(64 * n, n, n, heads, 1, d, e), dtype=torch.uint8, device="cuda")
    api.agc_diff_attn_forward(q, k, v, heads, 1, lam, q_end, k_end, 0.25, True, out, ws)
    rows = out.view(n, 64, heads, e)
    assert not rows[:, :63].any()
    want = v.float()[:, None] * (1 - lam[:, None])
    # the one power of two that a map consists of is rounded, and so is the result
    assert bool(((rows[:, 63].float() - want).abs() <= 2.0 ** -8 * (v.float().abs()[:, None] * (1 + lam.abs()[:, None]) + want.abs())).all())


@pytest.mark.parametrize("grad", [False, True])
@pytest.mark.parametrize("scale", [2.4e38, 3.4e38])
def test_scales_whose_binary_one_is_infinite_are_refused(grad, scale):
    """Scores enter powers of two: their factor is scale * log2(e)."""
    assert raw(grad, scale=scale) == api.AGC_EINVAL


@pytest.mark.parametrize("change", [
    dict(nq=2 ** 26, heads=10, ldq=4096, d=8, e=136), dict(nk=2 ** 26, heads=10, kv=10, ldq=2048, ldk=2048, ldv=2048, d=72, e=8)])
def test_more_wide_heads_than_a_launch_has_threads_for_are_refused(change):
    for grad in (False, True):
        assert raw(grad, **change) == api.AGC_ESHAPE


def test_more_rows_of_G_than_a_launch_has_threads_for_are_refused():
    assert raw(True, parts=(3,) * 256, heads=8192, kv=1, d=8, e=8, ldq=2 ** 17, lddq=2 ** 17, lddout=2 ** 16, ldg=8192) == api.AGC_ESHAPE
