"""Differential attention on the GPU against the formulas in 64 bits on the host.

Tolerances, element by element.  With u = 2^-24 and A the largest sum of |scale q k| of a pair, a score in binary32 is off by
(d + 4) u A at most and a map's value by as much of itself, with the sum it is divided by and the powers of two: below
F = 4 (d + e + 32) u (1 + A) of itself for all of binary32 together.  To that come the roundings to bfloat16, 2^-8 each: one of
every map's value in its product with v (out), and one of the result.  In the gradients the difference of the maps (dv) and dS
(dq, dk) enter as two bfloat16 parts: the first leaves 2^-8 of a value, the second 2^-8 of that.  A map's value below 2^-126 is
no binary32 any more and becomes zero: a sum of the 8192 at most that a test holds, each times factors below 2^7 and 2^5,
loses less than 2^-100 by it, which every bound of the gradients has on top.
    out  2^-8 |out| + (2^-8 + F) sum of (P1 + |lambda| P2) |v|
    dv   2^-8 |dv|  + 2^-16 sum of |P1 - lambda P2| |dout| + F sum of (P1 + |lambda| P2) |dout|
    dq   2^-8 |dq|  + scale (2^-16 sum of |dS| |k| + F sum of T |k|),  T = P (sum |dout v| + sum over keys of P sum |dout v|)
    dk   as dq, with q;   G  F times the sum of T;   lse  (d + 8) u A log2(e) + 2^-20
"""
import math

import numpy as np
import pytest

from paper_2605_15890_amd import api

U = 2.0 ** -24
HALF = 2.0 ** -8


def reference(q, k, v, lam, scale, causal, dout=None):
    """One sequence: q (Lq, H, 2, d), k (Lk, Hk, 2, d), v (Lk, Hk, e), dout (Lq, H, e), all 64 bits.  Results and the
    magnitudes that the tolerances multiply."""
    (lq, heads, _, d), (lk, kv_heads, e) = q.shape, v.shape
    group = heads // kv_heads
    r = dict(out=np.zeros((lq, heads, e)), lse=np.full((heads, 2, lq), -np.inf))
    r["out_size"], r["A"] = np.zeros_like(r["out"]), 0.0
    if dout is not None:
        r.update(dq=np.zeros_like(q), dk=np.zeros_like(k), dv=np.zeros_like(v), share=np.zeros((lq, heads)))
        for n in ("dq", "dk", "dv", "share"):
            r[n + "_half"], r[n + "_full"] = np.zeros_like(r[n]), np.zeros_like(r[n])
    if lq == 0 or lk == 0:
        return r
    seen = np.ones((lq, lk), bool)
    if causal:
        seen = np.arange(lk) <= np.arange(lq)[:, None] + lk - lq
    for h in range(heads):
        c = h // group
        P = []
        for m in range(2):
            s = scale * q[:, h, m] @ k[:, c, m].T
            r["A"] = max(r["A"], (abs(scale) * np.abs(q[:, h, m]) @ np.abs(k[:, c, m]).T).max())
            s = np.where(seen, s, -np.inf)
            top = s.max(1, keepdims=True)
            top = np.where(np.isfinite(top), top, 0)
            p = np.exp(s - top)
            total = p.sum(1, keepdims=True)
            with np.errstate(divide="ignore"):
                r["lse"][h, m] = ((top + np.log(total)) / math.log(2))[:, 0]
            P.append(p / np.where(total > 0, total, 1))
        mixed, size = P[0] - lam[h] * P[1], P[0] + abs(lam[h]) * P[1]
        r["out"][:, h], r["out_size"][:, h] = mixed @ v[:, c], size @ np.abs(v[:, c])
        if dout is None:
            continue
        dp, dp_size = dout[:, h] @ v[:, c].T, np.abs(dout[:, h]) @ np.abs(v[:, c]).T
        r["dv"][:, c] += mixed.T @ dout[:, h]
        r["dv_half"][:, c] += np.abs(mixed).T @ np.abs(dout[:, h])
        r["dv_full"][:, c] += size.T @ np.abs(dout[:, h])
        for m, f in enumerate((1.0, -lam[h])):
            mean, mean_size = (P[m] * dp).sum(1, keepdims=True), (P[m] * dp_size).sum(1, keepdims=True)
            ds, T = f * P[m] * (dp - mean), abs(f) * P[m] * (dp_size + mean_size)
            r["dq"][:, h, m] = scale * ds @ k[:, c, m]
            r["dq_half"][:, h, m], r["dq_full"][:, h, m] = (abs(scale) * x @ np.abs(k[:, c, m]) for x in (np.abs(ds), T))
            r["dk"][:, c, m] += scale * ds.T @ q[:, h, m]
            r["dk_half"][:, c, m] += abs(scale) * np.abs(ds).T @ np.abs(q[:, h, m])
            r["dk_full"][:, c, m] += abs(scale) * T.T @ np.abs(q[:, h, m])
            if m == 1:
                r["share"][:, h], r["share_full"][:, h] = -mean[:, 0], mean_size[:, 0]
    return r


def test_reference_by_differences():
    """The oracle's gradients against differences of its own forward pass: errors of the third order of a step of 1e-4."""
    rng = np.random.default_rng(0)
    q, k, v, dout = (rng.standard_normal(s) for s in ((5, 4, 2, 3), (6, 2, 2, 3), (6, 2, 4), (5, 4, 4)))
    lam = np.array([0.3, -0.7, 0.5, 1.2])
    r = reference(q, k, v, lam, 0.6, True, dout)

    def loss():
        return (reference(q, k, v, lam, 0.6, True)["out"] * dout).sum()

    for x, g in ((q, r["dq"]), (k, r["dk"]), (v, r["dv"]), (lam, r["share"].sum(0))):
        for i in rng.integers(0, x.size, 6):
            at = np.unravel_index(i, x.shape)
            was, x[at] = x[at], x[at] + 1e-4
            up = loss()
            x[at] = was - 1e-4
            down = loss()
            x[at] = was
            assert abs((up - down) / 2e-4 - g[at]) < 1e-6


def rows(rng, n, width, gap, shift, std=1.0):
    """(n, width) bfloat16 view on the GPU, NaN round it, and its values."""
    import torch
    flat = torch.full((n * (width + gap) + shift + 8,), float("nan"), dtype=torch.bfloat16, device="cuda")
    view = flat[shift:shift + n * (width + gap)].view(n, width + gap)[:, :width]
    view.copy_(torch.from_numpy((rng.standard_normal((n, width)) * std).astype(np.float32)))
    return view, view.double().cpu().numpy()


class Case:
    """Random operands for sequences of lens = [(queries, keys), ...], `behind` rows behind the last one."""
    def __init__(self, lens, heads, kv_heads, d, e, causal, gap=0, shift=0, behind=0, seed=0, std=1.0):
        import torch
        self.rng = rng = np.random.default_rng(seed + d)
        self.lens, self.heads, self.kv_heads, self.d, self.e, self.causal = lens, heads, kv_heads, d, e, causal
        self.lq, self.lk = [n for n, _ in lens], [n for _, n in lens]
        self.nq, self.nk = sum(self.lq) + behind, sum(self.lk) + behind
        self.gap, self.shift, self.scale = gap, shift, float(np.float32(d ** -0.5))
        self.q, self.qh = rows(rng, self.nq, 2 * heads * d, gap, shift, std)
        self.k, self.kh = rows(rng, self.nk, 2 * kv_heads * d, gap, shift, std)
        self.v, self.vh = rows(rng, self.nk, kv_heads * e, gap, shift)
        self.dout, self.douth = rows(rng, self.nq, heads * e, gap, shift)
        self.lam = torch.from_numpy(rng.uniform(-0.5, 1.0, heads).astype(np.float32)).cuda()
        self.q_end, self.k_end = (torch.tensor(np.cumsum(n), dtype=torch.int32, device="cuda") for n in (self.lq, self.lk))
        bytes_ = api.agc_diff_attn_workspace_bytes(self.nq, self.nk, len(lens), heads, kv_heads, d, e, True)
        self.ws = torch.full((bytes_,), 0xFF, dtype=torch.uint8, device="cuda")
        self.head = (self.q, self.k, self.v, heads, kv_heads, self.lam, self.q_end, self.k_end, self.scale, causal)
        self.lse = torch.full((2 * heads, self.nq), 7.0, device="cuda")

    def blank(self, n, width):
        import torch
        return torch.full((n, width + self.gap), 3.0, dtype=torch.bfloat16, device="cuda")

    def forward(self, lse=True, k_begin=None):
        out = self.blank(self.nq, self.heads * self.e)
        api.agc_diff_attn_forward(*self.head, out[:, :self.heads * self.e], self.ws, lse=self.lse if lse else None, k_begin=k_begin)
        return out

    def gradients(self, parts):
        import torch
        dq, dk, dv = (self.blank(t.shape[0], t.shape[1]) for t in (self.q, self.k, self.v))
        G = torch.full((len(parts), self.heads + 3), 9.0, device="cuda")
        api.agc_diff_attn_partial_gradients(*self.head, self.lse, self.dout, parts, *(g[:, :t.shape[1]] for g, t in ((dq, self.q), (dk, self.k), (dv, self.v))),
                                            G[:, 1:1 + self.heads], self.ws)
        assert torch.all(G[:, 0] == 9.0) and torch.all(G[:, 1 + self.heads:] == 9.0)
        return dq, dk, dv, G[:, 1:1 + self.heads].double().cpu().numpy()

    def references(self, gradients=True):
        i = j = 0
        lam = self.lam.double().cpu().numpy()
        for lq, lk in self.lens:
            yield slice(i, i + lq), slice(j, j + lk), reference(
                self.qh[i:i + lq].reshape(lq, self.heads, 2, self.d), self.kh[j:j + lk].reshape(lk, self.kv_heads, 2, self.d),
                self.vh[j:j + lk].reshape(lk, self.kv_heads, self.e), lam, self.scale, self.causal,
                self.douth[i:i + lq].reshape(lq, self.heads, self.e) if gradients else None)
            i, j = i + lq, j + lk

    def untouched(self, t, width, n):
        import torch
        assert torch.all(t[:, width:] == 3.0) and torch.all(t[n:] == 3.0)

    def full(self, r):
        return 4 * (self.d + self.e + 32) * U * (1 + r["A"])

    def check_forward(self, out):
        self.untouched(out, self.heads * self.e, sum(self.lq))
        got = out[:, :self.heads * self.e].double().cpu().numpy().reshape(self.nq, self.heads, self.e)
        lse = self.lse.double().cpu().numpy().reshape(self.heads, 2, self.nq)
        for at, _, r in self.references(False):
            tol = HALF * np.abs(r["out"]) + (HALF + self.full(r)) * r["out_size"]
            assert np.all(np.abs(got[at] - r["out"]) <= tol), np.max(np.abs(got[at] - r["out"]) / np.maximum(tol, 1e-30))
            mine, empty = lse[:, :, at], np.isinf(r["lse"])
            assert np.array_equal(np.isneginf(mine), empty)
            assert np.all(np.abs(np.where(empty, 0, mine) - np.where(empty, 0, r["lse"])) <= (self.d + 8) * U * r["A"] * 1.45 + 2.0 ** -20)
        assert np.all(lse[:, :, sum(self.lq):] == 7.0)

    def check_gradients(self, dq, dk, dv, G, parts):
        share, share_full = np.zeros((self.nq, self.heads)), np.zeros((self.nq, self.heads))
        got = {}
        for n, t, rows_, like in (("dq", dq, sum(self.lq), self.q), ("dk", dk, sum(self.lk), self.k), ("dv", dv, sum(self.lk), self.v)):
            self.untouched(t, like.shape[1], rows_)
            got[n] = t[:, :like.shape[1]].double().cpu().numpy()
        for at_q, at_k, r in self.references():
            for n, at in (("dq", at_q), ("dk", at_k), ("dv", at_k)):
                want = r[n].reshape(len(r[n]), got[n].shape[1])
                tol = HALF * np.abs(want) + (HALF ** 2 * r[n + "_half"] + self.full(r) * r[n + "_full"]).reshape(want.shape) + 2.0 ** -100
                off = np.abs(got[n][at] - want)
                assert np.all(off <= tol), (n, np.max(off / np.maximum(tol, 1e-30)))
            share[at_q], share_full[at_q] = r["share"], self.full(r) * r["share_full"]
        ends = [0] + list(parts)
        for p, (a, b) in enumerate(zip(ends, ends[1:])):
            assert np.all(np.abs(G[p] - share[a:b].sum(0)) <= share_full[a:b].sum(0) + U * np.abs(share[a:b].sum(0)))


LENS = {
    "one": [(1, 1)], "tiny": [(3, 5), (1, 1), (2, 2)], "edge": [(31, 31), (32, 32), (33, 33), (65, 65)], "tiles": [(257, 300), (64, 64)],
    "more_queries": [(40, 7), (300, 65)], "empty": [(0, 9), (5, 0), (0, 0), (70, 70), (8, 0)], "many": [(i % 7, (3 * i) % 11) for i in range(150)],
    "few_keys": [(700, 20), (900, 35)], "long_keys": [(33, 1500)], "long_both": [(300, 1400), (0, 3), (260, 1100)],
    "few_rows": [(1, 700), (2, 1300), (1, 64), (1, 0), (3, 2)], "one_query": [(1, 5000)], "one_query_long": [(1, 8100)],
}


@pytest.mark.gpu
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("heads,kv_heads,d,e", [(2, 2, 32, 64), (4, 1, 64, 128), (3, 3, 64, 128), (2, 1, 128, 256), (7, 1, 20, 33), (2, 2, 1, 1), (6, 2, 128, 7),
                                                (2, 1, 40, 200), (5, 5, 64, 100), (6, 2, 40, 72), (2, 2, 8, 16), (3, 1, 96, 128)])
@pytest.mark.parametrize("lens", list(LENS))
def test_against_the_formulas(lens, heads, kv_heads, d, e, causal):
    import torch
    c = Case(LENS[lens], heads, kv_heads, d, e, causal, seed=len(lens))
    out = c.forward()
    c.check_forward(out)
    assert torch.equal(c.forward(lse=False), out)
    cuts = sorted(int(x) for x in c.rng.integers(0, c.nq + 1, 3))
    parts = cuts + [c.nq]
    c.check_gradients(*c.gradients(parts), parts)


@pytest.mark.gpu
@pytest.mark.parametrize("d,e,gap,shift", [(64, 128, 8, 8), (64, 128, 64, 16), (20, 40, 1, 1), (32, 60, 8, 0), (33, 64, 8, 8), (128, 256, 24, 40), (40, 72, 24, 16),
                                             (40, 72, 4, 0), (40, 72, 8, 4), (8, 8, 0, 0)])
def test_strides_and_rows_behind_the_last_sequence(d, e, gap, shift):
    """NaN lies behind the sequences, between the rows and round the tensors."""
    import torch
    c = Case([(70, 90), (9, 3)], 4, 2, d, e, True, gap=gap, shift=shift, behind=37)
    for t, n in ((c.q, sum(c.lq)), (c.k, sum(c.lk)), (c.v, sum(c.lk)), (c.dout, sum(c.lq))):
        t[n:] = float("nan")
    c.check_forward(c.forward())
    # rows behind belong to a partition and count for nothing
    parts = [20, c.nq - 5, c.nq]
    c.check_gradients(*c.gradients(parts), parts)


@pytest.mark.gpu
@pytest.mark.parametrize("d,e", [(24, 40), (40, 72), (56, 64), (24, 120), (80, 136), (120, 248)])
@pytest.mark.parametrize("lens", ["edge", "empty", "one_query", "long_both"])
def test_widths_filled_up_on_the_way_or_in_the_workspace(d, e, lens):
    """Heads whose chunks of 16 bytes can be read where they lie, and the same ones two bytes off: the same sums, bit for bit."""
    import torch
    got = []
    for shift in (8, 9):
        c = Case(LENS[lens], 4, 2, d, e, True, gap=8, shift=shift, seed=e)
        out = c.forward()
        got.append([out, c.lse, *(torch.from_numpy(g) if isinstance(g, np.ndarray) else g for g in c.gradients([c.nq // 2, c.nq]))])
    for one, other in zip(*got):
        assert torch.equal(one, other)


@pytest.mark.gpu
@pytest.mark.parametrize("std", [0.0, 0.02, 6.0])
def test_flat_and_sharp_maps(std):
    c = Case([(90, 130), (33, 33)], 4, 2, 64, 128, True, std=std)
    c.check_forward(c.forward())
    c.check_gradients(*c.gradients([c.nq]), [c.nq])


@pytest.mark.gpu
def test_a_query_that_sees_one_key_has_no_gradient_of_its_scores():
    """Its map is 1 whatever the score: dq and dk are zeros to the last bit."""
    c = Case([(1, 1)] * 40 + [(9, 1)], 6, 2, 64, 128, True)
    c.forward()
    dq, dk, dv, G = c.gradients([c.nq])
    assert not dq.any() and not dk.any() and dv.any()


@pytest.mark.gpu
def test_rising_and_falling_scores():
    """Maxima that move on with every key, and that stay where they began."""
    import torch
    for order in (1, -1):
        c = Case([(40, 600)], 2, 1, 64, 128, False)
        ramp = torch.linspace(-4, 4, 600, device="cuda")[::order] if order == 1 else torch.linspace(-4, 4, 600, device="cuda").flip(0)
        c.k.copy_((ramp[:, None] * torch.ones(128, device="cuda")).to(torch.bfloat16))
        c.q.copy_(c.q.abs())
        c.kh, c.qh = c.k.double().cpu().numpy(), c.q.double().cpu().numpy()
        c.check_forward(c.forward())
        c.check_gradients(*c.gradients([c.nq]), [c.nq])


@pytest.mark.gpu
def test_caches_with_room_and_shared_keys():
    """Keys of each sequence where k_begin says, among NaN, some shared by two sequences."""
    import torch
    c = Case([(1, 300), (2, 41), (1, 300), (1, 0)], 4, 2, 64, 128, True)
    want = c.forward()
    at = [40, 400, 40, 5]
    k, v = (torch.full((700, t.shape[1]), float("nan"), dtype=torch.bfloat16, device="cuda") for t in (c.k, c.v))
    for t, from_ in ((k, c.k), (v, c.v)):
        t[40:340], t[400:441] = from_[:300], from_[300:341]
        from_[341:641] = from_[:300]      # the third sequence has the first one's keys
    want = c.forward()
    c.k, c.v = k, v
    begin = torch.tensor(at, dtype=torch.int32, device="cuda")
    end = begin + torch.tensor(c.lk, dtype=torch.int32, device="cuda")
    ws = torch.empty(api.agc_diff_attn_workspace_bytes(c.nq, 700, 4, 4, 2, 64, 128), dtype=torch.uint8, device="cuda")
    out = torch.full_like(want, 3.0)
    api.agc_diff_attn_forward(c.q, k, v, 4, 2, c.lam, c.q_end, end, c.scale, True, out, ws, k_begin=begin)
    # the keys are split in other places at most: the maps and the result are rounded in both
    size = float(v[~v.isnan()].abs().max()) * 2
    assert torch.isfinite(out.float()).all() and float((out.float() - want.float()).abs().max()) <= 4 * HALF * size
    assert torch.all(out[4:] == 0)


@pytest.mark.gpu
def test_ends_beyond_the_tensors_count_as_their_ends():
    import torch
    c = Case([(50, 60), (30, 40)], 2, 2, 64, 128, True)
    want = c.forward()
    c.q_end[1], c.k_end[1] = 2 ** 31 - 1, 2 ** 31 - 1
    assert torch.equal(c.forward(), want)
    # ends that descend leave sequences without rows or keys; every access stays inside
    c.q_end[:], c.k_end[:] = torch.tensor([60, -5], dtype=torch.int32), torch.tensor([200, 10], dtype=torch.int32)
    c.forward()
    c.gradients([c.nq])
    torch.cuda.synchronize()


@pytest.mark.gpu
@pytest.mark.parametrize("bad", ["nan", "inf"])
def test_bad_values_stay_in_their_sequence(bad):
    import torch
    lens = [(64, 64), (50, 50), (77, 77)]
    clean = Case(lens, 4, 2, 64, 128, True)
    out, grads = clean.forward(), clean.gradients([64, 114, 191])
    c = Case(lens, 4, 2, 64, 128, True)
    for t in (c.q, c.k, c.v, c.dout):
        t[70:80] = float(bad)
    got, bad_grads = c.forward(), c.gradients([64, 114, 191])
    fine = torch.tensor([i for i in range(191) if not 64 <= i < 114], device="cuda")
    assert torch.equal(got[fine], out[fine]) and torch.isnan(got[70:114].float()).any()
    for a, b in zip(bad_grads[:3], grads[:3]):
        assert torch.equal(a[fine], b[fine])
    assert np.array_equal(bad_grads[3][[0, 2]], grads[3][[0, 2]])


@pytest.mark.gpu
def test_gradient_of_lambda_by_differences():
    """out is linear in lambda; each of the two results is off by its own roundings."""
    import torch
    c = Case([(33, 70), (20, 20)], 3, 3, 64, 128, True)
    c.forward()
    *_, G = c.gradients([c.nq])
    base, total, size = c.lam.clone(), {}, 0.0
    for step in (64.0, -64.0):
        c.lam.copy_(base + step)
        out = c.forward()[:, :3 * 128].double() * c.dout.double()
        total[step] = out.view(-1, 3, 128).sum((0, 2)).cpu().numpy()
        size = max(size, float(out.abs().sum()))
    assert np.all(np.abs((total[64.0] - total[-64.0]) / 128 - G[0]) <= 2 * 2 * HALF * size / 128)


@pytest.mark.gpu
def test_graph_and_streams():
    """Forward and gradients captured, replayed with other inputs and other lengths; and on a side stream."""
    import torch
    c = Case([(40, 80), (25, 30), (1, 400)], 4, 2, 64, 128, True)
    out, dq, dk, dv = c.blank(c.nq, 4 * 128), torch.empty_like(c.q), torch.empty_like(c.k), torch.empty_like(c.v)
    G = torch.empty(2, 4, device="cuda")

    def both():
        api.agc_diff_attn_forward(*c.head, out, c.ws, lse=c.lse)
        api.agc_diff_attn_partial_gradients(*c.head, c.lse, c.dout, [30, c.nq], dq, dk, dv, G, c.ws)

    both()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for turn in range(3):
        c.q.mul_(0.75)
        c.q_end[0] -= turn
        c.k_end[1] -= 2 * turn
        both()
        want = [t.clone() for t in (out, dq, dk, dv, G)]
        for t in (out, dq, dk, dv, G):
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((out, dq, dk, dv, G), want))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for t in (out, dq, dk, dv, G):
        t.zero_()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        both()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip((out, dq, dk, dv, G), want))


@pytest.mark.gpu
def test_thousands_of_sequences():
    """Among five thousand, most of one query and one key, each finds its own."""
    import torch
    rng = np.random.default_rng(3)
    lens = [(int(rng.integers(0, 3)), int(rng.integers(0, 4))) for _ in range(5000)]
    lens[4321], lens[70] = (90, 200), (300, 33)
    c = Case(lens, 2, 1, 32, 64, True)
    c.check_forward(c.forward())
    c.check_gradients(*c.gradients([1000, c.nq]), [1000, c.nq])


@pytest.mark.gpu
@pytest.mark.parametrize("lens,heads,kv_heads,d,e,causal", [
    ([(1100, 1100)] * 12, 8, 8, 32, 64, True), ([(300, 300), (5000, 5000), (0, 0), (700, 700)], 4, 4, 64, 128, True), ([(2000, 2000)] * 2, 32, 16, 64, 128, True),
    ([(2100, 2100)] * 3, 3, 3, 64, 128, True), ([(1500, 1500)] * 4, 8, 8, 128, 256, True),
    ([(1500, 1500), (2600, 2300), (0, 0), (1900, 1950)], 8, 2, 128, 256, False), ([(9000, 900), (5000, 700)], 6, 3, 64, 128, False)])
def test_large_workgroups(lens, heads, kv_heads, d, e, causal):
    """Sizes that take the large workgroups and all orders of tiles, against sequence after sequence by itself, which takes
    small ones: the same formulas with sums cut in other places.  Two results, each off by its own rounding and, out, by
    those of its maps: 2^-8 sqrt(2) of a value in the root mean square at most, half a step being the largest."""
    import torch
    c = Case(lens, heads, kv_heads, d, e, causal)
    out = c.forward()[:, :heads * e]
    parts = [c.nq // 3, c.nq]
    dq, dk, dv, G = c.gradients(parts)
    total = np.zeros(heads)
    i = j = 0
    for lq, lk in lens:
        if lq == 0:
            continue
        one = (c.q[i:i + lq], c.k[j:j + lk], c.v[j:j + lk], heads, kv_heads, c.lam, torch.tensor([lq], dtype=torch.int32, device="cuda"),
               torch.tensor([lk], dtype=torch.int32, device="cuda"), c.scale, causal)
        ws = torch.empty(api.agc_diff_attn_workspace_bytes(lq, lk, 1, heads, kv_heads, d, e, True), dtype=torch.uint8, device="cuda")
        alone, lse = torch.empty_like(out[i:i + lq]), torch.empty(2 * heads, lq, device="cuda")
        api.agc_diff_attn_forward(*one, alone, ws, lse=lse)
        grads = [torch.empty_like(t) for t in one[:3]]
        g = torch.empty(1, heads, device="cuda")
        api.agc_diff_attn_partial_gradients(*one, lse, c.dout[i:i + lq], [lq], *grads, g, ws)
        for got, want in ((out[i:i + lq], alone), (dq[i:i + lq], grads[0]), (dk[j:j + lk], grads[1]), (dv[j:j + lk], grads[2])):
            assert float((got.double() - want.double()).norm() / want.double().norm()) < HALF * 2 ** 0.5
        assert float((c.lse[:, i:i + lq] - lse).abs().max()) < 2.0 ** -16
        total += g[0].double().cpu().numpy()
        i, j = i + lq, j + lk
    # binary32 sums of the same terms
    assert np.all(np.abs(G.sum(0) - total) <= 1e-5 * np.abs(G).sum(0).max())


@pytest.mark.gpu
def test_rows_beyond_four_gigabytes():
    """Keys, values and queries whose rows lie 2 MB apart."""
    import torch
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("needs 40 GB")
    want, got = [], []
    for far in (False, True):
        c = Case([(1, 2100), (500, 300)], 2, 1, 64, 128, True)
        if far:
            wide = torch.empty(2400, 1 << 20, dtype=torch.bfloat16, device="cuda")
            k, v = wide[:, 64:192], wide[:, 4096:4224]
            k.copy_(c.k)
            v.copy_(c.v)
            q = torch.empty(501, 1 << 20, dtype=torch.bfloat16, device="cuda")[:, :256]
            q.copy_(c.q)
            c.head = (q, k, v, *c.head[3:])
        out = c.forward()
        dq, dk, dv, G = c.gradients([c.nq])
        (got if far else want).extend((out, dq, dk, dv, torch.from_numpy(G)))
    assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.gpu
def test_queries_without_keys_get_zeros_whatever_the_values():
    import torch
    for d, e in ((64, 128), (128, 256), (20, 30)):
        c = Case([(40, 12)], 2, 1, d, e, True)
        c.v.fill_(float("nan"))
        out = c.forward()
        assert not out[:28].any() and torch.isnan(out[28:].float()).all()


@pytest.mark.gpu
def test_no_queries_or_no_keys():
    import torch
    c = Case([(0, 50)], 2, 1, 64, 128, True)
    c.forward()
    dq, dk, dv, G = c.gradients([0, 0])
    assert not dk.any() and not dv.any() and not G.any()
    c = Case([(50, 0)], 2, 1, 64, 128, False)
    assert not c.forward().any()
    dq, dk, dv, G = c.gradients([50])
    assert not dq.any() and not G.any()


# ------------------------------------------------------------------ refusals, on the CPU: nothing is dereferenced
def raw(grad=False, q=256, ldq=512, k=256, ldk=256, v=256, ldv=256, nq=3, nk=4, heads=4, kv=2, d=64, e=128, lam=4, qe=4, kb=0, ke=4, n=1, scale=1.0,
        out=256, ldo=512, lse=4, ws=256, dout=256, lddout=512, parts=(3,), dq=2, lddq=512, dk=2, lddk=256, dv=2, lddv=256, G=4, ldg=4):
    import struct
    L = api.load()
    head = (q, ldq, k, ldk, v, ldv, nq, nk, heads, kv, d, e, lam, qe)
    if not grad:
        return L.agc_diff_attn_forward(*head, kb, ke, n, scale, 1, out, ldo, lse, ws, None)
    part = None if parts is None else struct.pack(f"{len(parts)}q", *parts)
    return L.agc_diff_attn_partial_gradients(*head, ke, n, scale, 1, lse, dout, lddout, part, 0 if parts is None else len(parts), dq, lddq, dk, lddk, dv, lddv,
                                             G, ldg, ws, None)


@pytest.mark.parametrize("grad", [False, True])
@pytest.mark.parametrize("change,status", [
    (dict(nq=-1), -2), (dict(nq=2 ** 26 + 1), -2), (dict(nk=-1), -2), (dict(nk=2 ** 26 + 1), -2), (dict(n=0), -2), (dict(n=2 ** 20 + 1), -2),
    (dict(heads=3), -2), (dict(heads=0), -2), (dict(kv=0), -2), (dict(d=0), -2), (dict(d=129), -2), (dict(e=0), -2), (dict(e=257), -2),
    (dict(nq=2 ** 26, heads=32, ldq=4096), -2), (dict(nk=2 ** 26, heads=64, kv=32, ldk=4096, ldv=4096, ldq=8192), -2),
    (dict(nq=2 ** 26, heads=18, ldq=4096), -2), (dict(n=2 ** 19, heads=8, kv=8, ldq=1024, ldk=1024, ldv=1024), -2),
    (dict(n=2 ** 20, heads=32, kv=32, ldq=4096, ldk=4096, ldv=4096), -2), (dict(scale=math.inf), -1), (dict(scale=math.nan), -1),
    (dict(scale=-0.5), -1),
    (dict(q=0), -1), (dict(k=0), -1), (dict(v=0), -1), (dict(lam=0), -1), (dict(qe=0), -1), (dict(ke=0), -1), (dict(ws=0), -1),
    (dict(ldq=2 ** 24 + 8), -2), (dict(ldk=2 ** 24 + 8), -2), (dict(ldv=2 ** 24 + 8), -2), (dict(ldq=504), -2), (dict(ldk=248), -2),
    (dict(ldv=248), -2), (dict(q=258), -4), (dict(k=264), -4), (dict(v=258), -4), (dict(ldq=516), -4),
    (dict(ldk=257), -4), (dict(ldv=260), -4), (dict(q=257, d=60), -4), (dict(lam=6), -4), (dict(qe=2), -4), (dict(ke=2), -4),
    (dict(lse=2), -4), (dict(ws=128), -4)])
def test_refusals(grad, change, status):
    assert raw(grad, **change) == status


@pytest.mark.parametrize("change,status", [(dict(out=0), -1), (dict(ldo=511), -2), (dict(out=257), -4), (dict(kb=2), -4), (dict(nq=0, q=0, out=0), 0)])
def test_refusals_of_the_forward_pass(change, status):
    assert raw(**change) == status


@pytest.mark.parametrize("change,status", [
    (dict(parts=None), -1), (dict(parts=()), -2), (dict(parts=(2,)), -2), (dict(parts=(3, 2)), -2), (dict(parts=(2, 1, 3)), -2),
    (dict(parts=(3,) * 257), -2), (dict(parts=(3,) * 256, heads=2 ** 14, ldq=2 ** 21, lddout=2 ** 21, lddq=2 ** 21, ldg=2 ** 14), -2),
    (dict(dout=0), -1), (dict(lse=0), -1), (dict(dq=0), -1), (dict(dk=0), -1), (dict(dv=0), -1), (dict(G=0), -1), (dict(lddout=504), -2),
    (dict(lddout=2 ** 24 + 8), -2), (dict(lddq=511), -2),
    (dict(lddk=255), -2), (dict(lddv=255), -2), (dict(ldg=3), -2), (dict(dout=258), -4), (dict(lddout=516), -4), (dict(dq=1), -4),
    (dict(dk=1), -4), (dict(dv=1), -4),
    (dict(G=2), -4)])
def test_refusals_of_the_gradients(change, status):
    assert raw(True, **change) == status


def test_binding_refusals():
    import torch
    bf16 = torch.bfloat16
    ok = dict(q=torch.zeros(3, 512, dtype=bf16), k=torch.zeros(4, 256, dtype=bf16), v=torch.zeros(4, 256, dtype=bf16), heads=4, kv_heads=2, lam=torch.zeros(4),
              q_end=torch.zeros(1, dtype=torch.int32), k_end=torch.zeros(1, dtype=torch.int32), scale=1.0, causal=True, out=torch.zeros(3, 512, dtype=bf16),
              workspace=torch.zeros(1 << 20, dtype=torch.uint8), lse=torch.zeros(8, 3))

    def status(**change):
        with pytest.raises(api.AgcError) as e:
            api.agc_diff_attn_forward(**{**ok, **change})
        return e.value.status

    for change in (dict(q=ok["q"].float()), dict(q=ok["q"][:, :-1]), dict(k=ok["k"][:, :128]), dict(v=ok["v"].half()), dict(v=ok["v"][:3]), dict(heads=3), dict(heads=0),
                   dict(lam=ok["lam"][:3]), dict(lam=ok["lam"].double()), dict(q_end=torch.zeros(1, dtype=torch.int64)), dict(k_end=torch.zeros(2, dtype=torch.int32)),
                   dict(lse=torch.zeros(8, 2)), dict(lse=torch.zeros(8, 3, dtype=bf16)), dict(workspace=torch.zeros(16, dtype=torch.uint8))):
        assert status(**change) == api.AGC_ESHAPE, change
    assert status() == api.AGC_EINVAL     # host memory


def test_workspace():
    """Heads that are read where they lie ask for no room to copy; nothing for what is out of range."""
    need = api.agc_diff_attn_workspace_bytes
    assert need(1 << 16, 1 << 16, 8, 16, 4, 64, 128) == 256
    assert need(1 << 16, 1 << 16, 8, 16, 4, 63, 128) > (1 << 16) * 20 * 256
    assert need(1 << 16, 1 << 16, 8, 16, 4, 64, 128, True) == 256 + (1 << 16) * 16 * 16
    # forward and gradients share what splits leave; it does not grow with the keys
    assert need(8, 1 << 24, 8, 16, 4, 64, 128, True) >= need(8, 1 << 24, 8, 16, 4, 64, 128) < 1 << 24
    assert need(1, 1, 0, 1, 1, 1, 1) == 0 and need(1, 1, 1, 3, 2, 1, 1) == 0 and need(1, 1, 1, 1, 1, 129, 1) == 0
