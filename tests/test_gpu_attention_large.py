"""Differential attention in the large workgroups, every value of every row against the formulas in 64 bits, which run on the GPU
here (and are checked against the oracle of test_gpu_attention.py on the CPU).

Tolerances are those of test_gpu_attention.py, with what sums of n terms may lose: a lane adds up half of a row's powers and of its
D one after the other, a matrix unit's chain has one addition for 16 terms, below n u together for a map's value and as much again
for a product with it.  F becomes 4 (d + e + 32) u (1 + A) + 2 n u, n the longest sequence; lse has n u / 2 log2(e) more.
"""
import numpy as np
import pytest

from test_gpu_attention import HALF, U, Case, reference


def reference_in_torch(q, k, v, lam, scale, causal, dout):
    """As the oracle's `reference`, of float64 tensors of any device."""
    import torch
    (lq, heads, _, d), (lk, kv_heads, e) = q.shape, v.shape
    r = dict(out=q.new_zeros(lq, heads, e), lse=q.new_full((heads, 2, lq), -np.inf), dq=torch.zeros_like(q), dk=torch.zeros_like(k), dv=torch.zeros_like(v),
             share=q.new_zeros(lq, heads))
    r["out_size"], r["A"] = torch.zeros_like(r["out"]), 0.0
    for n in ("dq", "dk", "dv", "share"):
        r[n + "_half"], r[n + "_full"] = torch.zeros_like(r[n]), torch.zeros_like(r[n])
    if lq == 0 or lk == 0:
        return r
    hidden = torch.zeros(lq, lk, dtype=torch.bool, device=q.device)
    if causal:
        hidden = torch.ones_like(hidden).triu(lk - lq + 1)
    for h in range(heads):
        c, P = h // (heads // kv_heads), []
        for m in range(2):
            s = scale * q[:, h, m] @ k[:, c, m].t()
            r["A"] = max(r["A"], float((scale * q[:, h, m].abs() @ k[:, c, m].abs().t()).max()))
            s = s.masked_fill(hidden, -np.inf)
            top = s.amax(1, keepdim=True)
            top = torch.where(top.isinf(), 0, top)
            p = torch.exp(s - top)
            total = p.sum(1, keepdim=True)
            r["lse"][h, m] = ((top + total.log()) / np.log(2))[:, 0]
            P.append(p / torch.where(total > 0, total, 1))
        mixed, size = P[0] - lam[h] * P[1], P[0] + abs(lam[h]) * P[1]
        r["out"][:, h], r["out_size"][:, h] = mixed @ v[:, c], size @ v[:, c].abs()
        dp, dp_size = dout[:, h] @ v[:, c].t(), dout[:, h].abs() @ v[:, c].abs().t()
        r["dv"][:, c] += mixed.t() @ dout[:, h]
        r["dv_half"][:, c] += mixed.abs().t() @ dout[:, h].abs()
        r["dv_full"][:, c] += size.t() @ dout[:, h].abs()
        for m, f in enumerate((1.0, -float(lam[h]))):
            mean, mean_size = (P[m] * dp).sum(1, keepdim=True), (P[m] * dp_size).sum(1, keepdim=True)
            ds, T = f * P[m] * (dp - mean), abs(f) * P[m] * (dp_size + mean_size)
            r["dq"][:, h, m] = scale * ds @ k[:, c, m]
            r["dq_half"][:, h, m], r["dq_full"][:, h, m] = (scale * x @ k[:, c, m].abs() for x in (ds.abs(), T))
            r["dk"][:, c, m] += scale * ds.t() @ q[:, h, m]
            r["dk_half"][:, c, m] += scale * ds.abs().t() @ q[:, h, m].abs()
            r["dk_full"][:, c, m] += scale * T.t() @ q[:, h, m].abs()
            if m == 1:
                r["share"][:, h], r["share_full"][:, h] = -mean[:, 0], mean_size[:, 0]
    return r


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("lq,lk", [(7, 9), (9, 4), (0, 3)])
def test_both_references_are_one(lq, lk, causal):
    import torch
    rng = np.random.default_rng(lq)
    q, k, v, dout = (rng.standard_normal(s) for s in ((lq, 4, 2, 3), (lk, 2, 2, 3), (lk, 2, 5), (lq, 4, 5)))
    lam = np.array([0.3, -0.7, 0.5, 1.2])
    want = reference(q, k, v, lam, 0.6, causal, dout)
    got = reference_in_torch(*(torch.from_numpy(x) for x in (q, k, v, lam)), 0.6, causal, torch.from_numpy(dout))
    assert want.keys() == got.keys()
    for n, w in want.items():
        assert np.allclose(np.asarray(got[n]), w, rtol=1e-12, atol=1e-13), n


class LargeCase(Case):
    def __init__(self, *args, **kw):
        super().__init__(*args, **kw)
        assert self.takes_large_workgroups()

    def takes_large_workgroups(self):
        """In all three passes: as many rows a sequence as a workgroup has, and 192 workgroups."""
        D = 32 if self.d <= 32 and self.e <= 64 else 64 if self.d <= 64 and self.e <= 128 else 128
        wide = 128 if D == 128 else 256
        rows, n = self.nq * (self.heads // self.kv_heads), len(self.lens)
        return all(have // n >= own and have // own * self.kv_heads >= 192 for have, own in ((rows, wide), (rows, 128), (self.nk, wide)))

    def references(self, gradients=True):
        i = j = 0
        self.most = max(max(self.lq), max(self.lk))
        if not hasattr(self, "answers"):
            self.answers = []
            for lq, lk in self.lens:
                r = reference_in_torch(self.q[i:i + lq].double().reshape(lq, self.heads, 2, self.d), self.k[j:j + lk].double().reshape(lk, self.kv_heads, 2, self.d),
                                       self.v[j:j + lk].double().reshape(lk, self.kv_heads, self.e), self.lam.double(), self.scale, self.causal,
                                       self.dout[i:i + lq].double().reshape(lq, self.heads, self.e))
                self.answers.append((slice(i, i + lq), slice(j, j + lk), {n: x if n == "A" else x.cpu().numpy() for n, x in r.items()}))
                i, j = i + lq, j + lk
        yield from self.answers

    def full(self, r):
        return super().full(r) + 2 * self.most * U

    def check_forward(self, out):
        self.untouched(out, self.heads * self.e, sum(self.lq))
        got = out[:, :self.heads * self.e].double().cpu().numpy().reshape(self.nq, self.heads, self.e)
        lse = self.lse.double().cpu().numpy().reshape(self.heads, 2, self.nq)
        for at, _, r in self.references():
            tol = HALF * np.abs(r["out"]) + (HALF + self.full(r)) * r["out_size"]
            assert np.all(np.abs(got[at] - r["out"]) <= tol), np.max(np.abs(got[at] - r["out"]) / np.maximum(tol, 1e-30))
            mine, empty = lse[:, :, at], np.isinf(r["lse"])
            assert np.array_equal(np.isneginf(mine), empty)
            assert np.all(np.abs(np.where(empty, 0, mine) - np.where(empty, 0, r["lse"])) <= ((self.d + 8) * r["A"] + self.most / 2) * U * 1.45 + 2.0 ** -20)
        assert np.all(lse[:, :, sum(self.lq):] == 7.0)


RAGGED = [(1300, 1300), (2001, 1999), (0, 0), (1011, 1111), (2000, 2055)]


@pytest.mark.gpu
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("lens,heads,kv_heads,d,e,gap", [
    # the kernels' own widths
    (RAGGED, 8, 8, 32, 64, 0), (RAGGED, 16, 8, 64, 128, 8), (RAGGED, 8, 8, 128, 256, 0),
    # filled up on the way to LDS
    (RAGGED, 8, 8, 24, 40, 0), (RAGGED, 8, 8, 40, 72, 0), (RAGGED, 16, 8, 40, 72, 8), (RAGGED, 8, 8, 80, 160, 0), (RAGGED, 16, 8, 96, 192, 16), (RAGGED, 8, 8, 8, 248, 0),
    # copied: odd widths, values alone, rows that begin anywhere
    (RAGGED, 8, 8, 39, 71, 0), (RAGGED, 8, 8, 64, 100, 8), (RAGGED, 8, 8, 80, 160, 1),
    # key heads that do not go round the XCDs, one long sequence, queries and keys of very different lengths
    ([(3200, 3200)] * 4, 6, 6, 40, 72, 0), ([(8300, 8300)], 6, 6, 32, 64, 0), ([(4000, 7000), (4000, 700), (600, 800)], 6, 6, 64, 128, 0)])
def test_every_row(lens, heads, kv_heads, d, e, gap, causal):
    c = LargeCase(lens, heads, kv_heads, d, e, causal, gap=gap, behind=3)
    c.check_forward(c.forward())
    parts = [c.nq // 3, c.nq - 70, c.nq]
    c.check_gradients(*c.gradients(parts), parts)
