"""A small token model trained through the coded step, on one GPU.

    python -m paper_2605_15890_amd.token_model [--steps N] [--heads H]

Tokens pass an embedding and a gated feed-forward block; the loss is half the mean squared distance to what a block with
other (hidden) parameters makes of the same tokens.  Parameters lie in one vector beta = [table | Wg | Wu], and the
gradients of the data partitions are rows of G in the same order (Sec. II-A: g_j = grad L(D_j, beta)):

    ids -> agc_embed_forward -> agc_gated_forward -> loss
        <- agc_embed_partial_gradients <- agc_gated_partial_gradients     (rows of G)
    G -> agc_step -> g_hat -> agc_muon_update on both weights, agc_gd_update on the table

With heads the tokens see those before them in their sequence: the table's rows hold a token's queries, keys and values,

    ids -> agc_embed_forward -> agc_rotary_apply on queries and keys -> agc_diff_attn_forward -> agc_dropout onto the values
        <- agc_rotary_apply back <- agc_diff_attn_partial_gradients <- agc_dropout <-        (a row of G holds lambda's too)

and the block reads the sum.  beta = [table | Wg | Wu | lambda] then, and partitions are whole sequences.
"""
import argparse
import math

import numpy as np
import torch

from . import api


class TokenModel:
    def __init__(self, vocab=512, dim=64, d_ff=192, tokens=2048, workers=8, replication=2, bits=6, seed=0, device="cuda",
                 heads=0, seq_len=64, dropout=0.1):
        self.vocab, self.dim, self.d_ff, self.tokens, self.k = vocab, dim, d_ff, tokens, workers
        self.heads, self.dropout = heads, dropout
        # a token's row of the table: dim values, or queries and keys of both maps of each head, half as wide, and dim values
        self.head_dim = dim // heads // 2 if heads else 0
        self.wide = 4 * heads * self.head_dim + dim
        self.act, self.seed, self.device = "silu", seed, device
        self.half = d_ff * dim
        self.at_table, self.at_gate, self.at_up = 0, vocab * self.wide, vocab * self.wide + self.half
        self.at_lambda = self.at_up + self.half
        self.d = self.at_lambda + heads
        self.rng = np.random.default_rng(seed)
        g = torch.Generator(device=device).manual_seed(seed)
        self.beta, self.hidden = self._parameters(g), self._parameters(g)
        self.m1 = torch.zeros_like(self.beta)
        self.beta_bf16 = self.beta.to(torch.bfloat16)
        self.hidden_bf16 = self.hidden.to(torch.bfloat16)
        self.G = api.padded_rows(self.k, self.d, device)
        # one partition a worker and worker of the cyclic code, of slightly different sizes
        cuts = np.linspace(0, tokens, self.k + 1)[1:-1] + self.rng.integers(-9, 10, self.k - 1)
        self.part_end = [int(c) // seq_len * seq_len if heads else int(c) for c in cuts] + [tokens]
        # the code, and layer-wise scales for its three sections where they are whole blocks
        self.p = np.full(workers, 0.2)
        self.bits = np.full(workers, bits, dtype=np.uint8)
        phi = api.agc_phi_coef_balanced(self.p, int(self.bits.sum()))
        row_ptr, col, val, self.w = api.agc_build_cyclic_code(workers, self.k, replication, self.p, self.bits, phi)
        self.ctx = api.Context(workers, self.k, self.d)
        self.ctx.agc_set_code(row_ptr, col, val)
        if self.at_gate % 256 == 0 and self.half % 256 == 0:
            self.ctx.agc_set_layers([self.at_gate, self.at_up, self.at_lambda] + ([self.d] if heads else []))
        self.codes, self.scales, self.ghat = self.ctx.alloc_outputs(self.bits, device)
        # activations and workspaces, kept from step to step
        bf16 = torch.bfloat16
        self.x, self.dx = (torch.empty(tokens, dim, dtype=bf16, device=device) for _ in range(2))
        self.rows, self.drows = (self.x, self.dx) if not heads else (torch.empty(tokens, self.wide, dtype=bf16, device=device) for _ in range(2))
        self.h, self.y, self.dh = (torch.empty(tokens, d_ff, dtype=bf16, device=device) for _ in range(3))
        self.scale = math.sqrt(dim)
        sizes = [api.agc_embed_workspace_bytes(tokens, vocab, self.wide, self.k), api.agc_gated_workspace_bytes(tokens, dim, d_ff, self.k),
                 api.agc_muon_workspace_bytes(d_ff, dim, 2)]
        if heads:
            turns, _ = api.agc_rotary_frequencies(self.head_dim, base=100.0)
            self.turns = torch.from_numpy(turns).to(device)
            at = torch.arange(tokens, device=device)
            self.positions = (at % seq_len).to(torch.int32)
            self.seq_end = (at[::seq_len] + seq_len).clamp_(max=tokens).to(torch.int32)
            self.lse = torch.empty(2 * heads, tokens, device=device)
            self.attn, self.dattn = (torch.empty(tokens, dim, dtype=bf16, device=device) for _ in range(2))
            sizes.append(api.agc_diff_attn_workspace_bytes(tokens, tokens, len(self.seq_end), heads, heads, self.head_dim,
                                                           dim // heads, True))
        self.workspace = torch.empty(max(sizes), dtype=torch.uint8, device=device)   # the calls follow each other on a stream

    def _parameters(self, g):
        beta = torch.randn(self.d, generator=g, device=self.device)
        beta[:self.at_gate] /= self.scale_of_table()
        beta[self.at_gate:] /= math.sqrt(self.dim)
        if self.heads:
            beta[self.at_lambda:] = 0.5 + 0.2 * torch.randn(self.heads, generator=g, device=self.device)
        return beta

    def scale_of_table(self):
        return math.sqrt(self.dim)

    def table(self, beta):
        return beta[:self.at_gate].view(self.vocab, self.wide)

    def weights(self, beta_bf16):
        return (beta_bf16[self.at_gate:self.at_up].view(self.d_ff, self.dim), beta_bf16[self.at_up:self.at_lambda].view(self.d_ff, self.dim))

    def parts_of(self, rows):
        """Queries, keys and values of the rows, and the queries and keys as one."""
        n = 2 * self.heads * self.head_dim
        return rows[:, :n], rows[:, n:2 * n], rows[:, 2 * n:], rows[:, :2 * n]

    def maps(self, beta):
        """What both attention calls take behind q, k and v."""
        return self.heads, self.heads, beta[self.at_lambda:], self.seq_end, self.seq_end, self.head_dim ** -0.5, True

    def batch(self):
        return torch.from_numpy(self.rng.integers(0, self.vocab, self.tokens)).to(self.device)

    def forward(self, beta, beta_bf16, ids, out, t=0, p=0.0):
        api.agc_embed_forward(self.table(beta), ids, self.scale, self.rows)
        if self.heads:
            q, k, v, both = self.parts_of(self.rows)
            api.agc_rotary_apply(both, 4 * self.heads, self.positions, self.turns, "half", both)
            api.agc_diff_attn_forward(q, k, v, *self.maps(beta), self.attn, self.workspace, lse=self.lse)
            api.agc_dropout(self.attn, p, self.seed, t, 0, self.x, residual=v)
        w_gate, w_up = self.weights(beta_bf16)
        api.agc_gated_forward(self.x, w_gate, w_up, self.act, out, self.workspace)

    def partial_gradients(self, ids, t=0):
        """Rows of G, and the loss."""
        self.forward(self.hidden, self.hidden_bf16, ids, self.y)
        self.forward(self.beta, self.beta_bf16, ids, self.h, t, self.dropout)
        off = self.h.float() - self.y.float()
        self.dh.copy_(off / off.numel())
        w_gate, w_up = self.weights(self.beta_bf16)
        api.agc_gated_partial_gradients(self.x, w_gate, w_up, self.act, self.dh, self.part_end, self.dx,
                                        self.G[:, self.at_gate:self.at_up], self.G[:, self.at_up:self.at_lambda], self.workspace)
        if self.heads:
            q, k, v, _ = self.parts_of(self.rows)
            dq, dk, dv, dboth = self.parts_of(self.drows)
            api.agc_dropout(self.dx, self.dropout, self.seed, t, 0, self.dattn)
            api.agc_diff_attn_partial_gradients(q, k, v, *self.maps(self.beta), self.lse, self.dattn, self.part_end, dq, dk, dv,
                                                self.G[:, self.at_lambda:], self.workspace)
            api.agc_rotary_apply(dboth, 4 * self.heads, self.positions, self.turns, "half", dboth, inverse=True)
            dv.add_(self.dx)
        api.agc_embed_partial_gradients(self.drows, ids, self.part_end, self.vocab, self.scale, self.G[:, :self.at_gate],
                                        self.workspace)
        return 0.5 * off.square().mean()

    def step(self, t, lr=0.02, lr_table=20.0, lr_lambda=20.0):
        loss = self.partial_gradients(self.batch(), t)
        mask = (self.rng.random(len(self.p)) >= self.p).astype(np.uint8)
        self.ctx.agc_step(self.G, self.bits, self.w, mask, self.seed, t, self.codes, self.scales, self.ghat)
        api.agc_muon_update(self.beta, self.m1, self.ghat, [self.at_gate, self.at_up], self.d_ff, self.dim, lr, 0.9, True, 0.0,
                            math.sqrt(max(1.0, self.d_ff / self.dim)), 5, self.workspace, beta_bf16=self.beta_bf16)
        api.agc_gd_update(self.beta[:self.at_gate], self.ghat[:self.at_gate], lr_table)
        if self.heads:
            api.agc_gd_update(self.beta[self.at_lambda:], self.ghat[self.at_lambda:], lr_lambda)
        return loss

    def close(self):
        self.ctx.close()


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=300)
    ap.add_argument("--heads", type=int, default=0)
    args = ap.parse_args()
    steps = args.steps
    model = TokenModel(heads=args.heads)
    for t in range(steps):
        loss = model.step(t, lr=0.02 * (1 - t / steps))
        if t % 20 == 0 or t == steps - 1:
            print(f"step {t:4d}  loss {float(loss):.5f}", flush=True)
    model.close()


if __name__ == "__main__":
    main()
