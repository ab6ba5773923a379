"""A small token model trained through the coded step, on one GPU.

    python -m paper_2605_15890_amd.token_model [--steps N]

Tokens pass an embedding and a gated feed-forward block; the loss is half the mean squared distance to what a block with
other (hidden) parameters makes of the same tokens.  Parameters lie in one vector beta = [table | Wg | Wu], and the
gradients of the data partitions are rows of G in the same order (Sec. II-A: g_j = grad L(D_j, beta)):

    ids -> agc_embed_forward -> agc_gated_forward -> loss
        <- agc_embed_partial_gradients <- agc_gated_partial_gradients     (rows of G)
    G -> agc_step -> g_hat -> agc_muon_update on both weights, agc_gd_update on the table
"""
import argparse
import math

import numpy as np
import torch

from . import api


class TokenModel:
    def __init__(self, vocab=512, dim=64, d_ff=192, tokens=2048, workers=8, replication=2, bits=6, seed=0, device="cuda"):
        self.vocab, self.dim, self.d_ff, self.tokens, self.k = vocab, dim, d_ff, tokens, workers
        self.act, self.seed, self.device = "silu", seed, device
        self.half = d_ff * dim
        self.at_table, self.at_gate, self.at_up = 0, vocab * dim, vocab * dim + self.half
        self.d = self.at_up + self.half
        self.rng = np.random.default_rng(seed)
        g = torch.Generator(device=device).manual_seed(seed)
        self.beta, self.hidden = self._parameters(g), self._parameters(g)
        self.m1 = torch.zeros_like(self.beta)
        self.beta_bf16 = self.beta.to(torch.bfloat16)
        self.hidden_bf16 = self.hidden.to(torch.bfloat16)
        self.G = api.padded_rows(self.k, self.d, device)
        # one partition a worker and worker of the cyclic code, of slightly different sizes
        cuts = np.linspace(0, tokens, self.k + 1)[1:-1] + self.rng.integers(-9, 10, self.k - 1)
        self.part_end = [int(c) for c in cuts] + [tokens]
        # the code, and layer-wise scales for its three sections where they are whole blocks
        self.p = np.full(workers, 0.2)
        self.bits = np.full(workers, bits, dtype=np.uint8)
        phi = api.agc_phi_coef_balanced(self.p, int(self.bits.sum()))
        row_ptr, col, val, self.w = api.agc_build_cyclic_code(workers, self.k, replication, self.p, self.bits, phi)
        self.ctx = api.Context(workers, self.k, self.d)
        self.ctx.agc_set_code(row_ptr, col, val)
        if self.at_gate % 256 == 0 and self.half % 256 == 0:
            self.ctx.agc_set_layers([self.at_gate, self.at_up, self.d])
        self.codes, self.scales, self.ghat = self.ctx.alloc_outputs(self.bits, device)
        # activations and workspaces, kept from step to step
        bf16 = torch.bfloat16
        self.x, self.dx = (torch.empty(tokens, dim, dtype=bf16, device=device) for _ in range(2))
        self.h, self.y, self.dh = (torch.empty(tokens, d_ff, dtype=bf16, device=device) for _ in range(3))
        self.scale = math.sqrt(dim)
        sizes = (api.agc_embed_workspace_bytes(tokens, vocab, dim, self.k), api.agc_gated_workspace_bytes(tokens, dim, d_ff, self.k),
                 api.agc_muon_workspace_bytes(d_ff, dim, 2))
        self.workspace = torch.empty(max(sizes), dtype=torch.uint8, device=device)   # the calls follow each other on a stream

    def _parameters(self, g):
        beta = torch.randn(self.d, generator=g, device=self.device)
        beta[:self.at_gate] /= self.scale_of_table()
        beta[self.at_gate:] /= math.sqrt(self.dim)
        return beta

    def scale_of_table(self):
        return math.sqrt(self.dim)

    def table(self, beta):
        return beta[:self.at_gate].view(self.vocab, self.dim)

    def weights(self, beta_bf16):
        return (beta_bf16[self.at_gate:self.at_up].view(self.d_ff, self.dim), beta_bf16[self.at_up:].view(self.d_ff, self.dim))

    def batch(self):
        return torch.from_numpy(self.rng.integers(0, self.vocab, self.tokens)).to(self.device)

    def forward(self, beta, beta_bf16, ids, out):
        api.agc_embed_forward(self.table(beta), ids, self.scale, self.x)
        w_gate, w_up = self.weights(beta_bf16)
        api.agc_gated_forward(self.x, w_gate, w_up, self.act, out, self.workspace)

    def partial_gradients(self, ids):
        """Rows of G, and the loss."""
        self.forward(self.hidden, self.hidden_bf16, ids, self.y)
        self.forward(self.beta, self.beta_bf16, ids, self.h)
        off = self.h.float() - self.y.float()
        self.dh.copy_(off / off.numel())
        w_gate, w_up = self.weights(self.beta_bf16)
        api.agc_gated_partial_gradients(self.x, w_gate, w_up, self.act, self.dh, self.part_end, self.dx,
                                        self.G[:, self.at_gate:self.at_up], self.G[:, self.at_up:], self.workspace)
        api.agc_embed_partial_gradients(self.dx, ids, self.part_end, self.vocab, self.scale, self.G[:, :self.at_gate],
                                        self.workspace)
        return 0.5 * off.square().mean()

    def step(self, t, lr=0.02, lr_table=20.0):
        loss = self.partial_gradients(self.batch())
        mask = (self.rng.random(len(self.p)) >= self.p).astype(np.uint8)
        self.ctx.agc_step(self.G, self.bits, self.w, mask, self.seed, t, self.codes, self.scales, self.ghat)
        api.agc_muon_update(self.beta, self.m1, self.ghat, [self.at_gate, self.at_up], self.d_ff, self.dim, lr, 0.9, True, 0.0,
                            math.sqrt(max(1.0, self.d_ff / self.dim)), 5, self.workspace, beta_bf16=self.beta_bf16)
        api.agc_gd_update(self.beta[:self.at_gate], self.ghat[:self.at_gate], lr_table)
        return loss

    def close(self):
        self.ctx.close()


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=300)
    steps = ap.parse_args().steps
    model = TokenModel()
    for t in range(steps):
        loss = model.step(t, lr=0.02 * (1 - t / steps))
        if t % 20 == 0 or t == steps - 1:
            print(f"step {t:4d}  loss {float(loss):.5f}", flush=True)
    model.close()


if __name__ == "__main__":
    main()
