"""What the binding of the token models' operators refuses before anything reaches the GPU, and what it must not refuse."""
import pytest
import torch

from paper_2605_15890_amd import api


def refused(call, *args, **kw):
    with pytest.raises(api.AgcError) as e:
        call(*args, **kw)
    return e.value.status


@pytest.mark.parametrize("which", ["beta", "m1", "ghat", "beta_bf16"])
@pytest.mark.parametrize("dtype", [torch.int32, torch.float16, torch.int16, torch.float64])
def test_vectors_of_another_type(which, dtype):
    vectors = {"beta": torch.zeros(64), "m1": torch.zeros(64), "ghat": torch.zeros(64),
               "beta_bf16": torch.zeros(64, dtype=torch.bfloat16)}
    vectors[which] = torch.zeros(64, dtype=dtype)
    ws = torch.zeros(api.agc_muon_workspace_bytes(8, 8, 1), dtype=torch.uint8)
    assert refused(api.agc_muon_update, vectors["beta"], vectors["m1"], vectors["ghat"], [0], 8, 8, 0.1, 0.9, True, 0.0, 1.0,
                   5, ws, beta_bf16=vectors["beta_bf16"]) == api.AGC_ESHAPE


@pytest.mark.parametrize("dtype", [torch.complex64, torch.float32, torch.float64, torch.int16, torch.bool])
def test_ids_that_are_no_whole_numbers(dtype):
    table, out, ids = torch.zeros(4, 8), torch.zeros(3, 8), torch.zeros(3, dtype=dtype)
    assert refused(api.agc_embed_forward, table, ids, 1.0, out) == api.AGC_ESHAPE
    ws = torch.zeros(api.agc_embed_workspace_bytes(3, 4, 8, 1), dtype=torch.uint8)
    assert refused(api.agc_embed_partial_gradients, out, ids, [3], 4, 1.0, torch.zeros(1, 32), ws) == api.AGC_ESHAPE


@pytest.mark.gpu
def test_strides_of_a_single_row_do_not_matter():
    """One row of each weight, and one partition's gradients, from tensors of different strides."""
    bf16 = torch.bfloat16
    x = torch.randn(70, 16, device="cuda").to(bf16)
    gate, up = torch.randn(1, 16, device="cuda").to(bf16), torch.randn(4, 40, device="cuda").to(bf16)[2:3, :16]
    dh = torch.randn(70, 1, device="cuda").to(bf16)
    ws = torch.empty(api.agc_gated_workspace_bytes(70, 16, 1, 1), dtype=torch.uint8, device="cuda")
    got = []
    for w_up, G_up in ((up, torch.zeros(3, 50, device="cuda")[1:2, :16]), (up.contiguous(), torch.zeros(1, 16, device="cuda"))):
        h, G = torch.zeros(70, 1, dtype=bf16, device="cuda"), torch.zeros(1, 16, device="cuda")
        api.agc_gated_forward(x, gate, w_up, "silu", h, ws)
        api.agc_gated_partial_gradients(x, gate, w_up, "silu", dh, [70], None, G, G_up, ws)
        got.append((h, G, G_up))
    assert all(torch.equal(a, b) for a, b in zip(*got)) and got[0][0].abs().sum() > 0 and got[0][2].abs().sum() > 0


def test_workspace_of_a_forward_pass_of_few_tokens():
    """Up to 64 tokens nothing is laid out; more never need less."""
    sizes = [api.agc_gated_workspace_bytes(n, 1024, 4096) for n in (0, 1, 5, 64, 65, 66, 1000)]
    assert sizes[:4] == [256] * 4 and sizes == sorted(sizes) and sizes[4] > 1 << 20


@pytest.mark.gpu
@pytest.mark.parametrize("tokens", [1, 16, 64])
def test_forward_pass_of_few_tokens_leaves_the_workspace_alone(tokens):
    bf16 = torch.bfloat16
    x, w = torch.randn(tokens, 67, device="cuda").to(bf16), torch.randn(30, 67, device="cuda").to(bf16)
    h, ws = torch.empty(tokens, 30, dtype=bf16, device="cuda"), torch.full((256,), 9, dtype=torch.uint8, device="cuda")
    api.agc_gated_forward(x, w, w, "silu", h, ws)
    assert torch.all(ws == 9) and torch.isfinite(h.float()).all()
