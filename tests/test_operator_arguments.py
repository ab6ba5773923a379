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
