"""The operators together: a small token model trained through the coded step."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


def test_rows_of_G_add_up_to_the_gradient():
    """The partitions' rows add up to the gradient of the whole batch's loss, which autograd forms in 64 bits from the
    parameters as the block sees them.  Rounding to bfloat16 on the way (x, h, dh, and da, du, dx for the table) is off by
    up to 2^-8 each, as often up as down: 2^-8 of the weights' gradients, 2^-7 of the table's, against 64 bits."""
    import torch
    from paper_2605_15890_amd.token_model import TokenModel
    model = TokenModel()
    ids = model.batch()
    model.partial_gradients(ids)
    got = model.G.double().sum(0)
    beta = model.beta.double()
    beta[model.at_gate:] = model.beta_bf16[model.at_gate:].double()
    beta.requires_grad_(True)
    x = beta[:model.at_gate].view(model.vocab, model.dim)[ids] * model.scale
    a = x @ beta[model.at_gate:model.at_up].view(model.d_ff, model.dim).t()
    u = x @ beta[model.at_up:].view(model.d_ff, model.dim).t()
    h = a * torch.sigmoid(a) * u
    (h * model.dh.double()).sum().backward()
    want = beta.grad
    for name, at, end, tol in (("table", 0, model.at_gate, 2.0 ** -7), ("gate", model.at_gate, model.at_up, 2.0 ** -8),
                               ("up", model.at_up, model.d, 2.0 ** -8)):
        off = float((got[at:end] - want[at:end]).norm() / want[at:end].norm())
        assert off < tol, (name, off)
    model.close()


def test_training_lowers_the_loss():
    from paper_2605_15890_amd.token_model import TokenModel
    model = TokenModel()
    losses = [float(model.step(t)) for t in range(120)]
    assert np.mean(losses[-10:]) < 0.5 * np.mean(losses[:5]), (losses[:5], losses[-10:])
    model.close()
