"""Gates and their gradients as the binding takes them: shapes alone, no kernel is launched."""
import pytest
import torch

from paper_2406_02913_amd import szo


class OnDevice(torch.Tensor):
    """A host tensor that says it is on the device."""
    is_cuda = True


def device(*shape, dtype=torch.float32):
    return torch.zeros(*shape, dtype=dtype).as_subclass(OnDevice)


def desc(T, gate, H=64):
    return szo.make_block_desc(device(T, H), device(T, H), gate=gate)


def test_a_gate_that_is_expanded_over_tokens_has_the_gradient_of_a_row():
    """It is one row for the library, which writes one row of sums: a gradient for each token would be left unwritten but for its first row."""
    d = desc(5, device(64).expand(5, 64))
    assert d.gate_stride == 0
    for wrong in (device(5, 64), device(5, 64)[:, :], device(64).expand(5, 64)):
        with pytest.raises(ValueError):
            szo.make_block_grads(d, gate_grad=wrong)
    g = szo.make_block_grads(d, gate_grad=device(64))
    assert g.gate_grad and g.gate_stride == 0


def test_other_gates_have_gradients_of_their_own_shape():
    for T, gate, right, wrong in ((5, device(64), device(64), device(5, 64)), (5, device(5, 64), device(5, 64), device(64)), (1, device(1, 64), device(1, 64), device(64)),
                                  (1, device(64)[None], device(1, 64), device(64)), (5, device(5, 80)[:, :64], device(5, 72)[:, :64], device(64))):
        d = desc(T, gate)
        assert szo.make_block_grads(d, gate_grad=right).gate_grad
        with pytest.raises(ValueError):
            szo.make_block_grads(d, gate_grad=wrong)
    with pytest.raises(ValueError):
        szo.make_block_grads(desc(5, None), gate_grad=device(64))


@pytest.mark.gpu
def test_an_expanded_gate_gives_what_the_row_does():
    torch.manual_seed(1)
    y, h, gx = (torch.randn(37, 192, device="cuda") for _ in range(3))
    row = torch.randn(192, device="cuda")
    sums = []
    for gate in (row, row.expand(37, 192)):
        d = szo.make_block_desc(y, h, gate=gate, x_type=torch.float32)
        by_gate, by_y = torch.full((192,), 7.0, device="cuda"), torch.empty_like(y)
        szo.szo_block_norm_bwd(d, szo.make_block_grads(d, gx, y_grad=by_y, gate_grad=by_gate), torch.empty(szo.szo_block_workspace_bytes(d), dtype=torch.uint8, device="cuda"))
        sums.append((by_gate, by_y))
    assert torch.equal(sums[0][0], sums[1][0]) and torch.equal(sums[0][1], sums[1][1])
