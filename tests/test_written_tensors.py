"""Tensors that a call writes are known to autograd as changed: a later backward through what it saved of them raises, as after
torch's own calls in place.  The binding runs over a library that only takes notes."""
import pytest

import paper_1909_05073_amd as P
from test_gradient_lists import notes                    # noqa: F401  (a fixture)
from test_i8_outputs import notes as layer_notes         # noqa: F401  (a fixture)


@pytest.mark.parametrize("with_out", [False, True])
def test_clipped_gradients_count_as_changed(notes, with_out):     # noqa: F811
    import torch
    grads = [torch.ones(60), torch.ones(30)]
    outs = [torch.zeros(60), torch.zeros(30)] if with_out else None
    plan = P.GradList(grads, outs)
    written, read = (outs, grads) if with_out else (grads, [])
    was = [[t._version for t in ts] for ts in (written, read)]
    plan.norm()
    assert [[t._version for t in ts] for ts in (written, read)] == was
    plan.clip(1.0)
    assert all(t._version > v for t, v in zip(written, was[0])) and [t._version for t in read] == was[1]


def test_a_backward_through_gradients_that_were_clipped_raises(notes):     # noqa: F811
    import torch
    w = torch.ones(5, requires_grad=True)
    grad, = torch.autograd.grad((w ** 3).sum(), w, create_graph=True)
    penalty = (grad * grad).sum()                        # saves grad
    P.clip_grad_norm([grad], 1.0)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        penalty.backward()


def test_gradients_made_in_inference_mode_can_be_clipped(notes):     # noqa: F811
    import torch
    with torch.inference_mode():
        inside = torch.ones(7)
        P.clip_grad_norm([inside], 1.0)
    P.clip_grad_norm([inside, torch.ones(3)], 1.0)
    assert len(notes) == 2


@pytest.mark.parametrize("call", ["linear", "matmul"])
def test_outputs_of_a_layer_count_as_changed(layer_notes, call):     # noqa: F811
    import torch
    w, s, out = torch.zeros(3, 8, dtype=torch.int8), torch.ones(3), torch.zeros(4, 3)
    with torch.inference_mode():
        inside = torch.zeros(4, 3)
    for y in (out, inside):
        was = None if y is inside else y._version
        if call == "linear":
            P.linear_i8(torch.zeros(4, 8), w, s, out=y)
        else:
            P.matmul_i8(torch.zeros(4, 8, dtype=torch.int8), torch.ones(4), w, s, out=y)
        assert was is None or y._version > was
