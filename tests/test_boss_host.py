"""ExpertBlock's order of calls and what it hands over, on the CPU, where the library's calls are recorded and not made; and
wrong arguments of the Python calls, which are refused before anything is launched."""
import pytest
import torch

from paper_1905_03381_amd import api
from paper_1905_03381_amd.boss import ExpertBlock

CALLS = ["expert_forward", "route", "expert_combine", "expert_combine_grad", "expert_grad_weight", "expert_grad_input",
         "route_grad", "dropout"]


@pytest.fixture
def made(monkeypatch):
    """Names and arguments of the calls made."""
    calls = []
    monkeypatch.setattr(api, "ExpertWorkspace", lambda *a, **k: None)
    for name in CALLS:
        monkeypatch.setattr(api, name, lambda *a, _name=name: calls.append((_name, a)))
    return calls


def block(n_max=8, **change):
    return ExpertBlock(n_max, 16, 12, 4, 2, device="cpu", **change)


def rows(n, d=16):
    return torch.zeros(n, d, dtype=torch.bfloat16)


@pytest.mark.parametrize("count,rows_of_x,end", [(5, 8, 5), (8, 8, 8), (11, 8, 8), (11, 20, 8), (1 << 30, 64, 8), (0, 8, 0),
                                                 (-4, 20, 0)])
def test_the_routers_group_ends_inside_the_buffers(made, count, rows_of_x, end):
    """The router's product writes as many rows as its group has; its result has n_max."""
    b, x = block(), rows(rows_of_x)
    b.forward(x, torch.tensor([count], dtype=torch.int32), 0, torch.zeros_like(x))
    assert b.one.tolist() == [0, end]
    name, args = made[0]
    assert name == "expert_forward" and args[3] is b.one and args[6] is b.logits and b.logits.shape[0] >= end


def test_backward_needs_the_last_forward_to_have_trained(made):
    """A forward without training takes the buffers: what an earlier one kept is no longer there, and gradients of it
    would mix the two."""
    b, x, count = block(p=0.1), rows(8), torch.tensor([8], dtype=torch.int32)
    out, dx = torch.zeros_like(x), torch.zeros_like(x)
    with pytest.raises(api.AAError):
        b.backward(x, count, 0, x, dx)
    b.forward(x, count, 0, out)
    b.backward(x, count, 0, x, dx)
    b.backward(x, count, 0, x, dx)
    b.forward(x, count, 0, out, train=False)
    made.clear()
    with pytest.raises(api.AAError):
        b.backward(x, count, 0, x, dx)
    assert not made


def wrong(*shape, dtype="bfloat16"):
    return torch.zeros(*shape, dtype=getattr(torch, dtype))


@pytest.mark.parametrize("call", [
    lambda: api.dropout(wrong(4), None, None, 0.1, 0, 0, wrong(4)),
    lambda: api.dropout(wrong(2, 2, 2), None, None, 0.1, 0, 0, wrong(4)),
    lambda: api.dropout(None, None, None, 0.1, 0, 0, wrong(4)),
    lambda: api.expert_combine(wrong(4), wrong(2, 2, dtype="int32"), None, None, None, 0.0, 0, 0, wrong(4)),
    lambda: api.expert_combine(wrong(4, 4), None, None, None, None, 0.0, 0, 0, wrong(4)),
    lambda: api.expert_combine_grad(wrong(4), None, wrong(2, 2, dtype="int32"), None, None, 0.0, 0, 0, wrong(4), None),
    lambda: api.expert_forward(wrong(2, 2), None, 1, None, wrong(1, 2, 2), ["relu"], wrong(2, 2)),
    lambda: api.route(wrong(4), None, None, api.route_config("softmax", 1), None, None),
    lambda: api.route_config(None, 1),
])
def test_wrong_arguments_are_this_librarys_error(call):
    """Tensors of other dimensions, on the host, none at all: AAError, not what Python says about their shapes."""
    with pytest.raises(api.AAError):
        call()
