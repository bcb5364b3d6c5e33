"""ExpertBlock on the GPU: counts and buffers other than the block's own size."""
import pytest
import torch

from paper_1905_03381_amd import api
from paper_1905_03381_amd.boss import ExpertBlock
from test_gpu_experts import BF16, normal

pytestmark = pytest.mark.gpu


def counted(v):
    return torch.tensor([v], dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("n_max", [40, 300])
def test_more_rows_kept_than_the_block_has_room_for(n_max):
    """The block takes its first n_max rows, with the results of a call of exactly those; the rest is left alone."""
    n, E, K, d, f = n_max + 90, 8, 2, 64, 48
    x, dout = normal((n, d), BF16, 3).cuda(), normal((n, d), BF16, 4).cuda()
    got = []
    for rows, count in ((n_max, n_max), (n, n), (n, 1 << 30), (n_max, n)):
        block = ExpertBlock(n_max, d, f, E, K, p=0.2)
        out, dx = torch.full((rows, d), 7.0, dtype=BF16, device="cuda"), torch.full((rows, d), 7.0, dtype=BF16, device="cuda")
        block.forward(x[:rows], counted(count), 9, out)
        block.backward(x[:rows], counted(count), 9, dout[:rows], dx)
        assert (out[n_max:] == 7).all() and (dx[n_max:] == 7).all()
        got.append([out[:n_max], dx[:n_max], block.logits] + block.grads)
    for other in got[1:]:
        for a, b in zip(got[0], other):
            assert torch.equal(a, b)


def test_fewer_rows_than_the_block_are_refused():
    block, x = ExpertBlock(40, 64, 48, 8, 2), torch.zeros(39, 64, dtype=BF16, device="cuda")
    with pytest.raises(api.AAError):
        block.forward(x, counted(39), 0, torch.zeros_like(x))


def test_every_epoch_of_the_experts_workload_draws_anew(capsys, monkeypatch):
    """A row's keep draw comes from its position and the step: a step number that comes again would keep the same rows."""
    from paper_1905_03381_amd import workloads
    steps, call = [], api.score_shrink
    monkeypatch.setattr(api, "score_shrink", lambda *a: (steps.append(a[6:8]), call(*a))[1])
    workloads.main(["experts", "--n", "16384", "--threads", "4"])
    assert len(steps) == 12 and len(set(steps)) == 12, steps


def test_a_missing_workspace_is_refused():
    i32 = dict(dtype=torch.int32, device="cuda")
    ids, plan = torch.zeros(3, 2, **i32), [torch.zeros(5, **i32), torch.zeros(6, **i32), torch.zeros(3, 2, **i32)]
    x, dw = torch.zeros(6, 8, dtype=BF16, device="cuda"), torch.zeros(4, 8, 8, dtype=BF16, device="cuda")
    logits, weights = torch.zeros(3, 4, device="cuda"), torch.zeros(3, 2, device="cuda")
    for call in (lambda: api.expert_plan(ids, None, 4, *plan, None),
                 lambda: api.expert_grad_weight(x, x, None, 1, plan[0], dw, False, None),
                 lambda: api.route(logits, None, None, api.route_config("softmax", 2), ids, weights, plan, None)):
        with pytest.raises(api.AAError):
            call()
