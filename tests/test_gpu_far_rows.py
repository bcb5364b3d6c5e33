"""Products of rows that lie beyond 32 bits of 16-byte units from the first: 64 GiB and more."""
import pytest
import torch

from paper_1905_03381_amd import api
from test_gpu_experts import BF16, int_dev, normal

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("act,d_in,d_out,gathers", [
    ("none", 512, 136, 60), ("gated", 512, 72, 60), ("none", 64, 136, 60), ("none", 64, 40_000, 200), ("relu", 520, 72, 7)])
def test_gathered_rows_beyond_what_the_pairs_can_say(act, d_in, d_out, gathers):
    """A plan of few pairs may name rows far beyond their number: where those lie is not bounded by the pairs."""
    far, rows = 1 << 27, 257
    store = torch.empty((rows - 1) * far + 1024, dtype=BF16, device="cuda")
    x = store.as_strided((rows, d_in), (far, 1))
    named = [0, 1, 255, 256, 256, 250, 0] + list(range(rows - gathers + 7, rows))
    vals = normal((rows, d_in), BF16, 1).cuda()
    for r in set(named):
        x[r] = vals[r]
    w = normal((1, d_out * (2 if act == "gated" else 1), d_in), BF16, 2, d_in ** -0.5).cuda()
    offsets, order = int_dev([0, len(named)]), int_dev(named)
    got, want = (torch.empty(len(named), d_out, dtype=BF16, device="cuda") for _ in range(2))
    api.expert_forward(x, order, 1, offsets, w, act, got)
    api.expert_forward(vals, order, 1, offsets, w, act, want)
    assert torch.equal(got, want)
    if d_out == 136:
        dout = normal((len(named), d_out), BF16, 3).cuda()
        ws, dw = api.ExpertWorkspace(rows, 1, 1), [torch.empty(1, d_out, d_in, device="cuda") for _ in range(2)]
        api.expert_grad_weight(dout, x, order, 1, offsets, dw[0], False, ws)
        api.expert_grad_weight(dout, vals, order, 1, offsets, dw[1], False, ws)
        assert torch.equal(*dw)
    del store, x
    torch.cuda.empty_cache()
