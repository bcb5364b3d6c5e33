"""The gradient of routing at the ends of its range, against the references in 64 bits (experts_ref.py)."""
import numpy as np
import pytest
import torch

import experts_ref as R
from paper_1905_03381_amd import api
from test_gpu_experts import TYPES, U32, check, f64, half_step, int_dev, normal, tiny

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("near", [-60.0, -88.0, -89.0, -100.0, -300.0, -700.0])
@pytest.mark.parametrize("E,K", [(2, 2), (40, 8), (200, 30)])
def test_renormalised_sigmoid_of_low_logits(E, K, near, dtype):
    """Scores that only 64 bits hold have weights of ordinary size, and so has their gradient.  The bound is that of
    ordinary logits: a weight is rounded to 32 bits once, the sums and products that follow are of 32 bits."""
    n = 9
    x = (normal((n, E), torch.float32, E) * 0.7 + near).to(dtype)
    xs, dw = f64(x), normal((n, K), torch.float32, 9)
    ids = torch.empty(n, K, dtype=torch.int32, device="cuda")
    weights, out = torch.empty(n, K, device="cuda"), torch.empty(n, E, dtype=dtype, device="cuda")
    c = api.route_config("sigmoid", K, renormalise=True, scale=1.5)
    api.route(x.cuda(), None, None, c, ids, weights)
    api.route_grad(x.cuda(), None, c, ids, dw.cuda(), out)
    ids, got = ids.cpu().numpy(), f64(out)
    for t in range(n):
        row = torch.from_numpy(xs[t].copy()).requires_grad_(True)
        w = R.weights_of(row, ids[t].tolist(), "sigmoid", True, 1.5)
        check(f64(weights)[t], w.detach().numpy(), 4 * U32 * w.detach().numpy(), f"weights of row {t}")
        (w * dw[t].double()).sum().backward()
        want = row.grad.numpy()
        assert np.abs(want).max() > 1e-3
        mag = 1.5 * np.abs(dw[t].double().numpy()).sum()
        check(got[t], want, half_step(dtype) * np.abs(want) + 64 * U32 * mag + tiny(dtype), f"row {t}")


@pytest.mark.parametrize("dtype", TYPES)
def test_renormalised_sigmoid_beyond_64_bits(dtype):
    """Scores that 64 bits do not hold are 0, so are their weights, and the gradient with them."""
    x, K = torch.full((3, 8), -800.0, dtype=dtype, device="cuda"), 3
    ids = torch.empty(3, K, dtype=torch.int32, device="cuda")
    weights, out = torch.empty(3, K, device="cuda"), torch.full((3, 8), 7.0, dtype=dtype, device="cuda")
    c = api.route_config("sigmoid", K, renormalise=True)
    api.route(x, None, None, c, ids, weights)
    api.route_grad(x, None, c, ids, normal((3, K), torch.float32, 1).cuda(), out)
    assert (ids.cpu() == torch.arange(K)).all() and (weights == 0).all() and (out == 0).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("kind", ["softmax", "sigmoid"])
@pytest.mark.parametrize("n,E", [(5, 2), (300, 37), (70, 200)])
def test_one_renormalised_choice_has_no_gradient(n, E, kind, dtype):
    """The weight of a single renormalised choice is the scale whatever the logits are: its gradient is 0, exactly."""
    x = (normal((n, E), torch.float32, E) * 3).to(dtype).cuda()
    ids, weights, out = torch.empty(n, 1, dtype=torch.int32, device="cuda"), torch.empty(n, 1, device="cuda"), torch.ones_like(x)
    c = api.route_config(kind, 1, renormalise=True, scale=2.5)
    api.route(x, None, None, c, ids, weights)
    api.route_grad(x, None, c, ids, normal((n, 1), torch.float32, 3).cuda(), out)
    assert (weights == 2.5).all() and (out == 0).all()
