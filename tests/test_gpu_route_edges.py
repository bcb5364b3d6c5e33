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


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("high,low", [(0.5, None), (0.5, -10_000.0), (float("inf"), 0.25), (300.0, -500.0)])
@pytest.mark.parametrize("E,K", [(6, 2), (40, 5), (200, 9), (300, 20)])
def test_renormalised_softmax_of_choices_without_a_score(E, K, high, low, dtype):
    """A bias may choose masked experts alone: their scores are 0 beside the row's others, in 64 bits, so are their weights
    (there is nothing to divide by), and the gradient of those is 0.  low None: the type's lowest value."""
    if low is None:
        low = torch.finfo(dtype).min
    x = torch.full((4, E), low, dtype=dtype)
    x[:, ::3] = high
    x[0] = low                               # all alike: K equal weights, whose gradients are not 0
    x[2, 1] = high                           # one of the choices has a score
    bias = torch.zeros(E)
    bias[[e for e in range(E) if e % 3][:K]] = 3.0
    ids = torch.empty(4, K, dtype=torch.int32, device="cuda")
    weights, out = torch.empty(4, K, device="cuda"), torch.full((4, E), 7.0, dtype=dtype, device="cuda")
    c, dw = api.route_config("softmax", K, renormalise=True), normal((4, K), torch.float32, 5)
    api.route(x.cuda(), None, bias.cuda(), c, ids, weights)
    api.route_grad(x.cuda(), None, c, ids, dw.cuda(), out)
    ids, weights, got = ids.cpu().numpy(), f64(weights), f64(out)
    for t in range(4):
        want_ids, want_weights = R.choose(f64(x)[t], "softmax", K, bias.numpy(), renorm=True)
        assert ids[t].tolist() == want_ids
        check(weights[t], np.array(want_weights), 4 * U32, f"weights of row {t}")
    assert (weights[[1, 3]] == 0).all() and (got[[1, 3]] == 0).all()
    want = np.zeros(E)
    want[ids[0]] = (dw[0].double().numpy() - dw[0].double().mean().item()) / K
    mag = np.abs(dw[0].double().numpy()).sum()
    check(got[0], want, half_step(dtype) * np.abs(want) + 64 * U32 * mag + tiny(dtype), "row 0")
    assert (weights[2] > 0).sum() == 1 and (np.abs(got[2]) <= 64 * U32 * np.abs(dw[2].numpy()).sum()).all()
