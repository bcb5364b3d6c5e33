"""Layer norm and its gradient on the GPU against the references in 64 bits (layers_ref.py, with the tolerances)."""
import numpy as np
import pytest
import torch

import layers_ref as R
from layers_ref import BF16, F16, F32, TYPES, check, device_count, f64, in_use, normal, strided
from paper_1905_03381_amd import api

pytestmark = pytest.mark.gpu

# Either side of what a thread, 16 and 64 lanes, 4 and 8 waves hold, and rows that no block holds.
WIDTHS = [1, 2, 7, 8, 9, 65, 127, 128, 129, 255, 256, 257, 511, 512, 513, 1000, 1024, 1025, 2047, 2048, 2049, 4093, 4096, 4097, 8191,
          8192, 8193, 12_287, 12_288, 12_289, 16_384, 16_385, 70_001]


def vectors(d, seed, affine=True):
    if not affine:
        return None, None, np.ones(d), np.zeros(d)
    gamma, beta = 1 + normal((d,), F32, seed, 0.3), normal((d,), F32, seed + 1, 0.2)
    return gamma.cuda(), beta.cuda(), f64(gamma), f64(beta)


def rows(n, d, dtype, seed):
    """Rows of different size and mean."""
    x = normal((n, d), torch.float64, seed) * torch.exp(normal((n, 1), torch.float64, seed + 1))
    return (x + normal((n, 1), torch.float64, seed + 2, 2.0)).to(dtype)


def run_norm(x, gamma, beta, count, eps=1e-5, out=None, statistics=True):
    n, d = x.shape
    out = torch.full((n, d), 77.0, dtype=x.dtype, device="cuda") if out is None else out
    mean = torch.full((n,), 77.0, device="cuda") if statistics else None
    rstd = torch.full((n,), 77.0, device="cuda") if statistics else None
    api.layer_norm(x, gamma, beta, eps, device_count(count), out, mean, rstd)
    return out, mean, rstd


def check_norm(x, gamma, beta, count, got, eps=1e-5):
    m, dtype = in_use(count, x.shape[0]), x.dtype
    x64 = f64(x)[:m]
    want, bounds = R.norm(x64, gamma, beta, eps), R.norm_bounds(x64, gamma, beta, eps, dtype)
    for g, w, b, what in zip(got, want, bounds, ("out", "mean", "rstd")):
        if g is not None:
            check(g[:m], w, b, what)
            assert (f64(g[m:]) == 77.0).all(), what


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d", WIDTHS)
def test_widths(d, dtype):
    x = strided(rows(5, d, dtype, d), d + 3, 1)
    gamma, beta, g64, b64 = vectors(d, d + 50)
    check_norm(x, g64, b64, 4, run_norm(x, gamma, beta, 4))


@pytest.mark.parametrize("n,count", [(1, None), (1, 0), (3, -5), (3, 7), (17, 16), (300, 299), (9000, None)])
@pytest.mark.parametrize("d", [24, 200, 400, 640, 1500, 9000])
def test_rows(n, count, d):
    x = rows(n, d, BF16, n + d).cuda()
    gamma, beta, g64, b64 = vectors(d, 3)
    check_norm(x, g64, b64, count, run_norm(x, gamma, beta, count))


@pytest.mark.parametrize("d", [40, 1030, 20_000])
def test_without_vectors_and_statistics(d):
    x = rows(6, d, F16, 5).cuda()
    out, _, _ = run_norm(x, None, None, None, statistics=False)
    check_norm(x, np.ones(d), np.zeros(d), None, (out, None, None))
    gamma, beta, g64, b64 = vectors(d, 3)
    check_norm(x, g64, np.zeros(d), None, run_norm(x, gamma, None, None))
    check_norm(x, np.ones(d), b64, None, run_norm(x, None, beta, None))


@pytest.mark.parametrize("d", [12, 300, 700, 5000, 20_000])
def test_rows_that_are_not_in_use_may_hold_anything(d):
    n, m = 40, 17
    x, dout, res = (rows(n, d, BF16, 3 + i).cuda() for i in range(3))
    mean, rstd = statistics(x)
    for t in (x, dout, res, mean, rstd):
        t[m:] = float("nan")
    gamma, beta, g64, b64 = vectors(d, 3)
    check_norm(x, g64, b64, m, run_norm(x, gamma, beta, m))
    check_grad(dout, x, g64, mean, rstd, res, m, run_grad(dout, x, gamma, mean, rstd, res, m))


def test_one_workspace_for_all_widths():
    ws = api.LayerWorkspace(12_000)
    for d in (3, 500, 8192, 8193, 12_000):
        x, dout = rows(600, d, BF16, 3).cuda(), normal((600, d), BF16, 4).cuda()
        mean, rstd = statistics(x)
        dx, dgamma, dbeta = torch.zeros_like(x), torch.zeros(d, device="cuda"), torch.zeros(d, device="cuda")
        api.layer_norm_grad(dout, x, None, mean, rstd, None, None, dx, dgamma, dbeta, False, ws)
        check_grad(dout, x, np.ones(d), mean, rstd, None, None, (dx, dgamma, dbeta))


@pytest.mark.parametrize("d", [12, 700, 3000, 20_000])
def test_equal_columns_far_means_and_in_place(d):
    """Rows of one value have only eps; rows far from 0 keep the digits that their differences have."""
    x = normal((5, d), F32, 8)
    x[0], x[1] = 3.7, 0.0
    x[2] += 4096.0
    x[3] *= 1e-18
    x = x.cuda()
    gamma, beta, g64, b64 = vectors(d, 3)
    kept = x.clone()
    got = run_norm(x, gamma, beta, None, out=x)
    check_norm(kept, g64, b64, None, got)


@pytest.mark.parametrize("d", [100, 1500, 20_000])
def test_what_is_not_finite_stays_in_its_row(d):
    x = rows(4, d, F32, 9)
    x[1, d // 2], x[2, 0] = float("nan"), float("inf")
    got = run_norm(x.cuda(), None, None, None)
    out = f64(got[0])
    assert np.isnan(out[1]).all() and np.isnan(out[2]).all()
    for r in (0, 3):
        check_norm(x[r:r + 1].cuda(), np.ones(d), np.zeros(d), None, [g[r:r + 1] for g in got])


def run_grad(dout, x, gamma, mean, rstd, residual, count, sums=(True, True), accumulate=False, dx=None):
    n, d = x.shape
    dx = torch.full((n, d), 77.0, dtype=x.dtype, device="cuda") if dx is None else dx
    dgamma, dbeta = (torch.full((d,), 0.25, device="cuda") if s else None for s in sums)
    api.layer_norm_grad(dout, x, gamma, mean, rstd, residual, device_count(count), dx, dgamma, dbeta, accumulate,
                        api.LayerWorkspace(d) if any(sums) else None)
    return dx, dgamma, dbeta


def statistics(x, eps=1e-5):
    v = x.double()
    return v.mean(1).float(), (v.var(1, unbiased=False) + eps).rsqrt().float()


def check_grad(dout, x, g64, mean, rstd, residual, count, got, accumulate=False):
    m, dtype = in_use(count, x.shape[0]), x.dtype
    res = np.zeros((m, x.shape[1])) if residual is None else f64(residual)[:m]
    args = (f64(dout)[:m], f64(x)[:m], g64, f64(mean)[:m], f64(rstd)[:m], res)
    want, bounds = R.norm_grad(*args), R.norm_grad_bounds(*args, dtype)
    check(got[0][:m], want[0], bounds[0], "dx")
    assert (f64(got[0][m:]) == 77.0).all()
    for g, w, b, what in zip(got[1:], want[1:], bounds[1:], ("dgamma", "dbeta")):
        if g is not None:
            w = w + 0.25 if accumulate else w
            check(g, w, b + R.U32 * (np.abs(w) + 0.25), what)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d", WIDTHS)
def test_grad_widths(d, dtype):
    n = 7
    x, dout = strided(rows(n, d, dtype, d), d + 5, 3), strided(normal((n, d), dtype, d + 9), d + 1, 1)
    residual = strided(normal((n, d), dtype, d + 8), d + 2) if d % 2 else None
    gamma, _, g64, _ = vectors(d, d + 50)
    mean, rstd = statistics(x)
    check_grad(dout, x, g64, mean, rstd, residual, 6, run_grad(dout, x, gamma, mean, rstd, residual, 6))


@pytest.mark.parametrize("n,count", [(1, None), (2, 0), (3, -5), (3, 7), (17, 16), (300, 299), (9000, None)])
@pytest.mark.parametrize("d", [24, 200, 400, 640, 1500, 9000])
@pytest.mark.parametrize("accumulate", [False, True])
def test_grad_rows(n, count, d, accumulate):
    x, dout = rows(n, d, F16, n + d).cuda(), normal((n, d), F16, 4).cuda()
    gamma, _, g64, _ = vectors(d, 3)
    mean, rstd = statistics(x)
    got = run_grad(dout, x, gamma, mean, rstd, None, count, accumulate=accumulate)
    check_grad(dout, x, g64, mean, rstd, None, count, got, accumulate)


@pytest.mark.parametrize("d", [30, 1400, 20_000])
@pytest.mark.parametrize("sums", [(True, False), (False, True), (False, False)])
def test_grad_without(d, sums):
    x, dout = rows(9, d, BF16, 3).cuda(), normal((9, d), BF16, 4).cuda()
    mean, rstd = statistics(x)
    check_grad(dout, x, np.ones(d), mean, rstd, None, None, run_grad(dout, x, None, mean, rstd, None, None, sums))


@pytest.mark.parametrize("d", [30, 1400, 9000, 20_000])
@pytest.mark.parametrize("which", [0, 1, 2])
def test_grad_in_place(d, which):
    x, dout, res = (rows(9, d, BF16, 3 + i).cuda() for i in range(3))
    gamma, _, g64, _ = vectors(d, 3)
    mean, rstd = statistics(x)
    old = [t.clone() for t in (dout, x, res)]
    got = run_grad(dout, x, gamma, mean, rstd, res, None, dx=(dout, x, res)[which])
    check_grad(old[0], old[1], g64, mean, rstd, old[2], None, got)


def test_no_rows():
    d = 300
    x, mean = torch.zeros(0, d, device="cuda"), torch.zeros(0, device="cuda")
    run_norm(x, None, None, None)
    got = run_grad(x, x, None, mean, mean, None, None)
    assert (f64(got[1]) == 0).all() and (f64(got[2]) == 0).all()
    got = run_grad(x, x, None, mean, mean, None, None, accumulate=True)
    assert (f64(got[1]) == 0.25).all()


@pytest.mark.parametrize("d", [40, 900, 5000])
def test_gradient_is_the_differences(d):
    """Along random directions, in 32 bits: the second difference of the norm bounds what the step leaves."""
    n, h = 3, 2.0 ** -5
    x, dx_dir = rows(n, d, F32, 2), normal((n, d), F32, 5, 0.1)
    dout = normal((n, d), F32, 6)
    gamma, beta, g64, b64 = vectors(d, 3)
    mean, rstd = statistics(x.cuda())
    grad = f64(run_grad(dout.cuda(), x.cuda(), gamma, mean, rstd, None, None)[0])
    at = lambda s: (R.norm(f64(x) + s * f64(dx_dir), g64, b64, 1e-5)[0] * f64(dout)).sum(1)
    near, far = (at(h) - at(-h)) / (2 * h), (at(2 * h) - at(-2 * h)) / (4 * h)
    slope = (grad * f64(dx_dir)).sum(1)
    # (the difference's error falls with h^2, so that a third of near - far is most of it; near itself is nearer)
    assert (np.abs(slope - near) <= np.abs(near - far) + 1e-4 * np.abs(grad * f64(dx_dir)).sum(1)).all()


@pytest.mark.parametrize("d", [200, 3000, 8192])
def test_same_bits_and_streams(d):
    n = 2000
    x, dout = rows(n, d, BF16, 3).cuda(), normal((n, d), BF16, 4).cuda()
    gamma, beta, _, _ = vectors(d, 3)
    mean, rstd = statistics(x)
    first = run_norm(x, gamma, beta, None) + run_grad(dout, x, gamma, mean, rstd, dout, None)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        again = run_norm(x, gamma, beta, None) + run_grad(dout, x, gamma, mean, rstd, dout, None)
    side.synchronize()
    for a, b in zip(first, again):
        assert torch.equal(a, b)


def test_captured():
    n, d = 700, 1300
    x, dout = rows(n, d, BF16, 3).cuda(), normal((n, d), BF16, 4).cuda()
    gamma, beta, _, _ = vectors(d, 3)
    count, ws = device_count(n), api.LayerWorkspace(d)
    z = lambda *s, t=F32: torch.zeros(*s, dtype=t, device="cuda")
    out, dx, mean, rstd, dg, db = z(n, d, t=BF16), z(n, d, t=BF16), z(n), z(n), z(d), z(d)

    def step():
        api.layer_norm(x, gamma, beta, 1e-5, count, out, mean, rstd)
        api.layer_norm_grad(dout, x, gamma, mean, rstd, None, count, dx, dg, db, False, ws)

    step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for turn, m in enumerate((n, 13, 0, n)):
        x.copy_(rows(n, d, BF16, 20 + turn))
        count.fill_(m)
        g.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (out, dx, mean, rstd, dg, db)]
        step()
        torch.cuda.synchronize()
        for a, b in zip(got, (out, dx, mean, rstd, dg, db)):
            assert torch.equal(a, b)


def test_far_rows():
    """Rows whose places pass 32 bits."""
    n, d, ld = 5, 600, 1 << 29
    store = torch.zeros((n - 1) * ld + d, dtype=BF16, device="cuda")
    x = store.as_strided((n, d), (ld, 1))
    x.copy_(rows(n, d, BF16, 3))
    check_norm(x, np.ones(d), np.zeros(d), None, run_norm(x, None, None, None))
    mean, rstd = statistics(x)
    dout = normal((n, d), BF16, 4).cuda()
    check_grad(dout, x, np.ones(d), mean, rstd, None, None, run_grad(dout, x, None, mean, rstd, None, None))


@pytest.mark.parametrize("d", [120, 500, 1000, 2000, 5000, 9000])
@pytest.mark.parametrize("n", [2, 4, 5, 16, 32, 33, 128, 129])
def test_turns_of_one_block(n, d):
    """Either side of the rows that a block takes alone."""
    x, dout = rows(n, d, BF16, d).cuda(), normal((n, d), BF16, d + 9).cuda()
    gamma, _, g64, _ = vectors(d, d + 50)
    mean, rstd = statistics(x)
    check_grad(dout, x, g64, mean, rstd, None, n - 1, run_grad(dout, x, gamma, mean, rstd, None, n - 1))
