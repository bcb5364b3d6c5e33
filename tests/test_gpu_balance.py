"""Balance loss of a router, the experts' choices and shares, and the gradient, on the GPU against the references in 64
bits.

Tolerances.  A score is an exponential of a difference v (exact to a rounding of v: relative |v| U) by the hardware's
exp2 of v log2 e (another |v| U for that product, and 2 U), and what follows it: a sum over E, a division: a share is
off by at most (2 |v| + E / 8 + 12) U of itself (64 lanes' sums of E / 64 terms and 6 steps: at most E / 8 + 6
roundings), where below |v| < 104 for what 32 bits hold; smaller scores are 0 or off by 2^-126.  The losses and sums over
m rows add m + 64 roundings of the sum's magnitude."""
import numpy as np
import pytest
import torch

import layers_ref as R
from layers_ref import BF16, F16, F32, TYPES, U32, check, device_count, f64, half_step, in_use, normal, strided, tiny
from paper_1905_03381_amd import api

pytestmark = pytest.mark.gpu

KINDS = ["softmax", "sigmoid"]
# Experts of 16 lanes (1, 2, 4, 8 a lane) and of a wave (1 to 16), and sizes between.
EXPERTS = [1, 2, 5, 16, 17, 32, 60, 64, 100, 128, 129, 200, 256, 300, 512, 1000, 1024]


def case(n, E, K, dtype, seed, masked=True):
    x = normal((n, E), torch.float64, seed, 1.5) + normal((E,), torch.float64, seed + 1, 0.5)
    if masked and n > 2:
        g = torch.Generator().manual_seed(seed)
        x[torch.rand(n, E, generator=g) < 0.1] = -float("inf")
        x[1] = -float("inf")
    x = x.to(dtype)
    top, ids = torch.topk(x.double(), K, dim=1)
    ids = torch.where(top > -float("inf"), ids, -1).to(torch.int32)
    return x, ids.contiguous()


def run(x, ids, kind, count, coef=0.02, z_coef=0.003):
    E, K = x.shape[1], ids.shape[1]
    counts = torch.full((E,), -3, dtype=torch.int32, device="cuda")
    share, loss = torch.full((E,), 9.0, device="cuda"), torch.full((2,), 9.0, device="cuda")
    api.balance(x, device_count(count), api.route_config(kind, K), ids, coef, z_coef, counts, share, loss,
                api.LayerWorkspace(E))
    return counts, share, loss


def relative(x):
    """Of a share, in units of U."""
    with np.errstate(invalid="ignore"):
        v = np.where(np.isfinite(x), np.abs(x), 0.0)
    return 4 * v.max(initial=0.0) + x.shape[1] / 8 + 12  # (|x - top| <= 2 max |x|)


def check_balance(x, ids, kind, count, got, coef=0.02, z_coef=0.003):
    m = in_use(count, x.shape[0])
    x64, i = f64(x)[:m], ids.cpu().numpy()[:m]
    counts, share, loss = R.balance(x64, kind, i, coef, z_coef)
    assert (got[0].cpu().numpy() == counts).all()
    rel = (relative(x64) + m + 64) * U32
    check(got[1], share, rel * share + 2.0 ** -120, "share")
    # (log sum exp: its sum's relative error, and a rounding of the result)
    lse = R.shares(x64, kind)[2] if m else np.zeros(1)
    of_z = 2 * np.abs(lse) * U32 * (relative(x64) + np.abs(lse) * 4) + U32 * (m + 64) * lse ** 2
    check(got[2], loss, [rel * loss[0] + 2.0 ** -120, z_coef * of_z.mean() + 2.0 ** -120], "loss")


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("E", EXPERTS)
def test_experts(E, kind):
    K = min(E, 3)
    for dtype in TYPES:
        x, ids = case(37, E, K, dtype, E)
        x, ids = strided(x, E + 3, 1), ids.cuda()
        check_balance(x, ids, kind, 35, run(x, ids, kind, 35))


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("n,count", [(0, None), (1, None), (4, 0), (4, -2), (4, 9), (700, 650), (30_000, None)])
@pytest.mark.parametrize("E,K", [(8, 8), (64, 6), (256, 20), (1024, 64)])
def test_rows(n, count, E, K, kind):
    if n * E > 1 << 23:
        n = (1 << 23) // E
    x, ids = case(n, E, K, BF16, 5)
    x, ids = x.cuda(), ids.cuda()
    check_balance(x, ids, kind, count, run(x, ids, kind, count))


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("n", [15, 32, 33, 64, 65, 128, 129, 256, 257])
@pytest.mark.parametrize("E,K", [(8, 2), (64, 6), (200, 8), (700, 9)])
def test_turns_of_one_block(n, E, K, kind):
    """Either side of the rows that a block takes alone."""
    x, ids = case(n, E, K, F32, n)
    x, ids = x.cuda(), ids.cuda()
    check_balance(x, ids, kind, n - 1, run(x, ids, kind, n - 1))


@pytest.mark.parametrize("n", [60, 3000])
def test_counts_alone_and_rows_that_are_not_in_use(n):
    x, ids = case(n, 64, 4, BF16, 7)
    x, ids, m = x.cuda(), ids.cuda(), n // 2
    want = run(x, ids, "sigmoid", m)
    x[m:], ids[m:] = float("nan"), 5
    counts = torch.zeros(64, dtype=torch.int32, device="cuda")
    api.balance(x, device_count(m), api.route_config("sigmoid", 4), ids, 0.02, 0.003, counts, None, None, api.LayerWorkspace(64))
    assert torch.equal(counts, want[0])
    for a, b in zip(run(x, ids, "sigmoid", m), want):
        assert torch.equal(a, b)


def test_ids_outside_are_no_choices():
    x, ids = case(50, 16, 4, F32, 7)
    ids[3, 1], ids[4, 0], ids[5, 2] = 16, -9, 2 ** 31 - 1
    x, ids = x.cuda(), ids.cuda()
    check_balance(x, ids, "softmax", None, run(x, ids, "softmax", None))


@pytest.mark.parametrize("kind", KINDS)
def test_logits_that_are_not_finite_or_far(kind):
    inf, nan = float("inf"), float("nan")
    x = torch.zeros(8, 5)
    x[0] = torch.tensor([inf, 1.0, inf, -inf, 2.0])
    x[1] = torch.tensor([nan, 1.0, 2.0, -inf, 0.5])
    x[2] = torch.tensor([-inf] * 5)
    x[3] = torch.tensor([nan] * 5)
    x[4] = torch.tensor([-3e38, -3e38, 0.0, 1.0, 2.0])
    x[5] = torch.tensor([80.0, -80.0, 3.0, 0.0, 1.0])
    x[6] = torch.tensor([-90.0, -91.0, -92.0, -95.0, -inf])
    x[7] = torch.tensor([3e38, 0.0, 1.0, 2.0, 3.0])
    ids = torch.zeros(8, 2, dtype=torch.int32)
    x[4], x[7] = x[1], x[1]  # (lse^2 of what is far is beyond 32 bits: taken below)
    got = run(x.cuda(), ids.cuda(), kind, None)
    check_balance(x, ids, kind, None, got)
    counts = torch.tensor([7, 2, 0, 3, 4], dtype=torch.int32, device="cuda")
    out = torch.full((8, 5), 9.0, device="cuda")
    api.balance_grad(x.cuda(), None, api.route_config(kind, 2), None, None, counts, 0.02, 0.003, None, out)
    x64 = f64(x)
    want = R.balance_grad(x64, kind, f64(counts), 2, 0.02, 0.003)
    check(out, want, 400 * U32 * (np.abs(want) + 0.02 * 5 * 8 / 128 * R.shares(x64, kind)[0]) + 1e-30, "dlogits")
    assert np.isfinite(f64(out)).all()


def grad_bound(x, kind, counts, top_k, coef, z_coef, up, dtype, want):
    m, E = x.shape
    p, q, lse, rest = R.shares(x, kind)
    c = counts - counts.mean()
    rel = (relative(x) + 8) * U32
    size = coef * E / (m * m * top_k) * p * rest * (2 * np.abs(c) + 3 * (p * np.abs(c)).sum(1, keepdims=True))
    z = 2 * z_coef / m * q * (np.abs(lse)[:, None] * 6 + relative(x))
    b = abs(up) * (2 * rel * size + (rel * 2 * z_coef / m * q * np.abs(lse)[:, None] + U32 * z))
    return b + half_step(dtype) * (np.abs(want) + b) + tiny(dtype)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("E", EXPERTS)
def test_grad_experts(E, kind):
    K = min(E, 3)
    for dtype in TYPES:
        x, ids = case(9, E, K, dtype, E)
        x = strided(x, E + 3, 1)
        m = 8
        counts = torch.from_numpy(R.choices(ids.numpy()[:m], E).astype(np.int32)).cuda()
        out = strided(torch.full((9, E), 7.0, dtype=dtype), E + 1, 2)
        up = torch.tensor([1.5], device="cuda")
        api.balance_grad(x, device_count(m), api.route_config(kind, K), None, None, counts, 0.5, 0.25, up, out)
        x64 = f64(x)[:m]
        want = R.balance_grad(x64, kind, f64(counts), K, 0.5, 0.25, 1.5)
        check(out[:m], want, grad_bound(x64, kind, f64(counts), K, 0.5, 0.25, 1.5, dtype, want), (E, dtype))
        assert (f64(out[m:]) == 7.0).all()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("renorm", [False, True])
@pytest.mark.parametrize("E,K", [(16, 2), (64, 6), (100, 12), (256, 8), (1024, 40)])
def test_grad_with_the_routing(E, K, renorm, kind):
    """The sum of both gradients, rounded once: the routing's own call in 32 bits and the reference of the balance."""
    n, dtype = 300, F32
    x, ids = case(n, E, K, dtype, 3)
    x, ids = x.cuda(), ids.cuda()
    cfg = api.route_config(kind, K, renormalise=renorm, scale=1.5)
    dweights = normal((n, K), F32, 8, 0.01).cuda()
    counts = torch.from_numpy(R.choices(ids.cpu().numpy(), E).astype(np.int32)).cuda()
    alone, both = torch.zeros(n, E, device="cuda"), torch.zeros(n, E, device="cuda")
    api.route_grad(x, None, cfg, ids, dweights, alone)
    api.balance_grad(x, None, cfg, ids, dweights, counts, 0.5, 0.25, None, both)
    x64 = f64(x)
    want = R.balance_grad(x64, kind, f64(counts), K, 0.5, 0.25)
    bound = grad_bound(x64, kind, f64(counts), K, 0.5, 0.25, 1.0, dtype, want)
    # (the addition of the two is rounded)
    check(both, f64(alone) + want, bound + U32 * (np.abs(f64(alone)) + np.abs(want)), "dlogits")
    half = torch.zeros(n, E, dtype=BF16, device="cuda")
    api.balance_grad(x.to(BF16), None, cfg, ids, dweights, counts, 0.5, 0.25, None, half)
    x64 = f64(x.to(BF16))
    want = R.balance_grad(x64, kind, f64(counts), K, 0.5, 0.25)
    whole = torch.zeros(n, E, device="cuda")
    api.route_grad(x.to(BF16).float(), None, cfg, ids, dweights, whole)
    want = want + f64(whole)
    bound = grad_bound(x64, kind, f64(counts), K, 0.5, 0.25, 1.0, BF16, want)
    check(half, want, bound + U32 * np.abs(f64(whole)), "dlogits")


@pytest.mark.parametrize("kind", KINDS)
def test_gradient_is_the_differences(kind):
    """Of the reference's losses with the choices held."""
    n, E, K, h = 6, 12, 2, 1e-6
    x, ids = case(n, E, K, F32, 3, masked=False)
    counts = R.choices(ids.numpy(), E)
    grad = torch.zeros(n, E, device="cuda")
    api.balance_grad(x.cuda(), None, api.route_config(kind, K), None, None,
                     torch.from_numpy(counts.astype(np.int32)).cuda(), 0.5, 0.25, None, grad)
    x64 = f64(x)
    for t in range(n):
        for e in range(E):
            at = []
            for s in (h, -h):
                y = x64.copy()
                y[t, e] += s
                at.append(R.balance(y, kind, ids.numpy(), 0.5, 0.25)[2].sum())
            # (h^2 of the third derivative and 2^-52 / h of the losses, both below 1e-9; 32 bits: 2^-20 of the gradient's terms)
            assert abs(float(grad[t, e]) - (at[0] - at[1]) / (2 * h)) < 1e-8 + 2.0 ** -19


@pytest.mark.parametrize("E", [64, 256])
def test_captured_and_same_bits(E):
    n, K = 3000, 4
    x, ids = case(n, E, K, BF16, 3)
    x, ids = x.cuda(), ids.cuda()
    cfg, ws, count = api.route_config("softmax", K), api.LayerWorkspace(E), device_count(n)
    counts, share = torch.zeros(E, dtype=torch.int32, device="cuda"), torch.zeros(E, device="cuda")
    loss, out = torch.zeros(2, device="cuda"), torch.zeros_like(x)
    dweights = normal((n, K), F32, 3).cuda()

    def step():
        api.balance(x, count, cfg, ids, 0.02, 0.003, counts, share, loss, ws)
        api.balance_grad(x, count, cfg, ids, dweights, counts, 0.02, 0.003, None, out)

    step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for turn, m in enumerate((n, 11, 0, n)):
        new, new_ids = case(n, E, K, BF16, 40 + turn)
        x.copy_(new), ids.copy_(new_ids), count.fill_(m)
        g.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (counts, share, loss, out)]
        step()
        torch.cuda.synchronize()
        for a, b in zip(got, (counts, share, loss, out)):
            assert torch.equal(a, b)
        check_balance(x, ids, "softmax", m, (counts, share, loss))


def test_after_the_routing():
    """With what aa_route chose, on a side stream."""
    n, E, K = 500, 64, 6
    x, _ = case(n, E, K, F16, 12)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        x = x.cuda()
        ids, w = torch.zeros(n, K, dtype=torch.int32, device="cuda"), torch.zeros(n, K, device="cuda")
        offsets = torch.zeros(E + 1, dtype=torch.int32, device="cuda")
        plan = (offsets, torch.zeros(n * K, dtype=torch.int32, device="cuda"), torch.zeros_like(ids))
        api.route(x, None, None, api.route_config("softmax", K), ids, w, plan, api.ExpertWorkspace(n, K, E))
        got = run(x, ids, "softmax", None)
    side.synchronize()
    assert (got[0].cpu().numpy() == np.diff(offsets.cpu().numpy())).all()
    check_balance(x, ids, "softmax", None, got)


def routing_gradient(x, ids, kind, dweights, scale):
    """Of renormalised weights in 64 bits, relative to the highest choice; 0 where the scores' sum is 0 in 64 bits."""
    out = np.zeros_like(x)
    for t in range(len(x)):
        c = [e for e in ids[t] if e >= 0]
        v = x[t, c] if kind == "softmax" else np.minimum(x[t, c], 0.0)
        if v.max() - (x[t].max() if kind == "softmax" else 0.0) < -745.2:
            continue
        z = 1 / (1 + np.exp(-np.abs(x[t, c])))
        s = np.exp(v - v.max()) * (1.0 if kind == "softmax" else z)
        w, g = s / s.sum(), dweights[t, :len(c)] * scale
        rest = 1.0 if kind == "softmax" else np.where(x[t, c] > 0, 1 - z, z)
        out[t, c] = w * rest * (g - (w * g).sum())
    return out


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("E,K", [(5, 2), (16, 3), (32, 4), (60, 6), (128, 8), (256, 16), (64, 20), (200, 17), (300, 9), (1024, 40)])
def test_grad_of_choices_far_below_the_others(E, K, dtype, kind):
    """Renormalised choices (by a bias) that are 45 to 700 below the row's best, nothing in 32 bits beside them, or 800, nothing
    in 64; rows of ordinary choices between them."""
    n, scale = 70, 1.5
    x, g = normal((n, E), torch.float64, E, 1.5), torch.Generator().manual_seed(E)
    ids = torch.stack([torch.randperm(E, generator=g)[:K] for _ in range(n)])
    for t in range(n):
        deep = [0, 45, 90, 300, 700, 800][t % 6]
        if deep:
            x[t, ids[t]] = -deep + normal((K,), torch.float64, 100 + t)
    x = x.to(dtype)
    dweights = normal((n, K), F32, 8, 0.01)
    counts = R.choices(ids.numpy(), E)
    out = torch.full((n, E), 7.0, dtype=dtype, device="cuda")
    api.balance_grad(x.cuda(), None, api.route_config(kind, K, renormalise=True, scale=scale), ids.to(torch.int32).cuda(), dweights.cuda(),
                     torch.from_numpy(counts.astype(np.int32)).cuda(), 0.5, 0.25, None, out)
    x64, dw = f64(x), f64(dweights)
    route = routing_gradient(x64, ids.numpy(), kind, dw, scale)
    assert (np.abs(route[2::6]).max(1) > 1e-5).all() and (np.abs(route[4::6]).max(1) > 1e-5).all() and (route[5::6] == 0).all()
    want = R.balance_grad(x64, kind, counts.astype(float), K, 0.5, 0.25) + route
    # (a weight: an exponential of a difference of up to 10, a sum of K, a quotient)
    mag = scale * np.abs(dw).sum(1, keepdims=True)
    bound = grad_bound(x64, kind, counts.astype(float), K, 0.5, 0.25, 1.0, dtype, want)
    check(out, want, bound + (64 + K) * U32 * mag, "dlogits")
