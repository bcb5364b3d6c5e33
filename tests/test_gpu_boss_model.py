"""The operators around a block of experts together, as boss.Boss and boss.AdamW use them: gradients of the whole model
against a plain one in 64 bits, updates against torch's, a step in a graph.

Tolerance of the model's gradients: every buffer between two operators is rounded to 2^-8 of its values at most (bf16) and passes
at most about 14 buffers on its way (input layer, two blocks of norm, logits or hidden rows and sum, last norm, read-out, and back);
the operators between them are near isometries here (norms, residuals of unit size), so that in the 2-norm they add up to at
most 14 2^-8 = 5.5 %; f16 has an eighth of that."""
import numpy as np
import pytest
import torch

import layers_ref as R
from layers_ref import BF16, F16, F32, U32, check, device_count, f64, normal
from paper_1905_03381_amd import api
from paper_1905_03381_amd.boss import AdamW, Boss, ExpertBlock

pytestmark = pytest.mark.gpu

D64 = torch.float64


def plain_block(block, x, i, weights, m):
    """The block of experts with the choices that it made (no dropout)."""
    router, gate_up, down, gamma, beta = weights
    h = torch.nn.functional.layer_norm(x, x.shape[1:], gamma, beta, 1e-5)
    logits = h @ router[0].t()
    ids = block.ids[:m].cpu().long()
    s = torch.softmax(logits, 1).gather(1, ids)
    s = s / s.sum(1, keepdim=True)
    out = x
    f = down.shape[2]
    for k in range(ids.shape[1]):
        g = torch.bmm(gate_up[ids[:, k]], h.unsqueeze(2)).squeeze(2)
        y = torch.bmm(down[ids[:, k]], (torch.nn.functional.silu(g[:, :f]) * g[:, f:]).unsqueeze(2)).squeeze(2)
        out = out + s[:, k:k + 1] * y
    coef, z = block.balance
    E = router.shape[1]
    counts = torch.bincount(ids.view(-1), minlength=E).double()
    loss = coef * E / (m * ids.shape[1]) * (counts * torch.softmax(logits, 1).mean(0)).sum()
    return out, loss + z * (torch.logsumexp(logits, 1) ** 2).mean()


def plain(model, x, m):
    """out and the balance losses, and the weights that their gradients are asked of."""
    w = [v.detach().cpu().to(D64).requires_grad_(True) for v in model.weights()]
    h = torch.nn.functional.gelu(x @ w[0].t() + w[1], approximate="tanh")
    total, at = 0.0, 2
    for i, block in enumerate(model.blocks):
        h, loss = plain_block(block, h, i, w[at:at + 5], m)
        total, at = total + loss, at + 5
    h = torch.nn.functional.layer_norm(h, h.shape[1:], w[at], w[at + 1], 1e-5)
    return h @ w[at + 2].t() + w[at + 3], total, w


@pytest.mark.parametrize("dtype,off", [(BF16, 14 * 2.0 ** -8), (F16, 14 * 2.0 ** -11)])
@pytest.mark.parametrize("n_max,count", [(300, 300), (300, 190), (24, 24)])
def test_gradients_of_the_model(dtype, off, n_max, count):
    d_in, d, f, d_out, E, K = 40, 64, 48, 3, 8, 2
    model = Boss(n_max, d_in, d, f, d_out, E, K, dtype=dtype, balance=0.3, z_loss=0.01)
    for i, (w, g) in enumerate(zip(model.weights(), model.grads)):
        if w.dim() == 1:  # (weights of norms and biases that are not 1 and 0)
            w.add_(normal(tuple(w.shape), F32, i, 0.1).cuda())
    x, dout = normal((n_max, d_in), dtype, 3).cuda(), normal((n_max, d_out), dtype, 4, 1 / count).cuda()
    out = torch.full((n_max, d_out), 7.0, dtype=dtype, device="cuda")
    cnt = device_count(count)
    model.forward(x, cnt, 0, out)
    model.backward(x, cnt, 0, dout)
    want, balance, weights = plain(model, x[:count].cpu().to(D64), count)
    ((want * dout[:count].cpu().to(D64)).sum() + balance).backward()
    norm = np.linalg.norm
    got = f64(out)[:count]
    assert norm(got - want.detach().numpy()) <= off * norm(want.detach().numpy())
    assert (f64(out)[count:] == 7).all()
    for i, (g, w) in enumerate(zip(model.grads, weights)):
        g, w = f64(g), w.grad.numpy()
        assert norm(g - w) <= off * norm(w), (i, tuple(w.shape), norm(g - w) / norm(w))
    losses = sum(float(b.balance_loss.sum()) for b in model.blocks)
    assert abs(losses - float(balance.detach())) <= off * float(balance.detach())


def test_a_block_without_norm_and_balance_is_as_it_was():
    """The options off: the calls and results of before."""
    n, d = 50, 64
    x, dout = normal((n, d), BF16, 3).cuda(), normal((n, d), BF16, 4).cuda()
    a, b = ExpertBlock(n, d, 48, 8, 2, p=0.2), ExpertBlock(n, d, 48, 8, 2, p=0.2, balance=0.0, norm=False)
    assert len(a.weights()) == len(a.grads) == 3
    for block in (a, b):
        block.o, block.d = torch.zeros_like(x), torch.zeros_like(x)
        block.forward(x, device_count(n), 5, block.o)
        block.backward(x, device_count(n), 5, dout, block.d)
    assert torch.equal(a.o, b.o) and torch.equal(a.d, b.d)


def test_fewer_rows_than_the_model_are_refused():
    model, x = Boss(40, 16, 32, 16, 2, 4, 2), torch.zeros(39, 16, dtype=BF16, device="cuda")
    with pytest.raises(api.AAError):
        model.forward(x, device_count(39), 0, torch.zeros(40, 2, dtype=BF16, device="cuda"))


def small_model(n_max=64):
    return Boss(n_max, 24, 32, 16, 2, 4, 2, layers=1, balance=0.1)


def test_updates_are_torchs():
    """Three updates against torch.optim.AdamW in 64 bits on the same gradients: each is off by 40 U of the step's size and 4 U
    of the parameter, and hands that on."""
    model = small_model()
    opt = AdamW(model, 1e-2, weight_decay=0.1, max_norm=0.5)
    params = [torch.nn.Parameter(m.detach().cpu().to(D64)) for m in opt.masters]
    f = lambda v: float(np.float32(v))
    groups = [dict(params=[p], weight_decay=0.0 if p.dim() == 1 else f(0.1)) for p in params]
    theirs = torch.optim.AdamW(groups, lr=f(1e-2), betas=(f(0.9), f(0.999)), eps=f(1e-8))
    for step in range(3):
        for i, (g, p) in enumerate(zip(model.grads, params)):
            g.copy_(normal(tuple(g.shape), F32, 100 * step + i))
            p.grad = g.detach().cpu().to(D64)
        opt.step(device_count(5))
        torch.nn.utils.clip_grad_norm_(params, 0.5)
        theirs.step()
    assert int(opt.t.item()) == 3
    for m, p, w in zip(opt.masters, params, model.weights()):
        # (clip_grad_norm_ divides by the norm + 1e-6: 2e-8 of these norms, above 50; a step is at most about lr)
        check(m, p.detach().numpy(), 3 * (1e-2 * (60 * U32 + 1e-6) + 4 * U32 * np.abs(p.detach().numpy())), "master")
        assert torch.equal(w, m.to(w.dtype))


@pytest.mark.parametrize("bits", [32, 8])
def test_an_empty_batch_changes_nothing(bits):
    model = small_model()
    opt = AdamW(model, 1e-2, max_norm=1.0, state_bits=bits)
    x, dout = normal((64, 24), BF16, 3).cuda(), normal((64, 2), BF16, 4).cuda()
    out, cnt = torch.zeros(64, 2, dtype=BF16, device="cuda"), device_count(0)
    kept = [w.clone() for w in model.weights()]
    model.forward(x, cnt, 0, out)
    model.backward(x, cnt, 0, dout)
    assert all((g == 0).all() for g in model.grads)
    opt.step(cnt)
    assert all(torch.equal(a, b) for a, b in zip(kept, model.weights())) and int(opt.t.item()) == 0


@pytest.mark.parametrize("bits", [32, 8])
def test_a_step_in_a_graph(bits):
    """Forward, backward and update captured once and replayed on other batches, next to an eager model's."""
    n = 200
    make = lambda: Boss(n, 24, 64, 32, 2, 8, 2, layers=2, balance=0.1, p=0.1)
    a, b = make(), make()
    oa, ob = (AdamW(m, 1e-2, weight_decay=0.1, max_norm=0.5, state_bits=bits) for m in (a, b))
    x, dout = torch.zeros(n, 24, dtype=BF16, device="cuda"), torch.zeros(n, 2, dtype=BF16, device="cuda")
    out_a, out_b, cnt = torch.zeros_like(dout), torch.zeros_like(dout), device_count(0)

    def step(model, opt, out):
        model.forward(x, cnt, 3, out)
        model.backward(x, cnt, 3, dout)
        opt.step(cnt)

    step(a, oa, out_a)   # (loads the kernels; an empty batch)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step(a, oa, out_a)
    for turn, m in enumerate((n, 120, 0, 1, n)):
        x.copy_(normal((n, 24), BF16, 10 + turn)), dout.copy_(normal((n, 2), BF16, 30 + turn)), cnt.fill_(m)
        g.replay()
        torch.cuda.synchronize()
        step(b, ob, out_b)
        torch.cuda.synchronize()
        assert torch.equal(out_a[:m], out_b[:m]) and torch.equal(oa.norm, ob.norm)
        for s, t in zip(a.weights() + oa.masters + a.grads, b.weights() + ob.masters + b.grads):
            assert torch.equal(s, t)
        assert int(oa.t.item()) == int(ob.t.item())
    assert int(oa.t.item()) == 4


def test_state_bits_are_checked():
    with pytest.raises(api.AAError):
        AdamW(small_model(), 1e-3, state_bits=16)


def test_the_workload_runs(capsys):
    import json
    from paper_1905_03381_amd import workloads
    workloads.main(["boss", "--n", "16384", "--threads", "4"])
    got = json.loads(capsys.readouterr().out.strip().splitlines()[-1])
    assert len(got["stages"]) == 5 and got["kept_per_pool"] > 0
    assert all(np.isfinite(v) for v in [got["loss_first"], got["loss_last"]] + sum(got["balance_loss"], []))


@pytest.mark.parametrize("scale", [2.0 ** 16, 2.0 ** 10])
@pytest.mark.parametrize("norm", [False, True])
def test_the_balance_loss_follows_a_loss_scale(norm, scale):
    """f16, a pool whose balance gradient (1e-7 a logit here) is a step of the type or two: scaled with the loss it is as
    exact as any.  dout is 0, so that the router's gradient is the balance's alone: each logit's is off by half a step and what
    32 bits lose, 256 U at most, and the sum over m rows by m U of its terms."""
    n, m, d, E, K = 4200, 4096, 64, 16, 2
    block = ExpertBlock(n, d, 32, E, K, dtype=F16, balance=0.01, z_loss=1e-6, norm=norm)
    x, cnt = normal((n, d), F16, 3).cuda(), device_count(m)
    block.forward(x, cnt, 0, torch.zeros_like(x))
    block.backward(x, cnt, 0, torch.zeros_like(x), torch.zeros_like(x), loss_scale=torch.tensor([scale], device="cuda"))
    logits, rows = f64(block.logits)[:m], f64(block.norm.out if norm else x)[:m]
    dl = R.balance_grad(logits, "softmax", f64(block.counts), K, float(np.float32(0.01)), float(np.float32(1e-6)))
    assert np.abs(dl).max() < 2e-6
    off = R.half_step(F16) * np.abs(dl) + R.tiny(F16) / scale + 256 * U32 * np.abs(dl).max(1, keepdims=True)
    want, size = dl.T @ rows, np.abs(dl).T @ np.abs(rows)
    check(f64(block.grads[0])[0] / scale, want, off.T @ np.abs(rows) + (m + 64) * U32 * size, "router")


def test_gradients_under_a_loss_scale_are_as_many_times_larger():
    """A power of two moves no digits (bf16 has the range): bit by bit, in all of the model."""
    n, scale = 150, 8.0
    x, dout, cnt = normal((n, 24), BF16, 3).cuda(), normal((n, 2), BF16, 4).cuda(), device_count(140)
    a, b = (Boss(n, 24, 64, 32, 2, 8, 2, balance=0.1, z_loss=0.01) for _ in range(2))
    for model in (a, b):
        model.forward(x, cnt, 0, torch.zeros_like(dout))
    a.backward(x, cnt, 0, dout)
    b.backward(x, cnt, 0, dout * scale, loss_scale=torch.tensor([scale], device="cuda"))
    for g, h in zip(a.grads, b.grads):
        assert torch.equal(g * scale, h)


def test_an_update_of_scaled_gradients_is_the_unscaled():
    """grad_scale = 1 / loss_scale gives them back."""
    n, scale = 64, 1024.0
    x, dout, cnt = normal((n, 24), BF16, 3).cuda(), normal((n, 2), BF16, 4).cuda(), device_count(n)
    models = [small_model(n) for _ in range(2)]
    opts = [AdamW(m, 1e-2, weight_decay=0.1, max_norm=0.5) for m in models]
    for model, opt, s in zip(models, opts, (1.0, scale)):
        model.forward(x, cnt, 0, torch.zeros_like(dout))
        model.backward(x, cnt, 0, dout * s, loss_scale=torch.tensor([s], device="cuda"))
        opt.step(cnt, grad_scale=torch.tensor([1 / s], device="cuda"))
    for v, w in zip(opts[0].masters, opts[1].masters):
        assert torch.equal(v, w)


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("p", [0.0, 0.2])
def test_the_calls_of_a_block_without_norm_and_balance(dtype, p):
    """Its results, bit by bit, from the calls it stands for."""
    n, m, d, f, E, K, step = 90, 77, 64, 48, 8, 2, 5
    z = lambda *s, t=dtype: torch.zeros(*s, dtype=t, device="cuda")
    x, dout, cnt = normal((n, d), dtype, 3).cuda(), normal((n, d), dtype, 4).cuda(), device_count(m)
    block, out, dx = ExpertBlock(n, d, f, E, K, dtype=dtype, p=p), z(n, d), z(n, d)
    block.forward(x, cnt, step, out)
    block.backward(x, cnt, step, dout, dx)
    router, gate_up, down = block.weights()
    ws, one = api.ExpertWorkspace(n, K, E), torch.tensor([0, m], dtype=torch.int32, device="cuda")
    logits, ids, weights = z(n, E), z(n, K, t=torch.int32), z(n, K, t=F32)
    offsets, order, slot = z(E + 1, t=torch.int32), z(n * K, t=torch.int32), z(n, K, t=torch.int32)
    h, pre, y, o = z(n * K, f), z(n * K, 2 * f), z(n * K, d), z(n, d)
    api.expert_forward(x, None, 1, one, router, "none", logits)
    api.route(logits, cnt, None, block.cfg, ids, weights, (offsets, order, slot), ws)
    api.expert_forward(x, order, K, offsets, gate_up, "gated", h, pre)
    api.expert_forward(h, None, 1, offsets, down, "none", y)
    api.expert_combine(y, slot, weights, cnt, x, p, block.seed, step, o)
    assert torch.equal(out, o)
    dy, dpre, pairs, of_router = z(n * K, d), z(n * K, 2 * f), z(n * K, d), z(n, d)
    dweights, dlogits, back = z(n, K, t=F32), z(n, E), z(n, d)
    grads = [z(*w.shape, t=F32) for w in block.weights()]
    api.expert_combine_grad(dout, y, slot, weights, cnt, p, block.seed, step, dy, dweights)
    api.expert_grad_weight(dy, h, None, 1, offsets, grads[2], False, ws)
    api.expert_grad_input(dy, offsets, down, "gated", pre, dpre)
    api.expert_grad_weight(dpre, x, order, K, offsets, grads[1], False, ws)
    api.expert_grad_input(dpre, offsets, gate_up, "none", None, pairs)
    api.route_grad(logits, cnt, block.cfg, ids, dweights, dlogits)
    api.expert_grad_weight(dlogits, x, None, 1, one, grads[0], False, ws)
    api.expert_grad_input(dlogits, one, router, "none", None, of_router)
    api.dropout(of_router, cnt, dout, 0.0, 0, 0, back)
    api.expert_combine(pairs, slot, None, cnt, back, 0.0, 0, 0, back)
    assert torch.equal(dx, back) and all(torch.equal(a, b) for a, b in zip(block.grads, grads))
