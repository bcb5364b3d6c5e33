"""AdamW over many tensors and the gradients' norm on the GPU against the references in 64 bits.

Tolerances.  m and v are sums of two products: off by 4 U of their terms' magnitudes (a factor on the gradient adds 2
U, squared 4).  The step is a quotient of roots and products of those: where 1 - beta^t is worked out from t log beta in 32
bits it is off by 4 U; together 24 U of lr |m|' / (sqrt(v') + eps), m' the magnitudes' sum, and the parameter adds 3 U of
itself.  States of 8 bits: the value before rounding is off as above, so that the code is the reference's, or a neighbour's
where the place between two codes is nearer to a border than that."""
import numpy as np
import pytest
import torch

import layers_ref as R
from layers_ref import BF16, F16, F32, U32, check, device_count, f64, half_step, normal, tiny
from paper_1905_03381_amd import api

pytestmark = pytest.mark.gpu

F8 = torch.float8_e4m3fn
SEED = (5 << 33) + 77
F = lambda v: float(np.float32(v))
CFG = (F(1e-2), F(0.9), F(0.999), F(1e-8), F(0.1))


def config(cfg=CFG):
    return api.adamw_config(*cfg, SEED)


def codes_of(x):
    """Bytes and scales that hold x, to the nearest."""
    scale = R.scales(x)
    s = np.repeat(scale, R.BLOCK)[:len(x)]
    t = torch.from_numpy(x / np.where(s > 0, s, 1.0)).float().to(F8)
    return t, torch.from_numpy(scale).float()


class Tensor:
    """A tensor of the update with its state, on the GPU and as the reference has it."""

    def __init__(self, n, grad=F32, copy=None, bits=32, decay=1.0, seed=0, offset=0, empty=False):
        self.n, self.bits, self.decay = n, bits, F(decay)
        at = lambda t: torch.cat([torch.zeros(offset, dtype=t.dtype), t, torch.zeros(3, dtype=t.dtype)]).cuda()[offset:offset + n]
        size = torch.exp(normal((n,), torch.float64, seed, 1.5))
        self.g64 = normal((n,), torch.float64, seed + 1) * size
        m = (normal((n,), torch.float64, seed + 2) * size * 0.3).numpy() * (not empty)
        r = np.abs((normal((n,), torch.float64, seed + 3) * size * 0.7).numpy()) * (not empty)
        self.p = at(normal((n,), F32, seed + 4, 0.5))
        self.g = at(self.g64.to(grad))
        self.copy = None if copy is None else at(torch.zeros(n, dtype=copy))
        self.ms = self.vs = None
        if bits == 32:
            self.m, self.v = at(torch.from_numpy(m).float()), at(torch.from_numpy(r * r).float())
        else:
            (cm, sm), (cv, sv) = codes_of(m), codes_of(r)
            self.m, self.v, self.ms, self.vs = at(cm.view(torch.uint8)).view(F8), at(cv.view(torch.uint8)).view(F8), sm.cuda(), sv.cuda()

    def listed(self):
        return api.adamw_tensor(self.p, self.g, self.m, self.v, self.copy, self.ms, self.vs, self.decay)

    def states(self):
        if self.bits == 32:
            return f64(self.m), f64(self.v)
        value = lambda c, s: R.e4m3(c.view(torch.uint8).cpu().numpy()) * np.repeat(f64(s), R.BLOCK)[:self.n]
        return value(self.m, self.ms), value(self.v, self.vs) ** 2

    def before(self):
        return f64(self.p), f64(self.g), *self.states()

    def check(self, number, old, t, factor=1.0, lr_factor=1.0, cfg=CFG, seed=SEED):
        p, g, m, v = old
        lr, b1, b2, eps, wd = cfg
        want_p, want_m, want_v = R.adamw(p, g, m, v, t, cfg, self.decay, factor, lr_factor)
        of_m = 6 * U32 * (b1 * np.abs(m) + (1 - b1) * np.abs(g * factor)) + 2.0 ** -140
        of_v = 8 * U32 * want_v + 2.0 ** -140
        size = (b1 * np.abs(m) + (1 - b1) * np.abs(g * factor)) / (1 - b1 ** t)
        of_p = 32 * U32 * lr * lr_factor * size / (np.sqrt(want_v / (1 - b2 ** t)) + eps) + 4 * U32 * np.abs(p)
        check(self.p, want_p, of_p, "param")
        if self.copy is not None:
            dt = self.copy.dtype
            check(self.copy, want_p, of_p + half_step(dt) * (np.abs(want_p) + of_p) + tiny(dt), "copy")
            assert torch.equal(self.copy, self.p.to(dt))
        if self.bits == 32:
            check(self.m, want_m, of_m, "m")
            check(self.v, want_v, of_v, "v")
            return
        draw = R.draws(self.n, number, t, seed)
        root = np.sqrt(want_v)
        for what, value, off, codes, scale, one in (("m", want_m, of_m, self.m, self.ms, False),
                                                    ("v", root, 6 * U32 * root + 2.0 ** -140, self.v, self.vs, True)):
            s = R.scales(value)
            got_s = f64(scale)
            # (a largest value at a power of two may fall to either side)
            most = np.abs(R.blocks(value)).max(1)
            near = np.abs(most / np.exp2(np.round(np.log2(np.maximum(most, 1e-300)))) - 1) < 1e-5
            assert ((got_s == s) | near).all(), what
            got = R.e4m3(codes.view(torch.uint8).cpu().numpy())
            want, step, place = R.rounded(value, got_s, draw, one)
            per = np.repeat(got_s, R.BLOCK)[:self.n]
            slack = off / np.where(per > 0, per, 1.0) / step + 2.0 ** -19  # (the sum with the draw is rounded, too)
            border = np.abs(place - np.round(place)) <= slack
            differ = got != want
            assert (~differ | (border & (np.abs(got - want) <= 2 * step))).all(), what
            assert differ.mean() <= 1e-2, what


def update(tensors, t=0, cfg=CFG, lr_factor=None, factor=None, count=None):
    old = [x.before() for x in tensors]
    counter = torch.tensor([t], dtype=torch.int32, device="cuda")
    scalar = lambda v: None if v is None else torch.tensor([v], device="cuda")
    table = api.AdamWTable([x.listed() for x in tensors])
    api.adamw_step(table, config(cfg), scalar(lr_factor), scalar(factor), device_count(count), counter)
    torch.cuda.synchronize()
    return old, int(counter.item())


# One thread's eight, a block's scale, a chunk, and either side of them.
SIZES = [1, 2, 7, 8, 9, 255, 256, 257, 513, 2047, 2048, 2049, 5000, 70_001]


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("grad", [F32, BF16, F16])
@pytest.mark.parametrize("copy", [None, BF16, F16])
def test_sizes(bits, grad, copy):
    tensors = [Tensor(n, grad, copy, bits, decay=(i % 3) / 2, seed=10 * i, offset=i % 4) for i, n in enumerate(SIZES)]
    old, t = update(tensors, 6)
    assert t == 7
    for i, (x, o) in enumerate(zip(tensors, old)):
        x.check(i, o, 7)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("t", [0, 1, 999, 10_000_000])
def test_updates_and_factors(bits, t):
    tensors = [Tensor(n, BF16, BF16, bits, seed=n, empty=t == 0) for n in (100, 3001)]
    old, after = update(tensors, t, lr_factor=0.25, factor=0.125)
    assert after == t + 1
    for i, (x, o) in enumerate(zip(tensors, old)):
        x.check(i, o, t + 1, factor=0.125, lr_factor=0.25)


def test_many_tensors_of_all_kinds():
    """More than travel in one launch, empty ones among them; each as if it were alone."""
    g = np.random.default_rng(5)
    tensors = [Tensor(int(n), [F32, BF16, F16][i % 3], [None, BF16, F16][i % 3 - 1], [32, 8][i % 2], (i % 4) / 3, 100 * i, i % 5)
               for i, n in enumerate(np.where(g.random(150) < 0.1, 0, g.integers(1, 9000, 150)))]
    old, _ = update(tensors, 3)
    for i, (x, o) in enumerate(zip(tensors, old)):
        if x.n:
            x.check(i, o, 4)


@pytest.mark.parametrize("bits", [32, 8])
def test_a_run_of_updates(bits):
    """Every update from the state before it; nothing drifts between the copy and the parameters."""
    x = Tensor(5000, F32, BF16, bits, empty=True)
    counter = torch.zeros(1, dtype=torch.int32, device="cuda")
    table = api.AdamWTable([x.listed()])
    for t in range(1, 13):
        x.g.copy_(normal((x.n,), F32, 900 + t, 10.0 ** (t % 3 - 1)))
        old = x.before()
        api.adamw_step(table, config(), None, None, None, counter)
        x.check(0, old, t)
    assert int(counter.item()) == 12


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("why", ["count", "negative", "nan", "inf"])
def test_left_out(bits, why):
    x = Tensor(3000, BF16, BF16, bits, seed=3)
    kept = [None if t is None else t.clone() for t in (x.p, x.copy, x.m.view(torch.uint8), x.v.view(torch.uint8), x.ms, x.vs)]
    _, t = update([x], 5, factor={"nan": float("nan"), "inf": float("inf")}.get(why),
                  count={"count": 0, "negative": -1}.get(why))
    assert t == 5
    for a, b in zip(kept, (x.p, x.copy, x.m.view(torch.uint8), x.v.view(torch.uint8), x.ms, x.vs)):
        assert a is None or torch.equal(a, b)


def test_count_of_kept_rows():
    x = Tensor(300)
    old, t = update([x], 5, count=17)
    assert t == 6
    x.check(0, old[0], 6)


def test_what_is_not_finite_stays_where_it_is():
    for bits in (32, 8):
        x = Tensor(1000, F32, None, bits, seed=4)
        x.g[3], x.g[700], x.g[701] = float("nan"), float("inf"), float("-inf")
        old, _ = update([x], 0)
        ill = np.zeros(1000, bool)
        ill[[3, 700, 701]] = True
        assert not np.isfinite(f64(x.m.float()))[ill].any() and np.isfinite(f64(x.m.float()))[~ill].all()
        assert np.isfinite(f64(x.p))[~ill].all()
        if bits == 8:
            for scale in (x.ms, x.vs):
                assert np.isfinite(f64(scale)).all()
            y = Tensor(1000, F32, None, bits, seed=4)
            y.g[3], y.g[700], y.g[701] = 0.0, 0.0, 0.0
            update([y], 0)
            # (blocks without what is not finite; the others' scales are those of the rest)
            assert torch.equal(x.p[256:512], y.p[256:512]) and torch.equal(x.m[256:512].view(torch.uint8), y.m[256:512].view(torch.uint8))


def test_large_and_small_states():
    """Scales down to the smallest and gradients whose squares leave the range of 32 bits' normal numbers."""
    x = Tensor(2048, F32, None, 8, empty=True)
    size = np.repeat([1e-38, 1e-30, 1e-20, 1e-10, 1.0, 1e10, 1e18, 0.0], 256)
    x.g.copy_(torch.from_numpy(np.abs(f64(x.g)) * size + 0.0 * size).float())
    old, _ = update([x], 0)
    assert np.isfinite(f64(x.p)).all()
    m = x.states()[0]
    want = (1 - CFG[1]) * old[0][1]
    step = np.repeat(np.abs(R.blocks(want)).max(1), 256) * 2.0 ** -16 + np.abs(want) / 8 + 2.0 ** -134
    assert (np.abs(m - want) <= step).all()
    assert (f64(x.ms)[7] == 0) and (m[-256:] == 0).all()


def test_rounding_is_right_on_average():
    """A state that moves by less than half a step of its format moves all the same."""
    n, steps = 1 << 16, 200
    x = Tensor(n, F32, None, 8, empty=True)
    x.g.fill_(0.0)
    value = np.linspace(0.3, 1.0, n)
    (cm, sm), (cv, sv) = codes_of(value), codes_of(value)
    x.m.copy_(cm), x.v.copy_(cv), x.ms.copy_(sm), x.vs.copy_(sv)
    m0, v0 = x.states()
    table = api.AdamWTable([x.listed()])
    cfg = api.adamw_config(0.0, F(0.999), F(0.999), 1e-8, 0.0, SEED)
    counter = torch.zeros(1, dtype=torch.int32, device="cuda")
    for _ in range(steps):
        api.adamw_step(table, cfg, None, None, None, counter)
    m, v = x.states()
    # each rounding is off by at most a step, an eighth of the value, evenly: over 2^16 elements and 200 updates the mean is
    # off by at most 6 sqrt(200) / 8 / 2^8 of it (6 deviations); v is the square of what was rounded: sqrt(200) / 8 squared
    # at most may be added to its mean
    decay = F(0.999) ** steps
    assert abs(m.mean() / (m0.mean() * decay) - 1) <= 6 * np.sqrt(steps) / 8 / 2 ** 8
    root = np.sqrt(v).mean() / (np.sqrt(v0).mean() * F(0.999) ** (steps / 2))
    assert abs(root - 1) <= 6 * np.sqrt(steps) / 8 / 2 ** 8


def test_tensors_have_draws_of_their_own():
    a, b = Tensor(4096, F32, None, 8, seed=1), Tensor(4096, F32, None, 8, seed=1)
    update([a, b], 0)
    same = (a.m.view(torch.uint8) == b.m.view(torch.uint8)).float().mean().item()
    assert 0.2 < same < 0.99 and torch.equal(a.p, b.p)


# ---------------------------------------------------------------------------
# the norm


def run_norm(tensors, max_norm, scale=None):
    out = torch.full((2,), -1.0, device="cuda")
    api.grad_norm(api.AdamWTable([x.listed() for x in tensors]), max_norm,
                  None if scale is None else torch.tensor([scale], device="cuda"), out)
    return f64(out)


@pytest.mark.parametrize("max_norm", [1e-3, 7.0, float("inf")])
@pytest.mark.parametrize("scale", [None, 0.125, -2.0])
def test_norm(max_norm, scale):
    tensors = [Tensor(n, [F32, BF16, F16][i % 3], seed=i, offset=i % 3) for i, n in enumerate(SIZES + [0, 300_000])]
    got = run_norm(tensors, max_norm, scale)
    s = 1.0 if scale is None else scale
    norm = abs(s) * np.sqrt(sum((f64(x.g) ** 2).sum() for x in tensors))
    want = np.array([norm, s * min(1.0, F(max_norm) / norm)])
    check(got, want, 4 * U32 * np.abs(want), "norm")


def test_norm_beyond_32_bits_and_of_nothing():
    x = Tensor(5000)
    x.g.fill_(1e30)
    got = run_norm([x], 1.0)
    check(got, [np.float32(1e30) * np.sqrt(5000.0), 1 / (np.float32(1e30) * np.sqrt(5000.0))], [1e26, 1e-36], "norm")
    x.g.fill_(0.0)
    assert (run_norm([x], 1.0) == [0.0, 1.0]).all()
    assert (run_norm([Tensor(0)], 1.0) == [0.0, 1.0]).all()


@pytest.mark.parametrize("ill", [float("nan"), float("inf"), -float("inf")])
def test_norm_that_is_not_finite_leaves_the_update_out(ill):
    x, y = Tensor(5000, seed=1), Tensor(700, BF16, seed=2)
    y.g[699] = ill
    kept = x.p.clone(), y.p.clone()
    table = api.AdamWTable([x.listed(), y.listed()])
    out, t = torch.zeros(2, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    api.grad_norm(table, 1.0, None, out)
    assert not np.isfinite(f64(out)[0]) and np.isnan(f64(out)[1])
    api.adamw_step(table, config(), None, out[1:], None, t)
    assert torch.equal(x.p, kept[0]) and torch.equal(y.p, kept[1]) and int(t.item()) == 0


@pytest.mark.parametrize("bits", [32, 8])
def test_captured_with_clipping(bits):
    """The norm, the update and its counter in a graph, replayed with other gradients; an eager run beside it."""
    make = lambda: [Tensor(n, BF16, BF16, bits, seed=n) for n in (300, 40_000, 5000)]
    a, b = make(), make()
    ta, tb = api.AdamWTable([x.listed() for x in a]), api.AdamWTable([x.listed() for x in b])
    z = lambda k, t=F32: torch.zeros(k, dtype=t, device="cuda")
    out_a, out_b, ca, cb = z(2), z(2), z(1, torch.int32), z(1, torch.int32)

    def step(table, out, counter):
        api.grad_norm(table, 0.5, None, out)
        api.adamw_step(table, config(), None, out[1:], None, counter)

    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        step(ta, out_a, ca)
    for turn in range(4):
        for x, y in zip(a, b):
            new = normal((x.n,), BF16, 70 + turn, 10.0 ** turn)
            x.g.copy_(new), y.g.copy_(new)
        g.replay()
        torch.cuda.synchronize()
        step(tb, out_b, cb)
        torch.cuda.synchronize()
        assert torch.equal(out_a, out_b) and int(ca.item()) == int(cb.item()) == turn + 1
        for x, y in zip(a, b):
            for s, t in zip((x.p, x.copy, x.m.view(torch.uint8), x.v.view(torch.uint8)),
                            (y.p, y.copy, y.m.view(torch.uint8), y.v.view(torch.uint8))):
                assert torch.equal(s, t)


def test_many_elements():
    """More chunks than blocks, on a side stream; and what is past a tensor's end is left alone."""
    n = 9_000_001
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        x = Tensor(n, BF16, BF16, 8, seed=2, offset=5)
        old, _ = update([x, Tensor(77)], 9)
    side.synchronize()
    x.check(0, old[0], 10)
    assert (x.p.storage_offset() == 5) and (f64(x.p.as_strided((3,), (1,), 5 + n)) == 0).all()


def test_neighbours_and_shared_gradients():
    """Tensors that touch each other in one piece of memory are apart, and one gradient may be two tensors'."""
    n, m = 777, 512
    p, g = normal((n + m,), F32, 1).cuda(), normal((n,), BF16, 2).cuda()
    first, second = torch.zeros(n + m, device="cuda"), torch.zeros(n + m, device="cuda")
    old = f64(p)
    cut = lambda t: (t[:n], t[n:])
    listed = [api.adamw_tensor(x, g[:x.numel()], a, b) for x, a, b in zip(cut(p), cut(first), cut(second))]
    t = torch.zeros(1, dtype=torch.int32, device="cuda")
    api.adamw_step(api.AdamWTable(listed), CFG_ALONE, None, None, None, t)
    # after the first update of states that were 0 the step is lr g / (|g| + eps)
    both = np.concatenate([f64(g), f64(g)[:m]])
    want = -1e-2 * both / (np.abs(both) + 1e-8)
    assert np.abs(f64(p) - old - want).max() < 1e-2 * 16 * U32 + 4 * 2 * U32
    with pytest.raises(api.AAError):
        api.AdamWTable(listed + listed[:1])


CFG_ALONE = api.adamw_config(1e-2)


def test_numbers_that_are_not_the_tables():
    """A call whose numbers of tensors or chunks are others than the table's updates nothing."""
    x = [Tensor(5000), Tensor(300)]
    table = api.AdamWTable([k.listed() for k in x])
    before = [k.p.clone() for k in x]
    t, out = torch.zeros(1, dtype=torch.int32, device="cuda"), torch.zeros(2, device="cuda")
    for tensors, chunks in ((1, table.chunks), (2, table.chunks - 1)):
        other = type("Other", (), dict(ptr=table.ptr, bytes=table.bytes, device=table.device, n=tensors, chunks=chunks))
        api.adamw_step(other, CFG_ALONE, None, None, None, t)
        api.grad_norm(other, 1.0, None, out)
        assert out[0].item() == 0.0 and all(torch.equal(k.p, b) for k, b in zip(x, before))


def test_another_device_is_refused(monkeypatch):
    """Tensors of another device than the call's: here the call's device is said to be one that there is not."""
    z = lambda *s, t=F32: torch.zeros(*s, dtype=t, device="cuda")
    x, half, w, ws, c = z(4, 8), z(4, 8, t=BF16), z(8, 8, t=BF16), api.LayerWorkspace(8), z(1, t=torch.int32)
    tensor = api.adamw_tensor(z(9), z(9), z(9), z(9))
    table, cfg, ids, out = api.AdamWTable([tensor]), api.route_config("softmax", 2), z(4, 2, t=torch.int32), z(2)
    calls = [lambda: api.layer_norm(x, None, None, 1e-5, None, x),
             lambda: api.layer_norm_grad(x, x, None, z(4), z(4), None, None, x, z(8), z(8), False, ws),
             lambda: api.linear(half, w, None, "none", None, None, z(4, 8, t=BF16)),
             lambda: api.linear_grad(half, "none", None, c, None, z(8), False, ws),
             lambda: api.balance(x, c, cfg, ids, 0.1, 0.1, z(8, t=torch.int32), None, None, ws),
             lambda: api.balance_grad(x, c, cfg, None, None, z(8, t=torch.int32), 0.1, 0.1, None, x),
             lambda: api.AdamWTable([tensor]),
             lambda: api.grad_norm(table, 1.0, None, out),
             lambda: api.adamw_step(table, CFG_ALONE, None, None, None, c)]
    for call in calls[:1] + calls[2:6]:
        call()
    torch.cuda.synchronize()
    monkeypatch.setattr(api, "_current", lambda: 1)
    for call in calls:
        with pytest.raises(api.AAError, match="device"):
            call()


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("lr,factor,wd", [(1e-5, None, 1e-2), (1e-5, 0.5, 1e-2), (1e-4, None, 1e-3), (1e-3, 0.01, 1e-3)])
def test_a_small_decay_is_right_on_average(lr, factor, wd, bits):
    """lr weight_decay of about a rounding of the parameters.  A new parameter is rounded once, by half a step at most, to either
    side as often (the gradient's step, of many roundings and different everywhere, lies between): over n elements the mean
    decay, sum sign(p) (got - want) / sum |p|, is off by at most 6 deviations of those, 6 2^-24 sqrt(sum p^2) / sum |p|, and
    8 U of the decay and of the step's mean."""
    n = 1 << 19
    cfg = (F(lr), CFG[1], CFG[2], CFG[3], F(wd))
    x = Tensor(n, F32, None, bits, seed=11)
    old, _ = update([x], 9, cfg=cfg, lr_factor=factor)
    p, g, m, v = old[0]
    f = 1.0 if factor is None else F(factor)
    want = R.adamw(p, g, m, v, 10, cfg, 1.0, lr_factor=f)[0]
    drift = (np.sign(p) * (f64(x.p) - want)).sum() / np.abs(p).sum()
    decay = cfg[0] * f * cfg[4]
    deviation = 6 * 2.0 ** -24 * np.sqrt((p * p).sum()) / np.abs(p).sum()
    assert deviation < decay / 8   # (it would be seen)
    assert abs(drift) <= deviation + 8 * U32 * (decay + cfg[0] * f * 6), (drift, decay, deviation)


def test_numbers_of_another_table_count_no_update():
    """A call whose numbers of tensors or chunks are not the table's is no update: the counter stays, and the factor that the norm
    hands out leaves a following update out, too."""
    x = [Tensor(5000, F32, BF16, seed=1), Tensor(300, BF16, BF16, 8, seed=2)]
    table = api.AdamWTable([k.listed() for k in x])
    kept = [t.clone() for k in x for t in (k.p, k.copy, k.m.view(torch.uint8), k.v.view(torch.uint8))]
    t, out = torch.tensor([4], dtype=torch.int32, device="cuda"), torch.zeros(2, device="cuda")
    for tensors, chunks in ((1, table.chunks), (2, table.chunks - 1), (2, 0), (1, 0)):
        other = type("Other", (), dict(ptr=table.ptr, bytes=table.bytes, device=table.device, n=tensors, chunks=chunks))
        api.adamw_step(other, CFG_ALONE, None, None, None, t)
        assert int(t.item()) == 4
        out.fill_(7.0)
        api.grad_norm(other, 1.0, None, out)
        assert np.isnan(f64(out)[1])
        api.adamw_step(table, CFG_ALONE, None, out[1:], None, t)
        assert int(t.item()) == 4
    assert all(torch.equal(a, b) for a, b in zip(kept, [t for k in x for t in (k.p, k.copy, k.m.view(torch.uint8), k.v.view(torch.uint8))]))
    # the table's own numbers still count
    api.adamw_step(table, CFG_ALONE, None, None, None, t)
    api.grad_norm(table, 1.0, None, out)
    assert int(t.item()) == 5 and np.isfinite(f64(out)).all()


@pytest.mark.parametrize("bits,grad", [(32, F32), (8, BF16)])
def test_more_than_the_caches_hold(bits, grad):
    """8192 chunks and more, an odd end."""
    n = 8200 * 2048 + 1931
    x = Tensor(n, grad, BF16, bits, seed=6)
    old, t = update([Tensor(77), x], 9)
    assert t == 10
    x.check(1, old[1], 10)
    assert (f64(x.p.as_strided((3,), (1,), n)) == 0).all() and (f64(x.copy.as_strided((3,), (1,), n)) == 0).all()
