"""References in 64 bits of the operators around a Boss block of experts, and helpers their tests share.  Nothing here
calls the package."""
import numpy as np
import torch

U32 = 2.0 ** -23  # (2^-23 rather than 2^-24 for adders that cut instead of rounding)
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
TYPES = [F32, BF16, F16]
HALVES = [BF16, F16]


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def tiny(dtype):
    """Half a step below the smallest normal number."""
    return torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps / 2


def normal(shape, dtype, seed, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=g, dtype=torch.float64) * scale).to(dtype)


def strided(t, ld, offset=0):
    """t's values on the GPU as rows `ld` elements apart, the first `offset` elements into its storage; NaN between."""
    n, d = t.shape
    store = torch.full((offset + max(n, 1) * ld + 8,), float("nan"), dtype=t.dtype, device="cuda")
    v = store[offset:offset + n * ld].view(n, ld)[:, :d] if n else store[:0].view(0, ld)[:, :d]
    v.copy_(t)
    return v


def f64(t):
    return t.detach().cpu().to(torch.float64).numpy()


def device_count(count):
    return None if count is None else torch.tensor([count], dtype=torch.int32, device="cuda")


def in_use(count, n):
    return n if count is None else min(max(count, 0), n)


def check(got, want, bound, what):
    got, want = f64(got) if isinstance(got, torch.Tensor) else got, np.asarray(want)
    with np.errstate(invalid="ignore"):
        err = np.abs(got - want)
    same = (got == want) | (np.isnan(got) & np.isnan(want))
    bad = ~same & ~(err <= bound)
    assert not bad.any(), (what, int(bad.sum()), got[bad][:3], want[bad][:3], np.broadcast_to(bound, got.shape)[bad][:3])


# ---------------------------------------------------------------------------
# layer norm

# Additions that a term of a row's sum passes through: 16 of its thread, 6 between the lanes, 16 between the waves, and the
# division.
ROW_DEPTH = 40


def norm(x, gamma, beta, eps):
    """out, mean, rstd"""
    mean = x.mean(1, keepdims=True)
    rstd = 1 / np.sqrt(((x - mean) ** 2).mean(1, keepdims=True) + eps)
    return (x - mean) * rstd * gamma + beta, mean[:, 0], rstd[:, 0]


def norm_bounds(x, gamma, beta, eps, dtype):
    """How far out, mean and rstd may be off.  The mean is off by at most e = ROW_DEPTH U mean|x|; the squares around it sum
    to d (var + e^2) at most, with ROW_DEPTH + 4 roundings; the root halves what is relative, and adds a few."""
    out, mean, rstd = norm(x, gamma, beta, eps)
    xh = (x - mean[:, None]) * rstd[:, None]
    e = ROW_DEPTH * U32 * np.abs(x).mean(1)
    of_rstd = (ROW_DEPTH + 4) / 2 * U32 + 4 * U32 + (e * rstd) ** 2
    of_out = np.abs(gamma) * ((rstd * e)[:, None] + np.abs(xh) * (of_rstd + 4 * U32)[:, None])
    of_out = of_out + 2 * U32 * (np.abs(xh * gamma) + np.abs(beta))
    of_out += half_step(dtype) * (np.abs(out) + of_out) + tiny(dtype)
    return of_out, e, rstd * of_rstd


def norm_grad(dout, x, gamma, mean, rstd, residual):
    """dx, dgamma, dbeta"""
    xh = (x - mean[:, None]) * rstd[:, None]
    g = dout * gamma
    dx = rstd[:, None] * (g - g.mean(1, keepdims=True) - xh * (g * xh).mean(1, keepdims=True)) + residual
    return dx, (dout * xh).sum(0), dout.sum(0)


def norm_grad_bounds(dout, x, gamma, mean, rstd, residual, dtype):
    """xh is off by 2 roundings, g by one, their sums by ROW_DEPTH more; the sums over n rows by n (blocks, parts and their
    joining: at most 64 more) of their terms' magnitudes."""
    dx = norm_grad(dout, x, gamma, mean, rstd, residual)[0]
    xh = np.abs(x - mean[:, None]) * rstd[:, None]
    g = np.abs(dout * gamma)
    s1, s2 = g.mean(1, keepdims=True), (g * xh).mean(1, keepdims=True)
    of_dx = rstd[:, None] * U32 * (5 * g + (ROW_DEPTH + 6) * s1 + (ROW_DEPTH + 10) * xh * s2) + 2 * U32 * np.abs(residual)
    of_dx += half_step(dtype) * (np.abs(dx) + of_dx) + tiny(dtype)
    rows = len(x) + 64
    return of_dx, (rows + 3) * U32 * (np.abs(dout) * xh).sum(0), rows * U32 * np.abs(dout).sum(0)


# ---------------------------------------------------------------------------
# balance of a router


def shares(x, kind):
    """p, softmax, log sum exp (0 where it is not finite) and 1 - score of float64 logits; -inf and NaN are not free."""
    free = x > -np.inf  # (False for NaN)
    x = np.where(free, x, -np.inf)
    top = x.max(1, keepdims=True)
    with np.errstate(invalid="ignore", over="ignore"):
        e = np.where(free, np.where(x == top, 1.0, np.exp(x - np.where(np.isfinite(top), top, 0.0))), 0.0)
        e = np.where(np.isinf(top) & (x < top), 0.0, e)
    total = e.sum(1, keepdims=True)
    q = np.where(total > 0, e / np.where(total > 0, total, 1.0), 0.0)
    finite = np.isfinite(top[:, 0])
    lse = np.where(finite, np.where(finite, top[:, 0], 0.0) + np.log(np.where(total[:, 0] > 0, total[:, 0], 1.0)), 0.0)
    if kind == "softmax":
        return q, q, lse, np.ones_like(q)
    with np.errstate(over="ignore"):
        t = np.exp(-np.abs(x))
    low = np.minimum(x, 0.0)
    best = np.where(np.isfinite(low.max(1, keepdims=True)), low.max(1, keepdims=True), 0.0)
    s = np.where(free, np.exp(low - best) / (1 + t), 0.0)  # (relative to the row's highest)
    total = s.sum(1, keepdims=True)
    rest = np.where(x > 0, t / (1 + t), 1 / (1 + t))
    return np.where(total > 0, s / np.where(total > 0, total, 1.0), 0.0), q, lse, rest


def choices(ids, n_experts):
    ids = ids[(ids >= 0) & (ids < n_experts)]
    return np.bincount(ids.reshape(-1), minlength=n_experts)


def balance(x, kind, ids, coef, z_coef):
    """counts, shares, losses"""
    m, E = x.shape
    counts = choices(ids, E)
    if m == 0:
        return counts, np.zeros(E), np.zeros(2)
    p, _, lse, _ = shares(x, kind)
    share = p.sum(0) / m
    return counts, share, np.array([coef * E / (m * ids.shape[1]) * (counts * share).sum(), z_coef / m * (lse ** 2).sum()])


def balance_grad(x, kind, counts, top_k, coef, z_coef, up=1.0):
    m, E = x.shape
    p, q, lse, rest = shares(x, kind)
    d = coef * E / (m * m * top_k) * p * rest * (counts - (p * counts).sum(1, keepdims=True))
    return up * (d + 2 * z_coef / m * lse[:, None] * q)


# ---------------------------------------------------------------------------
# AdamW

BLOCK = 256


def e4m3(codes):
    """Values of bytes in the OCP format e4m3 (no infinities, NaN with all bits set)."""
    c = codes.astype(np.int64)
    e, f = (c >> 3) & 15, c & 7
    v = np.where(e == 0, f * 2.0 ** -9, (8 + f) * 2.0 ** (e - 10.0))
    v = np.where((c & 127) == 127, np.nan, v)
    return np.where(c & 128, -v, v)


def philox_words(c0, c1, c2, c3, seed):
    """Philox4x32-10 (Salmon et al., SC'11) on arrays of counters."""
    c = [np.asarray(v, np.uint64) + np.zeros_like(np.asarray(c0, np.uint64)) for v in (c0, c1, c2, c3)]
    k0, k1, low = seed & 0xFFFFFFFF, seed >> 32, np.uint64(0xFFFFFFFF)
    for _ in range(10):
        p0, p1 = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(p1 >> np.uint64(32)) ^ c[1] ^ np.uint64(k0), p1 & low, (p0 >> np.uint64(32)) ^ c[3] ^ np.uint64(k1), p0 & low]
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    return c


def draws(n, tensor, t, seed):
    """The 16-bit draws of elements 0 .. n - 1 of a tensor at update t."""
    group = np.arange((n + 7) // 8)
    words = philox_words(group, (1 << 31) + tensor, t & 0xFFFFFFFF, 0, seed)
    halves = [h for w in words for h in (w & np.uint64(0xFFFF), w >> np.uint64(16))]
    return np.stack(halves, 1).reshape(-1)[:n].astype(np.float64)


def blocks(x):
    """x in blocks of 256, zeros behind its end."""
    return np.pad(x, (0, -len(x) % BLOCK)).reshape(-1, BLOCK)


def scales(x):
    most = np.where(np.isfinite(blocks(x)), np.abs(blocks(x)), 0.0).max(1)
    _, e = np.frexp(most)
    return np.where(most > 0, np.ldexp(1.0, np.maximum(e - 8, -126)), 0.0)


def rounded(x, scale, draw, at_least_one):
    """Values of the codes, and the place of a in steps (to tell how near a border it was)."""
    s = np.repeat(scale, BLOCK)[:len(x)]
    a = np.abs(x) / np.where(s > 0, s, 1.0)
    _, e = np.frexp(a)
    step = np.ldexp(1.0, np.maximum(e - 4, -9))
    place = a / step + draw / 65536
    q = np.floor(place)
    if at_least_one:
        q = np.where(a > 0, np.maximum(q, 1), q)
    return np.sign(x) * q * step, step, place


def adamw(p, g, m, v, t, cfg, decay, factor=1.0, lr_factor=1.0):
    """p, m, v after update t (counted from 1); cfg: (lr, beta1, beta2, eps, weight_decay) as 32-bit values."""
    lr, b1, b2, eps, wd = cfg
    lr, g = lr * lr_factor, g * factor
    m, v = b1 * m + (1 - b1) * g, b2 * v + (1 - b2) * g * g
    step = m / (1 - b1 ** t) / (np.sqrt(v / (1 - b2 ** t)) + eps)
    return p * (1 - lr * wd * decay) - lr * step, m, v


# ---------------------------------------------------------------------------
# dense layer

ACTS = ["none", "relu", "silu", "gelu", "gated"]
GELU = 2 * np.sqrt(2 / np.pi)


def sigmoid(x):
    with np.errstate(over="ignore"):
        return 1 / (1 + np.exp(-x))


def activate(h, act):
    """The activation, and how far it is off for h exact, in units of U: |value| (2 |argument| (1 - z) + 8) for those with an
    exponential of the argument."""
    if act == "none":
        return h, 0 * h
    if act == "relu":
        return np.where(h < 0, 0.0, h), 0 * h
    gate, up = (h, 1.0) if act != "gated" else (h[:, :h.shape[1] // 2], h[:, h.shape[1] // 2:])
    arg = GELU * (gate + 0.044715 * gate ** 3) if act == "gelu" else gate
    z = sigmoid(arg)
    out = gate * z * up
    return out, np.abs(out) * (4 * np.abs(arg) * (1 - z) + 8)


def slopes(h, act):
    """(d out / d h, d out / d up) and the size of the terms the first is a sum of."""
    if act == "none":
        return np.ones_like(h), None, np.ones_like(h)
    if act == "relu":
        return (h > 0).astype(np.float64), None, (h > 0).astype(np.float64)
    gate, up = (h, 1.0) if act != "gated" else (h[:, :h.shape[1] // 2], h[:, h.shape[1] // 2:])
    arg = GELU * (gate + 0.044715 * gate ** 3) if act == "gelu" else gate
    inner = GELU * (1 + 3 * 0.044715 * gate ** 2) if act == "gelu" else 1.0
    z = sigmoid(arg)
    first, second = z, gate * z * (1 - z) * inner
    return (first + second) * up, gate * z if act == "gated" else None, (np.abs(first) + np.abs(second)) * np.abs(up)


def linear(x, w, bias, act, residual):
    h = x @ w.T + bias
    return activate(h, act)[0] + residual, h


def linear_bounds(x, w, bias, act, residual, dtype):
    """A sum of d_in products and the bias in 32 bits is off by (d_in + 3) U of its terms' magnitudes; the activations' slopes
    are at most 1.13."""
    h = x @ w.T + bias
    of_h = (x.shape[1] + 3) * U32 * (np.abs(x) @ np.abs(w).T + np.abs(bias))
    out, rel = activate(h, act)
    if act == "gated":
        f = out.shape[1]
        gate = np.abs(h[:, :f]) * sigmoid(h[:, :f])
        b = 1.13 * of_h[:, :f] * (np.abs(h[:, f:]) + of_h[:, f:]) + of_h[:, f:] * gate
    else:
        b = 1.13 * of_h
    b = b + rel * U32 + 2 * U32 * np.abs(residual)
    out = out + residual
    return b + half_step(dtype) * (np.abs(out) + b) + tiny(dtype), of_h + half_step(dtype) * (np.abs(h) + of_h) + tiny(dtype)


def linear_grad(dout, h, act):
    """dpre, its error, dbias, its error's terms (sum of magnitudes)."""
    s, u, size = slopes(h, act)
    d = dout * s
    with np.errstate(over="ignore"):
        arg = np.abs(h if act != "gated" else h[:, :h.shape[1] // 2])
    # (beyond 20 the slopes are 0 or 1)
    off = np.abs(dout) * size * (4 * np.minimum(1.6 * arg * (1 + 0.045 * arg ** 2), 120) + 16) * U32
    off = off * (act not in ("none", "relu"))
    if act == "gated":
        d, off = np.concatenate([d, dout * u], 1), np.concatenate([off, np.abs(dout * u) * (4 * np.minimum(arg, 120) + 16) * U32], 1)
    return d, off
