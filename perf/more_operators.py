"""Cases the operators around a Boss block of experts are timed on: layer norm, the dense product with its epilogue, the
router's balance loss and the optimizer's step over all tensors -- each in the direction and type that the case says.

A case is a dict of plain values; its "op" says which call a pass makes:

  norm           layer norm of the rows in use, with the rows' statistics
  norm_grad      gradient of the rows (and what comes along the residual), of the weight and of the offset
  linear         product with a matrix, bias, activation and residual
  linear_grad    gradients of its input, its matrix and its bias
  balance        choices of each expert, its mean share of the probability, balance loss and the loss on the logits' size
  balance_grad   their gradient, added to that of the routing weights
  adamw          one AdamW update of all tensors, states in 32 or 8 bits, with or without clipping by the gradients' norm

Where `own` is false `run` is the plain form in elementary torch operations, in 32 bits (bias corrections and the norm's
sum in 64); where it is true `run` calls the framework.  `exact` is the definition in 64 bits.  All inputs are drawn on the
GPU from the seed.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}
EPS = 1e-5                       # of the layer norm
LR, BETA1, BETA2, ADAM_EPS, DECAY = 1e-3, 0.9, 0.999, 1e-8, 0.01
MAX_NORM = 1.0
ROUND_SEED = (3 << 32) + 1905    # of the states' rounding
BLOCK = 256                      # neighbours that share a scale


def listed():
    return [
        # One row answered: launch and latency, nothing else.
        {"name": "norm_one_row", "op": "norm", "n": 1, "kept": 1, "d": 1024, "dtype": "bf16", "affine": True},
        # The norm before a block of experts of a training step, twice the benchmark's pool.
        {"name": "norm_rows", "op": "norm", "n": 32_768, "kept": 30_000, "d": 4096, "dtype": "bf16", "affine": True},
        # The backward pass of a norm whose rows are of odd width, in 32 bits, half of a pool kept.
        {"name": "norm_grad_odd", "op": "norm_grad", "n": 16_384, "kept": 8191, "d": 1021, "dtype": "f32",
         "affine": True, "residual": False},
        # The backward pass of a training step of wide rows, with the gradient that comes along the residual.
        {"name": "norm_grad_wide", "op": "norm_grad", "n": 16_384, "kept": 16_384, "d": 8192, "dtype": "bf16",
         "affine": True, "residual": True},
        # One row through a dense layer: the matrix is what is read.
        {"name": "linear_one_row", "op": "linear", "n": 1, "kept": 1, "d_in": 2048, "d_out": 4096, "act": "gelu",
         "bias": True, "residual": False, "pre": False, "dtype": "bf16"},
        # The wide half of a dense layer in a training step, with what its backward pass needs.
        {"name": "linear_gelu", "op": "linear", "n": 16_384, "kept": 16_384, "d_in": 2048, "d_out": 8192, "act": "gelu",
         "bias": True, "residual": False, "pre": True, "dtype": "bf16"},
        # The backward pass of a residual layer whose widths fill no tile, rows left over from a pool.
        {"name": "linear_grad_odd", "op": "linear_grad", "n": 8192, "kept": 6001, "d_in": 1000, "d_out": 1544,
         "act": "silu", "bias": True, "dtype": "f16"},
        # The balance loss of a wide router over a pool, sigmoid scores.
        {"name": "balance_pool", "op": "balance", "n": 16_384, "kept": 16_384, "E": 256, "K": 8, "dtype": "f32",
         "score": "sigmoid", "masked": 0.0},
        # Routing and balance gradient of the logits together; some experts are masked, some rows altogether.
        {"name": "balance_grad_softmax", "op": "balance_grad", "n": 65_536, "kept": 60_001, "E": 64, "K": 6,
         "dtype": "bf16", "score": "softmax", "masked": 0.02, "route": True, "renorm": True},
        # The tensors of a small block: the optimizer's shortest step.
        {"name": "adamw_small", "op": "adamw", "layers": 1, "d": 64, "f": 64, "E": 1, "bits": 32, "grad": "f32",
         "copy": "bf16", "clip": False},
        # The block of the experts workload, states in 32 bits, gradients as the block's products leave them.
        {"name": "adamw_block", "op": "adamw", "layers": 1, "d": 512, "f": 512, "E": 32, "bits": 32, "grad": "f32",
         "copy": "bf16", "clip": True},
        # 121 tensors of odd sizes, states in 8 bits, gradients in 16.
        {"name": "adamw_many_8bit", "op": "adamw", "layers": 24, "d": 517, "f": 310, "E": 4, "bits": 8, "grad": "bf16",
         "copy": "bf16", "clip": True},
    ]


MOST_FLOPS = 2 * 16_384 * 2048 * 8192  # of the largest listed product
MOST_BYTES = 850_000_000               # and of the largest listed pass over memory


def _log(rng, lo, hi):
    """A whole number from lo to hi, even over its logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _width(rng, lo, hi):
    """A row width: powers of two, odd multiples of eight, odd ones."""
    kind = rng.random()
    if kind < 0.35:
        return min(hi, 1 << rng.randint(max(0, lo.bit_length() - 1), hi.bit_length() - 1))
    if kind < 0.7:
        return min(hi, 8 * (_log(rng, max(1, lo // 8), hi // 8) | 1))
    return min(hi - 1, _log(rng, lo, hi) | 1)


def _kept(rng, n):
    return n if rng.random() < 0.6 else rng.randint(1, n)


def draw(rng):
    op = rng.choice(["norm", "norm", "norm_grad", "norm_grad", "linear", "linear", "linear_grad", "balance",
                     "balance_grad", "adamw", "adamw"])
    if op == "adamw":
        bits = rng.choice([32, 8])
        while True:
            case = {"op": op, "layers": _log(rng, 1, 40), "d": _width(rng, 16, 2048), "f": _width(rng, 16, 2048),
                    "E": _log(rng, 1, 32), "bits": bits, "grad": rng.choice(["f32", "bf16", "f16"]),
                    "copy": rng.choice(["none", "bf16", "f16"]), "clip": rng.random() < 0.6}
            if work(case)["bytes"] <= MOST_BYTES and sum(_sizes(case)) <= 50_000_000:
                return case
    if op in ("balance", "balance_grad"):
        E = rng.choice([4, 8, 16, 64, 128, 256]) if rng.random() < 0.6 else _log(rng, 2, 1000)
        n = _log(rng, 1, min(65_536, (1 << 24) // E))
        case = {"op": op, "n": n, "kept": _kept(rng, n), "E": E, "K": min(E, _log(rng, 1, 12)),
                "dtype": rng.choice(["f32", "bf16", "f16"]), "score": rng.choice(["softmax", "sigmoid"]),
                "masked": rng.choice([0.0, 0.0, 0.02, 0.3])}
        if op == "balance_grad":
            case["route"], case["renorm"] = rng.random() < 0.6, rng.random() < 0.5
        return case
    if op in ("norm", "norm_grad"):
        d = _width(rng, 8, 16_384)
        n = _log(rng, 1, min(40_000, (1 << 27) // d))
        case = {"op": op, "n": n, "kept": _kept(rng, n), "d": d, "dtype": rng.choice(["f32", "bf16", "bf16", "f16"]),
                "affine": rng.random() < 0.8}
        if op == "norm_grad":
            case["residual"] = rng.random() < 0.5
    else:
        d_in, d_out = _width(rng, 32, 8192), _width(rng, 32, 8192)
        act = rng.choice(["none", "relu", "silu", "gelu", "gated"])
        most = MOST_FLOPS // (d_in * d_out * (2 if act == "gated" else 1) * (4 if op == "linear_grad" else 2))
        n = _log(rng, 1, min(20_000, most))
        case = {"op": op, "n": n, "kept": _kept(rng, n), "d_in": d_in, "d_out": d_out, "act": act,
                "bias": rng.random() < 0.8, "dtype": rng.choice(["bf16", "bf16", "f16"])}
        if op == "linear":
            case["residual"], case["pre"] = rng.random() < 0.5, rng.random() < 0.5
    while work(case)["bytes"] > MOST_BYTES and case["n"] > 1:
        case["n"] //= 2
        case["kept"] = min(case["kept"], case["n"])
    return case


# ---------------------------------------------------------------------------
# inputs


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 6007 + 17)
    return g


def _normal(g, *shape, dtype=torch.float32, scale=1.0):
    """Normal values; large tensors in slices, so that no 32-bit copy of the whole is held."""
    out = torch.empty(*shape, dtype=dtype, device="cuda")
    flat = out.view(-1)
    for lo in range(0, flat.numel(), 1 << 26):
        hi = min(flat.numel(), lo + (1 << 26))
        flat[lo:hi] = torch.randn(hi - lo, generator=g, device="cuda") * scale
    return out


def _zeros(*shape, dtype=torch.float32):
    return torch.zeros(*shape, dtype=dtype, device="cuda")


def _wide(c):
    """Columns of a product's matrix rows: gated layers have two for each of the result's."""
    return c["d_out"] * (2 if c["act"] == "gated" else 1)


def _sizes(c):
    """Elements of the tensors of `layers` normed blocks of experts and a read-out."""
    d, f, E = c["d"], c["f"], c["E"]
    return [k for _ in range(c["layers"]) for k in (d, d, E * d, E * 2 * f * d, E * d * f)] + [d]


def _norm_inputs(c, g):
    n, d, dt = c["n"], c["d"], DTYPES[c["dtype"]]
    # a residual stream: rows of different size and mean, some columns larger than others
    spread = torch.exp(0.5 * torch.randn(d, generator=g, device="cuda"))
    size = torch.exp(0.3 * torch.randn(n, 1, generator=g, device="cuda"))
    x = torch.randn(n, d, generator=g, device="cuda") * spread * size
    x += 0.3 * torch.randn(n, 1, generator=g, device="cuda")
    s = {"x": x.to(dt), "gamma": None, "beta": None}
    if c["affine"]:
        s["gamma"] = 1 + 0.2 * torch.randn(d, generator=g, device="cuda")
        s["beta"] = 0.1 * torch.randn(d, generator=g, device="cuda")
    if c["op"] == "norm_grad":
        s["dout"] = _normal(g, n, d, dtype=dt)
        s["residual"] = _normal(g, n, d, dtype=dt) if c["residual"] else None
        v = s["x"].double()
        s["mean"] = v.mean(1).float()
        s["rstd"] = (v.var(1, unbiased=False) + EPS).rsqrt().float()
    return s


def _linear_inputs(c, g):
    n, dt = c["n"], DTYPES[c["dtype"]]
    s = {"x": _normal(g, n, c["d_in"], dtype=dt),
         "w": _normal(g, _wide(c), c["d_in"], dtype=dt, scale=c["d_in"] ** -0.5)}
    if c["op"] == "linear":
        s["bias"] = _normal(g, _wide(c), scale=0.1) if c["bias"] else None
        s["residual"] = _normal(g, n, c["d_out"], dtype=dt) if c["residual"] else None
    else:
        s["dout"] = _normal(g, n, c["d_out"], dtype=dt)
        s["pre"] = None if c["act"] == "none" else _normal(g, n, _wide(c), dtype=dt)
        s["group"] = torch.tensor([0, c["kept"]], dtype=torch.int32, device="cuda")  # the rows as one group
    return s


def _balance_inputs(c, g):
    n, E, K = c["n"], c["E"], c["K"]
    # logits of a router that has learned to prefer some experts
    x = torch.randn(n, E, generator=g, device="cuda") * 1.5
    x += 0.5 * torch.randn(E, generator=g, device="cuda")
    if c["masked"] > 0:
        x[torch.rand(n, E, generator=g, device="cuda") < c["masked"]] = -math.inf
        x[torch.rand(n, generator=g, device="cuda") < 0.01] = -math.inf
    x = x.to(DTYPES[c["dtype"]])
    top, ids = torch.topk(x.float(), K, dim=1)
    s = {"logits": x, "ids": torch.where(top > -math.inf, ids, -1).to(torch.int32).contiguous(), "coef": 0.01,
         "z_coef": 0.001}
    if c["op"] == "balance_grad":
        s["dweights"] = 0.01 * torch.randn(n, K, generator=g, device="cuda") if c["route"] else None
        s["dloss"] = torch.rand(1, generator=g, device="cuda") + 0.5
        live = s["ids"][:c["kept"]].reshape(-1).long()
        s["counts"] = torch.bincount(live[live >= 0], minlength=E).to(torch.int32)
    return s


def _adamw_inputs(c, g):
    """All tensors as parts of flat buffers, each on a multiple of BLOCK elements; what lies between is 0 and stays so."""
    sizes = _sizes(c)
    room = [-(-k // BLOCK) * BLOCK for k in sizes]
    total, starts = sum(room), [sum(room[:i]) for i in range(len(room))]
    tensor = torch.repeat_interleave(torch.arange(len(room), device="cuda"),
                                     torch.tensor([r // BLOCK for r in room], device="cuda"))
    first = torch.tensor(starts, device="cuda")[tensor] // BLOCK
    inside = torch.arange(total // BLOCK, device="cuda") - first  # a block's place in its tensor
    left = torch.tensor(sizes, device="cuda")[tensor] - inside * BLOCK
    live = torch.arange(BLOCK, device="cuda").view(1, -1) < left.view(-1, 1)
    live = live.view(-1)
    # (vectors of one row take no decay)
    s = {"sizes": sizes, "starts": starts, "tensor": tensor, "inside": inside,
         "decays": [0.0 if k <= c["d"] else 1.0 for k in sizes]}
    s["decay"] = torch.tensor(s["decays"], device="cuda")[tensor].view(-1, 1)
    size = torch.exp(torch.randn(total // BLOCK, 1, generator=g, device="cuda"))  # of a block's gradients
    own_size = torch.exp(0.7 * torch.randn(total, generator=g, device="cuda")).view(-1, BLOCK) * size * 1e-4
    grad = torch.randn(total, generator=g, device="cuda").view(-1, BLOCK) * own_size
    s["grad"] = (grad.view(-1) * live).to(DTYPES[c["grad"]])
    s["param"] = _normal(g, total, scale=0.03) * live
    s["copy"] = None if c["copy"] == "none" else s["param"].to(DTYPES[c["copy"]])
    m = torch.randn(total, generator=g, device="cuda").view(-1, BLOCK) * own_size * 0.3 * live.view(-1, BLOCK)
    r = own_size * (0.7 + 0.6 * torch.rand(total, generator=g, device="cuda").view(-1, BLOCK)) * live.view(-1, BLOCK)
    if c["bits"] == 32:
        s["m"], s["v"] = m.view(-1), (r * r).view(-1)
    else:
        for name, value in (("m", m), ("v", r)):
            scale = torch.exp2(torch.floor(torch.log2(value.abs().amax(1).clamp(min=1e-30))) - 7)
            s[name + "_scale"] = scale
            s[name] = (value / scale.view(-1, 1)).to(torch.float8_e4m3fn).view(-1)
    s["t"] = torch.full((1,), 100, dtype=torch.int32, device="cuda")
    s["norm"] = _zeros(2)
    return s


def _inputs(c, seed):
    """The inputs of a pass, and nothing else."""
    g, op = _gen(seed), c["op"]
    if op == "adamw":
        return dict(_adamw_inputs(c, g), case=c)
    make = {"norm": _norm_inputs, "linear": _linear_inputs, "balance": _balance_inputs}[op.replace("_grad", "")]
    return dict(make(c, g), case=c, count=torch.full((1,), c["kept"], dtype=torch.int32, device="cuda"))


def prepare(case, seed):
    s = _inputs(case, seed)
    if not own:
        return s
    from paper_1905_03381_amd import api
    c, op = case, case["op"]
    s["api"] = api
    if op == "norm":
        s["out"] = {"out": torch.zeros_like(s["x"]), "mean": _zeros(c["n"]), "rstd": _zeros(c["n"])}
    elif op == "norm_grad":
        s["out"] = {"dx": torch.zeros_like(s["x"])}
        if c["affine"]:
            s["out"].update(dgamma=_zeros(c["d"]), dbeta=_zeros(c["d"]))
        s["ws"] = api.LayerWorkspace(c["d"])
    elif op == "linear":
        dt = s["x"].dtype
        s["out"] = {"out": _zeros(c["n"], c["d_out"], dtype=dt)}
        if c["pre"]:
            s["out"]["pre"] = _zeros(c["n"], _wide(c), dtype=dt)
    elif op == "linear_grad":
        s["out"] = {"dx": torch.zeros_like(s["x"]), "dw": torch.zeros_like(s["w"])}
        if c["bias"]:
            s["out"]["dbias"] = _zeros(_wide(c))
        s["dpre"] = s["dout"] if c["act"] == "none" else torch.zeros_like(s["pre"])
        s["ws"], s["product_ws"] = api.LayerWorkspace(_wide(c)), api.ExpertWorkspace(c["n"], 1, 1)
    elif op in ("balance", "balance_grad"):
        s["cfg"] = api.route_config(c["score"], c["K"], renormalise=c.get("renorm", False))
        if op == "balance":
            s["out"] = {"counts": _zeros(c["E"], dtype=torch.int32), "share": _zeros(c["E"]), "loss": _zeros(2)}
            s["ws"] = api.LayerWorkspace(c["E"])
        else:
            s["out"] = {"dlogits": torch.zeros_like(s["logits"])}
    else:
        tensors = []
        for lo, k, decay in zip(s["starts"], s["sizes"], s["decays"]):
            t = {name: s[name][lo:lo + k] for name in ("param", "grad", "m", "v")}
            if s["copy"] is not None:
                t["copy"] = s["copy"][lo:lo + k]
            if c["bits"] == 8:
                at = slice(lo // BLOCK, lo // BLOCK - (-k // BLOCK))
                t["m_scale"], t["v_scale"] = s["m_scale"][at], s["v_scale"][at]
            tensors.append(api.adamw_tensor(decay=decay, **t))
        s["table"] = api.AdamWTable(tensors)
        s["cfg"] = api.adamw_config(LR, BETA1, BETA2, ADAM_EPS, DECAY, ROUND_SEED)
    return s


# ---------------------------------------------------------------------------
# the framework's calls


def _state_of(s):
    """What an optimizer's step leaves behind."""
    names = ["param", "copy", "m", "v", "t"] + (["m_scale", "v_scale"] if s["case"]["bits"] == 8 else [])
    out = {k: s[k] for k in names if s[k] is not None}
    if s["case"]["clip"]:
        out["norm"] = s["norm"]
    return out


def _run_own(s):
    api, c, out = s["api"], s["case"], s.get("out")
    op = c["op"]
    if op == "norm":
        api.layer_norm(s["x"], s["gamma"], s["beta"], EPS, s["count"], out["out"], out["mean"], out["rstd"])
    elif op == "norm_grad":
        api.layer_norm_grad(s["dout"], s["x"], s["gamma"], s["mean"], s["rstd"], s["residual"], s["count"], out["dx"],
                            out.get("dgamma"), out.get("dbeta"), False, s["ws"])
    elif op == "linear":
        api.linear(s["x"], s["w"], s["bias"], c["act"], s["residual"], s["count"], out["out"], out.get("pre"))
    elif op == "linear_grad":
        if c["bias"] or c["act"] != "none":
            api.linear_grad(s["dout"], c["act"], s["pre"], s["count"], None if c["act"] == "none" else s["dpre"],
                            out.get("dbias"), False, s["ws"])
        w = s["w"].unsqueeze(0)
        api.expert_grad_input(s["dpre"], s["group"], w, "none", None, out["dx"])
        api.expert_grad_weight(s["dpre"], s["x"], None, 1, s["group"], out["dw"].unsqueeze(0), False, s["product_ws"])
    elif op == "balance":
        api.balance(s["logits"], s["count"], s["cfg"], s["ids"], s["coef"], s["z_coef"], out["counts"], out["share"],
                    out["loss"], s["ws"])
    elif op == "balance_grad":
        api.balance_grad(s["logits"], s["count"], s["cfg"], s["ids"], s["dweights"], s["counts"], s["coef"],
                         s["z_coef"], s["dloss"], out["dlogits"])
    else:
        factor = None
        if c["clip"]:
            api.grad_norm(s["table"], MAX_NORM, None, s["norm"])
            factor = s["norm"][1:]
        api.adamw_step(s["table"], s["cfg"], None, factor, None, s["t"])
        return _state_of(s)
    return out


# ---------------------------------------------------------------------------
# the plain forms


def _run_norm(s):
    c, m = s["case"], s["case"]["kept"]
    x = s["x"][:m].float()
    mean = x.sum(1, keepdim=True) / c["d"]
    v = x - mean
    rstd = 1 / torch.sqrt((v * v).sum(1, keepdim=True) / c["d"] + EPS)
    y = v * rstd
    if c["affine"]:
        y = y * s["gamma"] + s["beta"]
    out = {"out": torch.zeros_like(s["x"]), "mean": _zeros(c["n"]), "rstd": _zeros(c["n"])}
    out["out"][:m], out["mean"][:m], out["rstd"][:m] = y, mean[:, 0], rstd[:, 0]
    return out


def _run_norm_grad(s):
    c, m = s["case"], s["case"]["kept"]
    dy, rstd = s["dout"][:m].float(), s["rstd"][:m].view(-1, 1)
    xh = (s["x"][:m].float() - s["mean"][:m].view(-1, 1)) * rstd
    g = dy * s["gamma"] if c["affine"] else dy
    d = rstd * (g - g.sum(1, keepdim=True) / c["d"] - xh * ((g * xh).sum(1, keepdim=True) / c["d"]))
    out = {"dx": torch.zeros_like(s["x"])}
    out["dx"][:m] = d if s["residual"] is None else d + s["residual"][:m].float()
    if c["affine"]:
        out["dgamma"], out["dbeta"] = (dy * xh).sum(0), dy.sum(0)
    return out


def _sigmoid(x):
    return 1 / (1 + torch.exp(-x))


def _gelu_slope(x):
    """2 u(x) of gelu(x) = x sigmoid(2 u), u = sqrt(2 / pi) (x + 0.044715 x^3), and its slope."""
    k = 2 * math.sqrt(2 / math.pi)
    return k * (x + 0.044715 * x * x * x), k * (1 + 3 * 0.044715 * x * x)


def _run_linear(s):
    c, m, f = s["case"], s["case"]["kept"], s["case"]["d_out"]
    h = s["x"][:m].float() @ s["w"].float().t()
    if s["bias"] is not None:
        h += s["bias"]
    if c["act"] == "relu":
        y = h.clamp(min=0)
    elif c["act"] == "silu":
        y = h * _sigmoid(h)
    elif c["act"] == "gelu":
        y = h * _sigmoid(_gelu_slope(h)[0])
    elif c["act"] == "gated":
        y = h[:, :f] * _sigmoid(h[:, :f]) * h[:, f:]
    else:
        y = h
    if s["residual"] is not None:
        y = y + s["residual"][:m].float()
    out = {"out": _zeros(c["n"], f, dtype=s["x"].dtype)}
    out["out"][:m] = y
    if c["pre"]:
        out["pre"] = _zeros(c["n"], h.shape[1], dtype=s["x"].dtype)
        out["pre"][:m] = h
    return out


def _run_linear_grad(s):
    c, m, f = s["case"], s["case"]["kept"], s["case"]["d_out"]
    d = s["dout"][:m].float()
    h = None if s["pre"] is None else s["pre"][:m].float()
    if c["act"] == "relu":
        d = torch.where(h > 0, d, 0.0)
    elif c["act"] == "silu":
        z = _sigmoid(h)
        d = d * z * (1 + h * (1 - z))
    elif c["act"] == "gelu":
        u, slope = _gelu_slope(h)
        z = _sigmoid(u)
        d = d * z * (1 + h * (1 - z) * slope)
    elif c["act"] == "gated":
        gate, up = h[:, :f], h[:, f:]
        z = _sigmoid(gate)
        d = torch.cat([d * up * z * (1 + gate * (1 - z)), d * gate * z], dim=1)
    out = {"dx": torch.zeros_like(s["x"])}
    out["dx"][:m] = d @ s["w"].float()
    out["dw"] = (d.t() @ s["x"][:m].float()).to(s["w"].dtype)
    if c["bias"]:
        out["dbias"] = d.sum(0)
    return out


def _probabilities(x, kind):
    """Scores, their shares of the row's sum and log sum exp of the free logits; -inf takes an expert out."""
    free = x > -math.inf
    top = x.amax(1, keepdim=True).clamp(min=-3e38)
    e = torch.where(free, torch.exp(x - top), 0.0)
    all_e = e.sum(1, keepdim=True)
    some = all_e > 0
    soft = torch.where(some, e / all_e, 0.0)
    lse = torch.where(some, top + torch.log(all_e), 0.0)
    if kind == "softmax":
        return soft, soft, soft, lse
    score = torch.where(free, _sigmoid(x), 0.0)
    total = score.sum(1, keepdim=True)
    return score, torch.where(total > 0, score / total, 0.0), soft, lse


def _run_balance(s):
    c, m, E = s["case"], s["case"]["kept"], s["case"]["E"]
    _, p, _, lse = _probabilities(s["logits"][:m].float(), c["score"])
    key = s["ids"][:m].reshape(-1).long()
    counts = torch.zeros(E + 1, dtype=torch.int32, device="cuda")
    counts.scatter_add_(0, torch.where(key < 0, E, key), torch.ones_like(key, dtype=torch.int32))
    counts, share = counts[:E], p.sum(0) / m
    loss = torch.stack([s["coef"] * E / (m * c["K"]) * (counts.float() * share).sum(),
                        s["z_coef"] / m * (lse * lse).sum()])
    return {"counts": counts, "share": share, "loss": loss}


def _run_balance_grad(s):
    c, m, E = s["case"], s["case"]["kept"], s["case"]["E"]
    x = s["logits"][:m].float()
    score, p, soft, lse = _probabilities(x, c["score"])
    counts = s["counts"].float()
    counts = counts - counts.sum() / E
    d = s["dloss"] * (s["coef"] * E / (m * c["K"]) / m) * p * (counts - (p * counts).sum(1, keepdim=True))
    if c["score"] == "sigmoid":
        d = d * (1 - score)
    d = d + s["dloss"] * (2 * s["z_coef"] / m) * lse * soft
    if s["dweights"] is not None:
        ids, there = s["ids"][:m].clamp(min=0).long(), s["ids"][:m] >= 0
        a = torch.where(there, s["dweights"][:m], 0.0)
        chosen = torch.where(there, score.gather(1, ids), 0.0)
        if c["renorm"]:
            total = chosen.sum(1, keepdim=True)
            a = (a - (a * chosen).sum(1, keepdim=True) / total) / total
            a = torch.where(there & (total > 0), a, 0.0)
        full = torch.zeros_like(score).scatter_add_(1, ids, a)
        if c["score"] == "sigmoid":
            d = d + full * score * (1 - score)
        else:
            d = d + score * (full - (a * chosen).sum(1, keepdim=True))
    out = torch.zeros_like(s["logits"])
    out[:m] = torch.where(x > -math.inf, d, 0.0)
    return {"dlogits": out}


def _mul32(a, b):
    """High and low word of the product of two 32-bit words held in 64-bit integers."""
    p = a * b  # wraps beyond 63 bits: the bits are those of the product
    return (p >> 32) & 0xFFFFFFFF, p & 0xFFFFFFFF


def _uniforms(s, t):
    """[blocks, BLOCK] of 2^-16 times a 16-bit draw: Philox4x32-10 on (element / 8, 2^31 + tensor, update), eight draws."""
    c0 = s["inside"].view(-1, 1) * (BLOCK // 8) + torch.arange(BLOCK // 8, device="cuda").view(1, -1)
    c1 = ((1 << 31) + s["tensor"]).view(-1, 1).expand_as(c0)
    c2, c3 = t.long().view(1, 1).expand_as(c0), torch.zeros_like(c0)
    k0, k1 = ROUND_SEED & 0xFFFFFFFF, ROUND_SEED >> 32
    for _ in range(10):
        hi0, lo0 = _mul32(c0, 0xD2511F53)
        hi1, lo1 = _mul32(c2, 0xCD9E8D57)
        c0, c1, c2, c3 = hi1 ^ c1 ^ k0, lo1, hi0 ^ c3 ^ k1, lo0
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    words = torch.stack([c0, c1, c2, c3], dim=2)
    return torch.stack([words & 0xFFFF, words >> 16], dim=3).view(-1, BLOCK).float() / 65536


def _to_8bit(x, u, floor_at_one):
    """Codes and scales of blocks x[., BLOCK]: a power of two that brings the largest into [128, 256), then rounding down of
    the code's steps plus u.  floor_at_one: what is above 0 is at least one step."""
    _, e = torch.frexp(x.abs().amax(1, keepdim=True))
    scale = torch.where(x.abs().amax(1, keepdim=True) > 0, torch.exp2((e - 8).clamp(min=-126).float()), 0.0)
    a = torch.where(scale > 0, x.abs() / scale, 0.0)
    _, e = torch.frexp(a)
    step = torch.exp2((e - 4).clamp(min=-9).float())
    q = torch.floor(a / step + u)
    if floor_at_one:
        q = torch.where(a > 0, q.clamp(min=1), q)
    return (torch.sign(x) * q * step).to(torch.float8_e4m3fn), scale.view(-1)


def _run_adamw(s):
    c = s["case"]
    f32 = lambda v: torch.tensor(v, dtype=torch.float32).item()
    b1, b2 = f32(BETA1), f32(BETA2)
    g = s["grad"].float().view(-1, BLOCK)
    if c["clip"]:
        norm = torch.sqrt(g.double().square().sum()).float()
        factor = torch.where(norm > MAX_NORM, MAX_NORM / norm, 1.0)
        s["norm"].copy_(torch.stack([norm, factor]))
        g = g * factor
    t = s["t"] + 1
    p = s["param"].view(-1, BLOCK)
    if c["bits"] == 8:
        m = s["m"].float().view(-1, BLOCK) * s["m_scale"].view(-1, 1)
        v = s["v"].float().view(-1, BLOCK) * s["v_scale"].view(-1, 1)
        v = v * v
    else:
        m, v = s["m"].view(-1, BLOCK), s["v"].view(-1, BLOCK)
    m = b1 * m + (1 - b1) * g
    v = b2 * v + (1 - b2) * (g * g)
    rate = (LR / (1 - b1 ** t.double())).float()
    root = (1 / torch.sqrt(1 - b2 ** t.double())).float()
    p = p * (1 - LR * DECAY * s["decay"]) - rate * m / (torch.sqrt(v) * root + ADAM_EPS)
    s["param"].copy_(p.view(-1))
    if s["copy"] is not None:
        s["copy"].copy_(p.view(-1))
    if c["bits"] == 8:
        u = _uniforms(s, t)
        for name, value in (("m", m), ("v", torch.sqrt(v))):
            codes, scale = _to_8bit(value, u, name == "v")
            s[name].copy_(codes.view(-1))
            s[name + "_scale"].copy_(scale)
    else:
        s["m"].copy_(m.view(-1))
        s["v"].copy_(v.view(-1))
    s["t"].copy_(t)
    return _state_of(s)


def run(state):
    if own:
        return _run_own(state)
    return {"norm": _run_norm, "norm_grad": _run_norm_grad, "linear": _run_linear, "linear_grad": _run_linear_grad,
            "balance": _run_balance, "balance_grad": _run_balance_grad, "adamw": _run_adamw}[state["case"]["op"]](state)


def work(case):
    c, op = case, case["op"]
    if op == "adamw":
        each = 8 + BYTES[c["grad"]] + (16 if c["bits"] == 32 else 4 + 16 / BLOCK)
        if c["copy"] != "none":
            each += 2
        if c["clip"]:  # the norm of all is known before the first is used
            each += BYTES[c["grad"]]
        total = sum(_sizes(c))
        return {"bytes": total * each, "flops": 15 * total}
    m, b = c["kept"], BYTES[c["dtype"]]
    if op == "norm":
        return {"bytes": m * c["d"] * 2 * b + 8 * m + (8 * c["d"] if c["affine"] else 0), "flops": 7 * m * c["d"]}
    if op == "norm_grad":
        return {"bytes": m * c["d"] * b * (4 if c["residual"] else 3) + 8 * m + (12 * c["d"] if c["affine"] else 0),
                "flops": 13 * m * c["d"]}
    if op == "linear":
        wide = _wide(c)
        out = m * (c["d_out"] * (2 if c["residual"] else 1) + (wide if c["pre"] else 0))
        return {"bytes": b * (m * c["d_in"] + wide * c["d_in"] + out) + (4 * wide if c["bias"] else 0),
                "flops": 2 * m * c["d_in"] * wide}
    if op == "linear_grad":
        wide = _wide(c)
        rows = m * (c["d_out"] + (0 if c["act"] == "none" else wide) + 2 * c["d_in"])
        return {"bytes": b * (rows + 2 * wide * c["d_in"]) + (4 * wide if c["bias"] else 0),
                "flops": 4 * m * c["d_in"] * wide}
    if op == "balance":
        return {"bytes": m * (c["E"] * b + 4 * c["K"]) + 8 * c["E"], "flops": 6 * m * c["E"]}
    return {"bytes": m * (2 * c["E"] * b + (8 * c["K"] if c["route"] else 0)) + 4 * c["E"], "flops": 12 * m * c["E"]}


# ---------------------------------------------------------------------------
# the definitions in 64 bits


def _exact_norm(c, s):
    m, f64 = c["kept"], torch.float64
    x = s["x"][:m].to(f64).requires_grad_(c["op"] == "norm_grad")
    gamma = torch.ones(c["d"], dtype=f64, device="cuda") if s["gamma"] is None else s["gamma"].to(f64)
    beta = torch.zeros_like(gamma) if s["beta"] is None else s["beta"].to(f64)
    if c["op"] == "norm":
        var, mean = torch.var_mean(x, dim=1, correction=0)
        rows = torch.zeros(2, c["n"], dtype=f64, device="cuda")
        rows[0, :m], rows[1, :m] = mean, torch.rsqrt(var + EPS)
        out = torch.zeros(c["n"], c["d"], dtype=f64, device="cuda")
        out[:m] = torch.addcmul(beta, (x - mean[:, None]) * rows[1, :m, None], gamma)
        return {"out": out, "mean": rows[0], "rstd": rows[1]}
    # by differentiation; a slice of the rows at a time
    gamma.requires_grad_(True)
    beta.requires_grad_(True)
    dx, step = torch.zeros(c["n"], c["d"], dtype=f64, device="cuda"), max(1, (1 << 25) // c["d"])
    for lo in range(0, m, step):
        v = s["x"][lo:min(m, lo + step)].to(f64).requires_grad_(True)
        var, mean = torch.var_mean(v, dim=1, correction=0, keepdim=True)
        y = (v - mean) * torch.rsqrt(var + EPS) * gamma + beta
        y.backward(s["dout"][lo:min(m, lo + step)].to(f64))
        dx[lo:lo + v.shape[0]] = v.grad
    if s["residual"] is not None:
        dx[:m] += s["residual"][:m].to(f64)
    out = {"dx": dx}
    if c["affine"]:
        out.update(dgamma=gamma.grad, dbeta=beta.grad)
    return out


def _exact_act(h, act, f):
    F = torch.nn.functional
    if act == "gated":
        gate, up = h.split(f, dim=1)
        return F.silu(gate) * up
    return {"none": lambda v: v, "relu": F.relu, "silu": F.silu, "gelu": lambda v: F.gelu(v, approximate="tanh")}[act](h)


def _exact_linear(c, s):
    m, f64 = c["kept"], torch.float64
    x, w = s["x"][:m].to(f64), s["w"].to(f64)
    whole = lambda v: torch.cat([v, torch.zeros(c["n"] - m, v.shape[1], dtype=f64, device="cuda")])
    if c["op"] == "linear":
        h = torch.matmul(w, x.t()).t()
        if s["bias"] is not None:
            h = h + s["bias"].to(f64)
        y = _exact_act(h, c["act"], c["d_out"])
        out = {"out": whole(y if s["residual"] is None else y + s["residual"][:m].to(f64))}
        if c["pre"]:
            out["pre"] = whole(h)
        return out
    d = s["dout"][:m].to(f64)
    if s["pre"] is not None:
        h = s["pre"][:m].to(f64).requires_grad_(True)
        _exact_act(h, c["act"], c["d_out"]).backward(d)
        d = h.grad
    out = {"dx": whole(torch.matmul(w.t(), d.t()).t()), "dw": torch.matmul(x.t(), d).t()}
    if c["bias"]:
        out["dbias"] = torch.ones(1, m, dtype=f64, device="cuda").matmul(d)[0]
    return out


def _exact_balance(c, s):
    m, E, f64 = c["kept"], c["E"], torch.float64
    x = s["logits"][:m].to(f64)
    gone = torch.isinf(x)  # the inputs hold no +inf
    empty = gone.all(1)
    x = x.masked_fill(gone, -1e4).requires_grad_(True)
    soft = torch.softmax(x, 1).masked_fill(gone, 0.0)
    score = soft if c["score"] == "softmax" else torch.sigmoid(x).masked_fill(gone, 0.0)
    total = score.sum(1, keepdim=True)
    p = score / total.masked_fill(total == 0, 1.0)
    lse = torch.logsumexp(x, 1).masked_fill(empty, 0.0)
    pairs = s["ids"][:m].reshape(-1)
    counts = torch.stack([(pairs == e).sum() for e in range(E)]).to(torch.int32)
    share = p.sum(0) / m
    loss = torch.stack([s["coef"] * E * (counts.to(f64) / (m * c["K"]) * share).sum(),
                        s["z_coef"] * lse.square().sum() / m])
    if c["op"] == "balance":
        return {"counts": counts, "share": share.detach(), "loss": loss.detach()}
    value = (loss * s["dloss"].to(f64)).sum()
    if s["dweights"] is not None:
        ids = s["ids"][:m].long()
        weights = torch.where(ids >= 0, score.gather(1, ids.clamp(min=0)), 0.0)
        if c["renorm"]:
            sums = weights.sum(1, keepdim=True)
            weights = weights / sums.masked_fill(sums == 0, 1.0)
        value = value + (weights * s["dweights"][:m].to(f64)).sum()
    value.backward()
    out = torch.zeros(c["n"], E, dtype=f64, device="cuda")
    out[:m] = x.grad.masked_fill(gone, 0.0)
    return {"dlogits": out}


def _exact_draws(s, t):
    """The generator again, its products in 16-bit halves."""
    low = 0xFFFF
    first = torch.arange(BLOCK // 8, device="cuda")[None] + s["inside"][:, None] * (BLOCK // 8)
    word = [first, (s["tensor"][:, None] + (1 << 31)) + 0 * first, torch.full_like(first, t), torch.zeros_like(first)]
    key = [ROUND_SEED % (1 << 32), ROUND_SEED // (1 << 32)]

    def times(a, m):
        x0, x1, m0, m1 = a & low, a >> 16, m & low, m >> 16
        mid = x1 * m0 + (x0 * m0 >> 16)
        mid2 = x0 * m1 + (mid & low)
        return x1 * m1 + (mid >> 16) + (mid2 >> 16), ((mid2 & low) << 16) | (x0 * m0 & low)

    for r in range(10):
        (ah, al), (bh, bl) = times(word[0], 0xD2511F53), times(word[2], 0xCD9E8D57)
        word = [bh ^ word[1] ^ ((key[0] + r * 0x9E3779B9) % (1 << 32)), bl,
                ah ^ word[3] ^ ((key[1] + r * 0xBB67AE85) % (1 << 32)), al]
    return torch.stack([h for w in word for h in (w & low, w >> 16)], dim=2).reshape(-1, BLOCK).to(torch.float64) / 65536


def _exact_codes(x, u, floor_at_one):
    """Between which two of the format's values, and past which of them the draw leads."""
    values = [k / 512 for k in range(8)] + [(1 + k / 8) * 2.0 ** e for e in range(-6, 9) for k in range(8)]
    values = torch.tensor([v for v in values if v <= 448], dtype=torch.float64, device="cuda")
    most = x.abs().max(1, keepdim=True).values
    power = torch.floor(torch.log2(most.clamp(min=1e-300)))
    power = power + (torch.exp2(power + 1) <= most) - (torch.exp2(power) > most).to(torch.float64)
    scale = torch.exp2((power - 7).clamp(min=-126)) * (most > 0)
    a = x.abs() / torch.where(scale > 0, scale, 1.0)
    at = (torch.searchsorted(values, a, right=True) - 1).clamp(max=values.numel() - 2)
    lo, hi = values[at], values[at + 1]
    code = torch.where((a - lo) / (hi - lo) + u >= 1, hi, lo)
    if floor_at_one:
        code = torch.where(a > 0, code.clamp(min=1 / 512), code)
    return (code * torch.sign(x)).reshape(-1), scale.reshape(-1)


def _exact_adamw(c, s):
    f64, one = torch.float64, lambda v: float(torch.tensor(v, dtype=torch.float32))
    b1, b2, t = one(BETA1), one(BETA2), int(s["t"].item()) + 1
    rate, decay, eps = one(LR), one(DECAY), one(ADAM_EPS)
    g, blocks = s["grad"].to(f64), (-1, BLOCK)
    out = {}
    if c["clip"]:
        norm = torch.linalg.vector_norm(g)
        factor = (MAX_NORM / norm).clamp(max=1.0)
        out["norm"] = torch.stack([norm, factor])
        g = g * factor
    m, v = s["m"].to(f64), s["v"].to(f64)
    if c["bits"] == 8:
        m = (m.view(blocks) * s["m_scale"].to(f64)[:, None]).view(-1)
        v = (v.view(blocks) * s["v_scale"].to(f64)[:, None]).view(-1).square()
    m = torch.lerp(g, m, b1)
    v = torch.lerp(g.square(), v, b2)
    step = (m / (1 - b1 ** t)) / ((v / (1 - b2 ** t)).sqrt() + eps)
    shrink = 1 - rate * decay * s["decay"].to(f64).expand(-1, BLOCK).reshape(-1)
    out["param"] = s["param"].to(f64) * shrink - rate * step
    if s["copy"] is not None:
        out["copy"] = out["param"]
    if c["bits"] == 8:
        u = _exact_draws(s, t)
        out["m"], out["m_scale"] = _exact_codes(m.view(blocks), u, False)
        out["v"], out["v_scale"] = _exact_codes(v.sqrt().view(blocks), u, True)
    else:
        out["m"], out["v"] = m, v
    out["t"] = torch.full_like(s["t"], t)
    return out


def exact(case, seed):
    s = _inputs(case, seed)
    return {"norm": _exact_norm, "linear": _exact_linear, "balance": _exact_balance,
            "adamw": _exact_adamw}[case["op"].replace("_grad", "")](case, s)
