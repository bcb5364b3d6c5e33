"""A Boss with blocks of experts: weights, buffers and the order of the library's calls.

The paper's Boss is whatever model the kept rows train (Algorithm 3).  ExpertBlock is a residual feed-forward block of gated
experts with a router and dropout, on request with a norm before it and with the router's balance loss; Boss puts an input
layer, such blocks, a last norm and a read-out together; AdamW updates the weights of either.  Everything a step decides -- how many rows there are, who gets which -- stays
on the device: `count` is the kept count as aa_score_shrink left it.  Nothing here synchronises, and after the
first step nothing allocates on the library's side, so a step can be captured into a graph (the seeds are then fixed).
"""
import torch

from . import api


class Norm:
    """Layer norm of up to n_max rows: its result, the rows' statistics, and weights gamma, beta in fp32."""

    def __init__(self, n_max, d, dtype=torch.bfloat16, device="cuda", eps=1e-5):
        f32 = lambda n: torch.zeros(n, device=device)
        self.eps, self.n_max = eps, n_max
        self.gamma, self.beta, self.mean, self.rstd = f32(d) + 1, f32(d), f32(n_max), f32(n_max)
        self.grads = [f32(d), f32(d)]
        self.out = torch.zeros(n_max, d, dtype=dtype, device=device)
        self.ws = api.LayerWorkspace(d, device=device)

    def weights(self):
        return [self.gamma, self.beta]

    def forward(self, x, count):
        api.layer_norm(x[:self.n_max], self.gamma, self.beta, self.eps, count, self.out, self.mean, self.rstd)
        return self.out

    def backward(self, x, count, dout, residual, dx):
        """residual: the gradient that is added to x's, or None."""
        residual = None if residual is None else residual[:self.n_max]
        api.layer_norm_grad(dout[:self.n_max], x[:self.n_max], self.gamma, self.mean, self.rstd, residual, count, dx,
                            *self.grads, False, self.ws)


def _need_kept(part):
    if not part.kept:
        raise api.AAError("backward: what the last forward kept is needed, and it ran without train=True or not at all")


class Dense:
    """act(w x + bias) for up to n_max rows: w [d_out, d_in] (gated: [2 d_out, d_in]) in dtype, bias in fp32."""

    def __init__(self, n_max, d_in, d_out, act="none", dtype=torch.bfloat16, seed=1905, device="cuda"):
        z = lambda *s, t=dtype: torch.zeros(*s, dtype=t, device=device)
        wide = 2 * d_out if act == "gated" else d_out
        g = torch.Generator(device=device)
        g.manual_seed(seed)
        self.n_max, self.act, self.kept = n_max, act, False
        self.w = (torch.randn(wide, d_in, generator=g, device=device) * d_in ** -0.5).to(dtype)
        self.bias = z(wide, t=torch.float32)
        self.grads = [z(wide, d_in, t=torch.float32), z(wide, t=torch.float32)]
        self.pre = None if act == "none" else z(n_max, wide)
        self.dpre = None if act == "none" else z(n_max, wide)
        self.one = z(2, t=torch.int32)   # the rows as a single group, for the gradients' products
        self.ws = api.LayerWorkspace(wide, device=device)
        self.product_ws = api.ExpertWorkspace(n_max, 1, 1, device=device)

    def weights(self):
        return [self.w, self.bias]

    def _rows(self, x, name):
        """The rows that a call of up to n_max may use: they must all be there, whatever the count says."""
        if x.shape[0] < self.n_max:
            raise api.AAError(f"{name}: {x.shape[0]} rows where {self.n_max} are needed")
        return x[:self.n_max]

    def forward(self, x, count, out, train=True):
        """train=False: nothing is kept for backward."""
        self.kept = False
        api.linear(self._rows(x, "x"), self.w, self.bias, self.act, None, count, out, self.pre if train else None)
        self.kept = train

    def backward(self, x, count, dout, dx=None):
        """Gradients of the last forward of the same x and count, which was one with train=True: self.grads, and of x into dx."""
        _need_kept(self)
        x, dout = self._rows(x, "x"), self._rows(dout, "dout")
        api.linear_grad(dout, self.act, self.pre, count, self.dpre, self.grads[1], False, self.ws)
        dpre = dout if self.dpre is None else self.dpre
        self.one[1:].copy_(count.clamp(0, self.n_max))
        api.expert_grad_weight(dpre, x, None, 1, self.one, self.grads[0][None], False, self.product_ws)
        if dx is not None:
            api.expert_grad_input(dpre, self.one, self.w[None], "none", None, self._rows(dx, "dx"))


class ExpertBlock:
    """out = x + dropout(sum_k weight_k expert_k(x)),  expert(x) = down silu(gate x) * (up x),  bf16 or f16.

    Weights: router [1, E, d], gate_up [E, 2 f, d], down [E, d, f]; gradients of the same shapes in fp32.  seed makes the first
    weights and, with the step, the masks: blocks of one model take seeds of their own.  Logits are rounded to dtype before
    they are routed: those that tie in it go to the lowest index.
    Rows [0, min(max(count, 0), n_max)) take part in a step; x, out, dout and dx have n_max rows or more, of which those
    at and beyond n_max are neither read nor written.

    norm: the router and the experts get norm(x) (eps 1e-5; weights gamma, beta [d] in fp32 behind the others) in the place
    of x, the residual stays x.  balance, z_loss: coefficients of the balance loss and of the loss on the logits' size; forward
    with train=True then leaves both in balance_loss, the experts' choices and shares in counts and share, and backward takes
    their gradient along.
    """

    def __init__(self, n_max, d, f, n_experts, top_k, dtype=torch.bfloat16, p=0.0, score="softmax", seed=1905,
                 device="cuda", norm=False, balance=0.0, z_loss=0.0, **routing):
        z = lambda *s, t=dtype: torch.zeros(*s, dtype=t, device=device)
        i32, f32, E, R = torch.int32, torch.float32, n_experts, n_max * top_k
        self.n_max, self.top_k, self.p, self.seed = n_max, top_k, p, seed
        routing.setdefault("renormalise", True)
        self.cfg = api.route_config(score, top_k, **routing)
        g = torch.Generator(device=device)
        g.manual_seed(seed)
        init = lambda *s: (torch.randn(*s, generator=g, device=device) * s[-1] ** -0.5).to(dtype)
        self.router, self.gate_up, self.down = init(1, E, d), init(E, 2 * f, d), init(E, d, f)
        self.norm = Norm(n_max, d, dtype, device) if norm else None
        self.balance = (balance, z_loss) if balance or z_loss else None
        if self.balance:
            self.counts, self.share, self.balance_loss = z(E, t=i32), z(E, t=f32), z(2, t=f32)
            self.balance_ws = api.LayerWorkspace(E, device=device)
        self.grads = [torch.zeros_like(w, dtype=f32) for w in self.weights()]
        if norm:
            self.norm.grads = self.grads[3:]
        self.one = z(2, t=i32)                       # the rows as a single group, for the router's product
        self.ids, self.route_weights = z(n_max, top_k, t=i32), z(n_max, top_k, t=f32)
        self.plan = (z(E + 1, t=i32), z(R, t=i32), z(n_max, top_k, t=i32))
        self.logits, self.h, self.pre, self.y = z(n_max, E), z(R, f), z(R, 2 * f), z(R, d)
        self.dy, self.dpre, self.dx_pairs = z(R, d), z(R, 2 * f), z(R, d)
        self.dweights, self.dlogits = z(n_max, top_k, t=f32), z(n_max, E)
        self.dx_router = z(n_max, d)
        # whether the buffers hold what backward needs (who replays a forward from a graph and calls backward outside it
        # sets this)
        self.kept = False
        self.ws = api.ExpertWorkspace(n_max, top_k, E, device=device)

    def weights(self):
        return [self.router, self.gate_up, self.down] + (self.norm.weights() if self.norm else [])

    def forward(self, x, count, step, out, train=True):
        """Rows in use of x into out; train=False: no dropout, and nothing is kept for backward (what an earlier
        call kept is gone, too)."""
        offsets, order, slot = self.plan
        p = self.p if train else 0.0
        self.kept = False
        residual = x
        if self.norm:
            x = self.norm.forward(x, count)
        # (the products go by the group's end alone: it must lie inside the block's own buffers)
        self.one[1:].copy_(count.clamp(0, self.n_max))
        api.expert_forward(x, None, 1, self.one, self.router, "none", self.logits)
        api.route(self.logits, count, None, self.cfg, self.ids, self.route_weights, self.plan, self.ws)
        api.expert_forward(x, order, self.top_k, offsets, self.gate_up, "gated", self.h, self.pre if train else None)
        api.expert_forward(self.h, None, 1, offsets, self.down, "none", self.y)
        api.expert_combine(self.y, slot, self.route_weights, count, residual, p, self.seed, step, out)
        if train and self.balance:
            api.balance(self.logits, count, self.cfg, self.ids, *self.balance, self.counts, self.share, self.balance_loss,
                        self.balance_ws)
        self.kept = train

    def backward(self, x, count, step, dout, dx, loss_scale=None):
        """Gradients of the last forward of the same x, count and step, which was one with train=True: self.grads, and of x
        into dx.  loss_scale: a float32 tensor of one, the factor that dout has been given (None: 1); the balance losses'
        gradients are given it, too.  In f16 they need one: of a pool of thousands of rows a logit's is below the type's
        smallest step."""
        _need_kept(self)
        offsets, order, slot = self.plan
        d_router, d_gate_up, d_down = self.grads[:3]
        below = x
        if self.norm:
            x = self.norm.out
        api.expert_combine_grad(dout, self.y, slot, self.route_weights, count, self.p, self.seed, step, self.dy,
                                self.dweights)
        api.expert_grad_weight(self.dy, self.h, None, 1, offsets, d_down, False, self.ws)
        api.expert_grad_input(self.dy, offsets, self.down, "gated", self.pre, self.dpre)
        api.expert_grad_weight(self.dpre, x, order, self.top_k, offsets, d_gate_up, False, self.ws)
        api.expert_grad_input(self.dpre, offsets, self.gate_up, "none", None, self.dx_pairs)
        if self.balance:
            api.balance_grad(self.logits, count, self.cfg, self.ids, self.dweights, self.counts, *self.balance, loss_scale,
                             self.dlogits)
        else:
            api.route_grad(self.logits, count, self.cfg, self.ids, self.dweights, self.dlogits)
        api.expert_grad_weight(self.dlogits, x, None, 1, self.one, d_router, False, self.ws)
        api.expert_grad_input(self.dlogits, self.one, self.router, "none", None, self.dx_router)
        if self.norm:  # the router and the pairs, through the norm, and the residual
            api.expert_combine(self.dx_pairs, slot, None, count, self.dx_router, 0.0, 0, 0, self.dx_router)
            self.norm.backward(below, count, self.dx_router, dout, dx)
            return
        # the block's input: the residual, the router and the pairs
        api.dropout(self.dx_router, count, dout, 0.0, 0, 0, dx)
        api.expert_combine(self.dx_pairs, slot, None, count, dx, 0.0, 0, 0, dx)


class Boss:
    """out = read-out(norm(blocks(input layer(x)))): features [., d_in] to [., d_out] by `layers` normed blocks of width d.

    Takes part in a step as ExpertBlock does: the first min(max(count, 0), n_max) rows.  options: those of ExpertBlock.
    """

    def __init__(self, n_max, d_in, d, f, d_out, n_experts, top_k, layers=2, dtype=torch.bfloat16, seed=1905,
                 device="cuda", **options):
        z = lambda w: torch.zeros(n_max, w, dtype=dtype, device=device)
        self.n_max = n_max
        self.enter = Dense(n_max, d_in, d, "gelu", dtype, seed, device)
        # (seeds: masks and first weights of each block are its own)
        self.blocks = [ExpertBlock(n_max, d, f, n_experts, top_k, dtype, seed=seed + 1 + i, device=device, norm=True, **options)
                       for i in range(layers)]
        self.norm = Norm(n_max, d, dtype, device)
        self.leave = Dense(n_max, d, d_out, "none", dtype, seed + 1 + layers, device)
        self.x = [z(d) for _ in range(layers + 1)]   # what goes into each block, and out of the last
        self.dx, self.dnorm = [z(d), z(d)], z(d)

    def parts(self):
        return [self.enter] + self.blocks + [self.norm, self.leave]

    def weights(self):
        return [w for part in self.parts() for w in part.weights()]

    @property
    def grads(self):
        return [g for part in self.parts() for g in part.grads]

    def forward(self, x, count, step, out, train=True):
        self.enter.forward(x, count, self.x[0], train)
        for block, below, above in zip(self.blocks, self.x, self.x[1:]):
            block.forward(below, count, step, above, train)
        self.leave.forward(self.norm.forward(self.x[-1], count), count, out, train)

    def backward(self, x, count, step, dout, loss_scale=None):
        """Gradients of the last forward of the same x, count and step, which was one with train=True, into grads; loss_scale as
        in ExpertBlock."""
        for part in [self.enter] + self.blocks + [self.leave]:  # (before any gradient is written)
            _need_kept(part)
        here, there = self.dx
        self.leave.backward(self.norm.out, count, dout, self.dnorm)
        self.norm.backward(self.x[-1], count, self.dnorm, None, here)
        for block, below in zip(self.blocks[::-1], self.x[-2::-1]):
            block.backward(below, count, step, here, there, loss_scale)
            here, there = there, here
        self.enter.backward(x, count, here)


class AdamW:
    """Updates of a model's weights (ExpertBlock, Boss: weights() and grads) by one launch, or two with clipping.

    Weights of 16 bits have an fp32 copy that is updated and from which they are rounded; vectors take no weight decay and keep
    states of 32 bits, the others of state_bits (8 or 32).  t counts the updates on the device; norm holds the gradients' norm
    and the factor they were taken with."""

    def __init__(self, model, lr, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.0, max_norm=None, state_bits=32, seed=0):
        if state_bits not in (8, 32):
            raise api.AAError(f"state_bits: {state_bits!r} is neither 8 nor 32")
        self.cfg, self.max_norm = api.adamw_config(lr, beta1, beta2, eps, weight_decay, seed), max_norm
        self.masters, self.states, tensors = [], [], []
        for w, g in zip(model.weights(), model.grads):
            master, vector = (w if w.dtype == torch.float32 else w.float()), w.dim() == 1
            z = lambda n, t: torch.zeros(n, dtype=t, device=w.device)
            if vector or state_bits == 32:
                state = dict(m=z(w.numel(), torch.float32), v=z(w.numel(), torch.float32))
            else:
                blocks = -(-w.numel() // api.STATE_BLOCK)
                state = dict(m=z(w.numel(), torch.uint8).view(torch.float8_e4m3fn),
                             v=z(w.numel(), torch.uint8).view(torch.float8_e4m3fn),
                             m_scale=z(blocks, torch.float32), v_scale=z(blocks, torch.float32))
            self.masters.append(master)
            self.states.append(state)
            tensors.append(api.adamw_tensor(master, g, copy=None if master is w else w, decay=0.0 if vector else 1.0, **state))
        device = self.masters[0].device
        self.table = api.AdamWTable(tensors, device=device)
        self.t, self.norm = torch.zeros(1, dtype=torch.int32, device=device), torch.zeros(2, device=device)

    def step(self, count=None, lr_factor=None, grad_scale=None):
        """count: the batch's rows, with none of them nothing changes; lr_factor, grad_scale: float32 tensors of one, factors
        of the step size and of the gradients (1 / loss_scale after a backward that had one)."""
        factor = grad_scale
        if self.max_norm is not None:
            api.grad_norm(self.table, self.max_norm, grad_scale, self.norm)
            factor = self.norm[1:]
        api.adamw_step(self.table, self.cfg, lr_factor, factor, count, self.t)
