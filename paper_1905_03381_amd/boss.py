"""A Boss with a block of experts: weights, buffers and the order of the library's calls.

The paper's Boss is whatever model the kept rows train (Algorithm 3); this one is a residual feed-forward block of gated
experts with a router and dropout.  Everything a step decides -- how many rows there are, who gets which -- stays
on the device: `count` is the kept count as aa_score_shrink left it.  Nothing here synchronises, and after the
first step nothing allocates on the library's side, so a step can be captured into a graph (the seeds are then fixed).
"""
import torch

from . import api


class ExpertBlock:
    """out = x + dropout(sum_k weight_k expert_k(x)),  expert(x) = down silu(gate x) * (up x),  bf16 or f16.

    Weights: router [1, E, d], gate_up [E, 2 f, d], down [E, d, f]; gradients of the same shapes in fp32.  seed makes the first
    weights and, with the step, the masks: blocks of one model take seeds of their own.  Logits are rounded to dtype before
    they are routed: those that tie in it go to the lowest index.
    Rows [0, min(max(count, 0), n_max)) take part in a step; x, out, dout and dx have n_max rows or more, of which those
    at and beyond n_max are neither read nor written.
    """

    def __init__(self, n_max, d, f, n_experts, top_k, dtype=torch.bfloat16, p=0.0, score="softmax", seed=1905,
                 device="cuda", **routing):
        z = lambda *s, t=dtype: torch.zeros(*s, dtype=t, device=device)
        i32, f32, E, R = torch.int32, torch.float32, n_experts, n_max * top_k
        self.n_max, self.top_k, self.p, self.seed = n_max, top_k, p, seed
        routing.setdefault("renormalise", True)
        self.cfg = api.route_config(score, top_k, **routing)
        g = torch.Generator(device=device)
        g.manual_seed(seed)
        init = lambda *s: (torch.randn(*s, generator=g, device=device) * s[-1] ** -0.5).to(dtype)
        self.router, self.gate_up, self.down = init(1, E, d), init(E, 2 * f, d), init(E, d, f)
        self.grads = [torch.zeros_like(w, dtype=f32) for w in self.weights()]
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
        return [self.router, self.gate_up, self.down]

    def forward(self, x, count, step, out, train=True):
        """Rows in use of x into out; train=False: no dropout, and nothing is kept for backward (what an earlier
        call kept is gone, too)."""
        offsets, order, slot = self.plan
        p = self.p if train else 0.0
        self.kept = False
        # (the products go by the group's end alone: it must lie inside the block's own buffers)
        self.one[1:].copy_(count.clamp(0, self.n_max))
        api.expert_forward(x, None, 1, self.one, self.router, "none", self.logits)
        api.route(self.logits, count, None, self.cfg, self.ids, self.route_weights, self.plan, self.ws)
        api.expert_forward(x, order, self.top_k, offsets, self.gate_up, "gated", self.h, self.pre if train else None)
        api.expert_forward(self.h, None, 1, offsets, self.down, "none", self.y)
        api.expert_combine(self.y, slot, self.route_weights, count, x, p, self.seed, step, out)
        self.kept = train

    def backward(self, x, count, step, dout, dx):
        """Gradients of the last forward of the same x, count and step, which was one with train=True: self.grads, and of x
        into dx."""
        if not self.kept:
            raise api.AAError("backward: what the last forward kept is needed, and it ran without train=True or not at all")
        offsets, order, slot = self.plan
        d_router, d_gate_up, d_down = self.grads
        api.expert_combine_grad(dout, self.y, slot, self.route_weights, count, self.p, self.seed, step, self.dy,
                                self.dweights)
        api.expert_grad_weight(self.dy, self.h, None, 1, offsets, d_down, False, self.ws)
        api.expert_grad_input(self.dy, offsets, self.down, "gated", self.pre, self.dpre)
        api.expert_grad_weight(self.dpre, x, order, self.top_k, offsets, d_gate_up, False, self.ws)
        api.expert_grad_input(self.dpre, offsets, self.gate_up, "none", None, self.dx_pairs)
        api.route_grad(self.logits, count, self.cfg, self.ids, self.dweights, self.dlogits)
        api.expert_grad_weight(self.dlogits, x, None, 1, self.one, d_router, False, self.ws)
        api.expert_grad_input(self.dlogits, self.one, self.router, "none", None, self.dx_router)
        # the block's input: the residual, the router and the pairs
        api.dropout(self.dx_router, count, dout, 0.0, 0, 0, dx)
        api.expert_combine(self.dx_pairs, slot, None, count, dx, 0.0, 0, 0, dx)
