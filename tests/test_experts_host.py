"""Refusals of the expert operators: every one is decided on the host before anything is launched, so these
run without a GPU.  The pointers handed over are never read."""
import ctypes as C

import pytest

from paper_1905_03381_amd import api

OK, NULL, SHAPE, ALIGN, WORKSPACE = 0, -1, -2, -3, -4
P = 0x10000  # stands for a device pointer, aligned to everything
F32, BF16, F16 = 0, 1, 2


@pytest.fixture(scope="module")
def L():
    import os
    if not os.path.exists(api.LIB_PATH):
        from paper_1905_03381_amd import build
        build.build(force=False)
    return api.lib()


def cfg(**change):
    c = api.route_config("softmax", 4)
    for k, v in change.items():
        setattr(c, k, v)
    return c


def call(fn, defaults, change):
    args = dict(defaults)
    assert set(change) <= set(args), change
    args.update(change)
    return fn(*args.values())


BIG = 1 << 40

ROUTE = dict(logits=P, dtype=F32, ld=16, count=None, n_max=8, n_experts=16, bias=None, cfg=cfg(), ids=P, weights=P,
             offsets=P, order=P, slot=P, ws=P, ws_bytes=BIG, stream=None)
ROUTE_GRAD = dict(logits=P, dtype=F32, ld=16, count=None, n_max=8, n_experts=16, cfg=cfg(), ids=P, dweights=P,
                  dlogits=P, ld_out=16, stream=None)
PLAN = dict(ids=P, count=None, n_max=8, top_k=4, n_experts=16, offsets=P, order=P, slot=P, ws=P, ws_bytes=BIG,
            stream=None)
FORWARD = dict(x=P, dtype=BF16, ldx=32, order=P, top_k=4, offsets=P, rows_max=32, n_experts=16, d_in=32, d_out=24,
               w=P, act=0, out=P, ldo=24, pre=None, ldpre=0, stream=None)
GRAD_INPUT = dict(dout=P, dtype=BF16, lddo=24, offsets=P, rows_max=32, n_experts=16, d_in=32, d_out=24, w=P, act=0,
                  saved=None, lds=0, dx=P, lddx=32, stream=None)
GRAD_WEIGHT = dict(dout=P, dtype=BF16, lddo=24, x=P, ldx=32, order=P, top_k=4, offsets=P, rows_max=32, n_experts=16,
                   d_in=32, d_out=24, dw=P, out_dtype=F32, accumulate=0, ws=P, ws_bytes=BIG, stream=None)
DROPOUT = dict(x=P, dtype=F32, ldx=32, count=None, n_max=8, d=32, residual=None, ldr=0, p=0.1, seed=1, step=2, out=P,
               ldo=32, stream=None)
COMBINE = dict(y=P, dtype=F32, ldy=32, slot=P, weights=P, count=None, n_max=8, top_k=4, d=32, residual=None, ldr=0,
               p=0.1, seed=1, step=2, out=P, ldo=32, stream=None)
COMBINE_GRAD = dict(dout=P, dtype=F32, lddo=32, y=P, ldy=32, slot=P, weights=P, count=None, n_max=8, top_k=4, d=32,
                    p=0.1, seed=1, step=2, dy=P, lddy=32, dweights=P, stream=None)

REFUSED = [
    ("aa_route", ROUTE, [
        (dict(logits=None), NULL), (dict(cfg=None), NULL), (dict(ids=None), NULL), (dict(weights=None), NULL),
        (dict(order=None), NULL), (dict(slot=None), NULL), (dict(offsets=None), NULL),
        (dict(dtype=3), SHAPE), (dict(dtype=-1), SHAPE), (dict(ld=15), SHAPE), (dict(n_max=-1), SHAPE),
        (dict(n_experts=0), SHAPE), (dict(n_experts=1025, ld=2000), SHAPE), (dict(n_max=1 << 30), SHAPE),
        (dict(cfg=cfg(top_k=0)), SHAPE), (dict(cfg=cfg(top_k=17)), SHAPE), (dict(cfg=cfg(top_k=65)), SHAPE),
        (dict(cfg=cfg(score=2)), SHAPE), (dict(cfg=cfg(n_groups=3)), SHAPE), (dict(cfg=cfg(n_groups=0)), SHAPE),
        (dict(cfg=cfg(n_groups=4, top_groups=5)), SHAPE), (dict(cfg=cfg(top_groups=0)), SHAPE),
        (dict(cfg=cfg(n_groups=8, top_groups=1)), SHAPE), (dict(cfg=cfg(group_best=3)), SHAPE),
        (dict(cfg=cfg(group_best=0)), SHAPE), (dict(cfg=cfg(scale=float("nan"))), SHAPE),
        (dict(cfg=cfg(scale=float("inf"))), SHAPE),
        (dict(logits=P + 2), ALIGN), (dict(logits=P + 1, dtype=BF16), ALIGN), (dict(ids=P + 2), ALIGN),
        (dict(bias=P + 1), ALIGN), (dict(count=P + 3), ALIGN),
        (dict(ws=None), WORKSPACE), (dict(ws=P + 128), WORKSPACE), (dict(ws_bytes=0), WORKSPACE)]),
    ("aa_route_grad", ROUTE_GRAD, [
        (dict(dlogits=None), NULL), (dict(dweights=None), NULL), (dict(ids=None), NULL), (dict(cfg=None), NULL),
        (dict(ld_out=15), SHAPE), (dict(dtype=7), SHAPE), (dict(n_max=-5), SHAPE), (dict(dlogits=P + 1), ALIGN)]),
    ("aa_expert_plan", PLAN, [
        (dict(ids=None), NULL), (dict(offsets=None), NULL), (dict(order=None), NULL), (dict(top_k=0), SHAPE),
        (dict(top_k=65), SHAPE), (dict(n_experts=0), SHAPE), (dict(n_experts=1025), SHAPE), (dict(n_max=-1), SHAPE),
        (dict(ws=None), WORKSPACE), (dict(ws_bytes=256), WORKSPACE), (dict(slot=P + 2), ALIGN)]),
    ("aa_expert_forward", FORWARD, [
        (dict(x=None), NULL), (dict(w=None), NULL), (dict(out=None), NULL), (dict(offsets=None), NULL),
        (dict(dtype=F32), SHAPE), (dict(act=3), SHAPE), (dict(pre=P, ldpre=48), SHAPE), (dict(top_k=0), SHAPE),
        (dict(ldx=31), SHAPE), (dict(ldo=23), SHAPE), (dict(d_in=0), SHAPE), (dict(d_out=0), SHAPE),
        (dict(rows_max=-1), SHAPE), (dict(act=2, pre=P, ldpre=47), SHAPE), (dict(ldx=(1 << 40) + 1), SHAPE),
        (dict(x=P + 1), ALIGN), (dict(w=P + 1), ALIGN), (dict(out=P + 1), ALIGN), (dict(order=P + 2), ALIGN)]),
    ("aa_expert_grad_input", GRAD_INPUT, [
        (dict(dout=None), NULL), (dict(dx=None), NULL), (dict(act=1, lds=32), NULL), (dict(act=2, lddx=64, lds=64), NULL),
        (dict(act=2, saved=P, lds=64), SHAPE), (dict(act=1, saved=P, lds=31), SHAPE), (dict(lddo=23), SHAPE),
        (dict(dtype=F32), SHAPE), (dict(n_experts=0), SHAPE), (dict(w=P + 1), ALIGN)]),
    ("aa_expert_grad_weight", GRAD_WEIGHT, [
        (dict(dout=None), NULL), (dict(x=None), NULL), (dict(dw=None), NULL), (dict(offsets=None), NULL),
        (dict(out_dtype=F16), SHAPE), (dict(dtype=F32), SHAPE), (dict(top_k=65), SHAPE), (dict(ldx=16), SHAPE),
        (dict(dw=P + 2), ALIGN), (dict(ws=None), WORKSPACE), (dict(ws_bytes=1024), WORKSPACE)]),
    ("aa_dropout", DROPOUT, [
        (dict(x=None), NULL), (dict(out=None), NULL), (dict(p=-0.1), SHAPE), (dict(p=1.5), SHAPE),
        (dict(p=float("nan")), SHAPE), (dict(d=0), SHAPE), (dict(n_max=-1), SHAPE), (dict(dtype=9), SHAPE),
        (dict(residual=P, ldr=31), SHAPE), (dict(ldx=8), SHAPE), (dict(x=P + 2), ALIGN), (dict(residual=P + 1, ldr=32), ALIGN)]),
    ("aa_expert_combine", COMBINE, [
        (dict(y=None), NULL), (dict(slot=None), NULL), (dict(out=None), NULL), (dict(top_k=0), SHAPE),
        (dict(top_k=65), SHAPE), (dict(p=2.0), SHAPE), (dict(ldo=31), SHAPE), (dict(weights=P + 1), ALIGN)]),
    ("aa_expert_combine_grad", COMBINE_GRAD, [
        (dict(y=None), NULL), (dict(dout=None), NULL), (dict(dy=None), NULL), (dict(slot=None), NULL),
        (dict(lddy=31), SHAPE), (dict(d=0), SHAPE), (dict(dweights=P + 2), ALIGN)]),
]


@pytest.mark.parametrize("name,defaults,change,status",
                         [(n, d, c, s) for n, d, rows in REFUSED for c, s in rows],
                         ids=[f"{n}-{'-'.join(c)}-{i}" for n, _, rows in REFUSED for i, (c, _) in enumerate(rows)])
def test_refusals(L, name, defaults, change, status):
    args = {k: C.byref(v) if isinstance(v, api.aa_route_config) else v for k, v in defaults.items()}
    new = {k: C.byref(v) if isinstance(v, api.aa_route_config) else v for k, v in change.items()}
    assert call(getattr(L, name), args, new) == status


def test_no_rows_is_not_an_error(L):
    """Nothing to do and nothing to launch: row buffers may then be NULL (an empty tensor's address)."""
    c = C.byref(cfg())
    rows = dict(n_max=0)
    assert call(L.aa_route, {**ROUTE, "cfg": c}, dict(rows, logits=None, ids=None, weights=None, offsets=None,
                                                       order=None, slot=None)) == OK
    assert call(L.aa_route_grad, {**ROUTE_GRAD, "cfg": c}, dict(rows, logits=None, ids=None, dweights=None,
                                                                dlogits=None)) == OK
    assert call(L.aa_dropout, DROPOUT, dict(rows, x=None, out=None)) == OK
    assert call(L.aa_expert_combine, COMBINE, dict(rows, y=None, slot=None, out=None)) == OK
    assert call(L.aa_expert_combine_grad, COMBINE_GRAD, dict(rows, y=None, slot=None, dout=None, dy=None)) == OK
    assert call(L.aa_expert_forward, FORWARD, dict(rows_max=0, x=None, out=None)) == OK
    assert call(L.aa_expert_grad_input, GRAD_INPUT, dict(rows_max=0, dout=None, dx=None)) == OK


def test_workspace_covers_the_plan(L):
    small = L.aa_expert_workspace_bytes(8, 4, 16)
    big = L.aa_expert_workspace_bytes(1 << 20, 8, 1024)
    assert 256 < small <= big
    # a count for every expert and every 2048 pairs
    assert big >= 256 + 4 * 1024 * ((1 << 23) // 2048)
    assert L.aa_expert_workspace_bytes(-1, -1, -1) > 0


def test_config_layout_matches_the_header():
    assert C.sizeof(api.aa_route_config) == 32
    assert api.aa_route_config.scale.offset == 24


def test_names_are_checked():
    with pytest.raises(api.AAError):
        api.route_config("tanh", 2)
