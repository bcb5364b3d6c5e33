"""Refusals of the operators around a Boss block of experts: every one is decided on the host before anything is
launched, so these run without a GPU.  The pointers handed over are never read."""
import pytest
import torch

from paper_1905_03381_amd import api

OK, NULL, SHAPE, ALIGN, WORKSPACE = 0, -1, -2, -3, -4
P = 0x10000  # stands for a device pointer, aligned to everything
F32, BF16, F16 = 0, 1, 2
BIG = 1 << 40
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def L():
    import os
    if not os.path.exists(api.LIB_PATH):
        from paper_1905_03381_amd import build
        build.build(force=False)
    return api.lib()


NORM = dict(x=P, dtype=BF16, ldx=32, count=None, n_max=8, d=32, gamma=P, beta=P, eps=1e-5, out=P, ldo=32, mean=P, rstd=P,
            stream=None)
NORM_GRAD = dict(dout=P, dtype=BF16, lddo=32, x=P, ldx=32, count=None, n_max=8, d=32, gamma=P, mean=P, rstd=P,
                 residual=None, ldr=0, dx=P, lddx=32, dgamma=P, dbeta=P, accumulate=0, ws=P, ws_bytes=BIG, stream=None)

LINEAR = dict(x=P, dtype=BF16, ldx=32, count=None, n_max=8, d_in=32, d_out=24, w=P, bias=P, act=0, residual=None, ldr=0, out=P,
              ldo=24, pre=None, ldpre=0, stream=None)
LINEAR_GRAD = dict(dout=P, dtype=BF16, lddo=24, count=None, n_max=8, d_out=24, act=2, pre=P, ldpre=48, dpre=P, lddp=48,
                   dbias=P, accumulate=0, ws=P, ws_bytes=BIG, stream=None)


def cfg(**change):
    c = api.route_config("softmax", 4)
    for k, v in change.items():
        setattr(c, k, v)
    return c


BALANCE = dict(logits=P, dtype=BF16, ld=16, count=None, n_max=8, n_experts=16, cfg=cfg(), ids=P, coef=0.1, z_coef=0.1,
               counts=P, share=P, loss=P, ws=P, ws_bytes=BIG, stream=None)
BALANCE_GRAD = dict(logits=P, dtype=BF16, ld=16, count=None, n_max=8, n_experts=16, cfg=cfg(), ids=P, dweights=P, counts=P,
                    coef=0.1, z_coef=0.1, dloss=None, dlogits=P, ld_out=16, stream=None)
OF_BOTH = [(dict(logits=None), NULL), (dict(cfg=None), NULL), (dict(dtype=3), SHAPE), (dict(n_max=-1), SHAPE),
           (dict(n_experts=0), SHAPE), (dict(n_experts=1025, ld=1025), SHAPE), (dict(ld=15), SHAPE),
           (dict(cfg=cfg(top_k=0)), SHAPE), (dict(cfg=cfg(top_k=17)), SHAPE), (dict(cfg=cfg(score=2)), SHAPE),
           (dict(cfg=cfg(scale=INF)), SHAPE), (dict(coef=NAN), SHAPE), (dict(z_coef=INF), SHAPE),
           (dict(logits=P + 1), ALIGN), (dict(count=P + 2), ALIGN), (dict(ids=P + 2), ALIGN), (dict(ids=None), NULL),
           (dict(counts=None), NULL), (dict(counts=P + 2), ALIGN)]


def tensors(*changes):
    """A host array of good tensors with changes."""
    out = (api.aa_adamw_tensor * len(changes))()
    for t, change in zip(out, changes):
        for k, v in dict(dict(param=P, grad=P, copy=None, m=P, v=P, m_scale=None, v_scale=None, n=5000, grad_dtype=BF16,
                              copy_dtype=BF16, state_bits=32, decay=1.0), **change).items():
            setattr(t, k, v)
    return out


def opt(**change):
    c = api.adamw_config(1e-3)
    for k, v in change.items():
        setattr(c, k, v)
    return c


GOOD = tensors({}, {})
ONE_BAD = lambda **change: tensors({}, change)
CHUNKS = dict(tensors=GOOD, n_tensors=2)
TABLE = dict(tensors=GOOD, n_tensors=2, table=P, table_bytes=BIG, stream=None)
OF_LIST = [
    (dict(tensors=None), NULL), (dict(n_tensors=0), SHAPE), (dict(n_tensors=-1), SHAPE), (dict(n_tensors=65537), SHAPE),
    (dict(tensors=ONE_BAD(n=-1)), SHAPE), (dict(tensors=ONE_BAD(n=(1 << 35) + 1)), SHAPE),
    (dict(tensors=ONE_BAD(grad_dtype=3)), SHAPE), (dict(tensors=ONE_BAD(copy=P, copy_dtype=F32)), SHAPE),
    (dict(tensors=ONE_BAD(state_bits=16)), SHAPE), (dict(tensors=ONE_BAD(decay=NAN)), SHAPE),
    (dict(tensors=ONE_BAD(param=None)), NULL), (dict(tensors=ONE_BAD(grad=None)), NULL), (dict(tensors=ONE_BAD(m=None)), NULL),
    (dict(tensors=ONE_BAD(v=None)), NULL), (dict(tensors=ONE_BAD(state_bits=8)), NULL),
    (dict(tensors=ONE_BAD(state_bits=8, m_scale=P)), NULL), (dict(tensors=ONE_BAD(param=P + 2)), ALIGN),
    (dict(tensors=ONE_BAD(grad=P + 1)), ALIGN), (dict(tensors=ONE_BAD(grad=P + 2, grad_dtype=F32)), ALIGN),
    (dict(tensors=ONE_BAD(copy=P + 1)), ALIGN), (dict(tensors=ONE_BAD(m=P + 1)), ALIGN), (dict(tensors=ONE_BAD(v=P + 2)), ALIGN),
    (dict(tensors=ONE_BAD(state_bits=8, m_scale=P + 2, v_scale=P)), ALIGN)]
GRAD_NORM = dict(table=P, table_bytes=BIG, n_tensors=2, n_chunks=6, max_norm=1.0, scale=None, out=P, stream=None)
STEP = dict(table=P, table_bytes=BIG, n_tensors=2, n_chunks=6, cfg=opt(), lr_factor=None, grad_factor=None, count=None,
            t=P, stream=None)
OF_TABLE = [(dict(table=None), WORKSPACE), (dict(table=P + 128), WORKSPACE), (dict(table_bytes=8192), WORKSPACE),
            (dict(n_tensors=0), SHAPE), (dict(n_tensors=65537), SHAPE), (dict(n_chunks=-1), SHAPE),
            (dict(n_chunks=1 << 31), SHAPE)]

REFUSED = [
    ("aa_linear", LINEAR, [
        (dict(x=None), NULL), (dict(w=None), NULL), (dict(out=None), NULL), (dict(dtype=F32), SHAPE), (dict(dtype=9), SHAPE),
        (dict(n_max=-1), SHAPE), (dict(d_in=0), SHAPE), (dict(d_out=0), SHAPE), (dict(act=5), SHAPE), (dict(act=-1), SHAPE),
        (dict(d_in=(1 << 24) + 1, ldx=BIG), SHAPE), (dict(d_out=(1 << 24) + 1, ldo=BIG), SHAPE), (dict(ldx=31), SHAPE),
        (dict(ldo=23), SHAPE), (dict(residual=P, ldr=23), SHAPE), (dict(pre=P, ldpre=23), SHAPE),
        (dict(act=2, pre=P, ldpre=47), SHAPE), (dict(x=P + 1), ALIGN), (dict(out=P + 1), ALIGN), (dict(w=P + 1), ALIGN),
        (dict(residual=P + 1, ldr=24), ALIGN), (dict(pre=P + 1, ldpre=24), ALIGN), (dict(bias=P + 2), ALIGN),
        (dict(count=P + 2), ALIGN), (dict(n_max=2 ** 31 - 1), SHAPE)]),
    ("aa_linear_grad", LINEAR_GRAD, [
        (dict(dout=None), NULL), (dict(pre=None), NULL), (dict(dpre=None, dbias=None), NULL), (dict(dtype=F32), SHAPE),
        (dict(n_max=-1), SHAPE), (dict(d_out=0), SHAPE), (dict(act=5), SHAPE), (dict(lddo=23), SHAPE), (dict(ldpre=47), SHAPE),
        (dict(lddp=47), SHAPE), (dict(dout=P + 1), ALIGN), (dict(pre=P + 1), ALIGN), (dict(dpre=P + 1), ALIGN),
        (dict(dbias=P + 2), ALIGN), (dict(ws=None), WORKSPACE), (dict(ws=P + 8), WORKSPACE), (dict(ws_bytes=4096), WORKSPACE)]),
    ("aa_adamw_chunks", CHUNKS, OF_LIST),
    ("aa_adamw_table", TABLE, OF_LIST + [(dict(table=None), WORKSPACE), (dict(table=P + 64), WORKSPACE),
                                         (dict(table_bytes=8192), WORKSPACE)]),
    ("aa_grad_norm", GRAD_NORM, OF_TABLE + [
        (dict(max_norm=0.0), SHAPE), (dict(max_norm=-1.0), SHAPE), (dict(max_norm=NAN), SHAPE), (dict(out=None), NULL),
        (dict(out=P + 2), ALIGN), (dict(scale=P + 1), ALIGN)]),
    ("aa_adamw_step", STEP, OF_TABLE + [
        (dict(cfg=None), NULL), (dict(cfg=opt(beta1=1.0)), SHAPE), (dict(cfg=opt(beta1=-0.1)), SHAPE),
        (dict(cfg=opt(beta2=NAN)), SHAPE), (dict(cfg=opt(eps=0.0)), SHAPE), (dict(cfg=opt(eps=1e-39)), SHAPE), (dict(cfg=opt(eps=INF)), SHAPE),
        (dict(cfg=opt(lr=-1.0)), SHAPE), (dict(cfg=opt(lr=INF)), SHAPE), (dict(cfg=opt(weight_decay=-1.0)), SHAPE),
        (dict(t=None), NULL), (dict(t=P + 2), ALIGN), (dict(lr_factor=P + 2), ALIGN), (dict(grad_factor=P + 2), ALIGN),
        (dict(count=P + 2), ALIGN)]),
    ("aa_balance", BALANCE, OF_BOTH + [
        (dict(share=P + 2), ALIGN), (dict(loss=P + 2), ALIGN), (dict(ws=None), WORKSPACE), (dict(ws_bytes=4096), WORKSPACE),
        (dict(ws=P + 64), WORKSPACE)]),
    ("aa_balance_grad", BALANCE_GRAD, OF_BOTH + [
        (dict(dlogits=None), NULL), (dict(ld_out=15), SHAPE), (dict(dlogits=P + 1), ALIGN), (dict(dloss=P + 2), ALIGN),
        (dict(dweights=P + 2), ALIGN)]),
    ("aa_layer_norm", NORM, [
        (dict(x=None), NULL), (dict(out=None), NULL), (dict(dtype=3), SHAPE), (dict(dtype=-1), SHAPE),
        (dict(n_max=-1), SHAPE), (dict(d=0), SHAPE), (dict(d=(1 << 24) + 1, ldx=BIG, ldo=BIG), SHAPE),
        (dict(ldx=31), SHAPE), (dict(ldo=31), SHAPE), (dict(ldx=BIG + 1), SHAPE), (dict(eps=-1e-9), SHAPE),
        (dict(eps=NAN), SHAPE), (dict(eps=INF), SHAPE), (dict(x=P + 1), ALIGN), (dict(out=P + 1), ALIGN),
        (dict(dtype=F32, x=P + 2), ALIGN), (dict(gamma=P + 2), ALIGN), (dict(beta=P + 2), ALIGN),
        (dict(mean=P + 2), ALIGN), (dict(rstd=P + 2), ALIGN), (dict(count=P + 2), ALIGN)]),
    ("aa_layer_norm_grad", NORM_GRAD, [
        (dict(dout=None), NULL), (dict(x=None), NULL), (dict(dx=None), NULL), (dict(mean=None), NULL),
        (dict(rstd=None), NULL), (dict(dtype=7), SHAPE), (dict(n_max=-1), SHAPE), (dict(d=0), SHAPE),
        (dict(lddo=31), SHAPE), (dict(ldx=31), SHAPE), (dict(lddx=31), SHAPE), (dict(residual=P, ldr=31), SHAPE),
        (dict(dout=P + 1), ALIGN), (dict(residual=P + 1, ldr=32), ALIGN), (dict(gamma=P + 1), ALIGN),
        (dict(dgamma=P + 2), ALIGN), (dict(dbeta=P + 2), ALIGN), (dict(ws=None), WORKSPACE),
        (dict(ws=P + 128), WORKSPACE), (dict(ws_bytes=256), WORKSPACE), (dict(ws=None, dgamma=None), WORKSPACE)]),
]


@pytest.mark.parametrize("name,args,change,want",
                         [(n, a, c, w) for n, a, cases in REFUSED for c, w in cases],
                         ids=lambda v: v if isinstance(v, str) else ",".join(v) if isinstance(v, dict) and len(v) < 4 else None)
def test_refused(L, name, args, change, want):
    call = dict(args)
    assert set(change) <= set(call), change
    call.update(change)
    assert getattr(L, name)(*call.values()) == want


def test_workspace_grows_with_the_columns(L):
    """One made for d_max columns serves every call of fewer: its size grows, and a call of d asks for no more than that of d."""
    widths = sorted({1, 2, 3, 64, 1000, 1024, 8191, 8192, 8193, 12_000, 16_383, 16_384, 70_001, 1 << 20, (1 << 22) - 1, 1 << 22,
                     (1 << 22) + 1, 1 << 24} | {(7919 * k) % 30_000 + 1 for k in range(200)})
    sizes = [L.aa_layer_workspace_bytes(d) for d in widths]
    assert L.aa_layer_workspace_bytes(0) == sizes[0]
    assert all(a <= b for a, b in zip(sizes, sizes[1:])) and sizes[-1] < 1 << 28 and all(s % 256 == 0 for s in sizes)


def test_a_workspace_serves_fewer_columns(L):
    """A call of no rows and no sums' room: refused for the workspace, or launched (which fails without a GPU)."""
    for d_max in (1, 5, 8192, 8193, 12_000, 16_383, 16_385, 70_001, (1 << 22) + 5):
        for d in {1, 4, 8192, 8193, 11_999, 16_384, d_max} - {w for w in (1, 4, 8192, 8193, 11_999, 16_384) if w > d_max}:
            call = dict(NORM_GRAD, n_max=0, d=d, lddo=d, ldx=d, lddx=d, ws_bytes=L.aa_layer_workspace_bytes(d_max), accumulate=1)
            assert L.aa_layer_norm_grad(*call.values()) == OK, (d_max, d)


T = torch.zeros(4, 8)  # (not a CUDA tensor)
HALF = torch.zeros(4, 8, dtype=torch.bfloat16)


@pytest.mark.parametrize("call", [
    lambda: api.layer_norm(T, None, None, 1e-5, None, T),
    lambda: api.layer_norm(None, None, None, 1e-5, None, T),
    lambda: api.layer_norm(torch.zeros(4), None, None, 1e-5, None, T),
    lambda: api.layer_norm(torch.zeros(4, 8, dtype=torch.float64), None, None, 1e-5, None, T),
    lambda: api.layer_norm_grad(T, T, None, None, None, None, None, T, None, None, False, None),
    lambda: api.linear(HALF, HALF, None, "gelu", None, None, HALF),
    lambda: api.linear(T, T, None, "gelu", None, None, T),
    lambda: api.linear(HALF, HALF, None, "tanh", None, None, HALF),
    lambda: api.linear(HALF, None, None, "none", None, None, HALF),
    lambda: api.linear_grad(HALF, "silu", None, None, HALF, None, False, None),
    lambda: api.linear_grad(None, "silu", None, None, HALF, None, False, None),
    lambda: api.balance(T, None, cfg(), None, 0.1, 0.1, None, None, None, None),
    lambda: api.balance(None, None, cfg(), None, 0.1, 0.1, None, None, None, None),
    lambda: api.balance_grad(T, None, cfg(), None, None, None, 0.1, 0.1, None, T),
    lambda: api.adamw_tensor(T, T, T, T),
    lambda: api.adamw_tensor(None, T, T, T),
    lambda: api.adamw_tensor(T, torch.zeros(4, dtype=torch.float64), T, T),
    lambda: api.AdamWTable([]),
    lambda: api.grad_norm(None, 1.0, None, None),
    lambda: api.adamw_step(None, None, None, None, None, None),
])
def test_python_refusals(call):
    with pytest.raises(api.AAError):
        call()


def test_chunks_of_tensors(L):
    n = lambda *sizes: L.aa_adamw_chunks(tensors(*(dict(n=k) for k in sizes)), len(sizes))
    assert n(0) == 0 and n(1) == 1 and n(2048) == 1 and n(2049, 0, 5) == 3 and n(1 << 35) == 1 << 24
    assert L.aa_adamw_table_bytes(3, 100) % 256 == 0 and L.aa_adamw_table_bytes(3, 100) < L.aa_adamw_table_bytes(300, 10_000)
    # a tensor without elements needs no memory
    assert L.aa_adamw_chunks(tensors(dict(n=0, param=None, grad=None, m=None, v=None)), 1) == 0


def apart(*changes):
    """tensors() with memory of their own, a megabyte for each array."""
    fields = ("param", "grad", "copy", "m", "v", "m_scale", "v_scale")
    place = lambda k: {f: P + ((k * len(fields) + i) << 20) for i, f in enumerate(fields)}
    return tensors(*(dict(place(k), state_bits=8, **change) for k, change in enumerate(changes)))


TWICE = [("param", "param", 0), ("param", "grad", 0), ("copy", "copy", 0), ("copy", "param", 19_996), ("m", "v", 4999),
         ("v", "v", 0), ("m_scale", "m_scale", 76), ("v_scale", "m", 0), ("grad", "copy", 9998), ("grad", "v_scale", 0)]


@pytest.mark.parametrize("field,other,by,same", [(f, o, by, s) for f, o, by in TWICE for s in (False, True) if not s or f != o])
def test_memory_listed_twice_is_refused(L, field, other, by, same):
    pair = apart({}, {})
    setattr(pair[1], field, getattr(pair[1 if same else 0], other) + by)
    call = dict(TABLE, tensors=pair)
    assert L.aa_adamw_table(*call.values()) == SHAPE
