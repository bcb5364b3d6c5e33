"""The experts' products where blocks take several tiles one after another, for every tile: the next tile's slices are
moved while the last one's results are written, groups are uneven, some are empty, and rows, columns and the summed
dimension end inside a tile.

Operands are -1, 0 and 1.  Sums are then whole numbers, exact in the matrix instructions' 32 bits and in torch's, and (this is
looked at) small enough for both 16-bit types: results are compared for equality.  What follows a sum in a gated product is worked
out in 32 bits and adds a few units of 2^-23, a rounding at most half a step."""
import numpy as np
import pytest
import torch

from paper_1905_03381_amd import api
from test_gpu_experts import F32, HALVES, U32, half_step, tiny

pytestmark = pytest.mark.gpu

PLACES = {256: 256, 128: 512, 32: 512}       # tiles the chip holds at once


def tile_of(mode, rows_max, E, d_in, d_out, act="none", aligned=True):
    """The tile that the library takes (0: the kernel for few rows), and how many of them its rule counts."""
    up = lambda a, b: -(-a // b)
    if mode == "grad_weight":
        tile = 128 if not aligned or d_in * d_out <= 256 * 256 else 256
        return tile, E * up(d_out, tile) * up(d_in, tile)
    groups = max(1, min(rows_max, E))
    rows = up(rows_max, groups)
    wide = (d_out if mode == "forward" else d_in) * (2 if mode == "forward" and act == "gated" else 1)
    steps = up(d_in if mode == "forward" else d_out, 64)
    n = {bm: groups * up(rows, bm) * up(wide, bn) for bm, bn in ((256, 256), (128, 128), (32, 64))}
    time = {256: up(n[256], 256) * (steps * 1.75 + 5.0),
            128: up(n[128], 512) * (steps * (0.6 if n[128] <= 256 else 1.05) + 3.0),
            32: up(n[32], 512) * (steps * 0.42 + 3.5)}
    if mode == "forward" and rows <= 32 and n[128] <= 320:
        return 0, 0
    if not aligned:
        return 128, n[128]
    best = 32 if time[32] < time[128] and time[32] < time[256] else 128 if time[128] < time[256] else 256
    return best, n[best]


def uneven(E, total, seed):
    """Ends of E groups of `total` rows: a third of them empty, one of a single row, the others of very unlike sizes."""
    g = np.random.default_rng(seed)
    share = g.random(E) ** 3 + 0.02
    share[g.permutation(E)[:E // 3]] = 0
    sizes = np.floor(share / share.sum() * total).astype(int)
    if E > 2:
        sizes[np.flatnonzero(share)[0]] = 1
    sizes[np.argmax(sizes)] += total - sizes.sum()
    return np.concatenate([[0], np.cumsum(sizes)]).astype(np.int32)


def whole(g, *shape, dtype, density):
    """-1, 0 and 1; density: the share that is not 0."""
    v = torch.rand(*shape, generator=g, device="cuda")
    return ((v < density / 2).to(F32) - (v > 1 - density / 2).to(F32)).to(dtype)


def generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def grouped(E, rows_max, K, seed):
    """offsets (their last below rows_max), an order of pairs of K choices a row, and numbers of the rows they read."""
    total = rows_max - rows_max // 40
    offsets = uneven(E, total, seed)
    order = torch.from_numpy(np.random.default_rng(seed + 1).permutation(rows_max).astype(np.int32)).cuda()
    return offsets, torch.from_numpy(offsets).cuda(), order, (order // K).long(), total


def assert_equal(got, want, what):
    assert float(want.abs().max()) <= 256, what
    assert torch.equal(got.to(F32), want), (what, int((got.to(F32) != want).sum()))


def assert_near(got, want, bound, what):
    off = (got.double() - want).abs()
    assert bool((off <= bound).all()), (what, float((off - bound).max()))


# mode, act, tile, rows_max, E, d_in, d_out, aligned
CASES = [
    ("forward", "none", 256, 32_768, 8, 200, 1003, True),
    ("forward", "relu", 256, 32_768, 8, 136, 1003, True),
    ("forward", "gated", 256, 32_768, 8, 200, 500, True),
    ("forward", "none", 128, 6400, 64, 136, 2555, True),
    ("forward", "gated", 128, 6400, 64, 200, 1274, True),
    ("forward", "relu", 32, 1920, 64, 2040, 760, True),
    ("forward", "gated", 32, 1920, 64, 2040, 380, True),
    ("forward", "none", 128, 8184, 8, 133, 1301, False),
    ("forward", "gated", 128, 8184, 8, 133, 651, False),
    ("grad_input", "none", 256, 32_768, 8, 1000, 200, True),
    ("grad_input", "relu", 256, 32_768, 8, 1000, 136, True),
    ("grad_input", "gated", 256, 32_768, 8, 1000, 200, True),
    ("grad_input", "relu", 128, 6400, 64, 2552, 136, True),
    ("grad_input", "gated", 32, 1920, 64, 632, 2040, True),
    ("grad_input", "none", 128, 8184, 8, 1301, 133, False),
    ("grad_input", "gated", 128, 8184, 8, 1301, 133, False),
]


@pytest.mark.parametrize("dtype", HALVES)
@pytest.mark.parametrize("gathered", [False, True])
@pytest.mark.parametrize("mode,act,tile,rows_max,E,d_in,d_out,aligned", [c for c in CASES if c[0] == "forward"])
def test_forward_over_several_tiles(mode, act, tile, rows_max, E, d_in, d_out, aligned, gathered, dtype):
    got_tile, tiles = tile_of(mode, rows_max, E, d_in, d_out, act, aligned)
    assert got_tile == tile and tiles > PLACES[tile], (got_tile, tiles)
    g, K, density = generator(E + d_in), 3, min(0.6, 200 / d_in)
    offsets, offsets_dev, order, rows, total = grouped(E, rows_max, K, d_out)
    x = whole(g, -(-rows_max // K) if gathered else rows_max, d_in, dtype=dtype, density=density)
    if not gathered:
        x[total:] = float("nan")                     # (rows of no group)
    w = whole(g, E, d_out * (2 if act == "gated" else 1), d_in, dtype=dtype, density=density)
    out = torch.full((rows_max, d_out), 55.0, dtype=dtype, device="cuda")
    pre = torch.full((rows_max, 2 * d_out), 55.0, dtype=dtype, device="cuda") if act == "gated" else None
    api.expert_forward(x, order if gathered else None, K, offsets_dev, w, act, out, pre)
    assert bool((out[total:] == 55).all()) and (pre is None or bool((pre[total:] == 55).all()))
    for e in range(E):
        lo, hi = int(offsets[e]), int(offsets[e + 1])
        if lo == hi:
            continue
        h = x[rows[lo:hi] if gathered else slice(lo, hi)].to(F32) @ w[e].to(F32).t()
        if act == "gated":
            assert_equal(pre[lo:hi], h, f"pre of expert {e}")
            gate, up = h[:, :d_out].double(), h[:, d_out:].double()
            want = gate * torch.sigmoid(gate) * up
            bound = 16 * U32 * (1 + gate.abs()) * want.abs()
            assert_near(out[lo:hi], want, bound + half_step(dtype) * (want.abs() + bound) + tiny(dtype), f"expert {e}")
        else:
            assert_equal(out[lo:hi], h.clamp(min=0) if act == "relu" else h, f"expert {e}")


@pytest.mark.parametrize("dtype", HALVES)
@pytest.mark.parametrize("mode,act,tile,rows_max,E,d_in,d_out,aligned", [c for c in CASES if c[0] == "grad_input"])
def test_grad_input_over_several_tiles(mode, act, tile, rows_max, E, d_in, d_out, aligned, dtype):
    got_tile, tiles = tile_of(mode, rows_max, E, d_in, d_out, act, aligned)
    assert got_tile == tile and tiles > PLACES[tile], (got_tile, tiles)
    g, density = generator(E + d_in), min(0.6, 200 / d_out)
    offsets, offsets_dev, _, _, total = grouped(E, rows_max, 1, d_out)
    dout = whole(g, rows_max, d_out, dtype=dtype, density=density)
    dout[total:] = float("nan")
    w = whole(g, E, d_out, d_in, dtype=dtype, density=density)
    wide = d_in * (2 if act == "gated" else 1)
    saved = None if act == "none" else whole(g, rows_max, wide, dtype=dtype, density=0.6)
    dx = torch.full((rows_max, wide), 55.0, dtype=dtype, device="cuda")
    api.expert_grad_input(dout, offsets_dev, w, act, saved, dx)
    assert bool((dx[total:] == 55).all())
    for e in range(E):
        q = slice(int(offsets[e]), int(offsets[e + 1]))
        if q.start == q.stop:
            continue
        d = dout[q].to(F32) @ w[e].to(F32)
        if act == "gated":
            gate, up = saved[q][:, :d_in].double(), saved[q][:, d_in:].double()
            z, D = torch.sigmoid(gate), d.double()
            want = torch.cat([D * up * (z + gate * z * (1 - z)), D * gate * z], 1)
            bound = 32 * U32 * D.abs().repeat(1, 2)   # (terms below 2 for gates and ups of at most 1)
            assert_near(dx[q], want, bound + half_step(dtype) * (want.abs() + bound) + tiny(dtype), f"expert {e}")
        else:
            assert_equal(dx[q], torch.where(saved[q] > 0, d, 0.0) if act == "relu" else d, f"expert {e}")


@pytest.mark.parametrize("dtype", HALVES)
@pytest.mark.parametrize("gathered,wide,accumulate", [(False, False, False), (True, True, False), (True, False, True),
                                                      (False, True, True)])
@pytest.mark.parametrize("tile,rows_max,E,d_in,d_out,aligned", [
    (256, 4100, 12, 1544, 1800, True), (256, 3000, 300, 256, 264, True), (128, 3000, 300, 136, 200, True),
    (128, 4100, 12, 707, 1301, False), (128, 3000, 300, 131, 203, False)])
def test_grad_weight_over_several_tiles(tile, rows_max, E, d_in, d_out, aligned, gathered, wide, accumulate, dtype):
    got_tile, tiles = tile_of("grad_weight", rows_max, E, d_in, d_out, aligned=aligned)
    assert got_tile == tile and tiles > PLACES[tile], (got_tile, tiles)
    g, K, out_type = generator(E + d_in), 3, F32 if wide else dtype
    offsets, offsets_dev, order, rows, total = grouped(E, rows_max, K, d_out)
    dout = whole(g, rows_max, d_out, dtype=dtype, density=0.3)
    dout[total:] = float("nan")
    x = whole(g, -(-rows_max // K) if gathered else rows_max, d_in, dtype=dtype, density=0.3)
    if not gathered:
        x[total:] = float("nan")
    old = whole(g, E, d_out, d_in, dtype=out_type, density=0.6)
    dw = old.clone()
    api.expert_grad_weight(dout, x, order if gathered else None, K, offsets_dev, dw, accumulate,
                           api.ExpertWorkspace(rows_max, 1, E))
    for e in range(E):
        lo, hi = int(offsets[e]), int(offsets[e + 1])
        want = dout[lo:hi].to(F32).t() @ x[rows[lo:hi] if gathered else slice(lo, hi)].to(F32)
        assert_equal(dw[e], want + old[e].to(F32) if accumulate else want, f"expert {e}")


@pytest.mark.parametrize("dtype", HALVES)
@pytest.mark.parametrize("act", ["none", "gated"])
@pytest.mark.parametrize("sizes", [[0, 190, 1, 0, 0, 0, 2, 7], [0, 0, 0, 0, 0, 0, 0, 100]])
@pytest.mark.parametrize("d_in", [136, 133])
def test_few_rows_that_are_nearly_all_one_experts(d_in, sizes, act, dtype):
    """The kernel for few rows goes by their average: 16 or 32 rows at a time of an expert that has many more."""
    E, d_out, rows_max = 8, 200, sum(sizes)
    assert tile_of("forward", rows_max, E, d_in, d_out, act)[0] == 0
    g = generator(d_in)
    offsets = np.concatenate([[0], np.cumsum(sizes)]).astype(np.int32)
    x, w = whole(g, rows_max, d_in, dtype=dtype, density=0.6), whole(g, E, (2 if act == "gated" else 1) * d_out, d_in, dtype=dtype, density=0.6)
    out, pre = torch.zeros(rows_max, d_out, dtype=dtype, device="cuda"), torch.zeros(rows_max, 2 * d_out, dtype=dtype, device="cuda")
    api.expert_forward(x, None, 1, torch.from_numpy(offsets).cuda(), w, act, out, pre if act == "gated" else None)
    for e in range(E):
        q = slice(int(offsets[e]), int(offsets[e + 1]))
        if q.start < q.stop:
            assert_equal((pre if act == "gated" else out)[q], x[q].to(F32) @ w[e].to(F32).t(), f"expert {e}")
