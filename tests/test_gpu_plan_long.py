"""The plan of many pairs: against torch's stable sort, on both sides of where a launch of its own adds the counts up, and
in a time that grows with the pairs and not with their square."""
import pytest
import torch

from paper_1905_03381_amd import api

pytestmark = pytest.mark.gpu


def made(n, K, E, rows, seed, out_of_range=0.0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    ids = torch.randint(0, E, (n, K), generator=g, device="cuda", dtype=torch.int32)
    if out_of_range:
        off = torch.rand(n, K, generator=g, device="cuda") < out_of_range
        ids[off] = torch.where(torch.rand(n, K, generator=g, device="cuda")[off] < 0.5, -1, E).to(torch.int32)
    count = None if rows is None else torch.tensor([rows], dtype=torch.int32, device="cuda")
    bufs = [torch.full(s, -7, dtype=torch.int32, device="cuda") for s in ((E + 1,), (n * K,), (n, K))]
    return ids, count, bufs, api.ExpertWorkspace(n, K, E)


def check_plan(ids, count, bufs, E):
    (n, K), (offsets, order, slot) = ids.shape, bufs
    m = n if count is None else int(count)
    key = ids[:m].reshape(-1).long()
    there = (key >= 0) & (key < E)
    where = torch.nonzero(there).view(-1)
    by = torch.sort(key[there], stable=True)
    want = where[by.indices].to(torch.int32)
    counts = torch.bincount(key[there], minlength=E)
    assert torch.equal(offsets[1:].long(), torch.cumsum(counts, 0)) and int(offsets[0]) == 0
    assert torch.equal(order[:want.numel()], want) and bool((order[want.numel():] == -7).all())
    places = torch.full((m * K,), -1, dtype=torch.int32, device="cuda")
    places[want.long()] = torch.arange(want.numel(), dtype=torch.int32, device="cuda")
    assert torch.equal(slot[:m].view(-1), places) and bool((slot[m:] == -7).all())


@pytest.mark.parametrize("E,n,K,rows", [
    (1, 3_000_000, 4, None), (5, 2_000_001, 2, None), (16, 700_001, 3, 650_000), (17, 1_300_000, 2, None), (63, 1_048_577, 1, None),
    (300, 500_001, 1, None), (1000, 262_145, 1, 0), (1000, 300_001, 1, 1), (1024, 300_001, 1, 300_000), (1024, 130_000, 2, None),
    (1024, 140_000, 2, None)])
def test_plan_of_many_pairs(E, n, K, rows):
    ids, count, bufs, ws = made(n, K, E, rows, E + n, 0.1)
    api.expert_plan(ids, count, E, *bufs, ws)
    check_plan(ids, count, bufs, E)


def test_plan_grows_with_the_pairs():
    """67 M pairs of 1024 experts, 32,768 tiles of pairs.  Read twice and written twice they are 1.1 GB, the counts 0.5: less than a
    millisecond; counts added up by every block for itself would be 4.4 TB."""
    E, n, K = 1024, 1 << 23, 8
    ids, count, bufs, ws = made(n, K, E, None, 1)
    api.expert_plan(ids, count, E, *bufs, ws)
    check_plan(ids, count, bufs, E)
    start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    start.record()
    api.expert_plan(ids, count, E, *bufs, ws)
    end.record()
    end.synchronize()
    assert start.elapsed_time(end) < 50.0
