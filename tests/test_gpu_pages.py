"""Page operations and rows of the cache on the GPU, at the sizes and arguments where they can
go wrong, against the plain model."""
import numpy as np
import pytest
import torch

from paper_2605_29657_amd import cache

import cache_model as M
from test_gpu_cache import Cache, i32, prefix, same, state, unchanged

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.mark.parametrize("n", [1, 3])
def test_no_survivor_in_any_sequence(n):
    # An empty list of survivors, whose tensor has no address.
    c = Cache(n, 16, 2, 64)
    c.append(list(range(n)), [40 + 3 * x for x in range(n)])
    none, offs = torch.zeros(0, dtype=torch.int32, device=DEV), i32([0] * (n + 1))
    starts, spans = [5, 0, 17][:n], [20, 43, 29][:n]
    cache.keep(c.pages, i32(range(n)), i32(starts), i32(spans), none, offs, c.plan)
    cache.move(c.pages, c.layer, c.plan, none, offs)
    for x in range(n):
        c.k[x].keep(starts[x], spans[x], []), c.v[x].keep(starts[x], spans[x], [])
    c.check()


@pytest.mark.parametrize("n", [2048, 4096])
def test_replacing_more_pages_than_32_bits_count(n):
    # Forks share a sequence of 2^20 pages; dropping the first token of each would take 2^31 or
    # 2^32 fresh pages, far more than the pool: all or nothing.
    big, page = 1 << 20, 16
    pages = cache.Pages(big + 64, page, n + 1, big)
    plan = cache.plan(pages, n)
    cache.reserve(pages, cache.Batch(1, rows=big * page), plan)
    cache.fork(pages, i32([0] * n), i32(range(1, n + 1)), plan)
    assert pages.status.item() == 0 and pages.refs[:big].unique().tolist() == [n + 1]
    taken, some = pages.taken.clone(), pages.table[[1, n // 2, n]].clone()
    none, offs = torch.zeros(0, dtype=torch.int32, device=DEV), i32([0] * (n + 1))
    cache.keep(pages, i32(range(1, n + 1)), i32([0] * n), i32([1] * n), none, offs, plan)
    assert pages.status.item() == cache.FULL
    assert pages.length.unique().tolist() == [big * page] and torch.equal(pages.taken, taken)
    assert pages.refs[:big].unique().tolist() == [n + 1] and pages.refs[big:].unique().tolist() == [0]
    assert torch.equal(pages.table[[1, n // 2, n]], some) and plan[:3].tolist()[2] == 0
    # One of them alone, with the tokens of 32 pages to go on with, goes on as before.
    pages.status.zero_()
    cache.keep(pages, i32([5]), i32([(big - 32) * page]), i32([1]), none, i32([0, 0]), plan)
    assert pages.status.item() == 0 and pages.length[5].item() == big * page - 1
