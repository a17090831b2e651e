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
