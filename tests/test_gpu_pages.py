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


# Two of four sequences with more rows than the stated bound, or offsets that descend.
@pytest.mark.parametrize("offsets,most", [([0, 3, 12, 15, 20], 8), ([4, 4, 2, 4, 20], 16), ([0, 9, 10, 20, 20], 8)])
def test_rows_that_the_offsets_and_the_bound_do_not_agree_on(offsets, most):
    c = Cache(4, 16, 2, 64)
    c.append([0, 1, 2, 3], [5, 20, 30, 40])
    was, x = state(c), c.rows(24)
    b = cache.Batch(4, row_offsets=i32(offsets), max_rows=most)
    cache.reserve(c.pages, b, c.plan)
    cache.append(c.pages, c.layer, b, c.plan, x, x)
    unchanged(c, was, cache.BAD_ROWS)
    # What reads the cache leaves such a sequence's rows as they were, and says so too.
    good = [i for i in range(4) if 0 < offsets[i + 1] - offsets[i] <= most]
    k, v = (torch.full((24, 2, 64), 9.0, device=DEV).bfloat16() for _ in range(2))
    cache.read(c.pages, c.layer, b, k, v)
    unchanged(c, was, cache.BAD_ROWS)
    q = torch.randn(24, 4, 64, device=DEV).bfloat16()
    out, lse = torch.full_like(q, 9.0), torch.full((24, 4), 9.0, device=DEV)
    cache.attend(c.pages, c.layer, b, q, out, cache.workspace(c.pages, c.layer, b, 4), lse=lse)
    unchanged(c, was, cache.BAD_ROWS)
    left = np.ones(24, bool)
    for i in good:
        at = slice(offsets[i], offsets[i + 1])
        left[at] = False
        n = min(at.stop - at.start, len(c.k[i].x))
        same(M.f64(k[at])[:n], c.k[i].x[:n])
        M.check_attention(M.f64(out[at]), M.f64(lse[at]), M.f64(q[at]), c.k[i].x, c.v[i].x, True)
    left = torch.from_numpy(left).to(DEV)
    assert (out[left] == 9).all() and (lse[left] == 9).all() and (k[left] == 9).all() and (v[left] == 9).all()


@pytest.mark.parametrize("T", [1, 40])
@pytest.mark.parametrize("n", [3, 400])
def test_reading_calls_say_which_slots_there_are_not(n, T):
    c = Cache(n, 16, 1, 64, num_pages=8 + n)
    c.append([0, 2], [50, 60])
    was = state(c)
    b = cache.Batch(n, rows=T, seq=i32([0] + [1] * (n - 2) + [n]))
    k = torch.full((n * T, 1, 64), 9.0, device=DEV).bfloat16()
    cache.read(c.pages, c.layer, b, k, None)
    unchanged(c, was, cache.BAD_SEQ)
    assert (k[T:] == 9).all()
    same(M.f64(k[:T]), c.k[0].x[:T])
    q = torch.randn(n * T, 8, 64, device=DEV).bfloat16()
    out, lse = torch.full_like(q, 9.0), torch.full((n * T, 8), 9.0, device=DEV)
    cache.attend(c.pages, c.layer, b, q, out, cache.workspace(c.pages, c.layer, b, 8), lse=lse)
    unchanged(c, was, cache.BAD_SEQ)
    assert (out[T:] == 0).all() and (lse[T:] == -np.inf).all()
    M.check_attention(M.f64(out[:T]), M.f64(lse[:T]), M.f64(q[:T]), c.k[0].x, c.v[0].x, True)
