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


# ------------------------------------------------------------- calls past a launch's workgroups
def fill(c, slots, rows, k, v, together):
    """Appends ``rows`` tokens each to ``slots`` (their keys and values packed), in one call or
    one call each: the same pages either way."""
    at = prefix(rows)
    for part in ([range(len(slots))] if together else [[x] for x in range(len(slots))]):
        b = c.batch([slots[x] for x in part], [rows[x] for x in part])
        cache.reserve(c.pages, b, c.plan)
        x = slice(at[part[0]], at[part[-1] + 1])
        cache.append(c.pages, c.layer, b, c.plan, k[x], v[x])


def values(c, slots, lens):
    k, v = (torch.empty(sum(lens), c.Hkv, c.d, device=DEV) for _ in range(2))
    for s, a, n in zip(slots, prefix(lens), lens):               # one by one: small calls
        cache.read(c.pages, c.layer, cache.Batch(1, rows=n, seq=i32([s])), k[a:a + n], v[a:a + n])
    return k, v


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("page,Hkv,d,tokens", [(64, 8, 128, 50000), (16, 64, 64, 12000), (128, 8, 128, 95000),
                                               (256, 16, 128, 46000), (256, 8, 256, 90000), (32, 12, 128, 32000)])
def test_more_blocks_than_workgroups(page, Hkv, d, tokens, dtype):
    # Appending and moving walk their blocks with 4096 workgroups at most: in one call here,
    # against small calls (which the other tests compare with the model), bit for bit.
    n = 5
    lens = [tokens // 8, tokens // 4 + 3, 7, tokens // 2 - 11, tokens // 8 + 1]
    num = sum(lens) // page + 4 * n
    units = page * (8 if d <= 64 else 16 if d <= 128 else 32) // 4
    side, heads = max(256 // units, 1), 2 if units <= 512 else 1         # blocks and heads of a workgroup
    fresh = sum(-(-x * 3 // 4 // page) for x in lens)
    assert sum(lens) // page * Hkv * 2 > 4096 * side and fresh * (Hkv // heads) * 2 > 4096 * side
    r = np.random.default_rng(page + d)
    cs = [Cache(n, page, Hkv, d, num_pages=2 * num, max_pages=num, seed=1, dtype=dtype) for _ in range(2)]
    g = torch.Generator(device=DEV).manual_seed(d)
    size = torch.exp2(torch.randint(-8, 9, (sum(lens), 1, 1), generator=g, device=DEV).float())
    for rows, z in ((lens, size), ([5, 1, 2, page, 3], 300.0)):   # the second raises most pages' scales
        k, v = (torch.randn(sum(rows), Hkv, d, generator=g, device=DEV).mul_(z).to(dtype) for _ in range(2))
        for c, together in zip(cs, (True, False)):
            fill(c, list(range(n)), rows, k, v, together)
    a, b = cs
    for x, y in ((a.pages.table, b.pages.table), (a.pages.length, b.pages.length), (a.layer.k, b.layer.k),
                 (a.layer.v, b.layer.v), (a.layer.k_scale.view(torch.int32), b.layer.k_scale.view(torch.int32)),
                 (a.layer.v_scale.view(torch.int32), b.layer.v_scale.view(torch.int32))):
        assert torch.equal(x, y)
    lens = a.pages.length.tolist()
    kept = [np.sort(r.choice(x, x * 3 // 4, replace=False)) for x in lens]
    for c, together in zip(cs, (True, False)):
        for part in ([range(n)] if together else [[x] for x in range(n)]):
            idx = i32(np.concatenate([kept[x] for x in part]))
            offs = i32(prefix([len(kept[x]) for x in part]))
            cache.keep(c.pages, i32(part), i32([0] * len(part)), i32([lens[x] for x in part]), idx, offs, c.plan)
            cache.move(c.pages, c.layer, c.plan, idx, offs)
        assert c.pages.status.item() == 0
    lens = [len(x) for x in kept]
    assert a.pages.length.tolist() == b.pages.length.tolist() == lens
    for x, y in zip(values(a, range(n), lens), values(b, range(n), lens)):
        assert torch.equal(x, y)
    k, v = (torch.empty(sum(lens), Hkv, d, device=DEV) for _ in range(2))              # and read in one call
    cache.read(a.pages, a.layer, a.batch(list(range(n)), lens), k, v)
    for x, y in zip((k, v), values(a, range(n), lens)):
        assert torch.equal(x, y)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("page,Hkv,d", [(64, 8, 128), (16, 3, 80), (128, 5, 256)])
def test_reading_more_than_the_caches_hold(page, Hkv, d, dtype):
    # Past 256 MB, outputs go past the caches: against parts, bit for bit, and rows behind the
    # sequences' ends stay.
    n = (300 << 20) // (2 * Hkv * d * dtype.itemsize)
    lens = [n // 3, n - n // 3 - 5]
    c = Cache(2, page, Hkv, d, num_pages=n // page + 4, max_pages=n // page + 2)
    k, v = (torch.randn(n, Hkv, d, generator=c.gen, device=DEV).bfloat16() for _ in range(2))
    fill(c, [0, 1], lens, k, v, True)
    rows = [lens[0] + 2, lens[1] + 3]
    k, v = (torch.full((n, Hkv, d), 9.0, device=DEV, dtype=dtype) for _ in range(2))
    cache.read(c.pages, c.layer, c.batch([0, 1], rows), k, v)
    wk, wv = (torch.full((n, Hkv, d), 9.0, device=DEV, dtype=dtype) for _ in range(2))
    for s, a in ((0, 0), (1, rows[0])):
        for x in range(0, lens[s], 9973):
            m = min(9973, lens[s] - x)
            cache.read(c.pages, c.layer, cache.Batch(1, rows=m, seq=i32([s])), wk[a + x:a + x + m], wv[a + x:a + x + m],
                       start=i32([x]))
    assert torch.equal(k, wk) and torch.equal(v, wv)
