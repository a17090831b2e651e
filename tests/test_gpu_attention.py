"""Attention over the 8-bit cache on the GPU, by the comparison of attention_model.py."""
import numpy as np
import pytest
import torch

from paper_2605_29657_amd import cache

import attention_model as A
import cache_model as M
from test_gpu_cache import Cache, i32, prefix

pytestmark = pytest.mark.gpu
DEV = "cuda"


def attend(c, seqs, rows, H, causal=True, scale=0.0, max_tokens=0, q=None):
    n = sum(rows)
    q = torch.randn(n, H, c.d, generator=c.gen, device=DEV).bfloat16() if q is None else q
    b = c.batch(seqs, rows)
    ws = cache.workspace(c.pages, c.layer, b, H, max_tokens)
    ws.fill_(0xff)
    out, lse = torch.empty_like(q), torch.empty(n, H, device=DEV)
    cache.attend(c.pages, c.layer, b, q, out, ws, lse=lse, causal=causal, softmax_scale=scale,
                 max_tokens=max_tokens)
    at = prefix(rows)
    for i, s in enumerate(seqs):
        x = slice(at[i], at[i + 1])
        A.check(M.f64(out[x]), M.f64(lse[x]), M.f64(q[x]), c.k[s].x, c.v[s].x, A.per_token(c.v[s]), causal, scale)
    return out, lse


@pytest.mark.parametrize("T", [1, 13, 40, 129, 300])
@pytest.mark.parametrize("page,H,Hkv,d", [(32, 7, 1, 80), (64, 8, 2, 128), (16, 8, 4, 64), (16, 4, 2, 256)])
def test_blocks_that_end_inside_a_tile_beside_unwritten_codes(page, H, Hkv, d, T):
    # The first page taken holds one token; what lies behind it there has never been written
    # (NaN codes).  Most row blocks of the longer sequence end inside a tile.
    c = Cache(2, page, Hkv, d, num_pages=200, max_pages=100, seed=T)
    c.append([0], [1])
    assert c.pages.table[0, 0].item() == 0
    c.append([1], [700])
    attend(c, [1], [T], H)
    attend(c, [1], [T], H, causal=False)
    attend(c, [1, 0], [T, 1], H)


# ------------------------------------------------------------------ pages of unequal scale
# A row's output follows from the keys that it sees and their weights (probability times scale):
# what a page weighs that it does not see, or gives next to nothing, leaves no trace in it.
def unequal(page, H, Hkv, d, sizes, logits=None, seed=0, max_pages=100, slots=1):
    """Slot 0 holds a page for each of ``sizes`` (powers of two), its values about that large, its
    keys such that a query of ones, scale 1, gives them about that logit (0, or ``logits``)."""
    c = Cache(slots, page, Hkv, d, num_pages=200, max_pages=max_pages, seed=seed, dtype=torch.float32)
    for x, z in zip(sizes, logits or [0.0] * len(sizes)):
        k = c.rows(page, 0.2 / d)
        k.add_(z / d)
        c.append([0], [page], k=k, v=c.rows(page, 2.0 ** x))
    return c


def ones(c, T, H):
    return (1 + 0.1 * torch.randn(T, H, c.d, generator=c.gen, device=DEV)).bfloat16()


SHAPES = [(16, 4, 2, 64), (16, 8, 1, 128), (32, 4, 2, 80), (64, 2, 1, 256), (16, 4, 4, 128)]


@pytest.mark.parametrize("T", [1, 3, 6, 14, 70, 200])
@pytest.mark.parametrize("page,H,Hkv,d", SHAPES)
def test_hidden_pages_of_any_scale(page, H, Hkv, d, T):
    # The last pages are hidden from the first rows and outweigh the earlier ones, or vanish
    # beside them.
    for sizes in ([0] * 5 + [30] * 3, [40, 0, 0, 0, 0, 0, 20, 60], [0, -30] * 4, [-60, -61, -30, 0, 30, 60, 90, 115]):
        c = unequal(page, H, Hkv, d, sizes, seed=T)
        attend(c, [0], [min(T, page * 8)], H, scale=1.0, q=ones(c, min(T, page * 8), H))


@pytest.mark.parametrize("T", [1, 6, 14, 70, 200])
@pytest.mark.parametrize("page,H,Hkv,d", SHAPES)
def test_visible_pages_of_no_weight(page, H, Hkv, d, T):
    # Pages 2^20 to 2^40 larger than the others, seen by every row with a weight of e^-200, of
    # about the others' or in between.
    T = min(T, page)
    for z in (-200.0, -14.0, -20.0, -28.0):
        for sizes in ([30, 0, 1, 0, 3, 0, -2, 0, 0], [0, 20, 0, 0, 40, 0, 0, 20, 0], [0, 0, 1, 0, 0, 0, 0, 40, 0]):
            c = unequal(page, H, Hkv, d, sizes, [z if x >= 20 else 0.0 for x in sizes], seed=T)
            attend(c, [0], [T], H, scale=1.0, q=ones(c, T, H))
            attend(c, [0], [T], H, scale=1.0, q=ones(c, T, H), causal=False)


@pytest.mark.parametrize("T", [1, 14, 70])
@pytest.mark.parametrize("step", [1, 2, 3, 4, 5, 6, 9, 17])
def test_scales_that_rise_or_fall_page_by_page(step, T):
    # Each page weighs less than the first one (or last one) although its scale is larger, so
    # that nothing that follows the scales alone keeps what the first one gave.
    n = min(24, 100 // step)
    for order in (1, -1):
        sizes = [step * x for x in range(n)][::order]
        logits = [-1.4 * x for x in sizes]
        for page, H, Hkv, d in ((16, 4, 1, 64), (64, 8, 2, 128)):
            c = unequal(page, H, Hkv, d, sizes, logits, seed=step)
            attend(c, [0], [min(T, page)], H, scale=1.0, q=ones(c, min(T, page), H))


@pytest.mark.parametrize("T", [1, 9, 14, 60, 150])
def test_scales_at_both_ends_of_their_range(T):
    # Weights that no float32 probability could carry: e^-140 times 2^110 beside 2^-95.
    for sizes, logits in (([-95, 110, -95, -95], [0.0, -140.0, 0.0, 0.0]), ([110, -95, -95, 60], [-141.0, 0.0, 0.0, -107.0]),
                          ([-95, -95, -95, 118], [0.0, 0.0, 0.0, -100.0]), ([118, 118, 118, 118], [0.0] * 4),
                          ([-99, -104, -99, -99], [0.0] * 4)):
        for page, d in ((16, 64), (64, 128)):
            c = unequal(page, 4, 2, d, sizes, logits, seed=T)
            attend(c, [0], [min(T, page)], 4, scale=1.0, q=ones(c, min(T, page), 4))


@pytest.mark.parametrize("T,H", [(1, 4), (4, 4), (1, 24), (40, 4)])
def test_unequal_scales_over_ranges_and_parts(T, H):
    # Many pages, so that ranges of work, parts of a block and the waves of a workgroup each
    # hold pages of other scales.
    r = np.random.default_rng(T)
    sizes = r.integers(-40, 40, 130).tolist()
    for logits in ([-0.69 * x for x in sizes], [-0.8 * x for x in sizes], [0.0] * 130):
        c = unequal(16, H, 1, 128, sizes, logits, seed=H, max_pages=1 << 16)
        q = ones(c, T, H)
        attend(c, [0], [T], H, scale=1.0, q=q)
        attend(c, [0], [T], H, scale=1.0, q=q, max_tokens=len(sizes) * 16)


@pytest.mark.parametrize("at", range(13))
@pytest.mark.parametrize("page,H,Hkv,d,T", [(64, 8, 2, 128, 150), (64, 4, 1, 128, 700), (64, 4, 1, 128, 20), (64, 8, 2, 64, 90),
                                            (64, 2, 1, 256, 90), (64, 4, 2, 128, 2), (64, 24, 1, 64, 1)])
def test_the_spread_is_passed_at_any_tile(page, H, Hkv, d, T, at):
    # Ordinary pages up to one of 2^21 (of no weight, or of all rows' largest), and behind it.
    for z in (-200.0, 0.0):
        c = unequal(page, H, Hkv, d, [x % 3 for x in range(at)] + [21] + [1] * (12 - at), [0.0] * at + [z] + [0.0] * (12 - at),
                    seed=at, max_pages=1 << 14)
        attend(c, [0], [T], H, scale=1.0, q=ones(c, T, H))
        attend(c, [0], [T], H, scale=1.0, q=ones(c, T, H), max_tokens=13 * page)


@pytest.mark.parametrize("T", [1, 5, 16, 150])
def test_values_next_to_the_largest_float(T):
    # Equal weights of values up to 240 * 2^120: a mean never passes its largest value.
    c = Cache(1, 64, 1, 64, num_pages=100, max_pages=80, dtype=torch.float32)
    v = torch.full((3000, 1, 64), 3.1e38, device=DEV)
    v[:, :, ::2] = -3.1e38
    c.append([0], [3000], k=torch.zeros(3000, 1, 64, device=DEV), v=v)
    attend(c, [0], [T], 4)
    attend(c, [0], [T], 4, max_tokens=64)


def test_outputs_do_not_depend_on_hidden_tokens():
    # The same first tokens with and without others behind them, which a causal row does not
    # see: equal bits where the same form handles both.
    page, H, Hkv, d, T = 16, 4, 1, 64, 64
    c = Cache(2, page, Hkv, d, num_pages=40, max_pages=20)
    k, v = c.rows(128), c.rows(128)
    q = torch.randn(T, H, d, generator=c.gen, device=DEV).bfloat16()
    outs = []
    for s, size in ((0, 1.0), (1, 2.0 ** 40)):
        w = v.clone()
        w[96:] *= size
        c.append([s], [128], k=k, v=w)
        outs.append(attend(c, [s], [T], H, q=q))
    # Rows 0 .. 31 see tokens 0 .. 64 to 95.
    assert torch.equal(outs[0][0][:32], outs[1][0][:32]) and torch.equal(outs[0][1], outs[1][1])


# ------------------------------------------------------------------- many keys in one part
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("page,H,Hkv,d,T,n", [(16, 16, 8, 64, 40, 64), (64, 8, 8, 128, 128, 64), (16, 8, 8, 128, 47, 64),
                                              (16, 16, 8, 256, 50, 32), (32, 16, 8, 128, 90, 32), (16, 32, 8, 80, 70, 16)])
def test_many_rows_over_many_keys_in_one_part(page, H, Hkv, d, T, n, causal):
    # As many row blocks as the chip holds, so that none is cut: a workgroup passes more keys
    # than the 1024 whose pages it has at hand, and again.  The sequences are forks of two.
    c = Cache(n, page, Hkv, d, num_pages=8000 // page + 9, max_pages=5100 // page, seed=T)
    lens = [2500 + page // 2 + 3, 4999]
    c.append([0, 1], lens)
    rest = list(range(2, n))
    c.fork([s % 2 for s in rest], rest)
    q = torch.randn(4, T, H, d, generator=c.gen, device=DEV).bfloat16()
    which = [s % 4 for s in range(n)]                             # slots 0 to 3 with a query each
    b = cache.Batch(n, rows=T)
    ws = cache.workspace(c.pages, c.layer, b, H, max(lens))
    out = torch.empty(n, T, H, d, device=DEV, dtype=torch.bfloat16)
    lse = torch.empty(n, T, H, device=DEV)
    cache.attend(c.pages, c.layer, b, q[which].flatten(0, 1), out.flatten(0, 1), ws, lse=lse.flatten(0, 1),
                 causal=causal, max_tokens=max(lens))
    assert torch.equal(out, out[which]) and torch.equal(lse, lse[which])
    for s in range(4):
        A.check(M.f64(out[s]), M.f64(lse[s]), M.f64(q[s]), c.k[s].x, c.v[s].x, A.per_token(c.v[s]), causal)


@pytest.mark.parametrize("T", [1, 3, 50])
def test_queries_and_outputs_as_slices_of_one_tensor(T):
    c = Cache(2, 32, 2, 64)
    c.append([0, 1], [70, 99])
    H = 4
    both = torch.randn(2 * T, 2 * H, 64, generator=c.gen, device=DEV).bfloat16()
    q, out = both[:, H:], both[:, :H]
    want, b = torch.empty(2 * T, H, 64, device=DEV, dtype=torch.bfloat16), cache.Batch(2, rows=T)
    ws = cache.workspace(c.pages, c.layer, b, H)
    cache.attend(c.pages, c.layer, b, q.contiguous(), want, ws)
    cache.attend(c.pages, c.layer, b, q, out, ws)
    assert torch.equal(out, want)


# ------------------------------------------------------- the attention tests of test_gpu_cache
# Once more, where outputs that are no numbers fail them.
from test_gpu_cache import (test_attend, test_attend_17_to_32_rows_in_one_block,                # noqa: E402,F401
                            test_attend_17_to_32_rows_of_unequal_scale, test_attend_long,
                            test_attend_more_row_blocks_than_threads, test_attend_pages_of_unequal_scale,
                            test_attend_sharp_and_flat_rows, test_attend_uniform_rows_and_strides,
                            test_attend_whatever_the_workspace_held)


@pytest.fixture(autouse=True)
def numbers_only(monkeypatch):
    check = M.check_attention

    def strict(got, lse, *rest):
        assert np.isfinite(got).all(), "%d of %d outputs are no numbers" % (np.sum(~np.isfinite(got)), got.size)
        check(got, lse, *rest)

    monkeypatch.setattr(M, "check_attention", strict)
