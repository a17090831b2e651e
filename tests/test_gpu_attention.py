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
