"""Attention arguments that no launch can hold, refused by the host (no call here reaches one)."""
import os

import pytest

from paper_2605_29657_amd import build as occam_build
from paper_2605_29657_amd import cache, occam

FAKE = 0x7f0000000000


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(occam.LIB_PATH):
        occam_build.build()
    return cache.lib()


def refused(L, status, n, rows, H, Hkv, **kw):
    p = cache._Pages(64, 64, 8192, 4, FAKE, FAKE, FAKE, FAKE, FAKE)
    c = cache._Cache(Hkv, 8, FAKE, FAKE, FAKE, FAKE)
    b = cache._Batch(n, None, rows, None, 0)
    a = cache._Attention(**dict(dict(num_heads=H, causal=1, softmax_scale=0.0, max_tokens=0), **kw))
    return L.occam_cache_workspace_size(p, c, b, a) == 0 and L.occam_cache_attend(
        p, c, b, a, FAKE, 8 * H, FAKE + (1 << 40), 8 * H, None, FAKE, 1 << 50, None) == status


@pytest.mark.parametrize("n,rows,H,Hkv", [(8192, 33, 2048, 2048), (8192, 129, 1024, 1024), (4096, 200, 2500, 2500)])
def test_more_workgroups_than_a_launch_holds(L, n, rows, H, Hkv):
    # 2^32 threads and more, by row blocks that their rows fill badly.
    assert refused(L, occam.ERR_UNSUPPORTED, n, rows, H, Hkv)


@pytest.mark.parametrize("scale", [2.4e38, 3.4e38])
def test_a_scale_past_float32_in_base_2(L, scale):
    assert refused(L, occam.ERR_INVALID_ARG, 4, 1, 8, 2, softmax_scale=scale)


@pytest.mark.parametrize("rows", [1, 5])
@pytest.mark.parametrize("n", [1, 3])
def test_queries_and_outputs_that_overlap(L, n, rows):
    # Of uniform rows, of which the host knows how many there are.
    p = cache._Pages(64, 64, 8, 16, FAKE, FAKE, FAKE, FAKE, FAKE)
    c, b = cache._Cache(2, 128, FAKE, FAKE, FAKE, FAKE), cache._Batch(n, None, rows, None, 0)
    a, row = cache._Attention(8, 1, 0.0, 0), 8 * 128
    size = L.occam_cache_workspace_size(p, c, b, a)
    for stride in (row, row + 256):
        for shift in (0, 256, 2 * row - 16, -256, (n * rows - 1) * stride * 2 + 2 * row - 16):
            assert L.occam_cache_attend(p, c, b, a, FAKE, stride, FAKE + shift, stride, None, FAKE + (1 << 40), size,
                                        None) == occam.ERR_INVALID_ARG, (stride, shift)
    if n * rows > 1:
        assert L.occam_cache_attend(p, c, b, a, FAKE, row, FAKE + 2 * row, 2 * row, None, FAKE + (1 << 40), size,
                                    None) == occam.ERR_INVALID_ARG
