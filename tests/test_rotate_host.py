"""Which tensors of one rotation may lie in one another: refused by the host before anything is
enqueued (no call here reaches a launch)."""
import os

import pytest

from paper_2605_29657_amd import build as occam_build
from paper_2605_29657_amd import cache, occam

FAKE = 0x7f0000000000
FAR = FAKE + (1 << 30)
E = 2                                          # bfloat16
ROW = 2 * 128 * E                              # two heads


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(occam.LIB_PATH):
        occam_build.build()
    return cache.lib()


def heads(src, dst, n=2, src_stride=256, dst_stride=None):
    return cache._Heads(src, dst, n, src_stride, dst_stride or src_stride)


def call(L, rows, *tensors):
    r = cache.Rotary(128, [1.0] * 64)
    return L.occam_rotate(r.ref, rows, FAKE, 0, occam.BF16, len(tensors), (cache._Heads * len(tensors))(*tensors), None)


@pytest.mark.parametrize("rows", [1, 16])
def test_the_same_rows_twice(L, rows):
    a = heads(FAKE, FAKE)
    assert call(L, rows, a, a) == occam.ERR_INVALID_ARG
    assert call(L, rows, a, heads(FAKE, FAKE, n=1, src_stride=256)) == occam.ERR_INVALID_ARG       # a head of it
    assert call(L, rows, heads(FAR, FAKE), heads(FAR + (1 << 20), FAKE)) == occam.ERR_INVALID_ARG  # one output
    assert call(L, rows, heads(FAR, FAKE), heads(FAKE, FAR + (1 << 20))) == occam.ERR_INVALID_ARG  # read and written
    assert call(L, rows, heads(FAKE, FAR), heads(FAR, FAKE)) == occam.ERR_INVALID_ARG


@pytest.mark.parametrize("shift", [E, ROW - E, -E, E - ROW])
def test_rows_that_overlap_in_part(L, shift):
    for stride in (256, 384, 512):
        for over in (0, 1, 15):
            b = heads(FAKE + over * stride * E + shift, FAKE + over * stride * E + shift, src_stride=stride)
            assert call(L, 16, heads(FAKE, FAKE, src_stride=stride), b) == occam.ERR_INVALID_ARG, (stride, over)


def test_rows_of_other_strides_that_lie_in_one_another(L):
    assert call(L, 16, heads(FAKE, FAKE, src_stride=512), heads(FAKE + ROW, FAKE + ROW, src_stride=768)) \
        == occam.ERR_INVALID_ARG
