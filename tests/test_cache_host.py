"""The cache's entry points on the CPU: exported symbols, sizes, and every refusal that the
host makes before anything is enqueued (no call here reaches a launch)."""
import ctypes
import os
import re
import types
from fractions import Fraction

import numpy as np
import pytest
import torch

from paper_2605_29657_amd import build as occam_build
from paper_2605_29657_amd import cache, occam

import cache_model as M

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 0x7f0000000000
INVALID, UNSUPPORTED, WORKSPACE = occam.ERR_INVALID_ARG, occam.ERR_UNSUPPORTED, occam.ERR_WORKSPACE


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(occam.LIB_PATH):
        occam_build.build()
    return cache.lib()


def pages(**kw):
    a = dict(num_pages=64, page_tokens=64, num_seqs=8, max_pages=16, table=FAKE, length=FAKE,
             refs=FAKE, taken=FAKE, status=FAKE)
    a.update(kw)
    return cache._Pages(**a)


def layer(**kw):
    a = dict(num_kv_heads=2, head_dim=128, k=FAKE, v=FAKE, k_scale=FAKE, v_scale=FAKE)
    a.update(kw)
    return cache._Cache(**a)


def batch(**kw):
    a = dict(n=4, seq=None, rows=1, row_offsets=None, max_rows=0)
    a.update(kw)
    return cache._Batch(**a)


def attention(**kw):
    a = dict(num_heads=8, causal=1, softmax_scale=0.0, max_tokens=0)
    a.update(kw)
    return cache._Attention(**a)


def test_header_functions_are_exported_and_bound(L):
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "occam_cache.h")).read(), flags=re.S)
    names = set(re.findall(r"\b(occam_[a-z_]+)\s*\(", text))
    assert names == set(cache.EXPORTS)
    for n in names:
        assert hasattr(L, n)


BAD_PAGES = [dict(num_pages=0), dict(num_pages=(1 << 24) + 1), dict(page_tokens=0),
             dict(page_tokens=8), dict(page_tokens=48), dict(page_tokens=512), dict(num_seqs=0),
             dict(num_seqs=65537), dict(max_pages=0)]


@pytest.mark.parametrize("kw", BAD_PAGES)
def test_bad_pages(L, kw):
    p, c, b = pages(**kw), layer(), batch()
    assert L.occam_pages_plan_size(p, 4) == 0
    assert L.occam_cache_storage_size(p, 2, 128) == 0
    assert L.occam_cache_workspace_size(p, c, b, attention()) == 0
    assert L.occam_pages_reset(p, None) == INVALID
    assert L.occam_pages_reserve(p, b, FAKE, 1 << 30, None) == INVALID
    assert L.occam_pages_fork(p, 4, FAKE, FAKE, FAKE, 1 << 30, None) == INVALID
    assert L.occam_pages_free(p, 4, FAKE, None) == INVALID
    assert L.occam_pages_keep(p, 4, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, 1 << 30, None) == INVALID
    assert L.occam_cache_append(p, c, b, FAKE, 1 << 30, 1, FAKE, 256, FAKE, 256, None) == INVALID
    assert L.occam_cache_read(p, c, b, None, 1, FAKE, 256, FAKE, 256, None) == INVALID
    assert L.occam_cache_move(p, c, 4, FAKE, 1 << 30, FAKE, FAKE, None) == INVALID
    assert L.occam_cache_attend(p, c, b, attention(), FAKE, 1024, FAKE, 1024, None, FAKE, 1 << 30, None) == INVALID


@pytest.mark.parametrize("name", ["table", "length", "refs", "taken", "status"])
@pytest.mark.parametrize("ptr", [None, FAKE + 2])
def test_page_arrays(L, name, ptr):
    assert L.occam_pages_reset(pages(**{name: ptr}), None) == INVALID


def test_positions_stay_in_32_bits(L):
    assert L.occam_pages_reset(pages(max_pages=1 << 25), None) == UNSUPPORTED
    assert L.occam_pages_plan_size(pages(max_pages=(1 << 25) - 1), 1) == 0     # no room to round up
    assert L.occam_pages_plan_size(pages(max_pages=(1 << 25) - 64), 1) > 0
    assert L.occam_cache_storage_size(pages(num_pages=1 << 24), 64, 128) == 0


@pytest.mark.parametrize("kw", [dict(num_kv_heads=0), dict(head_dim=0), dict(head_dim=4),
                                dict(head_dim=20), dict(head_dim=264), dict(k=None), dict(v=FAKE + 8),
                                dict(k_scale=FAKE + 2), dict(v_scale=None)])
def test_bad_layer(L, kw):
    p, c, b = pages(), layer(**kw), batch()
    st = 1 << 14
    assert L.occam_cache_append(p, c, b, FAKE, 1 << 30, 1, FAKE, st, FAKE, st, None) == INVALID
    assert L.occam_cache_read(p, c, b, None, 1, FAKE, st, FAKE, st, None) == INVALID
    assert L.occam_cache_move(p, c, 4, FAKE, 1 << 30, FAKE, FAKE, None) == INVALID
    assert L.occam_cache_attend(p, c, b, attention(), FAKE, st, FAKE, st, None, FAKE, 1 << 40, None) == INVALID


@pytest.mark.parametrize("kw", [dict(n=0), dict(n=8193), dict(rows=0), dict(row_offsets=FAKE, max_rows=0),
                                dict(seq=FAKE + 1), dict(row_offsets=FAKE + 2, max_rows=4), dict(n=9)])
def test_bad_batch(L, kw):
    p, c, b = pages(), layer(), batch(**kw)
    assert L.occam_pages_reserve(p, b, FAKE, 1 << 40, None) == INVALID
    assert L.occam_cache_append(p, c, b, FAKE, 1 << 40, 1, FAKE, 256, FAKE, 256, None) == INVALID
    assert L.occam_cache_read(p, c, b, None, 1, FAKE, 256, FAKE, 256, None) == INVALID
    assert L.occam_cache_workspace_size(p, c, b, attention()) == 0
    assert L.occam_cache_attend(p, c, b, attention(), FAKE, 1024, FAKE, 1024, None, FAKE, 1 << 40, None) == INVALID


def test_plans(L):
    p, b, c = pages(), batch(), layer()
    size = L.occam_pages_plan_size(p, 4)
    assert 0 < size < L.occam_pages_plan_size(p, 5)
    for n in (0, -1, 8193):
        assert L.occam_pages_plan_size(p, n) == 0
        assert L.occam_pages_fork(p, n, FAKE, FAKE, FAKE, 1 << 40, None) == INVALID
        assert L.occam_pages_free(p, n, FAKE, None) == INVALID
    assert L.occam_pages_reserve(p, b, FAKE, size - 1, None) == WORKSPACE
    assert L.occam_pages_fork(p, 4, FAKE, FAKE, FAKE, size - 1, None) == WORKSPACE
    assert L.occam_pages_keep(p, 4, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, size - 1, None) == WORKSPACE
    assert L.occam_cache_append(p, c, b, FAKE, size - 1, 1, FAKE, 256, FAKE, 256, None) == WORKSPACE
    assert L.occam_cache_move(p, c, 4, FAKE, size - 1, FAKE, FAKE, None) == WORKSPACE
    assert L.occam_pages_reserve(p, b, None, size, None) == INVALID
    assert L.occam_pages_reserve(p, b, FAKE + 2, size, None) == INVALID
    for i in range(2):
        args = [FAKE, FAKE]
        for bad in (None, FAKE + 1):
            args[i] = bad
            assert L.occam_pages_fork(p, 4, *args, FAKE, size, None) == INVALID
    for i in range(5):
        for bad in (None, FAKE + 1):
            args = [FAKE] * 5
            args[i] = bad
            assert L.occam_pages_keep(p, 4, *args, FAKE, size, None) == INVALID
    assert L.occam_pages_free(p, 4, None, None) == INVALID


@pytest.mark.parametrize("k,ks,v,vs,dtype", [
    (None, 256, FAKE, 256, 1), (FAKE, 256, None, 256, 1), (FAKE + 8, 256, FAKE, 256, 1),
    (FAKE, 255, FAKE, 256, 1), (FAKE, 252, FAKE, 256, 0), (FAKE, 260, FAKE, 256, 1),
    (FAKE, 256, FAKE, 258, 0), (FAKE, 256, FAKE, 256, 2)])
def test_bad_rows(L, k, ks, v, vs, dtype):
    p, c, b = pages(), layer(), batch()
    assert L.occam_cache_append(p, c, b, FAKE, 1 << 30, dtype, k, ks, v, vs, None) == INVALID
    if k and v:
        assert L.occam_cache_read(p, c, b, None, dtype, k, ks, v, vs, None) == INVALID


def test_read_needs_an_output_and_aligned_starts(L):
    p, c, b = pages(), layer(), batch()
    assert L.occam_cache_read(p, c, b, None, 1, None, 0, None, 0, None) == INVALID
    assert L.occam_cache_read(p, c, b, FAKE + 2, 1, FAKE, 256, None, 0, None) == INVALID


@pytest.mark.parametrize("kw", [dict(num_heads=0), dict(num_heads=7), dict(causal=2), dict(causal=-1),
                                dict(softmax_scale=-1.0), dict(softmax_scale=float("nan")),
                                dict(softmax_scale=float("inf")), dict(max_tokens=-1)])
def test_bad_attention(L, kw):
    p, c, b, a = pages(), layer(), batch(), attention(**kw)
    assert L.occam_cache_workspace_size(p, c, b, a) == 0
    assert L.occam_cache_attend(p, c, b, a, FAKE, 1 << 14, FAKE, 1 << 14, None, FAKE, 1 << 40, None) == INVALID


@pytest.mark.parametrize("q,qs,o,os_,lse", [
    (None, 1024, FAKE, 1024, None), (FAKE, 1024, None, 1024, None), (FAKE + 8, 1024, FAKE, 1024, None),
    (FAKE, 1016, FAKE, 1024, None), (FAKE, 1028, FAKE, 1024, None), (FAKE, 1024, FAKE, 1020, None),
    (FAKE, 1024, FAKE, 1024, FAKE + 2)])
def test_bad_attention_tensors(L, q, qs, o, os_, lse):
    p, c, b, a = pages(), layer(), batch(), attention()
    assert L.occam_cache_attend(p, c, b, a, q, qs, o, os_, lse, FAKE, 1 << 40, None) == INVALID


def test_attention_workspace(L):
    p, c, b, a = pages(), layer(), batch(), attention()
    size = L.occam_cache_workspace_size(p, c, b, a)
    assert size >= 256
    assert L.occam_cache_attend(p, c, b, a, FAKE, 1024, FAKE, 1024, None, FAKE, size - 1, None) == WORKSPACE
    assert L.occam_cache_attend(p, c, b, a, FAKE, 1024, FAKE, 1024, None, FAKE + 16, size, None) == INVALID
    assert L.occam_cache_attend(p, c, b, a, FAKE, 1024, FAKE, 1024, None, None, size, None) == INVALID
    huge = batch(n=8192, seq=FAKE, row_offsets=FAKE, max_rows=1 << 17)
    assert L.occam_cache_workspace_size(p, c, huge, a) == 0
    assert L.occam_cache_attend(p, c, huge, a, FAKE, 1024, FAKE, 1024, None, FAKE, 1 << 50, None) == UNSUPPORTED


def test_attention_does_not_work_in_place(L):
    p, c, b, a = pages(), layer(), batch(), attention()
    size = L.occam_cache_workspace_size(p, c, b, a)
    assert L.occam_cache_attend(p, c, b, a, FAKE, 1024, FAKE, 1024, None, FAKE, size, None) == INVALID


# ------------------------------------------------------------------------------- rotary
def rotary(d=128, freq=(1.0, 0.5), axis=None, axes=1, adjacent=False):
    return cache.Rotary(d, freq, axis, axes, adjacent)


@pytest.mark.parametrize("kw", [dict(d=0), dict(d=3), dict(d=258), dict(freq=()), dict(d=2),
                                dict(axes=0), dict(axes=5), dict(axis=[0, 1]), dict(axis=[0]),
                                dict(axis=[0, 300]), dict(freq=(1.0, float("inf"))),
                                dict(freq=(float("nan"), 1.0))])
def test_bad_rotary(L, kw):
    with pytest.raises(occam.OccamError) as e:
        rotary(**kw)
    assert e.value.status == INVALID


def test_turns_are_exact_fractions(L):
    # inv_freq / 2 pi to 80 digits; the fraction in 2^-64 within one unit of longdouble's.
    two_pi = Fraction("6.28318530717958647692528676655900576839433879875021")
    freq = [1.0, 1e6 ** -0.37, 1e-7, 6.5, -0.25, 0.0, 123456.789]
    r = rotary(freq=freq)
    for p, f in enumerate(freq):
        want = int(Fraction(f) / two_pi % 1 * (1 << 64) + Fraction(1, 2)) % (1 << 64)
        off = (int(r.c.turn[p]) - want) % (1 << 64)
        off = min(off, (1 << 64) - off)
        # 64-bit mantissa: half a unit of the quotient, which for large f has whole turns too.
        assert off <= 2 + abs(f), (f, off)


def test_axis_layouts():
    assert cache.sections([2, 1, 1]) == [0, 0, 1, 2]
    assert cache.interleaved([2, 1, 1]) == [0, 1, 2, 0]
    assert cache.interleaved([4, 2, 2]) == [0, 1, 2, 0, 1, 2, 0, 0]
    assert sorted(cache.interleaved([24, 20, 20])) == sorted(cache.sections([24, 20, 20]))


@pytest.mark.parametrize("kw", [dict(src=None), dict(dst=FAKE + 1), dict(heads=0), dict(src_row_stride=255),
                                dict(dst_row_stride=255), dict(dst=FAKE, dst_row_stride=512),
                                dict(dst=FAKE + 64)])
def test_bad_rotate_tensors(L, kw):
    r = rotary()
    a = dict(src=FAKE, dst=FAKE + (1 << 20), heads=2, src_row_stride=256, dst_row_stride=256)
    a.update(kw)
    assert L.occam_rotate(r.ref, 16, FAKE, 0, 1, 1, (cache._Heads * 1)(cache._Heads(**a)), None) == INVALID


def test_bad_rotate_arguments(L):
    r = rotary()
    h = (cache._Heads * 1)(cache._Heads(FAKE, FAKE, 2, 256, 256))
    assert L.occam_rotate(None, 4, FAKE, 0, 1, 1, h, None) == INVALID
    assert L.occam_rotate(r.ref, -1, FAKE, 0, 1, 1, h, None) == INVALID
    assert L.occam_rotate(r.ref, 4, None, 0, 1, 1, h, None) == INVALID
    assert L.occam_rotate(r.ref, 4, FAKE + 2, 0, 1, 1, h, None) == INVALID
    assert L.occam_rotate(r.ref, 4, FAKE, 0, 3, 1, h, None) == INVALID
    assert L.occam_rotate(r.ref, 4, FAKE, 0, 1, 0, h, None) == INVALID
    assert L.occam_rotate(r.ref, 4, FAKE, 0, 1, 9, h, None) == INVALID
    assert L.occam_rotate(r.ref, 4, FAKE, 0, 1, 1, None, None) == INVALID
    wide = (cache._Heads * 1)(cache._Heads(FAKE, FAKE, 4097, 4097 * 128, 4097 * 128))
    assert L.occam_rotate(r.ref, 4, FAKE, 0, 1, 1, wide, None) == UNSUPPORTED
    zero = cache._Rotary()
    assert L.occam_rotate(ctypes.byref(zero), 4, FAKE, 0, 1, 1, h, None) == INVALID
    assert L.occam_rotate(r.ref, 0, FAKE, 0, 1, 1, h, None) == occam.OK      # nothing to do


def test_more_rows_than_a_launch_has_threads(L):
    r = cache.Rotary(128, [1.0] * 64)
    h = (cache._Heads * 1)(cache._Heads(FAKE, FAKE, 1, 128, 128))
    assert L.occam_rotate(r.ref, (1 << 31) - 1, FAKE, 0, 1, 1, h, None) == UNSUPPORTED


# ------------------------------------------------------------------- the binding's checks
def test_binding_wants_one_offset_more_than_sequences():
    # move() takes the number of sequences from the offsets.
    two, four = torch.zeros(2, dtype=torch.int32), torch.zeros(4, dtype=torch.int32)
    here = types.SimpleNamespace(device=two.device)
    with pytest.raises(occam.OccamError, match="kept_offsets"):
        cache.keep(here, two, two, two, four, four, four)


def test_binding_refuses_what_is_not_on_the_device():
    with pytest.raises(occam.OccamError):
        cache.Pages(4, 16, 2, 2, device="cpu")


def test_binding_checks_rotate():
    r = rotary(d=8, freq=(1.0,))
    x = torch.zeros(3, 2, 8)
    for src, dst, pos in (([], None, torch.zeros(3, dtype=torch.int32)),
                          ([x], [x, x], torch.zeros(3, dtype=torch.int32)),
                          ([x], None, torch.zeros(2, dtype=torch.int32)),
                          ([x.half()], None, torch.zeros(3, dtype=torch.int32)),
                          ([x[:, :, :4]], None, torch.zeros(3, dtype=torch.int32)),
                          ([x, x[:2]], None, torch.zeros(3, dtype=torch.int32))):
        with pytest.raises(occam.OccamError):
            cache.rotate(r, pos, src, dst)


# ------------------------------------------------------------------------------- the model
def test_model_rounding_matches_torch_float8():
    x = torch.cat([torch.randn(4000) * 10.0 ** torch.randint(-3, 3, (4000,)), torch.tensor([0.0, 448, -448, 2.0 ** -10])])
    x = x.clamp(-448, 448)
    assert np.array_equal(M.round8(x.numpy()), x.to(torch.float8_e4m3fn).double().numpy())
    assert set(np.abs(M.E4M3[np.isfinite(M.E4M3)])) >= {448.0, 2.0 ** -9, 0.0}


def test_model_scale_rule():
    for a in (448.0, 448.0001, 224.0, 225.0, 1e-3, 1.75, 1.7500001, 3e38, 1e-45):
        s = M.scale_of(a)
        assert s >= 2.0 ** -100 and (a / s <= 448.0 or s == 2.0 ** 120)
        assert s == 2.0 ** -100 or a / (s / 2) > 448.0
    assert M.scale_of(0.0) == 2.0 ** -100
