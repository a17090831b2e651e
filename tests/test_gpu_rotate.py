"""Rotary positions on the GPU where the angle's own rounding would show."""
import math

import numpy as np
import pytest
import torch

from paper_2605_29657_amd import cache

import cache_model as M
from test_gpu_cache import check_rotated, i32

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.mark.parametrize("adjacent", [False, True])
@pytest.mark.parametrize("inverse", [False, True])
def test_small_sines_keep_the_angles_low_bits(adjacent, inverse):
    # Angles within 2^-8 of half and whole turns: the sine is small and the cosine next to 1 or
    # -1, so that (1, 0) turned shows the angle itself.  The fraction of a turn is good to 2^-40
    # of one here (positions times a fraction in 2^-64, then 2^-56), its sine and the correction
    # by what float32 could not hold to 2^-22 of each; the outputs are sums with zeros.
    r = np.random.default_rng(3)
    n, rows = 64, 40
    freq = [math.pi * (x % 3 + r.choice([-1.0, 1.0]) * 2.0 ** -r.uniform(8, 22)) for x in range(n)]
    pos = i32([1, -1, 3, -5, 2, 7, 0, 4096] * (rows // 8))
    x = torch.zeros(rows, 1, 2 * n, device=DEV)
    first = torch.arange(n, device=DEV) * 2 if adjacent else torch.arange(n, device=DEV)
    x[:, 0, first] = 1.0
    y = torch.empty_like(x)
    cache.rotate(cache.Rotary(2 * n, freq, adjacent=adjacent), pos, [x], [y], inverse=inverse)
    want = M.turned(M.f64(x), pos.cpu().numpy().reshape(rows, 1), [0] * n, freq, adjacent, inverse)
    got = M.f64(y)
    tol = 2 * np.pi * 2.0 ** -40 + 2.0 ** -22 * (np.abs(want) + 2.0 ** -22)
    assert np.all(np.abs(got - want) <= tol), (np.abs(got - want) / tol).max()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_positions_of_every_size(dtype):
    # Whole turns, quarter turns and their neighbours, and positions at both ends of 32 bits.
    freq = [math.pi, math.pi / 2, math.pi / 4, 2 * math.pi, 1.0, 1e-6, 2 * math.pi * (1 - 2.0 ** -30), 0.0]
    pos = torch.tensor([0, 1, -1, 2, 3, 4, 5, 2 ** 31 - 1, -2 ** 31, 2 ** 30, 12345677], dtype=torch.int32, device=DEV)
    x = torch.randn(len(pos), 3, 16, device=DEV).to(dtype)
    y = torch.empty_like(x)
    rot = cache.Rotary(16, freq)
    cache.rotate(rot, pos, [x], [y])
    # (far positions: a frequency's last bit in 2^-64 of a turn moves 2^31 positions by 2^-33)
    check_rotated(y, x, pos, [0] * 8, freq, False, False)
    z = torch.empty_like(x)
    cache.rotate(rot, -pos[:7], [x[:7]], [z[:7]], inverse=True)          # the same turn
    check_rotated(z[:7], x[:7], pos[:7], [0] * 8, freq, False, False)


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("dtype,d,pairs,heads,adjacent", [(torch.bfloat16, 128, 64, [14, 3], False),
                                                          (torch.bfloat16, 128, 32, [12, 8], True),
                                                          (torch.float32, 72, 36, [16, 16], False),
                                                          (torch.float32, 256, 128, [3, 2, 1], False)])
def test_more_rows_than_the_caches_hold(dtype, d, pairs, heads, adjacent, in_place):
    # Past 256 MB tensors go past the caches: against the same rows in parts, bit for bit.
    rows = (300 << 20) // (sum(heads) * d * dtype.itemsize)
    g = torch.Generator(device=DEV).manual_seed(d)
    pos = torch.randint(-9000, 9000, (rows, 3), generator=g, device=DEV, dtype=torch.int32)
    rot = cache.Rotary(d, [1e6 ** (-p / pairs) for p in range(pairs)], [p % 3 for p in range(pairs)], 3, adjacent)
    xs = [torch.randn(rows, h, d, generator=g, device=DEV).to(dtype) for h in heads]
    want = [torch.empty_like(x) for x in xs]
    for a in range(0, rows, 20011):
        z = slice(a, min(a + 20011, rows))
        cache.rotate(rot, pos[z], [x[z] for x in xs], [y[z] for y in want])
    out = xs if in_place else [torch.empty_like(x) for x in xs]
    cache.rotate(rot, pos, xs, None if in_place else out)
    for x, y in zip(out, want):
        assert torch.equal(x, y)
