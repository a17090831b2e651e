"""What the binding of the cache's entry points passes on and what it refuses, without a GPU:
its tensors lie on the CPU here (device index -1) and nothing is enqueued."""
import os
import re
import types

import pytest
import torch

from paper_2605_29657_amd import cache, occam


def i32(*x):
    return torch.tensor(x, dtype=torch.int32)


@pytest.fixture
def calls(monkeypatch):
    """The arguments of what would have been enqueued."""
    seen = []
    monkeypatch.setattr(cache, "_enqueue", lambda fn, index, stream, *args: seen.append(args))
    monkeypatch.setattr(cache, "lib", lambda: types.SimpleNamespace(**{n: n for n in cache.EXPORTS}))
    return seen


def pages(num_pages=8, page_tokens=16):
    return types.SimpleNamespace(index=-1, device=torch.device("cpu"), ref=None, num_pages=num_pages,
                                 page_tokens=page_tokens, num_seqs=4, max_pages=4)


def layer(**kw):
    a = dict(num_kv_heads=2, head_dim=8, ref=None, index=-1, num_pages=8, page_tokens=16)
    a.update(kw)
    return types.SimpleNamespace(**a)


def test_no_survivor_at_all(calls):
    # An empty tensor has no address, and the list of survivors may be empty.
    none = torch.zeros(0, dtype=torch.int32)
    offsets, two = i32(0, 0, 0), i32(0, 1)
    assert none.data_ptr() == 0
    cache.keep(pages(), two, two, two, none, offsets, two)
    cache.move(pages(), layer(), two, none, offsets)
    assert calls[0][5] == offsets.data_ptr()
    assert calls[1][5] == offsets.data_ptr() and calls[1][6] == offsets.data_ptr()


def test_status_bits_are_the_headers():
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    text = open(os.path.join(root, "include", "occam_cache.h")).read()
    bits = {n: int(v) for n, v in re.findall(r"OCCAM_PAGES_([A-Z_]+) = (\d+)", text)}
    assert bits == {n: getattr(cache, n) for n in ("FULL", "BAD_SEQ", "TOO_LONG", "BAD_SPAN", "BAD_ROWS")}


def ragged(n=2, most=4):
    return cache.Batch(n, row_offsets=torch.zeros(n + 1, dtype=torch.int32), max_rows=most)


def test_read_wants_keys_and_values_of_the_same_rows(calls):
    k, v = torch.zeros(8, 2, 8), torch.zeros(5, 2, 8)
    for a, b in ((k, v), (v, k)):
        with pytest.raises(occam.OccamError, match="same rows"):
            cache.read(pages(), layer(), ragged(), a, b)
    assert not calls
    for a, b in ((k, k.clone()), (k, None), (None, v)):
        cache.read(pages(), layer(), ragged(), a, b)
    assert len(calls) == 3


@pytest.mark.parametrize("kw", [dict(num_pages=7), dict(page_tokens=32), dict(index=1)])
def test_a_layer_of_other_pages(calls, kw):
    # Its storage has fewer pages, other ones, or lies on another GPU.
    p, c, b = pages(), layer(**kw), cache.Batch(1, rows=3)
    x, plan, idx, ws = torch.zeros(3, 2, 8), i32(0), i32(0, 1), torch.zeros(64, dtype=torch.uint8)
    q = torch.zeros(3, 2, 8, dtype=torch.bfloat16)
    for call in (lambda: cache.append(p, c, b, plan, x, x), lambda: cache.read(p, c, b, x),
                 lambda: cache.move(p, c, plan, idx, idx), lambda: cache.attend(p, c, b, q, q.clone(), ws)):
        with pytest.raises(occam.OccamError, match="layer"):
            call()
    assert not calls


def test_a_layer_of_its_pages_or_of_more(calls):
    b, x = cache.Batch(1, rows=3), torch.zeros(3, 2, 8)
    for c in (layer(), layer(num_pages=9)):
        cache.append(pages(), c, b, i32(0), x, x)
        cache.read(pages(), c, b, x)
        cache.move(pages(), c, i32(0), i32(0), i32(0, 1))
        cache.attend(pages(), c, b, x.bfloat16(), x.bfloat16(), torch.zeros(64, dtype=torch.uint8))
    assert len(calls) == 8


def test_the_workspace_is_one_piece(calls):
    b, q = cache.Batch(1, rows=3), torch.zeros(3, 2, 8, dtype=torch.bfloat16)
    for ws in (torch.zeros(1, dtype=torch.uint8).expand(1 << 20), torch.zeros(64, dtype=torch.uint8)[::2]):
        with pytest.raises(occam.OccamError, match="workspace"):
            cache.attend(pages(), layer(), b, q, q.clone(), ws)
    assert not calls
