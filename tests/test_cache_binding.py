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
