"""Operators of the serving side of the library, and what each computes in plain torch.

Each case is one pass through an operator of ``paper_2605_29657_amd.cache``:

  rotate   rotary positions with several axes (time, height, width) on query and key rows
  append   prompts written into a paged cache of 8-bit keys and values (one power-of-two
           scale for each page of tokens and head), read back as the values it stands for
  attend   attention of a sequence's last rows over that cache, with the log-normaliser
  prune    sequences forked once for every question, the survivors of their visual span
           kept, the rest dropped, the compacted cache read back, the forks given up
  step     one token of a second answer: fork, rotate, append, attend, free

``own`` chooses between the plain form and the library's calls.  In 8 bits a value is an
e4m3 number times the scale of its block: the smallest power of two that brings the
block's largest magnitude to at most 448, its exponent held within [-100, 120].
"""
from __future__ import annotations

import math
import random

import torch

own = False

DEV = "cuda"
TDT = {"bf16": torch.bfloat16, "f32": torch.float32}
ESZ = {"bf16": 2, "f32": 4}


def _rotate(name=None, **kw):
    c = dict(kind="rotate", rows=8, H=32, Hkv=8, d=128, pairs=64, axes=3, order="interleaved",
             adjacent=False, inverse=False, dtype="bf16", first=0)
    c.update(kw)
    return dict(c, name=name) if name else c


def _cached(kind, name=None, **kw):
    c = dict(kind=kind, B=1, T=1, T_lo=0, L=2880, L_lo=0, H=32, Hkv=8, d=128, page=64,
             dtype="bf16", causal=True, sizes=0)
    c.update(kw)
    return dict(c, name=name) if name else c


def listed():
    return [
        # One decoded token of eight requests: positions with three axes, the smallest launch.
        _rotate("rotate_step", first=4000),
        # A batch of sixteen images with their prompts, text-stage rows of a grouped-query model.
        _rotate("rotate_images", rows=16 * 2211),
        # Head dim 72 of a vision tower, height and width only, float32, the inverse rotation
        # (the gradient of the forward one) over a video's 16384 tokens.
        _rotate("rotate_vision_back", rows=16384, H=16, Hkv=16, d=72, pairs=36, axes=2,
                order="sections", inverse=True, dtype="f32"),
        # One short float32 prompt, odd length, head dim 80, the smallest pages.
        _cached("append", "append_one", L=131, Hkv=4, d=80, page=16, dtype="f32"),
        # A batch of images and prompts of all lengths going into the cache.
        _cached("append", "append_prompts", B=32, L=4608, L_lo=272, sizes=3),
        # One token of one request after a LLaVA-NeXT image: latency.
        _cached("attend", "attend_one", L=3011),
        # One token of 64 requests of all lengths, the smallest pages.
        _cached("attend", "attend_batch", B=64, L=4608, L_lo=272, page=16, sizes=5),
        # One token over eight long videos, as many key heads as query heads.
        _cached("attend", "attend_video", B=8, L=16640, Hkv=32, page=128),
        # Whole prompts of four LLaVA-NeXT images (4 registers, 2880 visual, 128 text tokens).
        _cached("attend", "attend_prompt", B=4, T=3012, L=3012, Hkv=32),
        # The text rows of a ragged batch over images in the cache: what Stage II scores with.
        _cached("attend", "attend_text", B=32, T=512, T_lo=16, L=4096, L_lo=256, sizes=7),
        # Eight images, eight questions each: every question prunes its own fork.
        _cached("prune", "prune_forks", B=8, T=8, L=2919, keep=0.1, before=39),
        # One token of another answer for each of 32 cached sequences.
        _cached("step", "step_forks", B=32, L=4608, L_lo=272, sizes=9),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


# A drawn case does at most the work of the largest listed one of its kind.
MAX_ROTATED = 1.4e8
MAX_CODES = 1.0e9
MAX_FLOPS = 2.9e11


def draw(rng):
    kind = rng.choice(["rotate", "rotate", "append", "attend", "attend", "attend", "attend",
                       "attend", "prune", "step"])
    Hkv = rng.choice([2, 4, 8, 8, 16, 32])
    H = Hkv * rng.choice([1, 2, 4, 7, 8]) if Hkv < 16 else Hkv * rng.choice([1, 2])
    d = rng.choice([64, 80, 96, 128, 128, 128, 256])
    if kind == "rotate":
        pairs = d // 2 if rng.random() < 0.7 else d // 4
        rows = max(1, min(_log_int(rng, 1, 60000), int(MAX_ROTATED / ((H + Hkv) * d))))
        return _rotate(rows=rows, H=H, Hkv=Hkv, d=d, pairs=pairs, axes=rng.choice([1, 2, 3, 3, 4]),
                       order=rng.choice(["interleaved", "sections"]),
                       adjacent=rng.random() < 0.3, inverse=rng.random() < 0.3,
                       dtype=rng.choice(["bf16", "bf16", "f32"]),
                       first=rng.choice([0, 1000, 2000000]))
    c = dict(B=_log_int(rng, 1, 64), L=_log_int(rng, 40, 17000), H=H, Hkv=Hkv, d=d,
             page=rng.choice([16, 32, 64, 64, 128]), sizes=rng.randrange(1, 1 << 20))
    if rng.random() < 0.5:
        c["L_lo"] = max(1, c["L"] // rng.randint(2, 16))
    if kind == "prune":
        c.update(T=rng.randint(1, 8), keep=round(rng.uniform(0.02, 0.4), 3), L_lo=0,
                 before=rng.randint(0, min(60, c["L"] // 4)))
    if kind == "append" and rng.random() < 0.3:
        c["dtype"] = "f32"
    if kind == "attend" and rng.random() < 0.6:
        c.update(T=_log_int(rng, 2, 2048), causal=rng.random() < 0.8)
        if rng.random() < 0.5:
            c["T_lo"] = max(1, c["T"] // rng.randint(2, 8))
    codes = 2 * c["L"] * Hkv * d
    if kind == "attend" and "T" in c:
        c["T"] = max(2, min(c["T"], int(MAX_FLOPS / (4.0 * (c["L"] + c["T"]) * H * d))))
        c["T_lo"] = min(c.get("T_lo", 0), c["T"])
        c["B"] = max(1, min(c["B"], int(MAX_FLOPS / (4.0 * c["T"] * (c["L"] + c["T"]) * H * d))))
    share = 0.15 if kind in ("append", "prune") else 1.0
    c["B"] = max(1, min(c["B"], int(share * MAX_CODES / codes)))
    return _cached(kind, **c)


# ------------------------------------------------------------------------------- shapes
def _counts(case):
    """(rows, keys) of every sequence: part of the case, not of the seed.  ``attend`` with
    one row: L keys in all; with more, the rows come after L cached ones (L == T: none)."""
    r = random.Random(case["sizes"])
    L = [r.randint(case["L_lo"], case["L"]) if case["L_lo"] else case["L"] for _ in range(case["B"])]
    T = [r.randint(case["T_lo"], case["T"]) if case["T_lo"] else case["T"] for _ in range(case["B"])]
    if case["kind"] == "attend" and case["T"] > 1 and case["L"] != case["T"]:
        L = [l + t for l, t in zip(L, T)]
    return T, L


def _kept(case):
    """Survivors of every fork."""
    r = random.Random(case["sizes"] + 1)
    n = case["L"] - case["before"]
    return [max(0, min(n, round(n * case["keep"] * r.uniform(0.5, 1.5))))
            for _ in range(case["B"] * case["T"])]


def _prefix(xs):
    out = [0]
    for x in xs:
        out.append(out[-1] + x)
    return out


def _axes(case):
    """The axis and the frequency (radians per position) of every pair."""
    n, a = case["pairs"], case["axes"]
    size = [n // a + (i < n % a) for i in range(a)]
    if case["order"] == "interleaved":
        axis = [p % a for p in range(n)]
    else:
        axis = [i for i in range(a) for _ in range(size[i])]
    return axis, [1e6 ** (-p / n) for p in range(n)]


def work(case):
    if case["kind"] == "rotate":
        x = float(case["rows"]) * (case["H"] + case["Hkv"]) * case["d"]
        return {"bytes": 2 * x * ESZ[case["dtype"]] + 4.0 * case["rows"] * case["axes"], "flops": 3 * x}
    T, L = _counts(case)
    row = case["Hkv"] * case["d"]
    if case["kind"] == "append":
        # Keys and values in, codes out, and the values that the codes stand for.
        return {"bytes": float(2 * sum(L) * row * (ESZ[case["dtype"]] + 1 + 2)), "flops": 0.0}
    if case["kind"] == "prune":
        # The survivors' codes moved; the compacted sequences read and given as bf16.
        held = sum(_kept(case)) + case["before"] * len(_kept(case))
        return {"bytes": float(2 * row * (2 * sum(_kept(case)) + 3 * held)), "flops": 0.0}
    qrow = case["H"] * case["d"]
    if case["kind"] == "step":
        b = 2 * sum(L) * row + case["B"] * (4 * 2 * row + 2 * 2 * qrow + 4 * case["H"])
        return {"bytes": float(b), "flops": 4.0 * sum(l + 1 for l in L) * qrow}
    seen = sum(t * l - (t * (t - 1) // 2 if case["causal"] else 0) for t, l in zip(T, L))
    return {"bytes": float(2 * sum(L) * row + sum(T) * (2 * 2 * qrow + 4 * case["H"])),
            "flops": 4.0 * seen * qrow}


# ------------------------------------------------------------------------------- inputs
def _i32(xs):
    return torch.tensor(xs, dtype=torch.int32, device=DEV)


def _positions(case):
    """Time, height and width of a run of images (24 patches a row) from position ``first``."""
    i = torch.arange(case["rows"], device=DEV)
    t = case["first"] + i // 576 * 7
    p = torch.stack([t, t + i % 576 // 24, t + i % 24, t + 5], 1)
    return p[:, :case["axes"]].int().contiguous()


def _keys_values(gen, B, L, Hkv, d, dtype):
    """Keys with channels of unequal size and a few tokens that draw attention, values."""
    k = torch.randn(B, L, Hkv, d, generator=gen, device=DEV)
    k.mul_(torch.randn(Hkv, d, generator=gen, device=DEV).mul_(0.5).exp_())
    k[:, :: max(1, L // 5)].mul_(3.0)
    v = torch.randn(B, L, Hkv, d, generator=gen, device=DEV)
    return k.to(TDT[dtype]), v.to(TDT[dtype])


def _inputs(case, seed):
    """The tensors of a case, padded over the batch where sequences differ in length."""
    gen = torch.Generator(device=DEV).manual_seed(int(seed))
    H, Hkv, d = case["H"], case["Hkv"], case["d"]
    if case["kind"] == "rotate":
        dt = TDT[case["dtype"]]
        return dict(pos=_positions(case),
                    q=torch.randn(case["rows"], H, d, generator=gen, device=DEV).to(dt),
                    k=torch.randn(case["rows"], Hkv, d, generator=gen, device=DEV).to(dt))
    B, page = case["B"], case["page"]
    T, L = _counts(case)
    k, v = _keys_values(gen, B, max(L), Hkv, d, case["dtype"])
    x = dict(T=T, L=L, k=k, v=v, lens=torch.tensor(L, device=DEV))
    if case["kind"] == "attend":
        x["q"] = torch.randn(sum(T), H, d, generator=gen, device=DEV).bfloat16()
    if case["kind"] == "step":
        x["q"] = torch.randn(B, H, d, generator=gen, device=DEV).bfloat16()
        x["k1"], x["v1"] = (y[:, 0] for y in _keys_values(gen, B, 1, Hkv, d, "bf16"))
        x["pos"] = (torch.tensor(L, device=DEV).view(B, 1) + torch.arange(3, device=DEV)).int()
    if case["kind"] == "prune":
        n = L[0] - case["before"]
        x["kept"] = [torch.sort(torch.randperm(n, generator=gen, device=DEV)[:c]).values
                     for c in _kept(case)]
    return x


def _step_axes(case):
    return _axes(dict(pairs=case["d"] // 2, axes=3, order="interleaved"))


def prepare(case, seed):
    x = _inputs(case, seed)
    st = dict(case=case)
    if case["kind"] == "rotate":
        axis, freq = _axes(case)
        st.update(x, axis=torch.tensor(axis, device=DEV),
                  freq=torch.tensor(freq, dtype=torch.float64, device=DEV))
        if own:
            from paper_2605_29657_amd import cache
            st["rotary"] = cache.Rotary(case["d"], freq, axis, axes=case["axes"],
                                        adjacent=case["adjacent"])
            st["out"] = [torch.empty_like(x["q"]), torch.empty_like(x["k"])]
        return st
    T, L, B = x["T"], x["L"], case["B"]
    st.update({n: x[n] for n in ("lens", "q", "k1", "v1", "pos") if n in x})
    token = torch.arange(max(L), device=DEV)
    st["held"] = torch.cat([token[:l] + b * max(L) for b, l in enumerate(L)])
    if case["kind"] == "append":
        st.update(k=x["k"].view(-1, case["Hkv"], case["d"])[st["held"]],
                  v=x["v"].view(-1, case["Hkv"], case["d"])[st["held"]])
    else:
        # What the cache holds when the call is made.
        st["k8"], st["ks"] = _quantise(_masked(x["k"], x["lens"]), case["page"])
        st["v8"], st["vs"] = _quantise(_masked(x["v"], x["lens"]), case["page"])
    if case["kind"] == "attend":
        row = torch.arange(max(T), device=DEV)
        rows = torch.tensor(T, device=DEV)
        st.update(rows=rows, at=(torch.tensor(_prefix(T)[:-1], device=DEV).view(B, 1) + row).clamp_(max=sum(T) - 1),
                  packed=torch.cat([row[:t] + b * max(T) for b, t in enumerate(T)]))
    if case["kind"] == "step":
        axis, freq = _step_axes(case)
        st.update(axis=torch.tensor(axis, device=DEV),
                  freq=torch.tensor(freq, dtype=torch.float64, device=DEV))
    if case["kind"] == "prune":
        before, keep = case["before"], x["kept"]
        width = before + max(len(i) for i in keep)
        src = torch.zeros(len(keep), width, dtype=torch.long, device=DEV)
        src[:, :before] = torch.arange(before, device=DEV)
        for f, i in enumerate(keep):
            src[f, before:before + len(i)] = before + i
        news = torch.tensor([before + len(i) for i in keep], device=DEV)
        st.update(src=src, image=torch.arange(len(keep), device=DEV) // case["T"], news=news,
                  packed=torch.cat([torch.arange(n, device=DEV) + f * width
                                    for f, n in enumerate(news.tolist())]))
    if own:
        st.update(_handles(case, x))
    return st


# ------------------------------------------------------------------------- the plain forms
def _masked(x, lens):
    """Tokens behind a sequence's end as zeros."""
    live = torch.arange(x.shape[1], device=DEV) < lens.view(-1, 1)
    return x * live.view(*live.shape, 1, 1).to(x.dtype)


def _exponent(amax):
    """The exponent of the block scale for these largest magnitudes."""
    m, e = torch.frexp(amax)
    return torch.where(amax > 0, e - 9 + (m > 0.875).int(), -100).clamp_(-100, 120)


def _blocks(x, page):
    B, L = x.shape[:2]
    pad = -L % page
    x = torch.cat([x, x.new_zeros(B, pad, *x.shape[2:])], 1) if pad else x
    return x.view(B, -1, page, *x.shape[2:])


def _quantise(x, page):
    """[B, L, Hkv, d] -> e4m3 codes and the scale of every block of ``page`` tokens and head."""
    L = x.shape[1]
    x = _blocks(x.float(), page)
    scale = torch.ldexp(torch.ones((), device=DEV), _exponent(x.abs().amax((2, 4))))
    codes = (x / scale[:, :, None, :, None]).to(torch.float8_e4m3fn)
    return codes.flatten(1, 2)[:, :L], scale


def _values(codes, scale, page):
    L = codes.shape[1]
    return codes.float() * scale.repeat_interleave(page, 1)[:, :L, :, None]


def _turned(x, pos, axis, freq, adjacent, inverse):
    """Rotary positions of rows [n, heads, d]; elements behind the pairs stay."""
    n = freq.numel()
    angle = pos[:, axis].double() * freq
    c, s = angle.cos().float()[:, None], angle.sin().float()[:, None]
    s = -s if inverse else s
    y = x.float()
    a, b = (y[..., 0:2 * n:2], y[..., 1:2 * n:2]) if adjacent else (y[..., :n], y[..., n:2 * n])
    r = (a * c - b * s, a * s + b * c)
    r = torch.stack(r, -1).flatten(-2) if adjacent else torch.cat(r, -1)
    return torch.cat([r, y[..., 2 * n:]], -1).to(x.dtype)


def _attention(q, k, v, last):
    """q [B, T, H, d], k and v [B, L, Hkv, d], last [B, T]: the last key that a row sees.
    Outputs [B, T, H, d] and the natural-log normalisers [B, T, H]."""
    B, T, H, d = q.shape
    Hkv = k.shape[2]
    q = q.float().view(B, T, Hkv, H // Hkv, d).permute(0, 2, 3, 1, 4).reshape(B, Hkv, -1, d)
    s = torch.matmul(q, k.permute(0, 2, 3, 1)).mul_(1.0 / math.sqrt(d)).view(B, Hkv, -1, T, k.shape[1])
    hidden = torch.arange(k.shape[1], device=DEV) > last[:, None, None, :, None]
    s.masked_fill_(hidden, -math.inf)
    m = s.amax(-1, keepdim=True)
    p = s.sub_(m.clamp(min=-3e38)).exp_()
    l = p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(B, Hkv, -1, k.shape[1]), v.transpose(1, 2)).view(B, Hkv, -1, T, d)
    o = o / torch.where(l > 0, l, torch.ones_like(l))
    lse = (m + l.log()).squeeze(-1)
    return o.permute(0, 3, 1, 2, 4).reshape(B, T, H, d), lse.permute(0, 3, 1, 2).reshape(B, T, H)


def run(state):
    c = state["case"]
    if own:
        return _run_own(state, c)
    page = c.get("page")
    if c["kind"] == "rotate":
        return dict(q=_turned(state["q"], state["pos"], state["axis"], state["freq"], c["adjacent"], c["inverse"]),
                    k=_turned(state["k"], state["pos"], state["axis"], state["freq"], c["adjacent"], c["inverse"]))
    if c["kind"] == "append":
        width = max(_counts(c)[1])
        full = state["k"].new_zeros(2, c["B"] * width, c["Hkv"], c["d"])
        full[:, state["held"]] = torch.stack([state["k"], state["v"]])
        y = _values(*_quantise(full.view(2 * c["B"], width, c["Hkv"], c["d"]), page), page)
        y = y.view(2, c["B"] * width, c["Hkv"], c["d"])[:, state["held"]].bfloat16()
        return dict(k=y[0], v=y[1])
    k, v = _values(state["k8"], state["ks"], page), _values(state["v8"], state["vs"], page)
    if c["kind"] == "attend":
        q = state["q"][state["at"]]
        t = torch.arange(q.shape[1], device=DEV)
        last = state["lens"].view(-1, 1) - 1 + ((t - state["rows"].view(-1, 1) + 1) if c["causal"] else 0 * t)
        o, lse = _attention(q, k, v, last)
        return dict(out=o.flatten(0, 1)[state["packed"]].bfloat16(), lse=lse.flatten(0, 1)[state["packed"]])
    if c["kind"] == "prune":
        at = (state["image"].view(-1, 1), state["src"])
        k = _quantise(_masked(k[at], state["news"]), page)
        v = _quantise(_masked(v[at], state["news"]), page)
        return dict(lengths=state["news"].int(),
                    k=_values(*k, page).flatten(0, 1)[state["packed"]].bfloat16(),
                    v=_values(*v, page).flatten(0, 1)[state["packed"]].bfloat16())
    q = _turned(state["q"], state["pos"], state["axis"], state["freq"], False, False)
    k1 = _turned(state["k1"], state["pos"], state["axis"], state["freq"], False, False)
    k, v = (_with_token(x, s, y.float(), state["lens"], page)
            for x, s, y in ((k, state["ks"], k1), (v, state["vs"], state["v1"])))
    o, lse = _attention(q[:, None], k, v, state["lens"].view(-1, 1))
    return dict(out=o[:, 0].bfloat16(), lse=lse[:, 0])


def _with_token(x, scale, new, lens, page):
    """One token more in every sequence: where it raises its block's scale, the block's
    earlier values are rounded once more."""
    B, L, Hkv, d = x.shape
    x = torch.cat([x, x.new_zeros(B, 1, Hkv, d)], 1)
    b = torch.arange(B, device=DEV)
    blk = lens // page
    scale = torch.cat([scale, scale.new_full((B, 1, Hkv), 2.0 ** -100)], 1)
    had = torch.where((lens % page > 0).view(B, 1), scale[b, blk], torch.full_like(scale[:, 0], 2.0 ** -100))
    s = torch.maximum(had, torch.ldexp(torch.ones((), device=DEV), _exponent(new.abs().amax(-1))))
    at = (blk * page).view(B, 1) + torch.arange(page, device=DEV)
    inside = at < lens.view(B, 1)
    at = torch.where(inside, at, lens.view(B, 1))
    old = torch.where(inside.view(B, page, 1, 1), x[b.view(B, 1), at], new[:, None])
    x[b.view(B, 1), at] = (old / s[:, None, :, None]).to(torch.float8_e4m3fn).float() * s[:, None, :, None]
    return x


# --------------------------------------------------------------------- the library's calls
def _handles(case, x):
    """The cache, filled in two rounds as a server does (so that the sequences' pages lie
    between each other), and what a program keeps beside it."""
    from paper_2605_29657_amd import cache
    T, L, B, page = x["T"], x["L"], case["B"], case["page"]
    Hkv, d, H = case["Hkv"], case["d"], case["H"]
    forks = B * case["T"] if case["kind"] == "prune" else B if case["kind"] == "step" else 0
    per_seq = -(-(max(L) + 1) // page)
    total = sum(-(-(l + 1) // page) for l in L) + forks * (per_seq if case["kind"] == "prune" else 2)
    pages = cache.Pages(total, page, B + forks, per_seq)
    layer = cache.Layer(pages, Hkv, d)
    plan = cache.plan(pages, max(B, forks))
    h = dict(pages=pages, layer=layer, plan=plan)
    if case["kind"] == "append":
        offs = _i32(_prefix(L))
        h["batch"] = cache.Batch(B, row_offsets=offs, max_rows=max(L))
        h["slots"] = _i32(list(range(B)))
        n = sum(L)
    else:
        half = [l // 2 // page * page for l in L]
        token = torch.arange(max(L), device=DEV)
        for lo, hi in (([0] * B, half), (half, L)):
            rows = [b - a for a, b in zip(lo, hi)]
            if not any(rows):
                continue
            at = torch.cat([token[a:b] + i * max(L) for i, (a, b) in enumerate(zip(lo, hi))])
            batch = cache.Batch(B, row_offsets=_i32(_prefix(rows)), max_rows=max(rows))
            cache.reserve(pages, batch, plan)
            cache.append(pages, layer, batch, plan, x["k"].view(-1, Hkv, d)[at], x["v"].view(-1, Hkv, d)[at])
        n = 0
    if case["kind"] == "attend":
        ragged = len(set(T)) > 1
        h["batch"] = cache.Batch(B, rows=T[0], row_offsets=_i32(_prefix(T)) if ragged else None, max_rows=max(T))
        h["ws"] = cache.workspace(pages, layer, h["batch"], H, max_tokens=max(L))
        h["out"] = torch.empty_like(x["q"])
        h["lse"] = torch.empty(sum(T), H, device=DEV)
        h["most"] = max(L)
    if case["kind"] == "step":
        axis, freq = _step_axes(case)
        h["rotary"] = cache.Rotary(d, freq, axis, axes=3)
        h["from"], h["to"] = _i32(list(range(B))), _i32(list(range(B, 2 * B)))
        h["batch"] = cache.Batch(B, rows=1, seq=h["to"])
        h["most"] = max(L) + 1
        h["ws"] = cache.workspace(pages, layer, h["batch"], H, max_tokens=h["most"])
        h["qr"], h["kr"], h["out"] = torch.empty_like(x["q"]), torch.empty_like(x["k1"]), torch.empty_like(x["q"])
        h["lse"] = torch.empty(B, H, device=DEV)
    if case["kind"] == "prune":
        counts = [len(i) for i in x["kept"]]
        n = sum(counts) + case["before"] * forks
        h["from"] = _i32([f // case["T"] for f in range(forks)])
        h["to"] = _i32(list(range(B, B + forks)))
        h["start"], h["span"] = _i32([case["before"]] * forks), _i32([L[0] - case["before"]] * forks)
        h["kept_idx"] = torch.cat(x["kept"]).int()
        h["kept_offsets"] = _i32(_prefix(counts))
        rows = [c + case["before"] for c in counts]
        h["batch"] = cache.Batch(forks, seq=h["to"], row_offsets=_i32(_prefix(rows)), max_rows=max(rows))
    if n:
        h["ko"] = torch.empty(n, Hkv, d, dtype=torch.bfloat16, device=DEV)
        h["vo"] = torch.empty(n, Hkv, d, dtype=torch.bfloat16, device=DEV)
    return h


def _run_own(s, c):
    from paper_2605_29657_amd import cache
    if c["kind"] == "rotate":
        cache.rotate(s["rotary"], s["pos"], [s["q"], s["k"]], s["out"], inverse=c["inverse"])
        return dict(q=s["out"][0], k=s["out"][1])
    pages, layer, plan, batch = s["pages"], s["layer"], s["plan"], s["batch"]
    if c["kind"] == "append":
        cache.reserve(pages, batch, plan)
        cache.append(pages, layer, batch, plan, s["k"], s["v"])
        cache.read(pages, layer, batch, s["ko"], s["vo"])
        cache.free(pages, s["slots"])
        return dict(k=s["ko"], v=s["vo"])
    if c["kind"] == "attend":
        cache.attend(pages, layer, batch, s["q"], s["out"], s["ws"], lse=s["lse"], causal=c["causal"],
                     max_tokens=s["most"])
        return dict(out=s["out"], lse=s["lse"])
    cache.fork(pages, s["from"], s["to"], plan)
    if c["kind"] == "prune":
        cache.keep(pages, s["to"], s["start"], s["span"], s["kept_idx"], s["kept_offsets"], plan)
        cache.move(pages, layer, plan, s["kept_idx"], s["kept_offsets"])
        cache.read(pages, layer, batch, s["ko"], s["vo"])
        lengths = pages.length[s["to"]]
        cache.free(pages, s["to"])
        return dict(lengths=lengths, k=s["ko"], v=s["vo"])
    cache.rotate(s["rotary"], s["pos"], [s["q"], s["k1"]], [s["qr"], s["kr"]])
    cache.reserve(pages, batch, plan)
    cache.append(pages, layer, batch, plan, s["kr"], s["v1"])
    cache.attend(pages, layer, batch, s["qr"], s["out"], s["ws"], lse=s["lse"], max_tokens=s["most"])
    cache.free(pages, s["to"])
    return dict(out=s["out"], lse=s["lse"])


# ------------------------------------------------------------------------------- 64 bits
def _round8(x):
    """Nearest e4m3 number, ties to even, of |x| <= 448 in float64."""
    step = torch.exp2(torch.frexp(x)[1].double().sub(1).clamp(min=-6) - 3)
    return torch.round(x / step) * step


def _scale64(x):
    """The block scale of one block [tokens, Hkv, d], per head."""
    top = x.abs().amax((0, 2))
    e = torch.ceil(torch.log2(top.clamp(min=1e-300) / 448.0))
    e = e + (top > 448.0 * torch.exp2(e)).double() - (top <= 448.0 * torch.exp2(e - 1)).double()
    return torch.exp2(torch.where(top > 0, e, torch.full_like(e, -100.0)).clamp(-100, 120))[:, None]


def _held64(x, page):
    """What the cache holds of one sequence [L, Hkv, d] written at once."""
    return torch.cat([_round8(b / _scale64(b)) * _scale64(b) for b in x.double().split(page)])


def _attend64(q, k, v, first_limit, causal):
    """One sequence: q [T, H, d]; row t sees the keys up to first_limit + t (causal) or all."""
    T, H, d = q.shape
    g = H // k.shape[1]
    out, lse = [], []
    for h in range(H):
        s = (q[:, h].double() @ k[:, h // g].t()) / math.sqrt(d)
        if causal:
            s = s.masked_fill(torch.ones_like(s, dtype=torch.bool).triu(first_limit + 1), -math.inf)
        z = torch.logsumexp(s, -1)
        out.append(torch.nan_to_num(torch.exp(s - z[:, None])) @ v[:, h // g])
        lse.append(z)
    return torch.stack(out, 1), torch.stack(lse, 1)


def _turn64(x, pos, axis, freq, adjacent, inverse):
    n = len(freq)
    angle = torch.stack([pos[:, a].double() * f for a, f in zip(axis, freq)], 1)[:, None]
    w = torch.polar(torch.ones_like(angle), -angle if inverse else angle)
    y = x.double().clone()
    i = torch.arange(n, device=DEV)
    a, b = (2 * i, 2 * i + 1) if adjacent else (i, i + n)
    z = torch.complex(y[..., a], y[..., b]) * w
    y[..., a], y[..., b] = z.real, z.imag
    return y


def exact(case, seed):
    x = _inputs(case, seed)
    if case["kind"] == "rotate":
        axis, freq = _axes(case)
        return {n: _turn64(x[n], x["pos"], axis, freq, case["adjacent"], case["inverse"]) for n in ("q", "k")}
    T, L, page = x["T"], x["L"], case["page"]
    held = {n: [_held64(x[n][b, :l], page) for b, l in enumerate(L)] for n in ("k", "v")}
    if case["kind"] == "append":
        return {n: torch.cat(y) for n, y in held.items()}
    if case["kind"] == "prune":
        at = [torch.cat([torch.arange(case["before"], device=DEV), case["before"] + i]) for i in x["kept"]]
        return dict(lengths=None, **{n: torch.cat([_held64(y[f // case["T"]][i], page) for f, i in enumerate(at)])
                                     for n, y in held.items()})
    if case["kind"] == "attend":
        got, first = [], _prefix(T)
        for b in range(case["B"]):
            got.append(_attend64(x["q"][first[b]:first[b + 1]], held["k"][b], held["v"][b],
                                 L[b] - T[b], case["causal"]))
        return dict(out=torch.cat([o for o, _ in got]), lse=torch.cat([z for _, z in got]))
    axis, freq = _step_axes(case)
    q = _turn64(x["q"], x["pos"], axis, freq, False, False).bfloat16()
    k1 = _turn64(x["k1"], x["pos"], axis, freq, False, False).bfloat16()
    got = []
    for b, l in enumerate(L):
        kv = [_held64(torch.cat([y, new[None]]), page) for y, new in
              ((x["k"][b, :l], k1[b].to(x["k"].dtype)), (x["v"][b, :l], x["v1"][b].to(x["v"].dtype)))]
        got.append(_attend64(q[b:b + 1], *kv, l, True))
    return dict(out=torch.cat([o for o, _ in got]), lse=torch.cat([z for _, z in got]))
