"""The operators on a K/V cache held in 4 bits, as measurable cases.

A next-scale generator appends keys and values at every scale and never drops any, so late scales attend to
tens of thousands of rows per layer. The operators here keep that cache in 4 bits (Cache4) and bound it:

  append     quantise a scale's new keys and values, write them behind the rows in the cache; read them back
  attention  attention of a scale's (kept) queries over the cache, with the log-sum-exp of every row
  weights    the attention weight that each cached row received, added to what it had
  evict      a shorter cache of the rows with the highest weight and the most recent ones; read it back

Format of a row of C channels: groups of 32 channels share a scale s (bf16 with five significant bits, the
largest magnitude over 7, rounded up); a channel is a whole number -7..7 times s, stored plus 8 in four bits.
Eight channels c..c+7 fill a 32-bit word: channel c+2i in bits 4i..4i+3, channel c+2i+1 in bits 16+4i..19+4i.

Sizes are those of the repository's configurations (the VAR-d16 256 shape, 16 heads of 64; the VAR-d30 512 shape,
30 heads of 64; the width-2048 shape at 1024 and 2048, 16 heads of 128) and generic ones around them.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda:0"
GROUP = 32
HEADS = {1024: 16, 1280: 20, 1536: 24, 1920: 30, 2048: 16}


def listed():
    return [
        # One image at its first small scales: a handful of new rows, all latency.
        {"name": "append_one", "kind": "append", "width": 1024, "batch": 1, "rows": 1, "len": 255, "spread": 0.0},
        # The last 1024x1024 scale of four images, about half of the tokens kept, counts that differ by image.
        {"name": "append_1024", "kind": "append", "width": 2048, "batch": 4, "rows": 2431, "len": 6425, "spread": 0.3},
        # A single query of one image against a short cache: the smallest call.
        {"name": "attend_single", "kind": "attention", "width": 1024, "batch": 1, "rows": 1, "len": 424, "spread": 0.0, "empty": False},
        # A late scale that pruning has left a few tokens of, four images with caches of different lengths; one of a
        # batch has no rows in the cache yet.
        {"name": "attend_few", "kind": "attention", "width": 2048, "batch": 5, "rows": 13, "len": 10521, "spread": 0.4, "empty": True},
        # An 8x8 scale's tokens against the longest cache.
        {"name": "attend_64_long", "kind": "attention", "width": 2048, "batch": 1, "rows": 64, "len": 29414, "spread": 0.0, "empty": False},
        # The last 512x512 scale of four images, head size 64, ragged.
        {"name": "attend_512", "kind": "attention", "width": 1920, "batch": 4, "rows": 563, "len": 1779, "spread": 0.35, "empty": False},
        # The last 2048x2048 scale with a fifth of the tokens kept: the largest.
        {"name": "attend_2048", "kind": "attention", "width": 2048, "batch": 1, "rows": 3277, "len": 29414, "spread": 0.0, "empty": False},
        # Weights of a small scale's rows, two images.
        {"name": "weigh_small", "kind": "weights", "width": 1024, "batch": 2, "rows": 9, "len": 680, "spread": 0.2},
        # Weights that the middle 1024x1024 scale gives to what is cached.
        {"name": "weigh_1024", "kind": "weights", "width": 2048, "batch": 2, "rows": 1024, "len": 7449, "spread": 0.25},
        # One layer of one image brought back to a small budget.
        {"name": "evict_one", "kind": "evict", "width": 1024, "batch": 1, "len": 680, "budget": 424, "recent": 100, "spread": 0.0},
        # A layer of eight images that have kept different numbers of rows; the shortest are under the budget.
        {"name": "evict_512", "kind": "evict", "width": 1920, "batch": 8, "len": 2237, "budget": 1216, "recent": 301, "spread": 0.6},
        # All layers of the width-2048 shape at once, after the 64x64 scale: one segment per layer.
        {"name": "evict_layers", "kind": "evict", "width": 2048, "batch": 32, "len": 10521, "budget": 4096, "recent": 2048, "spread": 0.0},
    ]


# ---- drawn cases ---------------------------------------------------------------------------------
def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("append", "attention", "attention", "weights", "evict"))
    width = rng.choice(sorted(HEADS))
    case = {"kind": kind, "width": width, "spread": rng.choice((0.0, round(rng.uniform(0.05, 0.6), 2)))}
    if kind == "append":
        case |= {"batch": rng.randint(1, 8), "rows": _log_int(rng, 1, 1500), "len": _log_int(rng, 1, 8000)}
    elif kind == "attention":
        length = _log_int(rng, 30, 29414)
        batch = max(1, min(rng.randint(1, 6), 60000 // length))
        most = min(3277, 90000000 // (length * batch))
        case |= {"batch": batch, "rows": _log_int(rng, 1, most), "len": length, "empty": batch > 1 and rng.random() < 0.25}
    elif kind == "weights":
        length = _log_int(rng, 30, 12000)
        batch = max(1, min(rng.randint(1, 4), 24000 // length))
        most = min(2048, 15000000 // (length * batch))
        case |= {"batch": batch, "rows": _log_int(rng, 1, most), "len": length}
    else:
        length = _log_int(rng, 40, 12000)
        budget = max(1, int(length * rng.uniform(0.2, 0.9)))
        case |= {"batch": max(1, min(rng.randint(1, 32), 150000 // length)), "len": length, "budget": budget,
                 "recent": int(budget * rng.uniform(0.0, 0.7))}
    return case


# ---- sizes ---------------------------------------------------------------------------------------
def _per_image(most, batch, spread):
    """Sizes of the images of a batch: `most`, and less by up to `spread` of it."""
    return [max(1, int(round(most * (1.0 - spread * i / max(1, batch - 1))))) if batch > 1 else most for i in range(batch)]


def _lengths(case):
    lens = _per_image(case["len"], case["batch"], case["spread"])
    if case.get("empty"):
        lens[-1] = 0
    return lens


def _rows(case):
    return list(reversed(_per_image(case["rows"], case["batch"], case["spread"])))


def _cumulative(counts):
    cu = [0]
    for n in counts:
        cu.append(cu[-1] + n)
    return cu


def work(case):
    C, H = case["width"], HEADS[case["width"]]
    row4 = C // 2 + C // 16                       # bytes of a row's keys, or values: codes and scales
    lens = _lengths(case)
    if case["kind"] == "append":
        m = sum(_rows(case))
        return {"bytes": m * (4 * C + 2 * row4) + m * (2 * row4 + 4 * C), "flops": 8 * m * C}
    if case["kind"] == "attention":
        rows = _rows(case)
        pairs = sum(r * n for r, n in zip(rows, lens))
        return {"bytes": sum(lens) * 2 * row4 + sum(rows) * (4 * C + 4 * H), "flops": 4 * pairs * C}
    if case["kind"] == "weights":
        rows = _rows(case)
        pairs = sum(r * n for r, n in zip(rows, lens))
        return {"bytes": sum(lens) * (row4 + 8) + sum(rows) * (2 * C + 4 * H), "flops": 2 * pairs * C}
    kept = sum(min(n, case["budget"]) for n in lens)
    return {"bytes": sum(lens) * 4 + kept * (4 * row4 + 8) + kept * (2 * row4 + 4 * C), "flops": 2 * kept * C}


# ---- the format ----------------------------------------------------------------------------------
def _quantise(x):
    """[..., C] bf16 -> codes int8 [..., C], scales bf16 [..., C / 32]."""
    g = x.float().unflatten(-1, (-1, GROUP))
    top = g.abs().amax(-1)
    raw = top / torch.full_like(top, 7.0)           # (divided by a number, torch multiplies by its reciprocal)
    s = ((raw.view(torch.int32) + 0x7FFFF) & ~0x7FFFF).view(torch.float32)      # five significant bits, upwards
    s = torch.where(raw > 0, s.clamp(min=2.0 ** -120), torch.zeros_like(s))
    q = torch.where(s[..., None] > 0, g / s[..., None], torch.zeros_like(g))
    return torch.round(q).to(torch.int8).flatten(-2), s.to(torch.bfloat16)


def _pack(codes):
    """int8 [..., C] -> uint8 [..., C / 2]."""
    u = (codes + 8).to(torch.uint8).unflatten(-1, (-1, 8))
    nib = u[..., [0, 2, 4, 6, 1, 3, 5, 7]].unflatten(-1, (4, 2))
    return (nib[..., 0] | (nib[..., 1] << 4)).flatten(-2)


def _unpack(packed):
    """uint8 [..., C / 2] -> int8 [..., C]."""
    p = packed.unflatten(-1, (-1, 4))
    nib = torch.stack((p & 15, p >> 4), -1).flatten(-2)                          # channels 0 2 4 6 1 3 5 7 of each eight
    return (nib[..., [0, 4, 1, 5, 2, 6, 3, 7]].to(torch.int8) - 8).flatten(-2)


def _decode(packed, scales):
    """The values that packed rows stand for, in 32 bits."""
    g = _unpack(packed).float().unflatten(-1, (-1, GROUP))
    return (g * scales.float()[..., None]).flatten(-2)


# ---- inputs --------------------------------------------------------------------------------------
def _randn(gen, *shape):
    return torch.randn(shape, generator=gen, device=DEV, dtype=torch.float32)


def _keys(gen, n, C):
    """Keys as projections give them: channels of different size, some with an offset of their own."""
    size = torch.exp(0.4 * _randn(gen, C))
    return (_randn(gen, n, C) * size + 0.5 * _randn(gen, C)).to(torch.bfloat16)


def _values(gen, n, C):
    return (_randn(gen, n, C) * torch.exp(0.3 * _randn(gen, C))).to(torch.bfloat16)


def _fill(gen, lens, lmax, C):
    """A cache of these lengths: packed keys and values and their scales."""
    B = len(lens)
    out = {n: torch.zeros((B, lmax, C // 2), dtype=torch.uint8, device=DEV) for n in ("k_codes", "v_codes")}
    out |= {n: torch.zeros((B, lmax, C // GROUP), dtype=torch.bfloat16, device=DEV) for n in ("k_scales", "v_scales")}
    for b, n in enumerate(lens):
        for which, make in (("k", _keys), ("v", _values)):
            if n:
                codes, scales = _quantise(make(gen, n, C))
                out[which + "_codes"][b, :n] = _pack(codes)
                out[which + "_scales"][b, :n] = scales
    return out


def _int32(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def _context(state, rows):
    """What a program that uses the framework holds: a context, the cache, its scratch memory."""
    import paper_2602_01345_b200 as nova
    state["nova"] = nova
    state["ctx"] = nova.Context(0)
    state["cache"] = nova.Cache4(state["k_codes"], state["v_codes"], state["k_scales"], state["v_scales"], state["kv_len"],
                                 n_heads=state["heads"])
    state["ctx"].ensure_cache4_workspace(state["cache"], rows)
    return state


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    C, H, B = case["width"], HEADS[case["width"]], case["batch"]
    lens = _lengths(case)
    state = {"kind": case["kind"], "heads": H, "lens": lens, "kv_len": _int32(lens)}
    if case["kind"] == "evict":
        lmax, cut = max(lens), [min(n, case["budget"]) for n in lens]
        state |= _fill(gen, lens, lmax, C)
        # accumulated weights: a few rows hold most, many have received nothing that 32 bits can hold (ties)
        weight = torch.exp(2.0 * _randn(gen, B, lmax)) * (_randn(gen, B, lmax) > -0.5)
        state |= {"weight": weight, "budget": case["budget"], "recent": case["recent"], "kept": cut, "m": sum(cut)}
        state["cu_kept"] = _int32(_cumulative(cut))
        if own:
            _context(state, 0)
            state["dst"] = state["nova"].Cache4.empty(B, case["budget"], C, H, device=DEV)
            state["weight_out"] = torch.empty((B, case["budget"]), dtype=torch.float32, device=DEV)
            state["src_row"] = torch.empty((B, case["budget"]), dtype=torch.int32, device=DEV)
            state["k_out"] = torch.empty((state["m"], C), dtype=torch.bfloat16, device=DEV)
            state["v_out"] = torch.empty((state["m"], C), dtype=torch.bfloat16, device=DEV)
        return state
    rows = _rows(case)
    m = sum(rows)
    state |= {"rows": rows, "cu": _int32(_cumulative(rows)), "m": m}
    lmax = max(n + r for n, r in zip(lens, rows)) if case["kind"] == "append" else max(lens)
    state |= _fill(gen, lens, lmax, C)
    if case["kind"] == "append":
        # a projection's output holds queries, keys and values next to each other
        qkv = torch.cat((_randn(gen, m, C).to(torch.bfloat16), _keys(gen, m, C), _values(gen, m, C)), -1)
        state |= {"k": qkv[:, C:2 * C], "v": qkv[:, 2 * C:]}
        if own:
            _context(state, m)
            state["k_out"] = torch.empty((m, C), dtype=torch.bfloat16, device=DEV)
            state["v_out"] = torch.empty((m, C), dtype=torch.bfloat16, device=DEV)
        return state
    # queries that make some rows attend widely and some to a few keys
    state["q"] = (1.3 * _randn(gen, m, C) * torch.exp(0.5 * _randn(gen, m, 1))).to(torch.bfloat16)
    if case["kind"] == "weights":
        state["lse"] = torch.empty((H, m), dtype=torch.float32, device=DEV)
        for b, h, q, k, _ in _heads(state, torch.float32):
            r0 = sum(rows[:b])
            state["lse"][h, r0:r0 + rows[b]] = torch.logsumexp(q @ k.t(), -1)
        weight = torch.rand((B, lmax), generator=gen, device=DEV) * 4.0
        for b, n in enumerate(lens):
            weight[b, n:] = 0.0
        state["weight"] = weight
    if own:
        _context(state, m)
        if case["kind"] == "weights":
            state["weight_out"] = torch.zeros_like(state["weight"])
        else:
            state["o"] = torch.empty((m, C), dtype=torch.bfloat16, device=DEV)
            state["lse_out"] = torch.empty((H, m), dtype=torch.float32, device=DEV)
    return state


# ---- plain forms ---------------------------------------------------------------------------------
def _heads(state, dtype):
    """Image, head, its scaled queries, keys and values in `dtype`, one after the other."""
    H, C = state["heads"], state["q"].shape[1]
    dh, r0 = C // H, 0
    for b, (n, r) in enumerate(zip(state["lens"], state["rows"])):
        if n and r:
            k = _decode(state["k_codes"][b, :n], state["k_scales"][b, :n]).to(dtype)
            v = _decode(state["v_codes"][b, :n], state["v_scales"][b, :n]).to(dtype) if state["kind"] == "attention" else None
            q = state["q"][r0:r0 + r].to(dtype) / math.sqrt(dh)
            for h in range(H):
                cols = slice(h * dh, (h + 1) * dh)
                yield b, h, q[:, cols], k[:, cols], v[:, cols] if v is not None else None
        r0 += r


def _plain_attention(state):
    H, C, m = state["heads"], state["q"].shape[1], state["m"]
    dh = C // H
    o = torch.zeros((m, C), dtype=torch.float32, device=DEV)
    lse = torch.full((H, m), -math.inf, dtype=torch.float32, device=DEV)
    starts = _cumulative(state["rows"])
    for b, h, q, k, v in _heads(state, torch.float32):
        s = q @ k.t()
        top = s.amax(-1, keepdim=True)
        p = torch.exp(s - top)
        total = p.sum(-1, keepdim=True)
        rows = slice(starts[b], starts[b + 1])
        o[rows, h * dh:(h + 1) * dh] = (p @ v) / total
        lse[h, rows] = (top + torch.log(total))[:, 0]
    return {"o": o.to(torch.bfloat16), "lse": lse}


def _plain_weights(state):
    out = torch.zeros_like(state["weight"])
    starts = _cumulative(state["rows"])
    for b, n in enumerate(state["lens"]):
        out[b, :n] = state["weight"][b, :n]
    for b, h, q, k, _ in _heads(state, torch.float32):
        p = torch.exp(q @ k.t() - state["lse"][h, starts[b]:starts[b + 1], None])
        out[b, :state["lens"][b]] += p.sum(0)
    return {"weight": out}


def _plain_append(state):
    return {which: (codes.float().unflatten(-1, (-1, GROUP)) * s.float()[..., None]).flatten(-2).to(torch.bfloat16)
            for which in ("k", "v") for codes, s in (_quantise(state[which]),)}


def _plain_evict(state):
    B, budget, recent = len(state["lens"]), state["budget"], state["recent"]
    weight_out = torch.zeros((B, budget), dtype=torch.float32, device=DEV)
    src = torch.full((B, budget), -1, dtype=torch.int32, device=DEV)
    k, v = [], []
    for b, n in enumerate(state["lens"]):
        if n <= budget:
            rows = torch.arange(n, device=DEV)
        else:
            old = n - recent
            best = torch.sort(state["weight"][b, :old], descending=True, stable=True).indices[:budget - recent]
            rows = torch.cat((torch.sort(best).values, torch.arange(old, n, device=DEV)))
        src[b, :rows.numel()] = rows.to(torch.int32)
        weight_out[b, :rows.numel()] = state["weight"][b, rows]
        k.append(_decode(state["k_codes"][b, rows], state["k_scales"][b, rows]).to(torch.bfloat16))
        v.append(_decode(state["v_codes"][b, rows], state["v_scales"][b, rows]).to(torch.bfloat16))
    return {"k": torch.cat(k), "v": torch.cat(v), "weight": weight_out, "src_row": src, "kv_len": state["kv_len"].clamp(max=budget)}


# ---- the framework's calls -----------------------------------------------------------------------
def _own_run(state):
    nova, ctx, cache = state["nova"], state["ctx"], state["cache"]
    if state["kind"] == "append":
        # (the lengths stay, as for a layer that is tried out: the next pass writes the same rows)
        nova.nova_cache4_append(ctx, cache, state["k"], state["v"], state["cu"], advance=False)
        nova.nova_cache4_read(ctx, cache, state["cu"], state["k_out"], state["v_out"], first=state["kv_len"])
        return {"k": state["k_out"], "v": state["v_out"]}
    if state["kind"] == "attention":
        nova.nova_cache4_attention(ctx, cache, state["q"], state["cu"], state["o"], lse=state["lse_out"])
        return {"o": state["o"], "lse": state["lse_out"]}
    if state["kind"] == "weights":
        nova.nova_cache4_weights(ctx, cache, state["q"], state["lse"], state["cu"], state["weight_out"], weight_in=state["weight"])
        return {"weight": state["weight_out"]}
    dst = state["dst"]
    nova.nova_cache4_evict(ctx, cache, state["weight"], state["budget"], state["recent"], dst, weight_out=state["weight_out"],
                           src_row=state["src_row"])
    nova.nova_cache4_read(ctx, dst, state["cu_kept"], state["k_out"], state["v_out"])
    return {"k": state["k_out"], "v": state["v_out"], "weight": state["weight_out"], "src_row": state["src_row"], "kv_len": dst.kv_len}


def run(state):
    if own:
        return _own_run(state)
    return {"append": _plain_append, "attention": _plain_attention, "weights": _plain_weights, "evict": _plain_evict}[state["kind"]](state)


# ---- the definition in 64 bits ---------------------------------------------------------------------
def _exact_values(words, scales):
    """Rows decoded one bit field at a time from 32-bit words."""
    w = words.contiguous().view(torch.int32).to(torch.int64)
    x = torch.empty(words.shape[:-1] + (words.shape[-1] * 2,), dtype=torch.float64, device=words.device)
    for i in range(4):
        x[..., 2 * i::8] = ((w >> (4 * i)) & 15).double() - 8.0
        x[..., 2 * i + 1::8] = ((w >> (16 + 4 * i)) & 15).double() - 8.0
    return x * scales.double().repeat_interleave(GROUP, -1)


def _exact_rounded(x):
    """Rows of bf16 values as the cache holds them: scale and whole number from their definitions."""
    g = x.double().reshape(x.shape[0], -1, GROUP)
    top = g.abs().amax(-1, keepdim=True)
    m, e = torch.frexp(torch.true_divide(top, torch.tensor([7.0], dtype=torch.float64, device=DEV)))
    s = torch.ldexp(torch.ceil(m * 32.0) / 32.0, e).clamp(min=2.0 ** -120)
    return (torch.round(g / s) * s).reshape(x.shape)


def exact(case, seed):
    state = prepare(case, seed)
    lens = state["lens"]
    if case["kind"] == "append":
        return {"k": _exact_rounded(state["k"]), "v": _exact_rounded(state["v"])}
    if case["kind"] == "evict":
        weight = torch.zeros((len(lens), case["budget"]), dtype=torch.float64, device=DEV)
        k, v = [], []
        for b, n in enumerate(lens):
            w = state["weight"][b, :n].double().cpu().tolist()
            spare = max(0, min(n, case["budget"]) - min(n, case["recent"]))
            old = sorted(range(n - min(n, case["recent"])), key=lambda j: (-w[j], j))[:spare]
            rows = torch.tensor(sorted(old) + list(range(n - min(n, case["recent"]), n)), device=DEV)
            weight[b, :rows.numel()] = state["weight"][b].double()[rows]
            k.append(_exact_values(state["k_codes"][b][rows], state["k_scales"][b][rows]))
            v.append(_exact_values(state["v_codes"][b][rows], state["v_scales"][b][rows]))
        return {"k": torch.cat(k), "v": torch.cat(v), "weight": weight, "src_row": None, "kv_len": None}
    H, C = state["heads"], case["width"]
    dh, cu = C // H, _cumulative(state["rows"])
    o = torch.zeros((state["m"], H, dh), dtype=torch.float64, device=DEV)
    lse = torch.full((H, state["m"]), -math.inf, dtype=torch.float64, device=DEV)
    weight = state["weight"].double() if case["kind"] == "weights" else None
    for b, n in enumerate(lens):
        if n == 0:
            continue
        q = state["q"][cu[b]:cu[b + 1]].double().view(-1, H, dh)
        k = _exact_values(state["k_codes"][b, :n], state["k_scales"][b, :n]).view(n, H, dh)
        v = _exact_values(state["v_codes"][b, :n], state["v_scales"][b, :n]).view(n, H, dh)
        for h in range(H):
            s = torch.einsum("qd,kd->qk", q[:, h], k[:, h]) * dh ** -0.5
            if weight is not None:
                weight[b, :n] += torch.exp(s - state["lse"][h, cu[b]:cu[b + 1]].double()[:, None]).sum(0)
                continue
            lse[h, cu[b]:cu[b + 1]] = torch.logsumexp(s, -1)
            o[cu[b]:cu[b + 1], h] = torch.softmax(s, -1) @ v[:, h]
    return {"weight": weight} if weight is not None else {"o": o.reshape(state["m"], C), "lse": lse}
