"""What serving over a paged key/value cache is judged by: rotary positions, new tokens written into the cache, attention of a chunk
of new tokens over it, and eviction by the attention weight that its keys have gathered.

`listed()` holds the fixed cases and `draw()` gives more of the same ranges; `prepare()` makes what a program has in hand
before the call, `run()` is one call of the public API (`own`) or the same in elementary torch operations, `exact()` the definition
in 64 bits, `work()` what the call cannot do without.

* ``rope``    ``rope``: rotary positions of queries or keys, or the gradient through them
* ``append``  ``cache_append``: new queries and keys rotated, keys and values written into their pages
* ``attn``    ``attn_paged``: each new token attends to its sequence's keys up to its own
* ``weigh``   ``attn_paged`` with ``mass``: the same, and the weights that every cached key received are added up
* ``evict``   ``cache_evict``: the keys of most weight and the latest ones move together, the others are dropped

A cache is ``[pages, kv_heads, page, d]``; the pages of a sequence are the rows of a table.  The new tokens of all sequences lie one
behind the other, ``[tokens, heads, d]``, and are the last ones of their sequences.
"""
from __future__ import annotations

import math
import random

import torch

own = False

_DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
_MOST_SCORES = 4 * 32 * 2048 * 8192  # of the plain form's padded scores
_MOST_CACHE = 1 << 20                # keys of all sequences and heads


def _rope(name, B, H, N, d, rotary, layout, dtype, inverse, at):
    return {"name": name, "op": "rope", "B": B, "H": H, "N": N, "d": d, "rotary": rotary, "layout": layout, "dtype": dtype,
            "inverse": inverse, "at": at}


def _append(name, B, new, kept, Hq, Hkv, d, page, rotary, layout, ragged):
    return {"name": name, "op": "append", "B": B, "new": new, "kept": kept, "Hq": Hq, "Hkv": Hkv, "d": d, "page": page, "rotary": rotary,
            "layout": layout, "ragged": ragged}


def _attn(name, op, B, new, kept, Hq, Hkv, d, page, ragged, sigma=1.0):
    return {"name": name, "op": op, "B": B, "new": new, "kept": kept, "Hq": Hq, "Hkv": Hkv, "d": d, "page": page, "ragged": ragged,
            "sigma": sigma}


def _evict(name, B, Hkv, kept, budget, recent, d, page, ragged):
    return {"name": name, "op": "evict", "B": B, "new": 0, "kept": kept, "Hkv": Hkv, "d": d, "page": page, "budget": budget, "recent": recent,
            "ragged": ragged}


def listed():
    return [
        # The queries of one new token far into a document, half of each head rotated: the latency of a call.
        _rope("rope_token_12x64", 1, 12, 1, 64, 32, "interleaved", "bf16", False, 131071),
        # Gradient of the headline layer's queries in float32, as a training step takes it.
        _rope("rope_grad_f32_4x32x4096", 4, 32, 4096, 128, 128, "half", "f32", True, 0),
        # One decoding step of a batch of 16.
        _append("append_decode_16", 16, 1, 2000, 32, 8, 128, 16, 128, "half", "kept"),
        # Four prompts of the headline's length written into their pages.
        _append("append_prompt_4x4096", 4, 4096, 0, 32, 8, 128, 64, 128, "half", "no"),
        # One new token of one short conversation, a head of keys for each of queries: the smallest decoding step.
        _attn("attn_decode_1x500", "attn", 1, 1, 500, 12, 12, 64, 16, "no"),
        # A decoding step of 24 conversations of all lengths up to 32768 keys, four query heads a key head.
        _attn("attn_decode_24x32768", "attn", 24, 1, 32767, 32, 8, 128, 64, "kept"),
        # A mixed step: prompts of all lengths up to 700 and continuations, over short caches, odd sizes.
        _attn("attn_mixed_20x1021", "attn", 20, 700, 1021, 12, 4, 64, 32, "both"),
        # Long prompts worked off in chunks of 2048: four of them, some 6000 keys behind each.
        _attn("attn_chunk_4x2048", "attn", 4, 2048, 6144, 32, 8, 128, 64, "kept", 2.0),
        # A decoding step that keeps count of what its keys are worth, eight conversations of 4096.
        _attn("weigh_decode_8x4096", "weigh", 8, 1, 4095, 32, 8, 128, 16, "kept"),
        # A chunk of a prompt that does.
        _attn("weigh_chunk_2x1024", "weigh", 2, 1024, 4000, 32, 8, 128, 64, "no", 2.0),
        # One conversation cut back to half.
        _evict("evict_1x4096", 1, 8, 4096, 2048, 128, 128, 16, "no"),
        # A batch of long ones cut back to a quarter.
        _evict("evict_16x16384", 16, 8, 16384, 4096, 1000, 128, 64, "kept"),
    ]


def _log_uniform(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    op = rng.choice(["rope", "append", "attn", "attn", "attn", "weigh", "weigh", "evict"])
    d = rng.choice([64, 128])
    rotary = rng.choice([d, d, d // 2, 16 * rng.randint(1, d // 16)])
    layout = rng.choice(["half", "interleaved"])
    Hkv = rng.choice([1, 2, 4, 8, 8, 12])
    Hq = Hkv * rng.choice([1, 2, 3, 4, 4, 7, 8])
    page = rng.choice([16, 32, 64, 128])
    ragged = rng.choice(["no", "kept", "both"])
    if op == "rope":
        H = rng.choice([1, 8, 12, 32])
        N = _log_uniform(rng, 1, 16384)
        B = rng.choice([1, 1, 2, 4]) if N <= 4096 else 1
        case = _rope("", B, H, N, d, rotary, layout, rng.choice(["bf16", "f32"]), rng.choice([False, True]), _log_uniform(rng, 1, 1 << 20))
    elif op == "append":
        B = _log_uniform(rng, 1, 32)
        new = rng.choice([1, _log_uniform(rng, 1, 16384 // B)])
        case = _append("", B, new, _log_uniform(rng, 1, 4096), min(Hq, 32), Hkv, d, page, rotary, layout, ragged)
        case["Hq"] = max(1, case["Hq"] // Hkv) * Hkv
    elif op == "evict":
        B = _log_uniform(rng, 1, 16)
        kept = _log_uniform(rng, 64, min(16384, 2 * _MOST_CACHE // (B * Hkv)))
        budget = _log_uniform(rng, 16, kept)
        case = _evict("", B, Hkv, kept, budget, rng.randint(0, budget // 2), d, page, ragged)
    else:
        new = rng.choice([1, 1, _log_uniform(rng, 2, 2048)])
        B = _log_uniform(rng, 1, 32 if new < 128 else 8)
        Hq = Hq if Hq <= 32 else 4 * Hkv if Hkv <= 8 else Hkv
        most = min(32768 if new < 128 else 8192, _MOST_SCORES // (4 * B * Hq * new), _MOST_CACHE * 4 // (B * Hkv))
        kept = _log_uniform(rng, 1, max(2, most - new))
        # (float32 sums of weights: scores of a few tens at most, as layers that are normalised have them)
        case = _attn("", op, B, new, kept, Hq, Hkv, d, page, ragged, rng.choice([1.0, 2.0, 4.0] if op == "attn" else [1.0, 1.0, 2.0]))
    del case["name"]
    return case


def _lengths(case):
    """(new tokens, length with them) of each sequence, from the case alone.  "kept": caches of all lengths; "both": new tokens too,
    some sequences with a single one."""
    rng = random.Random(repr(sorted((k, v) for k, v in case.items() if k != "name")))
    part = [(rng.uniform(0.0, 1.0), rng.uniform(0.0, 1.0)) for _ in range(case["B"])]
    kept = [case["kept"] if case["ragged"] == "no" or i == 0 else round(case["kept"] * u) for i, (u, _) in enumerate(part)]
    new = [case["new"] if case["ragged"] != "both" or i == 0 else 1 if w < 0.5 else max(1, round(case["new"] * (2 * w - 1)))
           for i, (_, w) in enumerate(part)]
    if case["op"] == "evict":
        return [(0, max(1, k)) for k in kept]
    return [(n, n + k) for n, k in zip(new, kept)]


def _frequencies(rotary):
    return 10000.0 ** (torch.arange(0, rotary, 2, dtype=torch.float64, device="cuda") / -rotary)


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)

    def normal(*shape, sigma=1.0, dtype=torch.bfloat16):
        return torch.randn(*shape, generator=gen, device="cuda", dtype=dtype).mul_(sigma)

    def int32(values):
        return torch.tensor(values, dtype=torch.int32, device="cuda")

    state = dict(case)
    if case["op"] == "rope":
        B, N = case["B"], case["N"]
        state["X"] = normal(B, case["H"], N, case["d"], dtype=_DTYPES[case["dtype"]])
        state["positions"] = (torch.arange(N, device="cuda") + case["at"]).to(torch.int32).expand(B, N).contiguous()
        state["frequencies"] = _frequencies(case["rotary"])
        return state
    B, Hkv, d, page = case["B"], case["Hkv"], case["d"], case["page"]
    pairs = _lengths(case)
    tokens = sum(n for n, _ in pairs)
    state["most_new"], state["most"] = max(n for n, _ in pairs), max(k for _, k in pairs)
    width = -(-state["most"] // page)
    out_width = -(-case["budget"] // page) if case["op"] == "evict" else 0
    order = torch.randperm(B * (width + out_width), generator=gen, device="cuda").to(torch.int32)  # a pool that has been in use for a while
    state["table"] = order[: B * width].view(B, width)
    state["lengths"] = int32([k for _, k in pairs])
    state["starts"] = int32([sum(n for n, _ in pairs[:i]) for i in range(B + 1)])
    state["K_cache"] = normal(B * (width + out_width), Hkv, page, d, sigma=case.get("sigma", 1.0))
    state["V_cache"] = normal(B * (width + out_width), Hkv, page, d)
    if case["op"] == "evict":
        state["table_out"] = order[B * width:].view(B, out_width)
        # what keys gather: most next to nothing, a few a lot; one in eight nothing at all
        mass = normal(B, Hkv, width * page, sigma=2.0, dtype=torch.float32).exp_()
        state["mass"] = mass * (torch.rand(mass.shape, generator=gen, device="cuda") >= 0.125)
        return state
    state["Q"] = normal(tokens, case["Hq"], d, sigma=case.get("sigma", 1.0))
    if case["op"] == "append":
        state["K"], state["V"] = normal(tokens, Hkv, d), normal(tokens, Hkv, d)
        state["positions"] = int32([k - n + i for n, k in pairs for i in range(n)])
        state["frequencies"] = _frequencies(case["rotary"])
    else:
        state["scale"] = d ** -0.5
        if case["op"] == "weigh":
            state["mass"] = torch.rand(B, Hkv, width * page, generator=gen, device="cuda")
    return state


# ---- the plain forms ---------------------------------------------------------------------------------------------------------


def _rotated(x, angles, layout, sign):
    """`x` [..., d] with its first 2 * angles.shape[-1] features rotated by `sign` times the angles, in 32 bits."""
    r = 2 * angles.shape[-1]
    cos, sin = angles.cos().float(), angles.sin().float() * sign
    x = x.float()
    if layout == "half":
        a, b = x[..., : r // 2], x[..., r // 2: r]
        turned = torch.cat((a * cos - b * sin, b * cos + a * sin), -1)
    else:
        a, b = x[..., 0:r:2], x[..., 1:r:2]
        turned = torch.stack((a * cos - b * sin, b * cos + a * sin), -1).flatten(-2)
    return torch.cat((turned, x[..., r:]), -1)


def _owner(state):
    """Of each new token: its sequence, and the place in it."""
    starts, lengths = state["starts"].long(), state["lengths"].long()
    tokens = torch.arange(state["Q"].shape[0], device="cuda")
    b = torch.searchsorted(starts, tokens, right=True) - 1
    return b, lengths[b] - (starts[b + 1] - tokens)


def _dense(cache, table):
    """The pages of each sequence side by side: [B, kv_heads, keys, d]."""
    x = cache[table.long()].transpose(1, 2)
    return x.reshape(x.shape[0], x.shape[1], -1, x.shape[-1])


def _plain_rope(s):
    angles = s["positions"].double()[:, None, :, None] * s["frequencies"]
    return _rotated(s["X"], angles, s["layout"], -1.0 if s["inverse"] else 1.0).to(s["X"].dtype)


def _plain_append(s):
    angles = s["positions"].double()[:, None, None] * s["frequencies"]
    q = _rotated(s["Q"], angles, s["layout"], 1.0).to(s["Q"].dtype)
    k = _rotated(s["K"], angles, s["layout"], 1.0).to(s["K"].dtype)
    b, at = _owner(s)
    page = s["table"].long()[b, at // s["page"]]
    s["K_cache"][page, :, at % s["page"]] = k
    s["V_cache"][page, :, at % s["page"]] = s["V"]
    return {"Q": q, "K_cache": s["K_cache"], "V_cache": s["V_cache"]}


def _plain_attn(s):
    B, Hkv, d, n = s["B"], s["Hkv"], s["d"], s["most_new"]
    G = s["Hq"] // Hkv
    starts, lengths = s["starts"].long(), s["lengths"].long()
    new = (starts[1:] - starts[:-1])[:, None]
    i = torch.arange(n, device="cuda")
    here = i < new                                                                    # [B, n]
    token = torch.where(here, starts[:-1, None] + i, 0)
    q = s["Q"][token].float().view(B, n, Hkv, G, d).permute(0, 2, 1, 3, 4).reshape(B, Hkv, n * G, d)
    j = torch.arange(s["table"].shape[1] * s["page"], device="cuda")
    seen = j <= (lengths[:, None] - new + i)[:, :, None]                                 # [B, n, keys]
    seen = (seen & here[:, :, None])[:, None, :, None, :]
    k = _dense(s["K_cache"], s["table"]).float()
    scores = (q @ k.transpose(2, 3)).mul_(s["scale"]).view(B, Hkv, n, G, -1).masked_fill_(~seen, -math.inf)
    top = scores.amax(-1, keepdim=True).clamp_min(-1e30)
    p = scores.sub_(top).exp_()
    p = p.div_(p.sum(-1, keepdim=True).clamp_min(1e-30))
    v = torch.where((j < lengths[:, None])[:, None, :, None], _dense(s["V_cache"], s["table"]).float(), 0.0)
    o = (p.view(B, Hkv, n * G, -1) @ v).view(B, Hkv, n, G, d).permute(0, 2, 1, 3, 4).reshape(B, n, Hkv * G, d)
    O = o[here].to(s["Q"].dtype)
    return {"O": O, "mass": s["mass"] + p.sum((2, 3))} if s["op"] == "weigh" else O


def _plain_evict(s):
    lengths, budget, recent, page, B, Hkv = s["lengths"].long(), s["budget"], s["recent"], s["page"], s["B"], s["Hkv"]
    j = torch.arange(s["mass"].shape[2], device="cuda")
    left = lengths.clamp_max(budget)
    rank = s["mass"].masked_fill((j >= (lengths - recent)[:, None])[:, None], math.inf).masked_fill((j >= lengths[:, None])[:, None], -math.inf)
    order = rank.sort(dim=-1, descending=True, stable=True).indices
    t = torch.arange(budget, device="cuda")
    there = (t < left[:, None])[:, None].expand(B, Hkv, budget)                          # [B, kv_heads, budget]
    order = torch.nn.functional.pad(order, (0, max(0, budget - order.shape[2])))[..., :budget]
    kept = order.masked_fill(~there, j.shape[0]).sort(dim=-1).values
    source = kept.masked_fill(~there, 0)
    b = torch.arange(B, device="cuda")[:, None, None].expand_as(kept)[there]
    h = torch.arange(Hkv, device="cuda")[None, :, None].expand_as(kept)[there]
    at = t.expand_as(kept)[there]
    from_page, to_page = s["table"].long()[b, source[there] // page], s["table_out"].long()[b, at // page]
    s["K_cache"][to_page, h, at % page] = s["K_cache"][from_page, h, source[there] % page]
    s["V_cache"][to_page, h, at % page] = s["V_cache"][from_page, h, source[there] % page]
    mass = torch.zeros(B, Hkv, s["table_out"].shape[1] * page, device="cuda")
    mass[..., :budget] = s["mass"].gather(2, source).masked_fill(~there, 0.0)
    return {"kept": kept.masked_fill(~there, -1).to(torch.int32), "lengths": left.to(torch.int32), "mass": mass, "K_cache": s["K_cache"],
            "V_cache": s["V_cache"]}


# ---- the framework's calls ---------------------------------------------------------------------------------------------------


def _own(s):
    from paper_2407_13885_b200 import binding
    op = s["op"]
    if op == "rope":
        return binding.rope(s["X"], s["positions"], s["frequencies"], layout=s["layout"], inverse=s["inverse"])
    if op == "append":
        q = binding.cache_append(s["Q"], s["K"], s["V"], s["K_cache"], s["V_cache"], s["table"], s["lengths"], s["starts"], s["positions"],
                                 s["frequencies"], layout=s["layout"])
        return {"Q": q, "K_cache": s["K_cache"], "V_cache": s["V_cache"]}
    if op == "evict":
        kept, lengths, mass = binding.cache_evict(s["K_cache"], s["V_cache"], s["table"], s["lengths"], s["mass"], s["budget"], s["recent"],
                                                  table_out=s["table_out"])
        return {"kept": kept, "lengths": lengths, "mass": mass, "K_cache": s["K_cache"], "V_cache": s["V_cache"]}
    if op == "weigh":
        O, mass = binding.attn_paged(s["Q"], s["K_cache"], s["V_cache"], s["table"], s["lengths"], s["starts"], s["scale"], mass=s["mass"])
        return {"O": O, "mass": mass}
    return binding.attn_paged(s["Q"], s["K_cache"], s["V_cache"], s["table"], s["lengths"], s["starts"], s["scale"])


_PLAIN = {"rope": _plain_rope, "append": _plain_append, "attn": _plain_attn, "weigh": _plain_attn, "evict": _plain_evict}


def run(state):
    return _own(state) if own else _PLAIN[state["op"]](state)


def work(case):
    if case["op"] == "rope":
        size, tokens = (4 if case["dtype"] == "f32" else 2), case["B"] * case["N"]
        return {"bytes": tokens * (2 * case["H"] * case["d"] * size + 4) + 4 * case["rotary"], "flops": 3 * tokens * case["H"] * case["rotary"]}
    pairs, Hkv, d = _lengths(case), case["Hkv"], case["d"]
    tokens, keys = sum(n for n, _ in pairs), sum(k for _, k in pairs)
    index = 4 * (2 * case["B"] + 1 + sum(-(-k // case["page"]) for _, k in pairs))  # lengths, starts, table
    if case["op"] == "append":
        rows = case["Hq"] + 2 * Hkv
        return {"bytes": tokens * (2 * rows * d * 2 + 4) + 4 * case["rotary"] + index, "flops": 3 * tokens * (case["Hq"] + Hkv) * case["rotary"]}
    if case["op"] == "evict":
        left = sum(min(k, case["budget"]) for _, k in pairs)
        out = case["B"] * Hkv * case["budget"] * 4 + case["B"] * Hkv * -(-case["budget"] // case["page"]) * case["page"] * 4
        return {"bytes": Hkv * (keys * 4 + left * 2 * 2 * d * 2) + out + index, "flops": 0}
    seen = sum(n * k - n * (n - 1) // 2 for n, k in pairs)
    mass = 2 * 4 * case["B"] * Hkv * -(-max(k for _, k in pairs) // case["page"]) * case["page"] if case["op"] == "weigh" else 0
    return {"bytes": 2 * d * (2 * tokens * case["Hq"] + 2 * keys * Hkv) + mass + index, "flops": 4 * seen * case["Hq"] * d}


# ---- the definition in 64 bits -----------------------------------------------------------------------------------------------


def _turn(x, position, frequencies, layout, inverse):
    """Every pair of features as a complex number times e^(i position frequency), the conjugate for the gradient; tokens first."""
    r = 2 * frequencies.numel()
    first, second = ((slice(0, r // 2), slice(r // 2, r)) if layout == "half" else (slice(0, r, 2), slice(1, r, 2)))
    x = x.double().clone()
    z = torch.complex(x[..., first], x[..., second])
    w = torch.polar(torch.ones_like(position.double())[..., None] * torch.ones_like(frequencies), position.double()[..., None] * frequencies)
    w = w.conj() if inverse else w
    z = z * w.view(w.shape[:-1] + (1,) * (z.dim() - w.dim()) + w.shape[-1:])
    x[..., first], x[..., second] = z.real, z.imag
    return x


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "rope":
        return _turn(s["X"].transpose(1, 2), s["positions"], s["frequencies"], s["layout"], s["inverse"]).transpose(1, 2).contiguous()
    page, Hkv, d, pairs = case["page"], case["Hkv"], case["d"], _lengths(case)
    if op == "append":
        k = _turn(s["K"], s["positions"], s["frequencies"], s["layout"], False)
        K, V = s["K_cache"].double(), s["V_cache"].double()
        t = 0
        for b, (n, length) in enumerate(pairs):
            at = torch.arange(length - n, length, device="cuda")
            pages = s["table"][b].long()[torch.div(at, page, rounding_mode="floor")]
            K[pages, :, at % page], V[pages, :, at % page] = k[t: t + n], s["V"][t: t + n].double()
            t += n
        return {"Q": _turn(s["Q"], s["positions"], s["frequencies"], s["layout"], False), "K_cache": K, "V_cache": V}
    if op == "evict":
        width = case["budget"]
        kept = torch.full((case["B"], Hkv, width), -1, dtype=torch.int64)
        mass = torch.zeros(case["B"], Hkv, s["table_out"].shape[1] * page, dtype=torch.float64)
        weights = s["mass"].double().cpu()
        for b, (_, length) in enumerate(pairs):
            for h in range(Hkv):
                if length <= width:
                    chosen = torch.arange(length)
                else:
                    recent = min(case["recent"], width)
                    old = weights[b, h, : length - recent]
                    best = torch.argsort(old, descending=True, stable=True)[: width - recent]
                    chosen = torch.cat((best.sort().values, torch.arange(length - recent, length)))
                kept[b, h, : len(chosen)] = chosen
                mass[b, h, : len(chosen)] = weights[b, h, chosen]
        return {"kept": kept.to(torch.int32), "lengths": torch.tensor([min(k, width) for _, k in pairs], dtype=torch.int32), "mass": mass,
                "K_cache": None, "V_cache": None}
    G = case["Hq"] // Hkv
    O = torch.zeros(s["Q"].shape, dtype=torch.float64, device="cuda")
    mass = s["mass"].double() if op == "weigh" else None
    t = 0
    for b, (n, length) in enumerate(pairs):
        pages = s["table"][b, : -(-length // page)].long()
        for h in range(Hkv):
            k, v = (c[pages, h].double().reshape(-1, d)[:length] for c in (s["K_cache"], s["V_cache"]))
            for at in range(0, n, 256):
                m = min(256, n - at)
                q = s["Q"][t + at: t + at + m, h * G: (h + 1) * G].double()
                z = torch.einsum("mgd,jd->mgj", q, k) * s["scale"]
                hidden = torch.arange(length, device="cuda")[None, :] > torch.arange(length - n + at, length - n + at + m, device="cuda")[:, None]
                p = torch.softmax(z.masked_fill(hidden[:, None], -math.inf), -1)
                O[t + at: t + at + m, h * G: (h + 1) * G] = torch.einsum("mgj,jd->mgd", p, v)
                if mass is not None:
                    mass[b, h, :length] += p.sum((0, 1))
        t += n
    return {"O": O, "mass": mass} if op == "weigh" else O
