"""The operators of models that look at images, video or an encoder's states, as a program uses them: rotary positions with
several axes, quantised into a paged cache (``hccs_cache_write_axes``) or into dense tensors (``hccs_states_write``), and
HCCS attention to states of another length (``hccs_attention_cross``).

``run`` computes them in their plain form with elementary torch operations, or, where ``own`` is true, by the
calls of this framework.  Codes (int8) are whole numbers here: they are what the integer attention consumes, so they
are returned and compared as such.
"""
import math
import random

import numpy as np
import torch

own = False

DEV = "cuda"
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32, "i32": torch.int32}
SHIFT = 20                 # requantisation of the logits: x = clamp((acc * M + 2^19) >> 20)


# ------------------------------------------------------------------------------------------------ cases
def _write(name, tokens, heads, kv_heads, dim, page, dtype, layout, pairs, order, restart, far, skip):
    """Tokens into a paged cache; ``pairs`` are the pairs of each axis, as text."""
    return {"name": name, "op": "write", "tokens": tokens, "heads": heads, "kv_heads": kv_heads, "dim": dim, "page": page,
            "dtype": dtype, "layout": layout, "pairs": pairs, "order": order, "restart": restart, "far": far, "skip": skip}


def _states(name, batch, length, heads, kv_heads, dim, dtype, layout, pairs, order, restart, heads_first):
    """Tokens into dense tensors; heads 0: keys and values alone, no pairs: no rotation."""
    return {"name": name, "op": "states", "batch": batch, "length": length, "heads": heads, "kv_heads": kv_heads, "dim": dim,
            "dtype": dtype, "layout": layout, "pairs": pairs, "order": order, "restart": restart, "heads_first": heads_first}


def _cross(name, batch, queries, length, heads, kv_heads, dim, norm, dtype, ragged, wide, share, fused, ranges):
    """``share`` sequences read the same states; fused: keys and values are views of one tensor; ranges: images per sequence, of
    which a query sees one or none (0: all keys are seen)."""
    return {"name": name, "op": "cross", "batch": batch, "queries": queries, "length": length, "heads": heads, "kv_heads": kv_heads,
            "dim": dim, "norm": norm, "dtype": dtype, "ragged": ragged, "wide": wide, "share": share, "fused": fused, "ranges": ranges}


def listed():
    return [
        # one generation step of four sequences whose prompts hold images: latency counts
        _write("axes step", 4, 32, 8, 128, 64, "bf16", "half", "16,24,24", "sections", False, 4000, False),
        # a batch of video prompts: frames, rows and columns in turn over the pairs
        _write("axes video", 16384, 32, 8, 128, 64, "bf16", "half", "24,20,20", "turns", False, 60000, False),
        # a padded batch, rows and columns on half of a head each with frequencies of its own, padding tokens skipped
        _write("axes padded", 1003, 12, 12, 64, 16, "f16", "interleaved", "16,16", "sections", True, 60, True),
        # patches of a batch of images, as the fused attention reads them
        _states("states image", 16, 1024, 12, 12, 64, "f16", "half", "16,16", "sections", True, True),
        # keys and values of an encoder's states, not rotated
        _states("states encoder", 8, 1499, 0, 16, 64, "f32", "half", "", "sections", False, False),
        # one token of one short sequence, integer output of the paper's int16 path
        _cross("cross one", 1, 1, 577, 12, 12, 64, "div", "i32", False, False, 1, False, 0),
        # a generation step of a batch of ragged inputs, two hypotheses each
        _cross("cross step", 32, 1, 1499, 16, 16, 64, "real", "bf16", True, False, 2, False, 0),
        # a generation step that looks at long videos
        _cross("cross video", 8, 1, 32768, 32, 8, 128, "real", "bf16", False, True, 1, True, 0),
        # positions of an image that look at a short text
        _cross("cross text", 8, 4096, 77, 16, 16, 64, "real", "f16", False, False, 1, False, 0),
        # ragged texts on the patches of one image each, leading-bit reciprocal
        _cross("cross patches", 24, 700, 256, 32, 8, 128, "clb", "bf16", True, False, 1, True, 0),
        # texts that see one image of four at a time, or none yet
        _cross("cross images", 2, 1001, 2404, 16, 4, 128, "real", "f32", True, True, 1, False, 4),
        # prompts on long states
        _cross("cross prompt", 2, 2048, 6404, 32, 8, 128, "real", "bf16", False, True, 1, False, 0),
    ]


def _spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _some_pairs(rng, dim, layout):
    """Pairs of each axis: all of a head, half of it, or odd shares."""
    total = rng.choice([dim // 2, dim // 2, dim // 4])
    axes = rng.choice([2, 3, 3, 4])
    if rng.random() < 0.5:
        cut = [total // axes + (1 if i < total % axes else 0) for i in range(axes)]
    else:
        at = sorted(rng.sample(range(1, total), axes - 1))
        cut = [b - a for a, b in zip([0] + at, at + [total])]
    return ",".join(str(c) for c in cut)


def draw(rng):
    op = rng.choice(["write", "write", "states", "states", "step", "step", "few", "text", "prompt", "images"])
    dim = rng.choice([64, 128])
    kv_heads = rng.choice([1, 2, 3, 4, 5, 8, 12, 16])
    group = rng.choice([1, 1, 2, 3, 4, 7, 8])
    if kv_heads * group > 64:
        group = 1
    heads = kv_heads * group
    layout, dtype = rng.choice(["half", "interleaved"]), rng.choice(["bf16", "f16", "f32"])
    most = 16384 * 48 * 128 // ((heads + 2 * kv_heads) * dim) // 2
    if op == "write":
        case = _write("", _spread(rng, 1, max(16, most)), heads, kv_heads, dim, rng.choice([16, 32, 64, 128, 256]), dtype, layout,
                      _some_pairs(rng, dim, layout), rng.choice(["sections", "turns"]), rng.random() < 0.4, _spread(rng, 1, 60000),
                      rng.random() < 0.3)
    elif op == "states":
        batch = rng.randint(1, 16)
        case = _states("", batch, _spread(rng, 1, max(16, most // batch)), rng.choice([0, heads, heads]), kv_heads, dim, dtype, layout,
                       rng.choice(["", _some_pairs(rng, dim, layout), _some_pairs(rng, dim, layout)]), rng.choice(["sections", "turns"]),
                       rng.random() < 0.5, rng.random() < 0.5)
    else:
        share = 1
        if op == "step":
            batch, queries = _spread(rng, 1, 48), 1
            share = rng.choice([1, 1, 2, 4])
            length = _spread(rng, 1, min(32768, max(2, 8 * 32768 * 8 * 128 // (batch * kv_heads * dim))))
        elif op == "few":
            batch, queries = rng.randint(1, 16), rng.randint(2, 40)
            length = _spread(rng, 1, min(16384, max(2, 4 * 32768 * 8 * 128 // (batch * kv_heads * dim))))
        elif op == "text":
            batch, queries = rng.randint(1, 12), _spread(rng, 64, 4096)
            length = _spread(rng, 1, 512)
        else:
            batch, queries = rng.randint(1, 4), _spread(rng, 64, 1500)
            length = _spread(rng, 200, 8000)
        # the cost of many queries grows with their pairs with keys, and the bytes with their rows
        while batch * queries * heads * length > 2 * 2048 * 6404 * 32 // 2 or batch * queries * heads * dim > 8 * 4096 * 16 * 64:
            if queries > 64:
                queries = queries * 2 // 3
            elif batch > 1:
                batch -= 1
            else:
                length = length * 2 // 3
        ranges = rng.randint(1, 5) if op == "images" else 0
        wide = length > 4000 or rng.random() < 0.3
        norm = "real" if wide else rng.choice(["real", "div", "clb"])
        out = rng.choice(["bf16", "f16", "f32"]) if norm == "real" or rng.random() < 0.5 else "i32"
        case = _cross("", batch, queries, max(length, ranges), heads, kv_heads, dim, norm, out, rng.random() < 0.6, wide, share,
                      rng.random() < 0.5, ranges)
    return {k: v for k, v in case.items() if k != "name"}


def _lengths(case):
    """(query lengths, key lengths) of the sequences: properties of the case, not of its seed.  Sequences that share their
    states have one length."""
    r = random.Random(case["length"] * 131 + case["batch"])
    n, share = case["batch"], case["share"]
    if not case["ragged"]:
        return [case["queries"]] * n, [case["length"]] * n
    q = [case["queries"]] + [r.randint(1, case["queries"]) for _ in range(n - 1)]
    k = [case["length"]] + [r.randint(max(1, case["length"] // 3), case["length"]) for _ in range(n - 1)]
    return q, [k[i - i % share] for i in range(n)]


def _ranges(case):
    """(first key, end) of what every query sees: nothing before the first image, then the image that came last."""
    r = random.Random(case["queries"] * 17 + case["ranges"])
    got = []
    for nq, n in zip(*_lengths(case)):
        images = case["ranges"]
        per = -(-n // images)
        at = sorted(r.randint(0, nq) for _ in range(images))
        for t in range(nq):
            last = sum(1 for a in at if a <= t) - 1
            got.append((min(last * per, n), min(last * per + per, n)) if last >= 0 else (0, 0))
    return got


def work(case):
    size = {"bf16": 2, "f16": 2, "f32": 4, "i32": 4}[case["dtype"]]
    if case["op"] in ("write", "states"):
        tokens = case["tokens"] if case["op"] == "write" else case["batch"] * case["length"]
        n = tokens * (case["heads"] + 2 * case["kv_heads"]) * case["dim"]
        axes = len(case["pairs"].split(",")) if case["pairs"] else 0
        return {"bytes": n * (size + 1) + tokens * (4 * axes + (8 if case["op"] == "write" else 0)), "flops": 4 * n}
    q, k = _lengths(case)
    pairs = sum(b - a for a, b in _ranges(case)) if case["ranges"] else sum(a * b for a, b in zip(q, k))
    states = sum(k[::case["share"]])
    row = case["heads"] * case["dim"]
    return {"bytes": 2 * states * case["kv_heads"] * case["dim"] + sum(q) * row * (1 + size), "flops": 4 * case["dim"] * pairs * case["heads"]}


# ------------------------------------------------------------------------------------------------ inputs
def axes_of(case):
    """(frequency, axis) of every pair: in sections, or in turn among the axes that have pairs left; frequencies over all of the
    rotated part, or each axis's own from the first on."""
    count = [int(c) for c in case["pairs"].split(",")] if case["pairs"] else []
    total = sum(count)
    if case["order"] == "sections":
        axis = [a for a, c in enumerate(count) for _ in range(c)]
    else:
        axis, left, a = [], list(count), 0
        while len(axis) < total:
            if left[a]:
                axis.append(a)
                left[a] -= 1
            a = (a + 1) % len(count)
    freq, seen = [], [0] * len(count)
    for i, a in enumerate(axis):
        freq.append(10000.0 ** (-seen[a] / count[a]) if case["restart"] else 10000.0 ** (-i / total))
        seen[a] += 1
    return freq, axis


def _positions(tokens, axes, far):
    """int32 [axes, tokens]: some text, then frames of 24 x 16 patches, then text again; a text token has one position on all axes."""
    t = torch.arange(tokens, device=DEV)
    text = tokens // 8
    patch = (t - text).clamp(min=0)
    grid = [patch // 384, patch // 16 % 24, patch % 16][-axes:] if axes <= 3 else [patch // 768, patch // 384 % 2, patch // 16 % 24, patch % 16]
    rows = [torch.where(t < text, t, torch.where(t < tokens - text, text + g, t)) + far for g in grid]
    return torch.stack(rows).to(torch.int32)


def _codes(shape, g):
    """int8 codes as attention reads them: a bell of width 32."""
    return torch.randn(shape, device=DEV, dtype=torch.float16, generator=g).mul_(32).round_().clamp_(-128, 127).to(torch.int8)


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(int(seed))
    host = random.Random(int(seed))
    h, dim, hq = case["kv_heads"], case["dim"], case["heads"]
    s = {"case": case}
    if case["op"] in ("write", "states"):
        dt = TYPES[case["dtype"]]
        t = case["tokens"] if case["op"] == "write" else case["batch"] * case["length"]
        qkv = torch.randn((t, (hq + 2 * h) * dim), device=DEV, generator=g).to(dt)           # as one projection leaves it
        s["q"] = qkv[:, :hq * dim].view(t, hq, dim) if hq else None
        s["k"] = qkv[:, hq * dim:(hq + h) * dim].view(t, h, dim)
        s["v"] = qkv[:, (hq + h) * dim:].view(t, h, dim)
        s["freq"], s["axis"] = axes_of(case)
        axes = len(case["pairs"].split(",")) if case["pairs"] else 0
        far = host.randint(0, case["far"]) if case["op"] == "write" else 0
        s["positions"] = _positions(t, axes, far) if axes else None
        s["scale"] = 1.0
        if case["op"] == "write":
            page = case["page"]
            pages = -(-t // page) + 1
            order = torch.randperm(pages, device=DEV, generator=g)
            at = torch.arange(t, device=DEV)
            slots = order[at // page] * page + at % page
            if case["skip"]:
                slots = torch.where(torch.rand(t, device=DEV, generator=g) < 0.25, torch.full_like(slots, -1), slots)
            s["slots"] = slots
            # one page more than the cache has: where the plain form puts what is skipped
            s["k_pool"], s["v_pool"] = _codes((pages + 1, h, page, dim), g), _codes((pages + 1, h, page, dim), g)
            s["q8"] = torch.empty((t, hq, dim), dtype=torch.int8, device=DEV)
        else:
            b, n = case["batch"], case["length"]
            shape = (lambda heads: (b, heads, n, dim)) if case["heads_first"] else (lambda heads: (t, heads, dim))
            s["q8"] = torch.empty(shape(hq), dtype=torch.int8, device=DEV) if hq else None
            s["k8"], s["v8"] = (torch.empty(shape(h), dtype=torch.int8, device=DEV) for _ in range(2))
        s["steps"] = [[round(host.uniform(0.02, 0.04), 5) for _ in range(n)] for n in (hq, h, h)]
        if own:
            import paper_2604_02292_b200 as pkg
            s["ctx"] = pkg.Context(0)
            s["steps"] = [np.array(v, dtype=np.float32) for v in s["steps"]]
            s["rope"] = pkg.RopeAxes(s["freq"], s["axis"], interleaved=case["layout"] == "interleaved", scale=s["scale"]) if axes else None
        else:
            s["dev_steps"] = [torch.tensor(v, device=DEV, dtype=torch.float32) for v in s["steps"]]
            s["dev_freq"] = torch.tensor(s["freq"], device=DEV, dtype=torch.float64)
            s["dev_axis"] = torch.tensor(s["axis"], device=DEV, dtype=torch.int64)
        return s
    qn, kn = _lengths(case)
    share = case["share"]
    start = torch.tensor([0] + qn).cumsum(0)
    total = int(start[-1])
    # the states of the inputs one behind the other, those of a shared input once
    at, firsts = 0, []
    for i, n in enumerate(kn):
        if i % share == 0:
            here, at = at, at + n
        firsts.append(here)
    s["q"] = _codes((total, hq, dim), g)
    if case["fused"]:
        kv = _codes((at, 2 * h, dim), g)
        s["k"], s["v"] = kv[:, :h], kv[:, h:]
    else:
        s["k"], s["v"] = _codes((at, h, dim), g), _codes((at, h, dim), g)
    s["start"] = start.to(torch.int32).to(DEV)
    s["k_start"], s["k_len"] = torch.tensor(firsts, dtype=torch.int32, device=DEV), torch.tensor(kn, dtype=torch.int32, device=DEV)
    s["host_start"] = firsts
    s["ranges"] = torch.tensor(_ranges(case), dtype=torch.int32, device=DEV).reshape(total, 2) if case["ranges"] else None
    s["out"] = torch.empty((total, hq, dim), dtype=TYPES[case["dtype"]], device=DEV)
    # logits with a spread of 10 to 30 units, a table inside the band of its kind
    spread = 32.0 * 32.0 * math.sqrt(dim)
    s["mult"] = [int(host.uniform(10, 30) / spread * (1 << SHIFT)) for _ in range(hq)]
    s["scale"] = [round(host.uniform(0.02, 0.04), 5) for _ in range(hq)]
    theta = []
    for _ in range(hq):
        if case["wide"]:
            d, sl = host.randint(60, 127), host.randint(1, 127)
            theta.append((d * sl + host.randint(0, 3 * sl), sl, d))
        else:
            n = max(case["length"], 1)
            floor, top = -(-256 // n), 32767 // n
            d = host.randint(max(1, min(4, top - floor)), max(1, min(127, top - floor)))
            sl = host.randint(min(1, (top - floor) // d), min(127, (top - floor) // d))
            theta.append((host.randint(sl * d + floor, top), sl, d))
    s["theta"] = theta
    if own:
        import paper_2604_02292_b200 as pkg
        s["ctx"] = pkg.Context(0)
        if case["wide"]:
            s["ctx"].hccs_params_upload_wide(np.array(theta, dtype=np.int32), case["length"])
        else:
            s["ctx"].hccs_params_upload(np.array(theta, dtype=np.int32), case["length"])
        s["mult"], s["scale"] = np.array(s["mult"], dtype=np.int32), np.array(s["scale"], dtype=np.float32)
        s["flags"] = {"div": pkg.HCCS_RECIP_DIV, "clb": pkg.HCCS_RECIP_CLB, "real": pkg.HCCS_RECIP_REAL}[case["norm"]]
    else:
        s["dev_mult"] = torch.tensor(s["mult"], device=DEV)
        s["dev_scale"] = torch.tensor(s["scale"], device=DEV, dtype=torch.float32)
        s["dev_theta"] = torch.tensor(theta, device=DEV)
    return s


# ------------------------------------------------------------------------------------------------ the operators
def run(s):
    op = s["case"]["op"]
    if own:
        return {"write": _own_write, "states": _own_states, "cross": _own_cross}[op](s)
    return {"write": _plain_write, "states": _plain_states, "cross": _plain_cross}[op](s)


def _own_write(s):
    k, v = s["k_pool"][:-1], s["v_pool"][:-1]
    s["ctx"].hccs_cache_write_axes(s["q"], s["k"], s["v"], s["q8"], k, v, s["positions"], s["slots"], *s["steps"], rope=s["rope"])
    return {"q": s["q8"], "k": k, "v": v}


def _own_states(s):
    s["ctx"].hccs_states_write(s["q"], s["k"], s["v"], s["q8"], s["k8"], s["v8"], s["positions"], *s["steps"], rope=s["rope"])
    out = {"k": s["k8"], "v": s["v8"]}
    if s["q"] is not None:
        out["q"] = s["q8"]
    return out


def _own_cross(s):
    c = s["case"]
    s["ctx"].hccs_attention_cross(s["q"], s["k"], s["v"], s["start"], s["k_start"], s["k_len"], s["out"], s["mult"], SHIFT,
                                  max_q=c["queries"], max_kv=c["length"], key_range=s["ranges"],
                                  out_scale=None if c["dtype"] == "i32" else s["scale"], flags=s["flags"])
    return s["out"]


def _quantised(y, step):
    """Codes of y [tokens, heads, dim] in double: values next to a border decide a whole step."""
    z = torch.round(y / step.double()[None, :, None]).clamp(-128, 127)
    return torch.nan_to_num(z, nan=0.0).to(torch.int8)


def _rotated(x, s):
    c = s["case"]
    x = x.double()
    if s["positions"] is None:
        return x
    rot = 2 * len(s["freq"])
    angle = s["positions"].double().t()[:, s["dev_axis"]] * s["dev_freq"][None, :]
    cos, sin = (torch.cos(angle) * s["scale"])[:, None, :], (torch.sin(angle) * s["scale"])[:, None, :]
    if c["layout"] == "half":
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        y = torch.cat([a * cos - b * sin, b * cos + a * sin], dim=-1)
    else:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        y = torch.stack([a * cos - b * sin, b * cos + a * sin], dim=-1).flatten(-2)
    return torch.cat([y, x[..., rot:]], dim=-1)


def _plain_write(s):
    page = s["case"]["page"]
    s["q8"].copy_(_quantised(_rotated(s["q"], s), s["dev_steps"][0]))
    last = (s["k_pool"].shape[0] - 1) * page
    slots = torch.where(s["slots"] < 0, torch.full_like(s["slots"], last), s["slots"])
    at, off = slots // page, slots % page
    s["k_pool"][at, :, off] = _quantised(_rotated(s["k"], s), s["dev_steps"][1])
    s["v_pool"][at, :, off] = _quantised(s["v"].double(), s["dev_steps"][2])
    return {"q": s["q8"], "k": s["k_pool"][:-1], "v": s["v_pool"][:-1]}


def _plain_states(s):
    c = s["case"]

    def put(out, codes):
        out.copy_(codes.unflatten(0, (c["batch"], c["length"])).transpose(1, 2) if c["heads_first"] else codes)
        return out

    out = {"k": put(s["k8"], _quantised(_rotated(s["k"], s), s["dev_steps"][1])), "v": put(s["v8"], _quantised(s["v"].double(), s["dev_steps"][2]))}
    if s["q"] is not None:
        out["q"] = put(s["q8"], _quantised(_rotated(s["q"], s), s["dev_steps"][0]))
    return out


def _plain_cross(s):
    c = s["case"]
    n_b, hq, h, dim, nq, n = c["batch"], c["heads"], c["kv_heads"], c["dim"], c["queries"], c["length"]
    g = hq // h
    start, k_len = s["start"].long(), s["k_len"].long()
    total, states = s["q"].shape[0], s["k"].shape[0]
    key = torch.arange(n, device=DEV)
    at = (s["k_start"].long()[:, None] + key[None, :]).clamp(max=states - 1)                            # [batch, key]
    rows = (start[:-1, None] + torch.arange(nq, device=DEV)[None, :]).clamp(max=total - 1)            # [batch, query]
    q = s["q"][rows].float().reshape(n_b, nq, h, g, dim).permute(0, 2, 1, 3, 4).reshape(n_b, h, nq * g, dim)
    acc = q @ s["k"][at].float().permute(0, 2, 3, 1)                                                    # whole numbers below 2^24
    valid = (key[None, :] < k_len[:, None])[:, None, :].expand(n_b, nq, n)                              # [batch, query, key]
    if s["ranges"] is not None:
        first, end = s["ranges"].long()[rows].unbind(-1)
        valid = valid & (key >= first[:, :, None]) & (key < end[:, :, None])
    valid = valid[:, None, :, None, :].expand(n_b, h, nq, g, n).reshape(n_b, h, nq * g, n)

    def per_row(v):                                                                                     # [heads] -> [kv head, row, 1]
        return v.reshape(h, 1, g).expand(h, nq, g).reshape(h, nq * g, 1)

    x = ((acc.long() * per_row(s["dev_mult"]) + (1 << (SHIFT - 1))) >> SHIFT).clamp(-128, 127).to(torch.int32)
    del acc
    big, slope, reach = (per_row(s["dev_theta"][:, i].to(torch.int32)) for i in range(3))
    m = torch.where(valid, x, -1000).amax(-1, keepdim=True)
    score = (big - slope * torch.minimum(m - x, reach)) * valid
    del x, valid
    z = score.sum(-1, keepdim=True)                                                                     # int64
    v = s["v"][at].float().permute(0, 2, 1, 3)
    if c["norm"] == "real":
        o = (score.float() / z.clamp(min=1).float()) @ v
        o = o * per_row(s["dev_scale"])
    else:
        if c["norm"] == "div":
            rho = 32767 // z.clamp(min=1)
        else:
            rho = 32767 >> (torch.frexp(z.clamp(min=1).float())[1].long() - 1)
        o = (score * rho).float() @ v                                                                   # whole numbers below 2^24
        if c["dtype"] != "i32":
            o = o * per_row(s["dev_scale"])
    o = o.to(TYPES[c["dtype"]]).reshape(n_b, h, nq, g, dim).permute(0, 2, 1, 3, 4).reshape(n_b, nq, hq, dim)
    t = torch.arange(total, device=DEV)
    b = torch.bucketize(t, start[1:], right=True)
    return o[b, t - start[b]]


# ------------------------------------------------------------------------------------------------ the definition, in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] in ("write", "states"):
        got = {}
        half = len(s["freq"])
        for name, step in (("q", s["steps"][0]), ("k", s["steps"][1]), ("v", s["steps"][2])):
            if s[name] is None:
                continue
            x = s[name].double().clone()
            if name != "v" and s["positions"] is not None:
                for i, (f, a) in enumerate(zip(s["freq"], s["axis"])):         # a rotation is a product of complex numbers
                    pos = s["positions"][a].double()
                    u, w = (i, i + half) if case["layout"] == "half" else (2 * i, 2 * i + 1)
                    turn = torch.polar(torch.full_like(pos, s["scale"]), pos * f)[:, None]
                    z = torch.complex(x[..., u], x[..., w]) * turn
                    x[..., u], x[..., w] = z.real, z.imag
            for i, w in enumerate(step):
                x[:, i] /= float(torch.tensor(float(w), dtype=torch.float32))
            got[name] = x.round().clamp(-128, 127)
        if case["op"] == "states":
            if case["heads_first"]:
                got = {k: v.reshape(case["batch"], case["length"], -1, case["dim"]).transpose(1, 2) for k, v in got.items()}
            return got
        out = {"q": got["q"]}
        keep = (s["slots"] >= 0).nonzero()[:, 0]
        at, off = s["slots"][keep] // case["page"], s["slots"][keep] % case["page"]
        for name in ("k", "v"):
            pool = s[name + "_pool"][:-1].double()
            pool[at, :, off] = got[name][keep]
            out[name] = pool
        return out
    qn, kn = _lengths(case)
    g, at = case["heads"] // case["kv_heads"], 0
    out = torch.zeros(s["out"].shape, dtype=torch.float64, device=DEV)
    for nq, n, k0 in zip(qn, kn, s["host_start"]):
        seen = torch.ones((nq, n), dtype=torch.bool, device=DEV)
        if s["ranges"] is not None:
            index = torch.arange(n, device=DEV)
            mine = s["ranges"][at:at + nq]
            seen = (index[None, :] >= mine[:, :1]) & (index[None, :] < mine[:, 1:])
        for kh in range(case["kv_heads"]):
            k, v = (t[k0:k0 + n, kh].double() for t in (s["k"], s["v"]))
            for hh in range(kh * g, kh * g + g):
                big, slope, reach = s["theta"][hh]
                x = s["q"][at:at + nq, hh].double() @ k.T
                x = torch.floor(x * (int(s["mult"][hh]) / 2.0 ** SHIFT) + 0.5).clamp(-128, 127)
                top = x.masked_fill(~seen, -math.inf).max(dim=1, keepdim=True).values
                w = (big - slope * (top - x).clamp(max=reach)).masked_fill(~seen, 0.0)
                z = w.sum(dim=1, keepdim=True).clamp(min=1.0)                  # rows that see nothing have no weights at all
                if case["norm"] == "real":
                    w = w / z
                elif case["norm"] == "div":
                    w = w * torch.floor(32767.0 / z)
                else:
                    w = w * torch.floor(32767.0 / torch.exp2(torch.frexp(z)[1].double() - 1.0))       # (log2 of 2^k may fall short of k)
                o = w @ v
                if case["dtype"] != "i32":
                    o = o * float(torch.tensor(float(s["scale"][hh]), dtype=torch.float32))
                out[at:at + nq, hh] = o
        at += nq
    return out
