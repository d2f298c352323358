"""The operators of generation over an int8 key/value cache, as a program uses them: tokens rotated, quantised and
written into a paged cache (``hccs_cache_write``), sequences read back from it (``hccs_cache_read``), and HCCS
attention of new tokens over it (``hccs_attention_cached``).

``run`` computes them in their plain form with elementary torch operations, or, where ``own`` is true, by the
calls of this framework.  Codes (int8) are whole numbers here, in the caches and in the quantised queries: they are
what the integer attention consumes, so they are returned and compared as such.
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
def _write(name, tokens, heads, kv_heads, dim, page, dtype, layout, rot, far, skip):
    return {"name": name, "op": "write", "tokens": tokens, "heads": heads, "kv_heads": kv_heads, "dim": dim, "page": page,
            "dtype": dtype, "layout": layout, "rot": rot, "far": far, "skip": skip}


def _read(name, batch, length, kv_heads, dim, page, dtype):
    return {"name": name, "op": "read", "batch": batch, "length": length, "kv_heads": kv_heads, "dim": dim, "page": page, "dtype": dtype}


def _attend(name, batch, queries, length, heads, kv_heads, dim, page, mask, norm, dtype, ragged, wide):
    return {"name": name, "op": "attend", "batch": batch, "queries": queries, "length": length, "heads": heads, "kv_heads": kv_heads,
            "dim": dim, "page": page, "mask": mask, "norm": norm, "dtype": dtype, "ragged": ragged, "wide": wide}


def listed():
    return [
        # one generation step of four sequences: latency counts
        _write("write step", 4, 32, 8, 128, 64, "bf16", "half", 128, 4000, False),
        # a batch of prompts, positions of a long context
        _write("write prompts", 16384, 32, 8, 128, 64, "bf16", "half", 128, 120000, False),
        # a padded batch of an encoder-sized model: part of the head rotated, padding tokens skipped
        _write("write padded", 1003, 12, 12, 64, 16, "f16", "interleaved", 32, 900, True),
        # short sequences handed to another program in their values
        _read("read short", 7, 1021, 12, 64, 16, "f32"),
        # long sequences read back for a layer that works on values
        _read("read long", 8, 8192, 8, 128, 64, "bf16"),
        # one token of one short sequence, integer output of the paper's int16 path
        _attend("decode one", 1, 1, 513, 12, 12, 64, 16, "causal", "div", "i32", False, False),
        # a serving batch of ragged sequences
        _attend("decode batch", 32, 1, 4096, 32, 8, 128, 64, "causal", "real", "bf16", True, False),
        # one token over a very long context: the keys have to be shared out
        _attend("decode long", 1, 1, 131072, 32, 8, 128, 64, "causal", "real", "bf16", False, True),
        # the largest serving batch
        _attend("decode full", 64, 1, 8192, 64, 8, 128, 64, "causal", "real", "bf16", False, True),
        # a small tree of drafted tokens, leading-bit reciprocal, integer output
        _attend("tree small", 3, 13, 700, 12, 12, 64, 16, "tree", "clb", "i32", True, False),
        # trees of drafted tokens of a serving batch
        _attend("tree batch", 8, 48, 8000, 32, 8, 128, 64, "tree", "real", "bf16", True, True),
        # a chunk of two long prompts
        _attend("prompt chunk", 2, 2048, 8192, 16, 4, 128, 64, "causal", "real", "bf16", False, True),
    ]


def _spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["write", "read", "decode", "decode", "tree", "chunk"])
    dim = rng.choice([64, 128])
    page = rng.choice([16, 32, 64, 128, 256])
    kv_heads = rng.choice([1, 2, 3, 4, 5, 8, 12])
    group = rng.choice([1, 1, 2, 3, 4, 7, 8])
    heads = kv_heads * group
    if op == "write":
        tokens = _spread(rng, 1, max(16, 16384 * 48 * 128 // ((heads + 2 * kv_heads) * dim) // 2))
        return {k: v for k, v in _write("", tokens, heads, kv_heads, dim, page, rng.choice(["bf16", "f16", "f32"]),
                                        rng.choice(["half", "interleaved"]), rng.choice([0, dim // 4, dim // 2, dim]),
                                        _spread(rng, 1, 120000), rng.random() < 0.3).items() if k != "name"}
    if op == "read":
        batch = rng.randint(1, 16)
        length = _spread(rng, 1, max(16, 8 * 8192 * 8 * 128 // (batch * kv_heads * dim) // 2))
        return {k: v for k, v in _read("", batch, min(length, 131072), kv_heads, dim, page, rng.choice(["bf16", "f16", "f32"])).items() if k != "name"}
    batch = _spread(rng, 1, 64) if op == "decode" else rng.randint(1, 8)
    most = 64 * 8192 * 8 * 128 // (batch * kv_heads * dim)
    if op == "decode":
        queries = 1
    elif op == "tree":
        queries = rng.randint(2, 70)
    else:
        queries = _spread(rng, 64, 1500)
    # the cost of a chunk grows with its rows: no more than the largest listed one
    if op != "decode":
        most = min(most, 2 * 2048 * 8192 * 16 // (batch * queries * heads))
    length = queries + _spread(rng, 1, max(2, min(131072 - queries, most // 2)))
    wide = length > 4000 or rng.random() < 0.3
    norm = "real" if wide else rng.choice(["real", "div", "clb"])
    dtype = rng.choice(["bf16", "f16", "f32"]) if norm == "real" or rng.random() < 0.3 else "i32"
    return {k: v for k, v in _attend("", batch, queries, length, heads, kv_heads, dim, page, "tree" if op == "tree" else "causal", norm, dtype,
                                     rng.random() < 0.6, wide).items() if k != "name"}


def _lengths(case):
    """(query lengths, key lengths) of the sequences: properties of the case, not of its seed."""
    r = random.Random(case["length"] * 131 + case["batch"])
    kv = [case["length"]] + [r.randint(max(1, case["length"] // 3), case["length"]) for _ in range(case["batch"] - 1)]
    if case["op"] == "read":
        return [0] * case["batch"], kv
    if not case["ragged"]:
        return [case["queries"]] * case["batch"], [case["length"]] * case["batch"]
    q = [case["queries"]] + [r.randint(1, case["queries"]) for _ in range(case["batch"] - 1)]
    return q, [max(a, b) for a, b in zip(q, kv)]


def work(case):
    size = {"bf16": 2, "f16": 2, "f32": 4, "i32": 4}[case["dtype"]]
    if case["op"] == "write":
        n = case["tokens"] * (case["heads"] + 2 * case["kv_heads"]) * case["dim"]
        return {"bytes": n * (size + 1) + 12 * case["tokens"], "flops": 4 * n}
    q, kv = _lengths(case)
    if case["op"] == "read":
        n = 2 * sum(kv) * case["kv_heads"] * case["dim"]
        return {"bytes": n * (size + 1), "flops": n}
    pairs = sum(a * (b - a) + a * (a + 1) / 2 for a, b in zip(q, kv)) * case["heads"]
    row = case["heads"] * case["dim"]
    return {"bytes": 2 * sum(kv) * case["kv_heads"] * case["dim"] + sum(q) * row * (1 + size), "flops": 4 * case["dim"] * pairs}


# ------------------------------------------------------------------------------------------------ inputs
def frequencies(rot, far):
    """Rotary frequencies in radians per position; a long context divides the slow ones by eight, by wavelength."""
    got = []
    for i in range(rot // 2):
        f = 10000.0 ** (-2.0 * i / rot)
        if far > 8192:
            turns = 8192 * f / (2 * math.pi)
            keep = min(1.0, max(0.0, (turns - 1.0) / 3.0))
            f = f * keep + f / 8.0 * (1.0 - keep)
        got.append(f)
    return got


def _codes(shape, g):
    """int8 codes as a cache holds them: a bell of width 32."""
    return torch.randn(shape, device=DEV, dtype=torch.float16, generator=g).mul_(32).round_().clamp_(-128, 127).to(torch.int8)


def _table(case, g, kv):
    """Pages of every sequence, shuffled over the pool."""
    per = -(-max(kv) // case["page"])
    pages = case["batch"] * per
    return torch.randperm(pages, device=DEV, generator=g).to(torch.int32).reshape(case["batch"], per), pages


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(int(seed))
    host = random.Random(int(seed))
    h, dim, page = case["kv_heads"], case["dim"], case["page"]
    s = {"case": case}
    if case["op"] == "write":
        t, hq, dt = case["tokens"], case["heads"], TYPES[case["dtype"]]
        qkv = torch.randn((t, (hq + 2 * h) * dim), device=DEV, generator=g).to(dt)           # as one projection leaves it
        s["q"] = qkv[:, :hq * dim].view(t, hq, dim)
        s["k"] = qkv[:, hq * dim:(hq + h) * dim].view(t, h, dim)
        s["v"] = qkv[:, (hq + h) * dim:].view(t, h, dim)
        s["positions"] = (torch.arange(t, device=DEV) + host.randint(0, case["far"])).to(torch.int32)
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
        s["steps"] = [[round(host.uniform(0.02, 0.04), 5) for _ in range(n)] for n in (hq, h, h)]
        s["freq"] = frequencies(case["rot"], case["far"])
        s["scale"] = 1.0 if case["far"] <= 8192 else 1.1
        if own:
            import paper_2604_02292_b200 as pkg
            s["ctx"] = pkg.Context(0)
            s["steps"] = [np.array(v, dtype=np.float32) for v in s["steps"]]
            s["rope"] = pkg.Rope(s["freq"], interleaved=case["layout"] == "interleaved", scale=s["scale"]) if case["rot"] else None
        else:
            s["dev_steps"] = [torch.tensor(v, device=DEV, dtype=torch.float32) for v in s["steps"]]
            s["dev_freq"] = torch.tensor(s["freq"], device=DEV, dtype=torch.float64)
        return s
    qn, kv = _lengths(case)
    s["table"], pages = _table(case, g, kv)
    s["k_pool"], s["v_pool"] = _codes((pages, h, page, dim), g), _codes((pages, h, page, dim), g)
    if case["op"] == "read":
        s["lens"] = kv
        s["steps"] = [[round(host.uniform(0.02, 0.04), 5) for _ in range(h)] for _ in range(2)]
        start = torch.tensor([0] + kv).cumsum(0)
        s["start"] = start.to(torch.int32).to(DEV)
        total = int(start[-1])
        s["k_out"], s["v_out"] = (torch.empty((total, h, dim), dtype=TYPES[case["dtype"]], device=DEV) for _ in range(2))
        if own:
            import paper_2604_02292_b200 as pkg
            s["ctx"] = pkg.Context(0)
            s["steps"] = [np.array(v, dtype=np.float32) for v in s["steps"]]
        else:
            s["dev_steps"] = [torch.tensor(v, device=DEV, dtype=torch.float32) for v in s["steps"]]
        return s
    hq = case["heads"]
    start = torch.tensor([0] + qn).cumsum(0)
    total = int(start[-1])
    s["q"] = _codes((total, hq, dim), g)
    s["start"], s["kv"] = start.to(torch.int32).to(DEV), torch.tensor(kv, dtype=torch.int32, device=DEV)
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
    s["tree"] = _tree(qn, case, g, host) if case["mask"] == "tree" else None
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


def _tree(qn, case, g, host):
    """Ancestor masks: bit j of a node's words says whether it sees node j of its sequence (itself and its ancestors)."""
    words = -(-case["queries"] // 32)
    rows = []
    for n in qn:
        seen = []
        for i in range(n):
            parent = host.randint(max(0, i - 6), i - 1) if i else -1
            seen.append((seen[parent] if parent >= 0 else 0) | (1 << i))
        rows += [[(b >> (32 * w)) & 0xFFFFFFFF for w in range(words)] for b in seen]
    t = torch.tensor(rows, dtype=torch.int64)
    return torch.where(t >= 1 << 31, t - (1 << 32), t).to(torch.int32).to(DEV)


# ------------------------------------------------------------------------------------------------ the operators
def run(s):
    op = s["case"]["op"]
    if own:
        return {"write": _own_write, "read": _own_read, "attend": _own_attend}[op](s)
    return {"write": _plain_write, "read": _plain_read, "attend": _plain_attend}[op](s)


def _own_write(s):
    k, v = s["k_pool"][:-1], s["v_pool"][:-1]
    s["ctx"].hccs_cache_write(s["q"], s["k"], s["v"], s["q8"], k, v, s["positions"], s["slots"], *s["steps"], rope=s["rope"])
    return {"q": s["q8"], "k": k, "v": v}


def _own_read(s):
    s["ctx"].hccs_cache_read(s["k_pool"], s["v_pool"], s["table"], s["start"], s["k_out"], s["v_out"], *s["steps"], max(s["lens"]))
    return {"k": s["k_out"], "v": s["v_out"]}


def _own_attend(s):
    c = s["case"]
    s["ctx"].hccs_attention_cached(s["q"], s["k_pool"], s["v_pool"], s["table"], s["start"], s["kv"], s["out"], s["mult"], SHIFT,
                                   max_q=c["queries"], max_kv=c["length"], tree_mask=s["tree"],
                                   out_scale=None if c["dtype"] == "i32" else s["scale"], flags=s["flags"])
    return s["out"]


def _quantised(y, step):
    """Codes of y [tokens, heads, dim] in double: values next to a border decide a whole step."""
    z = torch.round(y / step.double()[None, :, None]).clamp(-128, 127)
    return torch.nan_to_num(z, nan=0.0).to(torch.int8)


def _rotated(x, angle, s):
    c = s["case"]
    x = x.double()
    rot = c["rot"]
    if not rot:
        return x
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
    angle = s["positions"].double()[:, None] * s["dev_freq"][None, :]
    s["q8"].copy_(_quantised(_rotated(s["q"], angle, s), s["dev_steps"][0]))
    last = (s["k_pool"].shape[0] - 1) * page
    slots = torch.where(s["slots"] < 0, torch.full_like(s["slots"], last), s["slots"])
    at, off = slots // page, slots % page
    s["k_pool"][at, :, off] = _quantised(_rotated(s["k"], angle, s), s["dev_steps"][1])
    s["v_pool"][at, :, off] = _quantised(s["v"].double(), s["dev_steps"][2])
    return {"q": s["q8"], "k": s["k_pool"][:-1], "v": s["v_pool"][:-1]}


def _plain_read(s):
    page, dt = s["case"]["page"], TYPES[s["case"]["dtype"]]
    total = s["k_out"].shape[0]
    t = torch.arange(total, device=DEV)
    b = torch.bucketize(t, s["start"][1:].long(), right=True)
    i = t - s["start"].long()[b]
    at, off = s["table"].long()[b, i // page], i % page
    got = []
    for pool, step in zip((s["k_pool"], s["v_pool"]), s["dev_steps"]):
        got.append((pool[at, :, off].float() * step[None, :, None]).to(dt))
    return {"k": got[0], "v": got[1]}


def _plain_attend(s):
    c = s["case"]
    n_b, hq, h, dim, page, nq = c["batch"], c["heads"], c["kv_heads"], c["dim"], c["page"], c["queries"]
    g = hq // h
    start, kv = s["start"].long(), s["kv"].long()
    qn = start[1:] - start[:-1]
    n = s["table"].shape[1] * page
    total = s["q"].shape[0]

    def dense(pool):
        return pool[s["table"].long()].permute(0, 2, 1, 3, 4).reshape(n_b, h, n, dim).float()

    rows = (start[:-1, None] + torch.arange(nq, device=DEV)[None, :]).clamp(max=total - 1)            # [batch, query]
    q = s["q"][rows].float().reshape(n_b, nq, h, g, dim).permute(0, 2, 1, 3, 4).reshape(n_b, h, nq * g, dim)
    acc = q @ dense(s["k_pool"]).transpose(-1, -2)                                                      # whole numbers below 2^24
    key = torch.arange(n, device=DEV)
    new = key[None, :] - (kv - qn)[:, None]                                                             # [batch, key]: index among the new tokens
    if s["tree"] is None:
        valid = new[:, None, :] <= torch.arange(nq, device=DEV)[None, :, None]
    else:
        words = s["tree"][rows].long()                                                                  # [batch, query, word]
        at = new.clamp(0, 32 * words.shape[2] - 1)
        word = torch.gather(words, 2, (at // 32)[:, None, :].expand(-1, nq, -1))
        valid = (new < 0)[:, None, :] | ((word >> (at % 32)[:, None, :]) & 1).bool()
    valid = valid & (key[None, :] < kv[:, None])[:, None, :]                                            # [batch, query, key]
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
    v = dense(s["v_pool"])
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
    if case["op"] == "write":
        got = {}
        pos = s["positions"].double()
        for name, step in (("q", s["steps"][0]), ("k", s["steps"][1]), ("v", s["steps"][2])):
            x = s[name].double().clone()
            if name != "v":
                for i, f in enumerate(s["freq"]):                              # a rotation is a product of complex numbers
                    a, b = (i, i + case["rot"] // 2) if case["layout"] == "half" else (2 * i, 2 * i + 1)
                    turn = torch.polar(torch.full_like(pos, s["scale"]), pos * f)[:, None]
                    z = torch.complex(x[..., a], x[..., b]) * turn
                    x[..., a], x[..., b] = z.real, z.imag
            for i, w in enumerate(step):
                x[:, i] /= float(torch.tensor(w, dtype=torch.float32))
            got[name] = x.round().clamp(-128, 127)
        out = {"q": got["q"]}
        keep = (s["slots"] >= 0).nonzero()[:, 0]
        at, off = s["slots"][keep] // case["page"], s["slots"][keep] % case["page"]
        for name in ("k", "v"):
            pool = s[name + "_pool"][:-1].double()
            pool[at, :, off] = got[name][keep]
            out[name] = pool
        return out
    if case["op"] == "read":
        out = {}
        for name, pool, step in (("k", s["k_pool"], s["steps"][0]), ("v", s["v_pool"], s["steps"][1])):
            step = torch.tensor(step, dtype=torch.float32).double().to(DEV)
            seqs = []
            for b, n in enumerate(s["lens"]):
                seq = torch.cat([pool[p].transpose(0, 1) for p in s["table"][b].tolist()])[:n]
                seqs.append(seq.double() * step[None, :, None])
            out[name] = torch.cat(seqs)
        return out
    qn, kv = _lengths(case)
    g, at = case["heads"] // case["kv_heads"], 0
    out = torch.zeros(s["out"].shape, dtype=torch.float64, device=DEV)
    for b, (nq, n) in enumerate(zip(qn, kv)):
        pages = s["table"][b, :-(-n // case["page"])].long()
        seen = torch.ones((nq, n), dtype=torch.bool, device=DEV)
        if s["tree"] is None:
            seen[:, n - nq:] = torch.tril(seen[:, n - nq:])
        else:
            bits = (s["tree"][at:at + nq, :, None] >> torch.arange(32, device=DEV)[None, None, :]) & 1
            seen[:, n - nq:] = bits.flatten(1)[:, :nq].bool()
        for kh in range(case["kv_heads"]):
            k, v = (p[pages, kh].reshape(-1, case["dim"])[:n].double() for p in (s["k_pool"], s["v_pool"]))
            for hh in range(kh * g, kh * g + g):
                big, slope, reach = s["theta"][hh]
                x = s["q"][at:at + nq, hh].double() @ k.T
                x = torch.floor(x * (s["mult"][hh] / 2.0 ** SHIFT) + 0.5).clamp(-128, 127)
                top = x.masked_fill(~seen, -math.inf).max(dim=1, keepdim=True).values
                w = (big - slope * (top - x).clamp(max=reach)).masked_fill(~seen, 0.0)
                z = w.sum(dim=1, keepdim=True)
                if case["norm"] == "real":
                    w = w / z
                elif case["norm"] == "div":
                    w = w * torch.floor(32767.0 / z)
                else:
                    w = w * torch.floor(32767.0 / 2.0 ** torch.floor(torch.log2(z)))
                o = w @ v
                if case["dtype"] != "i32":
                    o = o * float(torch.tensor(s["scale"][hh], dtype=torch.float32))
                out[at:at + nq, hh] = o
        at += nq
    return out
