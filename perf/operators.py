"""Performance cases of the operators between a decoder layer's q/k/v launch and
its o launch: rotary positions, the paged key/value cache as it is written and
read back, and the attention of new tokens over it.

Each case is one call (or the two of a round trip) of the public Python API
(`rope`, `KVCache.write`, `KVCache.read`, `KVCache.attend`); with `own` false
the same mathematics runs in elementary torch operations.

  rope    x [T, heads, dim] turned by its tokens' positions
  write   the k and v (and q) columns of a fused q/k/v product: k and q are
          turned, k and v go to their slots of the cache; an 8-bit cache is
          read back, so that what it holds comes out as values
  read    cached tokens read back at the model's type
  attend  new tokens of every sequence over its pages

The cache is two tensors: keys [pages, kv_heads, page, dim] and values
[pages, kv_heads, page / I, dim, I] with I = 16 / bytes of an element (sixteen
bytes hold I consecutive tokens' values of one coordinate).  An 8-bit cache has
an f32 scale per token and head of each.  A slot is page · page_size + offset.
"""
from __future__ import annotations

import math

import torch

own = False
DEV = "cuda:0"
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16,
         "int8": torch.int8, "e4m3": torch.float8_e4m3fn}
SIZE = {"f32": 4, "f16": 2, "bf16": 2, "int8": 1, "e4m3": 1}
LARGEST = {"int8": 127.0, "e4m3": 448.0}


# ------------------------------------------------------------------- the cases
def listed():
    return [
        # one token's queries of a 14B-class layer (40 heads): a launch's latency
        {"name": "rope-1x40", "op": "rope", "T": 1, "heads": 40, "dim": 128, "rot": 128,
         "interleaved": False, "src": "f32", "dst": "f16", "first": 8191, "stretch": 1.0},
        # a prompt of an 8B-class layer, half of each head turned, in pairs of
        # neighbours, at positions near a million, stretched eightfold
        {"name": "rope-4096x32-far", "op": "rope", "T": 4096, "heads": 32, "dim": 128, "rot": 64,
         "interleaved": True, "src": "bf16", "dst": "bf16", "first": 999_000, "stretch": 8.0},
        # 64 concurrent sequences' next tokens, from the fused product's rows
        {"name": "write-64-e4m3", "op": "write", "T": 64, "q_heads": 40, "heads": 8, "dim": 128,
         "rot": 128, "interleaved": False, "cache": "e4m3", "dst": "f16", "page": 64,
         "scattered": True},
        # a prompt's chunk from the fused product of an 8B-class layer
        {"name": "write-4096-bf16", "op": "write", "T": 4096, "q_heads": 32, "heads": 8,
         "dim": 128, "rot": 128, "interleaved": False, "cache": "bf16", "dst": "bf16",
         "page": 128, "scattered": False},
        # a cached prefix read back (to move it, or to check it)
        {"name": "read-30000-int8", "op": "read", "T": 30_000, "heads": 8, "dim": 128,
         "cache": "int8", "dst": "bf16", "page": 64},
        # one sequence's next token after a short context: latency
        {"name": "attend-1x700", "op": "attend", "B": 1, "new": 1, "len": 700, "ragged": False,
         "q_heads": 40, "heads": 8, "dim": 128, "cache": "f16", "dst": "f16", "page": 64,
         "window": 0, "lse": False},
        # a serving batch's next tokens, contexts from a few tokens to 8000
        {"name": "attend-64x8000", "op": "attend", "B": 64, "new": 1, "len": 8000, "ragged": True,
         "q_heads": 32, "heads": 8, "dim": 128, "cache": "bf16", "dst": "bf16", "page": 128,
         "window": 0, "lse": False},
        # one long context: the work splits along it
        {"name": "attend-1x131071-e4m3", "op": "attend", "B": 1, "new": 1, "len": 131_071,
         "ragged": False, "q_heads": 32, "heads": 8, "dim": 128, "cache": "e4m3", "dst": "f16",
         "page": 256, "window": 0, "lse": True},
        # speculative tokens of sixteen sequences, 64-wide heads, a window
        {"name": "attend-16x5-window", "op": "attend", "B": 16, "new": 5, "len": 6000,
         "ragged": True, "q_heads": 24, "heads": 4, "dim": 64, "cache": "int8", "dst": "bf16",
         "page": 16, "window": 4000, "lse": False},
        # chunks of four prompts behind what is cached of them
        {"name": "attend-4x999-int8", "op": "attend", "B": 4, "new": 999, "len": 12_000,
         "ragged": True, "q_heads": 40, "heads": 8, "dim": 128, "cache": "int8", "dst": "f16",
         "page": 32, "window": 0, "lse": False},
        # a whole prompt through an 8B-class layer
        {"name": "attend-4096-prompt", "op": "attend", "B": 1, "new": 4096, "len": 4096,
         "ragged": False, "q_heads": 32, "heads": 8, "dim": 128, "cache": "f16", "dst": "f16",
         "page": 128, "window": 0, "lse": True},
        # wide heads without groups, two prompts of odd lengths
        {"name": "attend-2x2001-wide", "op": "attend", "B": 2, "new": 2001, "len": 2333,
         "ragged": True, "q_heads": 8, "heads": 8, "dim": 256, "cache": "bf16", "dst": "bf16",
         "page": 64, "window": 0, "lse": False},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["rope", "write", "write", "read"] + ["attend"] * 6)
    dim = rng.choice([64, 80, 96, 128, 128, 128, 192, 256])
    cache = rng.choice(["f16", "bf16", "int8", "e4m3"])
    dst = cache if cache in ("f16", "bf16") else rng.choice(["f16", "bf16"])
    page = rng.choice([16, 32, 64, 128, 256])
    if op == "rope":
        heads = rng.randint(1, 48)
        return {"op": op, "T": _log(rng, 1, 16e6 / (heads * dim)), "heads": heads, "dim": dim,
                "rot": 16 * rng.randint(1, dim // 16), "interleaved": rng.choice([True, False]),
                "src": rng.choice(["f32", "f16", "bf16"]), "dst": rng.choice(["f16", "bf16"]),
                "first": _log(rng, 1, 1e6), "stretch": rng.choice([1.0, 4.0])}
    heads = rng.choice([1, 2, 4, 8, 8])
    group = rng.choice([1, 2, 4, 4, 5, 6, 7, 8, 16])
    if op == "write":
        return {"op": op, "T": _log(rng, 1, 24e6 / (heads * (group + 2) * dim)),
                "q_heads": heads * group, "heads": heads, "dim": dim, "rot": dim,
                "interleaved": rng.choice([True, False]), "cache": cache, "dst": dst, "page": page,
                "scattered": rng.choice([True, False])}
    if op == "read":
        return {"op": op, "T": _log(rng, 1, 30e6 / (heads * dim)), "heads": heads, "dim": dim,
                "cache": cache, "dst": dst, "page": page}
    most = 68e9 / (4.0 * heads * group * dim)      # query-key pairs of a drawn case
    new = 1 if rng.random() < 0.5 else _log(rng, 1, 4096)
    length = max(new, _log(rng, 1, min(131_071, most / new)))
    b = _log(rng, 1, max(1.0, min(64.0, most / (new * length),
                                  2.9e8 / (length * heads * dim))))
    return {"op": op, "B": b, "new": new, "len": length, "ragged": rng.choice([True, False]),
            "q_heads": heads * group, "heads": heads, "dim": dim, "cache": cache, "dst": dst,
            "page": page, "window": rng.choice([0, 0, 0, max(1, length // 2)]),
            "lse": rng.choice([True, False])}


# ------------------------------------------------------------------ the inputs
def _lens(case):
    """(new tokens, cached tokens with them) of each sequence, before its order
    is drawn; a ragged batch's lie between a ninth and the whole of the largest."""
    b = case["B"]
    if not case["ragged"]:
        return [(case["new"], case["len"])] * b
    out = []
    for i in range(b):
        f = 1.0 if i == 0 else (i * 0.6180339887) % 1.0 * 8 / 9 + 1 / 9
        n = max(1, round(case["new"] * f))
        out.append((n, max(n, round(case["len"] * f))))
    return out


def _frequencies(rot, stretch):
    """Radians a position of each pair, in 64 bits, positions divided by `stretch`."""
    i = torch.arange(rot // 2, dtype=torch.float64)
    return (1e4 ** (-2.0 * i / rot) / stretch).to(DEV)


def _quantised(x, cache):
    """Codes and scales of x [..., dim] f32: scale = largest / 127 (448), code = x / scale."""
    scale = x.abs().amax(-1) / LARGEST[cache]
    y = torch.where(scale[..., None] > 0, x / scale[..., None], torch.zeros_like(x))
    y = y.round().clamp(-127, 127) if cache == "int8" else y
    return y.to(TYPES[cache]), scale


def _filled(gen, case, pages):
    """A cache of N(0, 1) tokens: keys, values and an 8-bit cache's scales."""
    cache, shape = case["cache"], (pages, case["heads"], case["page"], case["dim"])
    parts = []
    for kind in ("k", "v"):
        x = torch.randn(shape, generator=gen, device=DEV)
        x, scale = (x.to(TYPES[cache]), None) if SIZE[cache] == 2 else _quantised(x, cache)
        if kind == "v":
            i = 16 // SIZE[cache]
            x = x.reshape(pages, case["heads"], case["page"] // i, i, case["dim"])
            x = x.view(torch.uint8) if SIZE[cache] == 1 else x
            x = x.transpose(3, 4).contiguous().view(TYPES[cache])
        parts += [x.contiguous(), scale]
    return {"k": parts[0], "v": parts[2], "k_scale": parts[1], "v_scale": parts[3]}


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(int(seed))
    op, s = case["op"], {"case": case}

    def normal(*shape):
        return torch.randn(shape, generator=gen, device=DEV)

    def permutation(n):
        return torch.randperm(n, generator=gen, device=DEV)

    if op == "rope":
        s["x"] = normal(case["T"], case["heads"], case["dim"]).to(TYPES[case["src"]])
        s["positions"] = case["first"] + torch.arange(case["T"], device=DEV)
        s["freq"] = _frequencies(case["rot"], case["stretch"])
        return s
    page = case["page"]
    if op in ("write", "read"):
        T, start = case["T"], page // 2 + 1        # a chunk rarely starts with a page
        need = -(-(T + start) // page)
        pages = need + need // 4 + 1
        at = start + torch.arange(T, device=DEV)
        s["slots"] = permutation(pages)[at // page] * page + at % page
        if op == "read":
            s.update(_filled(gen, case, pages))
            return s
        if case["scattered"]:                      # tokens of as many sequences
            s["slots"] = s["slots"][permutation(T)]
        s["positions"] = (torch.randint(0, 100_000, (T,), generator=gen, device=DEV)
                          if case["scattered"] else at)
        hq, h, d = case["q_heads"], case["heads"], case["dim"]
        s["qkv"] = normal(T, (hq + 2 * h) * d)
        s["freq"] = _frequencies(case["rot"], 1.0)
        i = 16 // SIZE[case["cache"]]
        for part, shape in (("k", (pages, h, page, d)), ("v", (pages, h, page // i, d, i))):
            s[part] = torch.zeros(shape, dtype=torch.float32, device=DEV).to(TYPES[case["cache"]])
            s[part + "_scale"] = (torch.zeros(pages, h, page, device=DEV)
                                  if SIZE[case["cache"]] == 1 else None)
        return s
    order = permutation(case["B"]).tolist()
    lens = [_lens(case)[i] for i in order]
    starts = [0]
    for n, _ in lens:
        starts.append(starts[-1] + n)
    width = -(-case["len"] // page)                # pages a row of the table has room for
    used = [-(-length // page) for _, length in lens]
    s.update(_filled(gen, case, sum(used) + 1))
    which = permutation(sum(used) + 1)
    first = torch.tensor([0] + used, device=DEV).cumsum(0)
    column = torch.arange(width, device=DEV)
    inside = column < (first[1:] - first[:-1])[:, None]
    at = (first[:-1, None] + column).clamp(max=sum(used))
    s["table"] = torch.where(inside, which[at], 0).int()
    s["kv_len"] = torch.tensor([length for _, length in lens], dtype=torch.int32, device=DEV)
    s["q_start"] = torch.tensor(starts, dtype=torch.int32, device=DEV)
    s["max_new"] = max(n for n, _ in lens)
    s["q"] = (2 * normal(starts[-1], case["q_heads"], case["dim"])).to(TYPES[case["dst"]])
    return s


# ------------------------------------------------------------- the plain forms
def _turned(x, positions, freq, interleaved):
    """x [T, heads, dim] f32, its first 2·len(freq) coordinates turned in pairs."""
    rot = 2 * freq.numel()
    angle = positions.double()[:, None] * freq
    c, s = angle.cos().float()[:, None], angle.sin().float()[:, None]
    if interleaved:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        y = torch.stack([a * c - b * s, a * s + b * c], -1).flatten(-2)
    else:
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        y = torch.cat([a * c - b * s, a * s + b * c], -1)
    return torch.cat([y, x[..., rot:]], -1)


def _read_plain(s):
    """k and v of the slots as f32 [T, heads, dim]."""
    page = s["case"]["page"]
    p, o = s["slots"] // page, s["slots"] % page
    i = s["v"].shape[-1]
    bits = (lambda t: t.view(torch.uint8)) if i == 16 else (lambda t: t)
    k = bits(s["k"])[p, :, o].view(s["k"].dtype).float()
    v = bits(s["v"])[p, :, o // i, :, o % i].view(s["v"].dtype).float()
    if s["k_scale"] is None:
        return k, v
    return k * s["k_scale"][p, :, o][..., None], v * s["v_scale"][p, :, o][..., None]


def _write_plain(s):
    case, dst = s["case"], TYPES[s["case"]["dst"]]
    hq, h, d, page = case["q_heads"], case["heads"], case["dim"], case["page"]
    x = s["qkv"].reshape(case["T"], hq + 2 * h, d)
    turned = _turned(x[:, :hq + h], s["positions"], s["freq"], case["interleaved"])
    out = {"q": turned[:, :hq].to(dst)}
    p, o = s["slots"] // page, s["slots"] % page
    i = s["v"].shape[-1]
    for part, y in (("k", turned[:, hq:]), ("v", x[:, hq + h:])):
        to = s[part]
        if i == 16:
            y, scale = _quantised(y, case["cache"])
            s[part + "_scale"][p, :, o] = scale
            y, to = y.view(torch.uint8), to.view(torch.uint8)
        if part == "k":
            to[p, :, o] = y.to(to.dtype)
        else:
            to[p, :, o // i, :, o % i] = y.to(to.dtype)
    if i == 16:
        k, v = _read_plain(s)
        return {**out, "k": k.to(dst), "v": v.to(dst)}
    return {**out, "k": s["k"], "v": s["v"]}


def _attend_plain(s):
    case = s["case"]
    B, h, d, g = case["B"], case["heads"], case["dim"], case["q_heads"] // case["heads"]
    table, starts = s["table"].long(), s["q_start"].long()
    n, length, most = starts[1:] - starts[:-1], s["kv_len"].long(), s["max_new"]
    i = s["v"].shape[-1]
    bits = (lambda t: t.view(torch.uint8)) if i == 16 else (lambda t: t)
    k = bits(s["k"])[table].view(s["k"].dtype).float()             # [B, P, h, page, d]
    v = bits(s["v"])[table].view(s["v"].dtype).float()             # [B, P, h, page/I, d, I]
    k = k.permute(0, 2, 1, 3, 4).reshape(B, h, -1, d)
    v = v.permute(0, 2, 1, 3, 5, 4).reshape(B, h, -1, d)
    if s["k_scale"] is not None:
        k = k * s["k_scale"][table].permute(0, 2, 1, 3).reshape(B, h, -1, 1)
        v = v * s["v_scale"][table].permute(0, 2, 1, 3).reshape(B, h, -1, 1)
    row = torch.arange(most, device=DEV)
    at = (starts[:-1, None] + row).clamp(max=s["q"].shape[0] - 1)
    q = s["q"][at].float().reshape(B, most, h, g, d).permute(0, 2, 1, 3, 4).reshape(B, h, -1, d)
    score = torch.matmul(q, k.transpose(-1, -2).contiguous()) / math.sqrt(d)
    where = (length - n)[:, None] + row                            # [B, most]: a query's position
    key = torch.arange(k.shape[2], device=DEV)
    sees = (key <= where[..., None]) & (key < length[:, None, None])
    if case["window"]:
        sees &= key > where[..., None] - case["window"]
    sees = sees[:, None, :, None].expand(B, 1, most, g, -1).reshape(B, 1, most * g, -1)
    score.masked_fill_(~sees, -math.inf)
    top = score.amax(-1, keepdim=True)
    weight = torch.exp(score - torch.where(top > -math.inf, top, torch.zeros_like(top)))
    total = weight.sum(-1, keepdim=True)
    out = torch.matmul(weight, v) / total.clamp(min=1e-30)
    token = torch.arange(s["q"].shape[0], device=DEV)
    b = torch.searchsorted(starts[1:], token, right=True)
    out = out.reshape(B, h, most, g, d)[b, :, token - starts[b]].reshape(-1, h * g, d)
    got = {"out": out.to(s["q"].dtype)}
    if case["lse"]:
        lse = (top + total.log()).reshape(B, h, most, g)[b, :, token - starts[b]]
        got["lse"] = lse.reshape(-1, h * g)
    return got


# ---------------------------------------------------------------------- a pass
def _objects(s):
    """The package and what a program makes of its buffers once: cache, rotary."""
    import paper_2609_02652_amd as P
    if "own" not in s:
        cache = P.KVCache(s["k"], s["v"], s["k_scale"], s["v_scale"]) if "k" in s else None
        turn = P.Rotary(s["freq"], s["case"]["interleaved"]) if "freq" in s else None
        s["own"] = (P, cache, turn)
    return s["own"]


def run(s):
    case, op = s["case"], s["case"]["op"]
    if not own:
        if op == "rope":
            return _turned(s["x"].float(), s["positions"], s["freq"],
                           case["interleaved"]).to(TYPES[case["dst"]])
        if op == "write":
            return _write_plain(s)
        if op == "read":
            k, v = _read_plain(s)
            return {"k": k.to(TYPES[case["dst"]]), "v": v.to(TYPES[case["dst"]])}
        return _attend_plain(s)
    P, cache, turn = _objects(s)
    dst = TYPES[case["dst"]]
    if op == "rope":
        return P.rope(s["x"], s["positions"], turn, dtype=dst)
    if op == "read":
        k, v = cache.read(s["slots"], dtype=dst)
        return {"k": k, "v": v}
    if op == "write":
        hq, h, d = case["q_heads"], case["heads"], case["dim"]
        x = s["qkv"].view(case["T"], hq + 2 * h, d)
        q = cache.write(x[:, hq:hq + h], x[:, hq + h:], s["slots"], rotary=turn,
                        positions=s["positions"], q=x[:, :hq], dtype=dst)
        k, v = cache.read(s["slots"], dtype=dst) if SIZE[case["cache"]] == 1 else (s["k"], s["v"])
        return {"q": q, "k": k, "v": v}
    out = cache.attend(s["q"], s["table"], s["kv_len"], q_start=s["q_start"],
                       max_new=s["max_new"], window=case["window"], with_lse=case["lse"])
    return dict(zip(("out", "lse"), out)) if case["lse"] else {"out": out}


# ------------------------------------------------------------ what a pass needs
def work(case):
    op, d = case["op"], case["dim"]
    if op == "rope":
        n = case["T"] * case["heads"]
        return {"bytes": n * d * (SIZE[case["src"]] + SIZE[case["dst"]]) + 8.0 * case["T"]
                + 4.0 * case["rot"], "flops": 3.0 * n * case["rot"]}
    h, e = case["heads"], SIZE[case["cache"]]
    kept = 2.0 * d * e + (8 if e == 1 else 0)      # a cached token's bytes of one head
    out = 2.0 * SIZE[case["dst"]] * d if op != "attend" else 0.0
    if op == "read":
        return {"bytes": case["T"] * (h * (kept + out) + 8), "flops": 2.0 * case["T"] * h * d}
    if op == "write":
        T, hq = case["T"], case["q_heads"]
        back = h * (kept + out) + 8 if e == 1 else 0.0
        return {"bytes": T * (4.0 * (hq + 2 * h) * d + SIZE[case["dst"]] * hq * d + h * kept
                              + 16 + back) + 4.0 * case["rot"],
                "flops": T * (3.0 * (hq + h) * case["rot"] + 4.0 * h * d)}
    bytes_, pairs = 0.0, 0.0
    for n, length in _lens(case):
        seen = length if not case["window"] else min(length, case["window"] + n - 1)
        bytes_ += (2.0 * n * case["q_heads"] * d * SIZE[case["dst"]] + seen * h * kept
                   + 4.0 * seen / case["page"] + (4.0 * n * case["q_heads"] if case["lse"] else 0))
        # a query at position p sees min(p + 1, window) keys
        low, high, w = length - n + 1, length, case["window"] or length
        few = min(high, w)
        pairs += (max(0, few - low + 1) * (low + few) / 2.0 if low <= few else 0.0)
        pairs += w * max(0, high - max(low - 1, few))
    return {"bytes": bytes_ + 8.0 * case["B"], "flops": 4.0 * d * case["q_heads"] * pairs}


# ------------------------------------------------------------ the exact results
def _turn64(x, positions, freq, interleaved):
    """Each pair as a complex number times e^(i·angle)."""
    x, half = x.double().clone(), freq.numel()
    turn = torch.polar(torch.ones(1, dtype=torch.float64, device=DEV),
                       torch.outer(positions.double(), freq))[:, None]
    first = slice(0, 2 * half, 2) if interleaved else slice(0, half)
    second = slice(1, 2 * half, 2) if interleaved else slice(half, 2 * half)
    z = torch.complex(x[..., first].contiguous(), x[..., second].contiguous()) * turn
    x[..., first], x[..., second] = z.real, z.imag
    return x


def _token64(part, scale, slots, page, values):
    """The cached [T, heads, dim] of slots in 64 bits."""
    p, o = slots // page, slots % page
    x = part.float().double()
    if values:
        pages, h, chunks, d, i = x.shape
        x = x.transpose(3, 4).reshape(pages, h, chunks * i, d)
    x = x[p, :, o]
    return x if scale is None else x * scale.double()[p, :, o, None]


def _attend64(s):
    case = s["case"]
    d, h, g = case["dim"], case["heads"], case["q_heads"] // case["heads"]
    outs, lses = [], []
    starts, lens = s["q_start"].tolist(), s["kv_len"].tolist()
    for b, length in enumerate(lens):
        at = torch.arange(length, device=DEV)
        slots = s["table"][b].long()[at // case["page"]] * case["page"] + at % case["page"]
        pages = s["table"][b].long()[: -(-length // case["page"])]
        local = at                                   # the pages in order hold the tokens in order
        assert slots.numel() == length
        part = {n: (None if s[n] is None else s[n][pages] if s[n].element_size() > 1 else
                    s[n].view(torch.uint8)[pages].view(s[n].dtype))
                for n in ("k", "v", "k_scale", "v_scale")}
        k = _token64(part["k"], part["k_scale"], local, case["page"], False)
        v = _token64(part["v"], part["v_scale"], local, case["page"], True)
        n = starts[b + 1] - starts[b]
        where = torch.arange(length - n, length, device=DEV)
        sees = at <= where[:, None]
        if case["window"]:
            sees &= at > where[:, None] - case["window"]
        q = s["q"][starts[b]:starts[b + 1]].double()
        out = torch.empty(n, h * g, d, dtype=torch.float64, device=DEV)
        lse = torch.empty(n, h * g, dtype=torch.float64, device=DEV)
        for head in range(h * g):
            score = q[:, head] @ k[:, head // g].T.contiguous() * d ** -0.5
            score[~sees] = -math.inf
            lse[:, head] = torch.logsumexp(score, 1)
            out[:, head] = torch.softmax(score, 1) @ v[:, head // g]
        outs.append(out)
        lses.append(lse)
    got = {"out": torch.cat(outs)}
    if case["lse"]:
        got["lse"] = torch.cat(lses)
    return got


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "rope":
        return _turn64(s["x"], s["positions"], s["freq"], case["interleaved"])
    if op == "read":
        return {n: _token64(s[n], s[n + "_scale"], s["slots"], case["page"], n == "v")
                for n in ("k", "v")}
    if op == "attend":
        return _attend64(s)
    hq, h, d, page = case["q_heads"], case["heads"], case["dim"], case["page"]
    x = s["qkv"].reshape(-1, hq + 2 * h, d)
    args = (s["positions"], s["freq"], case["interleaved"])
    new = {"k": _turn64(x[:, hq:hq + h], *args), "v": x[:, hq + h:].double()}
    got = {"q": _turn64(x[:, :hq], *args)}
    for part, y in new.items():
        if case["cache"] in LARGEST:                # what the codes stand for
            step = y.abs().amax(-1, keepdim=True) / LARGEST[case["cache"]]
            c = y / step
            c = c.round() if case["cache"] == "int8" else c.float().to(TYPES["e4m3"]).double()
            got[part] = c * step
            continue
        buf = torch.zeros(s["k"].shape, dtype=torch.float64, device=DEV)
        p, o = s["slots"] // page, s["slots"] % page
        for t, (a, b) in enumerate(zip(p.tolist(), o.tolist())):
            buf[a, :, b] = y[t]
        if part == "v":
            i = s["v"].shape[-1]
            buf = buf.reshape(buf.shape[0], h, page // i, i, d).transpose(3, 4).contiguous()
        got[part] = buf
    return got
