"""What the speed of the long-context operators is measured on: rotary positions (forward and
backward), a microscaled key-value cache (written, read back and attended to), and attention of
one new token per sequence over a prefix that the whole batch shares.

A case is one pass on tensors that are already on the GPU.  Its fields:

  op        "rotary" (q and k of packed rows turned by their positions, or their gradients turned back),
            "cache" (new tokens quantised into the cache, and rows of it read back as bf16),
            "decode" (one token per sequence over a microscaled cache) or "prefix" (the same behind a shared prefix)
  d, hq, hkv  head dim, query heads, key-value heads
  seqs, tokens  sequences and, in all of them, their rows (rotary), new tokens (cache) or keys of their own (decode,
            prefix); the lengths are lengths(tokens, seqs), very different ones
  past      rotary: the first row's position; cache: keys that each sequence has before these tokens
  whole     cache: read back every key of each sequence, not the new ones alone
  prefix    keys that all sequences share
  page      rows of a cache page
  cache     "bf16", "e4m3" (a given scale per key-value head), "mxfp8" or "mxfp4" (a power of two for each 32 components)
  rotary, interleaved, scaled  components of a head that are rotated, in which pairs, and whether the
            frequencies and the amplitude are those of a context stretched eightfold
  backward  rotary: the gradients
  fused     rotary: q and k are views into one projection's output

`own` chooses between the elementary form of each operator and the framework's
calls; both take the same state.
"""
import math
import random

import torch

own = False

ELEMENTS = {"mxfp8": (448.0, 8, 0x600000), "mxfp4": (6.0, 2, 0x400000)}  # largest value, its exponent and fraction bits


def lengths(tokens, seqs):
    """`tokens` cut into `seqs` lengths at random places: a few long sequences, many short ones (as many tokens as
    sequences: one each)."""
    if tokens == seqs:
        return [1] * seqs
    r = random.Random(tokens * 1009 + seqs)
    cuts = [0] + sorted(r.randint(0, tokens) for _ in range(seqs - 1)) + [tokens]
    return [b - a for a, b in zip(cuts, cuts[1:])]


def _rotary(name, d, hq, hkv, seqs, tokens, past, rotary, interleaved, scaled, backward, fused):
    return {"name": name, "op": "rotary", "d": d, "hq": hq, "hkv": hkv, "seqs": seqs, "tokens": tokens, "past": past,
            "rotary": rotary, "interleaved": interleaved, "scaled": scaled, "backward": backward, "fused": fused}


def _cache(name, d, hq, hkv, seqs, tokens, past, page, cache, rotary, interleaved, whole):
    return {"name": name, "op": "cache", "d": d, "hq": hq, "hkv": hkv, "seqs": seqs, "tokens": tokens, "past": past,
            "page": page, "cache": cache, "rotary": rotary, "interleaved": interleaved, "whole": whole}


def _decode(name, d, hq, hkv, seqs, tokens, page, cache):
    return {"name": name, "op": "decode", "d": d, "hq": hq, "hkv": hkv, "seqs": seqs, "tokens": tokens, "page": page,
            "cache": cache}


def _prefix(name, d, hq, hkv, seqs, prefix, tokens, page, cache):
    return {"name": name, "op": "prefix", "d": d, "hq": hq, "hkv": hkv, "seqs": seqs, "prefix": prefix, "tokens": tokens,
            "page": page, "cache": cache}


def listed():
    return [
        # the next token of each of 64 running requests, deep in a stretched context
        _rotary("rotary-token-d128", 128, 32, 8, 64, 64, 100000, 128, False, True, False, False),
        # a training micro-batch of packed documents, straight from the fused projection
        _rotary("rotary-train-d128", 128, 32, 8, 12, 8192, 0, 128, False, True, False, True),
        # the gradients of a larger head of which half is rotated in adjacent pairs
        _rotary("rotary-back-d256", 256, 16, 4, 5, 5001, 0, 128, True, False, True, False),
        # one new token of each of 64 running requests into an 8-bit cache, and back
        _cache("cache-token-mxfp8", 128, 32, 8, 64, 64, 500, 16, "mxfp8", 128, False, False),
        # a batch of prompts into an 8-bit cache, and back for their attention
        _cache("cache-prompt-mxfp8", 128, 32, 8, 8, 8192, 0, 64, "mxfp8", 128, False, True),
        # the second part of four prompts into a 4-bit cache; the keys of both parts back
        _cache("cache-chunk-mxfp4", 128, 32, 8, 4, 3001, 4096, 32, "mxfp4", 96, True, True),
        # 64 running requests of very different lengths
        _decode("decode-mixed-mxfp8", 128, 32, 8, 64, 131072, 16, "mxfp8"),
        # one request with a very long context in a 4-bit cache
        _decode("decode-long-mxfp4", 128, 32, 8, 1, 131072, 64, "mxfp4"),
        # three requests of a small model behind one instruction
        _prefix("prefix-short-d64", 64, 8, 2, 3, 700, 150, 16, "bf16"),
        # 64 questions on one long document
        _prefix("prefix-long-bf16", 128, 32, 8, 64, 32768, 16384, 16, "bf16"),
        # 24 requests behind a shared conversation in an 8-bit cache
        _prefix("prefix-mixed-mxfp8", 128, 32, 8, 24, 16384, 6007, 64, "mxfp8"),
        # eight samples of one answer at the largest head dim, 4-bit cache
        _prefix("prefix-samples-mxfp4", 256, 16, 4, 8, 9001, 2000, 32, "mxfp4"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    top = {}
    for c in listed():
        w = work(c)
        top[c["op"]] = max(top.get(c["op"], 0), w["bytes"] + w["flops"])
    while True:
        op = rng.choice(["rotary", "cache", "decode", "prefix", "prefix"])
        d = rng.choice([64, 128, 128, 256])
        hkv = rng.choice([1, 2, 4, 8])
        hq = hkv * rng.choice([1, 2, 4, 8])
        seqs = _log(rng, 1, 64)
        rotary = rng.choice([d, d, d // 2, 3 * d // 4])
        if op == "rotary":
            tokens = seqs if rng.random() < 0.3 else _log(rng, 1, 8192)
            c = _rotary("", d, hq, hkv, seqs, tokens, rng.choice([0, _log(rng, 1, 131072)]), rotary, rng.random() < 0.5,
                        rng.random() < 0.5, rng.random() < 0.5, rng.random() < 0.5)
        elif op == "cache":
            tokens = seqs if rng.random() < 0.3 else _log(rng, 1, 8192)
            c = _cache("", d, hq, hkv, seqs, tokens, rng.choice([0, _log(rng, 1, 2048)]), rng.choice([16, 32, 64]),
                       rng.choice(["mxfp8", "mxfp4"]), rotary, rng.random() < 0.5, rng.random() < 0.5)
        elif op == "decode":
            c = _decode("", d, hq, hkv, seqs, _log(rng, 64, 131072), rng.choice([16, 32, 64]), rng.choice(["mxfp8", "mxfp4"]))
        else:
            c = _prefix("", d, hq, hkv, seqs, _log(rng, 64, 32768), _log(rng, 1, 16384), rng.choice([16, 32, 64]),
                        rng.choice(["bf16", "e4m3", "mxfp8", "mxfp4"]))
        del c["name"]
        w = work(c)
        if w["bytes"] + w["flops"] <= top[op]:
            return c


def _row_bytes(case):
    """Bytes of a cached row, its scales among them."""
    return case["d"] * {"bf16": 2, "e4m3": 1, "mxfp8": 33 / 32, "mxfp4": 17 / 32}[case["cache"]]


def work(case):
    d, hq, hkv, t = case["d"], case["hq"], case["hkv"], case["tokens"]
    if case["op"] == "rotary":
        return {"bytes": 2 * 2 * t * (hq + hkv) * d, "flops": 3 * t * (hq + hkv) * case["rotary"]}
    row = 2 * hkv * _row_bytes(case)  # K and V
    if case["op"] == "cache":  # q, k, v in, q and rows out; rows in, k, v out
        back = t + (case["seqs"] * case["past"] if case["whole"] else 0)
        return {"bytes": 2 * t * d * (2 * hq + 2 * hkv) + t * row + back * (row + 4 * hkv * d),
                "flops": 3 * t * (hq + hkv) * case["rotary"] + 2 * (t + back) * 2 * hkv * d}
    p = case.get("prefix", 0)
    return {"bytes": (t + p) * row + 2 * 2 * case["seqs"] * hq * d, "flops": 4 * hq * d * (t + p * case["seqs"])}


# ------------------------------------------------------------------ inputs
def _cu(lens):
    at = [0]
    for n in lens:
        at.append(at[-1] + n)
    return torch.tensor(at, dtype=torch.int32, device="cuda")


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _tables(lens, page, gen, shared=0):
    """Pages for `lens` tokens each, in random order, the first `shared` of them everybody's: a block table with -1 behind
    each sequence's last page."""
    need = [-(-n // page) for n in lens]
    ids = torch.randperm(sum(need) - (len(need) - 1) * shared + 3, generator=gen)
    table = torch.full((len(lens), max(max(need), 1)), -1, dtype=torch.int32)
    at = shared
    for s, n in enumerate(need):
        table[s, :shared] = ids[:shared]
        table[s, shared:n] = ids[at:at + n - shared].to(torch.int32)
        at += n - shared
    return table.cuda(), len(ids)


def _frequencies(case):
    """One per rotated pair, and the amplitude.  Stretched eightfold from 4096 positions: pairs that turn more than 32 times over
    those keep their frequency, those that turn less than once take an eighth of it, the others lie between."""
    n = case["rotary"]
    f = 10000.0 ** (-torch.arange(0, n, 2, dtype=torch.float64) / n)
    if not case.get("scaled"):
        return f.float().cuda(), 1.0
    place = [n * math.log(4096 / (turns * 2 * math.pi)) / (2 * math.log(10000.0)) for turns in (32, 1)]
    lo, hi = max(math.floor(place[0]), 0), min(math.ceil(place[1]), n - 1)
    slow = ((torch.arange(n // 2, dtype=torch.float64) - lo) / max(hi - lo, 1e-3)).clamp(0, 1)
    return (f * (1 - slow) + f / 8 * slow).float().cuda(), 0.1 * math.log(8.0) + 1.0


def prepare(case, seed):
    gpu = torch.Generator(device="cuda")
    gpu.manual_seed(int(seed))
    cpu = torch.Generator()
    cpu.manual_seed(int(seed) + 1)

    def normal(*shape):
        return torch.randn(shape, generator=gpu, device="cuda", dtype=torch.float32)

    d, hq, hkv, tokens, seqs = case["d"], case["hq"], case["hkv"], case["tokens"], case["seqs"]
    lens = lengths(tokens, seqs)
    st = dict(case, scale=1.0 / math.sqrt(d))
    if "rotary" in case:
        st["inv_freq"], st["amplitude"] = _frequencies(case)
    if case["op"] == "rotary":
        if case["fused"]:
            q, k, _ = normal(tokens, hq + 2 * hkv, d).to(torch.bfloat16).split([hq, hkv, hkv], dim=1)
        else:
            q, k = (normal(tokens, h, d).to(torch.bfloat16) for h in (hq, hkv))
        st |= {"q": q, "k": k, "cu": _cu(lens), "start": _i32([case["past"] + 7 * i for i in range(seqs)])}
        if tokens == seqs:  # one row each, anywhere
            st["positions"] = (case["past"] + torch.randint(0, 31072, (tokens,), generator=cpu)).to(torch.int32).cuda()
        return st
    # keys as behind a trained projection: a few components much larger than the others
    loud = 1.0 + 7.0 * (torch.rand((hkv, 1, d), generator=gpu, device="cuda") < 0.03)
    if case["op"] == "cache":
        old = [case["past"]] * seqs
        table, pages = _tables([a + b for a, b in zip(old, lens)], case["page"], cpu)
        first = [0 if case["whole"] else n for n in old]
        rows = [a + b - f for a, b, f in zip(old, lens, first)]
        st |= {"q": normal(tokens, hq, d).to(torch.bfloat16), "k": (normal(tokens, hkv, d) * loud[:, 0]).to(torch.bfloat16),
               "v": normal(tokens, hkv, d).to(torch.bfloat16), "cu": _cu(lens), "lens": _i32(old),
               "lens_after": _i32([a + b for a, b in zip(old, lens)]), "first": _i32(first), "cu_back": _cu(rows), "back": sum(rows)}
    else:
        prefix = case.get("prefix", 0)
        full = [prefix + n for n in lens]
        table, pages = _tables(full, case["page"], cpu, prefix // case["page"])
        st |= {"q": normal(seqs, hq, d).to(torch.bfloat16), "max_own": max(lens), "lens": _i32(full)}
        if case["op"] == "prefix":
            st |= {"prefix_table": table[0, :-(-prefix // case["page"])].contiguous(), "prefix_len": _i32([prefix])}
    st |= {"table": table, "k_scale": None, "v_scale": None}
    kc, vc = normal(pages, hkv, case["page"], d) * (loud if case["op"] == "cache" else 1.0), normal(pages, hkv, case["page"], d)
    if case["op"] == "prefix" and case["prefix"] % case["page"]:  # the prefix's last page: everybody has a copy, and goes on behind it
        n, at = case["prefix"] // case["page"], case["prefix"] % case["page"]
        for c in (kc, vc):
            c[table[:, n].long(), :, :at] = c[table[0, n].long(), :, :at].clone()
    if case["cache"] == "bf16":
        st["k_cache"], st["v_cache"] = kc.to(torch.bfloat16), vc.to(torch.bfloat16)
    elif case["cache"] == "e4m3":
        st["k_scale"], st["v_scale"] = (torch.linspace(0.02, 0.03, hkv, device="cuda") * f for f in (1.0, 0.9))
        kc, vc = kc / st["k_scale"][:, None, None], vc / st["v_scale"][:, None, None]
        st["k_cache"], st["v_cache"] = (c.clamp(-448.0, 448.0).to(torch.float8_e4m3fn) for c in (kc, vc))
    else:
        (st["k_cache"], st["k_scale"]), (st["v_cache"], st["v_scale"]) = (_quantise(c, case["cache"]) for c in (kc, vc))
    return st


# ------------------------------------------------------------------ elementary forms
def _rotate(x, place, inv_freq, interleaved, amplitude=1.0, back=False, wide=False):
    """The first components of each head rotated by place * inv_freq (angles in 64 bits), the others as they are.  wide: in 64
    bits throughout, for values that a quantisation decides on."""
    kind = torch.float64 if wide else torch.float32
    angle = place.double()[:, None] * inv_freq.double()
    cos, sin = (angle.cos() * amplitude).to(kind)[:, None], (angle.sin() * (-amplitude if back else amplitude)).to(kind)[:, None]
    n = 2 * inv_freq.shape[0]
    x, rest = x[..., :n].to(kind), x[..., n:].to(kind)
    a, b = (x[..., 0::2], x[..., 1::2]) if interleaved else x.chunk(2, dim=-1)
    a, b = a * cos - b * sin, a * sin + b * cos
    x = torch.stack((a, b), dim=-1).flatten(-2) if interleaved else torch.cat((a, b), dim=-1)
    return torch.cat((x, rest), dim=-1)


def _quantise(x, cache):
    """fp32 [..., d] -> elements (e4m3, or two e2m1 a byte, the lower half first) and a scale byte 127 + e for each 32: 2^e is the
    least power of two that puts the block's largest value in range."""
    largest, exponent, fraction = ELEMENTS[cache]
    x = x.unflatten(-1, (-1, 32))
    bits = x.abs().amax(-1, keepdim=True).view(torch.int32)
    byte = ((bits + (0x7FFFFF - fraction)) >> 23).sub(exponent).clamp(min=10)
    y = (x / ((byte << 23).view(torch.float32))).flatten(-2)
    scale = byte[..., 0].to(torch.uint8)
    if cache == "mxfp8":
        return y.clamp(-largest, largest).to(torch.float8_e4m3fn), scale
    a = y.abs()
    # borders between 0, 0.5, 1, 1.5, 2, 3, 4, 6; one that is met goes to the even code
    code = (a > 0.25).to(torch.uint8) + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5.0)
    code = code + 8 * (torch.signbit(y)).to(torch.uint8)
    return code[..., 0::2] + 16 * code[..., 1::2], scale


def _values(c, scale, cache):
    """What cached elements stand for, in fp32; scale: of the same rows."""
    if cache == "bf16":
        return c.float()
    if cache == "e4m3":
        return c.float() * scale
    if cache == "mxfp4":
        c = torch.stack((c & 15, c >> 4), dim=-1).flatten(-2).int()
        size, sub = (c >> 1) & 3, (c & 1).float()
        f = torch.where(size == 0, 0.5 * sub, (1.0 + 0.5 * sub) * torch.exp2((size - 1).float()))
        c = torch.where(c >= 8, -f, f)
    return (c.float().unflatten(-1, (-1, 32)) * (scale.int() << 23).view(torch.float32)[..., None]).flatten(-2)


def _places(tokens, cu):
    """The sequence of each token and its place there."""
    t = torch.arange(tokens, device=cu.device, dtype=torch.int32)
    s = (torch.searchsorted(cu, t, right=True) - 1).clamp(max=cu.shape[0] - 2)
    return s, (t - cu[s]).long()


def _plain_rotary(st):
    if "positions" in st:
        place = st["positions"]
    else:
        s, i = _places(st["q"].shape[0], st["cu"])
        place = i + st["start"][s]
    return tuple(_rotate(x, place, st["inv_freq"], st["interleaved"], st["amplitude"], st["backward"]).to(torch.bfloat16)
                 for x in (st["q"], st["k"]))


def _plain_cache(st):
    s, i = _places(st["k"].shape[0], st["cu"])
    place = st["lens"][s] + i
    at = (st["table"][s, place // st["page"]].long(), slice(None), place % st["page"])
    turn = (place, st["inv_freq"], st["interleaved"])
    q = _rotate(st["q"], *turn).to(torch.bfloat16)
    for name, x in (("k", _rotate(st["k"], *turn, wide=True).float()), ("v", st["v"].float())):
        elements, scale = _quantise(x, st["cache"])
        st[name + "_cache"].view(torch.uint8)[at] = elements.view(torch.uint8)
        st[name + "_scale"][at] = scale
    s, i = _places(st["back"], st["cu_back"])
    place = st["first"][s] + i
    at = (st["table"][s, place // st["page"]].long(), slice(None), place % st["page"])
    k, v = (_values(st[n + "_cache"].view(torch.uint8)[at].view(st[n + "_cache"].dtype), st[n + "_scale"][at], st["cache"]).to(torch.bfloat16)
            for n in "kv")
    return q, k, v


def _pages(st, name, ids):
    """The rows of pages `ids` [..., n], in fp32 [..., heads, n * page, d]."""
    c, scale = st[name + "_cache"], st[name + "_scale"]
    if scale is not None:
        scale = scale[:, None, None] if scale.dim() == 1 else scale[ids]
    raw = c.view(torch.uint8)[ids].view(c.dtype) if c.dtype != torch.bfloat16 else c[ids]
    return _values(raw, scale, st["cache"]).transpose(-4, -3).flatten(-3, -2)


def _softmax_part(s, v):
    """exp(s - max) v, the maximum and the sum."""
    top = s.amax(-1, keepdim=True)
    p = torch.exp(s - top.masked_fill(top == -math.inf, 0.0))
    return p @ v, top, p.sum(-1, keepdim=True)


def _plain_decode(st):
    d, hkv, page, g = st["d"], st["hkv"], st["page"], st["hq"] // st["hkv"]
    q = st["q"].float().reshape(-1, hkv, g, d)  # [S, Hkv, G, d]
    prefix = st.get("prefix", 0)
    parts = []
    if prefix:  # the shared keys, for all sequences at once
        k, v = (_pages(st, n, st["prefix_table"].long())[:, :prefix] for n in "kv")
        rows = q.transpose(0, 1).flatten(1, 2)  # [Hkv, S G, d]
        o, top, total = _softmax_part((rows @ k.transpose(1, 2)) * st["scale"], v)
        parts.append([x.unflatten(1, (-1, g)).transpose(0, 1) for x in (o, top, total)])
    skip = prefix // page
    width = -(-(prefix % page + st["max_own"]) // page)
    n = torch.arange(skip * page, (skip + width) * page, device=q.device)
    see = ((n >= prefix) & (n < st["lens"][:, None]))[:, None, None]
    k, v = (_pages(st, x, st["table"][:, skip:skip + width].long().clamp(min=0)) for x in "kv")
    parts.append(_softmax_part(((q @ k.transpose(2, 3)) * st["scale"]).masked_fill(~see, -math.inf), v))
    top = torch.stack([p[1] for p in parts]).amax(0)
    weight = [torch.exp(p[1] - top.masked_fill(top == -math.inf, 0.0)) for p in parts]
    o, total = (sum(w * p[i] for w, p in zip(weight, parts)) for i in (0, 2))
    return (o / total.masked_fill(total == 0, 1.0)).flatten(1, 2).to(torch.bfloat16)


# ------------------------------------------------------------------ one pass
def _own(st):
    from paper_2601_21824_amd import binding as dash
    if st["op"] == "rotary":
        where = {"positions": st["positions"]} if "positions" in st else {"cu": st["cu"], "start": st["start"]}
        return dash.rotary(st["q"], st["k"], st["inv_freq"], interleaved=st["interleaved"], amplitude=st["amplitude"],
                           backward=st["backward"], **where)
    scales = {"k_scale": st["k_scale"], "v_scale": st["v_scale"]}
    if st["op"] == "cache":
        q = torch.empty_like(st["q"])
        dash.dash_kv_append(st["k"], st["v"], st["k_cache"], st["v_cache"], st["table"], st["lens"], cu=st["cu"], q=st["q"],
                            q_out=q, inv_freq=st["inv_freq"], interleaved=st["interleaved"], **scales)
        return (q, *dash.kv_read(st["k_cache"], st["v_cache"], st["table"], st["lens_after"], st["cu_back"], st["back"],
                                 first=st["first"], **scales))
    if st["op"] == "decode":
        return dash.attn_decode(st["q"], st["k_cache"], st["v_cache"], st["table"], st["lens"], **scales)
    return dash.attn_prefix_decode(st["q"], st["k_cache"], st["v_cache"], st["table"], st["lens"], st["prefix_table"],
                                   st["prefix_len"], **scales)


def run(state):
    if own:
        return _own(state)
    return {"rotary": _plain_rotary, "cache": _plain_cache, "decode": _plain_decode, "prefix": _plain_decode}[state["op"]](state)


# ------------------------------------------------------------------ 64 bits
def _turned(x, place, st, amplitude=1.0, sign=1.0):
    n = st["rotary"] // 2
    turn = torch.polar(torch.full((), amplitude, dtype=torch.float64, device="cuda"), sign * place[:, None, None] * st["inv_freq"].double())
    x = x.double().clone()
    c = x[..., :2 * n]
    z = torch.complex(c[..., 0::2], c[..., 1::2]) if st["interleaved"] else torch.complex(c[..., :n], c[..., n:])
    z = z * turn
    if st["interleaved"]:
        c[..., 0::2], c[..., 1::2] = z.real, z.imag
    else:
        c[..., :n], c[..., n:] = z.real, z.imag
    return x


def _grid(cache):
    """The element type's values from 0 up, in the order of their codes."""
    if cache == "mxfp4":
        return torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64, device="cuda")
    return torch.arange(127, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn).double()


def _nearest(x, cache):
    """Each block of 32 by the least power of two that holds it, every value at the grid's nearest, ties to the even code."""
    grid = _grid(cache)
    x = x.unflatten(-1, (-1, 32))
    ratio = x.abs().amax(-1, keepdim=True) / grid[-1]
    frac, e = torch.frexp(ratio)  # ratio = frac 2^e, frac in [0.5, 1)
    e = torch.where(frac == 0.5, e - 1, e).clamp(min=-117)
    y = x.abs() * torch.exp2(-e.double())
    hi = torch.bucketize(y, grid).clamp(1, grid.numel() - 1)
    a, b = y - grid[hi - 1], grid[hi] - y
    code = torch.where((a < b) | ((a == b) & (hi % 2 == 1)), hi - 1, hi)
    return (torch.copysign(grid[code], x) * torch.exp2(e.double())).flatten(-2)


def _stored(st, name):
    """The whole pool's values as fp64 [pages, heads, page, d]."""
    c, scale = st[name + "_cache"], st[name + "_scale"]
    if st["cache"] == "mxfp4":
        grid = torch.cat((_grid("mxfp4"), -_grid("mxfp4")))
        c = torch.stack((grid[(c & 15).long()], grid[(c >> 4).long()]), dim=-1).flatten(-2)
    c = c.double()
    if st["cache"] == "e4m3":
        return c * scale.double()[:, None, None]
    if scale is not None:
        return (c.unflatten(-1, (-1, 32)) * torch.exp2(scale.double() - 127)[..., None]).flatten(-2)
    return c


def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] == "rotary":
        cu, start = st["cu"].tolist(), st["start"].tolist()
        place = torch.cat([torch.arange(o, o + b - a) for o, a, b in zip(start, cu, cu[1:])]).cuda()
        place = st["positions"].long() if "positions" in st else place
        return tuple(_turned(x, place, st, st["amplitude"], -1.0 if st["backward"] else 1.0) for x in (st["q"], st["k"]))
    if case["op"] == "cache":
        cu, old, back, first = (st[n].tolist() for n in ("cu", "lens", "cu_back", "first"))

        def rows(first, cu):  # rows of the whole pool
            at = []
            for s, (f, a, b) in enumerate(zip(first, cu, cu[1:])):
                j = torch.arange(f, f + b - a, device="cuda")
                at.append(st["table"][s].long()[j // st["page"]] * st["page"] + j % st["page"])
            return torch.cat(at)

        place = torch.cat([torch.arange(o, o + b - a) for o, a, b in zip(old, cu, cu[1:])]).cuda()
        to, of, out = rows(old, cu), rows(first, back), []
        for n, x in (("k", _turned(st["k"], place, st)), ("v", st["v"].double())):
            pool = _stored(st, n).transpose(1, 2).flatten(0, 1)
            pool[to] = _nearest(x, case["cache"])
            out.append(pool[of])
        return (_turned(st["q"], place, st), *out)
    g, lens, page = st["hq"] // st["hkv"], st["lens"].tolist(), st["page"]
    out = torch.zeros(st["q"].shape, dtype=torch.float64, device="cuda")
    k_all, v_all = _stored(st, "k"), _stored(st, "v")
    for s, n in enumerate(lens):
        if n == 0:
            continue
        ids = st["table"][s, :-(-n // page)].long()
        k, v = (c[ids].transpose(0, 1).flatten(1, 2)[:, :n].contiguous() for c in (k_all, v_all))  # [Hkv, n, d]
        for h in range(st["hkv"]):
            p = torch.softmax((st["q"][s, h * g:(h + 1) * g].double() @ k[h].t()) * st["scale"], -1)
            out[s, h * g:(h + 1) * g] = p @ v[h]
    return out
