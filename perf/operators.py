"""What the speed of the variable-length operators is measured on: attention over
packed prompts (forward and backward), appending to a paged key-value cache, and
attention of one new token over that cache.

A case is one call on tensors that are already on the GPU.  Its fields:

  op        "prompt" (forward: O and L), "train" (backward: dQ, dK, dV),
            "append" (rotate and store new tokens) or "decode" (one token per sequence)
  d, hq, hkv  head dim, query heads, key-value heads
  seqs, tokens  sequences and their new tokens in all (decode: cached keys in all);
            the lengths are lengths(tokens, seqs), very different ones
  past      prompt, append: keys that each sequence has before these tokens
  causal    mask (aligned to the last key); append, decode: not used
  fused     q, k and v are views into one projection's output
  page      rows of a cache page
  cache     "bf16" or "e4m3" (with a scale per key-value head)
  rotary    components of a head that are rotated, and in which pairs

`own` chooses between the elementary form of each operator and the framework's
calls; both take the same state.
"""
import math
import random

import torch

own = False


def lengths(tokens, seqs):
    """`tokens` cut into `seqs` lengths at random places: a few long sequences, many short ones (as many tokens as
    sequences: one each)."""
    if tokens == seqs:
        return [1] * seqs
    r = random.Random(tokens * 1009 + seqs)
    cuts = [0] + sorted(r.randint(0, tokens) for _ in range(seqs - 1)) + [tokens]
    return [b - a for a, b in zip(cuts, cuts[1:])]


def _prompt(name, op, d, hq, hkv, seqs, tokens, causal=True, past=0, fused=False):
    return {"name": name, "op": op, "d": d, "hq": hq, "hkv": hkv, "seqs": seqs, "tokens": tokens, "past": past,
            "causal": causal, "fused": fused}


def _append(name, d, hq, hkv, seqs, tokens, past, page, cache, rotary, interleaved):
    return {"name": name, "op": "append", "d": d, "hq": hq, "hkv": hkv, "seqs": seqs, "tokens": tokens, "past": past,
            "page": page, "cache": cache, "rotary": rotary, "interleaved": interleaved}


def _decode(name, d, hq, hkv, seqs, tokens, page, cache):
    return {"name": name, "op": "decode", "d": d, "hq": hq, "hkv": hkv, "seqs": seqs, "tokens": tokens, "page": page,
            "cache": cache}


def listed():
    return [
        # three short prompts of a small model: launches count
        _prompt("prompt-short-d64", "prompt", 64, 4, 2, 3, 250),
        # a batch of mixed prompts, straight from the fused projection
        _prompt("prompt-mixed-d128", "prompt", 128, 32, 8, 12, 8192, fused=True),
        # one long document
        _prompt("prompt-long-d128", "prompt", 128, 32, 8, 1, 8192),
        # the second part of two long prompts, on the keys of both parts, at the largest head dim
        _prompt("prompt-chunk-d256", "prompt", 256, 8, 4, 2, 1500, past=4096),
        # a fine-tuning step on a few short samples, one K/V head per query head
        _prompt("train-short-d64", "train", 64, 8, 8, 5, 600),
        # a training micro-batch of packed documents
        _prompt("train-mixed-d128", "train", 128, 32, 8, 12, 8192, fused=True),
        # training on one long document
        _prompt("train-long-d128", "train", 128, 32, 8, 1, 8192),
        # one new token of each of 64 running requests into the cache
        _append("append-token-bf16", 128, 32, 8, 64, 64, 500, 16, "bf16", 128, False),
        # a batch of prompts into an 8-bit cache, three quarters of each head rotated in adjacent pairs
        _append("append-prompt-e4m3", 128, 32, 8, 8, 8192, 0, 64, "e4m3", 96, True),
        # one request of a small model, early in its answer
        _decode("decode-one-d64", 64, 8, 2, 1, 901, 16, "bf16"),
        # 64 running requests of very different lengths
        _decode("decode-mixed-d128", 128, 32, 8, 64, 131072, 16, "bf16"),
        # one request with a very long context in an 8-bit cache
        _decode("decode-long-e4m3", 128, 32, 8, 1, 131072, 64, "e4m3"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _padded(case):
    """Scores of the padded elementary form."""
    q = lengths(case["tokens"], case["seqs"])
    return case["seqs"] * case["hq"] * max(q) * (max(q) + case["past"])


def draw(rng):
    top = {}
    for c in listed():
        w = work(c)
        top[c["op"]] = max(top.get(c["op"], 0), w["bytes"] + w["flops"])
    while True:
        op = rng.choice(["prompt", "train", "append", "decode"])
        d = rng.choice([64, 128, 128, 256])
        hkv = rng.choice([1, 2, 4, 8])
        hq = hkv * rng.choice([1, 2, 4, 8])
        seqs = _log(rng, 1, 48)
        if op in ("prompt", "train"):
            c = _prompt("", op, d, hq, hkv, seqs, _log(rng, 64, 8192), rng.random() < 0.8,
                        rng.choice([0, 0, _log(rng, 1, 4096)]), rng.random() < 0.5)
            if c["past"]:
                c["fused"] = False
            if _padded(c) > 1 << 31:
                continue
        elif op == "append":
            tokens = seqs if rng.random() < 0.5 else _log(rng, 64, 8192)
            c = _append("", d, hq, hkv, seqs, tokens, _log(rng, 1, 1024), rng.choice([16, 32, 64]),
                        rng.choice(["bf16", "e4m3"]), rng.choice([d, d, d // 2]), rng.random() < 0.5)
        else:
            c = _decode("", d, hq, hkv, seqs, _log(rng, 64, 131072), rng.choice([16, 32, 64]),
                        rng.choice(["bf16", "e4m3"]))
        del c["name"]
        w = work(c)
        if w["bytes"] + w["flops"] <= top[op]:
            return c


def _pairs(case):
    """Visible (query, key) pairs of all sequences, per query head."""
    total = 0
    for m in lengths(case["tokens"], case["seqs"]):
        n = m + case["past"]
        total += m * case["past"] + m * (m + 1) // 2 if case["causal"] else m * n
    return total


def work(case):
    d, hq, hkv, t = case["d"], case["hq"], case["hkv"], case["tokens"]
    if case["op"] in ("prompt", "train"):
        keys = t + case["seqs"] * case["past"]
        q, kv = 2 * t * hq * d, 2 * keys * hkv * d
        if case["op"] == "prompt":
            return {"bytes": 2 * q + 2 * kv + 4 * t * hq, "flops": 4 * d * hq * _pairs(case)}
        return {"bytes": 4 * q + 4 * kv + 4 * t * hq, "flops": 10 * d * hq * _pairs(case)}
    size = 2 if case["cache"] == "bf16" else 1
    if case["op"] == "append":  # q, k, v in; q, cache rows out
        return {"bytes": 2 * t * d * (2 * hq + 2 * hkv) + size * 2 * t * hkv * d, "flops": 3 * t * (hq + hkv) * case["rotary"]}
    return {"bytes": size * 2 * t * hkv * d + 2 * 2 * case["seqs"] * hq * d, "flops": 4 * t * hq * d}


# ------------------------------------------------------------------ inputs
def _cu(lens):
    at = [0]
    for n in lens:
        at.append(at[-1] + n)
    return torch.tensor(at, dtype=torch.int32, device="cuda")


def _tables(lens, page, gen):
    """Pages for `lens` tokens each, in random order: a block table with -1 behind each sequence's last page."""
    need = [-(-n // page) for n in lens]
    ids = torch.randperm(sum(need) + 3, generator=gen)
    table = torch.full((len(lens), max(max(need), 1)), -1, dtype=torch.int32)
    at = 0
    for s, n in enumerate(need):
        table[s, :n] = ids[at:at + n].to(torch.int32)
        at += n
    return table.cuda(), len(ids)


def prepare(case, seed):
    gpu = torch.Generator(device="cuda")
    gpu.manual_seed(int(seed))
    cpu = torch.Generator()
    cpu.manual_seed(int(seed) + 1)

    def normal(*shape):
        return torch.randn(shape, generator=gpu, device="cuda", dtype=torch.float32)

    d, hq, hkv, tokens = case["d"], case["hq"], case["hkv"], case["tokens"]
    lens = lengths(tokens, case["seqs"])
    st = dict(case, scale=1.0 / math.sqrt(d))
    if case["op"] in ("prompt", "train"):
        # scores of a few units, as behind a trained projection
        if case["fused"]:
            qkv = normal(tokens, hq + 2 * hkv, d).to(torch.bfloat16)
            q, k, v = qkv.split([hq, hkv, hkv], dim=1)
        else:
            keys = tokens + case["seqs"] * case["past"]
            q, k, v = (normal(n, h, d).to(torch.bfloat16) for n, h in ((tokens, hq), (keys, hkv), (keys, hkv)))
        st |= {"q": q, "k": k, "v": v, "cu_q": _cu(lens), "cu_k": _cu([n + case["past"] for n in lens]),
               "max_q": max(lens), "max_k": max(lens) + case["past"]}
        if case["op"] == "train":
            st["o"], st["lse"] = _plain_forward(st)
            st["do"] = normal(tokens, hq, d).to(torch.bfloat16)
        return st
    e4m3 = case["cache"] == "e4m3"
    if case["op"] == "append":
        old = [case["past"]] * case["seqs"]
        table, pages = _tables([a + b for a, b in zip(old, lens)], case["page"], cpu)
        st |= {"q": normal(tokens, hq, d).to(torch.bfloat16), "k": normal(tokens, hkv, d).to(torch.bfloat16),
               "v": normal(tokens, hkv, d).to(torch.bfloat16), "cu": _cu(lens),
               "lens": torch.tensor(old, dtype=torch.int32, device="cuda"),
               "inv_freq": (10000.0 ** (-torch.arange(0, case["rotary"], 2, dtype=torch.float64) / case["rotary"])).float().cuda()}
    else:
        table, pages = _tables(lens, case["page"], cpu)
        st |= {"q": normal(case["seqs"], hq, d).to(torch.bfloat16), "max_k": max(lens),
               "lens": torch.tensor(lens, dtype=torch.int32, device="cuda")}
    kc, vc = (normal(pages, hkv, case["page"], d) for _ in range(2))
    st |= {"table": table, "k_scale": None, "v_scale": None}
    if e4m3:  # a scale for each head: its values use a good part of the type's range
        st["k_scale"], st["v_scale"] = (torch.linspace(0.02, 0.03, hkv, device="cuda") * f for f in (1.0, 0.9))
        kc, vc = kc / st["k_scale"][:, None, None], vc / st["v_scale"][:, None, None]
        st["k_cache"], st["v_cache"] = (c.clamp(-448.0, 448.0).to(torch.float8_e4m3fn) for c in (kc, vc))
    else:
        st["k_cache"], st["v_cache"] = kc.to(torch.bfloat16), vc.to(torch.bfloat16)
    return st


# ------------------------------------------------------------------ elementary forms
def _pad(x, cu, longest):
    """[tokens, heads, d] -> fp32 [seqs, heads, longest, d] and which places are real."""
    at = torch.arange(longest, device=x.device)
    real = at < (cu[1:] - cu[:-1])[:, None]
    rows = (cu[:-1, None] + at).clamp(max=x.shape[0] - 1)
    return (x[rows].float() * real[..., None, None]).transpose(1, 2), real


def _places(tokens, cu):
    """The sequence of each token and its place there."""
    t = torch.arange(tokens, device=cu.device, dtype=torch.int32)
    s = (torch.searchsorted(cu, t, right=True) - 1).clamp(max=cu.shape[0] - 2)
    return s, (t - cu[s]).long()


def _scores(st):
    """Grouped, padded q [S, Hkv, G, M, d], k, v [S, Hkv, N, d], scaled scores and the visible pairs."""
    hkv, g, d = st["hkv"], st["hq"] // st["hkv"], st["d"]
    q, rows = _pad(st["q"], st["cu_q"], st["max_q"])
    k, cols = _pad(st["k"], st["cu_k"], st["max_k"])
    v, _ = _pad(st["v"], st["cu_k"], st["max_k"])
    q = q.reshape(-1, hkv, g, st["max_q"], d)
    s = (q.flatten(2, 3) @ k.transpose(2, 3)).reshape(-1, hkv, g, st["max_q"], st["max_k"]) * st["scale"]
    see = rows[:, :, None] & cols[:, None, :]
    if st["causal"]:
        m, n = (st[c][1:] - st[c][:-1] for c in ("cu_q", "cu_k"))
        i, j = torch.arange(st["max_q"], device=s.device), torch.arange(st["max_k"], device=s.device)
        see = see & (j - i[:, None] <= (n - m)[:, None, None])
    return q, k, v, s, see[:, None, None]


def _unpad(x, st, which):
    """fp32 [S, heads, longest, ...] -> [tokens, heads, ...]."""
    s, i = _places(st["q" if which == "cu_q" else "k"].shape[0], st[which])
    return x[s, :, i]


def _plain_forward(st):
    q, k, v, s, see = _scores(st)
    s = s.masked_fill(~see, -math.inf)
    top = s.amax(-1, keepdim=True)
    top = top.masked_fill(top == -math.inf, 0.0)
    p = torch.exp(s - top)
    total = p.sum(-1, keepdim=True)
    o = (p.flatten(2, 3) @ v).reshape(q.shape) / total.masked_fill(total == 0, 1.0)
    lse = torch.log(total) + top
    o = _unpad(o.flatten(1, 2), st, "cu_q").to(torch.bfloat16)
    return o, _unpad(lse.flatten(1, 2)[..., 0], st, "cu_q").t().contiguous()


def _plain_backward(st):
    q, k, v, s, see = _scores(st)
    g = st["hq"] // st["hkv"]
    do, _ = _pad(st["do"], st["cu_q"], st["max_q"])
    o, _ = _pad(st["o"], st["cu_q"], st["max_q"])
    lse, _ = _pad(st["lse"].t()[..., None], st["cu_q"], st["max_q"])
    do, o, lse = (x.reshape(-1, st["hkv"], g, st["max_q"], x.shape[-1]) for x in (do, o, lse))
    p = torch.exp(s - lse).masked_fill(~see, 0.0)
    dp = (do.flatten(2, 3) @ v.transpose(2, 3)).reshape(p.shape)
    ds = p * (dp - (do * o).sum(-1, keepdim=True))
    ds, p, do, flat = ds.flatten(2, 3), p.flatten(2, 3), do.flatten(2, 3), q.flatten(2, 3)
    dq = (ds @ k).reshape(q.shape).flatten(1, 2) * st["scale"]
    dk = ds.transpose(2, 3) @ flat * st["scale"]
    dv = p.transpose(2, 3) @ do
    return tuple(_unpad(x, st, c).to(torch.bfloat16) for x, c in ((dq, "cu_q"), (dk, "cu_k"), (dv, "cu_k")))


def _rotate(x, place, inv_freq, interleaved):
    """The first components of each head rotated by place * inv_freq (angles in 64 bits), the others as they are."""
    angle = place.double()[:, None] * inv_freq.double()
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    n = 2 * inv_freq.shape[0]
    x, rest = x[..., :n].float(), x[..., n:].float()
    a, b = (x[..., 0::2], x[..., 1::2]) if interleaved else x.chunk(2, dim=-1)
    a, b = a * cos - b * sin, a * sin + b * cos
    x = torch.stack((a, b), dim=-1).flatten(-2) if interleaved else torch.cat((a, b), dim=-1)
    return torch.cat((x, rest), dim=-1)


def _plain_append(st):
    s, i = _places(st["k"].shape[0], st["cu"])
    place = st["lens"][s] + i
    page, row = st["table"][s, place // st["page"]].long(), place % st["page"]
    q = _rotate(st["q"], place, st["inv_freq"], st["interleaved"]).to(torch.bfloat16)
    heads = torch.arange(st["hkv"], device=page.device)
    at = (page[:, None], heads, row[:, None])
    for_cache = (("k_cache", "k_scale", _rotate(st["k"], place, st["inv_freq"], st["interleaved"])),
                 ("v_cache", "v_scale", st["v"].float()))
    for name, scale, x in for_cache:
        if st["cache"] == "e4m3":
            x = (x / st[scale][:, None]).clamp(-448.0, 448.0).to(torch.float8_e4m3fn)
            st[name].view(torch.uint8)[at] = x.view(torch.uint8)
        else:
            st[name][at] = x.to(torch.bfloat16)
    return q, st["k_cache"], st["v_cache"]


def _plain_decode(st):
    d, hkv, n = st["d"], st["hkv"], st["max_k"]
    pages = st["table"].long().clamp(min=0)
    # [S, pages, Hkv, page, d] -> fp32 [S, Hkv, N, d]
    k, v = (st[c][pages].float().transpose(1, 2).flatten(2, 3)[:, :, :n] for c in ("k_cache", "v_cache"))
    if st["cache"] == "e4m3":
        k, v = k * st["k_scale"][:, None, None], v * st["v_scale"][:, None, None]
    q = st["q"].float().reshape(-1, hkv, st["hq"] // hkv, d)
    s = (q @ k.transpose(2, 3)) * st["scale"]
    see = (torch.arange(n, device=s.device) < st["lens"][:, None])[:, None, None]
    s = s.masked_fill(~see, -math.inf)
    top = s.amax(-1, keepdim=True)
    p = torch.exp(s - top.masked_fill(top == -math.inf, 0.0))
    total = p.sum(-1, keepdim=True)
    return ((p @ v) / total.masked_fill(total == 0, 1.0)).flatten(1, 2).to(torch.bfloat16)


# ------------------------------------------------------------------ one pass
def _own(st):
    from paper_2601_21824_amd import binding as dash
    if st["op"] == "prompt":
        return dash.attn_packed_fwd(st["q"], st["k"], st["v"], st["cu_q"], st["cu_k"], causal=st["causal"])
    if st["op"] == "train":
        return dash.attn_packed_bwd(st["q"], st["k"], st["v"], st["o"], st["do"], st["lse"], st["cu_q"], st["cu_k"],
                                    causal=st["causal"])
    if st["op"] == "append":
        q = torch.empty_like(st["q"])
        dash.dash_kv_append(st["k"], st["v"], st["k_cache"], st["v_cache"], st["table"], st["lens"], cu=st["cu"], q=st["q"],
                            q_out=q, inv_freq=st["inv_freq"], interleaved=st["interleaved"], k_scale=st["k_scale"],
                            v_scale=st["v_scale"])
        return q, st["k_cache"], st["v_cache"]
    return dash.attn_decode(st["q"], st["k_cache"], st["v_cache"], st["table"], st["lens"], k_scale=st["k_scale"],
                            v_scale=st["v_scale"])


def run(state):
    if own:
        return _own(state)
    return {"prompt": _plain_forward, "train": _plain_backward, "append": _plain_append,
            "decode": _plain_decode}[state["op"]](state)


# ------------------------------------------------------------------ 64 bits
def _exact_prompt(st, train):
    """One sequence and head at a time, from the definition: softmax over the visible keys, and its derivative."""
    g, scale = st["hq"] // st["hkv"], st["scale"]
    q, k, v = (st[x].double() for x in "qkv")
    o, lse = torch.zeros_like(q), torch.full((st["hq"], q.shape[0]), -math.inf, dtype=torch.float64, device="cuda")
    dq, dk, dv = (torch.zeros_like(x) for x in (q, k, v))
    cu_q, cu_k = st["cu_q"].tolist(), st["cu_k"].tolist()
    for a, b, x, y in zip(cu_q, cu_q[1:], cu_k, cu_k[1:]):
        if a == b or x == y:
            continue
        hidden = torch.zeros(b - a, y - x, dtype=torch.bool, device="cuda")
        if st["causal"]:
            hidden = torch.ones_like(hidden).triu((y - x) - (b - a) + 1)
        empty = hidden.all(-1, keepdim=True)
        for h in range(st["hq"]):
            kh, vh = k[x:y, h // g], v[x:y, h // g]
            s = (q[a:b, h] @ kh.t()).mul_(scale).masked_fill_(hidden, -math.inf)
            lse[h, a:b] = torch.logsumexp(s, -1)
            p = torch.softmax(s, -1).masked_fill_(empty, 0.0)
            o[a:b, h] = p @ vh
            if train:
                do = st["do"][a:b, h].double()
                dp = do @ vh.t()
                ds = p * (dp - (p * dp).sum(-1, keepdim=True)) * scale
                dq[a:b, h] = ds @ kh
                dk[x:y, h // g] += ds.t() @ q[a:b, h]
                dv[x:y, h // g] += p.t() @ do
    return (dq, dk, dv) if train else (o, lse)


def _exact_append(st):
    n, cu, old = st["rotary"] // 2, st["cu"].tolist(), st["lens"].tolist()
    place = torch.cat([torch.arange(o, o + b - a) for o, a, b in zip(old, cu, cu[1:])]).cuda()
    turn = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"), place[:, None, None] * st["inv_freq"].double())

    def rotated(x):
        x = x.double().clone()
        c = x[..., :2 * n]
        z = torch.complex(c[..., 0::2], c[..., 1::2]) if st["interleaved"] else torch.complex(c[..., :n], c[..., n:])
        z = z * turn
        if st["interleaved"]:
            c[..., 0::2], c[..., 1::2] = z.real, z.imag
        else:
            c[..., :n], c[..., n:] = z.real, z.imag
        return x

    caches = []
    seq = torch.cat([torch.full((b - a,), i) for i, (a, b) in enumerate(zip(cu, cu[1:]))]).cuda()
    where = st["table"].long()[seq, place // st["page"]] * st["page"] + place % st["page"]  # row of the whole pool
    for name, scale, x in (("k_cache", "k_scale", rotated(st["k"])), ("v_cache", "v_scale", st["v"].double())):
        pool = st[name].double().transpose(1, 2).flatten(0, 1)
        if st[scale] is not None:
            x = (x / st[scale].double()[:, None]).clamp(-448.0, 448.0)
        pool[where] = x
        caches.append(pool.unflatten(0, (-1, st["page"])).transpose(1, 2).contiguous())
    return (rotated(st["q"]), *caches)


def _exact_decode(st):
    g, lens = st["hq"] // st["hkv"], st["lens"].tolist()
    out = torch.zeros(st["q"].shape, dtype=torch.float64, device="cuda")
    for s, n in enumerate(lens):
        if n == 0:
            continue
        ids = st["table"][s, :-(-n // st["page"])].long()
        for h in range(st["hkv"]):
            k, v = (st[c][ids, h].double().flatten(0, 1)[:n] for c in ("k_cache", "v_cache"))
            if st["k_scale"] is not None:
                k, v = k * st["k_scale"][h].double(), v * st["v_scale"][h].double()
            p = torch.softmax((st["q"][s, h * g:(h + 1) * g].double() @ k.t()) * st["scale"], -1)
            out[s, h * g:(h + 1) * g] = p @ v
    return out


def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] in ("prompt", "train"):
        return _exact_prompt(st, case["op"] == "train")
    return _exact_append(st) if case["op"] == "append" else _exact_decode(st)
