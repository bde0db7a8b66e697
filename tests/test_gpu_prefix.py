"""Attention of one new token per sequence behind a shared prefix, against its definition in float64.

Bounds: those of the one-token attention without a shared prefix (o and P rounded to bf16, scores in fp32), and 8 u24 A more for
the parts' weights and their division by a sum and back.
"""
import math

import pytest
import torch

from mx_util import BF, Cache, used_rows
from paper_2601_21824_amd import binding as dash
from test_gpu_mx_cache import KINDS, attend64
from test_gpu_paged_cache import i32

pytestmark = pytest.mark.gpu

U24 = 2.0 ** -24


def tables(prefix, lens, page, seed=0):
    """Block table and page count of sequences of `lens` keys, the first `prefix` of them shared (sequences shorter than that
    have as many of the shared pages as they need), the prefix's own table, and each sequence's copy of the last shared page."""
    g = torch.Generator()
    g.manual_seed(seed)
    whole = prefix // page
    width = max([-(-n // page) for n in lens] + [-(-prefix // page), 1]) + 1
    pages = -(-prefix // page) + sum(max(-(-n // page) - whole, 0) for n in lens) + 2
    ids = torch.randperm(pages, generator=g).tolist()
    shared = [ids.pop() for _ in range(-(-prefix // page))]
    t = torch.full((len(lens), width), -1, dtype=torch.int32)
    copies = []
    for s, n in enumerate(lens):
        need = -(-n // page)
        t[s, :min(need, whole)] = torch.tensor(shared[:min(need, whole)], dtype=torch.int32)
        for i in range(whole, need):
            t[s, i] = ids.pop()
        if need > whole and prefix % page:
            copies.append(int(t[s, whole]))
    return t.cuda(), pages, torch.tensor(shared + [-1], dtype=torch.int32, device="cuda"), copies


def build(kind, d, hq, hkv, prefix, lens, page, order="phrd", seed=0, spoil=True):
    table, pages, shared, copies = tables(prefix, lens, page, seed)
    c = Cache(kind, pages, hkv, page, d, order, seed)
    g = torch.Generator(device="cuda")
    g.manual_seed(seed + d + hq)
    q = torch.randn((len(lens), hq + 1, d), generator=g, device="cuda").to(BF)[:, 1:] * 2  # strided, wide scores
    at = prefix % page
    u8 = torch.uint8
    for x in (*c.pools, *([c.k_scale, c.v_scale] if kind.startswith("mx") else [])):
        y = x.view(u8) if x.dtype is not BF else x
        for p in copies:
            y[p, :, :at] = y[int(shared[prefix // page]), :, :at]
    if spoil:  # what no sequence's key holds does not matter, nor the own pages' rows of the prefix, which are read from the shared ones
        used = used_rows(table, lens, page, pages)
        for i in range(-(-prefix // page)):
            used[int(shared[i])] = False
            used[int(shared[i]), :min(page, prefix - i * page)] = True
        c.spoil(used)
    return c, q, table, shared


def check(c, q, table, shared, prefix, lens, **kw):
    B, hq, d = q.shape
    o, lse, status = torch.full((B, hq, d), 9.0, device="cuda").to(BF), torch.full((B, hq), 9.0, device="cuda"), i32([0])
    dash.dash_attn_prefix_decode(q, *c.pools, table, i32(lens), shared, i32([prefix]), o, lse, status=status, **c.scales, **kw)
    assert int(status) == 0
    ro, rl, tol = attend64(c, q, table, lens, 1 / math.sqrt(d))
    over = ((o.double() - ro).abs() - tol - 8 * U24 * tol.clamp(min=ro.abs().amax())).max().item()
    assert over <= 0, over
    empty = i32(lens) == 0
    assert bool((o[empty] == 0).all()) and bool((lse[empty] == -math.inf).all())
    assert bool(((lse[~empty].double() - rl[~empty]).abs() <= 2e-5 * rl[~empty].abs().clamp(min=1)).all())
    again = dash.attn_prefix_decode(q, *c.pools, table, i32(lens), shared, i32([prefix]), **c.scales)
    assert torch.equal(o, again)
    return o, lse


# (d, hq, hkv, prefix, keys of each sequence in all, page, layout)
CASES = []
for d, page, order in ((64, 16, "phrd"), (128, 48, "prhd"), (256, 64, "hprd")):
    CASES += [
        (d, 4, 4, 300, [301, 300, 333, 700], page, order),
        (d, 8, 1, 1000, [1000 + 7 * i for i in range(20)], page, order),      # 160 rows: two tiles
        (d, 15, 3, 64 * 9, [64 * 9 + 1, 64 * 9, 5, 0, 64 * 9 - 1, 2000], page, order),  # shorter than the prefix, empty
        (d, 34, 2, 31, [31, 32, 40, 100], page, order),                       # a prefix inside one or two pages
        (d, 4, 2, 1, [1, 2, 20], page, order),
        (d, 4, 2, 0, [0, 5, 300], page, order),                               # nothing shared
    ]
CASES += [(128, 8, 2, 9001, [9001 + 13 * i for i in range(40)], 16, "phrd"), (256, 8, 1, 4999, [5000, 5400], 32, "phrd"),
          (64, 2, 1, 2048, [2048 - 100 * i for i in range(21)], 16, "phrd"), (128, 1, 1, 129, [130] * 130, 16, "phrd")]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("d,hq,hkv,prefix,lens,page,order", CASES)
def test_prefix(d, hq, hkv, prefix, lens, page, order, kind):
    check(*build(kind, d, hq, hkv, prefix, lens, page, order), prefix, lens)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("d", [64, 128, 256])
def test_scores_far_from_zero(d, kind):
    """Keys that score 2^25 and more above or below the others, in the prefix and behind it: the largest weighs exactly 1."""
    prefix, lens, page = 700, [800, 700, 90], 16
    for where in ("first", "last", "own"):
        c, q, table, shared = build(kind, d, 4, 2, prefix, lens, page, spoil=False)
        q = q.clone()
        at = {"first": 40, "last": 690, "own": 750}[where]
        # key 690 lies in the prefix's last page, which the sequences have copies of: the call reads the prefix's own
        p = [int(table[0, at // page])] + ([int(shared[at // page])] if at < prefix else [])
        if kind == "bf16":
            c.k[p, :, at % page, 0] = 3e8
            q[..., 0] = 1.0
        elif kind == "e4m3":
            c.k.view(torch.uint8)[p, :, at % page, 0] = 0x7C  # 384
            q[..., 0] = 2.0 ** 20
        else:
            c.k.view(torch.uint8)[p, :, at % page, 0] = 0x7C if kind == "mxfp8" else 0x07
            c.k_scale[p, :, at % page, 0] = 127 + 20
            q[..., 0] = 2.0 ** 6
        o, lse = torch.empty_like(q), torch.empty((3, 4), device="cuda")
        dash.dash_attn_prefix_decode(q, *c.pools, table, i32(lens), shared, i32([prefix]), o, lse, **c.scales)
        assert bool(o.isfinite().all()) and bool(lse.isfinite().all())
        sees = [n > at and (at < prefix or s == 0) for s, n in enumerate(lens)]
        v = c.all64()[1]
        for s in range(3):
            if sees[s] and kind != "e4m3":  # (2^20 times every key of column 0: no single key stands out there)
                want = v[int(table[s, at // page]), :, at % page].repeat_interleave(2, 0)
                assert bool(((o[s].double() - want).abs() <= 2.0 ** -8 * want.abs()).all())


def test_infinite_scores():
    """Keys that score -infinity take no weight; all of them: O = 0, L = -infinity."""
    d, prefix, lens, page = 128, 500, [600, 500, 40], 16
    c, q, table, shared = build("bf16", d, 4, 2, prefix, lens, page, spoil=False)
    q = q.clone()
    q[..., 0] = 1.0
    quiet = torch.zeros(c.k.shape[0], page, dtype=torch.bool, device="cuda")
    quiet[table[0, :6].long()] = True  # keys 0 .. 95
    c.k.transpose(1, 2)[quiet] = torch.cat((torch.full((1,), -math.inf), torch.zeros(d - 1))).to(BF).cuda()
    o, lse = torch.empty_like(q), torch.empty((3, 4), device="cuda")
    dash.dash_attn_prefix_decode(q, *c.pools, table, i32(lens), shared, i32([prefix]), o, lse)
    assert bool((o[2] == 0).all()) and bool((lse[2] == -math.inf).all())
    k64, v64 = c.all64()
    for s in (0, 1):
        j = torch.arange(96, lens[s], device="cuda")
        k, v = (x[table[s, j // page].long(), :, j % page].transpose(0, 1) for x in (k64, v64))
        qq = q[s].double().reshape(2, 2, d)
        sc = qq @ k.transpose(1, 2).contiguous() / math.sqrt(d)
        p = torch.softmax(sc, -1)
        off = (d + 4) * U24 * (qq.abs() @ k.abs().transpose(1, 2).contiguous()).amax() / math.sqrt(d)
        bound = 2.0 ** -8 * (p @ v).abs() + (2.0 ** -8 * (1 + 2.0 ** -8) + 2 * off + 2 * lens[s] * U24 + 24 * U24) * (p @ v.abs())
        assert bool(((o[s].double().reshape(2, 2, d) - p @ v).abs() <= bound).all())


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("d,hq,hkv,copies", [(64, 4, 2, 1), (128, 8, 1, 9), (256, 16, 1, 4)])  # few rows and many
def test_shared_keys_behind_a_shorter_sequence_do_not_reach_it(d, hq, hkv, copies, kind):
    """Sequences that end inside the prefix have their keys alone, whatever the prefix holds behind them."""
    prefix, page = 700, 16
    lens = [700, 50, 800, 49, 699, 0, 1] * copies
    c, q, table, shared = build(kind, d, hq, hkv, prefix, lens, page, spoil=False)
    want = dash.attn_prefix_decode(q, *c.pools, table, i32(lens), shared, i32([prefix]), **c.scales)
    for pool, scale in ((c.k, c.k_scale), (c.v, c.v_scale)):
        page_of, row = int(shared[50 // page]), 50 % page  # key 50
        if kind.startswith("mx"):
            scale[page_of, :, row] = 255
        elif kind == "e4m3":
            pool.view(torch.uint8)[page_of, :, row] = 0x7F
        else:
            pool[page_of, :, row] = float("nan")
    got = dash.attn_prefix_decode(q, *c.pools, table, i32(lens), shared, i32([prefix]), **c.scales)
    short = i32(lens) <= 50
    assert torch.equal(got[short], want[short]) and bool(got[~short].isnan().all())
    check(*build(kind, d, hq, hkv, prefix, lens, page), prefix, lens)


@pytest.mark.parametrize("kind", KINDS)
def test_as_without_a_shared_prefix(kind):
    """The same arguments give dash_attn_decode's result, both within their bounds."""
    prefix, lens, page, d = 2000, [2100, 2000, 2345, 2001], 16, 128
    c, q, table, shared = build(kind, d, 32, 8, prefix, lens, page)
    o, lse = check(c, q, table, shared, prefix, lens)
    # (with the sequences' own copies of the last page whole again)
    whole = prefix // page * page
    o2, lse2 = torch.empty_like(o), torch.empty_like(lse)
    dash.dash_attn_decode(q, *c.pools, table, i32(lens), o2, lse2, **c.scales)
    _, _, tol = attend64(c, q, table, lens, 1 / math.sqrt(d))
    assert whole == prefix
    assert bool(((o.double() - o2.double()).abs() <= 2.1 * tol).all())


def test_what_is_reported():
    prefix, lens, page = 100, [150, 120], 16
    c, q, table, shared = build("bf16", 64, 4, 2, prefix, lens, page)
    want = dash.attn_prefix_decode(q, *c.pools, table, i32(lens), shared, i32([prefix]))

    def run(table=table, lens=lens, shared=shared, prefix=prefix):
        status = i32([0])
        o = dash.attn_prefix_decode(q, *c.pools, table, i32(lens), shared, i32([prefix]), status=status)
        return int(status), o

    bad = shared.clone()
    bad[3] = 10 ** 6
    assert run(shared=bad)[0] == 1
    t = table.clone()
    t[0, 8] = -5
    code, o = run(table=t)
    assert code == 1 and torch.equal(o[1], want[1])
    t = table.clone()
    t[:, :prefix // page] = -7  # the shared pages' entries are not looked at
    code, o = run(table=t)
    assert code == 0 and torch.equal(o, want)
    for n in (-1, 16 * shared.numel() + 1):
        assert run(prefix=n)[0] == 1
    code, o = run(lens=[150, 10 ** 6])
    assert code == 1 and torch.equal(o[0], want[0])


def test_refusals():
    c, q, table, shared = build("bf16", 64, 4, 2, 100, [150, 120], 16)
    lens, n = i32([150, 120]), i32([100])
    for word, args in (("prefix_table", (q, *c.pools, table, lens, shared[None], n)), ("prefix_table", (q, *c.pools, table, lens, shared.long(), n)),
                       ("prefix_len", (q, *c.pools, table, lens, shared, i32([100, 100]))), ("prefix_len", (q, *c.pools, table, lens, shared, n.float())),
                       ("lens", (q[:1], *c.pools, table, lens, shared, n)), ("prefix_table", (q, *c.pools, table, lens, shared.cpu(), n))):
        with pytest.raises(dash.DashError, match=word):
            dash.attn_prefix_decode(*args)
    with pytest.raises(dash.DashError, match="workspace"):
        dash.attn_prefix_decode(q, *c.pools, table, lens, shared, n, workspace=torch.empty(512, dtype=torch.uint8, device="cuda"))


@pytest.mark.parametrize("kind", KINDS)
def test_answers_to_one_prompt(kind):
    """A prompt is stored once, eight answers go on from it, a token at a time: rotation, append, shared-prefix attention, eagerly
    and from two graphs that are replayed in turn on one workspace, a padded slot (length 0) among them; every
    step against float64, all the same bits.  One prefix ends inside a page."""
    d, hq, hkv, page, prefix, steps = 128, 8, 2, 16, 203, 4
    B = 9
    lens = [prefix + i for i in range(B - 1)] + [0]
    table, pages, shared, copies = tables(prefix, [n + steps if n else 0 for n in lens], page)
    g = torch.Generator(device="cuda")
    g.manual_seed(5)
    inv, amp = dash.dash_rotary_frequencies(d, scaling="parts", factor=4.0, original=64.0)
    inv = torch.from_numpy(inv).cuda()
    base = Cache(kind, pages, hkv, page, d, seed=2)
    # the prompt through the cache's own call, into the shared pages, and the last one's rows into each copy
    k, v = (torch.randn((prefix, hkv, d), generator=g, device="cuda").to(BF) for _ in range(2))
    for t in [shared[None]] + [torch.cat((shared[:prefix // page], i32([p])))[None] for p in copies]:
        dash.dash_kv_append(k, v, *base.pools, t.contiguous(), i32([0]), cu=i32([0, prefix]), inv_freq=inv, **base.scales)
    new = [[torch.randn((B, h, d), generator=g, device="cuda").to(BF) for h in (hq, hkv, hkv)] for _ in range(steps)]
    ws = torch.empty(dash.dash_prefix_decode_workspace_size(B, hq, hkv, d, page, table.shape[1], shared.numel()), dtype=torch.uint8, device="cuda")
    length = i32([prefix])
    grow = i32([1 if n else 0 for n in lens])

    def buffers():
        c = Cache(kind, pages, hkv, page, d, seed=2)
        for x, y in zip((*c.pools, c.k_scale, c.v_scale), (*base.pools, base.k_scale, base.v_scale)):
            if x is not None:
                x.copy_(y)
        return c, i32(lens), [torch.empty((B, h, d), device="cuda", dtype=BF) for h in (hq, hkv, hkv, hq, hq)]

    def step(b):
        c, n, (q, k, v, qr, o) = b
        dash.dash_kv_append(k, v, *c.pools, table, n, q=q, q_out=qr, inv_freq=inv, **c.scales)  # (the padded slot has no page)
        n += grow
        dash.dash_attn_prefix_decode(qr, *c.pools, table, n, shared, length, o, scale=amp * amp / math.sqrt(d), workspace=ws, **c.scales)

    def feed(b, t):
        for x, y in zip(b[2], new[t]):
            x.copy_(y)

    eager, outs = buffers(), []
    for t in range(steps):
        feed(eager, t)
        step(eager)
        outs.append(eager[2][4].clone())
        ro, _, tol = attend64(eager[0], eager[2][3], table, [n + t + 1 if n else 0 for n in lens], amp * amp / math.sqrt(d))
        assert bool(((outs[-1].double() - ro).abs() <= tol + 8 * U24 * ro.abs().amax()).all())
    graphs = []
    for _ in range(2):
        b = buffers()
        feed(b, 0)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step(b)
        graphs.append((graph, b))
    for t in range(steps):
        for graph, b in graphs:
            feed(b, t)
            graph.replay()
            dash.attn_prefix_decode(torch.ones_like(b[2][0]), *b[0].pools, table, b[1], shared, length, workspace=ws, **b[0].scales)
            torch.cuda.synchronize()
            assert torch.equal(b[2][4], outs[t])


def test_two_streams_and_a_later_length():
    prefix, lens, page = 1500, [1600, 1500, 1777], 16
    c, q, table, shared = build("bf16", 128, 8, 2, prefix, lens, page, spoil=False)
    n = dash.dash_prefix_decode_workspace_size(3, 8, 2, 128, page, table.shape[1], shared.numel())
    lens, length = i32(lens), i32([prefix])
    want = dash.attn_prefix_decode(q, *c.pools, table, lens, shared, length)
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = [[torch.zeros_like(want) for _ in range(6)] for _ in streams]
    spaces = [torch.empty(n, dtype=torch.uint8, device="cuda") for _ in streams]
    torch.cuda.synchronize()
    for i in range(6):
        for s, ws, o in zip(streams, spaces, outs):
            dash.dash_attn_prefix_decode(q, *c.pools, table, lens, shared, length, o[i], workspace=ws, stream=s)
    torch.cuda.synchronize()
    assert all(torch.equal(x, want) for o in outs for x in o)
    with pytest.raises(dash.DashError):
        dash.dash_attn_prefix_decode(q, *c.pools, table, lens, shared, length, outs[0][0], stream=streams[0])
    # a captured call follows the prefix's length
    o = torch.empty_like(want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        dash.dash_attn_prefix_decode(q, *c.pools, table, lens, shared, length, o, workspace=spaces[0])
    for m in (1500, 16, 0, 1488, 700):
        length.fill_(m)
        o.fill_(3.0)
        graph.replay()
        want = dash.attn_prefix_decode(q, *c.pools, table, lens, shared, length)
        torch.cuda.synchronize()
        assert torch.equal(o, want)
        ro, _, tol = attend64(c, q, table, lens.tolist(), 1 / math.sqrt(128))
        assert bool(((o.double() - ro).abs() <= tol + 8 * U24 * ro.abs().amax()).all())


def test_prefix_at_the_far_end_of_a_large_cache():
    """Pages past 2^32 bytes of the pool."""
    d, page, pages = 256, 65536, 132
    kc, vc = (torch.zeros((pages, 1, page, d), dtype=BF, device="cuda") for _ in range(2))
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    prefix, own = 1000, 300
    for c in (kc, vc):
        c[131, 0, :prefix] = torch.randn((prefix, d), generator=g, device="cuda").to(BF)
        for s in (129, 130):
            c[s, 0, :prefix] = c[131, 0, :prefix]
            c[s, 0, prefix:prefix + own] = torch.randn((own, d), generator=g, device="cuda").to(BF)
    q = torch.randn((2, 4, d), generator=g, device="cuda").to(BF)
    o = dash.attn_prefix_decode(q, kc, vc, i32([[129], [130]]), i32([prefix + own, prefix + 7]), i32([131]), i32([prefix]))
    for s, n in ((0, prefix + own), (1, prefix + 7)):
        k, v = (c[129 + s, 0, :n].double() for c in (kc, vc))
        p = torch.softmax((q[s].double() @ k.t().contiguous()) / 16, -1)
        a = p @ v.abs()
        off = (d + 4) * U24 * (q[s].double().abs() @ k.abs().t().contiguous()).amax() / 16
        tol = 2.0 ** -8 * (p @ v).abs() + (2.0 ** -8 * (1 + 2.0 ** -8) + 2 * off + 2 * n * U24 + 24 * U24) * a
        assert bool(((o[s].double() - p @ v).abs() <= tol).all())


@pytest.mark.parametrize("prefix,wide", [(704, 16.0), (701, 1.0)])
@pytest.mark.parametrize("d,copies", [(64, 1), (64, 3), (128, 1), (128, 3), (256, 1), (256, 6)])  # few rows and many
def test_scales_of_any_sign(d, copies, prefix, wide):
    """An e4m3 head whose keys' scale is negative, or 0 (every key of it scores 0), by either kernel, to the bounds of `check`, which
    take the scale by its absolute value; and the same call without the shared prefix."""
    hq, hkv, page = 16, 4, 16
    lens = [prefix, 50, 800, prefix + 2, 699, 0] * copies
    c, q, table, shared = build("e4m3", d, hq, hkv, prefix, lens, page)
    q = q * wide
    c.k_scale = torch.tensor([0.5, 0.0, -0.7, -0.0], device="cuda")
    c.v_scale = torch.tensor([-0.5, 0.6, 0.0, 0.8], device="cuda")
    o, lse = check(c, q, table, shared, prefix, lens)
    if prefix % page == 0:  # (the sequences' own copies of the last page are whole)
        o2, lse2 = torch.empty_like(o), torch.empty_like(lse)
        dash.dash_attn_decode(q, *c.pools, table, i32(lens), o2, lse2, **c.scales)
        _, _, tol = attend64(c, q, table, lens, 1 / math.sqrt(d))
        assert bool(((o.double() - o2.double()).abs() <= 2.1 * tol).all())


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("d,copies", [(64, 1), (128, 5), (256, 13)])  # few rows and many
def test_a_sequence_that_ends_with_the_prefix_needs_no_page(d, copies, kind):
    """Without keys of its own, a sequence has no page of its own either: its entries are not looked at, and nothing is reported."""
    prefix, page = 701, 16
    lens = [prefix, prefix + 1, prefix] * copies
    c, q, table, shared = build(kind, d, 16, 2, prefix, lens, page)
    want, lse = check(c, q, table, shared, prefix, lens)
    t = table.clone()
    t[i32(lens) == prefix] = -1
    status, o = i32([0]), torch.empty_like(want)
    dash.dash_attn_prefix_decode(q, *c.pools, t, i32(lens), shared, i32([prefix]), o, status=status, **c.scales)
    assert int(status) == 0 and torch.equal(o, want)
    alone = i32([prefix] * len(lens))  # nobody has a key of their own
    dash.dash_attn_prefix_decode(q, *c.pools, torch.full_like(t, -1), alone, shared, i32([prefix]), o, status=status, **c.scales)
    assert int(status) == 0
    ends = i32(lens) == prefix
    _, _, tol = attend64(c, q, table, lens, 1 / math.sqrt(d))
    assert bool(((o[ends].double() - want[ends].double()).abs() <= 2.1 * tol[ends]).all())


def first_block(c, rows, code, exponent=0):
    """Keys `rows` (truth values [pages, page]) get `code` in component 0 and, in a microscaled cache, 0 in the others of its
    block and the scale 2^exponent.  A code is a value (bf16) or an element's bits, of a tensor [heads, 1] or one for all."""
    k = (c.k if c.kind == "bf16" else c.k.view(torch.uint8)).transpose(1, 2)
    x = k[rows]
    x[..., 0] = code
    if c.kind.startswith("mx"):
        x[..., 1:32 if c.kind == "mxfp8" else 16] = 0
        s = c.k_scale.transpose(1, 2)
        y = s[rows]
        y[..., 0] = 127 + exponent
        s[rows] = y
    k[rows] = x


def rows_of_keys(table, shared, lens, prefix, keys, pages, page):
    """The cached rows of these keys of the prefix: the shared ones, and those of sequences' own copies."""
    r = torch.zeros((pages, page), dtype=torch.bool, device="cuda")
    for j in keys:
        r[int(shared[j // page]), j % page] = True
        for s, n in enumerate(lens):
            if n > j:
                r[int(table[s, j // page]), j % page] = True
    return r


# many rows: what the forward's pipelined loop leaves to its careful one, on rows that lie in pages
FAR = [(64, 6, 16, "phrd"), (128, 6, 48, "prhd"), (256, 14, 64, "hprd")]


@pytest.mark.parametrize("kind", KINDS + ["e4m3-"])
@pytest.mark.parametrize("prefix", [701, 640])
@pytest.mark.parametrize("d,copies,page,order", FAR)
def test_runs_that_begin_with_infinite_scores(d, copies, page, order, prefix, kind):
    """Of every 128 shared keys the first 32 score -infinity (overflowing, or an infinity in K), so that every run's rows are done
    again by the careful loop, on ordinary scores and all components.  Bounds of `check`; "-": scales of both signs."""
    lens = [prefix, 50, 800, 20, 1500] * copies
    c, q, table, shared = build(kind[:-1] if kind == "e4m3-" else kind, d, 8, 2, prefix, lens, page, order)
    if kind == "e4m3-":
        c.k_scale = torch.tensor([-0.7, 0.4], device="cuda")
    pages = c.k.shape[0]
    quiet = [j for j in range(prefix) if j % 128 < 32]
    live = ~(c.k.double().isnan() if kind == "bf16" else c.k.view(torch.uint8) == 0x7F).all(-1).all(1)
    if kind.startswith("mx"):
        live = (c.k_scale != 255).all(-1).all(1)
    k = (c.k if kind == "bf16" else c.k.view(torch.uint8)).transpose(1, 2)
    x = k[live]
    x[..., 0] = 0
    k[live] = x
    least = {"bf16": -math.inf, "mxfp8": 0xFE, "mxfp4": 0x0F}.get(kind)
    if least is None:  # e4m3: -448 times the scale's sign
        least = torch.where(c.k_scale > 0, 0xFE, 0x7E).to(torch.uint8)
    first_block(c, rows_of_keys(table, shared, lens, prefix, quiet, pages, page), least, 100)
    q = q.clone()
    q[..., 0] = {"bf16": 1.0, "mxfp8": 2.0 ** 100, "mxfp4": 2.0 ** 100}.get(kind, 2.0 ** 127)
    B, hq, _ = q.shape
    o, lse, status = torch.full((B, hq, d), 9.0, device="cuda").to(BF), torch.full((B, hq), 9.0, device="cuda"), i32([0])
    dash.dash_attn_prefix_decode(q, *c.pools, table, i32(lens), shared, i32([prefix]), o, lse, status=status, **c.scales)
    assert int(status) == 0
    k_all, v_all = c.all64()
    for s, n in enumerate(lens):
        j = torch.tensor([i for i in range(n) if i >= prefix or i % 128 >= 32], device="cuda", dtype=torch.long)
        if len(j) == 0:
            assert bool((o[s] == 0).all()) and bool((lse[s] == -math.inf).all())
            continue
        k, v = (x[table[s, j // page].long(), :, j % page].transpose(0, 1) for x in (k_all, v_all))
        qq = q[s].double().reshape(2, hq // 2, d)
        qq[..., 0] = 0
        sc = qq @ k.transpose(1, 2).contiguous() / math.sqrt(d)
        p = torch.softmax(sc, -1)
        a, oo = p @ v.abs(), p @ v
        off = (d + 4) * U24 / math.sqrt(d) * (qq.abs() @ k.abs().transpose(1, 2).contiguous()).amax(-1, keepdim=True)
        tol = 2.0 ** -8 * oo.abs() + (2.0 ** -8 * (1 + 2.0 ** -8) + 2 * off + 2 * n * U24 + 16 * U24) * a
        tol = tol + 8 * U24 * tol.clamp(min=oo.abs().amax())
        assert bool(((o[s].double().reshape(2, hq // 2, d) - oo).abs() <= tol).all()), (s, n)
        ref = torch.logsumexp(sc, -1).reshape(hq)
        assert bool(((lse[s].double() - ref).abs() <= 2e-5 * ref.abs().clamp(min=1)).all()), (s, n)
    assert torch.equal(o, dash.attn_prefix_decode(q, *c.pools, table, i32(lens), shared, i32([prefix]), **c.scales))


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("d,copies,page,order", FAR)
def test_many_rows_with_scores_far_from_zero(d, copies, page, order, kind):
    """One key far above all others, in a run's first unit, its last, partial one or behind the prefix: it weighs exactly 1, so that O
    is its V, rounded.  And all keys alike and far below 0: O is the mean of V, by P of exactly 1 and sums in fp32."""
    prefix, lens = 701, [701, 50, 800, 1500] * copies
    one = {"bf16": 1.0, "e4m3": 0x38, "mxfp8": 0x38, "mxfp4": 0x02}[kind]

    def run(key, q0):
        c, q, table, shared = build(kind, d, 8, 2, prefix, lens, page, order, spoil=False)
        everywhere = torch.ones(c.k.shape[0], page, dtype=torch.bool, device="cuda")
        first_block(c, everywhere, one if key is None else 0)
        if key is not None:
            first_block(c, rows_of_keys(table, shared, lens, prefix, [key], c.k.shape[0], page) if key < prefix else
                        used_key(table, lens, key, c.k.shape[0], page), one)
        q = torch.zeros_like(q) if key is None else q.clone()
        q[..., 0] = q0
        o, lse = torch.empty_like(q), torch.empty(q.shape[:2], device="cuda")
        dash.dash_attn_prefix_decode(q, *c.pools, table, i32(lens), shared, i32([prefix]), o, lse, **c.scales)
        return c, table, o, lse

    for key in (0, 31, 385, 700, 750):
        c, table, o, lse = run(key, 2.0 ** 30)
        v = c.all64()[1]
        for s, n in enumerate(lens):
            if n > key:
                want = v[int(table[s, key // page]), :, key % page].repeat_interleave(4, 0)
                assert bool(((o[s].double() - want).abs() <= 2.0 ** -8 * want.abs()).all()), (key, s)
            assert bool(o[s].isfinite().all()) and bool(lse[s].isfinite().all())
    c, table, o, lse = run(None, -2.0 ** 26)
    ks = c.k_scale.double() if kind == "e4m3" else torch.ones(2, dtype=torch.float64, device="cuda")
    for s, n in enumerate(lens):
        _, v = c.rows64(table, s, n)
        want, a = (x.repeat_interleave(4, 0) for x in (v.mean(1), v.abs().mean(1)))
        assert bool(((o[s].double() - want).abs() <= 2.0 ** -8 * want.abs() + (2 * n + 24) * U24 * a).all()), s
        ref = (-2.0 ** 26 / math.sqrt(d) * ks).repeat_interleave(4) + math.log(n)
        assert bool(((lse[s].double() - ref).abs() <= 8 * U24 * ref.abs()).all()), s


def used_key(table, lens, key, pages, page):
    """The cached row of one key behind the prefix, in every sequence that has it."""
    r = torch.zeros((pages, page), dtype=torch.bool, device="cuda")
    for s, n in enumerate(lens):
        if n > key:
            r[int(table[s, key // page]), key % page] = True
    return r
