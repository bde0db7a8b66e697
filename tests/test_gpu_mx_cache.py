"""Microscaled caches on the GPU: written, read back, attended to, against their definition in float64.

What is stored is compared for equality: the element nearest to value / 2^e (ties to even), where the value
is bf16 (V) or the rotated key, which the kernel computes in 64 bits and rounds to fp32 as the reference does.  (Two
computations in 64 bits differ by 2^-36 at most at these places, and would have to fall on two sides of a rounding to fp32 that
in turn is a tie of the element type: a chance of 10^-10 for each value.)

A rotated query is computed in 32 bits: beside its own rounding, u8 |y|, sine and cosine are rounded to fp32 (u24 each), and the two
products and their sum are (3 u24 of |x| + |y| at most): within 8 u24 (|x| + |y|), the bound of a query beside a bf16 cache.

The attention's bounds are those of the bf16 cache: the stored values are bf16 numbers, so u8 |o| for o's rounding, u8 A for P's
(A = sum_j P_j |v_j|), each score off by (d + 4) u24 times its sum of absolute products, sums over n keys n u24 A twice.
"""
import math

import pytest
import torch

from mx_util import BF, E4, Cache, pack, quantise64, used_rows, values64
from paper_2601_21824_amd import binding as dash
from test_gpu_paged_cache import LENS, i32, pair_size, rotate64, table_of

pytestmark = pytest.mark.gpu

U8, U24 = 2.0 ** -8, 2.0 ** -24
KINDS = ["bf16", "e4m3", "mxfp8", "mxfp4"]
MX = KINDS[2:]


def cat_places(old, new):
    return torch.cat([torch.arange(o, o + n) for o, n in zip(old, new)]).cuda()


def offsets(lens, first=0):
    at = [first]
    for n in lens:
        at.append(at[-1] + n)
    return at


# (d, hq, hkv, new tokens per sequence, lengths before, page, rotary, interleaved, layout)
APPENDS = [
    (128, 8, 2, [1, 1, 1], [0, 15, 16], 16, 128, False, "phrd"),
    (64, 4, 4, [5, 0, 40, 1], [3, 7, 0, 100], 16, 32, True, "prhd"),
    (64, 5, 1, [17, 33], [0, 47], 48, 64, True, "hprd"),
    (256, 6, 3, [9, 70], [131071, 2], 64, 256, False, "phrd"),
    (256, 2, 1, [9, 70], [131071, 2], 64, 208, True, "prhd"),
    (256, 3, 1, [3, 1], [7, 2], 16, 176, False, "phrd"),  # blocks of 32 across the halves and the rest
    (128, 32, 8, [700, 0, 1, 333], [0, 5, 99, 64], 32, 96, False, "phrd"),
    (128, 3, 3, [300, 600], [0, 0], 16, 0, False, "phrd"),  # no rotation
    (64, 2, 2, [9, 4], [3, 40], 16, 48, False, "phrd"),
]


@pytest.mark.parametrize("kind", MX)
@pytest.mark.parametrize("with_q", [True, False])
@pytest.mark.parametrize("d,hq,hkv,new,old,page,rotary,interleaved,order", APPENDS)
def test_append_and_read(d, hq, hkv, new, old, page, rotary, interleaved, order, with_q, kind):
    g = torch.Generator(device="cuda")
    g.manual_seed(d + hq)
    head, T = 2, sum(new)
    fused = torch.randn((T + head + 3, hq + 2 * hkv, d), generator=g, device="cuda")
    fused *= 2.0 ** torch.randint(-9, 9, (T + head + 3, hq + 2 * hkv, d // 32, 1), generator=g, device="cuda").expand(-1, -1, -1, 32).flatten(-2)
    q, k, v = fused.to(BF).split([hq, hkv, hkv], dim=1)
    table, pages = table_of([a + b for a, b in zip(old, new)], page)
    c = Cache(kind, pages, hkv, page, d, order, seed=1)
    before = [x.clone() for x in (*c.pools, c.k_scale, c.v_scale)]
    inv = (10000.0 ** (-torch.arange(0, rotary, 2, device="cuda") / rotary)).float() if rotary else None
    q_out, k_out, status = torch.full_like(q, 7.0), torch.full_like(k, 7.0), i32([0])
    kw = dict(q=q, q_out=q_out) if with_q else {}
    cu = i32(offsets(new, head))
    dash.dash_kv_append(k, v, *c.pools, table, i32(old), cu=cu, k_out=k_out, inv_freq=inv, interleaved=interleaved, status=status, **c.scales, **kw)
    assert int(status) == 0
    own, place = slice(head, head + T), cat_places(old, new)
    for x, out in ((q, q_out), (k, k_out))[0 if with_q else 1:]:
        ref = rotate64(x[own], place, inv, interleaved)
        tol = U8 * ref.abs() * (1 + U8) + (8 * U24 * pair_size(x[own], inv, interleaved) if x is q else 0.0)
        assert bool(((out[own].double() - ref).abs() <= tol).all())
        assert bool((out[:head] == 7).all()) and bool((out[head + T:] == 7).all())
    seq = torch.cat([torch.full((n,), s) for s, n in enumerate(new)]).cuda()
    ids, rows = table[seq, place // page].long(), place % page
    stored = []
    for x, pool, scale in ((rotate64(k[own], place, inv, interleaved).float(), c.k, c.k_scale), (v[own].float(), c.v, c.v_scale)):
        code, byte, _ = quantise64(x, kind)
        want = pack(code, kind)
        assert torch.equal(scale[ids, :, rows], byte)
        assert torch.equal(pool.view(torch.uint8)[ids, :, rows], want.view(torch.uint8))
        stored.append(values64(want, byte, kind))
    # nothing else moved
    for x, x0 in zip((*c.pools, c.k_scale, c.v_scale), before):
        keep = torch.ones(pages, page, dtype=torch.bool, device="cuda")
        keep[ids, rows] = False
        assert torch.equal(x.view(torch.uint8).transpose(1, 2)[keep], x0.view(torch.uint8).transpose(1, 2)[keep])
    # read back: what is stored, exactly
    after = i32([a + b for a, b in zip(old, new)])
    kr, vr = torch.full_like(k, 7.0), torch.full_like(v, 7.0)
    dash.dash_kv_read(*c.pools, table, after, cu, kr, vr, first=i32(old), status=status, **c.scales)
    assert int(status) == 0
    for out, want in ((kr, stored[0]), (vr, stored[1])):
        assert torch.equal(out[own].double(), want)
        assert bool((out[:head] == 7).all()) and bool((out[head + T:] == 7).all())


@pytest.mark.parametrize("kind", MX)
def test_blocks_at_the_ends_of_the_range(kind):
    """Zeros, the least and largest bf16 values, borders of scale and element, NaN and infinities."""
    top, inf, nan = float(torch.finfo(BF).max), math.inf, math.nan
    most = 448.0 if kind == "mxfp8" else 6.0
    rows = []
    for fill in ([0.0, -0.0], [top, -top], [1.5 * 2.0 ** 127, 2.0 ** 126], [2.0 ** -133, -2.0 ** -126], [2.0 ** -117, 2.0 ** -120],
                 [most, 1.0], [most * 2.0 ** -40, -most * 2.0 ** -41], [inf, 1.0], [-inf, 1.0], [nan, 1.0], [nan, inf]):
        rows.append((fill * 16)[:32])
    for m in (255 / 128, 7 / 4, 225 / 128, 3 / 2, 193 / 128, 1.0):  # fractions at which the exponent steps
        rows.append([m * 2.0 ** 5] + [(i / 16) * (-1) ** i for i in range(31)])
    ties = [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0] if kind == "mxfp4" else [17.0, 19.0, 25.0, 1.0625, 1.1875, 2.0 ** -10, 3 * 2.0 ** -10]
    rows.append([most] + [x * s for x in ties for s in (1, -1)] + [0.0] * (31 - 2 * len(ties)))
    x = torch.tensor(rows, device="cuda").to(BF)
    x = torch.cat((x, x.roll(1, 0)), 1)  # two blocks a row
    n = x.shape[0]
    k, v = x[:, None], x.flip(0)[:, None]
    c = Cache(kind, n, 1, 16, 64)
    table, old = torch.arange(n, dtype=torch.int32, device="cuda")[:, None], i32([3] * n)
    dash.dash_kv_append(k, v, *c.pools, table, old, **c.scales)
    kr, vr = dash.kv_read(*c.pools, table, i32([4] * n), i32(list(range(n + 1))), n, first=old, **c.scales)
    for src, pool, scale, out in ((k, c.k, c.k_scale, kr), (v, c.v, c.v_scale, vr)):
        code, byte, odd = quantise64(src.float(), kind)
        assert torch.equal(scale[:, :, 3], byte)
        plain = ~odd.repeat_interleave(32, -1)
        got = values64(pool[:, :, 3], scale[:, :, 3], kind)
        want = values64(pack(code, kind), byte, kind)
        assert torch.equal(got[plain], want[plain]) and bool(got[~plain].isnan().all())
        assert torch.equal(out.double()[plain], want[plain]) and bool(out[~plain].isnan().all())
        assert bool(out[plain].isfinite().all())


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("d,hkv,page,order", [(64, 3, 16, "phrd"), (128, 8, 48, "prhd"), (256, 1, 64, "hprd")])
def test_read(d, hkv, page, order, kind):
    """Any rows of any sequences, with gaps between and around them; keys that are not there are reported and left alone."""
    lens = [1, 0, 333, 16, 47, 130]
    table, pages = table_of(lens, page)
    c = Cache(kind, pages, hkv, page, d, order)
    k64, v64 = c.all64()
    first, n = [0, 0, 300, 3, 0, 129], [1, 0, 33, 13, 47, 1]
    at, rows = [5], 5
    for x in n:
        at.append(at[-1] + x)
    rows = at[-1] + 4
    k, v = (torch.full((rows, hkv + 1, d), 7.0, device="cuda").to(BF)[:, 1:] for _ in range(2))  # strided
    status = i32([0])
    dash.dash_kv_read(*c.pools, table, i32(lens), i32(at), k, v, first=i32(first), status=status, **c.scales)
    assert int(status) == 0
    for out, pool in ((k, k64), (v, v64)):
        for s, (f, m) in enumerate(zip(first, n)):
            j = torch.arange(f, f + m, device="cuda")
            want = pool[table[s, j // page].long(), :, j % page]
            got = out[at[s]:at[s + 1]].double()
            if kind == "e4m3":  # one product in fp32 and one rounding to bf16
                assert bool(((got - want).abs() <= (U8 + 2 * U24) * want.abs()).all())
            else:
                assert torch.equal(got, want)
        assert bool((out[:5] == 7).all()) and bool((out[at[-1]:] == 7).all())
    only = torch.full_like(v, 7.0)
    dash.dash_kv_read(*c.pools, table, i32(lens), i32(at), None, only, first=i32(first), **c.scales)
    assert torch.equal(only, v)
    # beyond a length, before the first key, no page, offsets that do not rise
    for kw in (dict(first=[0, 0, 301, 3, 0, 129]), dict(first=[-1, 0, 300, 3, 0, 129]), dict(at=[5, 6, 6, 5, 52, 99, 100])):
        a = i32(kw.get("at", at))
        k2 = torch.full_like(k, 7.0)
        status = i32([0])
        dash.dash_kv_read(*c.pools, table, i32(lens), a, k2, None, first=i32(kw.get("first", first)), status=status, **c.scales)
        assert int(status) == 1
        if "first" in kw and kw["first"][0] == 0:
            assert bool((k2[at[3] - 1] == 7).all()) and torch.equal(k2[at[3]:at[4]], k[at[3]:at[4]])
    t2 = table.clone()
    t2[4, 0] = pages
    k2, status = torch.full_like(k, 7.0), i32([0])
    dash.dash_kv_read(*c.pools, t2, i32(lens), i32(at), k2, None, first=i32(first), status=status, **c.scales)
    assert int(status) == 1 and bool((k2[at[4]:at[4] + min(page, 47)] == 7).all()) and torch.equal(k2[:at[4]], k[:at[4]])
    assert dash.kv_read(*c.pools, table, i32(lens), i32([0] * 7), 0, **c.scales)[0].shape == (0, hkv, d)


def attend64(c, q, table, lens, scale):
    """o, lse and the bound on o's error, in float64."""
    B, hq, d = q.shape
    hkv = c.k.shape[1]
    o, tol = (torch.zeros((B, hq, d), dtype=torch.float64, device="cuda") for _ in range(2))
    lse = torch.full((B, hq), -math.inf, dtype=torch.float64, device="cuda")
    k_all, v_all = c.all64()
    for s, n in enumerate(lens):
        if n == 0:
            continue
        ids = table[s, :-(-n // c.page)].long()
        k, v = (x[ids].transpose(0, 1).flatten(1, 2)[:, :n] for x in (k_all, v_all))
        qq = q[s].double().reshape(hkv, hq // hkv, d)
        sc = qq @ k.transpose(1, 2).contiguous() * scale
        p = torch.softmax(sc, -1)
        a = p @ v.abs()
        off = (d + 4) * U24 * scale * (qq.abs() @ k.abs().transpose(1, 2).contiguous()).amax(-1, keepdim=True)
        oo = p @ v
        o[s], lse[s] = oo.reshape(hq, d), torch.logsumexp(sc, -1).reshape(hq)
        tol[s] = (U8 * oo.abs() + (U8 * (1 + U8) + 2 * off + 2 * n * U24 + 16 * U24) * a).reshape(hq, d)
    return o, lse, tol


DECODES = [(d, hq, hkv, LENS, page, order) for d, page, order in ((64, 16, "phrd"), (128, 48, "prhd"), (256, 64, "hprd"))
           for hq, hkv in ((4, 4), (8, 1), (15, 3), (34, 2))]
DECODES += [(128, 8, 2, [20000], 16, "phrd"), (64, 64, 1, [9000, 1], 16, "phrd"), (256, 4, 4, [7001, 40, 3000], 32, "phrd"),
            (128, 4, 1, [1 + 37 * i % 211 for i in range(150)], 16, "phrd"),
            # more than two rounds of 64 sequences in several chunks each, whole ones only among them, and empty sequences
            (64, 4, 2, [128 * (i % 11) if i % 3 == 0 else 37 * i * i % 1500 for i in range(150)], 16, "phrd"),
            # more than 64 * 64 sequences
            (64, 4, 1, [1 + i % 3 if i % 400 else 1200 + i // 10 for i in range(4101)], 16, "phrd")]


@pytest.mark.parametrize("kind", MX)
@pytest.mark.parametrize("d,hq,hkv,lens,page,order", DECODES)
def test_decode(d, hq, hkv, lens, page, order, kind):
    g = torch.Generator(device="cuda")
    g.manual_seed(d + hq)
    q = torch.randn((len(lens), hq + 1, d), generator=g, device="cuda").to(BF)[:, 1:] * 2
    table, pages = table_of(lens, page)
    c = Cache(kind, pages, hkv, page, d, order)
    c.spoil(used_rows(table, lens, page, pages))  # what lies behind a sequence's last key does not matter
    o, lse, status = torch.full((len(lens), hq, d), 9.0, device="cuda").to(BF), torch.full((len(lens), hq), 9.0, device="cuda"), i32([0])
    dash.dash_attn_decode(q, *c.pools, table, i32(lens), o, lse, status=status, **c.scales)
    assert int(status) == 0
    ro, rl, tol = attend64(c, q, table, lens, 1 / math.sqrt(d))
    over = ((o.double() - ro).abs() - tol).max().item()
    assert over <= 0, over
    empty = i32(lens) == 0
    assert bool((o[empty] == 0).all()) and bool((lse[empty] == -math.inf).all())
    assert bool(((lse[~empty].double() - rl[~empty]).abs() <= 2e-5 * rl[~empty].abs().clamp(min=1)).all())
    assert torch.equal(o, dash.attn_decode(q, *c.pools, table, i32(lens), **c.scales))


@pytest.mark.parametrize("kind", MX)
def test_a_block_of_nan_reaches_its_own_sequence_alone(kind):
    lens, page, d = [40, 50, 60], 16, 128
    table, pages = table_of(lens, page)
    c = Cache(kind, pages, 2, page, d)
    q = torch.ones((3, 4, d), device="cuda").to(BF)
    want = dash.attn_decode(q, *c.pools, table, i32(lens), **c.scales)
    c.v_scale[int(table[1, 2]), 1, 3, 2] = 255  # columns 64 .. 95 of key 35, K/V head 1
    got = dash.attn_decode(q, *c.pools, table, i32(lens), **c.scales)
    hurt = torch.zeros_like(got, dtype=torch.bool)
    hurt[1, 2:, 64:96] = True
    assert bool(got[hurt].isnan().all()) and torch.equal(got[~hurt], want[~hurt])
    c.k_scale[int(table[0, 0]), 0, 3, 0] = 255
    got = dash.attn_decode(q, *c.pools, table, i32(lens), **c.scales)
    assert bool(got[0, :2].isnan().all()) and torch.equal(got[0, 2:], want[0, 2:]) and torch.equal(got[2], want[2])


@pytest.mark.parametrize("kind", MX)
def test_cache_beyond_32_bit_offsets(kind):
    """Pages at the far end of pools of over 4 GiB (MXFP4: 2^33 components)."""
    d, page = 256, 65536
    width = d if kind == "mxfp8" else d // 2
    pages = 4 * 2 ** 30 // (page * width) + 2
    kc, vc = (torch.zeros((pages, 1, page, width), dtype=torch.uint8, device="cuda") for _ in range(2))
    ks, vs = (torch.full((pages, 1, page, d // 32), 127, dtype=torch.uint8, device="cuda") for _ in range(2))
    if kind == "mxfp8":
        kc, vc = kc.view(E4), vc.view(E4)
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    q, k, v = (torch.randn((700, h, d), generator=g, device="cuda").to(BF) for h in (2, 1, 1))
    table, old = i32([[pages - 1, pages - 2]]), 65536 - 300
    dash.dash_kv_append(k, v, kc, vc, table, i32([old]), cu=i32([0, 700]), k_scale=ks, v_scale=vs)
    kr, vr = dash.kv_read(kc, vc, table, i32([old + 700]), i32([0, 700]), 700, first=i32([old]), k_scale=ks, v_scale=vs)
    for x, out in ((k, kr), (v, vr)):
        code, byte, _ = quantise64(x.float(), kind)
        assert torch.equal(out.double(), values64(pack(code, kind), byte, kind))
    o = dash.attn_decode(q[:1], kc, vc, table, i32([old + 700]), k_scale=ks, v_scale=vs)
    # the other keys are zeros: score 0, value 0
    s = (q[:1].double().transpose(0, 1) @ kr.double().permute(1, 2, 0).contiguous()) / 16
    top = s.amax(-1, keepdim=True).clamp(min=0)
    p = torch.exp(s - top)
    den = p.sum(-1, keepdim=True) + old * torch.exp(-top)
    ref = ((p @ vr.double().transpose(0, 1).contiguous()) / den).transpose(0, 1)
    a = ((p @ vr.double().abs().transpose(0, 1).contiguous()) / den).transpose(0, 1)
    off = (d + 4) * U24 * (q[:1].double().abs().transpose(0, 1) @ kr.double().abs().permute(1, 2, 0).contiguous()).amax() / 16
    assert bool(((o.double() - ref).abs() <= U8 * ref.abs() + (U8 * (1 + U8) + 2 * off + 2 * (old + 700) * U24) * a).all())


@pytest.mark.parametrize("kind", KINDS)
def test_second_part_of_a_prompt(kind):
    """Two parts of a prompt through the cache: the first part's keys, read back with the second's, give the attention
    over the values that the cache holds (its own bound: the packed forward's, P and O rounded)."""
    d, hq, hkv, page, parts = 128, 8, 2, 32, [[100, 7], [40, 65]]
    total = [sum(x) for x in zip(*parts)]
    table, pages = table_of(total, page)
    c = Cache(kind, pages, hkv, page, d)
    g = torch.Generator(device="cuda")
    g.manual_seed(4)
    inv = (10000.0 ** (-torch.arange(0, d, 2, device="cuda") / d)).float()
    old = [0, 0]
    for new in parts:
        T = sum(new)
        q, k, v = (torch.randn((T, h, d), generator=g, device="cuda").to(BF) for h in (hq, hkv, hkv))
        qr = torch.empty_like(q)
        dash.dash_kv_append(k, v, *c.pools, table, i32(old), cu=i32(offsets(new)), q=q, q_out=qr, inv_freq=inv, **c.scales)
        old = [a + b for a, b in zip(old, new)]
        cu_k = i32(offsets(old))
        k_all, v_all = dash.kv_read(*c.pools, table, i32(old), cu_k, sum(old), **c.scales)
        o, _ = dash.attn_packed_fwd(qr, k_all, v_all, i32(offsets(new)), cu_k)
    pos = 0
    for s, (n, m) in enumerate(zip(old, parts[1])):
        kk, vv = (x[sum(old[:s]):sum(old[:s + 1])].double().transpose(0, 1) for x in (k_all, v_all))
        if kind != "e4m3":
            want = c.rows64(table, s, n)
            assert torch.equal(kk, want[0]) and torch.equal(vv, want[1])
        qq = qr[pos:pos + m].double().transpose(0, 1).reshape(hkv, hq // hkv, m, d)
        sc = (qq.flatten(1, 2) @ kk.transpose(1, 2).contiguous()).reshape(hkv, hq // hkv, m, n) / math.sqrt(d)
        sc = sc.masked_fill(torch.ones(m, n, dtype=torch.bool, device="cuda").triu(n - m + 1), -math.inf)
        p = torch.softmax(sc, -1).flatten(1, 2)
        ref, a = (torch.reshape(p @ x, (hq, m, d)).transpose(0, 1) for x in (vv, vv.abs()))
        off = (d + 4) * U24 * (qq.flatten(1, 2).abs() @ kk.abs().transpose(1, 2).contiguous()).amax() / math.sqrt(d)
        assert bool(((o[pos:pos + m].double() - ref).abs() <= U8 * ref.abs() + (U8 * (1 + U8) + 2 * off + 2 * n * U24 + 16 * U24) * a).all())
        pos += m


@pytest.mark.parametrize("kind", MX)
def test_generation_step_captured(kind):
    """Append, read the new row back, attend: eagerly and replayed with later lengths, the same bits."""
    d, hq, hkv, page, steps, old = 128, 8, 2, 16, 5, [0, 15, 130, 77]
    B = len(old)
    table, pages = table_of([n + steps for n in old], page)
    inv = (10000.0 ** (-torch.arange(0, d, 2, device="cuda") / d)).float()
    g = torch.Generator(device="cuda")
    g.manual_seed(5)
    new = [[torch.randn((B, h, d), generator=g, device="cuda").to(BF) for h in (hq, hkv, hkv)] for _ in range(steps)]
    ws = torch.empty(dash.dash_decode_workspace_size(B, hq, hkv, d, page, table.shape[1]), dtype=torch.uint8, device="cuda")
    cu = i32(list(range(B + 1)))

    def buffers():
        c = Cache(kind, pages, hkv, page, d, seed=3)
        x = [torch.empty((B, h, d), device="cuda", dtype=BF) for h in (hq, hkv, hkv, hq, hq, hkv, hkv)]
        return c, i32(old), i32(old), x

    def step(b):
        c, lens, first, (q, k, v, qr, o, kr, vr) = b
        dash.dash_kv_append(k, v, *c.pools, table, lens, q=q, q_out=qr, inv_freq=inv, **c.scales)
        first.copy_(lens)
        lens += 1
        dash.dash_kv_read(*c.pools, table, lens, cu, kr, vr, first=first, **c.scales)
        dash.dash_attn_decode(qr, *c.pools, table, lens, o, workspace=ws, **c.scales)

    def feed(b, t):
        for x, y in zip(b[3], new[t]):
            x.copy_(y)

    eager, outs = buffers(), []
    for t in range(steps):
        feed(eager, t)
        step(eager)
        outs.append([x.clone() for x in eager[3][3:]])
    b = buffers()
    feed(b, 0)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        step(b)
    for t in range(steps):
        feed(b, t)
        graph.replay()
        dash.attn_decode(torch.ones_like(b[3][0]), *b[0].pools, table, b[1], workspace=ws, **b[0].scales)
        torch.cuda.synchronize()
        for x, want in zip(b[3][3:], outs[t]):
            assert torch.equal(x, want)


def test_refusals():
    table, pages = table_of([20, 30], 16)
    lens = i32([20, 30])
    x8, x4 = Cache("mxfp8", pages, 2, 16, 64), Cache("mxfp4", pages, 2, 16, 64)
    q = torch.ones((2, 4, 64), device="cuda").to(BF)
    k = q[:, :2].contiguous()
    for c in (x8, x4):
        for word, scales in (("k_scale", dict(k_scale=None, v_scale=c.v_scale)), ("v_scale", dict(k_scale=c.k_scale, v_scale=None)),
                             ("k_scale", dict(k_scale=c.k_scale[1:], v_scale=c.v_scale)), ("v_scale", dict(k_scale=c.k_scale, v_scale=c.v_scale[..., :1])),
                             ("k_scale", dict(k_scale=c.k_scale.transpose(0, 1).contiguous().transpose(0, 1), v_scale=c.v_scale)),
                             ("k_scale", dict(k_scale=c.k_scale.float(), v_scale=c.v_scale))):
            for call in (lambda: dash.attn_decode(q, *c.pools, table, lens, **scales), lambda: dash.dash_kv_append(k, k, *c.pools, table, lens, **scales),
                         lambda: dash.kv_read(*c.pools, table, lens, i32([0, 1, 2]), 2, **scales)):
                with pytest.raises(dash.DashError, match=word):
                    call()
    with pytest.raises(dash.DashError, match="cache"):
        dash.attn_decode(q, x4.k.view(torch.int8), x4.v.view(torch.int8), table, lens, **x4.scales)
    with pytest.raises(dash.DashError, match="head dim"):
        dash.attn_decode(torch.ones((2, 4, 128), device="cuda").to(BF), *x4.pools, table, lens, **x4.scales)
    kr = torch.empty((4, 2, 64), device="cuda", dtype=BF)
    for word, kw in (("k_out or v_out", dict(k_out=None, v_out=None)), ("cu", dict(cu=i32([0, 4]))), ("first", dict(first=i32([0]))),
                     ("v_out", dict(v_out=kr[:3])), ("k_out", dict(k_out=kr.float())), ("overlap", dict(k_out=kr[:, :1].expand(4, 2, 64)))):
        args = dict(dict(cu=i32([0, 2, 4]), k_out=kr, v_out=None), **kw)
        with pytest.raises(dash.DashError, match=word):
            dash.dash_kv_read(*x8.pools, table, lens, **args, **x8.scales)


@pytest.mark.parametrize("d,hq,hkv,rotary,interleaved", [(64, 16, 8, 64, False), (128, 32, 8, 96, True), (256, 16, 4, 256, False)])
@pytest.mark.parametrize("kind", KINDS)
def test_appends_and_reads_too_large_for_the_caches(d, hq, hkv, rotary, interleaved, kind):
    """Appends from 32 MB of q, k and v on (64 beside a bf16 or e4m3 cache), and reads of as much, go past the caches: the bits of
    calls of fewer rows, q and k also in place."""
    page, old = 32, [5, 0, 1000]
    tokens = (33 if kind in MX else 66) * 2 ** 20 // ((hq + 2 * hkv) * d * 2) + 1
    lens = [tokens // 4, tokens // 2, tokens - tokens // 4 - tokens // 2]
    assert max(lens) * (hq + 2 * hkv) * d * 2 < (32 if kind in MX else 64) * 2 ** 20
    table, pages = table_of([o + n for o, n in zip(old, lens)], page)
    g = torch.Generator(device="cuda")
    g.manual_seed(d + hq)
    q, k, v = (torch.randn((tokens, h, d), generator=g, device="cuda").to(BF) for h in (hq, hkv, hkv))
    inv = (10000.0 ** (-torch.arange(0, rotary, 2, device="cuda") / rotary)).float()
    at = offsets(lens)
    big, small, inside = (Cache(kind, pages, hkv, page, d) for _ in range(3))
    kw = dict(inv_freq=inv, interleaved=interleaved)
    q1, k1, status = torch.empty_like(q), torch.empty_like(k), i32([0])
    dash.dash_kv_append(k, v, *big.pools, table, i32(old), cu=i32(at), q=q, q_out=q1, k_out=k1, status=status, **kw, **big.scales)
    q2, k2 = torch.empty_like(q), torch.empty_like(k)
    for s, n in enumerate(lens):
        part = slice(at[s], at[s] + n)
        dash.dash_kv_append(k[part], v[part], *small.pools, table[s:s + 1], i32(old[s:s + 1]), cu=i32([0, n]), q=q[part], q_out=q2[part],
                            k_out=k2[part], status=status, **kw, **small.scales)
    dash.dash_kv_append(k, v, *inside.pools, table, i32(old), cu=i32(at), q=q, q_out=q, k_out=k, status=status, **kw, **inside.scales)
    assert int(status) == 0
    bits = lambda c: [x if x.dtype is BF else x.view(torch.uint8) for x in c.pools] + ([c.k_scale, c.v_scale] if kind in MX else [])  # noqa: E731
    for c in (big, inside):
        assert all(torch.equal(x, y) for x, y in zip(bits(c), bits(small)))
    assert all(torch.equal(x, q2) for x in (q1, q)) and all(torch.equal(x, k2) for x in (k1, k))
    # read back: all keys, and again, by few
    all_keys = i32([o + n for o, n in zip(old, lens)])
    rows = int(all_keys.sum())
    repeat = 33 * 2 ** 20 // (rows * hkv * d * 4) + 1  # sequences of the same keys
    t, n = table.repeat(repeat, 1), all_keys.repeat(repeat)
    cu = torch.cat((i32([0]), n.cumsum(0).to(torch.int32)))
    assert rows * repeat * hkv * d * 4 >= 32 * 2 ** 20
    ko, vo = dash.kv_read(*big.pools, t, n, cu, rows * repeat, status=status, **big.scales)
    first = 0
    for s, m in enumerate(all_keys.tolist()):
        for part in range(0, m, 900):
            few = min(900, m - part)
            kf, vf = dash.kv_read(*big.pools, table[s:s + 1], all_keys[s:s + 1], i32([0, few]), few, first=i32([part]), status=status, **big.scales)
            for r in range(repeat):
                own = slice(r * rows + first + part, r * rows + first + part + few)
                assert torch.equal(ko[own], kf) and torch.equal(vo[own], vf)
        first += m
    assert int(status) == 0


@pytest.mark.parametrize("kind", ["bf16", "mxfp8"])
@pytest.mark.parametrize("batch", [65, 66, 67, 69, 128, 130, 257, 259, 4097])
def test_lengths_at_any_address(batch, kind):
    """Batches that no share of 64 lanes divides, their lengths at the end of a tensor and at an address that only 4 divides."""
    d, hq, hkv, page = 64, 4, 2, 16
    lens = [1 + 7 * i % 53 if i % 97 else 600 + i % 400 for i in range(batch)]
    table, pages = table_of(lens, page)
    c = Cache(kind, pages, hkv, page, d)
    c.spoil(used_rows(table, lens, page, pages))
    g = torch.Generator(device="cuda")
    g.manual_seed(batch)
    q = torch.randn((batch, hq, d), generator=g, device="cuda").to(BF)
    ro, rl, tol = attend64(c, q, table, lens, 1 / math.sqrt(d))
    want = None
    for front in (0, 1, 2, 3):
        n = i32([10 ** 6] * front + lens)[front:]  # (what is before it does not matter)
        o, lse, status = torch.empty_like(q), torch.empty((batch, hq), device="cuda"), i32([0])
        dash.dash_attn_decode(q, *c.pools, table, n, o, lse, status=status, **c.scales)
        assert int(status) == 0 and bool(((o.double() - ro).abs() <= tol).all())
        assert bool(((lse.double() - rl).abs() <= 2e-5 * rl.abs().clamp(min=1)).all())
        assert want is None or torch.equal(o, want)
        want = o
        p = dash.attn_prefix_decode(q, *c.pools, table, n, table[0, :1].contiguous(), i32([0]), **c.scales)  # (nothing shared)
        assert bool(((p.double() - ro).abs() <= tol + 8 * U24 * tol.clamp(min=ro.abs().amax())).all())
