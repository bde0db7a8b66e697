"""The paged cache on the GPU: appending with rotation, attention of one token, and
both as a generation step uses them, against their definitions in float64.

Tolerances (u8 = 2^-8, half a bf16 step; u24 = 2^-24, half an fp32 step):
  rotated value  u8 |y| for its own rounding, and for sine and cosine (the angle in
                 half turns is rounded to fp32, pi u24, the functions 2 u24 more)
                 and the two products 8 u24 (|x| + |y|)
  e4m3           2^-4 |y| or half of the smallest step, 2^-10
  o              u8 |o| for its own rounding and u8 A for P's (A = sum_j P_j |v_j|);
                 each score is off by at most (d + 4) u24 times its sum of absolute
                 products, which moves o by twice that times A; sums over n keys in fp32
                 add at most n u24 A to each of numerator and denominator
"""
import math

import pytest
import torch

from paper_2601_21824_amd import binding as dash

pytestmark = pytest.mark.gpu

U8, U24 = 2.0 ** -8, 2.0 ** -24
BF, E4 = torch.bfloat16, torch.float8_e4m3fn


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def make_cache(pages, hkv, page, d, dtype, order="phrd", seed=0, fill=None):
    """[pages, hkv, page, d] view of a pool laid out in `order` of (p)ages, (h)eads, (r)ows, (d)."""
    size = {"p": pages, "h": hkv, "r": page, "d": d}
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    x = torch.randn([size[c] for c in order], generator=g, device="cuda")
    if fill is not None:
        x.fill_(fill)
    return x.clamp(-448, 448).to(dtype).permute([order.index(c) for c in "phrd"])


def table_of(lens, page, spare=2, seed=0):
    g = torch.Generator()
    g.manual_seed(seed)
    need = [-(-n // page) for n in lens]
    ids = torch.randperm(sum(need) + spare, generator=g).tolist()
    t = torch.full((len(lens), max(max(need), 1) + 1), -1, dtype=torch.int32)
    for s, n in enumerate(need):
        for i in range(n):
            t[s, i] = ids.pop()
    return t.cuda(), sum(need) + spare


def rows_of(cache, table, s, n, page):
    """Sequence s's first n rows [hkv, n, d] in float64."""
    ids = table[s, :-(-n // page)].long()
    return cache[ids].double().transpose(0, 1).flatten(1, 2)[:, :n]


# ------------------------------------------------------------------ append
def rotate64(x, place, inv_freq, interleaved):
    x = x.double().clone()
    if inv_freq is None:
        return x
    n = inv_freq.numel()
    ang = (place.double()[:, None] * inv_freq.double())[:, None]
    a, b = (x[..., 0:2 * n:2].clone(), x[..., 1:2 * n:2].clone()) if interleaved else (x[..., :n].clone(), x[..., n:2 * n].clone())
    y, z = a * ang.cos() - b * ang.sin(), a * ang.sin() + b * ang.cos()
    if interleaved:
        x[..., 0:2 * n:2], x[..., 1:2 * n:2] = y, z
    else:
        x[..., :n], x[..., n:2 * n] = y, z
    return x


def pair_size(x, inv_freq, interleaved):
    """|x| + |y| of each component's pair."""
    x = x.double().abs()
    out = torch.zeros_like(x)
    if inv_freq is None:
        return out
    n = inv_freq.numel()
    if interleaved:
        out[..., 0:2 * n:2] = out[..., 1:2 * n:2] = x[..., 0:2 * n:2] + x[..., 1:2 * n:2]
    else:
        out[..., :n] = out[..., n:2 * n] = x[..., :n] + x[..., n:2 * n]
    return out


# (d, hq, hkv, new tokens per sequence, lengths before, page, dtype, rotary, interleaved, layout)
APPENDS = [
    (128, 8, 2, [1, 1, 1], [0, 15, 16], 16, BF, 128, False, "phrd"),
    (128, 8, 2, [1, 1, 1], [0, 15, 16], 16, E4, 128, False, "phrd"),
    (64, 4, 4, [5, 0, 40, 1], [3, 7, 0, 100], 16, BF, 32, True, "prhd"),
    (64, 5, 1, [17, 33], [0, 47], 48, E4, 64, True, "hprd"),
    (256, 6, 3, [9, 70], [131071, 2], 64, BF, 256, False, "phrd"),
    (256, 2, 1, [9, 70], [131071, 2], 64, E4, 208, True, "prhd"),
    (128, 32, 8, [700, 0, 1, 333], [0, 5, 99, 64], 32, E4, 96, False, "phrd"),  # many rounds per wave
    (128, 3, 3, [300, 600], [0, 0], 16, BF, 0, False, "phrd"),  # no rotation
]


@pytest.mark.parametrize("d,hq,hkv,new,old,page,dtype,rotary,interleaved,order", APPENDS)
@pytest.mark.parametrize("with_q", [True, False])
def test_append(d, hq, hkv, new, old, page, dtype, rotary, interleaved, order, with_q):
    g = torch.Generator(device="cuda")
    g.manual_seed(d + hq)
    T, extra = sum(new), 3  # rows behind the last sequence
    fused = torch.randn((T + extra, hq + 2 * hkv, d), generator=g, device="cuda").to(BF)
    q, k, v = fused.split([hq, hkv, hkv], dim=1)  # strided views
    table, pages = table_of([a + b for a, b in zip(old, new)], page)
    kc, vc = (make_cache(pages, hkv, page, d, dtype, order, seed=i) for i in (1, 2))
    k0, v0 = kc.clone(), vc.clone()
    at = [0]
    for n in new:
        at.append(at[-1] + n)
    inv = (10000.0 ** (-torch.arange(0, rotary, 2, device="cuda") / rotary)).float() if rotary else None
    e4 = dtype is E4
    ks, vs = (torch.linspace(0.01, 0.02, hkv, device="cuda") * f if e4 else None for f in (1.0, 1.5))
    q_out, k_out = torch.full_like(q, 7.0), torch.full_like(k, 7.0)
    status = i32([0])
    kw = dict(q=q, q_out=q_out) if with_q else {}
    dash.dash_kv_append(k, v, kc, vc, table, i32(old), cu=i32(at), k_out=k_out, inv_freq=inv, interleaved=interleaved,
                        k_scale=ks, v_scale=vs, status=status, **kw)
    assert int(status) == 0
    place = torch.cat([torch.arange(o, o + n) for o, n in zip(old, new)]).cuda()
    for x, out in ((q, q_out), (k, k_out))[0 if with_q else 1:]:
        ref = rotate64(x[:T], place, inv, interleaved)
        tol = U8 * ref.abs() * (1 + U8) + 8 * U24 * pair_size(x[:T], inv, interleaved)
        assert bool(((out[:T].double() - ref).abs() <= tol).all())
        assert bool((out[T:] == 7.0).all()), "rows behind the last sequence are left alone"
    if not with_q:
        assert bool((q_out == 7.0).all())
    seq = torch.cat([torch.full((n,), s) for s, n in enumerate(new)]).cuda()
    ids, rows = table[seq, place // page].long(), place % page
    # values: the bits of one fp32 division and one rounding
    want_v = (v[:T].float() / vs[:, None]).clamp(-448, 448).to(E4) if e4 else v[:T]
    assert torch.equal(vc[ids, :, rows].float(), want_v.float())
    ref = rotate64(k[:T], place, inv, interleaved)
    tol = 8 * U24 * pair_size(k[:T], inv, interleaved)
    if e4:
        ref, tol = ref / ks.double()[:, None], tol / ks.double()[:, None]
        ref = ref.clamp(-448, 448)
        tol = tol + torch.maximum(2.0 ** -4 * ref.abs(), torch.full_like(ref, 2.0 ** -10)) * (1 + U8)
        assert bool((ref.abs() == 448).any()) or hkv < 3  # (some saturate)
    else:
        tol = tol + U8 * ref.abs() * (1 + U8)
        assert torch.equal(kc[ids, :, rows], k_out[:T])
    assert bool(((kc[ids, :, rows].double() - ref).abs() <= tol).all())
    # nothing else moved
    for c, c0 in ((kc, k0), (vc, v0)):
        keep = torch.ones(pages, page, dtype=torch.bool, device="cuda")
        keep[ids, rows] = False
        assert torch.equal(c.transpose(1, 2)[keep].float(), c0.transpose(1, 2)[keep].float())


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype", [BF, E4])
@pytest.mark.parametrize("d,rotary", [(d, r) for d in (64, 128, 256) for r in (16, d // 2, d // 2 + 16, d - 16)])
def test_append_keeps_the_components_behind_rotary_dim(d, rotary, dtype, interleaved):
    """Infinities, NaN and -0 behind rotary_dim: q_out and k_out have their bits, the cache the same values."""
    hq, hkv, T = 4, 2, 12
    g = torch.Generator(device="cuda")
    g.manual_seed(d + rotary)
    q, k = (torch.randn((T, h, d), generator=g, device="cuda").to(BF) for h in (hq, hkv))
    for i, odd in enumerate((float("inf"), float("-inf"), float("nan"), -0.0)):
        for x in (q, k):  # each at every component once in a row of four tokens and heads, then by itself
            x[i::4, :, rotary + i::4] = odd
            x[i, 0, rotary:] = 1.0
            x[i, 0, rotary + 4 + i] = odd
    table, lens = torch.arange(T, dtype=torch.int32, device="cuda")[:, None], i32([1 + i % 5 for i in range(T)])
    kc, vc = (make_cache(T, hkv, 16, d, dtype, fill=0.0) for _ in range(2))
    inv = (10000.0 ** (-torch.arange(0, rotary, 2, device="cuda") / rotary)).float()
    q_out, k_out = torch.empty_like(q), torch.empty_like(k)
    dash.dash_kv_append(k, k, kc, vc, table, lens, q=q, q_out=q_out, k_out=k_out, inv_freq=inv, interleaved=interleaved)
    for x, out in ((q, q_out), (k, k_out)):
        assert torch.equal(out[..., rotary:].view(torch.int16), x[..., rotary:].view(torch.int16))
        assert bool(out[..., :rotary].isfinite().all())
    got = kc[torch.arange(T), :, lens.long()][..., rotary:]
    want = k[..., rotary:] if dtype is BF else k[..., rotary:].float().clamp(-448, 448).to(E4)
    bits = torch.int16 if dtype is BF else torch.uint8
    same = (got.view(bits) == want.view(bits)) | (got.float().isnan() & want.float().isnan())
    assert bool(same.all())


def test_append_in_place_and_nan():
    """q_out = q and k_out = k; NaN and infinity pass (e4m3: infinity saturates, NaN stays)."""
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    q, k = (torch.randn((4, h, 64), generator=g, device="cuda").to(BF) for h in (4, 2))
    v = torch.randn((4, 2, 64), generator=g, device="cuda").to(BF)
    v[1, 0, 3], v[2, 1, 5], v[3, 1, 6] = float("nan"), float("inf"), float("-inf")
    inv = torch.full((32,), 0.5, device="cuda")
    table, lens = i32([[0], [1], [2], [3]]), i32([0, 1, 2, 3])
    kc, vc = (make_cache(4, 2, 16, 64, E4, fill=0.0) for _ in range(2))
    q1, k1 = torch.empty_like(q), torch.empty_like(k)
    dash.dash_kv_append(k, v, kc, vc, table, lens, q=q, q_out=q1, k_out=k1, inv_freq=inv)
    q2, k2 = q.clone(), k.clone()
    dash.dash_kv_append(k2, v, kc, vc, table, lens, q=q2, q_out=q2, k_out=k2, inv_freq=inv)
    assert torch.equal(q1, q2) and torch.equal(k1, k2)
    got = vc[torch.arange(4), :, torch.arange(4)].float()
    assert got[1, 0, 3].isnan() and got[2, 1, 5] == 448 and got[3, 1, 6] == -448
    assert int(got.isnan().sum()) == 1


def test_append_reports_missing_pages():
    """Tokens outside the table or in a page that does not exist are not stored, the others are."""
    k = torch.ones((5, 1, 64), device="cuda").to(BF)
    for table, old, cu, stored in (([[0, 9]], [14], [0, 5], 2),     # the second page does not exist
                                   ([[0, -1]], [14], [0, 5], 2),
                                   ([[0, 1]], [29], [0, 5], 3),     # behind the table
                                   ([[0, 1]], [-3], [0, 5], 0),     # a negative length
                                   ([[0, 1]], [2 ** 31 - 1], [0, 5], 0)):
        kc, vc = (make_cache(2, 1, 16, 64, BF, fill=0.0) for _ in range(2))
        status = i32([0])
        dash.dash_kv_append(k, k, kc, vc, i32(table), i32(old), cu=i32(cu), status=status)
        assert int(status) == 1
        assert int((kc == 1).sum()) == int((vc == 1).sum()) == stored * 64


# (offsets, lengths before, page): rows before the first sequence, few of them and more than a
# sequence has cached; one sequence; empty ones first; rows on both sides
OUTSIDE = [([3, 8], [10], 16), ([1, 1, 5, 9], [40, 7, 0], 16), ([6, 6, 6, 20], [2, 90, 33], 32), ([700, 1100, 1500], [900, 64], 64)]


@pytest.mark.parametrize("at,old,page", OUTSIDE)
@pytest.mark.parametrize("dtype", [BF, E4])
def test_append_leaves_rows_before_the_first_sequence_alone(at, old, page, dtype):
    d, hq, hkv, tail = 128, 8, 2, 4
    g = torch.Generator(device="cuda")
    g.manual_seed(sum(at))
    q, k, v = (torch.randn((at[-1] + tail, h, d), generator=g, device="cuda").to(BF) for h in (hq, hkv, hkv))
    new = [b - a for a, b in zip(at, at[1:])]
    table, pages = table_of([a + b for a, b in zip(old, new)], page)
    kc, vc = (make_cache(pages, hkv, page, d, dtype, seed=i) for i in (1, 2))
    inv = (10000.0 ** (-torch.arange(0, d, 2, device="cuda") / d)).float()

    def call(q, k, v, kc, vc, at):
        q_out, k_out, status = torch.full_like(q, 7.0), torch.full_like(k, 7.0), i32([0])
        dash.dash_kv_append(k, v, kc, vc, table, i32(old), cu=i32(at), q=q, q_out=q_out, k_out=k_out, inv_freq=inv, status=status)
        assert int(status) == 0
        return q_out, k_out

    # the same tokens alone, from row 0 on
    own = slice(at[0], at[-1])
    k1, v1 = kc.clone(), vc.clone()
    q_want, k_want = call(q[own], k[own], v[own], k1, v1, [a - at[0] for a in at])
    q_out, k_out = call(q, k, v, kc, vc, at)
    assert torch.equal(kc.view(torch.uint8), k1.view(torch.uint8)) and torch.equal(vc.view(torch.uint8), v1.view(torch.uint8))
    assert torch.equal(q_out[own], q_want) and torch.equal(k_out[own], k_want)
    for x in (q_out, k_out):
        assert bool((x[:at[0]] == 7).all()) and bool((x[at[-1]:] == 7).all())


@pytest.mark.parametrize("at,reported", [([0, 8, 5, 10], 1), ([0, 20, 3, 12], 1), ([-2, 4, 8, 12], 1), ([-2 ** 31, 4, 8, 12], 1),
                                         ([0, 2 ** 31 - 1, 3, 12], 1), ([4, 0, 12, 12], 0)])  # (the last: all in 0 .. 11)
def test_append_offsets_that_do_not_rise(at, reported):
    """Rows that no sequence holds are reported, and what the sequences have cached keeps its bits."""
    old, d = [20, 30, 25], 64
    k = torch.ones((12, 1, d), device="cuda").to(BF)
    table, pages = table_of([n + 12 for n in old], 16)
    kc, vc = (make_cache(pages, 1, 16, d, BF, seed=i) for i in (1, 2))
    before = [[rows_of(c, table, s, n, 16) for c in (kc, vc)] for s, n in enumerate(old)]
    status = i32([0])
    dash.dash_kv_append(k, k, kc, vc, table, i32(old), cu=i32(at), status=status)
    assert int(status) == reported
    for s, n in enumerate(old):
        for c, want in zip((kc, vc), before[s]):
            assert torch.equal(rows_of(c, table, s, n, 16), want)


# ------------------------------------------------------------------ one token
def decode64(q, kc, vc, table, lens, page, scale, ks=None, vs=None):
    """o, lse and the bound on o's error, in float64."""
    B, hq, d = q.shape
    hkv = kc.shape[1]
    o, tol = (torch.zeros((B, hq, d), dtype=torch.float64, device="cuda") for _ in range(2))
    lse = torch.full((B, hq), -math.inf, dtype=torch.float64, device="cuda")
    for s, n in enumerate(lens):
        if n == 0:
            continue
        k, v = rows_of(kc, table, s, n, page), rows_of(vc, table, s, n, page)
        if ks is not None:
            k, v = k * ks.double()[:, None, None], v * vs.double()[:, None, None]
        qq = q[s].double().reshape(hkv, hq // hkv, d)
        sc = qq @ k.transpose(1, 2) * scale
        p = torch.softmax(sc, -1)
        a = p @ v.abs()
        off = (d + 4) * U24 * scale * (qq.abs() @ k.abs().transpose(1, 2)).amax(-1, keepdim=True)
        oo = p @ v
        o[s], lse[s] = oo.reshape(hq, d), torch.logsumexp(sc, -1).reshape(hq)
        tol[s] = (U8 * oo.abs() + (U8 * (1 + U8) + 2 * off + 2 * n * U24 + 16 * U24) * a).reshape(hq, d)
    return o, lse, tol


LENS = [1, 0, 31, 32, 33, 127, 128, 129, 300, 16, 5]
# (d, hq, hkv, lengths, page, dtype, layout)
DECODES = [(d, hq, hkv, LENS, page, dt, order)
           for d, page, order in ((64, 16, "phrd"), (128, 48, "prhd"), (256, 64, "hprd"))
           for hq, hkv in ((4, 4), (8, 1), (15, 3), (34, 2)) for dt in (BF, E4)]
DECODES += [(128, 8, 2, [20000], 16, BF, "phrd"), (64, 64, 1, [9000, 1], 16, E4, "phrd"), (256, 4, 4, [7001, 40, 3000], 32, E4, "phrd"),
            (128, 4, 1, [1 + 37 * i % 211 for i in range(150)], 16, BF, "phrd"),  # more than two rounds of 64 sequences
            (64, 2, 2, [0] * 70 + [2000], 16, BF, "phrd")]
# tables short enough for one chunk per sequence (65536 / d keys), full and not, and one page more
DECODES += [(d, 8, 2, [n, 1, 0, n - 17, n // 3], 16, dt, "phrd") for d in (64, 128, 256) for dt in (BF, E4)
            for n in (65536 // d - 16, 65536 // d)]
DECODES += [(128, 20, 1, [1 + 29 * i % 490 for i in range(90)], 16, BF, "phrd")]


def decode_case(d, hq, hkv, lens, page, dtype, order, seed=0, garbage=float("nan")):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed + d + hq)
    q = torch.randn((len(lens), hq + 1, d), generator=g, device="cuda").to(BF)[:, 1:] * 2  # strided, wide scores
    table, pages = table_of(lens, page, seed=seed)
    kc, vc = (make_cache(pages, hkv, page, d, dtype, order, seed=seed + i) for i in (1, 2))
    # whatever lies behind a sequence's last key, and in pages of nobody, does not matter
    used = torch.zeros((pages, page), dtype=torch.bool, device="cuda")
    for s, n in enumerate(lens):
        for i in range(-(-n // page)):
            used[int(table[s, i]), :min(page, n - i * page)] = True
    for c in (kc, vc):
        f = c.float().transpose(1, 2)
        f[~used] = garbage
        c.copy_(f.transpose(1, 2).to(dtype))
    ks, vs = ((torch.linspace(0.3, 0.9, hkv, device="cuda") * f for f in (1.0, 1.5)) if dtype is E4 else (None, None))
    return q, kc, vc, table, ks, vs


@pytest.mark.parametrize("d,hq,hkv,lens,page,dtype,order", DECODES)
def test_decode(d, hq, hkv, lens, page, dtype, order):
    q, kc, vc, table, ks, vs = decode_case(d, hq, hkv, lens, page, dtype, order)
    o = torch.full((len(lens), hq, d), 9.0, device="cuda").to(BF)
    lse = torch.full((len(lens), hq), 9.0, device="cuda")
    status = i32([0])
    dash.dash_attn_decode(q, kc, vc, table, i32(lens), o, lse, None, ks, vs, status=status)
    assert int(status) == 0
    ro, rl, tol = decode64(q, kc, vc, table, lens, page, 1 / math.sqrt(d), ks, vs)
    over = ((o.double() - ro).abs() - tol).max().item()
    assert over <= 0, over
    empty = i32(lens) == 0
    assert bool((o[empty] == 0).all()) and bool((lse[empty] == -math.inf).all())
    err = (lse[~empty].double() - rl[~empty]).abs()
    assert bool((err <= 2e-5 * rl[~empty].abs().clamp(min=1)).all())
    # the same bits again, and without lse
    o2 = dash.attn_decode(q, kc, vc, table, i32(lens), k_scale=ks, v_scale=vs)
    assert torch.equal(o.view(torch.int16), o2.view(torch.int16))


@pytest.mark.parametrize("shift", [-1e30, -3e9, float("-inf"), 1e30])
@pytest.mark.parametrize("where", ["first", "last", "all"])
def test_decode_far_scores(shift, where):
    """Keys taken out (or in) by a huge score: the largest still weighs exactly 1; all -inf: O = 0, L = -inf."""
    d, page, n = 128, 16, 500
    q, kc, vc, table, _, _ = decode_case(d, 4, 2, [n], page, BF, "phrd", garbage=0.0)
    q, kc = q.clone(), kc.clone()
    q[..., 0] = 1
    at = {"first": range(0, 200), "last": range(300, n), "all": range(n)}[where]
    for j in at:
        kc[int(table[0, j // page]), :, j % page, 0] = shift
    o, lse = torch.empty_like(q), torch.empty((1, 4), device="cuda")
    dash.dash_attn_decode(q, kc, vc, table, i32([n]), o, lse)
    if where == "all" and math.isinf(shift):
        assert bool((o == 0).all()) and bool((lse == -math.inf).all())
        return
    assert bool(o.isfinite().all()) and bool(lse.isfinite().all())
    if where != "all" and shift < 0:  # the other keys alone
        ro, rl, tol = decode64(q, kc, vc, table, [n], page, 1 / math.sqrt(d))
        quiet = torch.tensor([j for j in range(n) if j not in set(at)], device="cuda")
        k, v = (rows_of(c, table, 0, n, page)[:, quiet] for c in (kc, vc))
        qq = q[0].double().reshape(2, 2, d)
        sc = qq @ k.transpose(1, 2) / math.sqrt(d)
        p = torch.softmax(sc, -1)
        off = (d + 4) * U24 * (qq.abs() @ k.abs().transpose(1, 2)).amax(-1, keepdim=True) / math.sqrt(d)
        bound = U8 * (p @ v).abs() + (U8 * (1 + U8) + 2 * off + 2 * n * U24 + 16 * U24) * (p @ v.abs())
        assert bool(((o[0].double().reshape(2, 2, d) - p @ v).abs() <= bound).all())


def test_decode_reports_bad_tables():
    """A page outside the cache, a length outside the table: reported, other sequences right."""
    q, kc, vc, table, _, _ = decode_case(64, 4, 2, [40, 40], 16, BF, "phrd")
    lens = i32([40, 40])
    good = dash.attn_decode(q, kc, vc, table, lens)
    for s, i, to in ((0, 1, 100), (0, 2, -1), (0, 0, 2 ** 31 - 1)):
        t = table.clone()
        t[s, i] = to
        status = i32([0])
        o = dash.attn_decode(q, kc, vc, t, lens, status=status)
        assert int(status) == 1 and torch.equal(o[1], good[1])
    for n, status_want in ((64, 1), (1000, 1), (-1, 1)):  # 64: the table's last entry is no page
        status = i32([0])
        o = dash.attn_decode(q, kc, vc, table, i32([n, 40]), status=status)
        assert int(status) == status_want and torch.equal(o[1], good[1])


def test_lengths_and_scales_of_another_shape_are_refused():
    q, kc, vc, table, ks, vs = decode_case(64, 8, 4, [5, 9, 20, 1], 16, E4, "phrd")
    lens, o = i32([5, 9, 20, 1]), torch.empty_like(q)
    want = dash.attn_decode(q, kc, vc, table, lens, k_scale=ks, v_scale=vs)
    assert torch.equal(dash.attn_decode(q, kc, vc, table, lens[:, None], k_scale=ks[None, :, None], v_scale=vs), want)
    lse = torch.empty((4, 8), device="cuda")
    for word, kw in (("lens", dict(lens=lens.reshape(2, 2))), ("k_scale", dict(k_scale=ks.reshape(2, 2))),
                     ("v_scale", dict(v_scale=vs.reshape(2, 2))), ("lse", dict(lse=lse.t().contiguous())),
                     ("lse", dict(lse=lse.flatten()))):
        args = dict(dict(lens=lens, lse=lse, k_scale=ks, v_scale=vs), **kw)
        with pytest.raises(dash.DashError, match=word):
            dash.dash_attn_decode(q, kc, vc, table, o=o, **args)
    k = q[:, :4].contiguous()
    for word, kw in (("lens", dict(lens=lens.reshape(2, 2))), ("k_scale", dict(k_scale=ks.reshape(2, 2))),
                     ("inv_freq", dict(inv_freq=torch.ones((4, 4), device="cuda")))):
        with pytest.raises(dash.DashError, match=word):
            dash.dash_kv_append(k, k, kc, vc, table, **dict(dict(lens=lens, k_scale=ks, v_scale=vs), **kw))


def test_tables_of_no_page():
    """No sequence has a page: nothing to attend to, nowhere to store."""
    q, kc = torch.ones((3, 4, 64), device="cuda").to(BF), make_cache(2, 2, 16, 64, BF)
    table, lens, status = torch.empty((3, 0), dtype=torch.int32, device="cuda"), i32([0, 0, 0]), i32([0])
    o, lse = torch.full_like(q, 3.0), torch.zeros((3, 4), device="cuda")
    dash.dash_attn_decode(q, kc, kc, table, lens, o, lse, status=status)
    assert bool((o == 0).all()) and bool((lse == -math.inf).all()) and int(status) == 0
    before = kc.clone()
    dash.dash_kv_append(q[:, :2], q[:, :2], kc, kc.clone(), table, lens, status=status)
    assert int(status) == 1 and torch.equal(kc, before)


# ------------------------------------------------------------------ together
def test_generation_step_captured_twice_on_one_workspace():
    """Append, then attend, for several tokens: eagerly, and from two graphs on one
    workspace that are replayed in turn with other work between them; every token of
    every sequence against float64, all three the same bits."""
    d, hq, hkv, page, steps = 128, 8, 2, 16, 6
    old = [0, 15, 130, 77]
    B = len(old)
    g = torch.Generator(device="cuda")
    g.manual_seed(5)
    table, pages = table_of([n + steps for n in old], page)
    inv = (10000.0 ** (-torch.arange(0, d, 2, device="cuda") / d)).float()
    base = [make_cache(pages, hkv, page, d, BF, seed=i) for i in (1, 2)]
    new = [[torch.randn((B, h, d), generator=g, device="cuda").to(BF) for h in (hq, hkv, hkv)] for _ in range(steps)]

    ws = torch.empty(dash.dash_decode_workspace_size(B, hq, hkv, d, page, table.shape[1]), dtype=torch.uint8, device="cuda")

    def buffers():
        return dict(kc=base[0].clone(), vc=base[1].clone(), lens=i32(old), q=torch.empty((B, hq, d), device="cuda", dtype=BF),
                    k=torch.empty((B, hkv, d), device="cuda", dtype=BF), v=torch.empty((B, hkv, d), device="cuda", dtype=BF),
                    qr=torch.empty((B, hq, d), device="cuda", dtype=BF), o=torch.empty((B, hq, d), device="cuda", dtype=BF))

    def step(b):
        dash.dash_kv_append(b["k"], b["v"], b["kc"], b["vc"], table, b["lens"], q=b["q"], q_out=b["qr"], inv_freq=inv)
        b["lens"] += 1
        dash.dash_attn_decode(b["qr"], b["kc"], b["vc"], table, b["lens"], b["o"], workspace=ws)

    def feed(b, t):
        for x, y in zip((b["q"], b["k"], b["v"]), new[t]):
            x.copy_(y)

    eager = buffers()
    outs = []
    for t in range(steps):
        feed(eager, t)
        step(eager)
        outs.append(eager["o"].clone())
        lens = [n + t + 1 for n in old]
        ro, _, tol = decode64(eager["qr"], eager["kc"], eager["vc"], table, lens, page, 1 / math.sqrt(d))
        assert bool(((outs[-1].double() - ro).abs() <= tol).all())
    graphs = []
    for _ in range(2):
        b = buffers()
        feed(b, 0)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            step(b)  # warm up on another stream
        torch.cuda.current_stream().wait_stream(side)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step(b)
        b["lens"].copy_(i32(old))
        graphs.append((graph, b))
    for t in range(steps):
        for graph, b in graphs:
            feed(b, t)
            graph.replay()
            dash.attn_decode(torch.ones_like(b["q"]), b["kc"], b["vc"], table, b["lens"], workspace=ws)  # eager, same workspace
            torch.cuda.synchronize()
            assert torch.equal(b["o"], outs[t])
    for _, b in graphs:
        assert torch.equal(b["kc"], eager["kc"]) and torch.equal(b["vc"], eager["vc"])


def test_two_streams_with_their_own_workspaces():
    q, kc, vc, table, _, _ = decode_case(128, 8, 2, [5000, 3, 900], 16, BF, "phrd")
    lens = i32([5000, 3, 900])
    want = dash.attn_decode(q, kc, vc, table, lens)
    torch.cuda.synchronize()
    n = dash.dash_decode_workspace_size(3, 8, 2, 128, 16, table.shape[1])
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = [[torch.zeros_like(want) for _ in range(8)] for _ in streams]
    spaces = [torch.empty(n, dtype=torch.uint8, device="cuda") for _ in streams]
    torch.cuda.synchronize()
    for i in range(8):
        for s, ws, o in zip(streams, spaces, outs):
            dash.dash_attn_decode(q, kc, vc, table, lens, o[i], workspace=ws, stream=s)
    torch.cuda.synchronize()
    assert all(torch.equal(x, want) for o in outs for x in o)
    with pytest.raises(dash.DashError):
        dash.dash_attn_decode(q, kc, vc, table, lens, outs[0][0], stream=streams[0])


def test_cache_beyond_32_bit_offsets():
    """A cache of over 4 GiB: pages at its far end."""
    d, hkv, page = 256, 1, 65536
    pages = 130  # 130 * 65536 * 256 * 1 byte = 2.2e9 elements of e4m3 each for K and V
    kc = torch.zeros((pages, hkv, page, d), dtype=torch.uint8, device="cuda").view(E4)
    vc = torch.zeros((pages, hkv, page, d), dtype=torch.uint8, device="cuda").view(E4)
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    new = [torch.randn((700, h, d), generator=g, device="cuda").to(BF) for h in (2, 1, 1)]
    table = i32([[129, 128]])
    old = 65536 - 300
    dash.dash_kv_append(new[1], new[2], kc, vc, table, i32([old]), cu=i32([0, 700]))
    assert torch.equal(kc[129, 0, old:].float(), new[1][:300, 0].to(E4).float())
    assert torch.equal(vc[128, 0, :400].float(), new[2][300:, 0].to(E4).float())
    q = new[0][:1]
    o = dash.attn_decode(q, kc, vc, table, i32([old + 700]))
    ro, _, tol = decode64(q, kc, vc, table, [old + 700], page, 1 / 16)
    assert bool(((o.double() - ro).abs() <= tol).all())
