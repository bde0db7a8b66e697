"""Attention over packed sequences on the GPU, forward and backward, against the
definition in float64 (packed_util.reference, which derives the bounds): sequences of no
and of one token, tiles that end inside and at a sequence, more queries than keys
(rows that see nothing), grouped heads, strided tensors, NaN in rows that belong to
nobody."""
import math

import pytest
import torch

from packed_util import BF, cu_of, over, packed_inputs, reference
from paper_2601_21824_amd import binding as dash

pytestmark = pytest.mark.gpu

EDGES = [1, 0, 31, 32, 33, 64, 0, 65, 127, 128, 129, 300]
# (d, hq, hkv, query lengths, key lengths, causal, layout)
CASES = [(d, hq, hkv, EDGES, EDGES, causal, layout)
         for d in (64, 128, 256) for causal in (True, False)
         for hq, hkv, layout in ((3, 3, "packed"), (8, 1, "fused"), (10, 2, "heads"))]
# keys before the queries, more queries than keys, no keys, no queries, one sequence
CASES += [(d, 4, 2, [5, 200, 64, 9, 0, 1, 130], [300, 260, 64, 0, 40, 257, 3], causal, "packed")
          for d in (64, 128, 256) for causal in (True, False)]
CASES += [(d, 4, 4, [600], [600], True, "packed") for d in (64, 128, 256)]
CASES += [(128, 16, 8, [257, 1023], [257, 1023], True, "fused"), (64, 2, 1, [3, 0], [0, 5], True, "packed"),
          (128, 1, 1, [1] * 150, [1 + i % 5 for i in range(150)], True, "packed")]


def ids(c):
    return f"d{c[0]}-{c[1]}over{c[2]}-{len(c[3])}x{max(c[3])}{'c' if c[5] else 'f'}-{c[6]}"


@pytest.mark.parametrize("d,hq,hkv,qlens,klens,causal,layout", CASES, ids=map(ids, CASES))
def test_forward(d, hq, hkv, qlens, klens, causal, layout):
    tail = 5
    q, k, v, do = packed_inputs(qlens, klens, hq, hkv, d, layout, tail, spread=2.0)
    o = torch.full((sum(qlens) + tail, hq, d), 7.0, device="cuda").to(BF)
    lse = torch.full((hq, sum(qlens) + tail), 7.0, device="cuda")
    cu_k = None if qlens == klens else cu_of(klens)
    dash.dash_attn_packed_fwd(q, k, v, o, lse, cu_of(qlens), cu_k, causal)
    n = sum(qlens)
    ref = reference(q, k, v, do, qlens, klens, causal, 1 / math.sqrt(d))
    assert over(o[:n], ref["o"][:n], ref["to"][:n]) <= 0
    rl, gl = ref["lse"][:, :n], lse[:, :n].double()
    assert torch.equal(rl == -math.inf, gl == -math.inf) and bool((o[:n][(rl == -math.inf).t()] == 0).all())
    ok = rl.isfinite()
    assert over(gl[ok], rl[ok], 2e-5 * rl[ok].abs().clamp(min=1)) <= 0
    assert bool((o[n:] == 7).all()) and bool((lse[:, n:] == 7).all()), "rows behind the last sequence"
    o2, lse2 = dash.attn_packed_fwd(q, k, v, cu_of(qlens), cu_k, causal)
    assert torch.equal(o[:n].view(torch.int16), o2[:n].view(torch.int16)) and torch.equal(lse[:, :n], lse2[:, :n])


# few query rows on many keys: split over the keys, evenly and not, beside sequences too
# short to be, and past the keys that a causal row sees
SPLITS = [(d, hq, hkv, q, k, causal) for d in (64, 128, 256) for causal in (True, False)
          for hq, hkv, q, k in ((2, 1, [1], [4097]), (4, 2, [130, 3], [5000, 700]), (8, 8, [64, 0, 200], [1023, 300, 3333]),
                                (2, 2, [2000], [2000]), (1, 1, [300, 5], [512, 6000]))]


@pytest.mark.parametrize("d,hq,hkv,qlens,klens,causal", SPLITS)
def test_forward_split(d, hq, hkv, qlens, klens, causal):
    tail = 3
    q, k, v, do = packed_inputs(qlens, klens, hq, hkv, d, "packed", tail, spread=2.0)
    cu_q, cu_k = cu_of(qlens), cu_of(klens)
    n, T, K = sum(qlens), sum(qlens) + tail, sum(klens) + tail
    size = dash.dash_packed_fwd_workspace_size(len(qlens), T, K, hq, hkv, d)
    assert size > 0
    ws = torch.full((size,), 255, dtype=torch.uint8, device="cuda")  # NaN, if it were read before it is written
    o, lse = torch.full_like(q, 7.0), torch.full((hq, T), 7.0, device="cuda")
    dash.dash_attn_packed_fwd(q, k, v, o, lse, cu_q, cu_k, causal, workspace=ws)
    ref = reference(q, k, v, do, qlens, klens, causal, 1 / math.sqrt(d))
    assert over(o[:n], ref["o"][:n], ref["to"][:n]) <= 0
    rl = ref["lse"][:, :n]
    assert bool(rl.isfinite().all()) and over(lse[:, :n], rl, 2e-5 * rl.abs().clamp(min=1)) <= 0
    assert bool((o[n:] == 7).all()) and bool((lse[:, n:] == 7).all())
    o1, lse1 = dash.attn_packed_fwd(q, k, v, cu_q, cu_k, causal)  # allocates its own
    assert torch.equal(o[:n].view(torch.int16), o1[:n].view(torch.int16)) and torch.equal(lse[:, :n], lse1[:, :n])
    o2, lse2 = torch.empty_like(o), torch.empty_like(lse)
    dash.dash_attn_packed_fwd(q, k, v, o2, lse2, cu_q, cu_k, causal)  # not split
    assert over(o2[:n], ref["o"][:n], ref["to"][:n]) <= 0 and over(lse2[:, :n], rl, 2e-5 * rl.abs().clamp(min=1)) <= 0


def test_forward_split_far_scores():
    """Runs whose keys all score -inf or far below the others: no weight, no NaN."""
    q, k, v, _ = packed_inputs([100], [4000], 2, 2, 128)
    q[..., 0] = 1
    for shift, lo, hi in ((float("-inf"), 0, 1500), (-1e30, 1000, 3000), (float("-inf"), 2500, 4000)):
        k2 = k.clone()
        k2[lo:hi, :, 0] = shift
        keep = torch.tensor([j for j in range(4000) if not lo <= j < hi], device="cuda")
        o, lse = dash.attn_packed_fwd(q, k2, v, cu_of([100]), cu_of([4000]), causal=False)
        for h in range(2):
            s = q[:, h].double() @ k2[keep, h].double().t() / math.sqrt(128)
            want = torch.softmax(s, -1) @ v[keep, h].double()
            assert float((o[:, h].double() - want).norm() / want.norm()) <= 5e-3
            assert float((lse[h].double() - torch.logsumexp(s, -1)).abs().max()) <= 1e-4
    k2[..., 0] = float("-inf")
    o, lse = dash.attn_packed_fwd(q, k2, v, cu_of([100]), cu_of([4000]), causal=False)
    assert bool((o == 0).all()) and bool((lse == -math.inf).all())


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("at", [0.0, 98304.0, -98304.0, 2.0 ** 20, -2.0 ** 20, 2.0 ** 24, 1e30, -1e30])
def test_forward_split_weighs_runs_by_their_keys(d, at):
    """All keys but some score the same, however far from 0, and those nothing (-2 |at| - 2^30): every
    run counts with as many keys as it has, one of them with a single one.

    O is the mean of V.  A key's P is 2^e, e = S log2(e) - m with m rounded, |e| <= U24 |m|, or 1
    where the rows are done again as far from 0: always from |m| = 2^20 on, and below it in a run
    that begins with keys that score nothing.  So the keys of all other runs have one weight; P's
    rounding makes a factor of it that is off by U8 at most.  With those of the one run that
    begins among the keys of no weight and ends behind them (v[hi:b], b unknown) another
    by d = U8 (1 + U8) + 2^(U24 |m|) - 1, O moves by d |sum over v[hi:b] of v - O| / n in first order,
    (1 + d) of it with the second.  Then U8 for the rounding of O and 2 n U24 A for the sums.
    L: log(n) added to S = at; the factor log2(e), the product, the sum with log2(n), the factor
    log(2) and the last product round by U24 each."""
    n, m = 4097, 3
    q, k, v, _ = packed_inputs([m], [n], 2, 2, d)
    q.zero_(), k.zero_()
    q[..., 0], k[..., 0], q[..., 1] = 1, at, 1
    U8, U24 = 2.0 ** -8, 2.0 ** -24
    s = torch.tensor(at).to(BF).double().item()
    size = dash.dash_packed_fwd_workspace_size(1, m, n, 2, 2, d)
    assert size > 0
    for lo, hi in ((0, 0), (1, 600), (n - 700, n - 1), (100, 4000)):
        k2 = k.clone()
        k2[lo:hi, :, 1] = -2 * abs(at) - 2.0 ** 30
        keep = torch.ones(n, dtype=torch.bool, device="cuda")
        keep[lo:hi] = False
        w = v[keep].double()
        want, top = w.mean(0), abs(s) / math.log(2)
        bound = 2 * U8 * (1 + U8) * want.abs() + 2 * n * U24 * w.abs().mean(0)
        if lo < hi and 0 < top < 2 ** 20:
            off = U8 * (1 + U8) + 2 ** (U24 * top) - 1
            bound = bound + off * (1 + off) * (v[hi:].double() - want).cumsum(0).abs().amax(0) / len(w)
        o, lse = dash.attn_packed_fwd(q, k2, v, cu_of([m]), cu_of([n]), causal=False, scale=1.0)
        o1, lse1 = torch.empty_like(o), torch.empty_like(lse)
        dash.dash_attn_packed_fwd(q, k2, v, o1, lse1, cu_of([m]), cu_of([n]), False, 1.0)  # not split
        L = s + math.log(int(keep.sum()))
        for oo, ll in ((o1, lse1), (o, lse)):
            assert over(oo, want.expand_as(oo), bound.expand_as(oo)) <= 0
            assert over(ll, torch.full_like(ll, L, dtype=torch.float64), 5 * U24 * abs(s) + 2e-5) <= 0


@pytest.mark.parametrize("shift", [-1e30, -3e9, float("-inf")])
@pytest.mark.parametrize("d", [64, 128, 256])
def test_forward_far_scores(d, shift):
    """Leading keys taken out by a huge negative score, whole units and half ones: the rows
    that see others ignore them, the rows that see only -inf have O = 0, L = -inf."""
    for lead in (20, 32, 130):
        lens = [200, 150]
        q, k, v, do = packed_inputs(lens, lens, 4, 2, d)
        q[..., 0] = 1
        k[:lead, :, 0] = shift
        o, lse = dash.attn_packed_fwd(q, k, v, cu_of(lens))
        k2 = k.clone()
        k2[:lead, :, 0] = float("-inf")
        assert bool(o[lead:].isfinite().all())
        for h in range(4):
            s = (q[:200, h].double() @ k2[:200, h // 2].double().t()) / math.sqrt(d)
            s = s.masked_fill(torch.ones_like(s, dtype=torch.bool).triu(1), -math.inf)[lead:]
            want = torch.softmax(s, -1) @ v[:200, h // 2].double()
            assert float((o[lead:200, h].double() - want).norm() / want.norm()) <= 5e-3
        if math.isinf(shift):
            assert bool((o[:lead] == 0).all()) and bool((lse[:, :lead] == -math.inf).all())
        else:
            assert bool(o[:lead].isfinite().all())


def test_forward_equals_the_dense_forward():
    """Equal lengths, a head each: the bits of the dense entry point."""
    B, H, N, d = 3, 4, 333, 128
    q, k, v, _ = packed_inputs([N] * B, [N] * B, H, H, d)
    o, lse = dash.attn_packed_fwd(q, k, v, cu_of([N] * B))
    dense = [x.reshape(B, N, H, d).transpose(1, 2).contiguous() for x in (q, k, v)]
    do, dl = dash.attn_fwd(*dense, True)
    assert torch.equal(o.reshape(B, N, H, d).transpose(1, 2), do)
    assert torch.equal(lse.reshape(H, B, N).transpose(0, 1), dl)


# ------------------------------------------------------------------ backward
def like(x, fill=7.0):
    """A tensor of x's shape and strides, filled."""
    return torch.full_like(x, fill, memory_format=torch.preserve_format) if x.is_contiguous() else \
        torch.empty_strided(x.shape, x.stride(), dtype=x.dtype, device=x.device).fill_(fill)


def train(q, k, v, do, cu_q, cu_k, causal, scale=None, status=None):
    o, lse = like(q), torch.full((q.shape[1], q.shape[0]), 7.0, device="cuda")
    dash.dash_attn_packed_fwd(q, k, v, o, lse, cu_q, cu_k, causal, scale)
    dq, dk, dv = like(do), like(k.contiguous()), like(v.contiguous())
    ws = torch.full((dash.dash_packed_workspace_size(cu_q.numel() - 1, q.shape[0], k.shape[0], q.shape[1], k.shape[1], q.shape[2]),),
                    255, dtype=torch.uint8, device="cuda")
    dash.dash_attn_packed_bwd(q, k, v, o, do, lse, dq, dk, dv, cu_q, cu_k, causal, scale, ws, status)
    assert dash.dash_bwd_check(ws) == dash.DASH_OK
    return dq, dk, dv


@pytest.mark.parametrize("d,hq,hkv,qlens,klens,causal,layout", CASES, ids=map(ids, CASES))
def test_backward(d, hq, hkv, qlens, klens, causal, layout):
    tail = 5
    q, k, v, do = packed_inputs(qlens, klens, hq, hkv, d, layout, tail)
    status = torch.full((1,), 9, dtype=torch.int32, device="cuda")
    scale = 0.7 / math.sqrt(d)
    cu_q, cu_k = cu_of(qlens), None if qlens == klens else cu_of(klens)
    dq, dk, dv = train(q, k, v, do, cu_q, cu_k, causal, scale, status)
    assert int(status) == 0
    ref = reference(q, k, v, do, qlens, klens, causal, scale)
    for name, got, lens in (("q", dq, qlens), ("k", dk, klens), ("v", dv, klens)):
        n = sum(lens)
        assert over(got[:n], ref["d" + name][:n], ref["t" + name][:n]) <= 0, "d" + name
        assert bool((got[n:] == 7).all()), "rows behind the last sequence"
    none = (ref["lse"] == -math.inf).t()[:sum(qlens)]
    assert bool((dq[:sum(qlens)][none] == 0).all())
    again = train(q, k, v, do, cu_q, cu_k, causal, scale)
    for a, b in zip((dq, dk, dv), again):
        assert torch.equal(a.view(torch.int16), b.view(torch.int16))


# wide KV tiles at d = 128, many chains per sequence, several workgroups' rounds
@pytest.mark.parametrize("d,hq,hkv,lens,causal", [
    (128, 16, 8, [4000, 1, 3000, 700, 600], True), (128, 8, 8, [2500, 513, 0, 6000], False), (128, 32, 8, [8192], True),
    (64, 32, 8, [2000, 900, 300, 1100], True), (256, 8, 4, [1500, 100, 2400], True), (256, 4, 4, [1025, 900], False)])
def test_backward_large(d, hq, hkv, lens, causal):
    q, k, v, do = packed_inputs(lens, lens, hq, hkv, d, "fused")
    out = train(q, k, v, do, cu_of(lens), None, causal)
    ref = reference(q, k, v, do, lens, lens, causal, 1 / math.sqrt(d))
    for name, got in zip("qkv", out):
        e = (got.double() - ref["d" + name])
        # (the elementwise bounds grow with the length; this is the repository's tolerance)
        assert float(e.norm() / ref["d" + name].norm()) <= 5e-3
        assert float(e.abs().max() / ref["d" + name].abs().max()) <= 2e-2
    for _ in range(8):
        again = train(q, k, v, do, cu_of(lens), None, causal)
        assert all(torch.equal(a.view(torch.int16), b.view(torch.int16)) for a, b in zip(out, again))


# 256-row KV tiles at d = 64: queries other than keys (rows that see nothing, keys that none
# sees), lengths at a tile's edges, split chains, the tile's last rows past a sequence
@pytest.mark.parametrize("hq,hkv,qlens,klens,causal,layout", [
    (32, 32, [1023, 1281, 1, 1500], [1023, 1281, 1, 1500], True, "packed"), (48, 8, [2049, 640], [2049, 640], True, "fused"),
    (64, 4, [257, 900, 31], [1700, 900, 900], True, "packed"), (64, 64, [1500, 700], [1100, 1000], True, "packed"),
    (20, 20, [300, 0, 256, 700], [257, 600, 256, 1300], False, "heads"), (40, 8, [64, 1000], [1025, 512], False, "packed")])
def test_backward_wide_d64(hq, hkv, qlens, klens, causal, layout):
    same = qlens == klens
    q, k, v, do = packed_inputs(qlens, klens, hq, hkv, 64, layout, tail=5)
    cu_q, cu_k = cu_of(qlens), None if same else cu_of(klens)
    out = train(q, k, v, do, cu_q, cu_k, causal)
    ref = reference(q, k, v, do, qlens, klens, causal, 1 / math.sqrt(64))
    for name, got, n in zip("qkv", out, (sum(qlens), sum(klens), sum(klens))):
        assert bool((got[n:] == 7).all()), "rows behind the last sequence"
        e = (got.double() - ref["d" + name])[:n]
        # (the repository's tolerance, as above)
        assert float(e.norm() / ref["d" + name].norm()) <= 5e-3
        assert float(e.abs().max() / ref["d" + name].abs().max()) <= 2e-2
    for _ in range(4):
        again = train(q, k, v, do, cu_q, cu_k, causal)
        assert all(torch.equal(a.view(torch.int16), b.view(torch.int16)) for a, b in zip(out, again))


# The same at d = 128, two key blocks a wave: sequences without queries and without keys, more
# queries than keys, keys that no query sees, lengths around the tile, a group of one and more
@pytest.mark.parametrize("hq,hkv,qlens,klens,causal,layout", [
    (32, 32, [1023, 1281, 1, 1500], [1023, 1281, 1, 1500], True, "packed"), (48, 8, [2049, 640], [2049, 640], True, "fused"),
    (64, 4, [257, 900, 0, 31], [1700, 900, 300, 900], True, "packed"), (64, 64, [1500, 700, 5], [1100, 1000, 0], True, "packed"),
    (32, 8, [700, 900, 600, 80], [511, 512, 513, 1600], True, "heads"), (20, 20, [300, 0, 256, 700], [257, 600, 256, 1300], False, "heads"),
    (40, 8, [64, 1000], [1025, 512], False, "packed"), (40, 10, [0, 700, 63], [255, 1280, 1], False, "packed")])
def test_backward_wide_d128(hq, hkv, qlens, klens, causal, layout):
    same, tail = qlens == klens, 5
    q, k, v, do = packed_inputs(qlens, klens, hq, hkv, 128, layout, tail=tail)
    # (packed_tile_rows' rule: 256-row tiles)
    T = k.shape[0]
    assert T // 256 * hq >= (320 if causal else 160) and T >= 480 * len(klens)
    cu_q, cu_k = cu_of(qlens), None if same else cu_of(klens)
    status = torch.full((1,), 9, dtype=torch.int32, device="cuda")
    out = train(q, k, v, do, cu_q, cu_k, causal, status=status)
    assert int(status) == 0
    ref = reference(q, k, v, do, qlens, klens, causal, 1 / math.sqrt(128))
    for name, got, n in zip("qkv", out, (sum(qlens), sum(klens), sum(klens))):
        assert bool((got[n:] == 7).all()), "rows behind the last sequence"
        assert over(got[:n], ref["d" + name][:n], ref["t" + name][:n]) <= 0, "d" + name
    none = (ref["lse"] == -math.inf).t()[:sum(qlens)]
    assert bool((out[0][:sum(qlens)][none] == 0).all())
    for _ in range(4):
        again = train(q, k, v, do, cu_q, cu_k, causal)
        assert all(torch.equal(a.view(torch.int16), b.view(torch.int16)) for a, b in zip(out, again))


def test_backward_accumulators_past_2_gib():
    """130 sequences of 1000, 32 heads over 8: dQ's fp32 blocks alone are 2.2 GB.  The last two
    sequences against the definition."""
    lens, hq, hkv, d = [1000] * 130, 32, 8, 128
    q, k, v, do = packed_inputs(lens, lens, hq, hkv, d)
    assert dash.dash_packed_workspace_size(len(lens), sum(lens), sum(lens), hq, hkv, d) > 1 << 31
    out = train(q, k, v, do, cu_of(lens), None, True)
    ref = reference(*(x[-2000:] for x in (q, k, v, do)), lens[-2:], lens[-2:], True, 1 / math.sqrt(d))
    for name, got in zip("qkv", out):
        e = got[-2000:].double() - ref["d" + name]
        assert float(e.norm() / ref["d" + name].norm()) <= 5e-3
        assert float(e.abs().max() / ref["d" + name].abs().max()) <= 2e-2
        assert bool(got.isfinite().all())


def test_no_queries_no_keys_one_row():
    """Tensors of no rows on either side; one row, whose strides say nothing (a broadcast)."""
    kv = torch.randn((300, 2, 64), device="cuda").to(BF)
    none = kv[:0, :1].expand(0, 4, 64)
    o, lse = dash.attn_packed_fwd(none, kv, kv, cu_of([0, 0]), cu_of([100, 200]))
    dq, dk, dv = dash.attn_packed_bwd(none, kv, kv, o, none.contiguous(), lse, cu_of([0, 0]), cu_of([100, 200]))
    assert bool((dk == 0).all()) and bool((dv == 0).all()) and dq.numel() == 0
    q = torch.randn((300, 4, 64), device="cuda").to(BF)
    empty = torch.empty((0, 2, 64), dtype=BF, device="cuda")
    o, lse = dash.attn_packed_fwd(q, empty, empty, cu_of([100, 200]), cu_of([0, 0]))
    assert bool((o == 0).all()) and bool((lse == -math.inf).all())
    dq, dk, dv = dash.attn_packed_bwd(q, empty, empty, o, q, lse, cu_of([100, 200]), cu_of([0, 0]))
    assert bool((dq == 0).all())
    for d in (64, 128, 256):
        one = torch.randn((1, 1, d), device="cuda").to(BF).as_strided((1, 2, d), (0, 0, 1))  # strides of 0
        qq = torch.randn((70, 4, d), device="cuda").to(BF)
        do = torch.randn_like(qq)
        want = reference(qq, one, one, do, [70], [1], False, 1 / math.sqrt(d))
        o, lse = dash.attn_packed_fwd(qq, one, one, cu_of([70]), cu_of([1]), causal=False)
        assert over(o, want["o"], want["to"]) <= 0
        dq, dk, dv = dash.attn_packed_bwd(qq, one, one, o, do, lse, cu_of([70]), cu_of([1]), causal=False)
        assert over(dq, want["dq"], want["tq"]) <= 0 and over(dk, want["dk"], want["tk"]) <= 0 and over(dv, want["dv"], want["tv"]) <= 0


def test_offsets_that_do_not_rise_are_reported():
    q, k, v, do = packed_inputs([200, 100], [200, 100], 4, 2, 64)
    good = cu_of([200, 100])
    o, lse = dash.attn_packed_fwd(q, k, v, good)
    want = dash.attn_packed_bwd(q, k, v, o, do, lse, good)
    ws = torch.empty(dash.dash_packed_workspace_size(2, 300, 300, 4, 2, 64), dtype=torch.uint8, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    for bad in ([0, 301, 300], [0, 200, 100], [-1, 200, 300], [0, 300, 2 ** 31 - 1], [300, 0, 300]):
        for cu_q, cu_k in ((bad, [0, 200, 300]), ([0, 200, 300], bad), (bad, bad)):
            a, b = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in (cu_q, cu_k))
            out = [torch.empty_like(x) for x in (q, k, v)]
            dash.dash_attn_packed_bwd(q, k, v, o, do, lse, *out, a, b, workspace=ws, status=status)
            assert int(status) == 1 and dash.dash_bwd_check(ws) == dash.DASH_ERR_TIMEOUT
            dash.attn_packed_fwd(q, k, v, a, b)  # some result, within the tensors
    dash.dash_attn_packed_bwd(q, k, v, o, do, lse, *out, good, workspace=ws, status=status)
    assert int(status) == 0 and dash.dash_bwd_check(ws) == dash.DASH_OK
    assert all(torch.equal(x, y) for x, y in zip(out, want))


def test_lse_of_another_shape_is_refused():
    """[tokens, heads] holds as many values as [heads, tokens]: refused, not read as it."""
    q, k, v, do = packed_inputs([90, 40], [90, 40], 4, 2, 64)
    cu = cu_of([90, 40])
    o, lse = dash.attn_packed_fwd(q, k, v, cu)
    for bad in (lse.t().contiguous(), lse.flatten(), lse.reshape(2, 260), lse[None], lse.t()):
        with pytest.raises(dash.DashError, match="lse"):
            dash.dash_attn_packed_fwd(q, k, v, o, bad, cu)
        with pytest.raises(dash.DashError, match="lse"):
            dash.attn_packed_bwd(q, k, v, o, do, bad, cu)
    with pytest.raises(dash.DashError, match="cu_k"):
        dash.attn_packed_fwd(q, k, v, cu_of([90, 20, 20]), cu_of([90, 20, 20]).reshape(2, 2))


@pytest.mark.parametrize("d", [64, 128, 256])
def test_rows_before_the_first_sequence(d):
    """Offsets that begin behind row 0: those rows are nobody's, like the ones behind the last sequence."""
    skip, lens = 70, [200, 0, 90]
    q, k, v, do = packed_inputs([skip, *lens], [skip, *lens], 4, 2, d, tail=3)
    cu = cu_of([skip, *lens])[1:].contiguous()
    own = slice(skip, skip + sum(lens))
    for x in (q, k, v, do):
        x[:skip] = float("nan")
    o, lse = torch.full_like(q, 7.0), torch.full((4, q.shape[0]), 7.0, device="cuda")
    dash.dash_attn_packed_fwd(q, k, v, o, lse, cu)
    o0, lse0 = dash.attn_packed_fwd(q[own], k[own], v[own], cu_of(lens))
    assert torch.equal(o[own], o0) and torch.equal(lse[:, own], lse0)
    dq, dk, dv = train(q, k, v, do, cu, None, True)
    want = train(q[own], k[own], v[own], do[own], cu_of(lens), None, True)
    for got, w in zip((dq, dk, dv), want):
        assert torch.equal(got[own], w)
    for x in (o, dq, dk, dv):
        assert bool((x[:skip] == 7).all()) and bool((x[own.stop:] == 7).all())


@pytest.mark.parametrize("d", [64, 128, 256])
def test_scores_that_overflow_to_minus_infinity(d):
    """Finite q and k whose products pass fp32's range: the keys weigh nothing, and a row of nothing
    else has O = 0, L = -inf and no gradient; the other rows and keys as without them."""
    q, k, v, do = packed_inputs([200], [200], 2, 2, d)
    q[:, :, 0], k[:, :, 0] = 2.0 ** 70, 0
    q[:70, :, 0] = 2.0 ** 90
    k[:100, :, 0] = -(2.0 ** 70)  # 2^160 and 2^140: -inf
    o, lse = dash.attn_packed_fwd(q, k, v, cu_of([200]))
    dq, dk, dv = dash.attn_packed_bwd(q, k, v, o, do, lse, cu_of([200]))
    for x in (o[:100], dq[:100], dk[:100], dv[:100]):
        assert bool((x == 0).all())
    assert bool((lse[:, :100] == -math.inf).all())
    o2, lse2 = dash.attn_packed_fwd(q[100:], k[100:], v[100:], cu_of([100]))
    ref = reference(q[100:], k[100:], v[100:], do[100:], [100], [100], True, 1 / math.sqrt(d))
    assert over(o[100:], ref["o"], ref["to"]) <= 0 and over(lse[:, 100:], ref["lse"], 2e-5 * ref["lse"].abs().clamp(min=1)) <= 0
    # (dQ's first component is 0 times k's)
    for name, got in (("q", dq), ("k", dk), ("v", dv)):
        assert over(got[100:, :, 1:], ref["d" + name][..., 1:], ref["t" + name][..., 1:]) <= 0, "d" + name


def test_thousands_of_sequences():
    """2100 sequences of 0 to 12 tokens: many rounds of the searches and of the chains' order."""
    lens = [(7 * i + i // 13) % 13 for i in range(2100)]
    q, k, v, do = packed_inputs(lens, lens, 4, 2, 64)
    o, lse = dash.attn_packed_fwd(q, k, v, cu_of(lens))
    out = train(q, k, v, do, cu_of(lens), None, True)
    ref = reference(q, k, v, do, lens, lens, True, 1 / math.sqrt(64))
    assert over(o, ref["o"], ref["to"]) <= 0 and over(lse, ref["lse"], 2e-5 * ref["lse"].abs().clamp(min=1)) <= 0
    for name, got in zip("qkv", out):
        assert over(got, ref["d" + name], ref["t" + name]) <= 0, "d" + name


def test_broadcast_heads():
    """K and V of one head read by all through a head stride of 0, gradients for each."""
    lens = [90, 40]
    q, k, v, do = packed_inputs(lens, lens, 4, 1, 128)
    kb, vb = k.expand(-1, 4, -1), v.expand(-1, 4, -1)
    cu = cu_of(lens)
    o, lse = dash.attn_packed_fwd(q, kb, vb, cu)
    got = dash.attn_packed_bwd(q, kb, vb, o, do, lse, cu)
    o2, lse2 = dash.attn_packed_fwd(q, kb.contiguous(), vb.contiguous(), cu)
    want = dash.attn_packed_bwd(q, kb.contiguous(), vb.contiguous(), o2, do, lse2, cu)
    assert torch.equal(o, o2) and all(torch.equal(a, b) for a, b in zip(got, want))


def test_many_sequences_and_heads():
    """More than 64 sequences (two rounds of a wave), empty ones among them; 34 heads over 2."""
    lens = [(37 * i) % 150 for i in range(140)]
    for d, hq, hkv in ((64, 4, 2), (128, 34, 2)):
        q, k, v, do = packed_inputs(lens, lens, hq, hkv, d)
        out = train(q, k, v, do, cu_of(lens), None, True)
        ref = reference(q, k, v, do, lens, lens, True, 1 / math.sqrt(d))
        for name, got in zip("qkv", out):
            assert over(got, ref["d" + name], ref["t" + name]) <= 0, "d" + name


def test_gradients_against_differences():
    """The gradients of sum(O * dO) against central differences of the float64
    definition's forward, along random directions (the forward itself is checked above)."""
    lens, hq, hkv, d, eps = [40, 3, 70], 4, 2, 64, 1e-4
    q, k, v, do = packed_inputs(lens, lens, hq, hkv, d)
    dq, dk, dv = train(q, k, v, do, cu_of(lens), None, True)
    base = [x.double() for x in (q, k, v)]
    for which, grad in ((0, dq), (1, dk), (2, dv)):
        g = torch.Generator(device="cuda")
        g.manual_seed(which)
        for _ in range(3):
            u = torch.randn(base[which].shape, generator=g, device="cuda", dtype=torch.float64)

            def value(sign):
                x = list(base)
                x[which] = x[which] + sign * eps * u
                r = reference(*x, do, lens, lens, True, 1 / math.sqrt(d))
                return (r["o"] * do.double()).sum()

            slope = float((value(1) - value(-1)) / (2 * eps))
            got = float((grad.double() * u).sum())
            # the gradient's bf16 errors (u8 of each value and of P, dS) along a random
            # direction add up like their 2-norm; six times that, and the difference's eps^2
            size = float((grad.double() * u).norm())
            assert abs(got - slope) <= 6 * 4 * 2.0 ** -8 * size + 1e-3


def test_backward_equals_the_dense_backward():
    """Equal lengths, a head each, narrow tiles: dQ is summed over the same KV tiles in the
    same order as by Descending, and has its bits.  dK and dV have them under a full mask;
    under a causal one the dense call visits 128-row query tiles from the last one down but
    the two 64-row blocks of each upwards, so that their sums are ordered differently."""
    for d, causal in ((64, True), (128, True), (128, False)):
        B, H, N = 2, 3, 500
        q, k, v, do = packed_inputs([N] * B, [N] * B, H, H, d)
        o, lse = dash.attn_packed_fwd(q, k, v, cu_of([N] * B), causal=causal)
        got = dash.attn_packed_bwd(q, k, v, o, do, lse, cu_of([N] * B), causal=causal)
        dense = [x.reshape(B, N, H, d).transpose(1, 2).contiguous() for x in (q, k, v, do)]
        od, ld = dash.attn_fwd(*dense[:3], causal)
        want = dash.attn_bwd(*dense[:3], od, dense[3], ld, causal, "descending")
        for a, b in list(zip(got, want))[:1 if causal else 3]:
            assert torch.equal(a.reshape(B, N, H, d).transpose(1, 2).contiguous().view(torch.int16), b.view(torch.int16))


def test_training_step_captured_and_replayed_with_other_lengths():
    """Forward and backward in two graphs on one workspace, replayed in turn with offsets
    that change between replays and eager calls between them: the eager bits every time."""
    d, hq, hkv, T, B = 128, 8, 2, 700, 4
    splits = ([100, 200, 0, 400], [700, 0, 0, 0], [1, 1, 1, 300], [350, 350, 0, 0])
    ws = torch.empty(dash.dash_packed_workspace_size(B, T, T, hq, hkv, d), dtype=torch.uint8, device="cuda")

    def step(b):
        dash.dash_attn_packed_fwd(b["q"], b["k"], b["v"], b["o"], b["lse"], b["cu"])
        dash.dash_attn_packed_bwd(b["q"], b["k"], b["v"], b["o"], b["do"], b["lse"], b["dq"], b["dk"], b["dv"], b["cu"],
                                  workspace=ws)

    def buffers(seed):
        q, k, v, do = packed_inputs([T], [T], hq, hkv, d, seed=seed)
        return dict(q=q, k=k, v=v, do=do, o=torch.zeros_like(q), lse=torch.zeros((hq, T), device="cuda"), dq=torch.zeros_like(q),
                    dk=torch.zeros_like(k), dv=torch.zeros_like(v), cu=cu_of(splits[0]))

    graphs = []
    for seed in (1, 2):
        b = buffers(seed)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            step(b)
        torch.cuda.current_stream().wait_stream(side)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step(b)
        graphs.append((graph, b))
    names = ("o", "lse", "dq", "dk", "dv")
    for lens in splits + splits:
        n = sum(lens)
        for graph, b in graphs:
            b["cu"].copy_(cu_of(lens))
            for x in names:
                b[x].fill_(7)
            graph.replay()
            torch.cuda.synchronize()
            got = {x: b[x].clone() for x in names}
            eager = dict(b, **{x: torch.full_like(b[x], 7) for x in names})
            step(eager)  # eager, on the same workspace, between the replays
            assert dash.dash_bwd_check(ws) == dash.DASH_OK
            assert all(torch.equal(got[x], eager[x]) for x in names)
            assert bool((got["dq"][n:] == 7).all()) and bool((got["dk"][n:] == 7).all())


def test_two_streams_with_their_own_workspaces():
    lens = [300, 1200, 64]
    q, k, v, do = packed_inputs(lens, lens, 8, 2, 128)
    cu = cu_of(lens)
    o, lse = dash.attn_packed_fwd(q, k, v, cu)
    want = dash.attn_packed_bwd(q, k, v, o, do, lse, cu)
    torch.cuda.synchronize()
    n = dash.dash_packed_workspace_size(3, sum(lens), sum(lens), 8, 2, 128)
    work = [(torch.cuda.Stream(), torch.empty(n, dtype=torch.uint8, device="cuda"),
             [[torch.zeros_like(x) for x in want] for _ in range(4)]) for _ in range(2)]
    torch.cuda.synchronize()
    for i in range(4):
        for s, ws, outs in work:
            dash.dash_attn_packed_bwd(q, k, v, o, do, lse, *outs[i], cu, workspace=ws, stream=s)
    torch.cuda.synchronize()
    for _, _, outs in work:
        assert all(torch.equal(a, b) for got in outs for a, b in zip(got, want))


def test_from_prompt_to_answer():
    """As a model's attention layer uses the operators: a prompt's queries and keys rotated
    and its keys stored, attention over the prompt, then tokens one by one over the
    cache.  Each token's output equals the packed forward's over the whole text so far."""
    d, hq, hkv, page, prompt, more = 128, 8, 2, 16, [37, 5, 120], 4
    g = torch.Generator(device="cuda")
    g.manual_seed(9)
    total = [n + more for n in prompt]
    qkv = [torch.randn((n, hq + 2 * hkv, d), generator=g, device="cuda").to(BF) for n in total]
    inv = (10000.0 ** (-torch.arange(0, d, 2, device="cuda") / d)).float()
    width = max(total) // page + 1
    table = torch.arange(3 * width, dtype=torch.int32, device="cuda").reshape(3, width)
    kc, vc = (torch.full((3 * width, hkv, page, d), float("nan"), device="cuda").to(BF) for _ in range(2))
    lens = torch.zeros(3, dtype=torch.int32, device="cuda")
    x = torch.cat([t[:n] for t, n in zip(qkv, prompt)])
    q, k, v = x.split([hq, hkv, hkv], dim=1)
    qr, kr = torch.empty_like(q), torch.empty_like(k)
    cu = cu_of(prompt)
    dash.dash_kv_append(k, v, kc, vc, table, lens, cu=cu, q=q, q_out=qr, k_out=kr, inv_freq=inv)
    lens += torch.tensor(prompt, dtype=torch.int32, device="cuda")
    first, _ = dash.attn_packed_fwd(qr, kr, v, cu)
    answers = []
    for t in range(more):
        x = torch.stack([s[n + t] for s, n in zip(qkv, prompt)])
        q, k, v = x.split([hq, hkv, hkv], dim=1)
        qt = torch.empty_like(q)
        dash.dash_kv_append(k, v, kc, vc, table, lens, q=q, q_out=qt, inv_freq=inv)
        lens += 1
        answers.append(dash.attn_decode(qt, kc, vc, table, lens))
    # the whole texts at once
    x = torch.cat(qkv)
    q, k, v = x.split([hq, hkv, hkv], dim=1)
    qr, kr = torch.empty_like(q), torch.empty_like(k)
    kc2, vc2 = torch.zeros_like(kc), torch.zeros_like(vc)
    cu = cu_of(total)
    dash.dash_kv_append(k, v, kc2, vc2, table, torch.zeros_like(lens), cu=cu, q=q, q_out=qr, k_out=kr, inv_freq=inv)
    whole, _ = dash.attn_packed_fwd(qr, kr, v, cu)
    ref = reference(qr, kr, v, torch.zeros_like(qr), total, total, True, 1 / math.sqrt(d))
    at, a = cu.tolist(), 0
    for s, n in enumerate(prompt):
        rows = slice(at[s], at[s] + n)
        assert over(first[a:a + n], ref["o"][rows], ref["to"][rows]) <= 0
        a += n
        for t in range(more):
            row = at[s] + n + t
            assert over(answers[t][s], ref["o"][row], ref["to"][row]) <= 0
            assert over(whole[row], ref["o"][row], ref["to"][row]) <= 0
