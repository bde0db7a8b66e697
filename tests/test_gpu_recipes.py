"""README's recipe of long contexts as it stands there, on the GPU: it serves what it trains."""
import math
import os

import pytest
import torch

import paper_2601_21824_amd as dash
from mx_util import BF, Cache
from test_gpu_mx_cache import KINDS, attend64, offsets
from test_gpu_paged_cache import i32, table_of
from test_gpu_rotary import bound, rotate64

pytestmark = pytest.mark.gpu

U8 = 2.0 ** -8


def recipe():
    text = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "README.md")).read()
    blocks = [b.split("```")[0] for b in text.split("```python\n")[1:]]
    (found,) = [b for b in blocks if "dash_rotary_frequencies" in b]
    return found


def test_long_contexts():
    """Queries and the cached keys have the frequencies and the amplitude of the training's rotation: q to the rotary call's bound; keys as
    MXFP8 holds them beside that, 2^-4 of themselves or, where they are small, 2^-10 of a scale of at most 2 max / 448, and one
    rounding to bf16 before it."""
    d, hq, hk, page = 128, 8, 2, 16
    old, new, prefix = [300, 203, 200], [40, 1, 77], 200  # (old: the first part of the prompts; three sequences share 200 keys of it)
    lens = [a + b for a, b in zip(old, new)]
    table, pages = table_of(lens, page)
    table[:, :prefix // page] = table[0, :prefix // page]
    T = sum(new)
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    random = lambda *s: torch.randn(s, generator=g, device="cuda").to(BF)  # noqa: E731
    q, k, v, dqr, dkr, q_new = random(T, hq, d), random(T, hk, d), random(T, hk, d), random(T, hq, d), random(T, hk, d), random(3, hq, d)
    c = Cache("mxfp8", pages, hk, page, d)
    names = dict(torch=torch, dash=dash, q=q, k=k, v=v, dqr=dqr, dkr=dkr, q_new=q_new, k_cache=c.k, v_cache=c.v, k_scale=c.k_scale,
                 v_scale=c.v_scale, block_table=table, cu=i32(offsets(new)), cu_all=i32(offsets(lens)), rows=sum(lens), lens=i32(old),
                 lens_after_append=i32(lens), prefix_table=table[0, :-(-prefix // page)].contiguous(), prefix_len=i32([prefix]))
    q0, k0 = q.clone(), k.clone()
    exec(recipe(), names)
    inv, amp = names["inv_freq"], names["amplitude"]
    assert amp > 1.2
    place = torch.cat([torch.arange(o, o + n) for o, n in zip(old, new)]).cuda()
    rq, rk = (rotate64(x, place, inv, False, amp) for x in (q0, k0))
    assert bool(((names["q"].double() - rq).abs() <= bound(q0, rq, inv, False, amp)).all())
    at = offsets(lens)
    stored = torch.cat([names["k_all"][at[s] + o:at[s + 1]] for s, o in enumerate(old)]).double()
    most = rk.abs().amax(-1, keepdim=True)
    assert bool(((stored - rk).abs() <= (2.0 ** -4 + U8 * (1 + 2.0 ** -4)) * rk.abs() + 2.0 ** -9 * most / 448 + bound(k0, rk, inv, False, amp)).all())
    # what is trained is what is served, to the rounding of the storage: places from 0 on, the same turns
    tq, tk = (rotate64(x, torch.cat([torch.arange(n) for n in new]).cuda(), inv, False, amp) for x in (q0, k0))
    assert bool(((names["qr"].double() - tq).abs() <= bound(q0, tq, inv, False, amp)).all())
    assert bool(((names["kr"].double() - tk).abs() <= bound(k0, tk, inv, False, amp)).all())
    assert all(bool(names[x].isfinite().all()) for x in ("o", "lse", "dq", "dk"))


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("rotary", [128, 64])
def test_a_context_by_parts_served_as_it_is_trained(rotary, kind):
    """The amplitude turns with the rotated components alone: rotated and then stored, a step of one token agrees with the last row
    of the attention over the same rows (those that the cache holds), both to their bounds; and with float64 on the definition's rotation,
    q and k rounded to bf16 once (u8 each, so that scores move by 2 u8 |q| |k|, and P by twice that)."""
    d, hq, hk, page, lens = 128, 8, 2, 16, [700, 1, 48]
    inv, amp = dash.dash_rotary_frequencies(rotary, scaling="parts", factor=8, original=64)
    inv = torch.from_numpy(inv).cuda()
    g = torch.Generator(device="cuda")
    g.manual_seed(rotary)
    T, at = sum(lens), offsets(lens)
    q, k, v = (torch.randn((T, h, d), generator=g, device="cuda").to(BF) for h in (hq, hk, hk))
    qr, kr = dash.rotary(q, k, inv, cu=i32(at), amplitude=amp)
    table, pages = table_of(lens, page)
    c = Cache(kind, pages, hk, page, d)
    dash.dash_kv_append(kr, v, *c.pools, table, i32([0, 0, 0]), cu=i32(at), **c.scales)
    k_all, v_all = dash.kv_read(*c.pools, table, i32(lens), i32(at), T, **c.scales)
    if kind == "bf16":
        assert torch.equal(k_all, kr) and torch.equal(v_all, v)
    last = torch.tensor(at[1:], device="cuda") - 1
    o, _ = dash.attn_packed_fwd(qr, k_all, v_all, i32(at))
    one = dash.attn_decode(qr[last].contiguous(), *c.pools, table, i32(lens), **c.scales)
    _, _, tol = attend64(c, qr[last], table, lens, 1 / math.sqrt(d))
    if kind != "e4m3":  # (read back, that type's values times their scale are rounded)
        assert bool(((one.double() - o[last].double()).abs() <= 2.1 * tol).all())
    if kind != "bf16":
        return
    place = torch.cat([torch.arange(n) for n in lens]).cuda()
    q64, k64 = (rotate64(x, place, inv, False, amp) for x in (q, k))
    for s, n in enumerate(lens):
        own = slice(at[s], at[s + 1])
        qs, ks, vs = q64[at[s + 1] - 1].reshape(hk, hq // hk, d), k64[own].transpose(0, 1), v[own].double().transpose(0, 1)
        p = torch.softmax(qs @ ks.transpose(1, 2).contiguous() / math.sqrt(d), -1)
        move = 2 * U8 * (qs.abs() @ ks.abs().transpose(1, 2).contiguous()).amax(-1, keepdim=True) / math.sqrt(d)
        a = (p @ vs.abs()) * (torch.expm1(2 * move * (1 + U8)) + 0.0)
        assert bool(((one[s].double().reshape(hk, hq // hk, d) - p @ vs).abs() <= tol[s].reshape(hk, hq // hk, d) + a).all())


@pytest.mark.parametrize("at", [[0, 10, 4], [0, 10, 4, 12], [5, 3], [0, 6, 6, 12]])
def test_offsets_that_fall(at):
    """The rotation and the read each report exactly when they leave a row of cu[0] .. cu[-1] - 1 alone (where offsets fall, two sequences
    may claim a row, and which of them it goes to, if any, is the call's own); rows outside those are nobody's, whatever an earlier
    sequence's end says, and are left alone."""
    d, rows, batch = 64, 12, len(at) - 1
    x = torch.ones((rows, 2, d), device="cuda").to(BF)
    out, s1, s2 = torch.full_like(x, 7.0), i32([0]), i32([0])
    inv = (10000.0 ** (-torch.arange(0, d, 2, device="cuda") / d)).float()
    dash.dash_rotary(x, None, out, None, inv, cu=i32(at), status=s1)
    table, pages = table_of([16] * batch, 16)
    c = Cache("bf16", pages, 2, 16, d)
    k, v = torch.full_like(x, 7.0), torch.full_like(x, 7.0)
    dash.dash_kv_read(*c.pools, table, i32([16] * batch), i32(at), k, v, status=s2)
    for status, ys in ((s1, [out]), (s2, [k, v])):
        for y in ys:
            left = (y == 7).flatten(1).all(-1)
            assert int(status) == int(left[at[0]:at[-1]].any()) and bool(left[:at[0]].all()) and bool(left[max(at[0], at[-1]):].all())
    for r in range(min(at[-1], 4) if at[0] == 0 else 0):  # (of sequence 0 alone)
        assert torch.equal(k[r], c.k[int(table[0, 0]), :, r]) and not bool((out[r] == 7).all())
