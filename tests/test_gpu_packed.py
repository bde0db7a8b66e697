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
