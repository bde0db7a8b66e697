"""Packed attention in float64, forward and backward from the definition, one sequence
and head at a time, with bounds on the kernels' errors."""
import math

import torch

U8, U24 = 2.0 ** -8, 2.0 ** -24
BF = torch.bfloat16


def cu_of(lens):
    at = [0]
    for n in lens:
        at.append(at[-1] + n)
    return torch.tensor(at, dtype=torch.int32, device="cuda")


def packed_inputs(qlens, klens, hq, hkv, d, layout="packed", tail=0, seed=0, spread=1.0):
    """q, k, v, dO of the given lengths with `tail` rows of NaN behind the last sequence.
    layout: "packed" [T, H, d]; "fused": views into one [T, hq + 2 hkv, d] (equal lengths only);
    "heads": [H, T, d] in memory."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed + d + hq + sum(qlens))
    tq, tk = sum(qlens) + tail, sum(klens) + tail

    def normal(t, h):
        if layout == "heads":
            return torch.randn((h, t, d), generator=g, device="cuda").to(BF).transpose(0, 1)
        return torch.randn((t, h, d), generator=g, device="cuda").to(BF)

    if layout == "fused":
        assert qlens == klens
        q, k, v = normal(tq, hq + 2 * hkv).split([hq, hkv, hkv], dim=1)
    else:
        q, k, v = normal(tq, hq), normal(tk, hkv), normal(tk, hkv)
    q.mul_(spread)
    do = normal(tq, hq)
    for x, n in ((q, sum(qlens)), (k, sum(klens)), (v, sum(klens)), (do, sum(qlens))):
        x[n:] = float("nan")
    return q, k, v, do


def visible(m, n, causal):
    see = torch.ones((m, n), dtype=torch.bool, device="cuda")
    return see.tril(n - m) if causal else see


def reference(q, k, v, do, qlens, klens, causal, scale):
    """float64 o [Tq, hq, d], lse [hq, Tq], dq, dk, dv, and bounds on |o - got| and the
    gradients' magnitudes (see bounds in the tests)."""
    hq, hkv, d = q.shape[1], k.shape[1], q.shape[2]
    G = hq // hkv
    Q, K, V, dO = (x.double().nan_to_num() for x in (q, k, v, do))
    out = {n: torch.zeros_like(x) for n, x in (("o", Q), ("dq", Q), ("dk", K), ("dv", K), ("to", Q), ("tq", Q), ("tk", K), ("tv", K))}
    lse = torch.full((hq, q.shape[0]), -math.inf, dtype=torch.float64, device="cuda")
    a = x = 0
    for m, n in zip(qlens, klens):
        b, y = a + m, x + n
        if m and n:
            see = visible(m, n, causal)
            some = see.any(-1, keepdim=True)
            for h in range(hq):
                qq, kk, vv, dd = Q[a:b, h], K[x:y, h // G], V[x:y, h // G], dO[a:b, h]
                s = (qq @ kk.t()).mul(scale).masked_fill(~see, -math.inf)
                lse[h, a:b] = torch.logsumexp(s, -1)
                p = torch.softmax(s, -1).masked_fill(~some, 0.0)
                o = p @ vv
                dp = dd @ vv.t()
                D = (dd * o).sum(-1, keepdim=True)
                ds = p * (dp - D)
                out["o"][a:b, h] = o
                out["dq"][a:b, h] = ds @ kk * scale
                out["dk"][x:y, h // G] += ds.t() @ qq * scale
                out["dv"][x:y, h // G] += p.t() @ dd
                # errors.  es: of a score (fp32 sums of d products), which moves P by as
                # much; el: of L, the same.  P and dS are rounded to bf16 once each.
                es = (d + 4) * U24 * scale * (qq.abs() @ kk.abs().t())
                es = es.masked_fill(~see, 0.0)
                ep = 2 * es.amax(-1, keepdim=True) + 2 * (n + 8) * U24 + 4 * U24 * lse[h, a:b, None].abs().nan_to_num(posinf=0.0)
                out["to"][a:b, h] = U8 * o.abs() + (U8 * (1 + U8) + 2 * ep) * (p @ vv.abs())
                # D from the bf16 O: rounded once more, off by the forward's error
                eD = (dd.abs() * (out["to"][a:b, h] + d * U24 * o.abs())).sum(-1, keepdim=True)
                eds = p * (ep * (dp - D).abs() + eD + (d + 4) * U24 * (dd.abs() @ vv.abs().t()) + 2 * U24 * (dp.abs() + D.abs()))
                eds = eds + U8 * (1 + U8) * (ds.abs() + eds)
                # fp32 sums over keys and queries
                out["tq"][a:b, h] = (eds @ kk.abs() + (n + 8) * U24 * (ds.abs() @ kk.abs())) * scale + U8 * out["dq"][a:b, h].abs()
                out["tk"][x:y, h // G] += (eds.t() @ qq.abs() + (m * G + 8) * U24 * (ds.abs().t() @ qq.abs())) * scale
                out["tv"][x:y, h // G] += ((U8 * (1 + U8) + ep) * p).t() @ dd.abs() + (m * G + 8) * U24 * (p.t() @ dd.abs())
        a, x = b, y
    out["tk"] += U8 * out["dk"].abs()
    out["tv"] += U8 * out["dv"].abs()
    for t in ("to", "tq", "tk", "tv"):
        out[t] = out[t] * (1 + U8)
    out["lse"] = lse
    return out


def over(got, want, bound):
    """The largest excess of |got - want| over its bound (<= 0: none); NaN counts as infinite."""
    e = (got.double() - want).abs() - bound
    return float(e.nan_to_num(nan=math.inf).max()) if e.numel() else 0.0
