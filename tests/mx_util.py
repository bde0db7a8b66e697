"""Microscaled rows from their definition, in 64 bits, and paged caches of every type for the tests."""
import torch

BF, E4, U8T = torch.bfloat16, torch.float8_e4m3fn, torch.uint8


def grid(kind):
    """Magnitudes of the element type in the order of their codes."""
    if kind == "mxfp4":
        return torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64)
    return torch.tensor([(c & 7) / 8 * 2.0 ** -6 if c < 8 else (1 + (c & 7) / 8) * 2.0 ** ((c >> 3) - 7) for c in range(127)],
                        dtype=torch.float64)


def quantise64(x, kind):
    """fp32 values [..., d] -> codes uint8 [..., d] (sign and magnitude), scale bytes [..., d / 32]."""
    g = grid(kind).to(x.device)
    sign = 8 if kind == "mxfp4" else 128
    b = x.double().unflatten(-1, (-1, 32))
    odd = ~b.isfinite().all(-1, keepdim=True)
    b = torch.where(odd, torch.zeros_like(b), b)
    most = b.abs().amax(-1, keepdim=True).clamp(max=1.5 * 2.0 ** 127)
    e = torch.full_like(most, -117.0)
    for _ in range(260):  # the least exponent that holds the block
        e = torch.where(most > g[-1] * torch.exp2(e), e + 1, e)
    y = b.abs() / torch.exp2(e)
    mid = (g[1:] + g[:-1]) / 2
    code = torch.bucketize(y, mid)  # ties go down ...
    tie = torch.cat((mid, mid[-1:] * 4))[code.clamp(max=mid.numel())] == y
    code = torch.where(tie & (code % 2 == 1), code + 1, code)  # ... or up to the even code
    code = (code + sign * torch.signbit(b)).to(U8T)
    byte = torch.where(odd, torch.full_like(e, 255), e + 127).to(U8T)
    return code.flatten(-2), byte[..., 0], odd[..., 0]


def pack(codes, kind):
    """Codes -> what a cache holds."""
    return codes.view(E4) if kind == "mxfp8" else codes[..., 0::2] + 16 * codes[..., 1::2]


def values64(elements, byte, kind):
    """What cached elements stand for: [..., d] float64 (NaN for a scale byte of 255)."""
    if kind == "mxfp4":
        c = torch.stack((elements & 15, elements >> 4), dim=-1).flatten(-2).long()
        g = grid(kind).to(c.device)
        v = torch.cat((g, -g))[c]
    else:
        v = elements.view(E4).double() if elements.dtype is U8T else elements.double()
    s = torch.where(byte == 255, torch.full(byte.shape, float("nan"), dtype=torch.float64, device=byte.device),
                    torch.exp2(byte.double() - 127))
    return (v.unflatten(-1, (-1, 32)) * s[..., None]).flatten(-2)


class Cache:
    """A pool of pages in one of the four types, its memory laid out in `order` of (p)ages, (h)eads, (r)ows, (d)."""

    def __init__(self, kind, pages, hkv, page, d, order="phrd", seed=0, spread=1.0):
        self.kind, self.page, self.d = kind, page, d
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        size = {"p": pages, "h": hkv, "r": page, "d": d}
        x, y = (torch.randn([size[c] for c in "phrd"], generator=g, device="cuda") * spread for _ in range(2))
        self.k_scale = self.v_scale = None
        laid = lambda t: t.permute([("phrd").index(c) for c in order]).contiguous().permute([order.index(c) for c in "phrd"])  # noqa: E731
        if kind == "bf16":
            self.k, self.v = laid(x.to(BF)), laid(y.to(BF))
        elif kind == "e4m3":
            self.k_scale, self.v_scale = (torch.linspace(0.3, 0.9, hkv, device="cuda") * f for f in (1.0, 1.5))
            self.k, self.v = (laid(t.clamp(-448, 448).to(E4).view(U8T)).view(E4) for t in (x, y))
        else:
            (a, self.k_scale, _), (b, self.v_scale, _) = (quantise64(t, kind) for t in (x, y))
            self.k, self.v = (laid(pack(t, kind).view(U8T)) for t in (a, b))
            if kind == "mxfp8":
                self.k, self.v = self.k.view(E4), self.v.view(E4)

    @property
    def scales(self):
        return {"k_scale": self.k_scale, "v_scale": self.v_scale}

    @property
    def pools(self):
        return self.k, self.v

    def all64(self):
        """Every row of K and V in float64 [pages, heads, page, d]."""
        out = []
        for c, s in ((self.k, self.k_scale), (self.v, self.v_scale)):
            if self.kind == "bf16":
                out.append(c.double())
            elif self.kind == "e4m3":
                out.append(c.double() * s.double()[:, None, None])
            else:
                out.append(values64(c, s, self.kind))
        return out

    def rows64(self, table, s, n):
        ids = table[s, :-(-n // self.page)].long()
        return [x[ids].transpose(0, 1).flatten(1, 2)[:, :n] for x in self.all64()]

    def spoil(self, used):
        """NaN wherever no sequence's key is: used [pages, page]."""
        off = ~used
        for c, s in ((self.k, self.k_scale), (self.v, self.v_scale)):
            t = (c if self.kind == "bf16" else c.view(U8T)).transpose(1, 2)
            t[off] = float("nan") if self.kind == "bf16" else 0x7F
            if self.kind.startswith("mx"):
                s.transpose(1, 2)[off] = 255


def used_rows(table, lens, page, pages):
    used = torch.zeros((pages, page), dtype=torch.bool, device="cuda")
    for s, n in enumerate(lens):
        for i in range(-(-n // page)):
            used[int(table[s, i]), :min(page, n - i * page)] = True
    return used
