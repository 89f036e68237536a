"""Paged caches in 64 bits on the CPU, for the tests: seeded sequences, the pool
that holds them, and what append, read-out and attention give. Written from
the operators' definitions with torch's elementary operations; it shares no
code with the library.

Rounding steps: a value rounded to a type is off by at most half a step,
torch.finfo(type).eps / 2 relative to it (bf16 2^-8).
"""
import math

import torch

E2M1 = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64)
HALF_BF16 = 2.0 ** -8
EPS32 = 2.0 ** -24


def e4m3(x):
    """The nearest E4M3 value (ties to even), saturated; NaN stays."""
    y = x.clamp(-448, 448)
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(y / step) * step


def mx_exponent(block):
    """floor(log2(largest)) - 2 of blocks [..., 32], within [-126, 127]."""
    top = block.abs().amax(-1, keepdim=True)
    return torch.where(top > 0, torch.frexp(top).exponent - 3, -126).clamp(-126, 127)


def mx_codes(x):
    """Rows [..., d] -> (code indices with sign bit [..., d], exponents [..., d/32])."""
    y = x.unflatten(-1, (-1, 32))
    e = mx_exponent(y)
    z = y.abs() * torch.exp2(-e.double())
    mid = (E2M1[1:] + E2M1[:-1]) / 2
    i = torch.bucketize(z.contiguous(), mid)
    tie = (i < 7) & (z == mid[i.clamp(max=6)]) & (i % 2 == 1)
    k = i + tie.long() + 8 * torch.signbit(y).long()
    return k.flatten(-2), e.squeeze(-1)


def mx_values(k, e):
    v = E2M1[(k & 7).long()] * torch.where(k > 7, -1.0, 1.0).double()
    return (v.unflatten(-1, (-1, 32)) * torch.exp2(e.double()).unsqueeze(-1)).flatten(-2)


def stored(x, kv, scale=None):
    """(bits, scale bytes or None, values) of rows x [..., g, rows, d] float64."""
    if kv == "bf16":
        b = x.float().to(torch.bfloat16)
        return b, None, b.double()
    if kv == "fp8_e4m3":
        s = torch.ones(x.shape[-3]) if scale is None else scale
        v = e4m3(x / s.double().view(-1, 1, 1))
        return v.float().to(torch.float8_e4m3fn).view(torch.uint8), None, v * s.double().view(-1, 1, 1)
    k, e = mx_codes(x)
    k8 = k.to(torch.uint8)
    return k8[..., 0::2] | (k8[..., 1::2] << 4), (e + 127).to(torch.uint8), mx_values(k, e)


class Problem:
    """Sequences (one context, b own ones) scattered over a pool whose every
    other row and page is poisoned with NaN, tables whose unused entries are
    not page ids."""

    def __init__(self, b, h, g, d, m_c, m_d, n=1, page=16, kv="bf16", maps=1, lens=None, seed=0,
                 spare=3, scaled=True):
        self.__dict__.update(b=b, h=h, g=g, d=d, m_c=m_c, m_d=m_d, n=n, page=page, kv=kv, maps=maps)
        r = torch.Generator().manual_seed(seed)
        self.rng = r
        self.q = torch.randn(b, h, n, d, generator=r).to(torch.bfloat16)
        self.lens = (torch.randint(0, m_d + 1, (b,), generator=r) if lens is None
                     else torch.tensor(lens)).to(torch.int32)
        self.k_scale = self.v_scale = None
        if kv == "fp8_e4m3" and scaled:
            self.k_scale, self.v_scale = (torch.exp2(2 * torch.rand(g, generator=r) - 7) for _ in range(2))
        cp, op = -(-m_c // page), -(-m_d // page)
        self.num_pages = max(1, cp + b * op + spare)
        order = torch.randperm(self.num_pages, generator=r).to(torch.int32)
        self.ctx_table = order[:cp].clone()
        self.tables = order[cp:cp + b * op].view(b, op).clone()
        cols = d // 2 if kv == "mxfp4" else d
        if kv == "bf16":
            self.pool = {x: torch.full((self.num_pages, g, page, cols), float("nan"), dtype=torch.bfloat16)
                         for x in "KV"}
        else:  # 0x7F: NaN in E4M3; MXFP4 rows are poisoned by their scale bytes
            self.pool = {x: torch.full((self.num_pages, g, page, cols), 0x7F, dtype=torch.uint8) for x in "KV"}
        self.exps = ({x: torch.full((self.num_pages, g, page, d // 32), 255, dtype=torch.uint8) for x in "KV"}
                     if kv == "mxfp4" else {"K": None, "V": None})
        self.ctx, self.own = {}, {}
        for x, sc in (("K", self.k_scale), ("V", self.v_scale)):
            self.ctx[x] = self._put(x, torch.randn(1, g, m_c, d, generator=r).double(), self.ctx_table.view(1, -1),
                                    torch.tensor([m_c]), sc)[0]
            self.own[x] = self._put(x, torch.randn(b, g, m_d, d, generator=r).double(), self.tables, self.lens, sc)
        for i in range(b):  # entries past the last valid row are not page ids
            self.tables[i, -(-int(self.lens[i]) // page):] = [-7, 1 << 30][i % 2]

    def _put(self, x, rows, tables, lens, scale):
        bits, exps, values = stored(rows, self.kv, scale)
        for i in range(rows.shape[0]):
            for t in range(int(lens[i])):
                at = int(tables[i, t // self.page]), t % self.page
                self.pool[x][at[0], :, at[1]] = bits[i, :, t]
                if exps is not None:
                    self.exps[x][at[0], :, at[1]] = exps[i, :, t]
        return values

    # what a call takes, on the GPU

    def plan(self, **kw):
        import paper_2403_08845_amd as bif
        return bif.PagedPlan(self.b, self.h, self.g, self.d, self.m_c, self.m_d, page=self.page,
                             num_pages=self.num_pages, n=self.n, kv=self.kv, maps=self.maps, **kw)

    def pages(self):
        import paper_2403_08845_amd as bif

        def dev(t):
            return None if t is None else t.cuda()
        return bif.Pages(dev(self.pool["K"]), dev(self.pool["V"]), dev(self.exps["K"]), dev(self.exps["V"]),
                         dev(self.k_scale), dev(self.v_scale))

    # what it gives

    def attention(self, scale=None, lam=None, weight=None, eps=1e-5, out_scale=1.0, q=None):
        """(out, tolerance) float64 [b, h, n, d]. The library's weights are off by
        2^-15 (two bf16 terms), by its 32-bit logits (d products each, exponent
        and conversions) and by the order of its 32-bit sums over the keys;
        magnitudes are those of the sums' terms. The output is rounded to bf16
        once.

        With codes in the pages and many query rows in a group the context's weights
        are one fp16 term instead: half a step of 2^-10 of each weight, and below
        fp16's normal range (2^-14) half a step of 2^-24, beside a chunk's largest
        weight and sum of 1 at least. MXFP4 values then count relative to the
        largest scale of their 32 elements in a chunk, which enters as 2^8: to half
        a step of 2^-24, 2^-33 of that scale; the largest value there is at least
        4 times it."""
        b, h, g, d, n, m_c, m_d = (getattr(self, k) for k in ("b", "h", "g", "d", "n", "m_c", "m_d"))
        w, p = d // self.maps, h // g
        R, M = self.maps * p * n, self.maps * b * p * n
        one_term = self.kv != "bf16" and (M > 64 or (M > 32 and R <= 32))
        scale = 1 / math.sqrt(w) if scale is None else scale
        q = (self.q if q is None else q).double().view(b, g, p, n, d)
        K, V = (torch.cat((self.ctx[x].expand(b, g, m_c, d), self.own[x]), 2)[:, :, None] for x in "KV")
        pos = torch.arange(m_c + m_d)
        seen = pos < m_c + (self.lens.view(-1, 1, 1) - n + 1 + torch.arange(n).view(-1, 1)).clamp(min=0)
        seen = seen[:, None, None]  # [b, 1, 1, n, keys]
        V = torch.where((pos < m_c + self.lens.view(-1, 1))[:, None, None, :, None], V, 0.0)
        maps = []
        for u in range(self.maps):
            f = slice(u * w, (u + 1) * w)
            x = torch.where(seen, scale * (q[..., f] @ K[..., f].transpose(-1, -2)), -math.inf)
            size = (torch.where(seen, abs(scale) * (q[..., f].abs() @ K[..., f].abs().transpose(-1, -2)), 0.0)
                    .amax(-1, keepdim=True))
            top = x.amax(-1, keepdim=True)
            e = torch.exp(x - torch.where(top == -math.inf, 0.0, top))
            total = e.sum(-1, keepdim=True)
            e = torch.where(total > 0, e / total, 0.0)
            tau = 2.0 ** -15 + (2.0 ** -11 if one_term else 0.0) + EPS32 * (2 * (m_c + m_d) + 4 * (w + 16) * (size + 1))
            less = torch.zeros(())
            if one_term and m_c:
                less = 2.0 ** -25 * self.ctx["V"].abs().sum(1)[:, None, None]
                if self.kv == "mxfp4":
                    top = self.ctx["V"].abs().amax(1).unflatten(-1, (-1, 32)).amax(-1).repeat_interleave(32, -1)
                    less = less + 2.0 ** -35 * top[:, None, None]
            maps.append((e @ V, tau * (e @ V.abs()) + torch.where(total > 0, less, 0.0)))
        y, err = maps[0]
        if self.maps == 2:
            lam = lam.double().view(g, p, 1, 1)
            y, err = y - lam * maps[1][0], err + lam.abs() * maps[1][1] + 4 * EPS32 * (y.abs() + (lam * maps[1][0]).abs())
            if weight is not None:
                r = torch.sqrt(y.square().mean(-1, keepdim=True) + eps)
                err = (err + y.abs() * err.square().mean(-1, keepdim=True).sqrt() / r) / r * weight.double().abs()
                y = y / r * weight.double()
            y, err = y * out_scale, err * abs(out_scale)
        return y.reshape(b, h, n, d), (HALF_BF16 * y.abs() + (1 + HALF_BF16) * err + 1e-30).reshape(b, h, n, d)


def rotated(x, position, freqs, neighbours, maps):
    """Rows x [..., d] float64 at positions [...] (broadcast): each part of d/maps
    has its first 2 len(freqs) elements rotated."""
    x = x.double().clone()
    half = freqs.numel()
    i = torch.arange(half)
    i, j = (2 * i, 2 * i + 1) if neighbours else (i, i + half)
    turns = position.double().unsqueeze(-1) * (freqs.double() / (2 * math.pi))
    a = 2 * math.pi * (turns - turns.round())
    c, s = a.cos(), a.sin()
    for u in range(maps):
        o = u * x.shape[-1] // maps
        lo, hi = x[..., o + i].clone(), x[..., o + j].clone()
        x[..., o + i], x[..., o + j] = lo * c - hi * s, lo * s + hi * c
    return x
