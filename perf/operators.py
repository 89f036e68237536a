"""The paged-cache operators: append with rotation, read-out, attention, differential attention.

A case is one call (or one generation step of two calls) of one layer, as a serving program makes it: the
caches of all sequences lie in one pool of pages, [pages][g][page][d], which a table per sequence names in
any order; the samples share the m_c rows of one context and own up to m_d rows each. Pools hold bf16, fp8
E4M3 codes with a scale per group, or MXFP4 (4-bit E2M1 codes, two a byte, one power-of-two scale byte per
32 elements).

Fields of a case: op; b samples, h query heads, g KV groups, d elements of a row, m_c context rows, m_d row
capacity of a sample, n new tokens per sample, page rows of a page, kv element type, ragged (each sample's
length its own). append: rot rotated elements of a head, pairs ("halves" or "neighbours" rotate together),
context (the rows go to the shared context: a prompt), padded (each sample has its own number of new tokens,
at most n). diff: norm (heads are normalised).
"""
import math

import torch

own = False

CODE_BITS = {"bf16": 16, "fp8_e4m3": 8, "mxfp4": 4}
SIGMAS = 4.5  # fp8: standard deviations at the largest code
E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _case(op, b, h, g, d, m_c, m_d, n=1, page=64, kv="bf16", ragged=False, rot=0, pairs="halves", context=False, padded=False, norm=False, **name):
    return dict(name, op=op, b=b, h=h, g=g, d=d, m_c=m_c, m_d=m_d, n=n, page=page, kv=kv, ragged=ragged, rot=rot, pairs=pairs,
                context=context, padded=padded, norm=norm)


def listed():
    return [
        # a 7B-shaped multi-head layer's generation step: one token of each of 32 samples
        _case("append", 32, 32, 32, 128, 8192, 512, rot=128, ragged=True, name="append_mha7b_b32"),
        # an 8k prompt of a grouped layer written into the context's 4-bit pages, and read back
        _case("append", 1, 32, 8, 128, 8192, 0, n=8192, kv="mxfp4", rot=128, context=True, name="append_prompt_8k_mxfp4"),
        # odd draft lengths behind a far context, part of a head rotated, neighbours paired
        _case("append", 37, 16, 4, 64, 262144, 300, n=5, page=16, kv="mxfp4", rot=32, pairs="neighbours", ragged=True, padded=True,
              name="append_padded_far_mxfp4"),
        # a toy layer: latency and launches only
        _case("decode", 4, 4, 4, 64, 128, 16, page=16, name="decode_tiny_b4_mc128"),
        # the 7B-shaped layer, 32 completions of an 8k prompt
        _case("decode", 32, 32, 32, 128, 8192, 512, name="decode_mha7b_b32_mc8k"),
        _case("decode", 32, 32, 32, 128, 8192, 512, kv="mxfp4", name="decode_mha7b_b32_mc8k_mxfp4"),
        # a multi-query layer, 128 completions of a 16k prompt
        _case("decode", 128, 32, 1, 128, 16384, 512, page=128, kv="fp8_e4m3", name="decode_mqa_b128_mc16k_fp8"),
        # a grouped layer, 256 completions of a 32k prompt that end at different lengths
        _case("decode", 256, 32, 8, 128, 32768, 1024, kv="mxfp4", ragged=True, name="decode_gqa8_b256_mc32k_mxfp4"),
        # sequences that share nothing, from empty ones to 4k rows, small pages
        _case("decode", 48, 32, 8, 128, 0, 4096, page=16, ragged=True, name="decode_gqa8_b48_own4k"),
        # differential heads (two maps over halves of 64): 32 completions of an 8k prompt
        _case("diff", 32, 16, 16, 128, 8192, 512, norm=True, name="diff_h16_b32_mc8k"),
        # grouped differential heads over 4-bit pages
        _case("diff", 64, 16, 4, 128, 16000, 384, kv="mxfp4", ragged=True, norm=True, name="diff_gqa4_b64_mc16k_mxfp4"),
        # a whole generation step of a small odd batch with 4 draft tokens: append, then attend
        _case("step", 5, 32, 8, 128, 3001, 200, n=4, page=32, kv="fp8_e4m3", rot=128, ragged=True, name="step_gqa8_b5_mc3001_fp8"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """A call between the listed ones, no dearer than the largest of its kind."""
    while True:
        op = rng.choice(("append", "append", "decode", "decode", "decode", "diff", "diff", "step"))
        limit = max(_cost(c) for c in listed() if c["op"] == ("decode" if op == "step" else op))
        h = rng.choice((4, 8, 12, 16, 32, 40))
        g = rng.choice([x for x in (1, 2, 4, 8, h) if h % x == 0])
        d = rng.choice((64, 128, 128))
        page = rng.choice((16, 32, 64, 128, 256))
        kv = rng.choice(("bf16", "fp8_e4m3", "mxfp4"))
        ragged = rng.random() < 0.6
        pairs, rot = rng.choice(("halves", "neighbours")), rng.choice((d, d, d // 2, d // 4, 0))
        if op == "append" and rng.random() < 0.5:  # a prompt, or a piece of one
            n = _log_int(rng, 1, 8192)
            c = _case(op, 1, h, g, d, n + rng.choice((0, rng.randint(0, 4096))), 0, n, page, kv, False, rot, pairs, context=True)
        elif op == "append":
            n = _log_int(rng, 1, 64)
            c = _case(op, _log_int(rng, 1, 256), h, g, d, _log_int(rng, 1, 1 << 20), n + _log_int(rng, 1, 500), n, page, kv, ragged, rot, pairs,
                      padded=rng.random() < 0.4)
        else:
            n = rng.choice((1, 1, 1, 2, 3, 4, 8))
            m_c = 0 if rng.random() < 0.15 else _log_int(rng, 1, 32768)
            m_d = _log_int(rng, 1, 1024 if m_c else 4096) + (n if op == "step" else 0)
            c = _case(op, _log_int(rng, 1, 256), h, g, d, m_c, m_d, n, page, kv, ragged, rot if op == "step" else 0, pairs if op == "step" else "halves",
                      norm=op == "diff" and rng.random() < 0.7)
        rows = c["b"] * h * c["n"] * (2 if op == "diff" else 1)
        if op != "append" and (h // g * n * (2 if op == "diff" else 1) > 64 or rows * (c["m_c"] + c["m_d"]) > 3e8):
            continue
        if c["b"] * c["m_d"] * g * d <= 3e8 and _cost(c) <= limit:
            return c


def _row_bytes(c):
    return c["d"] * CODE_BITS[c["kv"]] / 8 + (c["d"] / 32 if c["kv"] == "mxfp4" else 0)


def work(case):
    """append: the new rows read, rotated q and the encoded rows written (and, where the rows are read back, the
    encoded ones read and the bf16 ones written). Attention: one copy of the context, every sample's own rows,
    q and the tables read once, the outputs written once; the products of q and K and of the weights and V."""
    c = case
    b, h, g, d, n = (c[k] for k in ("b", "h", "g", "d", "n"))
    total, flops = 0, 0
    if c["op"] in ("append", "step"):
        rows = b * (n / 2 if c["padded"] else n)
        total += rows * ((h + 2 * g) * d * 2 + h * d * 2 + 2 * g * _row_bytes(c))
        flops += rows * (h + g) * c["rot"] * 3
        if c["kv"] == "mxfp4" and c["op"] == "append":
            total += rows * 2 * g * (_row_bytes(c) + d * 2)
    if c["op"] != "append":
        mean = (_least(c) + c["m_d"]) / 2 if c["ragged"] else c["m_d"]
        keys = c["m_c"] + b * mean
        total += 2 * g * keys * _row_bytes(c) + 4 * b * h * n * d + 4 * keys / c["page"]
        flops += (6 if c["op"] == "diff" else 4) * b * h * n * d * max(0, c["m_c"] + mean - (n - 1) / 2)
    return {"bytes": total, "flops": flops}


def _cost(c):
    w = work(c)
    return max(w["bytes"] / 5e12, w["flops"] / 1e15)


def _least(c):
    """Shortest length of a sample after the step: a step's own rows are among them."""
    return c["n"] if c["op"] == "step" else 0


def _grid(x):
    """The E2M1 value nearest to each |x|, as an index; ties to the even one, 6 at most."""
    y = x.abs()
    i = torch.where(y < 2, (y * 2).round(), torch.where(y < 4, y.round() + 2, (y / 2).round() + 4))
    return i.clamp_(max=7).to(torch.uint8)


def _to_mxfp4(x):
    """Rows [..., d] as codes [..., d/2] and scale bytes [..., d/32]."""
    y = x.unflatten(-1, (-1, 32))
    e = (torch.frexp(y.abs().amax(-1, keepdim=True)).exponent - 3).clamp_(-126, 127)
    e = torch.where(y.abs().amax(-1, keepdim=True) > 0, e, -126)
    y = torch.ldexp(y, -e)
    k = (_grid(y) | (torch.signbit(y).to(torch.uint8) << 3)).flatten(-2)
    return k[..., 0::2] | (k[..., 1::2] << 4), (e[..., 0] + 127).to(torch.uint8)


def _to_codes(x, kv, scale=None):
    """Rows [..., g, rows, d] as stored bits (and scale bytes)."""
    if kv == "mxfp4":
        return _to_mxfp4(x)
    if kv == "fp8_e4m3":
        return (x / scale.to(x.dtype).view(-1, 1, 1)).clamp_(-448, 448).float().to(torch.float8_e4m3fn).view(torch.uint8), None
    return x.to(torch.bfloat16), None


def _pool(c, gen, pages):
    """Pages of unit normal rows."""
    g, d, page = c["g"], c["d"], c["page"]
    scale = None
    if c["kv"] == "fp8_e4m3":  # groups differ by up to 2x either way
        scale = torch.exp2(2 * torch.rand(g, generator=gen, device="cuda") - 1) * (SIGMAS / 448)
    cols = d // 2 if c["kv"] == "mxfp4" else d
    bits = torch.empty(pages, g, page, cols, device="cuda", dtype=torch.bfloat16 if c["kv"] == "bf16" else torch.uint8)
    exps = torch.empty(pages, g, page, d // 32, device="cuda", dtype=torch.uint8) if c["kv"] == "mxfp4" else None
    step = max(1, (1 << 25) // (g * page * d))
    for p in range(0, pages, step):
        q = min(pages, p + step)
        x = torch.randn(q - p, g, page, d, generator=gen, device="cuda", dtype=torch.bfloat16).float()
        k, e = _to_codes(x * (448 / SIGMAS * scale.view(-1, 1, 1)) if scale is not None else x, c["kv"], scale)
        bits[p:q].copy_(k)
        if exps is not None:
            exps[p:q].copy_(e)
    return bits, exps, scale


def _inputs(c, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    b, h, g, d, n, m_c, m_d, page = (c[k] for k in ("b", "h", "g", "d", "n", "m_c", "m_d", "page"))
    s = {}
    ctx_pages = 0 if c["op"] == "append" and not c["context"] else -(-m_c // page)
    own_pages = -(-m_d // page)
    pages = max(1, ctx_pages + b * own_pages)
    for x in ("K", "V"):
        s[x], s[x + "_exp"], s["k_scale" if x == "K" else "v_scale"] = _pool(c, gen, pages)
    order = torch.randperm(pages, generator=gen, device="cuda").to(torch.int32)  # pages in the order that they came free
    s["ctx_table"] = order[:ctx_pages].clone()
    s["tables"] = order[ctx_pages:ctx_pages + b * own_pages].view(b, own_pages).clone()
    if c["context"]:
        s["lens"] = torch.full((1,), m_c - n, dtype=torch.int32, device="cuda")
    elif c["ragged"]:
        s["lens"] = torch.randint(_least(c), m_d + 1 - (n if c["op"] == "append" else 0), (b,), generator=gen, device="cuda", dtype=torch.int32)
    else:
        s["lens"] = torch.full((b,), m_d - (n if c["op"] == "append" else 0), dtype=torch.int32, device="cuda")
    if c["op"] == "step":
        s["lens"] -= n
    if c["op"] in ("append", "step"):
        # the layer's one projection of its new tokens: q, k and v rows side by side
        x = torch.randn(b, n, h + 2 * g, d, generator=gen, device="cuda", dtype=torch.bfloat16).transpose(1, 2)
        s["q"], s["k"], s["v"] = x[:, :h], x[:, h:h + g], x[:, h + g:]
        j = torch.arange(c["rot"] // 2, device="cuda", dtype=torch.float64)
        s["freqs"] = (10000.0 ** (-2 * j / max(1, c["rot"]))).float() if c["rot"] else None
        s["counts"] = torch.randint(0, n + 1, (b,), generator=gen, device="cuda", dtype=torch.int32) if c["padded"] else None
        s["q_out"] = torch.zeros(b, h, n, d, dtype=torch.bfloat16, device="cuda")
        s["lens_out"] = torch.zeros_like(s["lens"])
    else:
        s["q"] = torch.randn(b, h, n, d, generator=gen, device="cuda", dtype=torch.bfloat16)
    if c["op"] == "append" and c["kv"] == "mxfp4":
        s["k_back"], s["v_back"] = (torch.zeros(b, g, n, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    if c["op"] == "diff":
        s["lam"] = 0.2 + 0.6 * torch.rand(h, generator=gen, device="cuda")
        s["weight"] = 1 + 0.1 * torch.randn(d, generator=gen, device="cuda") if c["norm"] else None
        s["out_scale"] = 0.2
    s["out"] = torch.empty(b, h, n, d, dtype=torch.bfloat16, device="cuda")
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = dict(case)
    if own:
        import paper_2403_08845_amd as bif
        c = case
        s["plan"] = bif.PagedPlan(c["b"], c["h"], c["g"], c["d"], c["m_c"], c["m_d"], page=c["page"], num_pages=s["K"].shape[0],
                                  n=1 if c["op"] == "append" else c["n"], kv=c["kv"], maps=2 if c["op"] == "diff" else 1)
        s["pages"] = bif.Pages(s["K"], s["V"], s["K_exp"], s["V_exp"], s["k_scale"], s["v_scale"])
    return s


def run(state):
    s, c = state, state["case"]
    if own:
        _own(s, c)
    else:
        if c["op"] in ("append", "step"):
            _append(s, c)
        if c["op"] != "append":
            _attend(s, c)
    if c["op"] == "append" and c["kv"] == "mxfp4":
        return {"q": s["q_out"], "k": s["k_back"], "v": s["v_back"], "lens": s["lens_out"]}
    stored = {}
    if c["op"] in ("append", "step"):
        as_values = torch.float8_e4m3fn if c["kv"] == "fp8_e4m3" else torch.bfloat16
        stored = {"q": s["q_out"], "lens": s["lens_out"]}
        if c["kv"] != "mxfp4":
            stored.update(K=s["K"].view(as_values), V=s["V"].view(as_values))
    return stored if c["op"] == "append" else {"out": s["out"], **stored}


def _own(s, c):
    import paper_2403_08845_amd as bif
    plan, pages = s["plan"], s["pages"]
    q, lens = s["q"], s["lens"]
    if c["op"] in ("append", "step"):
        table = s["ctx_table"].view(1, -1) if c["context"] else s["tables"]
        bif.bifattn_paged_append(plan, pages, table, lens, s["k"], s["v"], s["lens_out"], q=q, q_out=s["q_out"], counts=s["counts"],
                                 freqs=s["freqs"], neighbours=c["pairs"] == "neighbours", context=c["context"])
        if "k_back" in s:
            bif.bifattn_paged_gather(plan, pages, table, s["lens_out"], s["k_back"], s["v_back"], first=lens, context=c["context"])
        q, lens = s["q_out"], s["lens_out"]
    if c["op"] == "diff":
        bif.bifattn_paged_decode_diff(plan, q, pages, s["ctx_table"], s["tables"], lens, s["lam"], s["out"], weight=s["weight"],
                                      eps=1e-5, out_scale=s["out_scale"])
    elif c["op"] != "append":
        bif.bifattn_paged_decode(plan, q, pages, s["ctx_table"], s["tables"], lens, s["out"])


# Plain forms.

def _rotated(x, position, freqs, pairs):
    """Rows x [..., n, d] at positions [..., n], in 64 bits."""
    x = x.double()
    if freqs is None:
        return x
    a = position.double().unsqueeze(-1) * freqs.double()
    r = 2 * freqs.numel()
    lo, hi = (x[..., 0:r:2], x[..., 1:r:2]) if pairs == "neighbours" else (x[..., :r // 2], x[..., r // 2:r])
    lo, hi = lo * a.cos() - hi * a.sin(), lo * a.sin() + hi * a.cos()
    y = torch.stack((lo, hi), -1).flatten(-2) if pairs == "neighbours" else torch.cat((lo, hi), -1)
    return torch.cat((y, x[..., r:]), -1)


def _append(s, c):
    n, page = c["n"], c["page"]
    table = s["ctx_table"].view(1, -1) if c["context"] else s["tables"]
    r = torch.arange(n, device="cuda")
    row = s["lens"].long().unsqueeze(1) + r
    count = torch.full_like(s["lens"], n) if s["counts"] is None else s["counts"]
    new = r < count.unsqueeze(1)
    position = (row + (0 if c["context"] else c["m_c"])).unsqueeze(1)
    place = table.long().gather(1, row // page), row % page
    s["q_out"].copy_(torch.where(new[:, None, :, None], _rotated(s["q"], position, s["freqs"], c["pairs"]).to(torch.bfloat16), s["q_out"]))
    k, ke = _to_codes(_rotated(s["k"], position, s["freqs"], c["pairs"]), c["kv"], s["k_scale"])
    v, ve = _to_codes(s["v"].double(), c["kv"], s["v_scale"])
    keep = new[..., None, None]

    def put(pool, x):
        if x is not None:
            pool[place[0], :, place[1]] = torch.where(keep, x.transpose(1, 2), pool[place[0], :, place[1]])

    put(s["K"], k)
    put(s["V"], v)
    put(s["K_exp"], ke)
    put(s["V_exp"], ve)
    s["lens_out"].copy_(s["lens"] + count)
    if "k_back" in s:
        for name, out in (("K", s["k_back"]), ("V", s["v_back"])):
            x = _values(s[name][place[0], :, place[1]], s[name + "_exp"][place[0], :, place[1]], None, c["kv"])
            out.copy_(torch.where(keep.transpose(1, 2), x.transpose(1, 2).to(torch.bfloat16), out))


def _values(bits, exps, scale, kv):
    """Stored rows [..., g, rows, cols] as 32-bit values."""
    if kv == "bf16":
        return bits.float()
    if kv == "fp8_e4m3":
        return bits.view(torch.float8_e4m3fn).float() * scale.view(-1, 1, 1)
    k = torch.stack((bits & 15, bits >> 4), -1).flatten(-2)
    x = torch.tensor(E2M1 + tuple(-v for v in E2M1), device="cuda")[k.int()]
    return torch.ldexp(x.unflatten(-1, (-1, 32)), (exps.int() - 127).unsqueeze(-1)).flatten(-2)


def _rows(s, c, name, table, rows):
    """The first rows of the sequences of a table [s, pages], [s, g, rows, d]."""
    def take(x):
        return None if x is None else x[table.long()].transpose(1, 2).flatten(2, 3)[:, :, :rows]
    return _values(take(s[name]), take(s[name + "_exp"]), s["k_scale" if name == "K" else "v_scale"], c["kv"])


def _attend(s, c):
    b, h, g, d, n, m_c, m_d = (c[k] for k in ("b", "h", "g", "d", "n", "m_c", "m_d"))
    p, parts = h // g, 2 if c["op"] == "diff" else 1
    q = (s["q_out"] if c["op"] == "step" else s["q"]).float().view(b, g, p * n, d)
    lens = s["lens_out"] if c["op"] == "step" else s["lens"]
    kc, vc = (_rows(s, c, x, s["ctx_table"].view(1, -1), m_c)[0] for x in ("K", "V"))  # [g, m_c, d]
    kd, vd = (_rows(s, c, x, s["tables"], m_d) for x in ("K", "V"))  # [b, g, m_d, d]
    pos = torch.arange(m_d, device="cuda")
    vd = torch.where((pos < lens.unsqueeze(1))[:, None, :, None], vd, 0)
    seen = pos < (lens.view(-1, 1, 1, 1) - n + 1 + torch.arange(p * n, device="cuda").view(-1, 1) % n)

    def attention(q, kc, kd):
        w = q.shape[-1]
        x = torch.bmm(q.transpose(0, 1).reshape(g, b * p * n, w), kc.transpose(1, 2)).view(g, b, p * n, m_c).transpose(0, 1)
        y = torch.bmm(q.reshape(b * g, p * n, w), kd.reshape(b * g, m_d, w).transpose(1, 2)).view(b, g, p * n, m_d)
        x = torch.cat((x, torch.where(seen, y, -math.inf)), -1) / math.sqrt(w)
        m = x.amax(-1, keepdim=True)
        x = (x - torch.where(m == -math.inf, 0, m)).exp_()
        total = x.sum(-1, keepdim=True)
        a = torch.bmm(x[..., :m_c].transpose(0, 1).reshape(g, b * p * n, m_c), vc).view(g, b, p * n, d).transpose(0, 1)
        a = a + torch.bmm(x[..., m_c:].reshape(b * g, p * n, m_d), vd.reshape(b * g, m_d, d)).view(b, g, p * n, d)
        return (a / torch.where(total > 0, total, 1)).reshape(b, h, n, d)

    if parts == 1:
        s["out"].copy_(attention(q, kc, kd))
        return
    lo, hi = slice(0, d // 2), slice(d // 2, d)
    y = attention(q[..., lo], kc[..., lo], kd[..., lo]) - s["lam"].view(-1, 1, 1) * attention(q[..., hi], kc[..., hi], kd[..., hi])
    if s["weight"] is not None:
        y = y * (y.square().mean(-1, keepdim=True) + 1e-5).rsqrt() * s["weight"]
    s["out"].copy_(y * s["out_scale"])


# From the definitions, in 64 bits.

def _exact_codes(x, kv, scale):
    """The values that rows x [g, d] are stored as."""
    if kv == "bf16":
        return x
    if kv == "fp8_e4m3":
        y = (x / scale.double().view(-1, 1)).clamp(-448, 448)
        step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
        return torch.round(y / step) * step
    grid = torch.tensor(E2M1, dtype=torch.float64, device="cuda")
    out = torch.empty_like(x)
    for j in range(0, x.shape[-1], 32):
        y = x[..., j:j + 32]
        top = y.abs().amax(-1, keepdim=True)
        unit = torch.exp2((torch.floor(torch.log2(top.clamp(min=1e-300))) - 2).clamp(-126, 127))
        z = (y.abs() / unit).contiguous()
        i = torch.bucketize(z, (grid[1:] + grid[:-1]) / 2)
        half = (i < 7) & (z == ((grid[1:] + grid[:-1]) / 2)[i.clamp(max=6)]) & (i % 2 == 1)  # ties to the even one
        out[..., j:j + 32] = grid[i + half.long()] * unit * torch.where(torch.signbit(y), -1.0, 1.0)
    return out


def _exact_rotated(x, position, freqs, pairs):
    """Rows x [..., d] at positions [...]: each pair a complex number, turned."""
    x = x.double().clone()
    if freqs is not None:
        half = freqs.numel()
        i = torch.arange(half, device="cuda")
        i, j = (2 * i, 2 * i + 1) if pairs == "neighbours" else (i, i + half)
        turns = position.double().unsqueeze(-1) * (freqs.double() / (2 * math.pi))
        z = torch.complex(x[..., i], x[..., j]) * torch.polar(torch.ones_like(turns), 2 * math.pi * (turns - turns.round()))
        x[..., i], x[..., j] = z.real, z.imag
    return x


def _exact_append(s, c):
    """What run() returns of an append; K and V [pages, g, page, d] of the pools afterwards."""
    page, kv = c["page"], c["kv"]
    table = (s["ctx_table"].view(1, -1) if c["context"] else s["tables"]).tolist()
    starts = s["lens"].tolist()
    counts = [c["n"]] * len(starts) if s["counts"] is None else s["counts"].tolist()
    place = [(i, r, table[i][(t + r) // page], (t + r) % page, t + r) for i, t in enumerate(starts) for r in range(counts[i])]
    res = {"q": torch.zeros(s["q_out"].shape, dtype=torch.float64, device="cuda"), "lens": s["lens"] + torch.tensor(counts, device="cuda", dtype=torch.int32)}
    pools = {}
    if kv != "mxfp4":
        for x in ("K", "V"):
            pools[x] = s[x].double() if kv == "bf16" else s[x].view(torch.float8_e4m3fn).double()
    else:
        res["k"], res["v"] = (torch.zeros(s["k_back"].shape, dtype=torch.float64, device="cuda") for _ in range(2)) if "k_back" in s else (None, None)
    if place:
        i, r, pg, off, row = torch.tensor(place, device="cuda").unbind(1)
        position = (row + (0 if c["context"] else c["m_c"])).unsqueeze(1)
        res["q"][i, :, r] = _exact_rotated(s["q"][i, :, r], position, s["freqs"], c["pairs"])
        rows = {"K": _exact_rotated(s["k"][i, :, r], position, s["freqs"], c["pairs"]), "V": s["v"][i, :, r].double()}
        for x, sc in (("K", s["k_scale"]), ("V", s["v_scale"])):
            y = _exact_codes(rows[x], kv, sc)
            if kv == "mxfp4":
                res[x.lower()][i, :, r] = y
            else:  # the pool holds codes: values without the group's scale
                pools[x][pg, :, off] = y
    return res, pools


def exact(case, seed):
    c = case
    s = _inputs(c, seed)
    if c["op"] == "append":
        res, pools = _exact_append(s, c)
        return {**res, **pools}
    b, h, g, d, n, m_c, m_d = (c[k] for k in ("b", "h", "g", "d", "n", "m_c", "m_d"))
    stored = {}
    if c["op"] == "step":
        if c["kv"] == "mxfp4":
            s["k_back"], s["v_back"] = (torch.empty(b, g, n, d, device="cuda") for _ in range(2))
        before = s["lens"].clone()
        res, pools = _exact_append(s, c)
        s["lens"] = before + n
        s["q"] = res["q"].to(torch.bfloat16)
        stored = {"q": res["q"], "lens": res["lens"], **pools}
    p, parts = h // g, 2 if c["op"] == "diff" else 1
    e2m1 = torch.tensor(E2M1, dtype=torch.float64, device="cuda")

    def values(name, pages, j, scale):  # rows of the pages of group j, in order
        x = s[name][pages.long(), j].flatten(0, -2)
        if c["kv"] == "bf16":
            return x.double()
        if c["kv"] == "fp8_e4m3":
            return x.view(torch.float8_e4m3fn).double() * scale[j].double()
        y = torch.empty(x.shape[0], d, dtype=torch.float64, device="cuda")
        for u in (0, 1):
            k = (x >> (4 * u)) & 15
            y[:, u::2] = torch.where(k > 7, -e2m1[(k & 7).long()], e2m1[(k & 7).long()])
        e = s[name + "_exp"][pages.long(), j].flatten(0, -2).double() - 127
        return y * torch.exp2(e).repeat_interleave(32, -1)

    out = torch.zeros(b, h, n, d, dtype=torch.float64, device="cuda")
    token = torch.arange(p * n, device="cuda") % n
    pos = torch.arange(m_d, device="cuda")
    for j in range(g):
        kc, vc = values("K", s["ctx_table"], j, s["k_scale"])[:m_c], values("V", s["ctx_table"], j, s["v_scale"])[:m_c]
        for i0 in range(0, b, 16):
            i1 = min(b, i0 + 16)
            q = s["q"][i0:i1, j * p:(j + 1) * p].double().reshape(i1 - i0, p * n, d)
            lens = s["lens"][i0:i1].view(-1, 1, 1)
            kd, vd = (values(x, s["tables"][i0:i1].flatten(), j, s[sc]).view(i1 - i0, -1, d)[:, :m_d] for x, sc in (("K", "k_scale"), ("V", "v_scale")))
            if c["op"] == "step":  # the step's own rows, as they are stored
                for i in range(i0, i1):
                    t = int(s["lens"][i]) - n
                    for x, y, sc in ((s["k"], kd, s["k_scale"]), (s["v"], vd, s["v_scale"])):
                        row = x[i, j].double()
                        if x is s["k"]:
                            row = _exact_rotated(row, m_c + t + torch.arange(n, device="cuda"), s["freqs"], c["pairs"])
                        one = None if sc is None else sc[j:j + 1]
                        row = _exact_codes(row.unsqueeze(1), c["kv"], one).squeeze(1)
                        if c["kv"] == "fp8_e4m3":
                            row = row * sc[j].double()
                        y[i - i0, t:t + n] = row.to(torch.bfloat16).double() if c["kv"] == "bf16" else row
            vd = torch.where((pos < lens).transpose(1, 2), vd, 0.0)
            seen = pos < (lens - n + 1 + token.view(-1, 1))
            maps = []
            for u in range(parts):
                f = slice(u * d // parts, (u + 1) * d // parts)
                x = torch.cat((torch.einsum("irw,tw->irt", q[..., f], kc[:, f]),
                               torch.where(seen, torch.einsum("irw,itw->irt", q[..., f], kd[..., f]), -math.inf)), -1) * (d / parts) ** -0.5
                top = x.amax(-1, keepdim=True)
                x = torch.exp(x - torch.where(top == -math.inf, 0.0, top))
                total = x.sum(-1, keepdim=True)
                a = torch.einsum("irt,tw->irw", x[..., :m_c], vc) + torch.einsum("irt,itw->irw", x[..., m_c:], vd)
                maps.append(torch.where(total > 0, a / total, 0.0).view(i1 - i0, p, n, d))
            y = maps[0]
            if parts == 2:
                y = y - s["lam"][j * p:(j + 1) * p].double().view(-1, 1, 1) * maps[1]
                if s["weight"] is not None:
                    y = y / torch.sqrt((y * y).sum(-1, keepdim=True) / d + 1e-5) * s["weight"].double()
                y = y * s["out_scale"]
            out[i0:i1, j * p:(j + 1) * p] = y
    return {"out": out, **({k: v for k, v in stored.items() if k in ("q", "lens", "K", "V")})}
