"""Rows in and out of paged caches against 64 bits (MI355X only): append with
rotation and encoding, read-out, and generation loops of append and attention."""
import pytest
import torch

import paper_2403_08845_amd as bif

from .paged_ref import HALF_BF16, Problem, mx_codes, mx_values, rotated, stored

pytestmark = pytest.mark.gpu


def freqs_of(rot):
    return (10000.0 ** (-torch.arange(0, rot, 2).double() / max(1, rot))).float()


def new_rows(x, n, fused, seed, samples=None):
    """q, k, v bf16 [s, heads, n, d]; fused: views into one projection's output."""
    r = torch.Generator().manual_seed(seed)
    s = x.b if samples is None else samples
    y = torch.randn(s, n, x.h + 2 * x.g, x.d, generator=r).to(torch.bfloat16).cuda().transpose(1, 2)
    parts = y[:, :x.h], y[:, x.h:x.h + x.g], y[:, x.h + x.g:]
    return parts if fused else [t.contiguous() for t in parts]


def values_of(bits, exps, kv):
    """Stored rows [..., cols] as float64 values without group scales."""
    bits = bits.cpu()
    if kv == "bf16":
        return bits.double()
    if kv == "fp8_e4m3":
        return bits.view(torch.float8_e4m3fn).double()
    k = torch.stack((bits & 15, bits >> 4), -1).flatten(-2)
    return mx_values(k, exps.cpu().int() - 127)


def rows_at(x, pages, name, i, t):
    table = x.ctx_table if i is None else x.tables[i]
    at = int(table[t // x.page]), t % x.page
    e = getattr(pages, name + "_exp")
    return values_of(getattr(pages, name)[at[0], :, at[1]], None if e is None else e[at[0], :, at[1]], x.kv)


def near(got, ref, kv):
    """Stored values [g, d] against what they stand for, 64 bits before rounding."""
    if kv == "bf16":
        return ((got - ref).abs() <= HALF_BF16 * ref.abs() + 1e-12).all()
    _, _, want = stored(ref.unsqueeze(-2), kv)
    return torch.equal(got, want.squeeze(-2))


APPEND = [
    # b, h, g, d, m_c, m_d, page, n, rot, neighbours, maps, fused
    (1, 1, 1, 64, 0, 1, 16, 1, 64, False, 1, False),
    (3, 8, 2, 128, 77, 40, 16, 1, 128, False, 1, True),
    (3, 8, 2, 128, 77, 40, 32, 5, 128, True, 1, True),
    (2, 4, 4, 64, 5000000, 30, 16, 3, 32, True, 1, False),   # far positions
    (2, 4, 4, 64, 5000000, 30, 16, 3, 16, False, 1, True),
    (4, 6, 3, 128, 10, 50, 64, 7, 64, False, 2, True),       # both halves rotate
    (4, 6, 3, 64, 10, 50, 64, 7, 32, True, 2, False),
    (2, 4, 2, 128, 9, 50, 16, 2, 48, False, 1, True),        # odd share of a row
    (2, 4, 2, 128, 9, 50, 16, 2, 0, False, 1, True),
]


@pytest.mark.parametrize("kv", ["bf16", "fp8_e4m3", "mxfp4"])
@pytest.mark.parametrize("case", APPEND, ids=lambda c: "b%d_h%d_g%d_d%d_mc%d_md%d_pg%d_n%d_rot%d_%d_maps%d_%d" % c)
def test_append(case, kv):
    b, h, g, d, m_c, m_d, page, n, rot, neighbours, maps, fused = case
    r = torch.Generator().manual_seed(1)
    lens = torch.randint(0, m_d - n + 1, (b,), generator=r).tolist()
    counts = torch.randint(0, n + 1, (b,), generator=r).to(torch.int32)
    counts[0] = n
    x = Problem(b, h, g, d, 0 if m_c > 1000 else m_c, m_d, 1, page, kv, maps=maps, lens=[m_d] * b, seed=2)
    x.m_c = m_c
    x.lens = torch.tensor(lens, dtype=torch.int32)
    q, k, v = new_rows(x, n, fused, 3)
    f = freqs_of(rot)
    pages = x.pages()
    before = [t.clone() for t in pages if t is not None]
    q_out = torch.full((b, h, n, d), 7.0, dtype=torch.bfloat16, device="cuda")
    lens_out = torch.zeros(b, dtype=torch.int32, device="cuda")
    with x.plan() as plan:
        bif.bifattn_paged_append(plan, pages, x.tables.cuda(), x.lens.cuda(), k, v, lens_out, q=q, q_out=q_out,
                                 counts=counts.cuda(), freqs=f.cuda() if rot else None, neighbours=neighbours)
        assert bif.bifattn_paged_plan_status(plan) == bif.OK
    assert torch.equal(lens_out.cpu(), x.lens + counts)
    q, k, v = q.cpu().double(), k.cpu().double(), v.cpu().double()
    unscaled = [torch.ones(g) if s is None else s for s in (x.k_scale, x.v_scale)]
    touched = torch.zeros(x.num_pages, page, dtype=torch.bool)
    for i in range(b):
        for t in range(n):
            row = int(x.lens[i]) + t
            if t >= int(counts[i]):
                assert (q_out[i, :, t] == 7.0).all()
                continue
            position = torch.tensor(m_c + row)
            want = rotated(q[i, :, t], position, f, neighbours, maps)
            assert ((q_out[i, :, t].cpu().double() - want).abs() <= HALF_BF16 * want.abs() + 1e-12).all()
            keys = rotated(k[i, :, t], position, f, neighbours, maps)
            for name, ref, s in (("K", keys, unscaled[0]), ("V", v[i, :, t], unscaled[1])):
                assert near(rows_at(x, pages, name, i, row), ref / s.double().view(-1, 1), kv), (name, i, t)
            touched[int(x.tables[i, row // page]), row % page] = True
    for t, old in zip([t for t in pages if t is not None and t.dim() == 4], before):  # every other row as it was
        keep = ~touched.cuda()
        assert torch.equal(t.transpose(1, 2)[keep].view(torch.uint8), old.transpose(1, 2)[keep].view(torch.uint8))


@pytest.mark.parametrize("kv", ["bf16", "mxfp4"])
def test_append_of_a_prompt_in_pieces(kv):
    """A prompt of the shared context appended in two pieces equals the same
    prompt at once, and read-out returns the stored values."""
    m_c, page = 1000, 32
    x = Problem(2, 4, 2, 128, m_c, 8, page=page, kv=kv, seed=4)
    q, k, v = new_rows(x, m_c, True, 5, samples=1)
    f, table = freqs_of(128).cuda(), x.ctx_table.view(1, -1).cuda()
    done = []
    for cuts in ([0, m_c], [0, 333, m_c]):
        pages = x.pages()
        q_out = torch.zeros(1, 4, m_c, 128, dtype=torch.bfloat16, device="cuda")
        lens = torch.zeros(1, dtype=torch.int32, device="cuda")
        with x.plan() as plan:
            for a, z in zip(cuts, cuts[1:]):
                piece = torch.zeros(1, 4, z - a, 128, dtype=torch.bfloat16, device="cuda")
                bif.bifattn_paged_append(plan, pages, table, lens, k[:, :, a:z], v[:, :, a:z], lens, q=q[:, :, a:z],
                                         q_out=piece, freqs=f, context=True)
                q_out[:, :, a:z] = piece
            assert lens.item() == m_c
            outs = [torch.full((1, 2, m_c + 5, 128), 3.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
            bif.bifattn_paged_gather(plan, pages, table, lens, *outs, context=True)
            assert bif.bifattn_paged_plan_status(plan) == bif.OK
        assert all((t[:, :, m_c:] == 3.0).all() for t in outs)
        done.append([pages.K[x.ctx_table.long()], pages.V[x.ctx_table.long()], q_out] + [t[:, :, :m_c] for t in outs])
        ref = rotated(k[0].cpu().double(), torch.arange(m_c), freqs_of(128), False, 1)
        for got, want in ((outs[0], ref), (outs[1], v[0].cpu().double())):
            got = got[0, :, :m_c].cpu().double()
            if kv == "bf16":
                assert ((got - want).abs() <= HALF_BF16 * want.abs() + 1e-12).all()
            else:
                assert torch.equal(got, mx_values(*mx_codes(want)))
    last = m_c % page  # the last page's rows past the prompt are poison in both
    for a, z in zip(*done):
        if a.dim() == 4 and a.shape[1] == 2 and a.shape[2] == page:
            a, z = a.clone(), z.clone()
            a[-1, :, last:], z[-1, :, last:] = 0, 0
        assert torch.equal(a, z)


def test_gather_ranges():
    """Rows from each sequence's own first one, group scales applied, the
    others left as they were."""
    for kv in ("bf16", "fp8_e4m3", "mxfp4"):
        x = Problem(4, 4, 2, 64, 3, 60, page=16, kv=kv, lens=[60, 17, 0, 33], seed=6)
        first = torch.tensor([40, 0, 0, 33], dtype=torch.int32)
        outs = [torch.full((4, 2, 20, 64), 9.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        with x.plan() as plan:
            bif.bifattn_paged_gather(plan, x.pages(), x.tables.cuda(), x.lens.cuda(), *outs, first=first.cuda())
            assert bif.bifattn_paged_plan_status(plan) == bif.OK
        for got, name in zip(outs, "KV"):
            got = got.cpu().double()
            for i in range(4):
                a, z = int(first[i]), min(int(x.lens[i]), int(first[i]) + 20)
                want = x.own[name][i, :, a:z]
                # fp8: a 32-bit product (off by 2^-24) rounded to bf16
                slack = HALF_BF16 * want.abs() * (1 + 2.0 ** -15) if kv == "fp8_e4m3" else 0 * want
                assert ((got[i, :, :z - a] - want).abs() <= slack).all()
                assert (got[i, :, max(0, z - a):] == 9.0).all()


def test_append_drops_what_does_not_fit():
    x = Problem(4, 4, 2, 64, 3, 20, page=16, lens=[20] * 4, seed=7)
    _, k, v = new_rows(x, 3, False, 8)
    pages = x.pages()
    before = pages.K.clone()
    lens = torch.tensor([17, 18, 20, -4], dtype=torch.int32, device="cuda")
    with x.plan() as plan:
        bif.bifattn_paged_append(plan, pages, x.tables.cuda(), lens, k, v, lens)
        assert bif.bifattn_paged_plan_status(plan) == bif.ELENS
        assert lens.tolist() == [20, 20, 20, 3]
        for i, start, fit in ((0, 17, 3), (1, 18, 2), (3, 0, 3)):
            for t in range(fit):
                assert torch.equal(rows_at(x, pages, "K", i, start + t), k[i, :, t].cpu().double())
        used = torch.zeros(x.num_pages, 16, dtype=torch.bool)
        for i, start, fit in ((0, 17, 3), (1, 18, 2), (3, 0, 3)):
            for t in range(start, start + fit):
                used[int(x.tables[i, t // 16]), t % 16] = True
        keep = ~used.cuda()
        assert torch.equal(pages.K.transpose(1, 2)[keep].view(torch.int16), before.transpose(1, 2)[keep].view(torch.int16))
        # a count outside [0, n] is clamped, an id outside the pool is skipped
        lens.zero_()
        bif.bifattn_paged_append(plan, pages, x.tables.cuda(), lens, k, v, lens,
                                 counts=torch.tensor([5, -1, 0, 2], dtype=torch.int32, device="cuda"))
        assert bif.bifattn_paged_plan_status(plan) == bif.ELENS and lens.tolist() == [3, 0, 0, 2]
        bad = x.tables.clone()
        bad[2, 0] = x.num_pages
        before = pages.K.clone()
        lens.zero_()
        counts = torch.tensor([0, 0, 3, 0], dtype=torch.int32, device="cuda")
        bif.bifattn_paged_append(plan, pages, bad.cuda(), lens, k, v, lens, counts=counts)
        assert bif.bifattn_paged_plan_status(plan) == bif.EPAGE
        assert torch.equal(pages.K.view(torch.int16), before.view(torch.int16))
        out = torch.full((4, 2, 3, 64), 5.0, dtype=torch.bfloat16, device="cuda")
        bif.bifattn_paged_gather(plan, pages, bad.cuda(), torch.tensor([0, 0, 3, 0], dtype=torch.int32, device="cuda"), out, out.clone())
        assert bif.bifattn_paged_plan_status(plan) == bif.EPAGE and (out == 5.0).all()


def test_encodings_at_borders():
    """Unrotated rows whose elements lie on rounding borders, blocks of zeros, of
    tiny and huge values, and blocks that are not finite."""
    x = Problem(1, 1, 1, 128, 0, 4, page=16, kv="mxfp4", lens=[4], seed=9)
    row = torch.zeros(4, 128)
    row[0, :32] = torch.tensor([6.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0] * 4) * torch.tensor([1.0, -1.0]).repeat_interleave(16)
    row[0, 32:64] = torch.linspace(-8, 8, 32)
    row[1, :32] = 2.0 ** -133
    row[1, 32:64] = torch.finfo(torch.bfloat16).max
    row[1, 64:96] = -0.0
    row[2, 3], row[2, 40], row[3, 70] = float("inf"), float("nan"), float("-inf")
    kv = row.to(torch.bfloat16).view(1, 1, 4, 128)
    pages = x.pages()
    lens = torch.zeros(1, dtype=torch.int32, device="cuda")
    with x.plan() as plan:
        bif.bifattn_paged_append(plan, pages, x.tables.cuda(), lens, kv.cuda(), kv.cuda(), lens)
        assert bif.bifattn_paged_plan_status(plan) == bif.OK
    page = int(x.tables[0, 0])
    for t in range(4):
        exps, codes = pages.K_exp[page, 0, t].cpu(), pages.K[page, 0, t].cpu()
        want, e = mx_codes(torch.nan_to_num(kv[0, 0, t].double(), nan=0.0, posinf=0.0, neginf=0.0))
        e = e + 127
        for blk in range(4):
            if not torch.isfinite(kv[0, 0, t, 32 * blk:32 * blk + 32]).all():
                assert exps[blk] == 255
            else:
                assert exps[blk] == e[blk]
                got = torch.stack((codes & 15, codes >> 4), -1).flatten()[32 * blk:32 * blk + 32]
                assert torch.equal(got.long(), want[32 * blk:32 * blk + 32])


def test_fp8_saturates_and_keeps_nan():
    x = Problem(1, 1, 1, 64, 0, 1, page=16, kv="fp8_e4m3", lens=[1], seed=9)
    x.k_scale, x.v_scale = torch.tensor([0.5]), torch.tensor([3.0])
    row = torch.zeros(64)
    row[:8] = torch.tensor([1e30, -1e30, float("inf"), float("-inf"), float("nan"), 232.0, 224.0, 2.0 ** -11])
    kv = row.to(torch.bfloat16).view(1, 1, 1, 64).cuda()
    pages = x.pages()
    lens = torch.zeros(1, dtype=torch.int32, device="cuda")
    with x.plan() as plan:
        bif.bifattn_paged_append(plan, pages, x.tables.cuda(), lens, kv, kv, lens)
        assert bif.bifattn_paged_plan_status(plan) == bif.OK
    got = pages.K[int(x.tables[0, 0]), 0, 0].cpu().view(torch.float8_e4m3fn).float()[:8]
    assert got[:4].tolist() == [448, -448, 448, -448] and torch.isnan(got[4]) and got[5:].tolist() == [448, 448, 0]


@pytest.mark.parametrize("kv", ["bf16", "fp8_e4m3", "mxfp4"])
@pytest.mark.parametrize("shape", [(3, 8, 2, 128, 77, 40, 1, 16, 1), (2, 4, 2, 64, 50, 30, 3, 32, 2),
                                   (40, 8, 2, 128, 130, 12, 1, 16, 1)], ids=["few", "diff", "many"])
def test_generation_loop(shape, kv):
    """Append, then attend, step after step on one pool: every step matches 64
    bits on the cache as stored; captured once and replayed for the later steps."""
    b, h, g, d, m_c, m_d, n, page, maps = shape
    x = Problem(b, h, g, d, m_c, m_d, n, page, kv, maps=maps, lens=[m_d] * b, seed=40)
    tables = x.tables.cuda()
    f = freqs_of(32 if maps == 2 else 64).cuda()
    lam = torch.rand(h, generator=x.rng)
    weight = torch.randn(d, generator=x.rng)
    pages = x.pages()
    lens = torch.zeros(b, dtype=torch.int32, device="cuda")
    buf = torch.zeros(b, n, h + 2 * g, d, dtype=torch.bfloat16, device="cuda").transpose(1, 2)
    q, k, v = buf[:, :h], buf[:, h:h + g], buf[:, h + g:]
    q_out, out = (torch.zeros(b, h, n, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    ctx, lam_d, weight_d = x.ctx_table.cuda(), lam.cuda(), weight.cuda()

    def step(plan):
        bif.bifattn_paged_append(plan, pages, tables, lens, k, v, lens, q=q, q_out=q_out, freqs=f)
        if maps == 2:
            bif.bifattn_paged_decode_diff(plan, q_out, pages, ctx, tables, lens, lam_d, out, weight=weight_d)
        else:
            bif.bifattn_paged_decode(plan, q_out, pages, ctx, tables, lens, out)

    with x.plan() as plan:
        graph = None
        for t in range(m_d // n):
            new = torch.randn(b, n, h + 2 * g, d, generator=x.rng).to(torch.bfloat16)
            buf.copy_(new.cuda().transpose(1, 2))
            if t < 2:
                step(plan)
            else:
                if graph is None:
                    torch.cuda.synchronize()
                    graph = torch.cuda.CUDAGraph()
                    with torch.cuda.graph(graph):
                        step(plan)
                graph.replay()
            torch.cuda.synchronize()
            assert lens.tolist() == [(t + 1) * n] * b
            if t in (0, 1, 2, 3, m_d // n - 1):
                x.lens = lens.cpu()
                for name, s in (("K", x.k_scale), ("V", x.v_scale)):
                    for i in range(b):
                        for r in range((t + 1) * n):
                            val = rows_at(x, pages, name, i, r)
                            x.own[name][i, :, r] = val if s is None else val * s.double().view(-1, 1)
                ref, tol = x.attention(lam=lam, weight=weight if maps == 2 else None, q=q_out.cpu())
                assert ((out.cpu().double() - ref).abs() <= tol).all(), t
        assert bif.bifattn_paged_plan_status(plan) == bif.OK


def test_streams_other_than_the_current_one():
    x = Problem(3, 8, 2, 128, 77, 40, page=32, lens=[40] * 3, seed=3)
    q, k, v = new_rows(x, 5, True, 8)
    res = []
    for stream in (None, torch.cuda.Stream()):
        pages = x.pages()
        lens = torch.tensor([0, 7, 35], dtype=torch.int32, device="cuda")
        q_out = torch.zeros(3, 8, 5, 128, dtype=torch.bfloat16, device="cuda")
        torch.cuda.synchronize()
        with x.plan() as plan:
            bif.bifattn_paged_append(plan, pages, x.tables.cuda(), lens, k, v, lens, q=q, q_out=q_out,
                                     freqs=freqs_of(128).cuda(), stream=stream)
            assert bif.bifattn_paged_plan_status(plan, stream) == bif.OK
        res.append((pages.K, q_out, lens))
    assert all(torch.equal(a.contiguous().view(torch.uint8), z.contiguous().view(torch.uint8)) for a, z in zip(*res))


def test_rotation_of_infinite_elements():
    """An infinite element makes its pair infinite (the sign of its cosine and
    sine) and leaves the others alone."""
    x = Problem(1, 1, 1, 64, 0, 1, page=16, lens=[1], seed=9)
    row = torch.randn(64, generator=x.rng)
    row[3], row[40] = float("inf"), float("-inf")
    kv = row.to(torch.bfloat16).view(1, 1, 1, 64).cuda()
    f = torch.linspace(0.1, 1.4, 32)
    pages = x.pages()
    lens = torch.zeros(1, dtype=torch.int32, device="cuda")
    x.m_c = 1  # position 1: angles in the first quadrant
    out = torch.zeros(1, 1, 1, 64, dtype=torch.bfloat16, device="cuda")
    with x.plan() as plan:
        bif.bifattn_paged_append(plan, pages, x.tables.cuda(), lens, kv, kv, lens, q=kv, q_out=out, freqs=f.cuda())
        assert bif.bifattn_paged_plan_status(plan) == bif.OK
    for got in (out[0, 0, 0].cpu(), pages.K[int(x.tables[0, 0]), 0, 0].cpu()):
        inf = torch.zeros(64)
        inf[3], inf[35], inf[40], inf[8] = 1, 1, -1, 1  # (x c - y s, x s + y c)
        assert torch.equal(torch.isinf(got.float()) * torch.sign(got.float()), inf)
        assert not torch.isnan(got).any()
