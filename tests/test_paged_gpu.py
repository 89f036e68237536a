"""Attention over paged caches against 64 bits (MI355X only). Every pool is
poisoned with NaN outside the valid rows and every table holds ids outside the
pool past its last valid page, so a read of either shows."""
import math

import pytest
import torch

import paper_2403_08845_amd as bif

from .paged_ref import Problem

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True, params=["parts", "one launch"])
def launches(request, monkeypatch):
    """Every test runs in parts and, where a unit's rows fit, as one launch."""
    monkeypatch.setenv("BIFATTN_WHOLE", "2" if request.param == "parts" else "1")
    return request.param


def attend(x, plan=None, pages=None, scale=None, lam=None, weight=None, eps=1e-5, out_scale=1.0, status=bif.OK,
           q=None, out=None):
    own = plan is None
    plan = plan or x.plan(scale=0.0 if scale is None else scale)
    try:
        out = torch.full((x.b, x.h, x.n, x.d), float("nan"), dtype=torch.bfloat16, device="cuda") if out is None else out
        args = ((x.q if q is None else q).cuda(), pages or x.pages(), x.ctx_table.cuda(), x.tables.cuda(), x.lens.cuda())
        if x.maps == 2:
            bif.bifattn_paged_decode_diff(plan, *args, lam.cuda(), out, weight=None if weight is None else weight.cuda(),
                                          eps=eps, out_scale=out_scale)
        else:
            bif.bifattn_paged_decode(plan, *args, out)
        assert bif.bifattn_paged_plan_status(plan) == status
        return out.cpu().double()
    finally:
        if own:
            plan.close()


def check(x, **kw):
    got = attend(x, **kw)
    kw = {k: v for k, v in kw.items() if k in ("scale", "lam", "weight", "eps", "out_scale")}
    ref, tol = x.attention(**kw)
    assert torch.isfinite(got).all()
    over = ((got - ref).abs() / tol).max().item()
    print(f"largest error {over:.3f} of the tolerance", flush=True)
    assert over <= 1


CASES = [
    # b, h, g, d, m_c, m_d, n, page, lens
    (1, 1, 1, 64, 1, 0, 1, 16, [0]),                          # one context key
    (1, 1, 1, 128, 0, 1, 1, 16, [1]),                         # one own key
    (2, 4, 2, 64, 0, 5, 1, 16, [0, 5]),                       # a sample without any key
    (4, 4, 4, 64, 128, 16, 1, 16, None),
    (3, 8, 2, 128, 77, 40, 1, 32, [0, 1, 40]),
    (2, 8, 8, 128, 33, 50, 3, 64, [2, 50]),                   # fewer own rows than tokens
    (3, 6, 3, 64, 0, 70, 4, 16, [0, 2, 70]),                  # tokens that see nothing
    (1, 16, 1, 64, 300, 33, 4, 16, [33]),                     # 64 query rows per unit, few in the group
    (3, 32, 2, 128, 200, 40, 4, 256, [4, 40, 17]),            # 64 per unit, many in the group
    (5, 32, 4, 128, 515, 65, 2, 16, None),                    # 80 rows per group
    (11, 16, 4, 64, 700, 130, 1, 128, None),                  # 44 rows
    (40, 32, 4, 128, 333, 20, 1, 64, None),                   # 320 rows: eight-wave work-groups
    (33, 8, 1, 64, 1031, 300, 1, 32, None),                   # 264 rows of 64 elements
    (2, 2, 2, 128, 5000, 2100, 1, 16, [2100, 1025]),          # several chunks of own rows
]


@pytest.mark.parametrize("kv", ["bf16", "fp8_e4m3", "mxfp4"])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "b%d_h%d_g%d_d%d_mc%d_md%d_n%d_pg%d" % c[:8])
def test_decode(case, kv):
    b, h, g, d, m_c, m_d, n, page, lens = case
    check(Problem(b, h, g, d, m_c, m_d, n, page, kv, lens=lens, seed=hash(case[:8]) % 1000))


DIFF = [
    (1, 1, 1, 64, 1, 0, 1, 16, [0]),
    (2, 4, 2, 128, 0, 6, 1, 16, [0, 6]),
    (4, 4, 4, 128, 130, 16, 1, 16, None),
    (3, 8, 2, 64, 77, 40, 4, 32, [0, 1, 40]),                 # 32 rows per unit
    (2, 16, 1, 128, 300, 33, 2, 64, [33, 1]),                 # 64 per unit
    (9, 16, 4, 128, 515, 65, 1, 16, None),                    # 72 rows per group
    (70, 16, 4, 128, 333, 20, 1, 64, None),                   # 280 rows of each map
    (70, 16, 4, 64, 261, 20, 1, 16, None),
]


@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("kv", ["bf16", "fp8_e4m3", "mxfp4"])
@pytest.mark.parametrize("case", DIFF, ids=lambda c: "b%d_h%d_g%d_d%d_mc%d_md%d_n%d_pg%d" % c[:8])
def test_differential(case, kv, norm):
    b, h, g, d, m_c, m_d, n, page, lens = case
    x = Problem(b, h, g, d, m_c, m_d, n, page, kv, maps=2, lens=lens, seed=7 + m_c)
    lam = torch.rand(h, generator=x.rng) * 1.2 - 0.2
    weight = torch.randn(d, generator=x.rng) if norm else None
    check(x, lam=lam, weight=weight, eps=1e-4, out_scale=-0.3)


@pytest.mark.parametrize("scale", [-0.2, 1.5])
@pytest.mark.parametrize("case", [CASES[4], CASES[9], CASES[11]], ids=["few", "many4", "many8"])
def test_scale(case, scale):
    b, h, g, d, m_c, m_d, n, page, lens = case
    check(Problem(b, h, g, d, m_c, m_d, n, page, "bf16", lens=lens, seed=5), scale=scale)


@pytest.mark.parametrize("kv", ["fp8_e4m3"])
def test_without_group_scales(kv):
    check(Problem(3, 8, 2, 128, 77, 40, page=32, kv=kv, scaled=False, seed=3))


@pytest.mark.parametrize("case", [CASES[4], CASES[9], CASES[11]], ids=["few", "many4", "many8"])
def test_rising_logits(case):
    """Keys whose logits rise along the sequence, so that the reference maximum is
    raised again and again."""
    b, h, g, d, m_c, m_d, n, page, lens = case
    x = Problem(b, h, g, d, m_c, m_d, n, page, "bf16", lens=lens, seed=6)
    x.q = x.q.abs()
    for name, rows in (("ctx", m_c), ("own", m_d)):
        ramp = torch.linspace(0.05, 3, max(1, rows)).view(-1, 1) if rows else torch.ones(0, 1)
        getattr(x, name)["K"] = (getattr(x, name)["K"].abs() * ramp).to(torch.bfloat16).double()
    x._put("K", x.ctx["K"][None], x.ctx_table.view(1, -1), torch.tensor([m_c]), None)
    x._put("K", x.own["K"], x.tables, x.lens, None)
    check(x)


def test_pools_past_32_bit_offsets():
    """Pages whose bytes lie past 2^32 of the pool, in both kernels."""
    for b, h in ((2, 2), (33, 2)):
        x = Problem(b, h, 1, 128, 200, 40, page=256, seed=9)
        far = (1 << 32) // (256 * 128 * 2) + 5
        pages = bif.Pages(*(torch.empty(far + x.num_pages, 1, 256, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2)))
        for t, k in ((pages.K, "K"), (pages.V, "V")):
            t[far:] = x.pool[k].cuda()
        x.ctx_table += far
        x.tables = torch.where((x.tables >= 0) & (x.tables < x.num_pages), x.tables + far, x.tables)
        x.num_pages += far
        check(x, pages=pages)
        del pages


def test_nonfinite_rows():
    """An infinite value reaches the samples that see it, a NaN block of an MXFP4
    row too; the others stay finite."""
    x = Problem(3, 4, 2, 64, 20, 40, page=16, lens=[40, 10, 3], seed=11)
    at = int(x.tables[0, 2]), 35 % 16
    x.pool["V"][at[0], 1, at[1], 5] = math.inf
    got = attend(x)
    assert torch.isposinf(got[0, 2:, 0, 5]).all()
    assert torch.isfinite(got[1:]).all() and torch.isfinite(got[0, :2]).all()
    x = Problem(3, 4, 2, 64, 20, 40, page=16, kv="mxfp4", lens=[40, 10, 3], seed=11)
    x.exps["V"][int(x.tables[0, 2]), 1, 3, 1] = 255
    got = attend(x)
    assert torch.isnan(got[0, 2:, 0, 32:]).all() and torch.isfinite(got[0, 2:, 0, :32]).all()
    assert torch.isfinite(got[1:]).all() and torch.isfinite(got[0, :2]).all()


@pytest.mark.parametrize("case", [CASES[4], CASES[9], CASES[11]], ids=["few", "many4", "many8"])
def test_bad_page_ids_and_lengths_are_flagged(case):
    """An id outside the pool reads page 0, a length outside its range is
    clamped: both are reported once, and later calls are clean."""
    b, h, g, d, m_c, m_d, n, page, _ = case
    x = Problem(b, h, g, d, m_c, m_d, n, page, "bf16", lens=[m_d] * b, seed=12)
    good = attend(x)
    with x.plan() as plan:
        first, x.ctx_table[0] = int(x.ctx_table[0]), x.num_pages
        x.pool["K"][0], x.pool["V"][0] = x.pool["K"][first].clone(), x.pool["V"][first].clone()
        if first not in (0,) and not (x.tables == 0).any() and not (x.ctx_table == 0).any():
            assert torch.equal(attend(x, plan, status=bif.EPAGE), good)
        else:
            attend(x, plan, status=bif.EPAGE)
        x.ctx_table[0] = first
        keep, x.tables[0, 0] = int(x.tables[0, 0]), -1
        attend(x, plan, status=bif.EPAGE)
        x.tables[0, 0] = keep
    x = Problem(b, h, g, d, m_c, m_d, n, page, "bf16", lens=[m_d] * b, seed=12)
    good = attend(x)
    with x.plan() as plan:
        x.lens[0] = m_d + 5
        assert torch.equal(attend(x, plan, status=bif.ELENS), good)
        x.lens[0] = m_d
        assert torch.equal(attend(x, plan), good)
    if b > 1:
        ref = Problem(b, h, g, d, m_c, m_d, n, page, "bf16", lens=[0] + [m_d] * (b - 1), seed=12)
        clean = attend(ref)
        ref.lens[0] = -3
        assert torch.equal(attend(ref, status=bif.ELENS), clean)


def test_bad_scales_are_flagged():
    x = Problem(3, 8, 2, 128, 77, 40, page=32, kv="fp8_e4m3", seed=3)
    good = attend(x)
    x.v_scale[1] = 0.0
    got = attend(x, status=bif.ESCALE)
    assert torch.equal(got[:, :4], good[:, :4])


@pytest.mark.parametrize("maps", [1, 2])
@pytest.mark.parametrize("case", [CASES[4], CASES[9], CASES[11]], ids=["few", "many4", "many8"])
def test_captured_steps_replay(case, maps):
    """A captured step replays with new inputs in its buffers, eager calls of
    another plan between the replays, on a stream of its own."""
    b, h, g, d, m_c, m_d, n, page, lens = case
    if maps * (h // g) * n > 64:
        pytest.skip("more query rows than a unit takes")
    x = Problem(b, h, g, d, m_c, m_d, n, page, "mxfp4", maps=maps, lens=lens, seed=21)
    lam = torch.rand(h, generator=x.rng)
    dev = dict(q=x.q.cuda(), pages=x.pages(), ctx=x.ctx_table.cuda(), tab=x.tables.cuda(), lens=x.lens.cuda(), lam=lam.cuda())
    out = torch.zeros(b, h, n, d, dtype=torch.bfloat16, device="cuda")
    side = torch.cuda.Stream()

    def step(plan):
        a = (plan, dev["q"], dev["pages"], dev["ctx"], dev["tab"], dev["lens"])
        if maps == 2:
            bif.bifattn_paged_decode_diff(*a, dev["lam"], out)
        else:
            bif.bifattn_paged_decode(*a, out)

    with x.plan() as plan, x.plan() as other:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.stream(side):
            step(plan)
            side.synchronize()
            with torch.cuda.graph(graph, stream=side):
                step(plan)
        for k in range(4):
            q = torch.randn(b, h, n, d, generator=x.rng).to(torch.bfloat16)
            dev["q"].copy_(q.cuda())
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            got = out.clone()
            out.zero_()
            step(other)
            assert torch.equal(got, out)
            ref, tol = x.attention(lam=lam, q=q)
            assert ((got.cpu().double() - ref).abs() <= tol).all()
        assert bif.bifattn_paged_plan_status(plan) == bif.OK


def test_small_steps_are_one_launch_by_estimate(monkeypatch):
    monkeypatch.delenv("BIFATTN_WHOLE")
    for dims, path in (((4, 4, 4, 64, 128, 16), "standard"), ((32, 32, 32, 128, 8192, 512), "bifurcated"),
                       ((2, 64, 1, 128, 10, 10), "bifurcated")):  # 64 query rows per unit
        with bif.PagedPlan(*dims, page=16, num_pages=9) as plan:
            assert plan.info()["path"] == bif.PATHS[path]


def test_two_plans_on_two_streams():
    x = Problem(5, 32, 4, 128, 515, 65, 2, 16, "bf16", seed=30)
    y = Problem(4, 4, 4, 64, 128, 16, 1, 16, "mxfp4", seed=31)
    want = [attend(x), attend(y)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    plans = [x.plan(), y.plan()]
    args = [(z.q.cuda(), z.pages(), z.ctx_table.cuda(), z.tables.cuda(), z.lens.cuda()) for z in (x, y)]
    outs = [torch.zeros(z.b, z.h, z.n, z.d, dtype=torch.bfloat16, device="cuda") for z in (x, y)]
    torch.cuda.synchronize()
    for _ in range(10):
        for plan, a, out, s in zip(plans, args, outs, streams):
            bif.bifattn_paged_decode(plan, *a, out, stream=s)
    torch.cuda.synchronize()
    for out, w in zip(outs, want):
        assert torch.equal(out.cpu().double(), w)
    for plan in plans:
        assert bif.bifattn_paged_plan_status(plan) == bif.OK
        plan.close()


def test_one_token_shapes():
    """[b, h, d] queries and outputs when n = 1."""
    x = Problem(3, 8, 2, 128, 77, 40, page=32, seed=3)
    want = attend(x)
    with x.plan() as plan:
        out = torch.zeros(x.b, x.h, x.d, dtype=torch.bfloat16, device="cuda")
        bif.bifattn_paged_decode(plan, x.q[:, :, 0].contiguous().cuda(), x.pages(), x.ctx_table.cuda(), x.tables.cuda(), x.lens.cuda(), out)
        assert torch.equal(out.cpu().double(), want[:, :, 0])


@pytest.mark.parametrize("kv", ["bf16", "mxfp4"])
@pytest.mark.parametrize("maps", [1, 2])
@pytest.mark.parametrize("lens", [[70, 33, 64, 2], [5, 35, 3, 32]])
def test_nonfinite_rows_of_later_tokens(lens, maps, kv):
    """A draft token's infinite or NaN row reaches that token and the later ones
    alone: the rows before it are as with any other value there."""
    x = Problem(4, 6, 2, 128, 20, 70, n=4, page=16, kv=kv, maps=maps, lens=lens, seed=13)
    lam = torch.full((x.h,), 0.5)
    want = attend(x, lam=lam)
    for back in (1, 3):  # the last token's row, the last but two's
        bad = [int(v) - back for v in lens]
        for i, t in enumerate(bad):
            if t < 0:
                continue
            at = int(x.tables[i, t // 16]), t % 16
            if kv == "mxfp4":
                x.exps["V"][at[0], 1, at[1], 2] = x.exps["K"][at[0], 1, at[1], 0] = 255
            else:
                x.pool["V"][at[0], 1, at[1], 5:9] = torch.tensor([math.inf, -math.inf, math.nan, 1.0])
                x.pool["K"][at[0], 1, at[1], 3] = math.nan
        got = attend(x, lam=lam)
        assert torch.equal(got[:, :3], want[:, :3])
        for i, t in enumerate(bad):
            first = x.n - (1 if t < 0 else back)  # the first token that sees a bad row
            assert torch.equal(got[i, 3:, :first], want[i, 3:, :first])
            assert torch.isnan(got[i, 3:, first:]).any(-1).all()


def test_values_of_unlike_columns():
    """MXFP4 value columns of very different size, in both context kernels: each
    column of 32 elements keeps its own precision."""
    for b in (2, 40):
        x = Problem(b, 8, 2, 128, 300, 20, page=16, kv="mxfp4", lens=[20] * b, seed=14)
        for name, tab, n in (("ctx", x.ctx_table.view(1, -1), [300]), ("own", x.tables, [20] * b)):
            v = getattr(x, name)["V"] * torch.tensor([1.0, 2.0 ** 40, 2.0 ** -50, 2.0 ** 90]).repeat_interleave(32).double()
            got = x._put("V", v if name == "own" else v[None], tab, torch.tensor(n), None)
            getattr(x, name)["V"] = got if name == "own" else got[0]
        got = attend(x)
        ref, tol = x.attention()
        assert ((got - ref).abs() <= tol).all()


def test_norm_without_eps_of_a_row_of_zeros():
    """A token that sees no key stays 0 under the norm, with eps = 0 too."""
    x = Problem(3, 8, 2, 128, 0, 40, page=32, maps=2, lens=[0, 7, 40], seed=15)
    lam, weight = torch.full((x.h,), 0.5), torch.randn(x.d, generator=x.rng)
    got = attend(x, lam=lam, weight=weight, eps=0.0)
    assert (got[0] == 0).all()
    ref, tol = x.attention(lam=lam, weight=weight, eps=0.0)
    assert ((got - ref).abs() <= tol)[1:].all()


def test_nonfinite_rows_of_many_draft_tokens():
    """As above with 40 tokens, whose hidden rows span two tiles, in fp8."""
    x = Problem(2, 2, 2, 64, 20, 90, n=40, page=16, kv="fp8_e4m3", lens=[90, 41], seed=16)
    want = attend(x)
    for i, length in enumerate((90, 41)):
        for t in (length - 1, length - 33):  # of the last token, of the 8th
            at = int(x.tables[i, t // 16]), t % 16
            x.pool["V"][at[0], 0, at[1], 7] = 0x7F
    got = attend(x)
    assert torch.equal(got[:, 1], want[:, 1]) and torch.equal(got[:, 0, :7], want[:, 0, :7])
    assert torch.isnan(got[:, 0, 7:, 7]).all()
    rest = torch.arange(64) != 7
    ref, tol = x.attention()
    assert ((got - ref).abs() <= tol)[:, 0, 7:, rest].all()


def test_two_parts_of_one_step_in_a_graph_with_a_second_plan():
    """Two plans' steps in one captured graph, replayed: each has a workspace of
    its own."""
    x = Problem(5, 32, 4, 128, 515, 65, 2, 16, "bf16", seed=30)
    y = Problem(3, 8, 2, 128, 77, 40, 1, 32, "mxfp4", seed=31)
    want = [attend(x), attend(y)]
    plans = [x.plan(), y.plan()]
    args = [(z.q.cuda(), z.pages(), z.ctx_table.cuda(), z.tables.cuda(), z.lens.cuda()) for z in (x, y)]
    outs = [torch.zeros(z.b, z.h, z.n, z.d, dtype=torch.bfloat16, device="cuda") for z in (x, y)]
    side = torch.cuda.Stream()

    def step():
        for plan, a, out in zip(plans, args, outs):
            bif.bifattn_paged_decode(plan, *a, out)

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        step()
        side.synchronize()
        with torch.cuda.graph(graph, stream=side):
            step()
    for _ in range(4):
        for out in outs:
            out.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for out, w in zip(outs, want):
            assert torch.equal(out.cpu().double(), w)
    for plan in plans:
        plan.close()
