"""Paged caches where fewer bits would show: context weights far below the
largest one, values far below the largest of their column, elements next to a
border between codes, results of a rotation that cancel, norms of tiny and huge
heads (MI355X only)."""
import math

import numpy as np
import pytest
import torch

import paper_2403_08845_amd as bif

from .paged_ref import EPS32, HALF_BF16, Problem, rotated
from .test_paged_gpu import attend

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def in_parts(monkeypatch):
    monkeypatch.setenv("BIFATTN_WHOLE", "2")


def bounds(x, lam=None):
    """(out, tolerance) float64: every weight is off by half a step of 11 bits (the
    context's with codes and many rows; 2^-15 and less elsewhere) and, below 2^-24
    of the largest weight, by half a step of 2^-34 of it (an fp16 step of 2^-24
    where the largest is 2^10); by its 32-bit logit (w products, exponent and
    conversions) and the order of the 32-bit sums over the keys; the output by
    half a bf16 step."""
    b, h, g, d, n, m_c, m_d = (getattr(x, k) for k in ("b", "h", "g", "d", "n", "m_c", "m_d"))
    w, p = d // x.maps, h // g
    q = x.q.double().view(b, g, p, n, d)
    K, V = (torch.cat((x.ctx[k].expand(b, g, m_c, d), x.own[k]), 2)[:, :, None] for k in "KV")
    pos = torch.arange(m_c + m_d)
    seen = (pos < m_c + (x.lens.view(-1, 1, 1) - n + 1 + torch.arange(n).view(-1, 1)).clamp(min=0))[:, None, None]
    V = torch.where((pos < m_c + x.lens.view(-1, 1))[:, None, None, :, None], V, 0.0)
    maps = []
    for u in range(x.maps):
        f = slice(u * w, (u + 1) * w)
        logit = torch.where(seen, (q[..., f] @ K[..., f].transpose(-1, -2)) / math.sqrt(w), -math.inf)
        size = torch.where(seen, (q[..., f].abs() @ K[..., f].abs().transpose(-1, -2)) / math.sqrt(w), 0.0).amax(-1, keepdim=True)
        e = torch.exp(logit - logit.amax(-1, keepdim=True))
        total = e.sum(-1, keepdim=True)
        tau = 2.0 ** -11 + EPS32 * (2 * (m_c + m_d) + 4 * (w + 16) * (size + 1))
        maps.append(((e / total) @ V, (tau * (e @ V.abs()) + 2.0 ** -35 * (seen.double() @ V.abs())) / total))
    y, err = maps[0]
    if x.maps == 2:
        l = lam.double().view(g, p, 1, 1)
        y, err = y - l * maps[1][0], err + l.abs() * maps[1][1] + 4 * EPS32 * (y.abs() + (l * maps[1][0]).abs())
    return y.reshape(b, h, n, d), (HALF_BF16 * y.abs() + (1 + HALF_BF16) * err + 1e-30).reshape(b, h, n, d)


def within(x, lam=None):
    with x.plan() as plan:
        assert plan.info()["ctx_kernel"] == 2  # the many-row kernel
        got = attend(x, plan, lam=lam)
    ref, tol = bounds(x, lam)
    over = ((got - ref).abs() / tol).max().item()
    print(f"largest error {over:.3f} of the tolerance", flush=True)
    assert over <= 1


def put(x, K=None, V=None):
    """Store the changed rows {"ctx": [g, rows, d], "own": [b, g, rows, d]}."""
    for name, rows, scale in (("K", K, x.k_scale), ("V", V, x.v_scale)):
        if rows is not None:
            x.ctx[name] = x._put(name, rows["ctx"][None], x.ctx_table.view(1, -1), torch.tensor([x.m_c]), scale)[0]
            x.own[name] = x._put(name, rows["own"], x.tables, x.lens, scale)


MANY = [
    # b, h, g, d, m_c, m_d, n, page, maps
    (5, 32, 4, 128, 700, 20, 2, 16, 1),                       # 80 rows per group: four-wave work-groups
    (40, 32, 4, 128, 1500, 20, 1, 64, 1),                     # 320
    (9, 16, 4, 128, 700, 33, 1, 16, 2),
    (70, 16, 4, 64, 900, 20, 1, 32, 2),
]
IDS = ["many4", "many8", "diff4", "diff8"]


@pytest.mark.parametrize("logit", [-45, 14, 16, 18, 21])
@pytest.mark.parametrize("kv", ["fp8_e4m3", "mxfp4"])
@pytest.mark.parametrize("case", MANY, ids=IDS)
def test_context_weights_beside_a_dominant_key(case, kv, logit):
    """The first context key has a logit far from all others and a value row of
    zeros (an attention sink): the output comes from the others' small weights."""
    *dims, maps = case
    x = Problem(*dims, kv, maps=maps, seed=50)
    w = x.d // maps
    K = {"ctx": x.ctx["K"].clone(), "own": x.own["K"].clone()}
    V = {"ctx": x.ctx["V"].clone(), "own": x.own["V"].clone()}
    K["ctx"][:, 0], V["ctx"][:, 0] = 0, 0
    for u in range(maps):
        x.q[..., u * w] = 64
        K["ctx"][:, 1:, u * w], K["own"][..., u * w] = 0, 0
        K["ctx"][:, 0, u * w] = logit * math.sqrt(w) / 64
    put(x, K, V)
    within(x, lam=torch.linspace(-0.2, 0.9, x.h))


@pytest.mark.parametrize("kv", ["fp8_e4m3", "mxfp4"])
@pytest.mark.parametrize("case", MANY, ids=IDS)
def test_rising_logits_over_codes(case, kv):
    *dims, maps = case
    x = Problem(*dims, kv, maps=maps, seed=51)
    x.q = x.q.abs()
    ramp = {name: torch.linspace(0.05, 2, rows).double().view(-1, 1) for name, rows in (("ctx", x.m_c), ("own", x.m_d))}
    put(x, {name: getattr(x, name)["K"].abs() * ramp[name] for name in ramp})
    within(x, lam=torch.linspace(-0.2, 0.9, x.h))


@pytest.mark.parametrize("case", MANY, ids=IDS)
def test_values_beside_a_far_larger_one_of_their_column(case):
    """MXFP4 values 2^-34 times the largest of their column, whose key has next to
    no weight."""
    *dims, maps = case
    x = Problem(*dims, "mxfp4", maps=maps, seed=52)
    w = x.d // maps
    K = {"ctx": x.ctx["K"].clone(), "own": x.own["K"].clone()}
    V = {"ctx": x.ctx["V"] * 2.0 ** -34, "own": x.own["V"] * 2.0 ** -34}
    K["ctx"][:, 0], V["ctx"][:, 0] = 0, 6
    for u in range(maps):
        x.q[..., u * w] = 64
        K["ctx"][:, 1:, u * w], K["own"][..., u * w] = 0, 0
        K["ctx"][:, 0, u * w] = -64 * math.sqrt(w) / 64
    put(x, K, V)
    within(x, lam=torch.linspace(-0.2, 0.9, x.h))


def test_fp8_read_out_is_rounded_once():
    """Products of a code and a scale just off the middle between two bf16 values:
    rounded to fp32 first they would meet it and go to the even one."""
    codes = torch.arange(256, dtype=torch.uint8)
    codes = codes[(codes & 127) != 127]
    values = codes.view(torch.float8_e4m3fn).double()
    r = torch.Generator().manual_seed(1)
    scale = torch.exp2(8 * torch.rand(1 << 16, generator=r) - 4)
    exact = values * scale.double().view(-1, 1)  # 28 bits

    def nearest(y):  # bf16, in one rounding
        step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -126))) - 7)
        return torch.round(y / step) * step

    twice = exact.float().to(torch.bfloat16).double()
    bad = (nearest(exact) != twice).any(1).nonzero().flatten()
    assert bad.numel() >= 2
    g, rows = 16, 4
    scale = torch.cat((scale[bad], scale))[:g].contiguous()
    x = Problem(1, g, g, 64, 0, rows, page=16, kv="fp8_e4m3", lens=[rows], seed=8)
    x.k_scale, x.v_scale = scale, scale.flip(0).contiguous()
    page = int(x.tables[0, 0])
    stored = torch.zeros(rows * 64, dtype=torch.uint8)
    stored[:codes.numel()] = codes
    stored = stored.view(rows, 64)
    for name in "KV":
        x.pool[name][page, :, :rows] = stored
    outs = [torch.zeros(1, g, rows, 64, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    with x.plan() as plan:
        bif.bifattn_paged_gather(plan, x.pages(), x.tables.cuda(), x.lens.cuda(), *outs)
        assert bif.bifattn_paged_plan_status(plan) == bif.OK
    for got, s in zip(outs, (x.k_scale, x.v_scale)):
        want = nearest(stored.view(torch.float8_e4m3fn).double() * s.double().view(-1, 1, 1))
        assert torch.equal(got[0].cpu().double(), want)


@pytest.mark.parametrize("rot", [0, 64])
def test_fp8_ties_of_quotients(rot):
    """x / scale exactly in the middle between two codes goes to the even one, also
    where x times the rounded reciprocal of the scale is below it (147 / 49)."""
    assert 147.0 * (1.0 / 49.0) < 3.0
    x = Problem(1, 1, 1, 64, 0, 1, page=16, kv="fp8_e4m3", lens=[1], seed=9)
    x.k_scale = x.v_scale = torch.tensor([49.0 / 64])
    row = torch.zeros(64)
    row[:4] = torch.tensor([147.0, -147.0, 49.0, 245.0]) * 2.0 ** -16  # 3, -3, 1 and 5 halves of the least code
    kv = row.to(torch.bfloat16).view(1, 1, 1, 64).cuda()
    pages = x.pages()
    lens = torch.zeros(1, dtype=torch.int32, device="cuda")
    with x.plan() as plan:  # position 0: no turn
        bif.bifattn_paged_append(plan, pages, x.tables.cuda(), lens, kv, kv, lens,
                                 freqs=torch.ones(32, device="cuda") if rot else None)
        assert bif.bifattn_paged_plan_status(plan) == bif.OK
    for t in (pages.K, pages.V):
        got = t[int(x.tables[0, 0]), 0, 0].cpu().view(torch.float8_e4m3fn).double()
        assert got[:5].tolist() == [2 * 2.0 ** -9, -2 * 2.0 ** -9, 0, 2 * 2.0 ** -9, 0]


# position, x, y, frequency near atan(x / y) / position: x cos - y sin cancels to
# about 2^-25 and lies within 2^-14 of a border between E2M1 codes of unit 2^-26
CANCELLED = [
    (1, 1.5703125, 1.984375, 0.6694372296333313),
    (4, 1.5703125, 1.984375, 0.16735930740833282),
    (7, 1.3203125, 1.1484375, 0.12212946265935898),
    (11, 1.7265625, 1.1328125, 0.09001261740922928),
    (27, 1.7265625, 1.7265625, 0.0290888212621212),
    (33, 1.578125, 1.1796875, 0.028147917240858078),
    (37, 1.015625, 1.9140625, 0.01318476814776659),
]


@pytest.mark.parametrize("case", CANCELLED, ids=lambda c: "position%d" % c[0])
def test_codes_of_cancelled_rotations(case):
    """Cosine and sine enter codes with 64 bits: the element falls on its side of
    the border (80-bit reference)."""
    position, a, c, f = case
    turn = np.longdouble(np.float32(f)) * position
    z = float(np.abs(np.longdouble(a) * np.cos(turn) - np.longdouble(c) * np.sin(turn)) * np.longdouble(2) ** 26)
    grid = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])
    middle = (grid[1:] + grid[:-1]) / 2
    assert 2.0 ** -20 < np.abs(z - middle).min() < 2.0 ** -14
    want = int(np.searchsorted(middle, z))
    x = Problem(1, 1, 1, 64, 0, 64, page=64, kv="mxfp4", lens=[64], seed=9)
    row, freqs = torch.zeros(64), torch.zeros(32)
    row[0] = 5 * 2.0 ** -26  # the largest of the block: unit 2^-26
    row[1], row[33], freqs[1] = a, c, f
    kv = row.to(torch.bfloat16).view(1, 1, 1, 64).cuda()
    assert torch.equal(kv.cpu().float().flatten(), row)
    pages = x.pages()
    lens = torch.tensor([position], dtype=torch.int32, device="cuda")
    with x.plan() as plan:
        bif.bifattn_paged_append(plan, pages, x.tables.cuda(), lens, kv, kv, lens, freqs=freqs.cuda())
        assert bif.bifattn_paged_plan_status(plan) == bif.OK
    at = int(x.tables[0, 0]), 0, position
    assert int(pages.K_exp[at][0]) == 127 - 26
    assert int(pages.K[at][0]) >> 4 & 7 == want


def test_rotations_that_cancel():
    """Rotated queries and bf16 keys against 80 bits: off by 2^-37 of |x| + |y| (the
    rest of cosine and sine, 2^-15 of them, its two products and the main part's
    excess over the result by as much, each rounded to 24 bits: four times 2^-39),
    by the angle's 2^-51 of itself times that, and by one rounding; also at
    positions near 2^29."""
    n = 32
    r = np.random.default_rng(4)
    for m_c in (0, 3, (1 << 29) - 100):
        x = Problem(1, 2, 1, 64, 0, 64, page=64, lens=[64], seed=9)
        x.m_c = m_c
        lo, hi = ((1 + r.integers(0, 128, 32) / 128) for _ in range(2))
        freqs = (np.arctan2(lo, hi) / max(1, m_c) if m_c < 100 else r.uniform(0.5, 1, 32)).astype(np.float32)
        row = torch.tensor(np.concatenate((lo, hi))).to(torch.bfloat16)
        kv = row.view(1, 1, 1, 64).expand(1, 1, n, 64).contiguous().cuda()
        q = kv.expand(1, 2, n, 64)
        pages = x.pages()
        out = torch.zeros(1, 2, n, 64, dtype=torch.bfloat16, device="cuda")
        lens = torch.zeros(1, dtype=torch.int32, device="cuda")
        with x.plan() as plan:
            bif.bifattn_paged_append(plan, pages, x.tables.cuda(), lens, kv, kv, lens, q=q, q_out=out,
                                     freqs=torch.from_numpy(freqs).cuda())
            assert bif.bifattn_paged_plan_status(plan) == bif.OK
        keys = pages.K[int(x.tables[0, 0]), 0].cpu().double().numpy()
        for t in range(n):
            turn = freqs.astype(np.longdouble) * (m_c + t)
            c, s = np.cos(turn), np.sin(turn)
            want = np.concatenate((lo * c - hi * s, lo * s + hi * c)).astype(np.float64)
            size = np.tile(lo + hi, 2)
            tol = 2.0 ** -8 * np.abs(want) + (2.0 ** -37 + 2.0 ** -51 * np.tile(turn.astype(np.float64), 2)) * size
            for got in (out[0, 0, t].cpu().double().numpy(), out[0, 1, t].cpu().double().numpy(), keys[t]):
                assert (np.abs(got - want) <= tol).all()


@pytest.mark.parametrize("launches", ["parts", "one launch"])
@pytest.mark.parametrize("power", [-95, -80, 64, 90])
@pytest.mark.parametrize("d", [64, 128])
def test_norm_of_tiny_and_huge_heads(d, power, launches, monkeypatch):
    """Heads whose squares leave fp32's range are normalised like others."""
    monkeypatch.setenv("BIFATTN_WHOLE", "2" if launches == "parts" else "1")
    x = Problem(3, 8, 2, d, 40, 40, page=32, maps=2, lens=[0, 7, 40], seed=15)
    put(x, V={name: getattr(x, name)["V"] * 2.0 ** power for name in ("ctx", "own")})
    lam, weight = torch.full((x.h,), 0.5), torch.randn(x.d, generator=x.rng)
    for eps in (0.0, 1e-5):
        got = attend(x, lam=lam, weight=weight, eps=eps)
        ref, tol = x.attention(lam=lam, weight=weight, eps=eps)
        assert ((got - ref).abs() <= tol).all(), eps


@pytest.mark.parametrize("launches", ["parts", "one launch"])
@pytest.mark.parametrize("map_", [0, 1])
@pytest.mark.parametrize("case", [(4, 4, 4, 128, 130, 16, 1, 16), (3, 8, 2, 64, 77, 40, 4, 32), (2, 16, 1, 128, 300, 33, 2, 64),
                                  (9, 16, 4, 128, 515, 65, 1, 16)], ids=["few", "drafts", "four_tiles", "many"])
def test_infinite_keys_of_one_map(case, map_, launches, monkeypatch):
    """A key element of one map that is -infinity takes the key's weight in that
    map alone, as a very negative finite one does."""
    monkeypatch.setenv("BIFATTN_WHOLE", "2" if launches == "parts" else "1")
    x = Problem(*case, "bf16", maps=2, lens=[case[5]] * case[0], seed=70)
    at = map_ * x.d // 2 + 3
    x.q[..., at] = 1
    lam = torch.linspace(0.2, 0.9, x.h)
    got = {}
    for value in (-2.0 ** 60, -math.inf):
        K = {name: getattr(x, name)["K"].clone() for name in ("ctx", "own")}
        K["ctx"][:, 5, at], K["own"][:, :, 1, at] = value, value
        put(x, K)
        got[value] = attend(x, lam=lam)
    assert torch.equal(got[-2.0 ** 60], got[-math.inf])
    for rows in (x.ctx, x.own):  # a logit of -62 or less instead: next to no weight
        rows["K"] = torch.where(rows["K"].isinf(), -500.0, rows["K"])
    ref, tol = bounds(x, lam)
    assert torch.isfinite(got[-math.inf]).all()
    assert ((got[-math.inf] - ref).abs() <= tol).all()


@pytest.mark.parametrize("scale", [1.0, 0.93, 0.87, 0.79, 0.71])
@pytest.mark.parametrize("kv", ["bf16", "fp8_e4m3", "mxfp4"])
@pytest.mark.parametrize("case", MANY[:2], ids=IDS[:2])
def test_differences_of_huge_logits(case, kv, scale):
    """Logits 2^25 and 2^25 + 4, whose differences are exact: the weights are those
    of 0 and 4."""
    *dims, _ = case
    x = Problem(*dims, kv, seed=71, scaled=False)
    x.q[:] = 0
    x.q[..., 0], x.q[..., 1] = 2.0 ** 25, 1
    K = {name: torch.zeros_like(getattr(x, name)["K"]) for name in ("ctx", "own")}
    for rows in K.values():
        rows[..., 0] = 1
    K["ctx"][:, 300:, 1] = 4
    put(x, K)
    got = attend(x, scale=scale)
    pos = torch.arange(x.m_c + x.m_d)
    own = (x.lens.view(-1, 1) - x.n + 1 + torch.arange(x.n)).clamp(min=0)  # [b, n]
    seen = pos < x.m_c + own.unsqueeze(-1)
    e = torch.where(seen, torch.where((pos >= 300) & (pos < x.m_c), 1.0, math.exp(-4 * scale)), 0.0).double()[:, None]
    V = torch.cat((x.ctx["V"].expand(x.b, *x.ctx["V"].shape), x.own["V"]), 2)
    V = torch.where((pos < x.m_c + x.lens.view(-1, 1))[:, None, :, None], V, 0.0)
    e = e / e.sum(-1, keepdim=True)
    ref, size = ((e @ v).repeat_interleave(x.h // x.g, 1) for v in (V, V.abs()))
    # the scale's own rounding, 2^-24 of the difference; the sums' order
    tol = HALF_BF16 * ref.abs() + (1 + HALF_BF16) * (2.0 ** -11 + EPS32 * (8 + 2 * pos.numel())) * size
    print("largest error", ((got - ref).abs() / tol).max().item(), "of the tolerance", flush=True)
    assert ((got - ref).abs() <= tol).all()


@pytest.mark.parametrize("launches", ["parts", "one launch"])
@pytest.mark.parametrize("value", [math.inf, math.nan])
def test_nonfinite_values_without_weight(value, launches, monkeypatch):
    """A draft token's row with an infinity or a NaN in its value and a key that
    leaves it no weight makes NaN of the tokens that see it, as 0 times it is, and
    of no other."""
    monkeypatch.setenv("BIFATTN_WHOLE", "2" if launches == "parts" else "1")
    lens = [70, 33, 64, 40]
    x = Problem(4, 6, 2, 128, 20, 70, n=4, page=16, kv="bf16", lens=lens, seed=13)
    x.q[..., 3] = 1
    K, V = ({name: getattr(x, name)[k].clone() for name in ("ctx", "own")} for k in "KV")
    for i, length in enumerate(lens):
        K["own"][i, 1, length - 3, 3] = -2.0 ** 40  # the second token's row
    put(x, K)
    want = attend(x)
    for i, length in enumerate(lens):
        V["own"][i, 1, length - 3, 5] = value
    put(x, V=V)
    got = attend(x)
    seen = torch.zeros_like(got, dtype=torch.bool)
    seen[:, 3:, 1:, 5] = True
    assert torch.isnan(got[seen]).all() and torch.equal(got[~seen], want[~seen])
