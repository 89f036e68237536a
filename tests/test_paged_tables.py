"""The README's example of paged caches runs as written, and one table of the
context serves append, read-out and attention (MI355X only)."""
import os
import re

import pytest
import torch

import paper_2403_08845_amd as bif

from .paged_ref import Problem

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_readme_paged_example_runs():
    src = open(os.path.join(ROOT, "README.md"), encoding="utf-8").read()
    blocks = re.findall(r"```python\n(.*?)```", src, re.S)
    paged = [t for t in blocks if "PagedPlan" in t]
    assert paged, "no example of paged caches in the README"
    scope = {}
    exec(compile(blocks[0], "README.md", "exec"), scope)  # the sizes
    for text in paged:
        exec(compile(text, "README.md", "exec"), scope)
    out, lens = scope["out"], scope["lens"]
    assert bool(out.isfinite().all()) and bool((out != 0).any())
    assert lens.unique().tolist() == [1] and scope["ctx_len"].item() == scope["m_c"]


@pytest.mark.parametrize("native", [True, False])
def test_one_context_table_for_all_calls(native):
    """[pages] and [1, pages], by the native checks (which take both) and Python's."""
    x = Problem(3, 4, 2, 64, 50, 12, page=16, kv="bf16", lens=[12, 5, 7], seed=2)
    new = torch.randn(2, 1, 2, 50, 64, generator=x.rng).to(torch.bfloat16).cuda()
    seen = []
    with x.plan() as plan:
        caller = plan._caller
        assert caller is not None
        if not native:
            plan._caller = None
        for table in (x.ctx_table.cuda(), x.ctx_table.view(1, -1).cuda()):
            pages = x.pages()
            length = torch.zeros(1, dtype=torch.int32, device="cuda")
            outs = [torch.zeros(1, 2, 50, 64, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
            out = torch.zeros(3, 4, 1, 64, dtype=torch.bfloat16, device="cuda")
            tables, lens, q = x.tables.cuda(), x.lens.cuda(), x.q.cuda()
            bif.bifattn_paged_append(plan, pages, table, length, new[0], new[1], length, context=True)
            bif.bifattn_paged_gather(plan, pages, table, length, *outs, context=True)
            bif.bifattn_paged_decode(plan, q, pages, table, tables, lens, out)
            if native:
                stream = torch.cuda.current_stream().cuda_stream
                assert caller.decode(q, pages, table, tables, lens, out, stream) == bif.OK
                assert caller.gather(pages, table, length, *outs, None, True, stream) == bif.OK
            assert bif.bifattn_paged_plan_status(plan) == bif.OK
            assert torch.equal(outs[0], new[0]) and torch.equal(outs[1], new[1])
            seen.append(out)
        assert torch.equal(*seen)
        with pytest.raises(ValueError):  # a sample's table keeps its two axes
            bif.bifattn_paged_append(plan, pages, x.tables[0].cuda(), lens[:1], new[0][:, :, :1], new[1][:, :, :1], lens[:1])
        with pytest.raises(ValueError):
            bif.bifattn_paged_gather(plan, pages, table[:, :-1], length, *outs, context=True)
        plan._caller = caller


def test_alignment_of_the_norm_weight():
    """A weight in the middle of a fused buffer is refused unless it lies at a
    multiple of 16 bytes; the output is left as it was."""
    x = Problem(2, 4, 2, 64, 20, 12, page=16, maps=2, lens=[12, 5], seed=2)
    fused = torch.randn(64 * 3, generator=x.rng).cuda()
    lam = fused[1:5]  # 4 bytes are enough
    args = (x.q.cuda(), x.pages(), x.ctx_table.cuda(), x.tables.cuda(), x.lens.cuda(), lam)
    out = torch.full((2, 4, 1, 64), 3.0, dtype=torch.bfloat16, device="cuda")
    with x.plan() as plan:
        for at in (1, 2, 3, 66):
            with pytest.raises(bif.BifattnError) as e:
                bif.bifattn_paged_decode_diff(plan, *args, out, weight=fused[at:at + 64])
            assert e.value.status == bif.EALIGN
        torch.cuda.synchronize()
        assert (out == 3.0).all()
        other = torch.zeros_like(out)
        bif.bifattn_paged_decode_diff(plan, *args, out, weight=fused[68:132])
        bif.bifattn_paged_decode_diff(plan, *args, other, weight=fused[68:132].clone())
        assert bif.bifattn_paged_plan_status(plan) == bif.OK
        assert torch.equal(out, other) and bool(out.isfinite().all())
