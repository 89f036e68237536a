"""Appends whose arrays of lengths and counts are the same memory: on the CPU
which are refused, on an MI355X that every work-group has its inputs."""
import os
import shutil
import subprocess

import pytest
import torch

import paper_2403_08845_amd as bif

from .paged_ref import Problem
from .test_sanitizers import ROCM, ROOT, SAN, _run


@pytest.mark.skipif(shutil.which("g++") is None or not os.path.isdir(os.path.join(ROCM, "include", "hip")),
                    reason="g++ or the HIP headers missing")
def test_overlapping_lengths_on_the_host(tmp_path):
    exe = str(tmp_path / "paged_overlap")
    csrc = os.path.join(ROOT, "paper_2403_08845_amd", "csrc")
    subprocess.check_call(["g++", "-std=c++17", *SAN, "-Wall", "-Wno-unused-function", "-D__HIP_PLATFORM_AMD__",
                           f"-I{ROCM}/include", f"-I{ROOT}/include", f"-I{csrc}",
                           os.path.join(csrc, "bifattn_paged_host.cpp"),
                           os.path.join(ROOT, "tests", "sanitize", "paged_overlap_driver.cpp"), "-o", exe])
    assert "all checks passed" in _run(exe, leaks=True)


@pytest.mark.gpu
@pytest.mark.parametrize("b,n", [(3, 5), (40, 70)])
def test_counts_replaced_by_lengths(b, n):
    """Prompts of different lengths into empty sequences, whose lengths the counts'
    array holds and receives: every row of every sample is written."""
    x = Problem(b, 8, 2, 128, 7, 80, page=16, kv="bf16", lens=[80] * b, seed=60)
    r = torch.Generator().manual_seed(61)
    y = torch.randn(b, n, 12, 128, generator=r).to(torch.bfloat16).cuda().transpose(1, 2)
    q, k, v = y[:, :8], y[:, 8:10], y[:, 10:]
    start = torch.randint(0, 80 - n + 1, (b,), generator=r).to(torch.int32)
    count = torch.randint(0, n + 1, (b,), generator=r).to(torch.int32)
    freqs = torch.rand(64, generator=r).cuda()
    tables = x.tables.cuda()
    seen = []
    with x.plan() as plan:
        for form in ("apart", "lengths", "counts", "counts", "counts"):
            pages = x.pages()
            q_out = torch.zeros(b, 8, n, 128, dtype=torch.bfloat16, device="cuda")
            lens, counts = start.cuda(), count.cuda()
            out = {"apart": torch.zeros_like(lens), "lengths": lens, "counts": counts}[form]
            bif.bifattn_paged_append(plan, pages, tables, lens, k, v, out, q=q, q_out=q_out, counts=counts, freqs=freqs)
            assert bif.bifattn_paged_plan_status(plan) == bif.OK
            assert torch.equal(out.cpu(), start + count)
            seen.append((pages.K.view(torch.int16), pages.V.view(torch.int16), q_out.view(torch.int16)))
        for got in seen[1:]:
            assert all(torch.equal(a, z) for a, z in zip(got, seen[0]))
        both = torch.zeros(b + 1, dtype=torch.int32, device="cuda")
        with pytest.raises(bif.BifattnError):
            bif.bifattn_paged_append(plan, pages, tables, both[:-1], k, v, both[1:])
