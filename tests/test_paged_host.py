"""The paged caches' host side (CPU only): refusals of the C ABI and of the
binding, the work split, and the 64-bit reference of the GPU tests."""
import ctypes
import math
import os
import shutil

import pytest
import torch

import paper_2403_08845_amd as bif

from .paged_ref import Problem, e4m3, mx_codes, mx_values, rotated, stored
from .test_sanitizers import ROCM, ROOT, SAN, _run


@pytest.mark.skipif(shutil.which("g++") is None or not os.path.isdir(os.path.join(ROCM, "include", "hip")),
                    reason="g++ or the HIP headers missing")
def test_refusals_and_work_splits_under_sanitizers(tmp_path):
    import subprocess
    exe = str(tmp_path / "paged_san")
    csrc = os.path.join(ROOT, "paper_2403_08845_amd", "csrc")
    subprocess.check_call(["g++", "-std=c++17", *SAN, "-Wall", "-D__HIP_PLATFORM_AMD__", f"-I{ROCM}/include",
                           f"-I{ROOT}/include", f"-I{csrc}", os.path.join(csrc, "bifattn_paged_host.cpp"),
                           os.path.join(ROOT, "tests", "sanitize", "paged_driver.cpp"), "-o", exe])
    assert "all checks passed" in _run(exe, leaks=True)


def test_plan_create_refuses_bad_dims_without_a_device():
    L = bif.lib()
    for dims, want in (((0, 4, 4, 64, 128, 16, 16, 9), bif.EINVAL), ((4, 4, 4, 64, 0, 0, 16, 9), bif.EINVAL),
                       ((4, 4, 4, 64, 128, 16, 8, 9), bif.EUNSUPPORTED), ((4, 4, 4, 64, 128, 16, 16, 0), bif.EINVAL)):
        d, handle = bif.PagedDims(*dims), ctypes.c_void_p(77)
        assert L.bifattn_paged_plan_create(ctypes.byref(d), ctypes.byref(handle)) == want and handle.value is None
    assert L.bifattn_paged_plan_create(None, None) == bif.EINVAL
    # the contiguous caches' plans do not take the paged element type
    d, handle = bif.Dims(2, 4, 2, 64, 128, 16, 0.0, 1, 4), ctypes.c_void_p()
    assert L.bifattn_plan_create(ctypes.byref(d), ctypes.byref(handle)) == bif.EINVAL
    with pytest.raises(ValueError):
        bif.PagedPlan(2, 4, 2, 64, 128, 16, kv="int8")
    assert bif.status_string(bif.EPAGE) != bif.status_string(12345)


class FakePlan:
    def __init__(self, kv="bf16", maps=1):
        self.kv = kv
        self.dims = bif.PagedDims(2, 4, 2, 64, 32, 20, 16, 9, 0.0, 1, bif.PAGED_KV_TYPES[kv], maps)
        self.handle = ctypes.c_void_p(0)
        self.device = torch.device("cpu")  # host tensors pass the device check up to is_cuda


def test_binding_refuses_before_any_call():
    bf, i32 = torch.bfloat16, torch.int32
    k = torch.zeros(2, 2, 3, 64, dtype=bf)
    lens = torch.zeros(2, dtype=i32)
    table = torch.zeros(2, 2, dtype=i32)
    pages = bif.Pages(*(torch.zeros(9, 2, 16, 64, dtype=bf) for _ in range(2)))
    plan = FakePlan()
    with pytest.raises(TypeError):
        bif.bifattn_paged_append(plan, pages, table, lens, k.float(), k, lens, stream=0)
    with pytest.raises(TypeError):
        bif.bifattn_paged_append(plan, pages, table, lens, None, k, lens, stream=0)
    with pytest.raises(ValueError):  # q without q_out
        bif.bifattn_paged_append(plan, pages, table, lens, k, k, lens, q=k, stream=0)
    with pytest.raises(ValueError):  # groups
        bif.bifattn_paged_append(plan, pages, table, lens, k[:, :1], k, lens, stream=0)
    with pytest.raises(ValueError):  # host memory
        bif.bifattn_paged_append(plan, pages, table, lens, k, k, lens, stream=0)
    with pytest.raises(TypeError):
        bif.bifattn_paged_append(plan, pages, table, lens, k, k, lens, freqs=[1.0], stream=0)
    with pytest.raises(TypeError):
        bif.bifattn_paged_gather(plan, pages, table, lens, k[0], k, stream=0)
    q = torch.zeros(2, 4, 1, 64, dtype=bf)
    with pytest.raises(TypeError):
        bif.bifattn_paged_decode(plan, q.float(), pages, table[0], table, lens, q, stream=0)
    with pytest.raises(ValueError):
        bif.bifattn_paged_decode(plan, q[:1], pages, table[0], table, lens, q, stream=0)
    with pytest.raises(TypeError):
        bif._pages(plan, (pages.K, pages.V))
    with pytest.raises(ValueError):
        bif._pages(plan, pages._replace(K_exp=pages.K))
    with pytest.raises(ValueError):
        bif._pages(plan, pages._replace(k_scale=torch.ones(2)))
    with pytest.raises(ValueError):
        bif._pages(FakePlan("mxfp4"), pages)


def test_reference_attention_is_the_softmax():
    """The reference against torch's own softmax, row by row, with and without
    keys."""
    x = Problem(2, 4, 2, 64, 5, 9, n=3, page=16, kv="bf16", maps=2, lens=[9, 1], seed=1)
    lam = torch.rand(4)
    y, tol = x.attention(lam=lam)
    for i in range(2):
        for j in range(4):
            for r in range(3):
                seen = 5 + max(0, int(x.lens[i]) - 3 + r + 1)
                K = torch.cat((x.ctx["K"][j // 2], x.own["K"][i, j // 2]))[:seen]
                V = torch.cat((x.ctx["V"][j // 2], x.own["V"][i, j // 2]))[:seen]
                q = x.q[i, j, r].double()
                a = [torch.softmax(K[:, f] @ q[f] / math.sqrt(32), 0) @ V for f in (slice(0, 32), slice(32, 64))]
                assert torch.allclose(a[0] - lam[j].double() * a[1], y[i, j, r], rtol=1e-12, atol=1e-12)
    empty = Problem(1, 1, 1, 64, 0, 4, n=2, lens=[1], seed=1).attention()[0]
    assert (empty[0, 0, 0] == 0).all() and (empty[0, 0, 1] != 0).any()


def test_reference_encodings():
    x = torch.linspace(-500, 500, 4001, dtype=torch.float64)
    want = x.clamp(-448, 448).float().to(torch.float8_e4m3fn).double()
    assert torch.equal(e4m3(x), want)
    tie = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0]).double().repeat(4)
    k, e = mx_codes(tie)
    assert e.tolist() == [0] and mx_values(k, e)[:8].tolist() == [0, 1, 1, 2, 2, 4, 4, 6]
    assert mx_codes(torch.zeros(32).double())[1].tolist() == [-126]
    bits, exps, values = stored(torch.randn(1, 3, 64, dtype=torch.float64), "mxfp4")
    assert bits.shape == (1, 3, 32) and exps.shape == (1, 3, 2) and values.shape == (1, 3, 64)
    row = torch.arange(64, dtype=torch.float64)
    turned = rotated(row, torch.tensor(0), torch.ones(16), True, 2)
    assert torch.equal(turned, row)
    quarter = rotated(row, torch.tensor(1), torch.full((16,), math.pi / 2), False, 1)
    # the angle is fp32's pi / 2: off by 4.4e-8
    assert torch.allclose(quarter[:16], -row[16:32], atol=1e-5) and torch.allclose(quarter[16:32], row[:16], atol=1e-5)
