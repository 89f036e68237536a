"""The paged calls' native argument checks take and refuse what the Python
checks do, with the same results and errors (MI355X only)."""
import pytest
import torch

import paper_2403_08845_amd as bif

from .paged_ref import Problem

pytestmark = pytest.mark.gpu


def both_ways(plan, call, state):
    native = plan._caller
    assert native is not None  # the module that was built loads
    seen = []
    for caller in (native, None):
        plan._caller = caller
        try:
            s = {k: v.clone() if isinstance(v, torch.Tensor) else v for k, v in state().items()}
            call(plan, s)
            torch.cuda.synchronize()
            seen.append(("ok", {k: v for k, v in s.items() if isinstance(v, torch.Tensor)}))
        except Exception as e:
            seen.append((type(e).__name__, str(e)))
    plan._caller = native
    return seen


def same(seen, name):
    assert seen[0][0] == seen[1][0], (name, seen)
    if seen[0][0] != "ok":
        assert seen[0][1] == seen[1][1], (name, seen)
    else:
        for k, v in seen[0][1].items():
            assert torch.equal(v.contiguous().view(torch.uint8), seen[1][1][k].contiguous().view(torch.uint8)), (name, k)


def misaligned(t):
    base = torch.empty(t.numel() + 1, dtype=t.dtype, device=t.device)
    base[1:].copy_(t.reshape(-1))
    return base[1:].view(t.shape)


@pytest.mark.parametrize("kv,maps,n", [("bf16", 1, 1), ("fp8_e4m3", 2, 2), ("mxfp4", 1, 2)])
def test_native_and_python_checks_agree(kv, maps, n):
    x = Problem(3, 4, 2, 64, 20, 12, n, 16, kv, maps=maps, lens=[12, 5, 7], seed=2)
    pages = x.pages()
    r = torch.Generator().manual_seed(3)

    class Sub(torch.Tensor):
        pass

    with x.plan() as plan:
        def attention():
            return dict(q=x.q.cuda(), ctx=x.ctx_table.cuda(), tab=x.tables.cuda(), lens=x.lens.cuda(),
                        lam=torch.rand(4, device="cuda"), weight=torch.ones(64, device="cuda"),
                        out=torch.zeros(3, 4, n, 64, dtype=torch.bfloat16, device="cuda"))
        fixed = attention()

        def attend(plan, s):
            p = s.get("pages", pages)
            if maps == 2:
                bif.bifattn_paged_decode_diff(plan, s["q"], p, s["ctx"], s["tab"], s["lens"], s["lam"], s["out"],
                                              weight=s["weight"], eps=s.get("eps", 1e-5))
            else:
                bif.bifattn_paged_decode(plan, s["q"], p, s["ctx"], s["tab"], s["lens"], s["out"])

        wide = torch.cat([pages.K, pages.K], dim=1)
        forms = {"valid": {}, "parameter": dict(q=torch.nn.Parameter(fixed["q"], requires_grad=False)),
                 "subclass": dict(q=fixed["q"].as_subclass(Sub)), "row of a table": dict(ctx=fixed["ctx"].view(1, -1)),
                 "long lens": dict(lens=fixed["lens"].long()), "short table": dict(tab=fixed["tab"][:, :0]),
                 "half": dict(q=fixed["q"].half()), "fp32 out": dict(out=fixed["out"].float()),
                 "host": dict(lens=x.lens), "none": dict(tab=None), "list": dict(ctx=[1]),
                 "misaligned": dict(q=misaligned(fixed["q"])), "no weight": dict(weight=None),
                 "short weight": dict(weight=fixed["weight"][:5]), "negative eps": dict(eps=-1.0), "whole eps": dict(eps=0),
                 "pages tuple": dict(pages=tuple(pages)), "few pages": dict(pages=pages._replace(K=pages.K[1:])),
                 "strided pages": dict(pages=pages._replace(K=wide[:, ::2])),
                 "scales": dict(pages=pages._replace(k_scale=torch.ones(2, device="cuda"))),
                 "exps": dict(pages=pages._replace(V_exp=torch.ones(x.num_pages, 2, 16, 2, dtype=torch.uint8, device="cuda"))),
                 "no exps": dict(pages=pages._replace(K_exp=None))}
        if n == 1:
            forms["flat"] = dict(q=fixed["q"][:, :, 0], out=fixed["out"][:, :, 0])
        for name, change in forms.items():
            if name in ("no weight", "short weight", "negative eps", "whole eps") and maps == 1:
                continue
            print(f"[case] attention {kv} {name}", flush=True)
            same(both_ways(plan, attend, lambda: dict(fixed, **change)), name)

        y = torch.randn(3, 5, 4 + 2 + 2, 64, generator=r).to(torch.bfloat16).cuda().transpose(1, 2)
        new = dict(k=y[:, 4:6], v=y[:, 6:], q=y[:, :4], q_out=torch.zeros(3, 4, 5, 64, dtype=torch.bfloat16, device="cuda"),
                   counts=torch.tensor([5, 0, 3], dtype=torch.int32, device="cuda"), freqs=torch.rand(16, device="cuda"),
                   tab=fixed["tab"], lens=torch.zeros(3, dtype=torch.int32, device="cuda"),
                   lens_out=torch.zeros(3, dtype=torch.int32, device="cuda"),
                   K=pages.K, V=pages.V, **({} if pages.K_exp is None else dict(K_exp=pages.K_exp, V_exp=pages.V_exp)))

        def append(plan, s):
            # clones are contiguous: strided ones are made here
            for k in ("k", "v", "q"):
                if s.get("strided") and s[k] is not None:
                    s[k] = s[k].transpose(1, 2).contiguous().transpose(1, 2)
            p = pages._replace(**{k: s[k] for k in ("K", "V", "K_exp", "V_exp") if k in s})
            bif.bifattn_paged_append(plan, p, s["tab"], s["lens"], s["k"], s["v"], s["lens_out"], q=s["q"], q_out=s["q_out"],
                                     counts=s["counts"], freqs=s["freqs"], neighbours=s.get("neighbours", False),
                                     context=s.get("context", False), stream=s.get("stream"))

        forms = {"valid": {}, "strided": dict(strided=True), "neighbours": dict(neighbours=True), "truthy": dict(neighbours=1),
                 "no q": dict(q=None, q_out=None), "q alone": dict(q_out=None), "no freqs": dict(freqs=None),
                 "odd freqs": dict(freqs=torch.rand(3, device="cuda")), "many freqs": dict(freqs=torch.rand(90, device="cuda")),
                 "double freqs": dict(freqs=torch.rand(16, device="cuda").double()), "no counts": dict(counts=None),
                 "long counts": dict(counts=new["counts"].long()), "wrong groups": dict(v=new["v"][:, :1]),
                 "wrong rank": dict(k=new["k"][0]), "wrong type": dict(v=new["v"].float()), "host": dict(k=new["k"].cpu()),
                 "context of three": dict(context=True), "other rows": dict(q=new["q"][:, :, :2]), "none": dict(lens=None),
                 "on a stream": dict(stream=torch.cuda.Stream()), "misaligned": dict(q_out=None, q=None, k=misaligned(new["k"]))}
        for name, change in forms.items():
            print(f"[case] append {kv} {name}", flush=True)
            torch.cuda.synchronize()
            same(both_ways(plan, append, lambda: dict(new, **change)), name)

        out = dict(ko=torch.zeros(3, 2, 6, 64, dtype=torch.bfloat16, device="cuda"),
                   vo=torch.zeros(3, 2, 6, 64, dtype=torch.bfloat16, device="cuda"), tab=fixed["tab"], lens=fixed["lens"],
                   first=torch.tensor([1, 0, 4], dtype=torch.int32, device="cuda"))

        def gather(plan, s):
            bif.bifattn_paged_gather(plan, pages, s["tab"], s["lens"], s["ko"], s["vo"], first=s["first"],
                                     context=s.get("context", False))

        forms = {"valid": {}, "from 0": dict(first=None), "context": dict(context=True), "other shapes": dict(vo=out["vo"][:, :, :5]),
                 "fp32": dict(ko=out["ko"].float()), "none": dict(vo=None), "long": dict(first=out["first"].long())}
        for name, change in forms.items():
            print(f"[case] gather {kv} {name}", flush=True)
            same(both_ways(plan, gather, lambda: dict(out, **change)), name)
