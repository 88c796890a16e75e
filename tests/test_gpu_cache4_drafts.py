"""Drafted decode steps on a 4-bit cache: written, attended to behind a shared prompt,
verified, and those that were not kept written over."""
import pytest
import torch

import cache4_ref as ref
from paper_2606_03026_gb300 import spikeproj as sp

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("B,n,Hq,Hkv,D,C,dtype", [(3, 2, 8, 2, 64, 60, "bf16"), (5, 4, 24, 4, 128, 900, "fp16")],
                         ids=["one-launch", "many-rows"])
def test_drafts_are_written_verified_and_written_over(B, n, Hq, Hkv, D, C, dtype):
    P, V, T = 150, 300, n + 1
    t = torch.bfloat16 if dtype == "bf16" else torch.float16
    g = torch.Generator(device=DEV).manual_seed(81)
    new = lambda *s: torch.randn(*s, generator=g, device=DEV).to(t)          # noqa: E731
    uniform = lambda *s: torch.rand(s, generator=g, device=DEV)              # noqa: E731
    pk, pv, head = new(P, Hkv, D), new(P, Hkv, D), torch.randn(Hq * D, V, generator=g, device=DEV) * 0.1
    prefix, cache = sp.Cache(B, Hq, Hkv, D, 1, max_T=T, dtype=dtype), sp.Cache4(Hq, Hkv, D, C, max_T=T, dtype=dtype)
    none, unused = torch.zeros(B, dtype=torch.int32, device=DEV), new(B, 1, Hkv, D)
    k4, v4 = cache.new(B)
    lens = torch.tensor([(7 * b) % 5 for b in range(B)], dtype=torch.int32, device=DEV)
    cache.write(new(B, 4, Hkv, D), new(B, 4, Hkv, D), k4, v4, n=lens)
    k, v = (ref.values(x[0].cpu(), x[1].cpu()) for x in (k4, v4))            # what the caches stand for
    kept_of_all = []
    for step in range(8):
        query, nk, nv = new(B, T, Hq, D), new(B, T, Hkv, D), new(B, T, Hkv, D)
        cache.write(nk, nv, k4, v4, at=lens)
        for b, at in enumerate(lens.tolist()):
            k[b, at:at + T], v[b, at:at + T] = (ref.quantise(x[b].cpu())[2] for x in (nk, nv))
        lens += T
        out, lse = torch.empty_like(query), torch.empty(B, T, Hq, device=DEV)
        prefix.attend(query, unused, unused, none, out, prefix_k=pk, prefix_v=pv, lse=lse)
        other = out.cpu(), lse.cpu()
        cache.attend(query, k4, v4, lens, out, lse=lse, other_out=out, other_lse=lse)
        want, wlse, tol, lse_tol = ref.attend(query.cpu(), k, v, lens.cpu(), other=other)
        assert ((out.cpu().double() - want).abs() <= tol).all() and ((lse.cpu().double() - wlse).abs() <= lse_tol).all()
        p = torch.softmax(out.flatten(2).float() @ head, -1)
        q = torch.softmax((p[:, :n] + 1e-6).log() + 0.3 * torch.randn(B, n, V, generator=g, device=DEV), -1).contiguous()
        draft = torch.multinomial(q.flatten(0, 1), 1, generator=g).view(B, n).int()
        kept, tokens = torch.empty(B, dtype=torch.int32, device=DEV), torch.empty(B, T, dtype=torch.int32, device=DEV)
        sp.verify(p, q, draft, uniform(B, n), uniform(B), kept, tokens)
        lens += kept - n                    # the last token and the kept drafts stay
        kept_of_all += kept.tolist()
    assert min(kept_of_all) < n and max(kept_of_all) > 0 and cache.status() == prefix.status() == sp.SP_OK
    for x, held in ((k, k4), (v, v4)):
        assert torch.equal(ref.values(held[0].cpu(), held[1].cpu()), x)      # (also what is not in use)
    cache.close()
    prefix.close()
