"""An attend call whose waits run out (copies that are never issued, waits of
about 2 ms): the status says so once, whatever the workspace held, and the
next call of the handle is right."""
import time

import pytest
import torch

from paper_2606_03026_gb300 import spikeproj as sp

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("B,T,Hq,Hkv,P,C", [(2, 1, 4, 2, 9000, 300), (24, 6, 24, 2, 700, 200), (40, 3, 33, 11, 700, 260),
                                            (3, 2, 4, 2, 0, 400)], ids=["few-rows", "more", "many-rows", "no-prefix"])
def test_waits_that_run_out(B, T, Hq, Hkv, P, C, D, dtype):
    g = torch.Generator(device=DEV).manual_seed(B)

    def normal(*shape):
        return torch.randn(shape, generator=g, device=DEV).to(dtype)

    q, k, v = normal(B, T, Hq, D), normal(B, C, Hkv, D), normal(B, C, Hkv, D)
    pk, pv = (normal(P, Hkv, D), normal(P, Hkv, D)) if P else (None, None)
    lens = torch.randint(T, C + 1, (B,), generator=g, device=DEV, dtype=torch.int32)
    cache = sp.Cache(B, Hq, Hkv, D, C, max_T=T, weights=True, dtype="bf16" if dtype == torch.bfloat16 else "fp16")

    def attend(b=B):
        out, w, lse = torch.zeros_like(q[:b]), torch.zeros(b, Hkv, C, device=DEV), torch.zeros(b, T, Hq, device=DEV)
        cache.attend(q[:b], k[:b], v[:b], lens[:b], out, pk, pv, w, lse)
        return out, w, lse

    def stalled(b=B):
        cache.inject_fault(sp.SP_FAULT_STALL)
        torch.cuda.synchronize()
        start = time.perf_counter()
        attend(b)
        torch.cuda.synchronize()
        assert time.perf_counter() - start < 1.0
        assert cache.status() == sp.SP_EKERNEL and cache.status() == sp.SP_OK

    stalled()                               # nothing has written the workspace
    want = attend()
    assert cache.status() == sp.SP_OK and want[0].isfinite().all()
    stalled(1)                              # units numbered otherwise than the last call's
    stalled()
    for _ in range(2):
        for x, y in zip(attend(), want):
            assert torch.equal(x, y)
    assert cache.status() == sp.SP_OK
    cache.close()
