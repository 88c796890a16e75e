"""Waits of the 4-bit cache's attention that run out, after calls of other kinds on the
same handle."""
import pytest
import torch

from paper_2606_03026_gb300 import spikeproj as sp
from test_gpu_cache4 import check, make

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("B,Hq,Hkv,D,C,T,before", [
    (12, 64, 8, 128, 6000, 8, (1, 8)),       # 64 rows after units of 8 that all warps have parts of
    (1, 16, 4, 128, 60000, 5, (1, 2, 4)),
    (3, 34, 2, 64, 9000, 6, (1,)),           # two units of 51 rows after some of 17
    (9, 16, 2, 96, 3000, 4, (2, 1)),
], ids=str)
def test_a_wait_runs_out_after_calls_of_other_lengths(B, Hq, Hkv, D, C, T, before):
    """Where the rows' kernel gives up, its units' notes are those of the calls before,
    for other numbers of tokens, workers and rows: they are not taken further than the
    workspace, the status says what happened, and the next call is right."""
    lens = [C - 97 * b for b in range(B)]
    q, k4, v4, lens = make(51, B, T, Hq, Hkv, D, C, lens, "bf16", garbage=False)
    on = tuple(x.to(DEV) for x in k4), tuple(x.to(DEV) for x in v4), lens.to(DEV)
    cache = sp.Cache4(Hq, Hkv, D, C, max_T=T)

    def attend(t):
        out, lse = torch.zeros(B, t, Hq, D, dtype=torch.bfloat16, device=DEV), torch.zeros(B, t, Hq, device=DEV)
        cache.attend(q[:, T - t:].to(DEV), *on, out, lse=lse)
        return out, lse

    for t in before:
        attend(t)
        cache.inject_fault(sp.SP_FAULT_STALL)
        attend(T)
        assert cache.status() == sp.SP_EKERNEL and cache.status() == sp.SP_OK
    out, lse = attend(T)
    assert cache.status() == sp.SP_OK
    check(q, k4, v4, lens, (out.cpu(), lse.cpu()))
    cache.close()
