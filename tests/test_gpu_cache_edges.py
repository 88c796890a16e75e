"""Attention, eviction and verification where sums vanish, offsets are long and
rows are wide."""
import itertools
import math

import pytest
import torch

from paper_2606_03026_gb300 import spikeproj as sp

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("B,G,P", [(1, 1, 40000), (40, 60, 700), (3, 3, 700)], ids=["long", "rows", "few"])
@pytest.mark.parametrize("score", [0.0, -math.inf], ids=["vanishing", "zero"])
def test_a_value_that_is_nan_stays_where_its_weight_vanishes(dtype, B, G, P, score):
    """One prefix value is NaN; its weight beside the last entry's, 128 nats above,
    is nothing in 32 bits, or it has none at all.  Its column of every row that
    sees it is NaN all the same, however the entries are cut up."""
    D, C = 64, 70
    q = torch.ones(B, 1, G, D, dtype=dtype, device=DEV)
    pk, pv = torch.full((P, 1, D), score, dtype=dtype, device=DEV), torch.ones(P, 1, D, dtype=dtype, device=DEV)
    pk[-1] = 16.0
    pk[64:] = pk[64:].nan_to_num(neginf=0.0)                 # only the first tile's are without weight
    k, v = torch.zeros(B, C, 1, D, dtype=dtype, device=DEV), torch.ones(B, C, 1, D, dtype=dtype, device=DEV)
    lens = torch.full((B,), C, dtype=torch.int32, device=DEV)
    cache = sp.Cache(B, G, 1, D, C, dtype="bf16" if dtype == torch.bfloat16 else "fp16")
    out = torch.zeros_like(q)
    cache.attend(q, k, v, lens, out, pk, pv)
    assert (out == 1).all()
    pv[5, 0, 7] = math.nan
    cache.attend(q, k, v, lens, out, pk, pv)
    assert out[..., 7].isnan().all() and (out[..., :7] == 1).all() and (out[..., 8:] == 1).all()
    # the same in an own cache
    pv[5, 0, 7] = 1.0
    k[0, 0], v[0, 0, 0, 3] = score, math.nan
    cache.attend(q, k, v, lens, out, pk, pv)
    assert out[0, ..., 3].isnan().all() and (out[0, ..., :3] == 1).all() and (out[0, ..., 4:] == 1).all()
    assert (out[1:] == 1).all()
    assert cache.status() == sp.SP_OK
    cache.close()


@pytest.mark.parametrize("B,T,V", [(1, 4, 57344), (40, 4, 57344), (400, 7, 999), (3, 64, 5000)])
def test_a_verification_in_the_place_of_its_drafts(B, T, V):
    """n_accept in n_draft's buffer, tokens in that of the drafts, whose CTAs all read them."""
    g = torch.Generator(device=DEV).manual_seed(B)
    z = 2 * torch.randn(B, T + 1, V, generator=g, device=DEV)
    p = torch.softmax(z, 2)
    q = torch.softmax(z[:, :T] + 0.6 * torch.randn(B, T, V, generator=g, device=DEV), 2)
    draft = torch.multinomial(q.view(-1, V), 1, generator=g).view(B, T).to(torch.int32)
    u, us = torch.rand(B, T, generator=g, device=DEV), torch.rand(B, generator=g, device=DEV)
    count = torch.randint(0, T + 1, (B,), generator=g, device=DEV, dtype=torch.int32)
    n, tokens = torch.empty_like(count), torch.empty(B, T + 1, dtype=torch.int32, device=DEV)
    sp.verify(p, q, draft, u, us, n, tokens, n_draft=count)
    for _ in range(20):
        both, row = count.clone(), torch.cat([draft, draft[:, :1]], 1)
        sp.verify(p, q, row[:, :T], u, us, both, row, n_draft=both)
        assert torch.equal(both, n) and torch.equal(row, tokens)


@pytest.mark.parametrize("V", [1, 2, 3, 4, 5, 6, 7, 9, 66, 511, 512, 514, 1025, 4097, 30002])
def test_a_verification_of_rows_that_begin_anywhere(V):
    """p and q off 16 bytes by 0 to 12, all of the residual at either end of the
    row; what lies beside the rows would be drawn if it were read."""
    for shift_p, shift_q, end in itertools.product(range(4), range(4), (0, 1)):
        some = min(V, 3)
        at = torch.arange(some) if end == 0 else torch.arange(V - some, V)
        p, q = (torch.full((V + 8,), math.inf, device=DEV) for _ in range(2))
        p, q = p[shift_p:shift_p + V], q[shift_q:shift_q + V]
        p.zero_(), q.zero_()
        p[at.to(DEV)] = 0.5
        q[at[0]] = 0.5                       # (its residual is 0)
        first, second = (at[1], at[-1]) if some > 1 else (at[0], at[0])
        for u, want in ((0.0, first), (0.999, second)):
            n, token = torch.zeros(1, dtype=torch.int32, device=DEV), torch.zeros(1, 2, dtype=torch.int32, device=DEV)
            sp.verify(p.expand(1, 2, V), q.view(1, 1, V), torch.full((1, 1), -1, dtype=torch.int32, device=DEV),
                      torch.zeros(1, 1, device=DEV), torch.tensor([u], device=DEV), n, token)
            assert token.tolist() == [[int(want), -1]] and int(n) == 0, (shift_p, shift_q, end, u)


@pytest.mark.parametrize("B,Hkv,C,budget", [(16, 8, 12000, 3000), (3, 2, 300, 250), (64, 4, 2056, 2048)])
def test_calls_back_to_back_see_each_others_results(B, Hkv, C, budget):
    """attend, evict, attend, evict, .. on two sets of buffers in turn, each launched
    while the one before may still run: as with the device waited for in between."""
    D, T = 64, 2

    def run(wait):
        g = torch.Generator(device=DEV).manual_seed(6)
        k, v = (torch.randn(B, C, Hkv, D, generator=g, device=DEV).bfloat16() for _ in range(2))
        q = torch.randn(B, T, 2 * Hkv, D, generator=g, device=DEV).bfloat16()
        pk, pv = (torch.randn(100, Hkv, D, generator=g, device=DEV).bfloat16() for _ in range(2))
        lens = torch.zeros(2, B, dtype=torch.int32, device=DEV)             # (both in one sector for few sequences)
        lens[0] = torch.randint(C // 2, C + 1, (B,), generator=g, device=DEV)
        now, w = lens[0].clone(), torch.zeros(2, B, Hkv, C, device=DEV)
        pos = torch.arange(C, dtype=torch.int32, device=DEV).expand(2, B, Hkv, C).contiguous()
        outs = [torch.zeros_like(q) for _ in range(6)]
        torch.cuda.synchronize()
        for i in range(6):
            a, b = i % 2, 1 - i % 2
            cache.attend(q, k, v, lens[a], outs[i], pk, pv, w[a])
            if wait:
                torch.cuda.synchronize()
            cache.evict(k, v, w[a], pos[a], lens[a], now, budget - 10 * i, 16, w[b], pos[b], lens[b])
            if wait:
                torch.cuda.synchronize()
        torch.cuda.synchronize()
        return [*outs, k, v, w, pos, lens]

    cache = sp.Cache(B, 2 * Hkv, Hkv, D, C, max_T=T, weights=True)
    want = run(True)
    for _ in range(10):
        for x, y in zip(run(False), want):
            assert torch.equal(x, y)
    assert cache.status() == sp.SP_OK
    cache.close()
