"""Tensors and workspaces whose last elements lie more than 2^31 from their
first, in every dimension, and rows of several pieces per group."""
import pytest
import torch

from paper_2606_03026_gb300 import spikeproj as sp
from test_gpu_cache import check, check_evict, evict_case, make

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def far(x, dim):
    """The values of x on the GPU with dimension `dim` (or the last but one) so
    far apart that its last index lies past 2^31 elements."""
    dim = max(0, min(dim, x.dim() - 2))
    while x.shape[dim] == 1:
        dim -= 1
    rest = [i for i in range(x.dim()) if i != dim]
    stride, n = [0] * x.dim(), 1
    for i in reversed(rest):
        stride[i], n = n, n * x.shape[i]
    stride[dim] = (max(n, 2 ** 31 // (x.shape[dim] - 1)) // 8 + 2) * 8
    last = sum((a - 1) * b for a, b in zip(x.shape, stride))
    assert (x.shape[dim] - 1) * stride[dim] > 2 ** 31
    y = torch.empty(last + 1, dtype=x.dtype, device=DEV).as_strided(x.shape, stride)
    y.copy_(x)
    return y


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("dim", [0, 1, 2], ids=["sequences", "entries", "heads"])
def test_attend_past_32_bits(dim, D):
    x = make(51, 2, 3, 4, 2, D, 40, 150, [5, 150], "bf16")
    q, pk, pv, k, v, lens = x
    cache = sp.Cache(2, 4, 2, D, 150, max_T=3, weights=True)
    out, w = far(torch.zeros_like(q), dim), far(torch.full((2, 2, 150), 0.25), dim)
    lse = torch.zeros(2, 3, 4, device=DEV)
    cache.attend(far(q, dim), far(k, dim), far(v, dim), lens.to(DEV), out, far(pk, dim - 1), far(pv, dim - 1), w, lse)
    torch.cuda.synchronize()
    assert cache.status() == sp.SP_OK
    check(*x, (out.cpu(), lse.cpu(), w.cpu()))
    cache.close()


@pytest.mark.parametrize("dim", [0, 1, 2], ids=["sequences", "entries", "heads"])
def test_evict_past_32_bits(dim):
    x = evict_case(52, 2, 2, 64, 90, [90, 70], 50, 9, "spread")
    k, v, w, pos, lens, now = x
    cache = sp.Cache(2, 2, 2, 64, 90)
    gk, gv, lo = far(k, dim), far(v, dim), torch.zeros(2, dtype=torch.int32, device=DEV)
    wo, po = far(torch.full((2, 2, 50), 7.0), dim), far(torch.full((2, 2, 50), 7, dtype=torch.int32), dim)
    cache.evict(gk, gv, far(w, dim), far(pos, dim), lens.to(DEV), now.to(DEV), 50, 9, wo, po, lo)
    torch.cuda.synchronize()
    check_evict(x, 50, 9, (gk.cpu(), gv.cpu(), wo.cpu(), po.cpu(), lo.cpu()))
    cache.close()


def test_scores_past_32_bits():
    """8.9 GB of scores: 2^20 entries that 1056 query rows see, all alike."""
    T, G, C = 32, 33, 1 << 20
    q = torch.ones(2, T, G, 64, dtype=torch.bfloat16, device=DEV)
    k, v = torch.zeros(2, C, 1, 64, dtype=torch.bfloat16, device=DEV), torch.ones(2, C, 1, 64, dtype=torch.bfloat16, device=DEV)
    assert 2 * C * T * G > 2 ** 31
    cache = sp.Cache(2, G, 1, 64, C, max_T=T, weights=True)
    out, w, lse = torch.zeros_like(q), torch.zeros(2, 1, C, device=DEV), torch.zeros(2, T, G, device=DEV)
    cache.attend(q, k, v, torch.tensor([3, C], dtype=torch.int32, device=DEV), out, weights=w, lse=lse)
    torch.cuda.synchronize()
    assert cache.status() == sp.SP_OK
    seen = torch.arange(C - T + 1, C + 1, dtype=torch.float64, device=DEV)        # by each query token
    assert (out[1] == 1).all() and ((lse[1].double() - seen.log().view(T, 1)).abs() <= 2.0 ** -18).all()
    # a row's share of an entry is 1 / seen; what the last entries get of the later rows alone
    all_rows = G * (1 / seen).sum()
    late = G * (1 / seen).flip(0).cumsum(0).flip(0)
    want = torch.cat([all_rows.expand(C - T), late])
    # a term is off by the rounding of its exponent, near 2^-18, their sum by as many roundings
    assert ((w[1, 0].double() - want).abs() <= want * (2.0 ** -18 + (T * G + 8) * 2.0 ** -24)).all()
    assert (w[0, 0, 3:] == 0).all()
    cache.close()


# ---------------------------------------------------------------------------
def drafted(B, T, V, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    z = 2 * torch.randn(B, T + 1, V, generator=g, device=DEV)
    p = torch.softmax(z, 2)
    q = torch.softmax(z[:, :T] + 0.6 * torch.randn(B, T, V, generator=g, device=DEV), 2)
    draft = torch.randint(0, V, (B, T), generator=g, device=DEV, dtype=torch.int32)
    return p, q, draft, torch.rand(B, T, generator=g, device=DEV)


def first_past(r, u):
    """The token of the residual r (float32 [V]) at u, by whole sums."""
    w = torch.round(r.double().clamp(0, 1) * 2.0 ** 36).long()
    return int(torch.searchsorted(w.cumsum(0), int(u * 2 ** 24) * int(w.sum()) // 2 ** 24, right=True))


@pytest.mark.parametrize("dim", [0, 1])
def test_verify_past_32_bits(dim):
    p, q, draft, u = drafted(2, 3, 5000, 53)
    us = torch.tensor([0.3, 0.8], device=DEV)
    n, tokens = torch.zeros(2, dtype=torch.int32, device=DEV), torch.zeros(2, 4, dtype=torch.int32, device=DEV)
    sp.verify(p, q, draft, u, us, n, tokens)
    far_n, far_tokens = torch.zeros_like(n), far(torch.zeros_like(tokens), 0)
    sp.verify(far(p, dim), far(q, dim), far(draft, 0), far(u, 0), us, far_n, far_tokens)
    assert torch.equal(far_n, n) and torch.equal(far_tokens, tokens) and (tokens[:, 0] >= 0).all()


@pytest.mark.parametrize("B,T,V", [(1, 1, 1 << 24), (1, 0, (1 << 24) - 1), (160, 1, 300001), (160, 0, 1 << 20)])
def test_verify_rows_of_several_pieces_per_group(B, T, V):
    """A group is several pieces above 2^18 entries a CTA: tokens in the first,
    middle and last groups of all warps, and at both ends."""
    p, q, draft, u = drafted(B, T, V, 54)
    u.fill_(1.0)                            # no draft is kept
    if T:
        p[:, 0].scatter_(1, draft.long(), 0.0)
    grid = torch.tensor([0.0, 1 - 2.0 ** -24, *[(i + 0.5) / 29 for i in range(29)]], device=DEV)
    for at in range(0, len(grid), B):
        us = grid[at:at + B].repeat(B)[:B].contiguous()
        n, tokens = torch.zeros(B, dtype=torch.int32, device=DEV), torch.zeros(B, T + 1, dtype=torch.int32, device=DEV)
        sp.verify(p, q if T else None, draft if T else None, u if T else None, us, n, tokens)
        assert not n.any()
        for b in range(min(B, 40)):
            assert int(tokens[b, 0]) == first_past(p[b, 0] - q[b, 0] if T else p[b, 0], float(us[b])), (b, float(us[b]))
