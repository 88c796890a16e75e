"""Attention, eviction and verification where sums vanish, offsets are long and
rows are wide."""
import pytest
import torch

from paper_2606_03026_gb300 import spikeproj as sp

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


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
