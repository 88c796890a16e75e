"""Verification of drafted tokens against a plain implementation in whole numbers."""
import math

import numpy as np
import pytest
import torch

import serving_ref as ref
from paper_2606_03026_gb300 import spikeproj as sp

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def make(seed, B, T, V, sharp=2.0, noise=0.6):
    r = np.random.default_rng(seed)

    def soft(z):
        e = np.exp(z - z.max(-1, keepdims=True))
        return (e / e.sum(-1, keepdims=True)).astype(np.float32)

    z = sharp * r.standard_normal((B, T + 1, V))
    p, q = soft(z), soft(z[:, :T] + noise * r.standard_normal((B, T, V)))
    draft = np.array([[r.choice(V, p=q[b, t] / q[b, t].astype(np.float64).sum()) for t in range(T)] for b in range(B)],
                     dtype=np.int32).reshape(B, T)
    return p, q, draft, r.random((B, T), dtype=np.float32), r.random(B, dtype=np.float32)


def run(p, q, draft, u, us, n_draft=None, pad=0):
    def gpu(x):
        x = torch.from_numpy(np.ascontiguousarray(x)).to(DEV)
        if not pad or x.dim() < 2:
            return x
        wide = torch.full((*x.shape[:-1], x.shape[-1] + 2 * pad), 77, dtype=x.dtype, device=DEV)
        wide[..., pad:pad + x.shape[-1]] = x
        return wide[..., pad:pad + x.shape[-1]]

    B, T = draft.shape
    n = torch.full((B,), -9, dtype=torch.int32, device=DEV)
    tokens = torch.full((B, T + 1), -9, dtype=torch.int32, device=DEV)
    sp.verify(gpu(p), gpu(q) if T else None, gpu(draft) if T else None, gpu(u) if T else None, gpu(us), n, tokens,
              None if n_draft is None else gpu(np.array(n_draft, dtype=np.int32)))
    torch.cuda.synchronize()
    return n.cpu().numpy(), tokens.cpu().numpy()


def check(p, q, draft, u, us, n_draft=None, pad=0):
    n, tokens = run(p, q, draft, u, us, n_draft, pad)
    B, T = draft.shape
    for b in range(B):
        nd = T if n_draft is None else min(max(n_draft[b], 0), T)
        wn, wt = ref.verify(p[b], q[b] if T else None, draft[b], u[b], us[b], nd)
        assert (int(n[b]), tokens[b].tolist()) == (wn, wt), b
    return n, tokens


@pytest.mark.parametrize("B,T,V", [(1, 1, 1), (1, 4, 2), (3, 0, 100), (2, 3, 31), (5, 4, 1000), (2, 7, 4099),
                                   (1, 2, 50001), (400, 2, 65), (30, 5, 9000), (2, 64, 50)])
def test_verify_matches_the_definition(B, T, V):
    check(*make(B + T + V, B, T, V))


def test_verify_ragged_drafts_and_strides():
    x = make(5, 6, 4, 777)
    check(*x, n_draft=[0, 1, 2, 3, 4, 9])
    check(*x, n_draft=[-3, 4, 4, 0, 2, 4], pad=3)
    check(*x, pad=4)


def test_verify_kept_and_refused_drafts_both_occur():
    n, _ = check(*make(6, 200, 4, 300))
    assert len(set(n.tolist())) == 5


def test_verify_random_numbers_at_their_ends():
    p, q, draft, u, us = make(7, 8, 2, 500)
    u[:] = np.array([0, 1 - 2.0 ** -24, 1, 2, -1, math.nan, math.inf, 0.5], dtype=np.float32)[:, None]
    us[:] = np.array([0, 1 - 2.0 ** -24, 1, 2, -1, math.nan, -math.inf, 0.5], dtype=np.float32)
    check(p, q, draft, u, us)


def test_verify_tokens_outside_the_vocabulary_are_refused():
    p, q, draft, u, us = make(8, 4, 3, 300)
    draft[0, 0], draft[1, 1], draft[2, 0], draft[3, 2] = -1, 300, 2 ** 31 - 1, -2 ** 31
    u[:] = 0
    n, _ = check(p, q, draft, u, us)
    assert n.tolist() == [0, 1, 0, 2]


def test_verify_equal_distributions_and_degenerate_rows():
    p, q, draft, u, us = make(9, 6, 1, 2000)
    q[0] = p[0, :1]                       # p = q, and refused: drawn from p
    p[0, 0, draft[0, 0]] = q[0, 0, draft[0, 0]]
    u[0] = 1
    p[1] = 0                              # nothing anywhere
    p[2, 0] = 0
    p[2, 0, 1999] = 1                     # the last token alone
    p[3, 0] = 0
    p[3, 0, 0] = 1                        # the first
    p[4, 0, 5] = math.nan
    p[4, 0, 6] = math.inf                 # taken as 1
    p[5, 0] = 2.0 ** -37                  # half of the unit: rounds to even, 0
    u[1:] = 1
    n, tokens = check(p, q, draft, u, us)
    assert tokens[1].tolist() == [-1, -1]


def test_verify_whole_sums_in_any_split():
    # a flat row, every weight 2^36 / V: the token is floor(u V) whatever the split
    for V in (4096, 65536):
        p = np.full((3, 1, V), 1.0 / V, dtype=np.float32)
        us = np.array([0.25, 0.5 - 2.0 ** -24, 0.75], dtype=np.float32)
        n, tokens = run(p, np.zeros((3, 0, V), np.float32), np.zeros((3, 0), np.int32), np.zeros((3, 0), np.float32), us)
        assert tokens[:, 0].tolist() == [V // 4, V // 2 - 1, 3 * V // 4]


def test_verify_keeps_the_target_distribution():
    """Drafted and corrected tokens follow p: a chi-square over 20000 sequences (15 degrees of freedom, 1e-6 tail 57)."""
    V, B = 16, 20000
    r = np.random.default_rng(10)
    p1, q1 = r.dirichlet(np.ones(V)), r.dirichlet(np.ones(V))
    p = np.broadcast_to(p1.astype(np.float32), (B, 2, V))
    q = np.broadcast_to(q1.astype(np.float32), (B, 1, V))
    draft = r.choice(V, size=(B, 1), p=q1).astype(np.int32)
    n, tokens = run(p, q, draft, r.random((B, 1), dtype=np.float32), r.random(B, dtype=np.float32))
    seen = np.bincount(tokens[:, 0], minlength=V)
    assert ((seen - B * p1) ** 2 / (B * p1)).sum() < 57


def test_verify_refusals():
    p, q, draft, u, us = (torch.from_numpy(x).to(DEV) for x in make(11, 2, 2, 50))
    n = torch.zeros(2, dtype=torch.int32, device=DEV)
    tokens = torch.zeros(2, 3, dtype=torch.int32, device=DEV)

    def status(**change):
        call = sp.SpVerify(p.data_ptr(), 150, 50, q.data_ptr(), 100, 50, draft.data_ptr(), 2, None, u.data_ptr(), 2,
                           us.data_ptr(), n.data_ptr(), tokens.data_ptr(), 3, 2, 2, 50)
        for k, v in change.items():
            setattr(call, k, v)
        with pytest.raises(sp.SpikeProjError) as e:
            sp.spike_proj_verify(call)
        return e.value.status

    for name in ("p", "q", "draft", "u", "u_sample", "n_accept", "tokens"):
        assert status(**{name: None}) == sp.SP_EINVAL, name
        assert status(**{name: (1 << 20) + 2}) == sp.SP_EALIGN, name
    for change in ({"T": -1}, {"T": 65}, {"V": 0}, {"V": (1 << 24) + 1}, {"B": 0}, {"B": 65536}):
        assert status(**change) == sp.SP_ERANGE, change
    for change in ({"ld_draft": 1}, {"ld_u": 1}, {"ld_tokens": 2}):
        assert status(**change) == sp.SP_EINVAL, change
    with pytest.raises(ValueError):
        sp.verify(p, q[:, :1], draft, u, us, n, tokens)
    with pytest.raises(ValueError):
        sp.verify(p, q, draft.long(), u, us, n, tokens)
    torch.cuda.synchronize()
