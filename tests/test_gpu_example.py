"""The drafted decoding example: its calls in the order in which a user makes
them, each checked against the plain implementation on what it was given."""
import importlib.util
from pathlib import Path

import numpy as np
import pytest
import torch

import serving_ref as ref
from paper_2606_03026_gb300 import spikeproj as sp

pytestmark = pytest.mark.gpu


def load():
    path = Path(__file__).resolve().parent.parent / "examples" / "drafted_decode.py"
    spec = importlib.util.spec_from_file_location("drafted_decode", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def test_drafted_decoding(monkeypatch):
    d = load().DraftedDecoder(batch=3, prompt=70, drafts=2, vocab=160, width=64, Hq=4, Hkv=2, D=64, capacity=14, budget=9,
                              recent=4)
    calls = []
    attend, evict, verify = d.cache.attend, d.cache.evict, sp.verify

    def cpu(*tensors):
        return [x.cpu().clone() for x in tensors]

    def checked_attend(q, k, v, lens, out, pk, pv, weights):
        before = weights.cpu().clone()
        attend(q, k, v, lens, out, pk, pv, weights)
        calls.append("attend")
        want, _, ww, mass, size = ref.attend(*cpu(q, k, v, lens, pk, pv))
        top = float(torch.cat([v.flatten(), pv.flatten()]).abs().max())
        tol, _, w_rel = ref.attend_bounds(q.dtype, 64, 70 + 14, mass, size, want, top)
        assert ((out.cpu().double() - want).abs() <= tol).all()
        gain = weights.cpu().double() - before
        assert ((gain - ww).abs() <= ww * (w_rel.max() + 2.0 ** -20) + 2.0 ** -23 * (ww + before)).all()

    def checked_evict(k, v, weights, pos, lens, now, budget, recent, weights_out, pos_out, lens_out):
        bk, bw, bp, bl, bn = cpu(k, weights, pos, lens, now)
        evict(k, v, weights, pos, lens, now, budget, recent, weights_out, pos_out, lens_out)
        calls.append("evict")
        for b in range(3):
            for h in range(2):
                src = ref.evict(bw[b, h], bp[b, h], int(bl[b]), bn[b], budget, recent)
                assert torch.equal(k[b, :len(src), h].cpu(), bk[b, src, h])
                assert torch.equal(pos_out[b, h, :len(src)].cpu(), bp[b, h, src])
                assert int(lens_out[b]) == len(src)

    def checked_verify(p, q, draft, u, u_sample, kept, tokens):
        verify(p, q, draft, u, u_sample, kept, tokens)
        calls.append("verify" if q is not None else "draw")
        none = np.zeros((3, 0), np.float32)
        P, U, K, X = (x.cpu().numpy() for x in (p, u_sample, kept, tokens))
        Q, R, A = (none if x is None else x.cpu().numpy() for x in (q, draft, u))
        for b in range(3):
            n, want = ref.verify(P[b], Q[b], R[b], A[b], U[b], P.shape[1] - 1)
            assert K[b] == n and X[b].tolist() == want

    monkeypatch.setattr(d.cache, "attend", checked_attend)
    monkeypatch.setattr(d.cache, "evict", checked_evict)
    monkeypatch.setattr(sp, "verify", checked_verify)
    for _ in range(8):
        tokens = d.step()
        made = (tokens >= 0).sum(1)
        assert (made >= 1).all() and (tokens < 160).all()
        assert torch.equal(d.last, tokens.gather(1, made.unsqueeze(1) - 1)[:, 0])
        lens, now = d.lens.tolist(), d.now.tolist()
        assert all(1 <= n <= 14 and n <= t for n, t in zip(lens, now))
        # every entry in use is of a token of its own
        for b in range(3):
            for h in range(2):
                pos = d.pos[b, h, :lens[b]].tolist()
                assert len(set(pos)) == lens[b] and max(pos) == now[b] - 1
    assert calls.count("evict") >= 2 and calls.count("attend") == 8
    assert calls.count("verify") == 8 and calls.count("draw") == 16
    d.close()
