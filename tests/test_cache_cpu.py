"""The cache and verification operators without a GPU: what their entry points
refuse, their launches on fake devices, and the plain implementations that the
GPU tests compare with, pinned by hand and by laws."""
import ctypes
import itertools
import math

import numpy as np
import pytest
import torch

import serving_ref as ref
from paper_2606_03026_gb300 import spikeproj as sp
from test_host_cpu import FAKE, lib  # noqa: F401  (a fixture)

B, T, HQ, HKV, D, C, P = 2, 3, 8, 2, 64, 32, 100


def attend_call(**over):
    f = dict(q=FAKE, q_batch=T * HQ * D, q_token=HQ * D, q_head=D, prefix_k=FAKE, prefix_v=FAKE, pk_entry=HKV * D,
             pk_head=D, pv_entry=HKV * D, pv_head=D, k=FAKE, v=FAKE, k_batch=C * HKV * D, k_entry=HKV * D, k_head=D,
             v_batch=C * HKV * D, v_entry=HKV * D, v_head=D, lens=FAKE, out=FAKE, out_batch=T * HQ * D,
             out_token=HQ * D, out_head=D, lse=None, weights=None, weights_batch=HKV * C, weights_head=C, B=B, T=T,
             prefix_len=P, scale=0.125)
    return sp.SpAttend(**{**f, **over})


def evict_call(**over):
    f = dict(k=FAKE, v=FAKE, k_batch=C * HKV * D, k_entry=HKV * D, k_head=D, v_batch=C * HKV * D, v_entry=HKV * D,
             v_head=D, weights=FAKE, pos=FAKE, in_batch=HKV * C, in_head=C, weights_out=2 * FAKE, pos_out=2 * FAKE,
             out_batch=HKV * C, out_head=C, lens=FAKE, now=FAKE, lens_out=2 * FAKE, B=B, budget=16, recent=4)
    return sp.SpEvict(**{**f, **over})


def verify_call(**over):
    f = dict(p=FAKE, p_batch=4 * 100, p_row=100, q=FAKE, q_batch=3 * 100, q_row=100, draft=FAKE, ld_draft=3,
             n_draft=None, u=FAKE, ld_u=3, u_sample=FAKE, n_accept=FAKE, tokens=FAKE, ld_tokens=4, B=2, T=3, V=100)
    return sp.SpVerify(**{**f, **over})


def make(lib, max_batch=B, max_T=T, Hq=HQ, Hkv=HKV, D=D, capacity=C, dtype=0, flags=1):
    h = ctypes.c_void_p()
    st = lib.spike_proj_cache_create(ctypes.byref(h), max_batch, max_T, Hq, Hkv, D, capacity, dtype, flags, None)
    return h, st


@pytest.fixture
def cache(lib):                                                  # noqa: F811
    lib.fake_device(0)
    lib.fake_fail(b"")
    h, st = make(lib)
    assert st == sp.SP_OK
    yield h
    assert lib.spike_proj_cache_destroy(h) == sp.SP_OK


@pytest.mark.parametrize("over, want", [
    (dict(max_batch=0), sp.SP_ERANGE), (dict(max_batch=1025), sp.SP_ERANGE),
    (dict(max_T=0), sp.SP_ERANGE), (dict(max_T=33), sp.SP_ERANGE),
    (dict(Hq=0), sp.SP_ERANGE), (dict(Hq=514), sp.SP_ERANGE), (dict(Hq=7), sp.SP_EINVAL), (dict(Hkv=0), sp.SP_EINVAL),
    (dict(D=0), sp.SP_ERANGE), (dict(D=136), sp.SP_ERANGE), (dict(D=60), sp.SP_EALIGN),
    (dict(capacity=0), sp.SP_ERANGE), (dict(capacity=(1 << 24) + 1), sp.SP_ERANGE),
    (dict(dtype=2), sp.SP_EINVAL), (dict(flags=2), sp.SP_EINVAL),
], ids=str)
def test_a_cache_is_refused(lib, over, want):                    # noqa: F811
    h, st = make(lib, **over)
    assert st == want and not h.value
    # the library itself says so before it looks for a device
    assert make(sp.lib(), **over)[1] == want


@pytest.mark.parametrize("over, want", [
    *[({name: None}, sp.SP_EINVAL) for name in ("q", "k", "v", "lens", "out", "prefix_k", "prefix_v")],
    *[({name: FAKE + 8}, sp.SP_EALIGN) for name in ("q", "k", "v", "out", "prefix_k", "prefix_v")],
    *[({name: FAKE + 2}, sp.SP_EALIGN) for name in ("lens", "lse", "weights")],
    *[({name: 68}, sp.SP_EALIGN) for name in ("q_batch", "q_token", "q_head", "k_batch", "k_entry", "k_head", "v_batch",
                                              "v_entry", "v_head", "out_batch", "out_token", "out_head", "pk_entry",
                                              "pk_head", "pv_entry", "pv_head")],
    *[({name: 0}, sp.SP_EALIGN) for name in ("q_head", "k_batch", "v_head", "pk_head", "out_token")],
    (dict(q_token=-512), sp.SP_EALIGN), (dict(out_head=-32), sp.SP_EALIGN),
    (dict(B=0), sp.SP_EINVAL), (dict(T=0), sp.SP_EINVAL), (dict(prefix_len=-1), sp.SP_EINVAL),
    (dict(B=B + 1), sp.SP_ERANGE), (dict(T=T + 1), sp.SP_ERANGE), (dict(prefix_len=(1 << 24) + 1), sp.SP_ERANGE),
    *[(dict(scale=x), sp.SP_EINVAL) for x in (0.0, -1.0, math.inf, math.nan)],
], ids=str)
def test_an_attend_call_is_refused(lib, cache, over, want):      # noqa: F811
    lib.fake_launches()
    assert lib.spike_proj_cache_attend(cache, ctypes.byref(attend_call(**over)), None) == want
    assert lib.fake_launches() == 0


def test_attend_calls_at_the_limits(lib, cache):                 # noqa: F811
    ok = [dict(), dict(lse=FAKE, weights=FAKE), dict(prefix_len=0, prefix_k=None, prefix_v=None, pk_head=3),
          dict(B=1, q_batch=0, k_batch=5, out_batch=1), dict(T=1, q_token=0), dict(prefix_len=1, pk_entry=0),
          dict(out_head=-D, out_token=-HQ * D)]
    for over in ok:
        assert lib.spike_proj_cache_attend(cache, ctypes.byref(attend_call(**over)), None) == sp.SP_OK, over
    assert lib.spike_proj_cache_attend(None, ctypes.byref(attend_call()), None) == sp.SP_EINVAL
    assert lib.spike_proj_cache_attend(cache, None, None) == sp.SP_EINVAL
    assert lib.spike_proj_cache_status(cache, None) == sp.SP_OK
    assert lib.spike_proj_cache_status(None, None) == sp.SP_EINVAL
    plain, st = make(lib, flags=0)
    assert st == sp.SP_OK
    assert lib.spike_proj_cache_attend(plain, ctypes.byref(attend_call(weights=FAKE)), None) == sp.SP_EUNSUPPORTED
    assert lib.spike_proj_cache_destroy(plain) == sp.SP_OK
    assert lib.spike_proj_cache_destroy(None) == sp.SP_OK


def test_a_call_of_too_many_tiles_is_refused(lib):               # noqa: F811
    # the 128 query rows of each of 64 sequences and 128 K/V heads are a unit of
    # their own: 2^13 units, with the 2^12 tiles of 2^18 prefix entries 2^25
    h, st = make(lib, max_batch=64, max_T=32, Hq=512, Hkv=128, D=8, capacity=1, flags=0)
    assert st == sp.SP_OK
    wide = dict(q_batch=32 * 512 * 8, q_token=512 * 8, q_head=8, pk_entry=128 * 8, pk_head=8, pv_entry=128 * 8, pv_head=8,
                k_batch=1024, k_head=8, v_batch=1024, v_head=8, out_batch=32 * 512 * 8, out_token=512 * 8, out_head=8)
    for prefix, want in ((1 << 18, sp.SP_ERANGE), (1 << 17, sp.SP_OK)):
        call = attend_call(B=64, T=32, prefix_len=prefix, **wide)
        assert lib.spike_proj_cache_attend(h, ctypes.byref(call), None) == want
    assert lib.spike_proj_cache_destroy(h) == sp.SP_OK


@pytest.mark.parametrize("over, want", [
    *[({name: None}, sp.SP_EINVAL) for name in ("k", "v", "weights", "pos", "weights_out", "pos_out", "lens", "now",
                                                "lens_out")],
    (dict(weights_out=FAKE), sp.SP_EINVAL), (dict(pos_out=FAKE), sp.SP_EINVAL), (dict(lens_out=FAKE), sp.SP_EINVAL),
    *[({name: FAKE + 8}, sp.SP_EALIGN) for name in ("k", "v")],
    *[({name: 3 * FAKE + 1}, sp.SP_EALIGN) for name in ("weights", "pos", "weights_out", "pos_out", "lens", "now",
                                                       "lens_out")],
    *[({name: 68}, sp.SP_EALIGN) for name in ("k_batch", "k_entry", "k_head", "v_batch", "v_entry", "v_head")],
    (dict(k_entry=-128), sp.SP_EALIGN), (dict(B=0), sp.SP_EINVAL), (dict(B=B + 1), sp.SP_ERANGE),
    (dict(budget=-1, recent=0), sp.SP_EINVAL), (dict(recent=-1), sp.SP_EINVAL), (dict(recent=17), sp.SP_EINVAL),
], ids=str)
def test_an_evict_call_is_refused(lib, cache, over, want):       # noqa: F811
    lib.fake_launches()
    assert lib.spike_proj_cache_evict(cache, ctypes.byref(evict_call(**over)), None) == want
    assert lib.fake_launches() == 0


@pytest.mark.parametrize("over, want", [
    *[({name: None}, sp.SP_EINVAL) for name in ("p", "q", "draft", "u", "u_sample", "n_accept", "tokens")],
    *[({name: FAKE + 2}, sp.SP_EALIGN) for name in ("p", "q", "draft", "n_draft", "u", "u_sample", "n_accept", "tokens")],
    (dict(T=-1), sp.SP_ERANGE), (dict(T=65, ld_draft=65, ld_u=65, ld_tokens=66), sp.SP_ERANGE),
    (dict(V=0), sp.SP_ERANGE), (dict(V=(1 << 24) + 1), sp.SP_ERANGE), (dict(B=0), sp.SP_ERANGE),
    (dict(B=65536), sp.SP_ERANGE), (dict(ld_draft=2), sp.SP_EINVAL), (dict(ld_u=2), sp.SP_EINVAL),
    (dict(ld_tokens=3), sp.SP_EINVAL),
], ids=str)
def test_a_verify_call_is_refused(lib, over, want):              # noqa: F811
    lib.fake_launches()
    assert lib.spike_proj_verify(ctypes.byref(verify_call(**over)), None) == want
    assert lib.fake_launches() == 0
    assert sp.lib().spike_proj_verify(ctypes.byref(verify_call(**over)), None) == want
    assert lib.spike_proj_verify(None, None) == sp.SP_EINVAL


@pytest.mark.parametrize("first", [0, 1])
def test_every_launch_on_either_device(lib, first):              # noqa: F811
    """Head widths, types, few and many rows, few and many long caches, one
    and all sequences of a verification: each variant finds its attributes on
    the device that is current, and a handle serves its own device alone."""
    lib.fake_fail(b"")
    for dev in (first, 1 - first):
        lib.fake_device(dev)
        for d, dtype, (b, t) in itertools.product((8, 64, 72, 128), (0, 1), ((1, 1), (3, 5), (64, 8))):
            h, st = make(lib, max_batch=b, max_T=t, D=d, dtype=dtype)
            assert st == sp.SP_OK
            strides = dict(q_batch=t * HQ * d, q_token=HQ * d, q_head=d, pk_entry=HKV * d, pk_head=d, pv_entry=HKV * d,
                           pv_head=d, out_batch=t * HQ * d, out_token=HQ * d, out_head=d)
            kv = dict(k_batch=C * HKV * d, k_entry=HKV * d, k_head=d, v_batch=C * HKV * d, v_entry=HKV * d, v_head=d)
            lib.fake_launches()
            assert lib.spike_proj_cache_attend(h, ctypes.byref(attend_call(B=b, T=t, weights=FAKE, **strides, **kv)),
                                               None) == sp.SP_OK
            assert lib.fake_launches() == 3
            assert lib.spike_proj_cache_attend(h, ctypes.byref(attend_call(B=b, T=t, **strides, **kv)), None) == sp.SP_OK
            assert lib.fake_launches() == 2
            lib.fake_device(1 - dev)
            assert lib.spike_proj_cache_attend(h, ctypes.byref(attend_call(B=b, T=t, **strides, **kv)),
                                               None) == sp.SP_EDEVICE
            assert lib.spike_proj_cache_evict(h, ctypes.byref(evict_call(B=b, **kv)), None) == sp.SP_EDEVICE
            lib.fake_device(dev)
            assert lib.spike_proj_cache_destroy(h) == sp.SP_OK
        for heads, capacity, budget in itertools.product((1, 4, 20, 200), (1, 1000, 10000, 100000), (0, 60, 5000, 200000)):
            h, st = make(lib, max_batch=1, Hq=heads, Hkv=heads, D=8, capacity=capacity, flags=0)
            assert st == sp.SP_OK
            kv = dict(k_batch=8, k_entry=heads * 8, k_head=8, v_batch=8, v_entry=heads * 8, v_head=8)
            lib.fake_launches()
            assert lib.spike_proj_cache_evict(h, ctypes.byref(evict_call(B=1, budget=budget, recent=0, **kv)),
                                              None) == sp.SP_OK
            assert lib.fake_launches() == (2 if min(budget, capacity - budget) > 64 else 1)
            assert lib.spike_proj_cache_destroy(h) == sp.SP_OK
        for b, t, v in itertools.product((1, 20, 300, 65535), (0, 4, 64), (1, 1000, 57344, 1 << 24)):
            call = verify_call(B=b, T=t, V=v, ld_draft=t, ld_u=t, ld_tokens=t + 1)
            lib.fake_launches()
            assert lib.spike_proj_verify(ctypes.byref(call), None) == sp.SP_OK, (b, t, v)
            assert lib.fake_launches() == 1


@pytest.mark.parametrize("kernel", [b"attend_kernel", b"combine_kernel", b"weights_kernel", b"evict_kernel", b"move_kernel",
                                    b"verify_kernel"])
def test_a_failed_launch_is_reported(lib, cache, kernel):        # noqa: F811
    h, st = make(lib, capacity=1000)
    assert st == sp.SP_OK
    kv = dict(k_batch=1000 * HKV * D, v_batch=1000 * HKV * D)
    calls = [lambda: lib.spike_proj_cache_attend(h, ctypes.byref(attend_call(weights=FAKE, **kv)), None),
             lambda: lib.spike_proj_cache_evict(h, ctypes.byref(evict_call(budget=500, **kv)), None),
             lambda: lib.spike_proj_verify(ctypes.byref(verify_call()), None)]
    lib.fake_fail(kernel)
    assert [f() for f in calls].count(sp.SP_ECUDA) == 1
    lib.fake_fail(b"")
    assert [f() for f in calls] == [sp.SP_OK] * 3
    assert lib.spike_proj_cache_destroy(h) == sp.SP_OK


def test_the_packed_calls_have_the_structures_layout():
    """The binding packs a call's values itself; ctypes reads the same ones back."""
    for cls, pack in ((sp.SpAttend, sp._pack_attend), (sp.SpEvict, sp._pack_evict), (sp.SpVerify, sp._pack_verify)):
        values = [0.5 if t is ctypes.c_float else 3 * i + 1 for i, (_, t) in enumerate(cls._fields_)]
        got = cls.from_buffer_copy(pack(*values))
        assert [getattr(got, name) for name, _ in cls._fields_] == values


# ---- the plain implementations -------------------------------------------------
def test_attend_by_hand():
    # one K/V head, two query tokens: the first sees the prefix entry and one own
    # entry with equal scores, the second one more that weighs three times as much
    q = torch.ones(1, 2, 1, 1, dtype=torch.float64)
    pk, pv = torch.zeros(1, 1, 1), torch.full((1, 1, 1), 4.0)
    k = torch.tensor([0.0, math.log(3.0), 99.0]).view(1, 3, 1, 1).double()
    v = torch.tensor([8.0, 16.0, math.nan]).view(1, 3, 1, 1).double()
    out, lse, w, _, _ = ref.attend(q, k, v, [2], pk, pv, scale=1.0)
    assert torch.allclose(out.flatten(), torch.tensor([6.0, (4 + 8 + 48) / 5]).double())
    assert torch.allclose(lse.flatten(), torch.tensor([2.0, 5.0]).double().log())
    assert torch.allclose(w.flatten(), torch.tensor([0.5 + 0.2, 0.6, 0.0]).double())
    out, lse, w, _, _ = ref.attend(q, k, v, [0])
    assert (out == 0).all() and (lse == -math.inf).all() and (w == 0).all()


def test_attend_is_masked_attention():
    g = torch.Generator().manual_seed(5)
    Bn, Tn, H, Dn, Pn, Cn = 2, 3, 4, 16, 7, 9
    q = torch.randn(Bn, Tn, H, Dn, generator=g).double()
    pk, pv = (torch.randn(Pn, 2, Dn, generator=g).double() for _ in range(2))
    k, v = (torch.randn(Bn, Cn, 2, Dn, generator=g).double() for _ in range(2))
    lens = [9, 4]
    out, lse, w, _, _ = ref.attend(q, k, v, lens, pk, pv)
    keys, vals = (torch.cat([p.expand(Bn, -1, -1, -1), x], 1).repeat_interleave(2, 2).transpose(1, 2)
                  for p, x in ((pk, k), (pv, v)))
    seen = torch.zeros(Bn, 1, Tn, Pn + Cn, dtype=torch.bool)
    for b in range(Bn):
        for t in range(Tn):
            seen[b, 0, t, :Pn + lens[b] - (Tn - 1 - t)] = True
    want = torch.nn.functional.scaled_dot_product_attention(q.transpose(1, 2), keys, vals, attn_mask=seen)
    assert torch.allclose(out, want.transpose(1, 2))
    # a row's weights on prefix and own entries are 1 together
    total = torch.zeros(Bn)
    s = (q.transpose(1, 2) @ keys.transpose(2, 3) / 4).masked_fill(~seen, -math.inf)
    total = torch.softmax(s, -1)[..., Pn:].sum((1, 2))
    assert torch.allclose(w.sum(1), total)
    assert torch.allclose(lse, torch.logsumexp(s, -1).transpose(1, 2))


def test_evict_by_hand():
    w = torch.tensor([5.0, 1.0, 4.0, 1.0, 3.0, 2.0])
    pos = torch.tensor([0, 1, 2, 3, 4, 5])
    assert ref.evict(w, pos, 3, 6, 4, 1) == [0, 1, 2]                     # nothing leaves
    assert ref.evict(w, pos, 6, 6, 4, 1) == [0, 4, 2, 5]                  # 1 and 3 go
    assert ref.evict(w, pos, 6, 6, 4, 4) == [4, 5, 2, 3]                  # the newest four
    assert ref.evict(torch.ones(6), pos, 6, 6, 3, 0) == [0, 1, 2]         # equal: the lower slots
    assert ref.evict(torch.tensor([0.0, math.inf, math.nan]), pos, 3, 9, 1, 0) == [2]
    assert ref.evict(w, pos, 6, 6, 0, 0) == []


def test_verify_by_hand():
    f = np.float32
    p = np.array([[0.5, 0.25, 0.25, 0], [0, 0.5, 0, 0.5], [0.25] * 4], f)
    q = np.array([[0.25] * 4, [0.5, 0.5, 0, 0]], f)
    run = lambda draft, u, us, n=2: ref.verify(p, q, np.array(draft), np.array(u, f), f(us), n)   # noqa: E731
    assert run([0, 1], [0.99, 0.99], 0.5) == (2, [0, 1, 2])               # both kept, the next from p alone
    assert run([3, 1], [0.0, 0.0], 0.9) == (0, [0, -1, -1])               # p is 0; the residual is token 0's
    assert run([0, 0], [0.5, 0.1], 0.0) == (1, [0, 3, -1])                # the residual of row 1 is token 3's
    assert run([0, 1], [0.5, 0.5], 0.74, 1) == (1, [0, 3, -1])            # one draft: then p of row 1
    assert run([7, 1], [0.0, 0.0], 0.0) == (0, [0, -1, -1])               # no such token
    assert ref.verify(p[:1] * 0, q[:0], np.zeros(0), np.zeros(0, f), f(0), 0) == (0, [-1])


def test_verify_gives_the_targets_distribution():
    """Drafts drawn from q, kept or replaced, are distributed as p: summed over
    all drafts and grids of both random numbers, on which these probabilities
    are exact."""
    p = np.array([[1 / 2, 1 / 4, 1 / 8, 1 / 8], [1, 0, 0, 0]], np.float32)
    q = np.array([[1 / 4, 1 / 4, 1 / 2, 0]], np.float32)
    got = np.zeros(4)
    for x in range(4):
        for u, us in itertools.product((np.arange(8) + 0.5) / 8, (np.arange(6) + 0.5) / 6):
            got[ref.verify(p, q, np.array([x]), np.array([u], np.float32), np.float32(us), 1)[1][0]] += q[0, x] / 48
    assert np.allclose(got, p[0], atol=1e-7)
