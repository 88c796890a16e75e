"""Attention over a shared prefix and own caches, and eviction from them,
against plain 64-bit implementations."""
import ctypes
import math

import numpy as np
import pytest
import torch

import serving_ref as ref
from paper_2606_03026_gb300 import spikeproj as sp

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}


def make(seed, B, T, Hq, Hkv, D, P, C, lens, dtype, layout="entries", garbage=math.nan):
    """CPU tensors of a call; own entries that are not in use hold `garbage`."""
    g = torch.Generator().manual_seed(seed)
    t = TYPES[dtype]
    q = (1.5 * torch.randn(B, T, Hq, D, generator=g)).to(t)
    pk, pv = (torch.randn(P, Hkv, D, generator=g).to(t) for _ in range(2))
    k, v = (torch.randn(B, C, Hkv, D, generator=g).to(t) for _ in range(2))
    lens = torch.tensor(lens, dtype=torch.int32)
    for b in range(B):
        k[b, max(0, int(lens[b])):] = garbage
        v[b, max(0, int(lens[b])):] = garbage
    return q, pk, pv, k, v, lens


def on_gpu(x, layout):
    """The same values on the GPU: as they are, heads before entries, or in a wider buffer."""
    if layout == "heads":
        return x.to(DEV).transpose(-3, -2).contiguous().transpose(-3, -2)
    if layout == "padded":
        wide = torch.full((*x.shape[:-1], x.shape[-1] + 16), math.nan, dtype=x.dtype, device=DEV)
        wide[..., 8:8 + x.shape[-1]] = x.to(DEV)
        return wide[..., 8:8 + x.shape[-1]]
    return x.to(DEV)


def run(q, pk, pv, k, v, lens, layout="entries", weights=True, scale=None, start=0.25):
    B, T, Hq, D = q.shape
    C, Hkv = k.shape[1:3]
    name = "bf16" if q.dtype == torch.bfloat16 else "fp16"
    cache = sp.Cache(B, Hq, Hkv, D, C, max_T=T, dtype=name, weights=weights)
    out = on_gpu(torch.full_like(q, 7.0), layout)
    lse = torch.full((B, T, Hq), 7.0, device=DEV)
    w = torch.full((B, Hkv, C), start, device=DEV) if weights else None
    cache.attend(on_gpu(q, layout), on_gpu(k, layout), on_gpu(v, layout), lens.to(DEV), out,
                 prefix_k=on_gpu(pk, layout) if len(pk) else None,
                 prefix_v=on_gpu(pv, layout) if len(pv) else None, weights=w, lse=lse, scale=scale)
    torch.cuda.synchronize()
    assert cache.status() == sp.SP_OK
    cache.close()
    return out.cpu(), lse.cpu(), None if w is None else w.cpu()


def check(q, pk, pv, k, v, lens, got, scale=None, start=0.25):
    out, lse, w = got
    want, wlse, ww, mass, size = ref.attend(q, k, v, lens, pk, pv, scale)
    used = torch.cat([pv.double().abs().flatten(), v.double().abs().nan_to_num(0).flatten(), torch.zeros(1)])
    out_tol, lse_tol, w_rel = ref.attend_bounds(q.dtype, q.shape[3], pk.shape[0] + k.shape[1], mass, size, want,
                                                float(used.max()))
    empty = wlse == -math.inf
    assert torch.equal(lse.isneginf(), empty)
    assert (out[empty] == 0).all(), "a row that sees nothing is not zero"
    err = (out.double() - want).abs()
    assert (err <= out_tol).all(), f"out: {(err / out_tol).max()} of its bound"
    e = (lse.double() - wlse).abs()[~empty]
    assert (e <= (lse_tol + 2.0 ** -22 * wlse.abs())[~empty]).all(), "lse"
    if w is not None:
        n = lens.clamp(0, k.shape[1])
        inside = torch.arange(k.shape[1]).view(1, 1, -1) < n.view(-1, 1, 1)
        assert (w[~inside.expand_as(w)] == start).all(), "weights of entries that are not in use changed"
        # each of the T * Hq / Hkv terms has the relative error of a probability
        tol = ww * (w_rel.max() + 2.0 ** -20) + 2.0 ** -23 * (ww + start)
        e = (w.double() - start - ww).abs()
        assert (e <= tol)[inside.expand_as(w)].all(), f"weights: {(e / tol)[inside.expand_as(w)].max()} of the bound"


CASES = [
    # B, T, Hq, Hkv, D, P, C, lens
    (1, 1, 1, 1, 64, 1, 1, [1]),
    (1, 1, 4, 2, 128, 0, 5, [3]),
    (2, 1, 12, 4, 128, 129, 300, [300, 1]),
    (3, 1, 3, 1, 64, 127, 128, [128, 127, 0]),
    (5, 2, 8, 2, 128, 128, 257, [257, 256, 130, 2, 1]),
    (4, 5, 6, 2, 64, 300, 140, [140, 133, 128, 5]),
    (2, 8, 16, 2, 128, 1000, 200, [200, 131]),
    (3, 3, 4, 4, 80, 77, 90, [90, 41, 3]),
    (2, 4, 8, 8, 96, 513, 64, [64, 7]),
    (2, 2, 5, 5, 8, 33, 20, [20, 19]),
    (2, 3, 12, 3, 72, 65, 150, [129, 150]),
    (40, 1, 6, 2, 128, 260, 33, [i % 34 for i in range(40)]),       # more rows than a tile
    (16, 6, 24, 3, 64, 200, 150, [9 * i + 6 for i in range(16)]),
    (1, 32, 16, 2, 128, 250, 64, [40]),                             # 256 rows of one head
    (2, 1, 200, 1, 64, 70, 140, [140, 3]),                          # 200 query heads on one
]


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(map(str, c[:7])))
def test_attend_matches_the_definition(case, dtype):
    x = make(11, *case, dtype)
    check(*x, run(*x))


@pytest.mark.parametrize("layout", ["heads", "padded"])
@pytest.mark.parametrize("case", [CASES[5], CASES[7], CASES[2]], ids=["T5", "D80", "T1"])
def test_attend_strides(case, layout):
    x = make(12, *case, "bf16")
    check(*x, run(*x, layout=layout))


def test_attend_long_prefix_splits_over_the_device():
    x = make(13, 3, 2, 8, 2, 128, 40001, 700, [700, 333, 2], "bf16")
    check(*x, run(*x))


def test_attend_long_own_caches():
    x = make(14, 2, 1, 4, 2, 64, 5, 9000, [9000, 8191], "fp16")
    check(*x, run(*x))


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_attend_rows_that_see_nothing(dtype):
    # no prefix: sequence 0 has nothing, 1 fewer entries than queries, 2 exactly as many
    x = make(15, 4, 3, 4, 2, 64, 0, 130, [0, 2, 3, 130], dtype)
    check(*x, run(*x))


def test_attend_lens_are_taken_into_the_capacity():
    q, pk, pv, k, v, lens = make(16, 3, 1, 2, 1, 64, 10, 40, [40, 0, 40], "bf16")
    check(q, pk, pv, k, v, torch.tensor([40, 0, 40]), run(q, pk, pv, k, v, torch.tensor([41, -5, 2 ** 31 - 1], dtype=torch.int32)))


def test_attend_scores_that_keep_rising_and_extreme_ones():
    # later tiles always beat the maximum so far; then scores far apart, where all but one vanish
    for factor in (1.0, 30.0):
        q, pk, pv, k, v, lens = make(17, 2, 2, 4, 2, 64, 700, 300, [300, 200], "bf16")
        ramp = torch.linspace(-8, 8, 700).view(-1, 1, 1) * factor
        pk = (q[0, 0, 0].float().sign() * ramp).to(torch.bfloat16).expand(700, 2, 64).contiguous()
        check(q, pk, pv, k, v, lens, run(q, pk, pv, k, v, lens))


def test_attend_half_precision_keeps_a_long_flat_tail():
    # one entry 14 nats above 30000 others, which together weigh 2.5 %: their
    # probabilities lie below half precision's subnormals
    q, pk, pv, k, v, lens = make(18, 1, 1, 1, 1, 64, 30000, 4, [1], "fp16")
    q = torch.ones_like(q)
    pk = torch.zeros_like(pk)
    pk[77] = 14.0 / 8.0
    k[0, 0] = 0
    pv = (1 + pv.float().abs()).half()
    check(q, pk, pv, k, v, lens, run(q, pk, pv, k, v, lens))


def test_attend_nan_and_infinity_stay_with_the_rows_that_see_them():
    q, pk, pv, k, v, lens = make(19, 3, 4, 4, 2, 64, 200, 140, [135, 64, 4], "bf16")
    clean = run(q, pk, pv, k, v, lens)
    # the last draft's entry of sequence 0: value NaN; of sequence 1: key NaN; of
    # sequence 2: value infinite.  Only the last query token of each sees them.
    v[0, 134] = math.nan
    k[1, 63] = math.nan
    v[2, 3] = math.inf
    out, lse, w = run(q, pk, pv, k, v, lens)
    assert torch.equal(out[:, :3], clean[0][:, :3])
    assert out[0, 3].isnan().all() and out[1, 3].isnan().all() and (out[2, 3] == math.inf).all()
    assert torch.equal(lse[:, :3], clean[1][:, :3]) and torch.equal(lse[0], clean[1][0])


def test_attend_is_reproducible_and_leaves_its_inputs():
    x = make(20, 6, 3, 12, 4, 128, 3001, 600, [600, 5, 77, 128, 400, 3], "bf16")
    a, b = run(*x), run(*x)
    for i, j in zip(a, b):
        assert torch.equal(i, j)


def test_attend_a_sequence_does_not_depend_on_its_neighbours():
    q, pk, pv, k, v, lens = make(21, 4, 2, 4, 2, 64, 300, 200, [200, 100, 50, 7], "bf16")
    want, _, _, mass, size = ref.attend(q[1:2], k[1:2], v[1:2], lens[1:2], pk, pv)
    v[0] = math.nan
    q[2] = math.nan
    out, lse, w = run(q, pk, pv, k, v, lens)
    tol = ref.attend_bounds(q.dtype, 64, 500, mass, size, want, 8.0)[0]
    assert ((out[1:2].double() - want).abs() <= tol).all()
    assert out[0].isnan().all() and out[2].isnan().all() and not out[3].isnan().any()


def test_attend_smaller_calls_than_the_handle_on_another_stream():
    cache = sp.Cache(8, 8, 2, 64, 100, max_T=6, dtype="bf16", weights=True)
    stream = torch.cuda.Stream()
    for B, T in ((8, 6), (3, 2), (1, 1)):
        x = make(22 + T, B, T, 8, 2, 64, 90, 100, [100 - 3 * b for b in range(B)], "bf16")
        q, pk, pv, k, v, lens = [a.to(DEV) for a in x]
        out, lse, w = torch.empty_like(q), torch.empty(B, T, 8, device=DEV), torch.zeros(B, 2, 100, device=DEV)
        torch.cuda.synchronize()
        cache.attend(q, k, v, lens, out, pk, pv, w, lse, stream=stream)
        stream.synchronize()
        check(*x, (out.cpu(), lse.cpu(), w.cpu()), start=0.0)
    cache.close()


def test_attend_in_a_graph():
    x = make(30, 4, 2, 8, 2, 128, 500, 200, [200, 100, 50, 7], "bf16")
    q, pk, pv, k, v, lens = [a.to(DEV) for a in x]
    cache = sp.Cache(4, 8, 2, 128, 200, max_T=2, weights=True)
    out, lse, w = torch.zeros_like(q), torch.empty(4, 2, 8, device=DEV), torch.zeros(4, 2, 200, device=DEV)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        cache.attend(q, k, v, lens, out, pk, pv, w, lse)
    torch.cuda.synchronize()
    w.zero_()
    out.zero_()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        cache.attend(q, k, v, lens, out, pk, pv, w, lse)
    g.replay()
    torch.cuda.synchronize()
    check(*x, (out.cpu(), lse.cpu(), w.cpu()), start=0.0)
    # other lengths, read on the device
    lens.copy_(torch.tensor([2, 200, 199, 64], dtype=torch.int32))
    k2, v2 = (torch.randn(4, 200, 2, 128, device=DEV).bfloat16() for _ in range(2))
    k.copy_(k2), v.copy_(v2), w.zero_()
    g.replay()
    torch.cuda.synchronize()
    check(x[0], x[1], x[2], k.cpu(), v.cpu(), lens.cpu(), (out.cpu(), lse.cpu(), w.cpu()), start=0.0)
    cache.close()


@pytest.mark.parametrize("D", [40, 64, 72, 128])
def test_attend_many_rows_of_odd_number(D):
    # 2277 rows, two to a warp of the merge; neighbours of other lengths, some empty
    lens = [(7 * b) % 41 for b in range(23)]
    x = make(32, 23, 3, 33, 11, D, 70, 40, lens, "bf16")
    check(*x, run(*x))


def test_attend_more_heads_than_a_grid_is_high():
    """1024 sequences x 65 K/V heads, one own entry each: it has all of the weight."""
    B, H, D = 1024, 65, 8
    g = torch.Generator().manual_seed(31)
    q, k, v = (torch.randn(B, 1, H, D, generator=g).bfloat16().to(DEV) for _ in range(3))
    cache = sp.Cache(B, H, H, D, 1, weights=True)
    out, w = torch.empty_like(q), torch.zeros(B, H, 1, device=DEV)
    cache.attend(q, k, v, torch.ones(B, dtype=torch.int32, device=DEV), out, weights=w)
    torch.cuda.synchronize()
    assert cache.status() == sp.SP_OK
    assert torch.equal(out, v) and ((w - 1).abs() <= 2.0 ** -20).all()
    cache.close()


# ---------------------------------------------------------------------------
def evict_case(seed, B, Hkv, D, C, lens, budget, recent, kind, dtype="bf16", layout="entries"):
    g = torch.Generator().manual_seed(seed)
    k, v = (torch.randn(B, C, Hkv, D, generator=g).to(TYPES[dtype]) for _ in range(2))
    w = torch.exp(2 * torch.randn(B, Hkv, C, generator=g))
    if kind == "ties":
        w = (w * 0.7).floor()
    if kind == "equal":
        w = torch.ones_like(w)
    if kind == "odd":              # every kind of value that a float has
        pool = torch.tensor([0.0, -0.0, math.nan, math.inf, -math.inf, -1.0, 1e-45, 1.0, 3e38, -math.nan])
        w = pool[torch.randint(0, len(pool), w.shape, generator=g)]
    pos = torch.argsort(torch.rand(B, Hkv, C, generator=g), dim=2).to(torch.int32)
    lens = torch.tensor(lens, dtype=torch.int32)
    now = torch.full((B,), C, dtype=torch.int32)
    return k, v, w, pos, lens, now


def run_evict(k, v, w, pos, lens, now, budget, recent, layout="entries", room=None):
    B, C, Hkv, D = k.shape
    cache = sp.Cache(B, Hkv, Hkv, D, C, dtype="bf16" if k.dtype == torch.bfloat16 else "fp16")
    room = min(budget, C) if room is None else room
    gk, gv = on_gpu(k, layout), on_gpu(v, layout)
    wo, po = torch.full((B, Hkv, room), 7.0, device=DEV), torch.full((B, Hkv, room), 7, dtype=torch.int32, device=DEV)
    lo = torch.full((B,), -7, dtype=torch.int32, device=DEV)
    cache.evict(gk, gv, w.to(DEV), pos.to(DEV), lens.to(DEV), now.to(DEV), budget, recent, wo, po, lo)
    torch.cuda.synchronize()
    cache.close()
    return gk.cpu(), gv.cpu(), wo.cpu(), po.cpu(), lo.cpu()


def check_evict(x, budget, recent, got):
    k, v, w, pos, lens, now = x
    gk, gv, wo, po, lo = got
    B, C, Hkv, D = k.shape
    for b in range(B):
        n = min(max(int(lens[b]), 0), C)
        assert int(lo[b]) == min(n, budget)
        for h in range(Hkv):
            src = ref.evict(w[b, h], pos[b, h], n, now[b], budget, recent)
            wk, wv = k[b, :, h].clone(), v[b, :, h].clone()
            wk[:len(src)], wv[:len(src)] = k[b, src, h], v[b, src, h]
            assert torch.equal(gk[b, :, h], wk) and torch.equal(gv[b, :, h], wv), (b, h)
            assert np.array_equal(wo[b, h, :len(src)].numpy().view(np.uint32), w[b, h, src].numpy().view(np.uint32))
            assert torch.equal(po[b, h, :len(src)], pos[b, h, src])
            assert (wo[b, h, len(src):] == 7).all() and (po[b, h, len(src):] == 7).all()


EVICT = [
    # B, Hkv, D, C, lens, budget, recent
    (1, 1, 64, 1, [1], 0, 0),
    (1, 1, 64, 2, [2], 1, 1),
    (2, 2, 128, 40, [40, 33], 32, 8),
    (4, 1, 8, 700, [700, 513, 512, 0], 512, 0),
    (3, 2, 80, 1100, [1100, 1024, 77], 600, 600),
    (2, 1, 64, 300, [300, 250], 400, 10),          # budget beyond the capacity
    (2, 2, 64, 513, [513, 100], 0, 0),             # nothing stays
    (1, 2, 64, 5000, [4999], 300, 50),             # most goes
    (1, 1, 64, 20000, [20000], 12000, 77),         # several CTAs per head
    (3, 1, 8, 200000, [200000, 150001, 9], 70001, 5),   # more keys than shared memory holds
]


@pytest.mark.parametrize("kind", ["spread", "ties", "equal", "odd"])
@pytest.mark.parametrize("case", EVICT, ids=lambda c: "-".join(map(str, c[:4])) + f"-{c[5]}")
def test_evict_matches_the_definition(case, kind):
    x = evict_case(41, *case, kind)
    check_evict(x, *case[5:], run_evict(*x, *case[5:]))


@pytest.mark.parametrize("layout", ["heads", "padded"])
def test_evict_strides_and_half_precision(layout):
    case = (2, 3, 72, 500, [500, 400], 256, 30)
    x = evict_case(42, *case, "ties", "fp16")
    check_evict(x, 256, 30, run_evict(*x, 256, 30, layout=layout, room=300))


def test_evict_takes_lens_into_the_capacity_and_now_to_its_ends():
    k, v, w, pos, lens, now = evict_case(43, 3, 1, 64, 100, [100, 0, 100], 60, 20, "spread")
    pos[2] = torch.randint(-2 ** 31, 2 ** 31 - 1, (1, 100), generator=torch.Generator().manual_seed(1)).to(torch.int32)
    now[2] = -2 ** 31                                # now - recent leaves 32 bits
    x = k, v, w, pos, torch.tensor([101, -1, 2 ** 31 - 1], dtype=torch.int32), now
    check_evict((k, v, w, pos, lens, now), 60, 20, run_evict(*x, 60, 20))


def test_attend_after_evict_sees_the_kept_entries():
    case = (2, 2, 64, 400, [400, 390], 200, 16)
    k, v, w, pos, lens, now = evict_case(44, *case, "spread")
    gk, gv, wo, po, lo = run_evict(k, v, w, pos, lens, now, 200, 16)
    q, pk, pv = make(45, 2, 1, 4, 2, 64, 50, 400, [0, 0], "bf16")[:3]
    got = run(q, pk, pv, gk, gv, lo)
    check(q, pk, pv, gk, gv, lo, got)
    # the same entries in their old order
    ok, ov = k.clone(), v.clone()
    for b in range(2):
        for h in range(2):
            src = sorted(ref.evict(w[b, h], pos[b, h], int(lens[b]), now[b], 200, 16))
            ok[b, :200, h], ov[b, :200, h] = k[b, src, h], v[b, src, h]
    check(q, pk, pv, ok, ov, lo, (got[0], got[1], None))


# ---------------------------------------------------------------------------
def test_offsets_past_32_bits():
    """Caches of 6 GB each (more than 2^31 elements): the last sequence lies past 32-bit offsets."""
    B, C, Hkv, D = 3, 400_000, 8, 128
    k = torch.zeros(B, C, Hkv, D, dtype=torch.bfloat16, device=DEV)
    v = torch.zeros_like(k)
    assert (B - 1) * k.stride(0) * 2 > 2 ** 30 and k.numel() > 2 ** 30
    lens = torch.tensor([0, 0, C], dtype=torch.int32, device=DEV)
    k[2, C - 1], v[2, C - 1] = 1.0, 3.0
    k[2, 5], v[2, 5] = 1.0, 1.0
    q = torch.full((B, 1, Hkv, D), 2.0, dtype=torch.bfloat16, device=DEV)
    out = torch.empty_like(q)
    cache = sp.Cache(B, Hkv, Hkv, D, C, dtype="bf16")
    cache.attend(q, k, v, lens, out, scale=1.0)
    # two entries share all of the weight: 256 nats above the rest
    assert (out[2] == 2.0).all() and (out[:2] == 0).all()
    w = torch.zeros(B, Hkv, C, device=DEV)
    w[2, :, C - 1] = 1
    pos = torch.arange(C, dtype=torch.int32, device=DEV).expand(B, Hkv, C).contiguous()
    wo, po = torch.zeros(B, Hkv, 10, device=DEV), torch.zeros(B, Hkv, 10, dtype=torch.int32, device=DEV)
    lo = torch.zeros_like(lens)
    cache.evict(k, v, w, pos, lens, lens, 10, 0, wo, po, lo)
    torch.cuda.synchronize()
    assert (v[2, 9] == 3.0).all() and (v[2, 5] == 1.0).all() and (po[2, :, 9] == C - 1).all()
    assert lo.tolist() == [0, 0, 10] and (wo[2, :, 9] == 1).all() and not v[:2].any()
    cache.close()


# ---------------------------------------------------------------------------
def test_refusals():
    cache = sp.Cache(2, 4, 2, 64, 32, max_T=2)
    q = torch.zeros(2, 2, 4, 64, dtype=torch.bfloat16, device=DEV)
    k = torch.zeros(2, 32, 2, 64, dtype=torch.bfloat16, device=DEV)
    lens = torch.zeros(2, dtype=torch.int32, device=DEV)
    w = torch.zeros(2, 2, 32, device=DEV)

    def status(f, *a, **kw):
        with pytest.raises(sp.SpikeProjError) as e:
            f(*a, **kw)
        return e.value.status

    out = torch.zeros_like(q)
    assert status(cache.attend, q, k, k, lens, out, weights=w) == sp.SP_EUNSUPPORTED
    for scale in (0.0, -1.0, math.inf, math.nan):
        assert status(cache.attend, q, k, k, lens, out, scale=scale) == sp.SP_EINVAL
    big = torch.zeros(3, 2, 4, 64, dtype=torch.bfloat16, device=DEV)
    assert status(cache.attend, big, torch.zeros(3, 32, 2, 64, dtype=torch.bfloat16, device=DEV),
                  torch.zeros(3, 32, 2, 64, dtype=torch.bfloat16, device=DEV),
                  torch.zeros(3, dtype=torch.int32, device=DEV), torch.zeros_like(big)) == sp.SP_ERANGE
    long = torch.zeros(2, 3, 4, 64, dtype=torch.bfloat16, device=DEV)
    assert status(cache.attend, long, k, k, lens, torch.zeros_like(long)) == sp.SP_ERANGE
    # a K that starts off 16 bytes, rows 68 elements apart, heads that share one
    odd = torch.zeros(2 * 32 * 2 * 64 + 8, dtype=torch.bfloat16, device=DEV)[4:-4].view(2, 32, 2, 64)
    assert status(cache.attend, q, odd, k, lens, out) == sp.SP_EALIGN
    assert status(cache.attend, q, torch.zeros(2, 32, 2, 68, dtype=torch.bfloat16, device=DEV)[..., :64], k, lens, out) \
        == sp.SP_EALIGN
    assert status(cache.attend, q, k[:, :, :1].expand(2, 32, 2, 64), k, lens, out) == sp.SP_EALIGN
    # shapes and types that the binding refuses
    for bad in (lambda: cache.attend(q, k[:, :31], k, lens, out), lambda: cache.attend(q.half(), k, k, lens, out),
                lambda: cache.attend(q, k, k, lens.long(), out), lambda: cache.attend(q, k, k.cpu(), lens, out),
                lambda: cache.attend(q, k, k, lens, out, prefix_k=k[0], prefix_v=k[0, :5])):
        with pytest.raises(ValueError):
            bad()
    pos, wo, po = (torch.zeros(2, 2, 32, dtype=t, device=DEV) for t in (torch.int32, torch.float32, torch.int32))
    lo = torch.zeros_like(lens)
    assert status(cache.evict, k, k, w, pos, lens, lens, 8, 9, wo, po, lo) == sp.SP_EINVAL
    assert status(cache.evict, k, k, w, pos, lens, lens, -1, 0, wo, po, lo) == sp.SP_EINVAL
    assert status(cache.evict, k, k, w, pos, lens, lens, 8, 0, w, po, lo) == sp.SP_EINVAL
    assert status(cache.evict, k, k, w, pos, lens, lens, 8, 0, wo, pos, lo) == sp.SP_EINVAL
    assert status(cache.evict, k, k, w, pos, lens, lens, 8, 0, wo, po, lens) == sp.SP_EINVAL
    with pytest.raises(ValueError):
        cache.evict(k, k, w, pos, lens, lens, 8, 0, wo[:, :, :7], po[:, :, :7], lo)
    torch.cuda.synchronize()
    cache.close()
