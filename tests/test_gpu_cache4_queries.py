"""Queries of any size of their type, with scales that bring their scores to what a
softmax tells apart, and with scales that do not."""
import math

import pytest
import torch

import cache4_ref as ref
from test_gpu_cache4 import TYPES, check, held_entries, make, run

pytestmark = pytest.mark.gpu

# by blocks for themselves, by warps in line, by CTAs
KERNELS = [(1, 6, 300), (2, 14, 900), (6, 14, 900)]


@pytest.mark.parametrize("D", [64, 80, 128])
@pytest.mark.parametrize("T,Hq,C", KERNELS, ids=str)
@pytest.mark.parametrize("power", [-130, -126, -120, -110, -100, -87, -84, -60, 60, 100, 124])
def test_scores_of_order_one(power, T, Hq, C, D):
    """Rows of 2^power (bf16's numbers begin at 2^-133 and have 8 bits from 2^-126 on)
    and scales that bring their scores to order one."""
    q, k4, v4, lens = make(61, 2, T, Hq, 2, D, C, [C, C // 3], "bf16")
    q = (q.double() * 2.0 ** power).bfloat16()
    scale = min(0.05 * 2.0 ** -power, 2.0 ** 127)
    check(q, k4, v4, lens, run(q, k4, v4, lens, scale=scale), scale=scale)


@pytest.mark.parametrize("T,Hq,C", KERNELS, ids=str)
def test_rows_of_all_sizes_together(T, Hq, C):
    """A row of 2^-120 beside others of up to 2^-100 in one unit, zeros among them, and
    infinities and NaN in the place of some elements."""
    q, k4, v4, lens = make(62, 2, T, Hq, 2, 128, C, [C, C // 2], "bf16")
    sizes = torch.exp2(-100 - 20 * torch.rand(2, T, Hq, 1, generator=torch.Generator().manual_seed(63)).double())
    sizes[:, :, 0], sizes[:, :, Hq // 2] = 2.0 ** -120, 0.0
    q = (q.double() * sizes).bfloat16()
    got = run(q, k4, v4, lens, scale=2.0 ** 100)
    check(q, k4, v4, lens, got, scale=2.0 ** 100)
    bad = q.clone()
    bad[:, :, 1, 7], bad[:, :, 2, 9] = math.nan, math.inf
    out, lse = run(bad, k4, v4, lens, scale=2.0 ** 100)
    assert out[:, -1, 1:3].isnan().all() and lse[:, -1, 1:3].isnan().all()
    rest = [i for i in range(Hq) if i not in (1, 2)]
    assert torch.equal(out[:, :, rest], got[0][:, :, rest]) and torch.equal(lse[:, :, rest], got[1][:, :, rest])


def one_element(T, Hq, C, D, dtype, element, code, byte):
    """Queries of one element, keys of one element: scores are a product of two numbers."""
    g = torch.Generator().manual_seed(64)
    q = torch.zeros(2, T, Hq, D, dtype=TYPES[dtype])
    q[..., 5] = element
    k4 = torch.zeros(2, C, 2, D // 2, dtype=torch.uint8), torch.full((2, C, 2, D // 16), byte, dtype=torch.uint8)
    k4[0][..., 2] = 16 * code               # element 5
    return q, k4, held_entries(g, 2, C, 2, D), torch.tensor([C, C // 2], dtype=torch.int32)


# the type, an element of the queries, a scale: with keys of 2^-18 scores within FP32
LARGE = [("bf16", 2.0 ** 126, 2.0 ** 15), ("bf16", 2.0 ** 127, 2.0 ** 17), ("bf16", -(2.0 ** 120), 2.0 ** 22),
         ("bf16", 2.0 ** 14, 2.0 ** 127), ("bf16", 2.0 ** -20, 3e38), ("bf16", 2.0 ** -133, 3e38), ("fp16", 2.0 ** -24, 3e38),
         ("fp16", 2.0 ** 10, 2.0 ** 127), ("fp16", -1.0, 3.4e38), ("bf16", 2.0 ** -120, 2.0 ** -120), ("bf16", 0.0, 3e38),
         ("fp16", 0.0, 3e38), ("fp16", 0.0, 1e-44)]


@pytest.mark.parametrize("T,Hq,C", KERNELS, ids=str)
@pytest.mark.parametrize("dtype,element,scale", LARGE, ids=str)
def test_scales_of_any_size(dtype, element, scale, T, Hq, C):
    """Equal scores give the mean of the values whatever their size, and their lse; a
    score above the others by 2^20 and more is all of the weight."""
    q, k4, v4, lens = one_element(T, Hq, C, 64, dtype, element, 1, 1)          # keys of 2^-18
    G = Hq // 2
    out, lse = run(q, k4, v4, lens, causal=False, scale=scale)
    v = ref.values(*v4)
    score = float(q[0, 0, 0, 5]) * 2.0 ** -18 * float(torch.tensor(scale, dtype=torch.float32))
    assert abs(score) < 2.0 ** 127
    for b in range(2):
        n = int(lens[b])
        mean, size = (x.mean(0).repeat_interleave(G, 0) for x in (v[b, :n], v[b, :n].abs()))
        # a probability's rounding and its sum's; the sums; the result's, and half precision's last step
        tol = size * (2 * 2.0 ** -11 + 2.0 ** -16) + (mean.abs() + size * 2.0 ** -10) * torch.finfo(q.dtype).eps / 2 + 2.0 ** -25
        assert ((out[b].double() - mean).abs() <= tol).all()
        want = score + math.log(n)
        assert ((lse[b].double() - want).abs() <= 2.0 ** -22 * abs(want) + 2.0 ** -19).all()
    if abs(score) >= 2.0 ** 20:
        k4[0][:, 100, :, 2] = 16 * (2 if score > 0 else 0)                     # twice the score, or nothing below 0
        out, lse = run(q, k4, v4, lens, causal=False, scale=scale)
        assert torch.equal(out, v[:, 100].to(q.dtype).repeat_interleave(G, 1).unsqueeze(1).expand(out.shape))
        want = max(0.0, 2 * score)
        assert ((lse.double() - want).abs() <= 2.0 ** -22 * want + 2.0 ** -19).all()


@pytest.mark.parametrize("T,Hq,C", KERNELS, ids=str)
@pytest.mark.parametrize("dtype,element,scale", [x for x in LARGE if x[1]], ids=str)
def test_rows_that_see_nothing_whatever_the_scale(dtype, element, scale, T, Hq, C):
    """Masks hold at every size: fewer entries than tokens, joined with other attention."""
    q, k4, v4, _ = one_element(T, Hq, C, 64, dtype, element, 1, 1)
    lens = torch.tensor([T - 1, 0], dtype=torch.int32)
    other = torch.full_like(q, 2.0), torch.full((2, T, Hq), -math.inf)
    other[1][:, :, 1] = -3.0
    out, lse = run(q, k4, v4, lens, scale=scale, other=other)
    assert (out[1, :, 1] == 2).all() and ((lse[1, :, 1] + 3).abs() <= 2.0 ** -20).all()
    assert (out[0, 0, 1] == 2).all() and ((lse[0, 0, 1] + 3).abs() <= 2.0 ** -20).all()
    rest = [i for i in range(Hq) if i != 1]
    assert (out[1][:, rest] == 0).all() and (lse[1][:, rest] == -math.inf).all()
    assert (out[0, 0, rest] == 0).all() and (lse[0, 0, rest] == -math.inf).all()
    assert out.isfinite().all()


@pytest.mark.parametrize("T,Hq,C", KERNELS, ids=str)
@pytest.mark.parametrize("dtype,element,scale", [("bf16", 2.0 ** 127, 3e38), ("bf16", 2.0 ** 100, 2.0 ** 100), ("bf16", 2.0 ** 127, 2.0 ** 19),
                                                 ("fp16", 2.0 ** 15, 3e38)], ids=str)
def test_scores_below_the_range(dtype, element, scale, T, Hq, C):
    """Entries whose scores FP32 does not hold have no weight: a row of them alone sees
    nothing, beside one score of 0 they vanish."""
    q, k4, v4, lens = one_element(T, Hq, C, 64, dtype, element, 15, 8)         # keys of -6 * 2^-14
    out, lse = run(q, k4, v4, lens, causal=False, scale=scale)
    assert (out == 0).all() and (lse == -math.inf).all()
    other = torch.full_like(q, 2.0), torch.full((2, T, Hq), -3.0)
    out, lse = run(q, k4, v4, lens, causal=False, scale=scale, other=other)
    assert (out == 2).all() and ((lse + 3).abs() <= 2.0 ** -20).all()
    k4[0][:, 77] = 0
    out, lse = run(q, k4, v4, lens, causal=False, scale=scale)
    assert torch.equal(out, ref.values(*v4)[:, 77].to(q.dtype).repeat_interleave(Hq // 2, 1).unsqueeze(1).expand(out.shape))
    assert (lse.abs() <= 2.0 ** -19).all()
