"""A KV cache held in 4 bits: writing, reading and attention against plain 64-bit
implementations."""
import math

import pytest
import torch

import cache4_ref as ref
import serving_ref
from paper_2606_03026_gb300 import spikeproj as sp

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}


def place(x, layout):
    """The values of [B, C or T, H, W] on the GPU: as they are, heads before entries, or in a wider buffer."""
    if layout == "heads":
        return x.to(DEV).transpose(1, 2).contiguous().transpose(1, 2)
    if layout == "padded":
        room = 32 if x.dtype == torch.uint8 else 16
        wide = torch.full((*x.shape[:-1], x.shape[-1] + 2 * room), 77, dtype=x.dtype, device=DEV)
        wide[..., room:room + x.shape[-1]] = x.to(DEV)
        return wide[..., room:room + x.shape[-1]]
    return x.to(DEV)


def activations(g, *shape, dtype):
    x = torch.randn(*shape, generator=g) * torch.exp2(torch.randint(-6, 7, (*shape[:-1], 1), generator=g).float())
    return x.to(TYPES[dtype])


# ---------------------------------------------------------------------------
def check_codes(x, layout="entries"):
    """x [rows, D]: one token each of a batch of one sequence with one head."""
    D = x.shape[1]
    rows = x.view(1, -1, 1, D)
    name = "bf16" if x.dtype == torch.bfloat16 else "fp16"
    cache = sp.Cache4(1, 1, D, rows.shape[1], dtype=name)
    k4, v4 = cache.new(1)
    k_out, v_out = (torch.zeros_like(rows, device=DEV) for _ in range(2))
    cache.write(rows.to(DEV), rows.flip(1).to(DEV), k4, v4, k_out=k_out, v_out=v_out)
    codes, scales, values = ref.quantise(x)
    for held, out, order in ((k4, k_out, 1), (v4, v_out, -1)):
        assert torch.equal(held[0].cpu()[0, ::1, 0], codes if order > 0 else codes.flip(0))
        assert torch.equal(held[1].cpu()[0, :, 0], scales if order > 0 else scales.flip(0))
        want = (values if order > 0 else values.flip(0)).to(x.dtype)
        assert torch.equal(want.double().nan_to_num(9e9), (values if order > 0 else values.flip(0)).nan_to_num(9e9)), "not exact in the type"
        got = out.cpu()[0, :, 0]
        assert torch.equal(got.isnan(), want.isnan()) and torch.equal(got.nan_to_num(0), want.nan_to_num(0))
    back_k, back_v = (torch.zeros_like(rows, device=DEV) for _ in range(2))
    cache.read(k4, v4, back_k, back_v)
    assert torch.equal(back_k.view(torch.int16), k_out.view(torch.int16))
    assert torch.equal(back_v.view(torch.int16), v_out.view(torch.int16))
    cache.close()


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_every_largest_element(dtype):
    """All 2^16 bit patterns as a group's largest element (NaN and infinities too)."""
    top = torch.arange(-2 ** 15, 2 ** 15).to(torch.int16).view(TYPES[dtype])
    g = torch.Generator().manual_seed(1)
    x = (top.double().unsqueeze(1) * (2 * torch.rand(2 ** 16, 16, generator=g) - 1)).to(TYPES[dtype])
    x[torch.arange(2 ** 16), torch.randint(0, 16, (2 ** 16,), generator=g)] = top
    check_codes(x)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_elements_on_and_beside_the_borders(dtype):
    """Every scale times every border between two codes, and the numbers of the type beside it."""
    borders = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0], dtype=torch.float64)
    scales = ref.SCALES[1:]
    x = (scales.unsqueeze(1) * borders).to(TYPES[dtype])
    rows = []
    for step in (-1, 0, 1):
        y = (x.view(torch.int16) + step).view(TYPES[dtype])
        rows.append(torch.cat([y, -y, torch.zeros_like(y[:, :1]), (6 * scales).unsqueeze(1).to(TYPES[dtype])], 1))
    check_codes(torch.cat(rows))


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_scales_on_and_beside_their_borders(dtype):
    """Largest elements six times what lies halfway between two scales, and the numbers beside them."""
    half = 6 * (ref.SCALES[1:] + ref.SCALES[:-1]) / 2
    x = half.to(TYPES[dtype]).view(torch.int16)
    x = torch.cat([(x + i).view(TYPES[dtype]) for i in range(-3, 4)])
    check_codes(x.unsqueeze(1) * torch.linspace(-1, 1, 16).to(TYPES[dtype]))


def test_special_groups():
    x = torch.randn(10, 128, generator=torch.Generator().manual_seed(2)).bfloat16()
    x[9, ::3], x[9, 1::3] = -0.0, 0.0
    x[0], x[1], x[2] = 0.0, -0.0, 1e-30
    x[3, 17], x[4, 127], x[5, 0] = math.nan, math.inf, -math.inf
    x[6], x[7, 5] = 3e38, 3e38
    x[8] = torch.where(torch.arange(128) % 2 == 0, -1e-6, 2e-5).bfloat16()
    check_codes(x)
    check_codes(x.half())


# ---------------------------------------------------------------------------
def written(B, T, Hkv, D, C, at, n, dtype, layout, out, seed=3):
    g = torch.Generator().manual_seed(seed)
    k, v = (activations(g, B, T, Hkv, D, dtype=dtype) for _ in range(2))
    held = [torch.randint(0, top, (B, C, Hkv, w), generator=g).to(torch.uint8) for w, top in ((D // 2, 256), (D // 16, 227)) * 2]
    outs = [torch.full_like(k, 5.0) for _ in range(2)]
    cache = sp.Cache4(Hkv, Hkv, D, C, dtype=dtype)
    gk4 = tuple(place(x, layout) for x in held[:2])
    gv4 = tuple(place(x, layout) for x in held[2:])
    gouts = [place(x, layout) for x in outs] if out else [None, None]
    ints = [None if x is None else torch.tensor(x, dtype=torch.int32) for x in (at, n)]
    cache.write(place(k, layout), place(v, layout), gk4, gv4, *(None if x is None else x.to(DEV) for x in ints),
                *gouts)
    for b in range(B):
        a = 0 if at is None else at[b]
        for t in range(T if n is None else min(max(n[b], 0), T)):
            for i, x in enumerate((k, v)):
                codes, scales, values = ref.quantise(x[b, t])
                if 0 <= a + t < C:
                    held[2 * i][b, a + t], held[2 * i + 1][b, a + t] = codes, scales
                outs[i][b, t] = values.to(x.dtype)
    for got, want in zip(gk4 + gv4, held):
        assert torch.equal(got.cpu(), want)
    if out:
        for got, want in zip(gouts, outs):
            assert torch.equal(got.cpu(), want)
    # and back: slots from one before the first on, one token more
    reads = [torch.full((B, T + 1, Hkv, D), 3.0, dtype=TYPES[dtype]) for _ in range(2)]
    greads = [place(x, layout) for x in reads]
    before = None if at is None else torch.tensor([x - 1 for x in at], dtype=torch.int32, device=DEV)
    cache.read(gk4, gv4, *greads, before, None if n is None else ints[1].to(DEV))
    for b in range(B):
        a = 0 if at is None else at[b] - 1
        for t in range(T + 1 if n is None else min(max(n[b], 0), T + 1)):
            if 0 <= a + t < C:
                for i in range(2):
                    reads[i][b, t] = ref.values(held[2 * i][b, a + t], held[2 * i + 1][b, a + t]).to(TYPES[dtype])
    for got, want in zip(greads, reads):
        got = got.cpu()
        assert torch.equal(got.isnan(), want.isnan()) and torch.equal(got.nan_to_num(0, 1e4, -1e4), want.nan_to_num(0, 1e4, -1e4))
    # a padded buffer's bytes beside the rows are as they were
    if layout == "padded":
        for x in gk4 + gv4 + tuple(gouts if out else ()) + tuple(greads):
            room = 32 if x.dtype == torch.uint8 else 16
            wide = x.as_strided((*x.shape[:-1], x.shape[-1] + 2 * room), x.stride(), x.storage_offset() - room)
            assert (wide[..., :room] == 77).all() and (wide[..., -room:] == 77).all()
    cache.close()


@pytest.mark.parametrize("layout", ["entries", "heads", "padded"])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("case", [
    # B, T, Hkv, D, C, at, n
    (1, 1, 1, 16, 1, [0], None),
    (1, 1, 4, 128, 5, [4], [1]),
    (3, 5, 2, 64, 9, [0, 4, 7], [5, 0, 3]),                    # the last runs past the end
    (3, 5, 2, 80, 9, [-2, 9, 2 ** 31 - 1], [5, 5, 5]),         # slots before the first, past the last
    (2, 7, 3, 96, 30, [3, 11], [-5, 900]),                     # counts outside 0 .. T
    (2, 65, 8, 112, 70, [2, 5], None),
    (2, 130, 5, 32, 131, None, None),
    (33, 2, 7, 48, 4, [i % 4 for i in range(33)], [i % 3 for i in range(33)]),
], ids=lambda c: "-".join(map(str, c[:5])))
def test_write_and_read(case, dtype, layout):
    written(*case, dtype, layout, True)


def test_write_without_values():
    written(2, 3, 2, 128, 8, [1, 5], [3, 2], "bf16", "heads", False)


def test_values_in_the_place_of_the_tokens():
    g = torch.Generator().manual_seed(4)
    k, v = (activations(g, 2, 40, 3, 64, dtype="fp16").to(DEV) for _ in range(2))
    want = [ref.quantise(x.cpu())[2].half() for x in (k, v)]
    cache = sp.Cache4(3, 3, 64, 40, dtype="fp16")
    k4, v4 = cache.new(2)
    cache.write(k, v, k4, v4, k_out=k, v_out=v)
    assert torch.equal(k.cpu(), want[0]) and torch.equal(v.cpu(), want[1])
    assert torch.equal(ref.values(*(x.cpu() for x in k4)).half(), want[0])
    # written once more they are the same
    codes = k4[0].clone()
    cache.write(k, v, k4, v4, k_out=k, v_out=v)
    assert torch.equal(k.cpu(), want[0]) and torch.equal(ref.values(*(x.cpu() for x in k4)).half(), want[0]) and codes.shape
    cache.close()


# ---------------------------------------------------------------------------
def held_entries(g, B, C, Hkv, D):
    """Codes and scales of what normal numbers of different size give."""
    x = torch.randn(B, C, Hkv, D, generator=g) * (0.5 + 2 * torch.rand(1, 1, Hkv, 1, generator=g))
    codes, scales, _ = ref.quantise(x.bfloat16())
    return codes, scales


def make(seed, B, T, Hq, Hkv, D, C, lens, dtype, garbage=True):
    """CPU tensors; slots that are not in use hold NaN scales."""
    g = torch.Generator().manual_seed(seed)
    q = (1.5 * torch.randn(B, T, Hq, D, generator=g)).to(TYPES[dtype])
    k4, v4 = held_entries(g, B, C, Hkv, D), held_entries(g, B, C, Hkv, D)
    if garbage:
        for b in range(B):
            for x in (k4, v4):
                x[1][b, max(0, lens[b]):] = 255
    return q, k4, v4, torch.tensor(lens, dtype=torch.int32)


def run(q, k4, v4, lens, layout="entries", causal=True, scale=None, other=None, stream=None, cache=None):
    B, T, Hq, D = q.shape
    C, Hkv = k4[0].shape[1:3]
    name = "bf16" if q.dtype == torch.bfloat16 else "fp16"
    own = cache or sp.Cache4(Hq, Hkv, D, C, max_T=T, dtype=name)
    out, lse = place(torch.full_like(q, 7.0), layout), torch.full((B, T, Hq), 7.0, device=DEV)
    more = {} if other is None else dict(other_out=place(other[0], layout), other_lse=other[1].to(DEV))
    own.attend(place(q, layout), tuple(place(x, layout) for x in k4), tuple(place(x, layout) for x in v4), lens.to(DEV), out,
               lse=lse, causal=causal, scale=scale, **more)
    torch.cuda.synchronize()
    assert own.status() == sp.SP_OK
    if cache is None:
        own.close()
    return out.cpu(), lse.cpu()


def check(q, k4, v4, lens, got, causal=True, scale=None, other=None):
    want, wlse, tol, lse_tol = ref.attend(q, ref.values(*k4), ref.values(*v4), lens, causal, scale, other)
    out, lse = got[0].double(), got[1].double()
    empty = wlse == -math.inf
    assert torch.equal(lse.isneginf(), empty) and (out[empty] == 0).all()
    err = (out - want).abs()
    assert (err <= tol).all(), f"out: {(err / tol).max()} of its bound"
    err = (lse - wlse).abs()[~empty]
    assert (err <= lse_tol[~empty]).all(), f"lse: {(err / lse_tol[~empty]).max()} of its bound"


CASES = [
    # B, T, Hq, Hkv, D, C, lens
    (1, 1, 1, 1, 16, 1, [1]),
    (1, 1, 4, 2, 128, 5, [3]),
    (2, 1, 12, 4, 128, 300, [300, 1]),
    (4, 1, 3, 1, 64, 128, [128, 127, 0, 17]),
    (3, 1, 8, 1, 128, 700, [700, 16, 15]),
    (5, 2, 8, 2, 128, 257, [257, 256, 130, 2, 1]),
    (4, 5, 6, 2, 64, 140, [140, 133, 3, 0]),                      # fewer entries than tokens
    (2, 8, 16, 2, 128, 200, [200, 131]),                          # 64 rows of a head
    (3, 3, 4, 4, 80, 90, [90, 41, 3]),
    (2, 4, 8, 8, 96, 64, [64, 7]),
    (2, 2, 5, 5, 32, 20, [20, 19]),
    (2, 3, 12, 3, 112, 150, [129, 150]),
    (2, 3, 15, 3, 48, 150, [-3, 1000]),                           # lengths outside the cache
    (40, 1, 6, 2, 128, 33, [i % 34 for i in range(40)]),
    (16, 6, 24, 3, 64, 150, [9 * i + 6 for i in range(16)]),      # 48 rows
    (3, 7, 9, 3, 128, 99, [99, 98, 6]),                           # 21 rows
    (2, 3, 9, 1, 64, 400, [400, 33]),                             # 27 rows
    (1, 32, 16, 2, 128, 64, [40]),                                # 256 rows of one head
    (2, 1, 200, 1, 64, 140, [140, 3]),                            # 200 query heads on one
]


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(map(str, c[:6])))
def test_attend_matches_the_definition(case, dtype):
    x = make(11, *case, dtype)
    check(*x, run(*x))


@pytest.mark.parametrize("layout", ["heads", "padded"])
@pytest.mark.parametrize("D", [64, 80, 112, 128])
def test_attend_on_other_layouts(layout, D):
    x = make(12, 3, 2, 6, 3, D, 70, [70, 33, 2], "bf16")
    check(*x, run(*x, layout=layout))


@pytest.mark.parametrize("G", [1, 5, 8, 9, 16, 17, 24, 25, 32, 33, 40, 48, 50, 64, 65])
@pytest.mark.parametrize("D", [64, 128])
def test_every_number_of_query_heads(G, D):
    x = make(13, 2, 1, 2 * G, 2, D, 260, [260, 31], "bf16")
    check(*x, run(*x))


def test_all_entries_seen():
    x = make(14, 3, 4, 8, 2, 128, 90, [90, 17, 0], "bf16")
    check(*x, run(*x, causal=False), causal=False)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_joined_with_other_attention(dtype):
    q, k4, v4, lens = make(15, 4, 3, 8, 2, 64, 150, [150, 2, 0, 77], dtype)
    g = torch.Generator().manual_seed(16)
    other = torch.randn(4, 3, 8, 64, generator=g).to(q.dtype), 4 * torch.randn(4, 3, 8, generator=g)
    other[1][0, 0, :3], other[1][2, :, 5] = -math.inf, -math.inf
    other[0][0, 0, :3], other[0][2, :, 5] = math.nan, math.inf        # of no weight
    other[1][3, 1, 0], other[1][3, 1, 1] = 300.0, -300.0
    check(q, k4, v4, lens, run(q, k4, v4, lens, other=other), other=other)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("T,Hq,C", [(1, 32, 40), (4, 40, 40), (1, 32, 2000)], ids=str)
def test_parts_are_weighed_by_unrounded_sums(T, Hq, C, dtype):
    """Values of nothing beside other attention of 1: what comes out is the weight."""
    q, k4, v4, lens = make(42, 40, T, Hq, 4, 64, C, [2 + b for b in range(39)] + [C], dtype)
    v4[0][:] = 0
    lse = ref.attend(q, ref.values(*k4), ref.values(*v4), lens, scale=0.02)[1]
    lse = torch.where(lse.isfinite(), lse, 0.0)
    other = torch.ones_like(q), (lse + torch.linspace(-3, 3, Hq)).float()
    check(q, k4, v4, lens, run(q, k4, v4, lens, scale=0.02, other=other), scale=0.02, other=other)


@pytest.mark.parametrize("T,Hq,D", [(1, 6, 128), (5, 10, 64), (1, 6, 64), (4, 40, 128), (9, 42, 64)], ids=str)
def test_joined_in_place(T, Hq, D):
    """Into the tensors of what is joined, by calls of other lengths one after the other:
    sequences without entries beside some that are cut up between the workers."""
    cache = sp.Cache4(Hq, 2, D, 900, max_T=T)
    for i, lens in enumerate(([900, 5, 0], [0, 900, 70], [40, 0, 0], [0, 0, 0], [700, 900, 800])):
        q, k4, v4, lens = make(17 + i, 3, T, Hq, 2, D, 900, lens, "bf16")
        g = torch.Generator().manual_seed(18 + i)
        other = torch.randn(3, T, Hq, D, generator=g).bfloat16(), torch.randn(3, T, Hq, generator=g)
        out, lse = other[0].to(DEV), other[1].to(DEV)
        on = [tuple(y.to(DEV) for y in x) for x in (k4, v4)]
        cache.attend(q.to(DEV), *on, lens.to(DEV), out, lse=lse, other_out=out, other_lse=lse)
        check(q, k4, v4, lens, (out.cpu(), lse.cpu()), other=other)
        check(q, k4, v4, lens, run(q, k4, v4, lens, cache=cache))
    cache.close()


@pytest.mark.parametrize("layout", ["entries", "heads"])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(map(str, c[:6])))
def test_the_same_sequences_in_a_larger_cache(case, layout):
    """Where blocks share out the tiles of all sequences, not those of one."""
    B, T, Hq, Hkv, D, _, lens = case
    x = make(11, B, T, Hq, Hkv, D, 1100, lens, "bf16")
    check(*x, run(*x, layout=layout))


@pytest.mark.parametrize("layout", ["entries", "heads"])
@pytest.mark.parametrize("Hq,Hkv", [(7, 7), (40, 20), (150, 150), (400, 200), (480, 60), (500, 500)])
def test_numbers_of_heads(Hq, Hkv, layout):
    """Workers that are left over where so many walk side by side; more heads than workers."""
    x = make(35, 3, 1, Hq, Hkv, 16, 800, [800, 33, 401], "bf16")
    check(*x, run(*x, layout=layout))
    if Hq < 500:
        x = make(36, 2, 9, Hq, Hkv, 16, 80, [80, 77], "bf16")
        check(*x, run(*x, layout=layout))


@pytest.mark.parametrize("C", [768, 769])
@pytest.mark.parametrize("T,Hq,D", [(1, 6, 128), (4, 4, 112), (2, 14, 128), (1, 12, 64), (5, 6, 64), (3, 6, 32)], ids=str)
def test_every_number_of_tiles(T, Hq, D, C):
    """Fewer tiles than a block's warps, as many, more; joined in place."""
    lens = [0, 1, 31, 32, 33, 64, 65, 96, 97, 128, 129, 160, 161, 224, 257, 767, 768]
    q, k4, v4, lens = make(31, len(lens), T, Hq, 2, D, C, lens, "bf16")
    check(q, k4, v4, lens, run(q, k4, v4, lens))
    g = torch.Generator().manual_seed(32)
    other = torch.randn(q.shape, generator=g).bfloat16(), 4 * torch.randn(q.shape[:3], generator=g)
    cache = sp.Cache4(Hq, 2, D, C, max_T=T)
    out, lse = other[0].to(DEV), other[1].to(DEV)
    cache.attend(q.to(DEV), *(tuple(y.to(DEV) for y in x) for x in (k4, v4)), lens.to(DEV), out, lse=lse, other_out=out,
                 other_lse=lse)
    check(q, k4, v4, lens, (out.cpu(), lse.cpu()), other=other)
    cache.close()


@pytest.mark.parametrize("T,Hq,D", [(1, 6, 128), (2, 12, 128), (3, 6, 64), (4, 10, 64)], ids=str)
@pytest.mark.parametrize("B", [1, 8, 20, 100])
def test_few_and_many_parts_of_a_row(B, T, Hq, D):
    x = make(33, B, T, Hq, 2, D, 1600, [1600 - 11 * b for b in range(B)], "bf16")
    check(*x, run(*x))


@pytest.mark.parametrize("T,Hq", [(1, 4), (2, 8), (7, 50)], ids=str)
@pytest.mark.parametrize("D", [64, 128])
def test_a_nan_value_of_no_weight_in_a_short_cache(T, Hq, D):
    """As in a long cache, where the parts of one block meet."""
    nan_beside_all_of_the_weight(T, Hq, D, 600)


@pytest.mark.parametrize("T,Hq", [(1, 4), (2, 8), (4, 16), (7, 50)], ids=str)
@pytest.mark.parametrize("D", [64, 128])
def test_a_nan_value_stays_where_its_weight_vanishes(T, Hq, D):
    """A value's group is NaN; its weight beside another entry's, 128 nats above, is
    nothing in 32 bits, whatever workers have the two."""
    nan_beside_all_of_the_weight(T, Hq, D, 5000)


def nan_beside_all_of_the_weight(T, Hq, D, C):
    q = torch.ones(2, T, Hq, D, dtype=torch.float16)
    k4 = torch.zeros(2, C, 2, D // 2, dtype=torch.uint8), torch.full((2, C, 2, D // 16), 120, dtype=torch.uint8)
    v4 = torch.full((2, C, 2, D // 2), 0x22, dtype=torch.uint8), torch.full((2, C, 2, D // 16), 120, dtype=torch.uint8)
    k4[0][:, C - T - 1] = 0x77
    k4[1][:, C - T - 1] = 144              # 6 * 16 an element
    v4[1][0, 3, 0, 1] = 255
    lens = torch.tensor([C, C], dtype=torch.int32)
    out, lse = run(q, k4, v4, lens, scale=1.0)
    assert out[0, :, :Hq // 2, 16:32].isnan().all()
    out[0, :, :Hq // 2, 16:32] = 1.0       # (code 2, as all values)
    assert (out == 1).all() and lse.isfinite().all()


@pytest.mark.parametrize("D,B,n", [(128, 1, 200_003), (64, 2, 70_001)])
def test_long_caches(D, B, n):
    x = make(19, B, 2, 3, 1, D, n, [n - 5] * B, "bf16", garbage=False)
    check(*x, run(*x))


def test_more_units_than_the_gpu_holds():
    lens = [(7 * b) % 40 for b in range(1024)]
    x = make(20, 1024, 1, 4, 4, 32, 40, lens, "fp16")
    check(*x, run(*x))


@pytest.mark.parametrize("B", [5, 31, 127, 128, 129, 131])
@pytest.mark.parametrize("T,Hq", [(1, 2), (3, 12)], ids=str)
def test_numbers_of_sequences(B, T, Hq):
    lens = [(37 * b) % 200 if b % 3 else 0 for b in range(B)]
    x = make(34, B, T, Hq, 2, 64, 800, lens, "bf16")
    check(*x, run(*x))


def test_one_entry_with_all_of_the_weight_comes_out_exactly():
    q, k4, v4, lens = make(21, 2, 1, 4, 2, 128, 500, [500, 333], "fp16")
    k4[1][:, 250] = 120                    # a scale of 2, above all others
    k4[0][:, 250] = 0x77                   # all 6
    q[:] = 4.0
    out, _ = run(q, k4, v4, lens, scale=1.0)
    want = ref.values(*v4)[:, 250].half().repeat_interleave(2, 1)
    assert torch.equal(out[:, 0], want)


def test_large_and_small_queries():
    """Rows of bf16 queries beyond half precision's range, and far below it."""
    q, k4, v4, lens = make(22, 2, 1, 6, 2, 128, 100, [100, 64], "bf16")
    for i, f in enumerate((1e30, 1e-30, 1.0, 1e36, 1e-36, 0.0)):
        q[:, :, i] *= f
    q[1, 0, 2, 5] = 3e30                   # one element far above its row
    for scale in (1e-30, 1e28, 1.0):
        s = scale * (q.double().unsqueeze(3) * ref.values(*k4)[:, None, :, [0, 0, 0, 1, 1, 1]].transpose(2, 3)).sum(-1)
        fine = s.abs().amax((1, 3)) < 1e3  # (others are one entry's, by a wide margin or a narrow one)
        want, wlse, tol, lse_tol = ref.attend(q, ref.values(*k4), ref.values(*v4), lens, True, scale)
        out, lse = run(q, k4, v4, lens, scale=scale)
        assert ((out.double() - want).abs() <= tol)[:, 0][fine].all()
        assert ((lse.double() - wlse).abs() <= lse_tol)[:, 0][fine].all()
        assert fine.any()


@pytest.mark.parametrize("T,Hq,C", [(1, 4, 700), (1, 4, 3000), (5, 6, 3000), (9, 8, 3000)], ids=str)
@pytest.mark.parametrize("power", [10, 20, 22, 26, 30, 60, 100])
def test_scores_of_any_size(T, Hq, C, power):
    """Equal scores of 2^power and more give the mean of the values, one score above
    them its value, however far apart FP32 numbers of that size are."""
    g = torch.Generator().manual_seed(41)
    q = torch.full((2, T, Hq, 64), 2.0 ** (power - 11), dtype=torch.bfloat16)
    k4 = torch.full((2, C, 2, 32), 0x77, dtype=torch.uint8), torch.full((2, C, 2, 4), 120, dtype=torch.uint8)  # 6 * 1
    _, v4 = held_entries(g, 2, C, 2, 64), held_entries(g, 2, C, 2, 64)
    lens = torch.tensor([C, C // 2], dtype=torch.int32)
    out, lse = run(q, k4, v4, lens, causal=False, scale=1.0)
    v = ref.values(*v4)
    for b in range(2):
        mean, size = v[b, :lens[b]].mean(0).repeat_interleave(Hq // 2, 0), v[b, :lens[b]].abs().mean(0).repeat_interleave(Hq // 2, 0)
        tol = size * (2 * 2.0 ** -11 + 2.0 ** -16) + mean.abs() * 2.0 ** -8
        assert ((out[b].double() - mean).abs() <= tol).all()
    want = 64 * 6 * 2.0 ** (power - 11) + torch.log(lens.double())
    assert ((lse.double() - want.view(2, 1, 1)).abs() <= 2.0 ** -22 * want.view(2, 1, 1)).all()
    if power >= 20:                        # (others' scores are half of it, more than 2^18 less)
        k4[1][:, 300] = 128                # twice the scale
        out, _ = run(q, k4, v4, lens, causal=False, scale=1.0)
        assert torch.equal(out, v[:, 300].bfloat16().repeat_interleave(Hq // 2, 1).unsqueeze(1).expand(out.shape))


def test_nan_entries():
    """A NaN is that of the rows that see it, and of its 16 elements in a value."""
    T, n = 4, 60
    q, k4, v4, lens = make(23, 3, T, 4, 2, 64, 64, [n, n, n], "bf16")
    k4[1][0, n - 2, 1, 3] = 255            # seen by the last two tokens
    v4[1][1, n - 3, 0, 2] = 255            # by the last three
    v4[1][2, 7, 1] = 255                   # by all
    out, lse = run(q, k4, v4, lens)
    nan = torch.zeros(out.shape, dtype=torch.bool)
    nan[0, T - 2:, 2:] = True
    nan[1, T - 3:, :2, 32:48] = True
    nan[2, :, 2:] = True
    assert torch.equal(out.isnan(), nan)
    assert torch.equal(lse.isnan(), nan.all(-1) & (torch.arange(3) == 0).view(3, 1, 1))
    clean = [tuple(torch.where(y == 255, 56, y) if i else y for i, y in enumerate(x)) for x in (k4, v4)]
    want, _, tol, _ = ref.attend(q, *(ref.values(*x) for x in clean), lens)
    mixed = nan | (torch.arange(3) == 0).view(3, 1, 1, 1) & nan
    assert ((out.double() - want).abs() <= tol)[~mixed].all()


def test_nan_and_infinite_queries():
    q, k4, v4, lens = make(24, 1, 1, 4, 2, 128, 40, [40], "bf16")
    q[0, 0, 1, 9], q[0, 0, 2, 100] = math.nan, math.inf
    out, lse = run(q, k4, v4, lens)
    assert out[0, 0, 1:3].isnan().all() and lse[0, 0, 1:3].isnan().all()
    q[0, 0, 1:3] = 0
    check(*(x[:, :, [0, 3]] if i == 0 else x for i, x in enumerate((q, k4, v4, lens))), (out[:, :, [0, 3]], lse[:, :, [0, 3]]))


def test_results_repeat():
    """Bit for bit, whichever block comes last."""
    x = make(25, 3, 1, 8, 2, 128, 5000, [5000, 100, 3333], "bf16", garbage=False)
    cache = sp.Cache4(8, 2, 128, 5000)
    first = run(*x, cache=cache)
    for _ in range(20):
        again = run(*x, cache=cache)
        assert torch.equal(first[0].view(torch.int16), again[0].view(torch.int16)) and torch.equal(first[1], again[1])
    cache.close()


# ---------------------------------------------------------------------------
def test_a_decode_as_it_is_used():
    """A shared prompt in 16 bits, entries of each step written and attended to in 4
    bits, joined; then all of them back in 16 bits for the other operators."""
    B, T, Hq, Hkv, D, C, P = 3, 2, 8, 2, 64, 40, 90
    g = torch.Generator(device=DEV).manual_seed(26)
    new = lambda *s: torch.randn(*s, generator=g, device=DEV).bfloat16()     # noqa: E731
    pk, pv = new(P, Hkv, D), new(P, Hkv, D)
    prefix, cache = sp.Cache(B, Hq, Hkv, D, 1, max_T=T), sp.Cache4(Hq, Hkv, D, C, max_T=T)
    none, unused = torch.zeros(B, dtype=torch.int32, device=DEV), new(B, 1, Hkv, D)
    k4, v4 = cache.new(B)
    lens = torch.tensor([0, 3, 1], dtype=torch.int32, device=DEV)
    k, v = (torch.zeros(B, C, Hkv, D, dtype=torch.bfloat16) for _ in range(2))     # what the caches stand for
    for step in range(5):
        q, nk, nv = new(B, T, Hq, D), new(B, T, Hkv, D), new(B, T, Hkv, D)
        n = torch.randint(1, T + 1, (B,), generator=g, device=DEV, dtype=torch.int32)
        cache.write(nk, nv, k4, v4, at=lens, n=n)
        for b in range(B):
            for held, x in ((k, nk), (v, nv)):
                at = int(lens[b])
                held[b, at:at + int(n[b])] = ref.quantise(x[b, :int(n[b])].cpu())[2].bfloat16()
        lens += n
        out, lse = torch.empty_like(q), torch.empty(B, T, Hq, device=DEV)
        prefix.attend(q, unused, unused, none, out, prefix_k=pk, prefix_v=pv, lse=lse)
        other = out.cpu(), lse.cpu()
        cache.attend(q, k4, v4, lens, out, lse=lse, other_out=out, other_lse=lse)
        want, wlse, tol, lse_tol = ref.attend(q.cpu(), k.double(), v.double(), lens.cpu(), other=other)
        assert ((out.cpu().double() - want).abs() <= tol).all() and ((lse.cpu().double() - wlse).abs() <= lse_tol).all()
        # the same attention in one piece, but for the rounding of the part over the prompt
        whole, _, _, mass, size = serving_ref.attend(q.cpu(), k, v, lens.cpu(), pk.cpu(), pv.cpu())
        assert ((out.cpu().double() - whole).abs() <= tol + 2.0 ** -7 * mass).all()
    back_k, back_v = (torch.full((B, C, Hkv, D), 9.0, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    cache.read(k4, v4, back_k, back_v, n=lens)
    for b in range(B):
        n = int(lens[b])
        assert torch.equal(back_k[b, :n].cpu(), k[b, :n]) and torch.equal(back_v[b, :n].cpu(), v[b, :n])
        assert (back_k[b, n:] == 9).all()
    cache.close()
    prefix.close()


@pytest.mark.parametrize("layout", ["entries", "heads"])
@pytest.mark.parametrize("T,Hq,C", [(1, 4, 200), (1, 4, 1000), (4, 12, 1000)], ids=str)
def test_back_to_back_calls_see_each_others_results(T, Hq, C, layout):
    """Writes over the same slots, attention in two parts, reads, nothing between them."""
    B, Hkv, D, steps = 24, 2, 128, 12
    g = torch.Generator(device=DEV).manual_seed(37)
    new = lambda *s: torch.randn(*s, generator=g, device=DEV).bfloat16()     # noqa: E731
    cache = sp.Cache4(Hq, Hkv, D, C, max_T=T)
    k4, v4 = (tuple(place(y, layout) for y in held_entries(torch.Generator().manual_seed(s), B, C, Hkv, D)) for s in (38, 39))
    lens = torch.randint(T, C + 1, (B,), generator=g, device=DEV, dtype=torch.int32)
    at, half = lens - T, lens // 2
    k, v, q = new(steps, B, T, Hkv, D), new(steps, B, T, Hkv, D), new(steps, B, T, Hq, D)

    def calls(wait):
        out, first = torch.zeros_like(q), torch.zeros_like(q)
        lse, lse1 = (torch.zeros(steps, B, T, Hq, device=DEV) for _ in range(2))
        kb, vb = torch.zeros_like(k), torch.zeros_like(v)
        torch.cuda.synchronize()
        for i in range(steps):
            for call in (lambda: cache.write(k[i], v[i], k4, v4, at=at),
                         lambda: cache.attend(q[i], k4, v4, half, first[i], lse=lse1[i], causal=False),
                         lambda: cache.attend(q[i], k4, v4, lens, out[i], lse=lse[i], other_out=first[i], other_lse=lse1[i]),
                         lambda: cache.read(k4, v4, kb[i], vb[i], at=at)):
                call()
                if wait:
                    torch.cuda.synchronize()
        torch.cuda.synchronize()
        return [x.cpu() for x in (out, first, lse, lse1, kb, vb)]

    want = calls(True)
    for _ in range(3):
        for x, y in zip(calls(False), want):
            assert torch.equal(x, y)
    cache.close()


@pytest.mark.parametrize("T,Hq", [(1, 8), (5, 24)], ids=str)
def test_handles_on_streams_at_once(T, Hq):
    """Two 4-bit caches and one in 16 bits, each on a stream of its own."""
    B, Hkv, D, C = 6, 2, 128, 6000
    x = [make(43 + i, B, T, Hq, Hkv, D, C, [C - 900 * b - i for b in range(B)], "bf16", garbage=False) for i in range(2)]
    on = [[q.to(DEV), tuple(y.to(DEV) for y in k4), tuple(y.to(DEV) for y in v4), lens.to(DEV)] for q, k4, v4, lens in x]
    caches, streams = [sp.Cache4(Hq, Hkv, D, C, max_T=T) for _ in range(2)], [torch.cuda.Stream() for _ in range(3)]
    outs = [[torch.zeros_like(o[0]) for _ in range(15)] for o in on]
    own = sp.Cache(B, Hq, Hkv, D, 1000, max_T=T)
    g = torch.Generator(device=DEV).manual_seed(45)
    k, v = (torch.randn(B, 1000, Hkv, D, generator=g, device=DEV).bfloat16() for _ in range(2))
    lens16, outs16 = torch.full((B,), 1000, dtype=torch.int32, device=DEV), [torch.zeros_like(on[0][0]) for _ in range(15)]
    torch.cuda.synchronize()
    for i in range(15):
        for cache, o, out, stream in zip(caches, on, outs, streams):
            cache.attend(o[0], o[1], o[2], o[3], out[i], stream=stream)
        own.attend(on[0][0], k, v, lens16, outs16[i], stream=streams[2])
    torch.cuda.synchronize()
    for cache, o, out, y in zip(caches, on, outs, x):
        alone = run(*y)[0]
        assert cache.status() == sp.SP_OK and all(torch.equal(z.cpu(), alone) for z in out)
        cache.close()
    assert own.status() == sp.SP_OK and all(torch.equal(z, outs16[0]) for z in outs16)
    own.close()


def test_replayed_from_graphs_on_another_stream():
    """Two graphs on one handle, replayed in turn on new inputs."""
    x = [make(27 + i, 2, 1, 4, 2, 128, 3000, [3000, 40 + i], "bf16") for i in range(3)]
    cache = sp.Cache4(4, 2, 128, 3000)
    stream = torch.cuda.Stream()
    on = [t.clone() for t in (x[0][0].to(DEV), *(y.to(DEV) for y in x[0][1] + x[0][2]), x[0][3].to(DEV))]
    out, lse = torch.zeros(2, 1, 4, 128, dtype=torch.bfloat16, device=DEV), torch.zeros(2, 1, 4, device=DEV)
    out2 = torch.zeros_like(out)
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    torch.cuda.synchronize()
    for graph, o in zip(graphs, (out, out2)):
        with torch.cuda.graph(graph, stream=stream):
            cache.attend(on[0], (on[1], on[2]), (on[3], on[4]), on[5], o, lse=lse)
    for i in (1, 2, 0):
        for to, new in zip(on, (x[i][0], *x[i][1], *x[i][2], x[i][3])):
            to.copy_(new)
        with torch.cuda.stream(stream):
            stream.wait_stream(torch.cuda.default_stream())
            graphs[0].replay()
            graphs[1].replay()
        torch.cuda.synchronize()
        check(*x[i], (out.cpu(), lse.cpu()))
        assert torch.equal(out, out2)
    cache.close()


def test_refusals():
    cache = sp.Cache4(4, 2, 64, 8, max_T=2)
    k4, v4 = cache.new(2)
    q = torch.zeros(2, 2, 4, 64, dtype=torch.bfloat16, device=DEV)
    k = torch.zeros(2, 3, 2, 64, dtype=torch.bfloat16, device=DEV)
    lens, out = torch.zeros(2, dtype=torch.int32, device=DEV), torch.empty_like(q)
    with pytest.raises(ValueError, match="k4"):
        cache.attend(q, None, v4, lens, out)
    with pytest.raises(ValueError, match="shape"):
        cache.attend(q, (k4[0], v4[0]), v4, lens, out)
    with pytest.raises(ValueError, match="one without"):
        cache.attend(q, k4, v4, lens, out, other_out=out)
    with pytest.raises(sp.SpikeProjError) as e:
        cache.attend(q.repeat(1, 2, 1, 1), k4, v4, lens, out.repeat(1, 2, 1, 1))
    assert e.value.status == sp.SP_ERANGE
    with pytest.raises(sp.SpikeProjError) as e:
        cache.write(k, k.clone(), k4, k4)
    assert e.value.status == sp.SP_EINVAL
    with pytest.raises(ValueError, match="expected"):
        cache.write(k.half(), k, k4, v4)
    with pytest.raises(ValueError, match="k_out"):
        cache.read(k4, v4, None, k)
    cache.close()
