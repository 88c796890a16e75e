"""The 4-bit cache without a GPU: what its entry points and its binding refuse, its
launches on fake devices, and the plain implementations that the GPU tests compare
with, pinned by hand and by laws."""
import ctypes
import itertools
import math

import pytest
import torch

import cache4_ref as ref
import serving_ref
from paper_2606_03026_gb300 import spikeproj as sp
from test_cache_binding_cpu import Tensor, library                # noqa: F401  (a fixture)
from test_host_cpu import FAKE, lib                               # noqa: F401  (a fixture)

B, T, HQ, HKV, D, C = 2, 3, 8, 2, 64, 32
U8, I32, F32, BF16 = torch.uint8, torch.int32, torch.float32, torch.bfloat16


def held(name, at):
    return {name + "_codes": at, name + "_batch": C * HKV * D // 2, name + "_entry": HKV * D // 2, name + "_head": D // 2,
            name + "_scales": at + (1 << 20), name + "_scales_batch": C * HKV * D // 16, name + "_scales_entry": HKV * D // 16,
            name + "_scales_head": D // 16}


def rows(name, heads=HKV):
    return {name + "_batch": T * heads * D, name + "_token": heads * D, name + "_head": D}


def write_call(**over):
    f = dict(k=FAKE, v=2 * FAKE, **rows("k"), **rows("v"), **held("k4", 3 * FAKE), **held("v4", 4 * FAKE), at=FAKE, n=FAKE,
             k_out=5 * FAKE, v_out=6 * FAKE, **rows("k_out"), **rows("v_out"), B=B, T=T)
    return sp.SpWrite4(**{**f, **over})


def read_call(**over):
    f = dict(**held("k4", 3 * FAKE), **held("v4", 4 * FAKE), at=FAKE, n=FAKE, k_out=5 * FAKE, v_out=6 * FAKE, **rows("k_out"),
             **rows("v_out"), B=B, T=T)
    return sp.SpRead4(**{**f, **over})


def attend_call(**over):
    f = dict(q=FAKE, **rows("q", HQ), **held("k4", 3 * FAKE), **held("v4", 4 * FAKE), lens=FAKE, out=2 * FAKE, **rows("out", HQ),
             lse=FAKE, other_out=5 * FAKE, **rows("other", HQ), other_lse=FAKE, B=B, T=T, causal=1, scale=0.125)
    return sp.SpAttend4(**{**f, **over})


def make(lib, max_T=T, Hq=HQ, Hkv=HKV, D=D, capacity=C, dtype=0):  # noqa: F811
    h = ctypes.c_void_p()
    return h, lib.spike_proj_cache4_create(ctypes.byref(h), max_T, Hq, Hkv, D, capacity, dtype, None)


@pytest.fixture
def cache(lib):                                                   # noqa: F811
    lib.fake_device(0)
    lib.fake_fail(b"")
    h, st = make(lib)
    assert st == sp.SP_OK
    yield h
    assert lib.spike_proj_cache4_destroy(h) == sp.SP_OK


@pytest.mark.parametrize("over, want", [
    (dict(max_T=0), sp.SP_ERANGE), (dict(max_T=33), sp.SP_ERANGE), (dict(Hq=0), sp.SP_ERANGE), (dict(Hq=514), sp.SP_ERANGE),
    (dict(Hq=7), sp.SP_EINVAL), (dict(Hkv=0), sp.SP_EINVAL), (dict(D=8), sp.SP_ERANGE), (dict(D=144), sp.SP_ERANGE),
    (dict(D=72), sp.SP_EALIGN), (dict(capacity=0), sp.SP_ERANGE), (dict(capacity=(1 << 24) + 1), sp.SP_ERANGE),
    (dict(dtype=2), sp.SP_EINVAL),
], ids=str)
def test_a_cache_is_refused(lib, over, want):                     # noqa: F811
    h, st = make(lib, **over)
    assert st == want and not h.value
    # the library itself says so before it looks for a device
    assert make(sp.lib(), **over)[1] == want


KV_NULL = [name + part for name in ("k4", "v4") for part in ("_codes", "_scales")]
KV_BAD = [*[({name + "_codes": 3 * FAKE + 8}, sp.SP_EALIGN) for name in ("k4", "v4")],
          *[({name + "_scales": 3 * FAKE + 2}, sp.SP_EALIGN) for name in ("k4", "v4")],
          *[({name + d: 72}, sp.SP_EALIGN) for name in ("k4", "v4") for d in ("_batch", "_entry", "_head")],
          *[({name + d: 6}, sp.SP_EALIGN) for name in ("k4", "v4") for d in ("_scales_batch", "_scales_entry", "_scales_head")]]


@pytest.mark.parametrize("over, want", [
    *[({name: None}, sp.SP_EINVAL) for name in ("k", "v", "k_out", "v_out", *KV_NULL)], *KV_BAD,
    *[({name: 3 * FAKE + 8}, sp.SP_EALIGN) for name in ("k", "v", "k_out", "v_out")],
    *[({name: 3 * FAKE + 2}, sp.SP_EALIGN) for name in ("at", "n")],
    *[({name + d: 68}, sp.SP_EALIGN) for name in ("k", "v", "k_out", "v_out") for d in ("_batch", "_token", "_head")],
    *[({name + d: x}, sp.SP_EALIGN) for name in ("k_out", "v_out") for d in ("_batch", "_token", "_head") for x in (0, 32, -32)],
    *[({name + d: 0}, sp.SP_EALIGN) for name in ("k4", "v4") for d in ("_batch", "_entry", "_scales_head")],
    (dict(v4_codes=3 * FAKE), sp.SP_EINVAL), (dict(v4_scales=3 * FAKE + (1 << 20)), sp.SP_EINVAL),
    (dict(v_out=5 * FAKE), sp.SP_EINVAL), (dict(k_out=2 * FAKE), sp.SP_EINVAL), (dict(v_out=FAKE), sp.SP_EINVAL),
    (dict(k_out=FAKE, k_out_token=2 * HKV * D), sp.SP_EINVAL), (dict(v_out=2 * FAKE, v_out_head=2 * D), sp.SP_EINVAL),
    (dict(B=0), sp.SP_EINVAL), (dict(T=0), sp.SP_EINVAL), (dict(B=1025), sp.SP_ERANGE), (dict(T=1 << 27), sp.SP_ERANGE),
], ids=str)
def test_a_write_call_is_refused(lib, cache, over, want):         # noqa: F811
    lib.fake_launches()
    assert lib.spike_proj_cache4_write(cache, ctypes.byref(write_call(**over)), None) == want
    assert lib.fake_launches() == 0


@pytest.mark.parametrize("over, want", [
    *[({name: None}, sp.SP_EINVAL) for name in ("k_out", "v_out", *KV_NULL)], *KV_BAD,
    *[({name: 3 * FAKE + 8}, sp.SP_EALIGN) for name in ("k_out", "v_out")],
    *[({name: 3 * FAKE + 2}, sp.SP_EALIGN) for name in ("at", "n")],
    *[({name + d: x}, sp.SP_EALIGN) for name in ("k_out", "v_out") for d in ("_batch", "_token", "_head") for x in (68, 0, -32)],
    (dict(v_out=5 * FAKE), sp.SP_EINVAL),
    (dict(B=0), sp.SP_EINVAL), (dict(T=-1), sp.SP_EINVAL), (dict(B=1025), sp.SP_ERANGE), (dict(T=1 << 27), sp.SP_ERANGE),
], ids=str)
def test_a_read_call_is_refused(lib, cache, over, want):          # noqa: F811
    lib.fake_launches()
    assert lib.spike_proj_cache4_read(cache, ctypes.byref(read_call(**over)), None) == want
    assert lib.fake_launches() == 0


@pytest.mark.parametrize("over, want", [
    *[({name: None}, sp.SP_EINVAL) for name in ("q", "lens", "out", "other_out", "other_lse", *KV_NULL)], *KV_BAD,
    *[({name: 3 * FAKE + 8}, sp.SP_EALIGN) for name in ("q", "out", "other_out")],
    *[({name: 3 * FAKE + 2}, sp.SP_EALIGN) for name in ("lens", "lse", "other_lse")],
    *[({name + d: 68}, sp.SP_EALIGN) for name in ("q", "out", "other") for d in ("_batch", "_token", "_head")],
    *[({"out" + d: x}, sp.SP_EALIGN) for d in ("_batch", "_token", "_head") for x in (0, 32, -32)],
    (dict(out=FAKE), sp.SP_EINVAL), (dict(other_out=2 * FAKE, other_head=2 * D), sp.SP_EINVAL),
    (dict(B=0), sp.SP_EINVAL), (dict(T=0), sp.SP_EINVAL), (dict(B=1025), sp.SP_ERANGE), (dict(T=T + 1), sp.SP_ERANGE),
    *[(dict(scale=x), sp.SP_EINVAL) for x in (0.0, -1.0, math.inf, math.nan)],
], ids=str)
def test_an_attend_call_is_refused(lib, cache, over, want):       # noqa: F811
    lib.fake_launches()
    assert lib.spike_proj_cache4_attend(cache, ctypes.byref(attend_call(**over)), None) == want
    assert lib.fake_launches() == 0


def test_calls_at_the_limits(lib, cache):                         # noqa: F811
    writes = [dict(), dict(at=None, n=None), dict(k_out=None, v_out=None), dict(k_out=FAKE, v_out=2 * FAKE),
              dict(B=1, k_batch=3, k4_batch=1, k4_scales_batch=1, v_out_batch=0), dict(T=1, k_token=1, v_out_token=0),
              dict(k_head=0, v_token=0), dict(k4_entry=-HKV * D // 2), dict(k_out_head=-D, k_out_token=-HKV * D)]
    for over in writes:
        assert lib.spike_proj_cache4_write(cache, ctypes.byref(write_call(**over)), None) == sp.SP_OK, over
    for over in (dict(), dict(at=None, n=None), dict(k4_entry=0, v4_scales_batch=0), dict(T=1, k_out_token=0)):
        assert lib.spike_proj_cache4_read(cache, ctypes.byref(read_call(**over)), None) == sp.SP_OK, over
    for over in (dict(), dict(lse=None), dict(other_out=None, other_lse=None), dict(other_out=2 * FAKE), dict(causal=0),
                 dict(q_head=0, k4_batch=0), dict(T=1, q_token=1), dict(B=1, out_batch=0, other_batch=1)):
        assert lib.spike_proj_cache4_attend(cache, ctypes.byref(attend_call(**over)), None) == sp.SP_OK, over
    for call in (lib.spike_proj_cache4_write, lib.spike_proj_cache4_read, lib.spike_proj_cache4_attend):
        assert call(None, FAKE, None) == sp.SP_EINVAL and call(cache, None, None) == sp.SP_EINVAL
    assert lib.spike_proj_cache4_status(cache, None) == sp.SP_OK
    assert lib.spike_proj_cache4_status(None, None) == sp.SP_EINVAL
    assert lib.spike_proj_cache4_inject_fault(cache, sp.SP_FAULT_STALL) == sp.SP_OK
    assert lib.spike_proj_cache4_inject_fault(cache, sp.SP_FAULT_ABORT) == sp.SP_EINVAL
    assert lib.spike_proj_cache4_inject_fault(None, 0) == sp.SP_EINVAL
    assert lib.spike_proj_cache4_destroy(None) == sp.SP_OK


def test_a_handle_serves_its_own_device(lib, cache):              # noqa: F811
    lib.fake_device(1)
    lib.fake_launches()
    assert lib.spike_proj_cache4_write(cache, ctypes.byref(write_call()), None) == sp.SP_EDEVICE
    assert lib.spike_proj_cache4_read(cache, ctypes.byref(read_call()), None) == sp.SP_EDEVICE
    assert lib.spike_proj_cache4_attend(cache, ctypes.byref(attend_call()), None) == sp.SP_EDEVICE
    assert lib.fake_launches() == 0
    lib.fake_device(0)


def test_a_launch_that_fails_is_reported(lib, cache):             # noqa: F811
    large, st = make(lib, capacity=1024)    # (a short cache has no launch of a merge)
    assert st == sp.SP_OK
    for name, call in ((b"write4", lambda: lib.spike_proj_cache4_write(cache, ctypes.byref(write_call()), None)),
                       (b"read4", lambda: lib.spike_proj_cache4_read(cache, ctypes.byref(read_call()), None)),
                       (b"attend4", lambda: lib.spike_proj_cache4_attend(cache, ctypes.byref(attend_call()), None)),
                       (b"attend4", lambda: lib.spike_proj_cache4_attend(large, ctypes.byref(attend_call()), None)),
                       (b"merge4", lambda: lib.spike_proj_cache4_attend(large, ctypes.byref(attend_call()), None))):
        lib.fake_fail(name)
        assert call() == sp.SP_ECUDA
        lib.fake_fail(b"")
        assert call() == sp.SP_OK
    assert lib.spike_proj_cache4_destroy(large) == sp.SP_OK


@pytest.mark.parametrize("heads, B, capacity, launches", [(4, 1, 64, 1), (4, 1, 768, 1), (4, 1, 769, 2), (8, 152 * 4, 768, 1),
                                                          (8, 152 * 4 + 1, 768, 2), (17, 1, 64, 2)])
def test_a_short_cache_takes_one_launch(lib, heads, B, capacity, launches):  # noqa: F811
    h, st = make(lib, Hq=heads, Hkv=1, D=128, max_T=1, capacity=capacity)
    assert st == sp.SP_OK
    lib.fake_launches()
    strides = {x + s: n * 128 for x in ("q", "out") for s, n in (("_batch", heads), ("_token", heads), ("_head", 1))}
    kv = {x + "4" + s: n * 64 for x in "kv" for s, n in (("_batch", capacity), ("_entry", 1), ("_head", 1))}
    call = attend_call(T=1, B=B, other_out=None, other_lse=None, **strides, **kv)
    assert lib.spike_proj_cache4_attend(h, ctypes.byref(call), None) == sp.SP_OK
    assert lib.fake_launches() == launches
    assert lib.spike_proj_cache4_destroy(h) == sp.SP_OK


@pytest.mark.parametrize("heads, D, rows_kernel", [(8, 128, False), (9, 128, False), (16, 128, False), (17, 128, True), (16, 64, False), (17, 64, True),
                                                  (512, 16, True)])
def test_query_rows_decide_the_kernel(lib, heads, D, rows_kernel):  # noqa: F811
    h, st = make(lib, Hq=heads, Hkv=1, D=D, max_T=1, capacity=64)
    assert st == sp.SP_OK
    lib.fake_fail(b"attend4_rows")
    strides = {x + s: n * D for x in ("q", "out", "other") for s, n in (("_batch", heads), ("_token", heads), ("_head", 1))}
    kv = {x + "4" + s: n * D // 2 for x in "kv" for s, n in (("_batch", 64), ("_entry", 1), ("_head", 1))}
    sc = {x + "4_scales" + s: n * D // 16 for x in "kv" for s, n in (("_batch", 64), ("_entry", 1), ("_head", 1))}
    call = attend_call(T=1, **strides, **kv, **sc)
    assert lib.spike_proj_cache4_attend(h, ctypes.byref(call), None) == (sp.SP_ECUDA if rows_kernel else sp.SP_OK)
    lib.fake_fail(b"")
    assert lib.spike_proj_cache4_destroy(h) == sp.SP_OK


def test_a_call_of_too_many_tiles_is_refused(lib):                # noqa: F811
    # 1024 sequences and 512 heads of 2^17 entries each: 2^19 units of 2^12 + 2 tiles
    call = dict(B=1024, T=1, q_batch=512 * 16, q_token=512 * 16, q_head=16, out_batch=512 * 16, out_token=512 * 16, out_head=16,
                other_out=None, other_lse=None,
                **{x + "4" + s: n for x in "kv" for s, n in (("_batch", 8), ("_entry", 8), ("_head", 8), ("_scales_batch", 1),
                                                             ("_scales_entry", 1), ("_scales_head", 1))})
    for capacity, want in (((1 << 17) + 1, sp.SP_ERANGE), ((1 << 16), sp.SP_OK)):
        h, st = make(lib, Hq=512, Hkv=512, D=16, max_T=1, capacity=capacity)
        assert st == sp.SP_OK
        assert lib.spike_proj_cache4_attend(h, ctypes.byref(attend_call(**call)), None) == want
        assert lib.spike_proj_cache4_destroy(h) == sp.SP_OK


@pytest.mark.parametrize("cls, pack", [(sp.SpWrite4, sp._pack_write4), (sp.SpRead4, sp._pack_read4),
                                       (sp.SpAttend4, sp._pack_attend4)])
def test_calls_are_packed_as_their_structures(cls, pack):
    values = [0.5 if t is ctypes.c_float else 3 * i + 1 for i, (_, t) in enumerate(cls._fields_)]
    got = cls.from_buffer_copy(pack(*values))
    assert [getattr(got, name) for name, _ in cls._fields_] == values


# ---- the binding -----------------------------------------------------------------
@pytest.fixture
def bound(library):                                               # noqa: F811
    cache = sp.Cache4(HQ, HKV, D, C, max_T=T)
    cache.handle = 1                        # (nothing made one)
    library.calls.clear()
    yield cache
    cache.handle = None


def pair4(device=0):
    return Tensor((B, C, HKV, D // 2), U8, device=device), Tensor((B, C, HKV, D // 16), U8, device=device)


def args_of(call):
    kv = lambda: Tensor((B, T, HKV, D), BF16)                     # noqa: E731
    one = lambda: Tensor((B,), I32)                               # noqa: E731
    if call == "write":
        return dict(k=kv(), v=kv(), k4=pair4(), v4=pair4(), at=one(), n=one(), k_out=kv(), v_out=kv())
    if call == "read":
        return dict(k4=pair4(), v4=pair4(), k_out=kv(), v_out=kv(), at=one(), n=one())
    q = lambda: Tensor((B, T, HQ, D), BF16)                       # noqa: E731
    lse = lambda: Tensor((B, T, HQ), F32)                         # noqa: E731
    return dict(q=q(), k4=pair4(), v4=pair4(), lens=one(), out=q(), lse=lse(), other_out=q(), other_lse=lse())


CALLS = ("write", "read", "attend")


@pytest.mark.parametrize("call", CALLS)
def test_the_calls_as_they_are_meant_reach_the_library(library, bound, call):  # noqa: F811
    getattr(bound, call)(**args_of(call))
    assert [n for n, _ in library.calls] == ["spike_proj_cache4_" + call]


@pytest.mark.parametrize("call, name", [(c, n) for c in CALLS for n in args_of(c)])
@pytest.mark.parametrize("wrong", ["device", "host", "type", "shape", "rows"])
def test_a_tensor_of_another_kind_is_refused(library, bound, call, name, wrong):  # noqa: F811
    args = args_of(call)
    for i in range(2 if name in ("k4", "v4") else 1):
        x = args[name][i] if name in ("k4", "v4") else args[name]
        bad = Tensor(x.shape, x.dtype, x.stride(), x.device)
        if wrong == "device":
            bad.device = 1
        elif wrong == "host":
            bad.device = -1
        elif wrong == "type":
            bad.dtype = torch.float64
        elif wrong == "shape":
            bad.shape = (*x.shape[:-1], x.shape[-1] + 16)
        else:
            bad._stride = (*x.stride()[:-1], 2)
        now = {**args, name: (bad, x) if name in ("k4", "v4") and i == 0 else (args[name][0], bad) if name in ("k4", "v4") else bad}
        if name in ("k4", "v4") and i == 0:
            now[name] = bad, args[name][1]
        with pytest.raises(ValueError, match="k|v|q|lens|out|lse|at|n"):
            getattr(bound, call)(**now)
    assert not library.calls


@pytest.mark.parametrize("call, name", [(c, n) for c in CALLS for n in args_of(c)])
def test_a_missing_tensor_is_refused(library, bound, call, name):  # noqa: F811
    args = {**args_of(call), name: None}
    if name in ("at", "n", "lse"):
        return getattr(bound, call)(**args)
    with pytest.raises(ValueError, match=name):
        getattr(bound, call)(**args)
    assert not library.calls
    if name in ("k4", "v4"):
        for i in range(2):
            x = list(pair4())
            x[i] = None
            with pytest.raises(ValueError, match=name):
                getattr(bound, call)(**{**args_of(call), name: tuple(x)})


# ---- the plain implementations -----------------------------------------------------
def test_quantise_by_hand():
    x = torch.tensor([6.0, -3.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -0.25, -0.3, 5.5, 0.0, -0.0, 0.1, 2.4])
    codes, scales, values = ref.quantise(x.bfloat16().view(1, 16))
    assert scales.tolist() == [[15 * 8]]                          # 1
    assert values.tolist() == [[6, -3, 0, 1, 1, 2, 2, 4, 4, 0, -0.5, 6, 0, 0, 0, 2]]
    assert codes.tolist() == [[7 + 16 * 13, 0 + 16 * 2, 2 + 16 * 4, 4 + 16 * 6, 6 + 16 * 8, 9 + 16 * 7, 0 + 16 * 8, 0 + 16 * 4]]
    # the scale: 6 * 1.0625 lies between 1 and 1.125, and goes to the even one, 1
    assert ref.quantise(torch.full((1, 16), 6.375).half())[1].item() == 120
    assert ref.quantise(torch.full((1, 16), 6.40625).half())[1].item() == 121
    assert ref.quantise(torch.full((1, 16), 65504.0).half())[1].item() == 226 and ref.SCALES[226] == 10240
    codes, scales, values = ref.quantise(torch.full((1, 16), -1e-30).bfloat16())
    assert not codes.any() and not scales.any() and not values.any()
    codes, scales, values = ref.quantise(torch.tensor([[1.0] * 15 + [math.nan], [math.inf] * 16]).half())
    assert not codes.any() and (scales == 255).all() and values.isnan().all()


def test_quantise_is_idempotent_and_near():
    g = torch.Generator().manual_seed(1)
    x = (torch.randn(500, 64, generator=g) * torch.exp2(torch.randint(-10, 10, (500, 1), generator=g).float())).bfloat16()
    codes, scales, values = ref.quantise(x)
    assert torch.equal(ref.values(codes, scales), values)
    again = ref.quantise(values.bfloat16())
    assert torch.equal(again[2], values)
    # half a step: of 2 from 4 on, of 1 from 2 on, of 0.5 below; the largest may lie 6.4 times the scale up
    s = ref.SCALES[scales.long()].repeat_interleave(16, 1)
    step = torch.where(x.double().abs() >= 4 * s, 2.0, torch.where(x.double().abs() >= 2 * s, 1.0, 0.5)) * s
    assert ((x.double() - values).abs() <= step / 2 + 1e-12).all()


def test_attend_agrees_with_the_16_bit_definition():
    g = torch.Generator().manual_seed(2)
    q = torch.randn(2, 3, 4, 32, generator=g).bfloat16()
    k, v = (ref.quantise(torch.randn(2, 20, 2, 32, generator=g).bfloat16())[2] for _ in range(2))
    out, lse, _, _ = ref.attend(q, k, v, [20, 2])
    want, wlse, _, _, _ = serving_ref.attend(q, k, v, [20, 2])
    assert torch.allclose(out, want) and torch.allclose(lse, wlse)
    # joined with the attention over the first entries, what is left gives the whole
    first = ref.attend(q, k[:, :7], v[:, :7], [7, 7], causal=False)
    rest = ref.attend(q, k[:, 7:], v[:, 7:], [13, 13], other=(first[0], first[1]))
    whole = ref.attend(q, k, v, [20, 20])
    assert torch.allclose(rest[0], whole[0]) and torch.allclose(rest[1], whole[1])
    nothing = ref.attend(q, k, v, [0, 0], other=(first[0], first[1]))
    assert torch.allclose(nothing[0], first[0]) and torch.allclose(nothing[1], first[1])


# ---- the arithmetic of the write kernel --------------------------------------------
def test_every_quotient_is_a_tie_or_far_from_one():
    """What write4_kernel's comment says: with x of 11 bits and scales of 4, |x| / s is
    a border between two codes or at least 2^-12 of itself away; and a / 6 likewise for
    the borders between two scales."""
    borders = [(1, 4), (3, 4), (5, 4), (7, 4), (5, 2), (7, 2), (5, 1)]
    for m in range(8, 16):
        for num, den in borders:
            for e in range(-16, 17):
                # |x| 2^e / m against num / den: x den 2^e - num m, in whole numbers
                for x in {x for t in (num * m / den / 2.0 ** e,) for x in range(int(t) - 1, int(t) + 3)}:
                    if 1 <= x < 2048:
                        left, right = (x * den * 2 ** e, num * m) if e >= 0 else (x * den, num * m * 2 ** -e)
                        assert left == right or abs(left - right) * 4096 >= right
    # a is x 2^k, the border 6 times halfway between two scales, (2 m + 1) / 16 of a power of two
    for m, k in itertools.product(range(8, 16), range(-4, 5)):
        for x in range(1, 2048):
            left, right = x * 2 ** (k + 4), 6 * (2 * m + 1) * 2 ** 4
            assert left == right or abs(left - right) * 4096 >= right
