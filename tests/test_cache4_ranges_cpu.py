"""What the merge of the 4-bit cache's attention reads, as far as arithmetic that it
shares with the host decides it.  No GPU."""
import ctypes
import random
import subprocess
from pathlib import Path

import pytest

from paper_2606_03026_gb300 import _build

HERE = Path(__file__).resolve().parent


@pytest.fixture(scope="module")
def arith(tmp_path_factory):
    out = tmp_path_factory.mktemp("arith4") / "libcache4_arith.so"
    cuda = Path(_build.nvcc()).resolve().parent.parent / "include"
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", f"-I{cuda}", f"-I{_build.INCLUDE}", f"-I{_build.CSRC}",
                    str(HERE / "cache4_arith.cpp"), "-o", str(out)], check=True)
    lib = ctypes.CDLL(str(out))
    lib.arith4_merge.restype = ctypes.c_int64
    return lib


def merged(arith, shape, sms, R, side, slot, last):
    parts, at, end = ctypes.c_int32(), (ctypes.c_int64 * 2)(), (ctypes.c_int64 * 2)()
    size = arith.arith4_merge(*shape, sms, R, side, slot, last, ctypes.byref(parts), at, end)
    return size, parts.value, tuple(at), tuple(end)


# max_T, Hq, Hkv, D: plans by warps and by CTAs, of 8 to 96 rows a slot
SHAPES = [(8, 64, 8, 128), (5, 16, 4, 128), (5, 8, 2, 128), (32, 12, 4, 64), (32, 12, 4, 128), (9, 40, 2, 112), (32, 2, 2, 32),
          (2, 512, 1, 64)]


@pytest.mark.parametrize("sms", [132, 148, 152])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "-".join(map(str, s)))
def test_a_merge_stays_within_the_workspace_whatever_was_noted(arith, shape, sms):
    """After a wait that ran out a unit's note is what an earlier call of the handle left,
    for another number of query tokens: notes of every plan, read under every plan, and
    any other numbers."""
    rng = random.Random(sms)
    max_T, G = shape[0], shape[1] // shape[2]
    plans = sorted({T * G for T in range(1, max_T + 1)})
    notes = []
    for R in plans:
        w = arith.arith4_workers(R, shape[3], sms)
        notes += [(s, x) for s in (0, 1, w - 1, w, 2 * w - 2, 2 * w - 1) for x in (0, 1, w // 2, w - 2, w - 1)]
        notes += [(rng.randrange(2 * w), rng.randrange(w)) for _ in range(20)]
    notes += [(0, 2 ** 31 - 1), (2 ** 31 - 1, 0), (2 ** 31 - 1, 2 ** 31 - 1), (5, -7), (1, -2 ** 31)]
    slots = (ctypes.c_int64 * 3)()
    for R in plans:
        arith.arith4_slots(*shape, sms, R, slots)
        for slot, last in notes:
            for side in (1, 2, shape[2]):
                size, parts, at, end = merged(arith, shape, sms, R, side, slot, last)
                w = arith.arith4_workers(R, shape[3], sms)
                assert parts >= (1 if slot < 2 * w and last < w else 0)
                if parts:
                    assert slots[0] <= at[0] and end[0] <= slots[1], (R, side, slot, last)
                    assert slots[1] <= at[1] and end[1] <= slots[2] <= size, (R, side, slot, last)


@pytest.mark.parametrize("side", [1, 2, 8])
def test_the_parts_that_a_call_notes_are_merged(arith, side):
    """What a kernel writes down itself is taken as it is: the slot, then the first ones
    of the workers beside it up to the last."""
    shape, sms = (8, 64, 8, 128), 152
    for R in (8, 16, 24, 64):
        w, slots, row = arith.arith4_workers(R, shape[3], sms), (ctypes.c_int64 * 3)(), 8 * ((min(R, 8) if R <= 16 else R) // 8)
        arith.arith4_slots(*shape, sms, R, slots)
        for first in (0, 1, w // 2, w - 1):
            for count in range(1, (w - 1 - first) // side + 2):
                for second in (0, 1):
                    last = first + (count - 1) * side
                    _, parts, at, end = merged(arith, shape, sms, R, side, 2 * first + second, last)
                    assert parts == count
                    assert at[1] == slots[1] + (2 * first + second if count == 1 else min(2 * first + second, 2 * (first + side))) * row * 512
                    assert end[1] == slots[1] + (1 + (2 * first + second if count == 1 else 2 * last)) * row * 512
