"""What the cache kernels read and write, as far as arithmetic that they share
with the host decides it, and what their entry points refuse besides.  No GPU."""
import ctypes
import itertools
import subprocess
from pathlib import Path

import pytest

from paper_2606_03026_gb300 import _build, spikeproj as sp
from test_cache_cpu import cache, evict_call                     # noqa: F401  (a fixture)
from test_host_cpu import FAKE, lib                              # noqa: F401  (a fixture)

HERE = Path(__file__).resolve().parent


@pytest.fixture(scope="module")
def arith(tmp_path_factory):
    out = tmp_path_factory.mktemp("arith") / "libcache_arith.so"
    cuda = Path(_build.nvcc()).resolve().parent.parent / "include"
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", f"-I{cuda}", f"-I{_build.INCLUDE}", f"-I{_build.CSRC}",
                    str(HERE / "cache_arith.cpp"), "-o", str(out)], check=True)
    return ctypes.CDLL(str(out))


def two(f, *args):
    a, b = ctypes.c_int32(), ctypes.c_int32()
    f(*args, ctypes.byref(a), ctypes.byref(b))
    return a.value, b.value


ANY = [-2 ** 31, -2 ** 31 + 1, -305, -194, -8, -2, -1, 0, 1, 2, 7, 150, 302, 303, 304, 305, 2 ** 30, 2 ** 31 - 1]


@pytest.mark.parametrize("grid", [1, 304])
def test_partial_results_are_within_the_workspace_whatever_was_noted(arith, grid):
    """After a wait that ran out a unit's CTAs are what an earlier call or
    nobody wrote: reversed, negative, huge."""
    for first, last in itertools.product(ANY, ANY):
        at, count = two(arith.arith_results, first, last, grid)
        assert 0 <= at < grid and 0 <= count and at + count <= grid, (first, last)
        if 0 <= first <= last < grid:
            assert (at, count) == (first, last - first + 1)


@pytest.mark.parametrize("parts", [1, 2, 8])
def test_shares_of_the_results_are_all_of_them_once(arith, parts):
    for n in (0, 1, 2, 7, 8, 9, 71, 304, 608):
        have = []
        for sub in range(parts):
            begin, end = two(arith.arith_share, n, sub, parts)
            assert end <= n and begin >= 0
            have += range(begin, end)
        assert have == list(range(n))


@pytest.mark.parametrize("pieces", [(0,), (1,), (2, 1), (3, 5), (5, 4), (7, 0, 3)])
def test_no_copy_of_a_verification_is_left_on_its_way(arith, pieces):
    """Rows of so many pieces, one after another through one ring, whatever one
    copy does: late ones are waited for before the CTA may leave."""
    total = sum(pieces)
    rows = (ctypes.c_int * len(pieces))(*pieces)
    for at, what, rest in itertools.product(range(total + 1), (1, 2), (0, 1)):
        how = [0] * at + [what] + [rest] * total
        assert arith.arith_ring(len(pieces), rows, (ctypes.c_int * len(how))(*how)) == 0, (at, what, rest)


@pytest.mark.parametrize("V", [*range(1, 24), 511, 512, 513, 1030, (1 << 24) - 1])
def test_a_verification_copies_nothing_outside_its_rows(arith, V):
    """Copies are of whole 16-byte pieces of a row, and with the entries read by
    themselves at its ends they are all of it, wherever both rows begin and
    however they are cut."""
    copy = (ctypes.c_int32 * 3)()
    for p, q in itertools.product((0, 4, 8, 12), repeat=2):
        lead, trail = two(arith.arith_row_ends, p, q, V)
        assert 0 <= lead <= 3 and 0 <= trail <= 3 and lead + trail <= V
        for skip, cut in itertools.product({p, q}, (1, 2, 3, 5, 64, 512)):
            for v in range(0, V, cut) if V < 2000 else [0, cut, (V - 1) // cut * cut - cut, (V - 1) // cut * cut]:
                n = min(cut, V - v)
                arith.arith_row_copy(skip, V, v, n, copy)
                base, start, size = copy
                end = start + max(size, 0)
                if size > 0:
                    assert start % 16 == 0 and size % 16 == 0 and skip <= start and end <= skip + 4 * V
                # the place in the ring: from the 16 bytes on that hold the piece's first entry
                assert base == (skip + 4 * v) // 16 * 16 and start >= base and end - base <= 4 * n + 32
                for e in range(max(v, lead), min(v + n, V - trail)):
                    assert start <= skip + 4 * e and skip + 4 * e + 4 <= end


OWN = {name: (i + 1) * FAKE for i, name in enumerate(("weights", "pos", "lens", "now", "weights_out", "pos_out", "lens_out"))}


@pytest.mark.parametrize("out", ["weights_out", "pos_out", "lens_out"])
@pytest.mark.parametrize("given", ["weights", "pos", "lens", "now"])
def test_an_eviction_whose_output_is_an_input_is_refused(lib, cache, out, given):      # noqa: F811
    """`now` in the place of lens_out, for one: head 0 writes the lengths while
    the other heads may not have read the time yet."""
    assert lib.spike_proj_cache_evict(cache, ctypes.byref(evict_call(**OWN)), None) == sp.SP_OK
    lib.fake_launches()
    assert lib.spike_proj_cache_evict(cache, ctypes.byref(evict_call(**{**OWN, out: OWN[given]})), None) == sp.SP_EINVAL
    assert lib.fake_launches() == 0


def test_an_eviction_of_everything_needs_no_outputs_of_entries(lib, cache):     # noqa: F811
    call = evict_call(**{**OWN, "weights_out": None, "pos_out": None, "budget": 0, "recent": 0})
    assert lib.spike_proj_cache_evict(cache, ctypes.byref(call), None) == sp.SP_OK


def test_a_fault_of_a_cache_is_a_stall(lib, cache):                             # noqa: F811
    for fault, want in ((sp.SP_FAULT_STALL, sp.SP_OK), (sp.SP_FAULT_NONE, sp.SP_OK), (sp.SP_FAULT_ABORT, sp.SP_EINVAL),
                        (3, sp.SP_EINVAL), (-1, sp.SP_EINVAL)):
        assert lib.spike_proj_cache_inject_fault(cache, fault) == want
    assert lib.spike_proj_cache_inject_fault(None, sp.SP_FAULT_STALL) == sp.SP_EINVAL
