"""What the Python binding of the cache and verification operators refuses and
takes, on stand-ins of tensors: no GPU and no call of the library."""
import pytest
import torch

from paper_2606_03026_gb300 import spikeproj as sp

B, T, HQ, HKV, D, C, P, V = 2, 3, 4, 2, 64, 8, 5, 30
BF16, F32, I32 = torch.bfloat16, torch.float32, torch.int32


class Tensor:
    """As much of a CUDA tensor as the binding looks at."""

    def __init__(self, shape, dtype, stride=None, device=0):
        self.shape, self.dtype, self.device = tuple(shape), dtype, device
        if stride is None:
            stride, n = [], 1
            for x in reversed(self.shape):
                stride.insert(0, n)
                n *= x
        self._stride = tuple(stride)

    def stride(self, dim=None):
        return self._stride if dim is None else self._stride[dim]

    is_cuda = property(lambda self: self.device >= 0)
    get_device = lambda self: self.device                        # noqa: E731
    data_ptr = lambda self: 1 << 30                              # noqa: E731
    is_contiguous = lambda self: True                            # noqa: E731


class Library:
    """Takes the calls that reach it."""

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        return lambda *args: self.calls.append((name, args)) or sp.SP_OK


@pytest.fixture
def library(monkeypatch):
    library = Library()
    monkeypatch.setattr(sp, "lib", lambda: library)
    monkeypatch.setattr(sp, "_stream", lambda stream: 0)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    return library


@pytest.fixture
def cache(library):
    cache = sp.Cache(B, HQ, HKV, D, C, max_T=T, weights=True)
    cache.handle = 1                        # (nothing made one)
    library.calls.clear()
    yield cache
    cache.handle = None


def attend_args(batch=B, **over):
    a = dict(q=Tensor((batch, T, HQ, D), BF16), k=Tensor((batch, C, HKV, D), BF16), v=Tensor((batch, C, HKV, D), BF16),
             lens=Tensor((batch,), I32), out=Tensor((batch, T, HQ, D), BF16), prefix_k=Tensor((P, HKV, D), BF16),
             prefix_v=Tensor((P, HKV, D), BF16), weights=Tensor((batch, HKV, C), F32), lse=Tensor((batch, T, HQ), F32))
    return {**a, **over}


def evict_args(batch=B, **over):
    a = dict(k=Tensor((batch, C, HKV, D), BF16), v=Tensor((batch, C, HKV, D), BF16), weights=Tensor((batch, HKV, C), F32),
             pos=Tensor((batch, HKV, C), I32), lens=Tensor((batch,), I32), now=Tensor((batch,), I32), budget=4, recent=1,
             weights_out=Tensor((batch, HKV, C), F32), pos_out=Tensor((batch, HKV, C), I32), lens_out=Tensor((batch,), I32))
    return {**a, **over}


def verify_args(batch=B, **over):
    a = dict(p=Tensor((batch, T + 1, V), F32), q=Tensor((batch, T, V), F32), draft=Tensor((batch, T), I32),
             u=Tensor((batch, T), F32), u_sample=Tensor((batch,), F32), n_accept=Tensor((batch,), I32),
             tokens=Tensor((batch, T + 1), I32), n_draft=Tensor((batch,), I32))
    return {**a, **over}


MAKE = {"attend": attend_args, "evict": evict_args, "verify": verify_args}
TENSORS = [(call, name) for call, make in MAKE.items() for name, x in make().items() if isinstance(x, Tensor)]


def run(cache, call, args):
    (sp.verify if call == "verify" else getattr(cache, call))(**args)


@pytest.mark.parametrize("call", MAKE)
def test_the_calls_as_they_are_meant_reach_the_library(library, cache, call):
    run(cache, call, MAKE[call]())
    assert len(library.calls) == 1


@pytest.mark.parametrize("call, name", TENSORS)
@pytest.mark.parametrize("device", [1, -1])
def test_a_tensor_elsewhere_is_refused(library, cache, call, name, device):
    """On another GPU than the handle's (the current one), or on none."""
    args = MAKE[call]()
    args[name].device = device
    with pytest.raises(ValueError, match=name):
        run(cache, call, args)
    assert not library.calls


OPTIONAL = {("attend", "weights"), ("attend", "lse"), ("verify", "n_draft")}


@pytest.mark.parametrize("call, name", TENSORS)
def test_a_missing_tensor_is_refused(library, cache, call, name):
    """Also one half of a prefix, and drafts without what goes with them."""
    args = {**MAKE[call](), name: None}
    if (call, name) in OPTIONAL:
        return run(cache, call, args)
    with pytest.raises(ValueError, match=name):
        run(cache, call, args)
    assert not library.calls


def test_what_a_call_can_do_without(library, cache):
    run(cache, "attend", attend_args(prefix_k=None, prefix_v=None, weights=None, lse=None))
    run(cache, "verify", verify_args(p=Tensor((B, 1, V), F32), tokens=Tensor((B, 1), I32), q=None, draft=None, u=None))
    assert len(library.calls) == 2


def test_positions_have_the_weights_strides(library, cache):
    """Where a dimension has more than one element."""
    for name, dtype in (("pos", I32), ("pos_out", I32)):
        for stride in ((HKV * C + 1, C, 1), (HKV * C, C + 1, 1)):
            with pytest.raises(ValueError, match="strides"):
                run(cache, "evict", evict_args(**{name: Tensor((B, HKV, C), dtype, stride)}))
        # one sequence: cut out of a cache whose heads come before its sequences
        run(cache, "evict", evict_args(batch=1, **{name: Tensor((1, HKV, C), dtype, (C, C, 1))}))
        # one head
        one = sp.Cache(B, 2, 1, D, C)
        one.handle = 1
        kv = {x: Tensor((B, C, 1, D), BF16) for x in ("k", "v")}
        entries = {x: Tensor((B, 1, C), F32) for x in ("weights", "weights_out")} | {x: Tensor((B, 1, C), I32) for x in ("pos", "pos_out")}
        run(one, "evict", evict_args(**kv, **{**entries, name: Tensor((B, 1, C), dtype, (C, 7 * C, 1))}))
        one.handle = None
    assert [n for n, _ in library.calls].count("spike_proj_cache_evict") == 4
