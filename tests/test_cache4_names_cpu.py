"""What the binding of the 4-bit cache says of a tensor of another kind: its name, and
of a cache which of its two.  No GPU."""
import re

import pytest
import torch

from test_cache4_cpu import CALLS, args_of, bound                  # noqa: F401  (a fixture)
from test_cache_binding_cpu import Tensor, library                # noqa: F401  (a fixture)


def bad_ones(x):
    """x on another device, on the host, of another type and of two other shapes, and with gaps in its rows."""
    yield Tensor(x.shape, x.dtype, x.stride(), 1)
    yield Tensor(x.shape, x.dtype, x.stride(), -1)
    yield Tensor(x.shape, torch.float64, x.stride(), x.device)
    yield Tensor((*x.shape[:-1], x.shape[-1] + 16), x.dtype, x.stride(), x.device)
    yield Tensor((x.shape[0] + 1, *x.shape[1:]), x.dtype, x.stride(), x.device)
    yield Tensor(x.shape, x.dtype, (*x.stride()[:-1], 2), x.device)


# the tensor that a call takes its batch and tokens from: of another batch, the others do not fit
FIRST = {"write": "k", "read": "k_out", "attend": "q"}


@pytest.mark.parametrize("call, name", [(c, n) for c in CALLS for n in args_of(c)])
def test_a_refusal_names_the_tensor(library, bound, call, name):  # noqa: F811
    args, held = args_of(call), name in ("k4", "v4")
    for i in range(2 if held else 1):
        for n, bad in enumerate(bad_ones(args[name][i] if held else args[name])):
            if n == 4 and name == FIRST[call]:
                continue
            now = {**args, name: tuple(bad if j == i else x for j, x in enumerate(args[name])) if held else bad}
            with pytest.raises(ValueError, match="^" + re.escape(f"{name}[{i}]" if held else name) + ":"):
                getattr(bound, call)(**now)
    assert not library.calls


@pytest.mark.parametrize("call", CALLS)
def test_a_call_whose_first_tensor_is_of_another_batch_is_refused(library, bound, call):  # noqa: F811
    args = args_of(call)
    x = args[FIRST[call]]
    with pytest.raises(ValueError, match=r"^\w+(\[[01]\])?:"):
        getattr(bound, call)(**{**args, FIRST[call]: Tensor((x.shape[0] + 1, *x.shape[1:]), x.dtype)})
    assert not library.calls


@pytest.mark.parametrize("call, name, shape", [(c, n, s) for c in CALLS for n in args_of(c) for s in ((), (2,), (2, 3), (2, 3, 4, 5, 6))],
                         ids=str)
def test_tensors_of_other_ranks_are_refused(library, bound, call, name, shape):  # noqa: F811
    args, held = args_of(call), name in ("k4", "v4")
    for i in range(2 if held else 1):
        x = args[name][i] if held else args[name]
        if shape == x.shape or (len(shape) < 2 and name == FIRST[call]):     # (an IndexError, as for 16-bit caches)
            continue
        bad = Tensor(shape, x.dtype)
        now = {**args, name: tuple(bad if j == i else y for j, y in enumerate(args[name])) if held else bad}
        with pytest.raises(ValueError, match="^" + re.escape(f"{name}[{i}]" if held else name) + ":"):
            getattr(bound, call)(**now)
    assert not library.calls
