"""Values of a 4-bit cache written once more: in the place of the tokens, and what is
read back.  The codes and scales are the definition's of these values."""
import pytest
import torch

import cache4_ref as ref
from paper_2606_03026_gb300 import spikeproj as sp
from test_gpu_cache4 import DEV, activations, place

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("layout", ["entries", "heads"])
@pytest.mark.parametrize("D", [16, 64, 112])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_values_written_once_more(dtype, D, layout):
    g = torch.Generator().manual_seed(71)
    B, T, H, C = 2, 33, 3, 40
    # (sizes down to where scales are multiples of 2^-17: codes may change there, values do not)
    x = [(activations(g, B, T, H, D, dtype=dtype).double() * 2.0 ** -i).to(torch.bfloat16 if dtype == "bf16" else torch.float16)
         for i in (0, 9)]
    cache = sp.Cache4(H, H, D, C, dtype=dtype)
    k4, v4 = (tuple(place(torch.zeros(B, C, H, w, dtype=torch.uint8), layout) for w in (D // 2, D // 16)) for _ in range(2))
    k, v = (place(y, layout) for y in x)
    for _ in range(3):
        want = [ref.quantise(y) for y in x]
        cache.write(k, v, k4, v4, k_out=k, v_out=v)
        for (codes, scales, values), held, out in zip(want, (k4, v4), (k, v)):
            assert torch.equal(held[0][:, :T].cpu(), codes) and torch.equal(held[1][:, :T].cpu(), scales)
            assert torch.equal(out.cpu().double(), values)
        x = [w[2].to(k.dtype) for w in want]
    # what is read back and written again, into other slots
    back = [torch.empty(B, T, H, D, dtype=k.dtype, device=DEV) for _ in range(2)]
    cache.read(k4, v4, *back)
    at = torch.full((B,), C - T, dtype=torch.int32, device=DEV)
    cache.write(*back, k4, v4, at=at)
    for y, held in zip(x, (k4, v4)):
        codes, scales, _ = ref.quantise(y)
        assert torch.equal(held[0][:, C - T:].cpu(), codes) and torch.equal(held[1][:, C - T:].cpu(), scales)
    cache.close()
