"""The 4-bit cache on tensors whose last elements lie more than 2^31 bytes or
elements from their first, in every dimension; and waits that run out."""
import time

import pytest
import torch

import cache4_ref as ref
from paper_2606_03026_gb300 import spikeproj as sp
from test_gpu_cache_far import far
from test_gpu_cache4 import activations, check, make

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def far4(x, dim):
    """far() for bytes: strides in multiples of 16."""
    stride, n = [0] * 4, 1
    for i in reversed([i for i in range(4) if i != dim]):
        stride[i], n = n, n * x.shape[i]
    stride[dim] = (max(n, 2 ** 31 // (x.shape[dim] - 1)) // 16 + 2) * 16
    last = sum((a - 1) * b for a, b in zip(x.shape, stride))
    y = torch.empty(last + 1, dtype=x.dtype, device=DEV).as_strided(x.shape, stride)
    y.copy_(x)
    return y


@pytest.mark.parametrize("T", [1, 4, 9], ids=["8-rows", "some", "many"])
@pytest.mark.parametrize("dim", [0, 1, 2], ids=["sequences", "entries", "heads"])
def test_attend4_past_32_bits(dim, T):
    q, k4, v4, lens = make(41, 2, T, 8, 2, 128, 150, [5, 150], "bf16")
    cache = sp.Cache4(8, 2, 128, 150, max_T=T)
    out, lse = far(torch.zeros_like(q), dim), torch.zeros(2, T, 8, device=DEV)
    cache.attend(far(q, dim), tuple(far4(x, dim) for x in k4), tuple(far4(x, dim) for x in v4), lens.to(DEV), out, lse=lse)
    torch.cuda.synchronize()
    assert cache.status() == sp.SP_OK
    check(q, k4, v4, lens, (out.cpu(), lse.cpu()))
    cache.close()


@pytest.mark.parametrize("dim", [0, 1, 2], ids=["sequences", "entries", "heads"])
def test_write4_and_read4_past_32_bits(dim):
    g = torch.Generator().manual_seed(42)
    k, v = (activations(g, 2, 3, 2, 64, dtype="fp16") for _ in range(2))
    cache = sp.Cache4(2, 2, 64, 5, dtype="fp16")
    held = [far4(torch.full((2, 5, 2, w), 7, dtype=torch.uint8), dim) for w in (32, 4, 32, 4)]
    at = torch.tensor([2, 1], dtype=torch.int32, device=DEV)
    outs = [far(torch.zeros_like(k), dim) for _ in range(2)]
    cache.write(far(k, dim), far(v, dim), tuple(held[:2]), tuple(held[2:]), at=at, k_out=outs[0], v_out=outs[1])
    for i, x in enumerate((k, v)):
        codes, scales, values = ref.quantise(x)
        for b, a in enumerate((2, 1)):
            assert torch.equal(held[2 * i][b, a:a + 3].cpu(), codes[b]) and torch.equal(held[2 * i + 1][b, a:a + 3].cpu(), scales[b])
            assert (held[2 * i][b, :a] == 7).all()
        assert torch.equal(outs[i].cpu(), values.half())
    back = [far(torch.zeros_like(k), dim) for _ in range(2)]
    cache.read(tuple(held[:2]), tuple(held[2:]), *back, at=at)
    assert torch.equal(back[0].cpu(), outs[0].cpu()) and torch.equal(back[1].cpu(), outs[1].cpu())
    cache.close()


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("B,T,Hq,Hkv,C", [(2, 5, 8, 2, 3000), (24, 6, 24, 2, 200), (40, 3, 33, 1, 260)],
                         ids=["long", "more", "many-rows"])
def test_waits_that_run_out(B, T, Hq, Hkv, C, D, dtype):
    """Keys that are never handed over, waits of about 2 ms: the status says so once,
    whatever the workspace held, and the next call of the handle is right."""
    g = torch.Generator().manual_seed(B)
    lens = torch.randint(T, C + 1, (B,), generator=g).tolist()
    q, k4, v4, lens = make(43, B, T, Hq, Hkv, D, C, lens, dtype)
    on = q.to(DEV), tuple(x.to(DEV) for x in k4), tuple(x.to(DEV) for x in v4), lens.to(DEV)
    cache = sp.Cache4(Hq, Hkv, D, C, max_T=T, dtype=dtype)

    def attend():
        out, lse = torch.zeros_like(on[0]), torch.zeros(B, T, Hq, device=DEV)
        cache.attend(*on, out, lse=lse)
        return out, lse

    def stalled():
        cache.inject_fault(sp.SP_FAULT_STALL)
        torch.cuda.synchronize()
        start = time.perf_counter()
        attend()
        torch.cuda.synchronize()
        assert time.perf_counter() - start < 1.0
        assert cache.status() == sp.SP_EKERNEL and cache.status() == sp.SP_OK

    stalled()                               # nothing has written the workspace
    want = attend()
    assert cache.status() == sp.SP_OK and want[0].isfinite().all()
    stalled()
    for _ in range(2):
        for x, y in zip(attend(), want):
            assert torch.equal(x, y)
    assert cache.status() == sp.SP_OK
    cache.close()
