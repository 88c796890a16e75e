"""ctypes binding of libspikeproj.so (``include/spike_proj.h``).

Argument marshalling only: every step of the projection runs in the CUDA
library.  Functions keep the C names; device buffers are passed as torch CUDA
tensors (or raw integer device addresses), streams default to torch's current
stream.  A missing library is an error, never a fallback.
"""
from __future__ import annotations

import ctypes
import struct
from pathlib import Path

LIB_PATH = Path(__file__).resolve().parent / "_build" / "libspikeproj.so"

# sp_status
SP_OK, SP_EINVAL, SP_EALIGN, SP_EDEVICE, SP_ECUDA, SP_ENOMEM, SP_ERANGE, \
    SP_EKERNEL, SP_EUNSUPPORTED, SP_ESCRATCH = range(10)
# sp_fmt
SP_SPIKES_BITS32, SP_SPIKES_U8, SP_SPIKES_BOOL8 = 0, 1, 2
# sp_kernel
SP_AUTO, SP_GATHER, SP_UNION, SP_GEMM = 0, 1, 2, 3
# sp_fault (tests of the error path only)
SP_FAULT_NONE, SP_FAULT_ABORT, SP_FAULT_STALL = 0, 1, 2
SP_PLAN_GEMM = 0x1
# sp_dtype
SP_BF16, SP_FP16 = 0, 1
SP_CACHE_WEIGHTS = 0x1
SPIKE_PROJ_MAX_K = 131072
SPIKE_PROJ_MAX_GROUP = 64
SPIKE_PROJ_NOALLOC_MAX_N = 32768
SPIKE_PROJ_DENSE_MAX_B = 4
SPIKE_PROJ_DENSE_MAX_GROUP = 128
SPIKE_PROJ_CACHE_MAX_B = 1024
SPIKE_PROJ_CACHE_MAX_T = 32
SPIKE_PROJ_CACHE_MAX_HEADS = 512
SPIKE_PROJ_CACHE_MAX_D = 128
SPIKE_PROJ_CACHE_MAX_LEN = 1 << 24
SPIKE_PROJ_VERIFY_MAX_T = 64
SPIKE_PROJ_VERIFY_MAX_V = 1 << 24

FMTS = {"bits": SP_SPIKES_BITS32, "u8": SP_SPIKES_U8, "bool8": SP_SPIKES_BOOL8}
KERNELS = {"auto": SP_AUTO, "gather": SP_GATHER, "union": SP_UNION, "gemm": SP_GEMM}
DTYPES = {"bf16": SP_BF16, "fp16": SP_FP16}
KERNEL_NAMES = {v: k for k, v in KERNELS.items()}

# every entry point of the C ABI with its ctypes signature
_P, _I32, _I64, _U32 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_uint32
_SIGNATURES = {
    "spike_proj_plan": ([_P, _P, _I64, _P, _I32, _I32, _I32, _U32, _P], ctypes.c_int),
    "spike_proj_plan_destroy": ([_P], ctypes.c_int),
    "spike_proj_decode": ([_P, _P, ctypes.c_int, _P, _P, _P], ctypes.c_int),
    "spike_proj_batched": ([_P, _P, ctypes.c_int, _I32, _I64, _P, _P, ctypes.c_int, _P],
                           ctypes.c_int),
    "spike_proj_prefill": ([_P, _P, _I32, _I64, _P, _P, ctypes.c_int, _P], ctypes.c_int),
    "spike_proj_last_dispatch": ([_P, _P, _P], ctypes.c_int),
    "spike_proj_plan_status": ([_P, _P], ctypes.c_int),
    "spike_proj_group_create": ([_P, _P, _I32, _P], ctypes.c_int),
    "spike_proj_group_destroy": ([_P], ctypes.c_int),
    "spike_proj_group_decode": ([_P, _P, ctypes.c_int, _I64, _P, _P, _I64, _P], ctypes.c_int),
    "spike_proj_group_decode_host": ([_P, _P, ctypes.c_int, _I64, _P, _P, _I64, _P],
                                     ctypes.c_int),
    "spike_proj_group_decode_lif": ([_P, _P, _P, _P, _I64, ctypes.c_float, ctypes.c_float, _P,
                                     _I64, _P, _P, _I64, _P], ctypes.c_int),
    "spike_proj_group_status": ([_P, _P], ctypes.c_int),
    "spike_proj_group_prefill": ([_P, _P, ctypes.c_int, _I32, _I64, _P, _P, _P], ctypes.c_int),
    "spike_proj_decode_noalloc": ([_P, _I64, _P, _I32, _I32, _P, ctypes.c_int, _P, _P, _P],
                                  ctypes.c_int),
    "spike_proj_dense": ([_P, _I32, _I32, _P], ctypes.c_int),
    "spike_proj_lif": ([_P, _P, _I32, _I32, _I64, ctypes.c_float, ctypes.c_float, _P, _I64, _P],
                       ctypes.c_int),
    "spike_proj_head_create": ([_P, _P, _I64, _P, _I32, _I32, _P], ctypes.c_int),
    "spike_proj_head_destroy": ([_P], ctypes.c_int),
    "spike_proj_head": ([_P, _P, _I64, _I32, ctypes.c_float, _I32, _P, _P, _P, _P, _P, _P, _I64,
                         _P], ctypes.c_int),
    "spike_proj_cache_create": ([_P, _I32, _I32, _I32, _I32, _I32, _I32, _I32, _U32, _P],
                                ctypes.c_int),
    "spike_proj_cache_destroy": ([_P], ctypes.c_int),
    "spike_proj_cache_status": ([_P, _P], ctypes.c_int),
    "spike_proj_cache_attend": ([_P, _P, _P], ctypes.c_int),
    "spike_proj_cache_evict": ([_P, _P, _P], ctypes.c_int),
    "spike_proj_verify": ([_P, _P], ctypes.c_int),
    "spike_proj_probe_gather": ([_P, _P, _I32, _I32, _P, _P], ctypes.c_int),
    "spike_proj_plan_inject_fault": ([_P, _I32], ctypes.c_int),
    "spike_proj_group_inject_fault": ([_P, _I32], ctypes.c_int),
    "spike_proj_cache_inject_fault": ([_P, _I32], ctypes.c_int),
    "spike_proj_strerror": ([ctypes.c_int], ctypes.c_char_p),
    "spike_proj_last_cuda_error": ([], ctypes.c_int),
    "spike_proj_abi_version": ([], ctypes.c_int),
}

_lib = None


class SpikeProjError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        msg = lib().spike_proj_strerror(status).decode()
        if status == SP_ECUDA:
            msg += f" (cudaError {lib().spike_proj_last_cuda_error()})"
        super().__init__(f"{where}: {msg} [status {status}]")


def lib():
    """The loaded library (opened on first use).  Raises if it is not built."""
    global _lib
    if _lib is None:
        if not LIB_PATH.exists():
            raise RuntimeError(
                f"{LIB_PATH} is missing: build the CUDA library first "
                "(python -c 'import __graft_entry__ as g; g.build()')")
        L = ctypes.CDLL(str(LIB_PATH))
        for name, (args, res) in _SIGNATURES.items():
            fn = getattr(L, name)
            fn.argtypes = args
            fn.restype = res
        _lib = L
    return _lib


def _addr(x):
    """Device (or host) address of a tensor / numpy array / int / None."""
    if x is None:
        return None
    if isinstance(x, int):
        return x
    try:
        return x.data_ptr()
    except AttributeError:
        pass
    if hasattr(x, "ctypes"):
        return x.ctypes.data
    raise TypeError(f"cannot take the address of {type(x)!r}")


def _current_stream_object() -> int:
    import torch
    return torch.cuda.current_stream().cuda_stream


def _first_current_stream() -> int:
    """torch's current stream of the current device, and the function for the
    calls that follow.  torch.cuda.current_stream() builds a Stream object:
    2.9 of the 7.5 us that a single decode took on the host (Grace, torch 2.9;
    4.2 us with the raw handle, 0.1 us).  The call here also initialises
    torch's CUDA state, which the raw query needs."""
    global _current_stream
    handle = _current_stream_object()
    import torch
    device = getattr(torch._C, "_cuda_getDevice", None)
    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    _current_stream = (lambda: raw(device())) if device and raw else _current_stream_object
    return handle


_current_stream = _first_current_stream


def _stream(stream):
    if stream is None:
        return _current_stream()
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


def _check(status: int, where: str):
    if status != SP_OK:
        raise SpikeProjError(status, where)


def _fmt(fmt):
    return FMTS[fmt] if isinstance(fmt, str) else int(fmt)


def _kernel(k):
    return KERNELS[k] if isinstance(k, str) else int(k)


# ---------------------------------------------------------------------------
# thin wrappers, same names as the C ABI
# ---------------------------------------------------------------------------
def spike_proj_plan(W, ldw, scale, N, K, max_batch=1, flags=0, stream=None) -> int:
    h = ctypes.c_void_p()
    _check(lib().spike_proj_plan(ctypes.byref(h), _addr(W), ldw, _addr(scale), N, K,
                                 max_batch, flags, _stream(stream)), "spike_proj_plan")
    return h.value


def spike_proj_plan_destroy(plan):
    _check(lib().spike_proj_plan_destroy(plan), "spike_proj_plan_destroy")


def spike_proj_decode(plan, spikes, fmt, acc=None, y=None, stream=None):
    _check(lib().spike_proj_decode(plan, _addr(spikes), _fmt(fmt), _addr(acc), _addr(y),
                                   _stream(stream)), "spike_proj_decode")


def spike_proj_batched(plan, spikes, fmt, B, ld_spikes, acc=None, y=None, strategy="auto",
                       stream=None):
    _check(lib().spike_proj_batched(plan, _addr(spikes), _fmt(fmt), B, ld_spikes, _addr(acc),
                                    _addr(y), _kernel(strategy), _stream(stream)),
           "spike_proj_batched")


def spike_proj_prefill(plan, X, T, ldx, acc=None, y=None, strategy="auto", stream=None):
    _check(lib().spike_proj_prefill(plan, _addr(X), T, ldx, _addr(acc), _addr(y),
                                    _kernel(strategy), _stream(stream)), "spike_proj_prefill")


def spike_proj_last_dispatch(plan):
    k = ctypes.c_int(0)
    n = ctypes.c_int32(0)
    _check(lib().spike_proj_last_dispatch(plan, ctypes.byref(k), ctypes.byref(n)),
           "spike_proj_last_dispatch")
    return KERNEL_NAMES.get(k.value, k.value), n.value


def spike_proj_plan_status(plan, stream=None) -> int:
    return lib().spike_proj_plan_status(plan, _stream(stream))


def spike_proj_group_create(plans, stream=None) -> int:
    arr = (ctypes.c_void_p * len(plans))(*plans)
    h = ctypes.c_void_p()
    _check(lib().spike_proj_group_create(ctypes.byref(h), arr, len(plans), _stream(stream)),
           "spike_proj_group_create")
    return h.value


def spike_proj_group_destroy(group):
    _check(lib().spike_proj_group_destroy(group), "spike_proj_group_destroy")


def spike_proj_group_decode(group, spikes, fmt, ld_spikes, acc=None, y=None, ld_out=0,
                            stream=None):
    _check(lib().spike_proj_group_decode(group, _addr(spikes), _fmt(fmt), ld_spikes, _addr(acc),
                                         _addr(y), ld_out, _stream(stream)),
           "spike_proj_group_decode")


def spike_proj_group_decode_host(group, h_spikes, fmt, ld_spikes, h_acc=None, h_y=None,
                                 ld_out=0, stream=None):
    _check(lib().spike_proj_group_decode_host(group, _addr(h_spikes), _fmt(fmt), ld_spikes,
                                              _addr(h_acc), _addr(h_y), ld_out,
                                              _stream(stream)),
           "spike_proj_group_decode_host")


def spike_proj_group_decode_lif(group, v_in, v_out, I, ld, beta, theta, bits=None, ld_bits=0,
                                acc=None, y=None, ld_out=0, stream=None):
    _check(lib().spike_proj_group_decode_lif(group, _addr(v_in), _addr(v_out), _addr(I), ld, beta,
                                             theta, _addr(bits), ld_bits, _addr(acc), _addr(y),
                                             ld_out, _stream(stream)),
           "spike_proj_group_decode_lif")


def _ptr_array(xs):
    """Host array of device addresses (ctypes), or None."""
    if xs is None:
        return None
    return (ctypes.c_void_p * len(xs))(*[_addr(x) for x in xs])


def spike_proj_group_prefill(group, X, fmt, T, ldx, acc=None, y=None, stream=None):
    """X, acc, y: sequences with one device tensor (or address) per member."""
    _check(lib().spike_proj_group_prefill(group, _ptr_array(X), _fmt(fmt), T, ldx,
                                          _ptr_array(acc), _ptr_array(y), _stream(stream)),
           "spike_proj_group_prefill")


def spike_proj_group_status(group, stream=None) -> int:
    return lib().spike_proj_group_status(group, _stream(stream))


def spike_proj_lif(v, I, K, rows, ld, beta, theta, bits, ld_bits, stream=None):
    _check(lib().spike_proj_lif(_addr(v), _addr(I), K, rows, ld, beta, theta, _addr(bits), ld_bits,
                                _stream(stream)), "spike_proj_lif")


def lif(v, I, beta, theta, bits, K=None, stream=None):
    """One LIF step of every row of v / I (float32 [rows, ld] tensors),
    spikes into bits (uint32 [rows, >= ceil(K/32)])."""
    rows, ld = v.shape
    spike_proj_lif(v, I, ld if K is None else K, rows, v.stride(0), beta, theta, bits,
                   bits.stride(0), stream)


class SpDense(ctypes.Structure):
    """struct sp_dense of spike_proj.h (one continuous-input projection)."""
    _fields_ = [("W", ctypes.c_void_p), ("ldw", ctypes.c_int64), ("scale", ctypes.c_void_p),
                ("x", ctypes.c_void_p), ("ldx", ctypes.c_int64), ("y", ctypes.c_void_p),
                ("ldy", ctypes.c_int64), ("N", ctypes.c_int32), ("K", ctypes.c_int32)]


def spike_proj_dense(problems, B, stream=None):
    """problems: sequence of (W, ldw, scale, x, ldx, y, ldy, N, K), the fields
    of struct sp_dense (tensors or addresses); all run in one launch."""
    arr = (SpDense * len(problems))()
    for i, (W, ldw, scale, x, ldx, y, ldy, N, K) in enumerate(problems):
        arr[i] = SpDense(_addr(W), ldw, _addr(scale), _addr(x), ldx, _addr(y), ldy, N, K)
    _check(lib().spike_proj_dense(ctypes.addressof(arr), len(problems), B, _stream(stream)),
           "spike_proj_dense")


def dense(W, scale, x, y, K=None, stream=None):
    """One continuous-input projection: W int8 [N, ldw] row-major, scale
    float32 [N], x float32 [B, ldx], y float32 [B, ldy] (torch tensors)."""
    N, ldw = W.shape
    xs = x if x.dim() == 2 else x.reshape(1, -1)
    ys = y if y.dim() == 2 else y.reshape(1, -1)
    K = ldw if K is None else K
    spike_proj_dense([(W, ldw, scale, xs, xs.stride(0), ys, ys.stride(0), N, K)], xs.shape[0],
                     stream)


def spike_proj_decode_noalloc(W, ldw, scale, N, K, spikes, fmt, acc=None, y=None,
                              stream=None):
    """Batch-1 decode without a plan and without any allocation (the
    library's fixed per-device scratch; N <= SPIKE_PROJ_NOALLOC_MAX_N)."""
    _check(lib().spike_proj_decode_noalloc(_addr(W), ldw, _addr(scale), N, K, _addr(spikes),
                                           _fmt(fmt), _addr(acc), _addr(y), _stream(stream)),
           "spike_proj_decode_noalloc")


def spike_proj_probe_gather(base, offsets16, count, sink, piece_bytes=512, stream=None):
    """Measurement aid: read `count` pieces of `piece_bytes` at base + 16 * offsets16[i]."""
    _check(lib().spike_proj_probe_gather(_addr(base), _addr(offsets16), count, piece_bytes,
                                         _addr(sink), _stream(stream)), "spike_proj_probe_gather")


def spike_proj_plan_inject_fault(plan, fault):
    """Tests of the error path only: arm a fault for the plan's next launch."""
    _check(lib().spike_proj_plan_inject_fault(plan, fault), "spike_proj_plan_inject_fault")


def spike_proj_group_inject_fault(group, fault):
    """Tests of the error path only: arm a fault for the group's next launch."""
    _check(lib().spike_proj_group_inject_fault(group, fault), "spike_proj_group_inject_fault")


def spike_proj_cache_inject_fault(cache, fault):
    """Tests of the error path only: arm a fault for the cache's next attend call."""
    _check(lib().spike_proj_cache_inject_fault(cache, fault), "spike_proj_cache_inject_fault")


def spike_proj_strerror(status) -> str:
    return lib().spike_proj_strerror(status).decode()


def spike_proj_abi_version() -> int:
    return lib().spike_proj_abi_version()


# ---------------------------------------------------------------------------
# convenience owners (hold references to the borrowed tensors)
# ---------------------------------------------------------------------------
class Plan:
    """One projection: column-major INT8 W (torch int8 CUDA tensor whose
    storage is [K][ldw]) and FP32 scale [N]."""

    def __init__(self, W, scale, N, K, ldw=None, max_batch=1, gemm=False, stream=None):
        self.W, self.scale = W, scale            # borrowed by the library
        self.N, self.K = N, K
        self.ldw = N if ldw is None else ldw
        self.max_batch = max_batch
        self.handle = spike_proj_plan(W, self.ldw, scale, N, K, max_batch,
                                      SP_PLAN_GEMM if gemm else 0, stream)

    def decode(self, spikes, fmt, acc=None, y=None, stream=None):
        spike_proj_decode(self.handle, spikes, fmt, acc, y, stream)

    def batched(self, spikes, fmt, B, ld_spikes, acc=None, y=None, strategy="auto",
                stream=None):
        spike_proj_batched(self.handle, spikes, fmt, B, ld_spikes, acc, y, strategy, stream)

    def prefill(self, X, T, ldx, acc=None, y=None, strategy="auto", stream=None):
        spike_proj_prefill(self.handle, X, T, ldx, acc, y, strategy, stream)

    def last_dispatch(self):
        return spike_proj_last_dispatch(self.handle)

    def status(self, stream=None) -> int:
        return spike_proj_plan_status(self.handle, stream)

    def inject_fault(self, fault):
        """Tests of the error path only (SP_FAULT_ABORT / SP_FAULT_STALL)."""
        spike_proj_plan_inject_fault(self.handle, fault)

    def close(self):
        if self.handle:
            spike_proj_plan_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class Group:
    """Independent batch-1 projections decoded in one launch."""

    def __init__(self, plans, stream=None):
        self.plans = list(plans)
        self.handle = spike_proj_group_create([p.handle for p in self.plans], stream)

    def decode(self, spikes, fmt, ld_spikes, acc=None, y=None, ld_out=0, stream=None):
        spike_proj_group_decode(self.handle, spikes, fmt, ld_spikes, acc, y, ld_out, stream)

    def decode_host(self, h_spikes, fmt, ld_spikes, h_acc=None, h_y=None, ld_out=0,
                    stream=None):
        spike_proj_group_decode_host(self.handle, h_spikes, fmt, ld_spikes, h_acc, h_y,
                                     ld_out, stream)

    def decode_lif(self, v_in, v_out, I, beta, theta, bits=None, acc=None, y=None, ld_out=0,
                   stream=None):
        """One LIF step of row j of v_in / I (float32 [count, ld] tensors) into
        v_out, its spikes projected by plan j, in one launch; bits (uint32
        [count, >= ceil(maxK/32)]) optionally receives the spike words."""
        spike_proj_group_decode_lif(self.handle, v_in, v_out, I, v_in.stride(0), beta, theta, bits,
                                    0 if bits is None else bits.stride(0), acc, y, ld_out, stream)

    def prefill(self, X, fmt, T, ldx, acc=None, y=None, stream=None):
        """T rows per member through the tensor-core contraction, all members
        in one launch: X, acc, y hold one device tensor per member."""
        spike_proj_group_prefill(self.handle, X, fmt, T, ldx, acc, y, stream)

    def status(self, stream=None) -> int:
        return spike_proj_group_status(self.handle, stream)

    def inject_fault(self, fault):
        """Tests of the error path only (SP_FAULT_ABORT)."""
        spike_proj_group_inject_fault(self.handle, fault)

    def close(self):
        if self.handle:
            spike_proj_group_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def spike_proj_head_create(W, ldw, scale, V, K, stream=None) -> int:
    h = ctypes.c_void_p()
    _check(lib().spike_proj_head_create(ctypes.byref(h), _addr(W), ldw, _addr(scale), V, K,
                                        _stream(stream)), "spike_proj_head_create")
    return h.value


def spike_proj_head_destroy(head):
    _check(lib().spike_proj_head_destroy(head), "spike_proj_head_destroy")


def spike_proj_head(head, h, ldh, B, tau, k_sel, token, verified=None, gap=None, cand=None, r=None,
                    z=None, ld_z=0, stream=None):
    _check(lib().spike_proj_head(head, _addr(h), ldh, B, tau, k_sel, _addr(token), _addr(verified),
                                 _addr(gap), _addr(cand), _addr(r), _addr(z), ld_z,
                                 _stream(stream)), "spike_proj_head")


class Head:
    """Vocabulary head with INT8 activations and candidate-row verification
    over row-major INT8 weights W [V, ldw] and row scales [V] (borrowed)."""

    def __init__(self, W, scale, K=None, stream=None):
        self.W, self.scale = W, scale
        self.V, self.ldw = W.shape
        self.K = self.ldw if K is None else K
        self.handle = spike_proj_head_create(W, self.ldw, scale, self.V, self.K, stream)

    def __call__(self, h, tau, k_sel, token, verified=None, gap=None, cand=None, r=None, z=None,
                 stream=None):
        """h float32 [B, ldh]; outputs as spike_proj_head (tensors)."""
        hs = h if h.dim() == 2 else h.reshape(1, -1)
        spike_proj_head(self.handle, hs, hs.stride(0), hs.shape[0], tau, k_sel, token, verified,
                        gap, cand, r, z, 0 if z is None else z.stride(0), stream)

    def close(self):
        if self.handle:
            spike_proj_head_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


# ---------------------------------------------------------------------------
# a KV cache with a shared prefix, and the verification of drafted tokens
# ---------------------------------------------------------------------------
class SpAttend(ctypes.Structure):
    """struct sp_attend of spike_proj.h."""
    _fields_ = [("q", _P), ("q_batch", _I64), ("q_token", _I64), ("q_head", _I64),
                ("prefix_k", _P), ("prefix_v", _P),
                ("pk_entry", _I64), ("pk_head", _I64), ("pv_entry", _I64), ("pv_head", _I64),
                ("k", _P), ("v", _P), ("k_batch", _I64), ("k_entry", _I64), ("k_head", _I64),
                ("v_batch", _I64), ("v_entry", _I64), ("v_head", _I64),
                ("lens", _P), ("out", _P), ("out_batch", _I64), ("out_token", _I64),
                ("out_head", _I64), ("lse", _P), ("weights", _P), ("weights_batch", _I64),
                ("weights_head", _I64), ("B", _I32), ("T", _I32), ("prefix_len", _I32),
                ("scale", ctypes.c_float)]


class SpEvict(ctypes.Structure):
    """struct sp_evict of spike_proj.h."""
    _fields_ = [("k", _P), ("v", _P), ("k_batch", _I64), ("k_entry", _I64), ("k_head", _I64),
                ("v_batch", _I64), ("v_entry", _I64), ("v_head", _I64),
                ("weights", _P), ("pos", _P), ("in_batch", _I64), ("in_head", _I64),
                ("weights_out", _P), ("pos_out", _P), ("out_batch", _I64), ("out_head", _I64),
                ("lens", _P), ("now", _P), ("lens_out", _P),
                ("B", _I32), ("budget", _I32), ("recent", _I32)]


class SpVerify(ctypes.Structure):
    """struct sp_verify of spike_proj.h."""
    _fields_ = [("p", _P), ("p_batch", _I64), ("p_row", _I64),
                ("q", _P), ("q_batch", _I64), ("q_row", _I64),
                ("draft", _P), ("ld_draft", _I64), ("n_draft", _P), ("u", _P), ("ld_u", _I64),
                ("u_sample", _P), ("n_accept", _P), ("tokens", _P), ("ld_tokens", _I64),
                ("B", _I32), ("T", _I32), ("V", _I32)]


def spike_proj_cache_create(max_batch, max_T, Hq, Hkv, D, capacity, dtype, flags=0,
                            stream=None) -> int:
    h = ctypes.c_void_p()
    _check(lib().spike_proj_cache_create(ctypes.byref(h), max_batch, max_T, Hq, Hkv, D, capacity,
                                         DTYPES[dtype] if isinstance(dtype, str) else int(dtype),
                                         flags, _stream(stream)), "spike_proj_cache_create")
    return h.value


def spike_proj_cache_destroy(cache):
    _check(lib().spike_proj_cache_destroy(cache), "spike_proj_cache_destroy")


def spike_proj_cache_status(cache, stream=None) -> int:
    return lib().spike_proj_cache_status(cache, _stream(stream))


def spike_proj_cache_attend(cache, call, stream=None):
    """call: an SpAttend."""
    _check(lib().spike_proj_cache_attend(cache, ctypes.addressof(call), _stream(stream)),
           "spike_proj_cache_attend")


def spike_proj_cache_evict(cache, call, stream=None):
    """call: an SpEvict."""
    _check(lib().spike_proj_cache_evict(cache, ctypes.addressof(call), _stream(stream)),
           "spike_proj_cache_evict")


def spike_proj_verify(call, stream=None):
    """call: an SpVerify."""
    _check(lib().spike_proj_verify(ctypes.addressof(call), _stream(stream)), "spike_proj_verify")


def _packer(struct_type):
    """struct.Struct with the layout of a ctypes structure (its fields in order,
    native alignment): packing one call's values this way takes a fifth of the
    time of filling the ctypes structure field by field."""
    codes = {_P: "Q", _I64: "q", _I32: "i", ctypes.c_float: "f"}
    s = struct.Struct("@" + "".join(codes[t] for _, t in struct_type._fields_))
    assert ctypes.sizeof(struct_type) - s.size in range(8)       # padding at the end
    return struct.Struct(s.format + "x" * (ctypes.sizeof(struct_type) - s.size)).pack


_pack_attend, _pack_evict, _pack_verify = map(_packer, (SpAttend, SpEvict, SpVerify))


def _reject(x, name, shape, dtype, device):
    """Says what is wrong with a tensor that a call does not take as it is."""
    if x.shape != shape:
        raise ValueError(f"{name}: shape {tuple(x.shape)}, expected {tuple(shape)}")
    if x.dtype is not dtype:
        raise ValueError(f"{name}: {x.dtype}, expected {dtype}")
    if not x.is_cuda:
        raise ValueError(f"{name}: not a CUDA tensor")
    if x.get_device() != device:
        raise ValueError(f"{name}: on CUDA device {x.get_device()}, expected {device}")
    if x.shape and x.shape[-1] > 1 and x.stride(-1) != 1:
        raise ValueError(f"{name}: the last dimension is not contiguous")


def _want(x, name, shape, dtype, device):
    """The strides of a tensor of the shape and type that a call needs, rows
    contiguous, on the CUDA device of that number."""
    if x is None:
        raise ValueError(f"{name}: missing")
    st = x.stride()
    if x.shape != shape or x.dtype is not dtype or x.get_device() != device or st[-1] != 1:
        _reject(x, name, shape, dtype, device)
    return st


class Cache:
    """Attention over own caches [B, capacity, Hkv, D] of sequences that share a
    prefix [P, Hkv, D], and eviction from the own caches.  Owns workspace for
    max_batch sequences of max_T query tokens; the tensors are the caller's."""

    def __init__(self, max_batch, Hq, Hkv, D, capacity, max_T=1, dtype="bf16", weights=False,
                 stream=None):
        import torch
        self.Hq, self.Hkv, self.D, self.capacity, self.max_T = Hq, Hkv, D, capacity, max_T
        self.dtype = {"bf16": torch.bfloat16, "fp16": torch.float16}[dtype]
        self._f32, self._i32 = torch.float32, torch.int32
        self._scale = D ** -0.5
        self.handle = spike_proj_cache_create(max_batch, max_T, Hq, Hkv, D, capacity, dtype,
                                              SP_CACHE_WEIGHTS if weights else 0, stream)
        self._device = torch.cuda.current_device()             # the handle's

    def attend(self, q, k, v, lens, out, prefix_k=None, prefix_v=None, weights=None, lse=None,
               scale=None, stream=None):
        """T query tokens per sequence, q [B, T, Hq, D] -> out [B, T, Hq, D]; the
        own caches already hold the T tokens' entries, which lens (int32 [B])
        counts.  weights (float32 [B, Hkv, capacity]) gains the attention that
        the own entries get from all T tokens (of drafts that are refused later
        too); lse (float32 [B, T, Hq]) is optional."""
        t, dev = self.dtype, self._device
        if q is None:
            raise ValueError("q: missing")
        B, T = q.shape[0], q.shape[1]
        rows, own = (B, T, self.Hq, self.D), (B, self.capacity, self.Hkv, self.D)
        qs, os = _want(q, "q", rows, t, dev), _want(out, "out", rows, t, dev)
        ks, vs = _want(k, "k", own, t, dev), _want(v, "v", own, t, dev)
        _want(lens, "lens", (B,), self._i32, dev)
        P, pk, pv, pks, pvs = 0, 0, 0, (0, 0), (0, 0)
        if (prefix_k is None) != (prefix_v is None):
            raise ValueError("prefix_k, prefix_v: one without the other")
        if prefix_k is not None and prefix_k.shape[0]:
            P = prefix_k.shape[0]
            pks = _want(prefix_k, "prefix_k", (P, self.Hkv, self.D), t, dev)
            pvs = _want(prefix_v, "prefix_v", (P, self.Hkv, self.D), t, dev)
            pk, pv = prefix_k.data_ptr(), prefix_v.data_ptr()
        w, ws, l = 0, (0, 0), 0
        if weights is not None:
            ws, w = _want(weights, "weights", own[:1] + (self.Hkv, self.capacity), self._f32, dev), weights.data_ptr()
        if lse is not None:
            _want(lse, "lse", rows[:3], self._f32, dev)
            if not lse.is_contiguous():
                raise ValueError("lse: not contiguous")
            l = lse.data_ptr()
        call = _pack_attend(q.data_ptr(), qs[0], qs[1], qs[2], pk, pv, pks[0], pks[1], pvs[0], pvs[1],
                            k.data_ptr(), v.data_ptr(), ks[0], ks[1], ks[2], vs[0], vs[1], vs[2],
                            lens.data_ptr(), out.data_ptr(), os[0], os[1], os[2], l, w, ws[0], ws[1],
                            B, T, P, self._scale if scale is None else scale)
        _check(lib().spike_proj_cache_attend(self.handle, call, _stream(stream)),
               "spike_proj_cache_attend")

    def evict(self, k, v, weights, pos, lens, now, budget, recent, weights_out, pos_out, lens_out,
              stream=None):
        """Keeps `budget` entries of every own cache, the `recent` newest (pos >=
        now - recent) and then those of the most weight; K and V [B, capacity,
        Hkv, D] in place, weights and pos [B, Hkv, capacity] into weights_out
        and pos_out [B, Hkv, >= min(budget, capacity)]."""
        if k is None or weights_out is None:
            raise ValueError("k, weights_out: missing")
        t, B, dev = self.dtype, k.shape[0], self._device
        own = (B, self.capacity, self.Hkv, self.D)
        ks, vs = _want(k, "k", own, t, dev), _want(v, "v", own, t, dev)
        have = (B, self.Hkv, self.capacity)
        ws, ps = _want(weights, "weights", have, self._f32, dev), _want(pos, "pos", have, self._i32, dev)
        room = weights_out.shape[-1]
        if room < min(budget, self.capacity):
            raise ValueError("weights_out: no room for the budget")
        left = (B, self.Hkv, room)
        wos, pos_s = _want(weights_out, "weights_out", left, self._f32, dev), _want(pos_out, "pos_out", left, self._i32, dev)
        for i, n in ((0, B), (1, self.Hkv)):                   # (a dimension of size 1 has no stride)
            if n > 1 and (ps[i] != ws[i] or pos_s[i] != wos[i]):
                raise ValueError("pos: other strides than weights")
        one = (B,)
        _want(lens, "lens", one, self._i32, dev)
        _want(now, "now", one, self._i32, dev)
        _want(lens_out, "lens_out", one, self._i32, dev)
        call = _pack_evict(k.data_ptr(), v.data_ptr(), ks[0], ks[1], ks[2], vs[0], vs[1], vs[2],
                           weights.data_ptr(), pos.data_ptr(), ws[0], ws[1], weights_out.data_ptr(),
                           pos_out.data_ptr(), wos[0], wos[1], lens.data_ptr(), now.data_ptr(),
                           lens_out.data_ptr(), B, budget, recent)
        _check(lib().spike_proj_cache_evict(self.handle, call, _stream(stream)), "spike_proj_cache_evict")

    def status(self, stream=None) -> int:
        return spike_proj_cache_status(self.handle, stream)

    def inject_fault(self, fault):
        """Tests of the error path only (SP_FAULT_STALL)."""
        spike_proj_cache_inject_fault(self.handle, fault)

    def close(self):
        if self.handle:
            spike_proj_cache_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def verify(p, q, draft, u, u_sample, n_accept, tokens, n_draft=None, stream=None):
    """How many of the drafts [B, T] the target keeps and the token after them:
    p [B, T+1, V] and q [B, T, V] float32 probabilities (q, draft and u may be
    None when T is 0), u [B, T] and u_sample [B] uniform float32 in [0, 1),
    n_draft int32 [B] or None; n_accept int32 [B], tokens int32 [B, T+1]."""
    import torch
    f32, i32 = torch.float32, torch.int32
    if p is None:
        raise ValueError("p: missing")
    B, rows, V = p.shape
    T, dev = rows - 1, torch.cuda.current_device()
    ps = _want(p, "p", (B, rows, V), f32, dev)
    qa, qs, da, ds, ua, us = 0, (0, 0), 0, (0,), 0, (0,)
    if T:
        drafts = (B, T)
        qs = _want(q, "q", (B, T, V), f32, dev)
        ds, us = _want(draft, "draft", drafts, i32, dev), _want(u, "u", drafts, f32, dev)
        qa, da, ua = q.data_ptr(), draft.data_ptr(), u.data_ptr()
    one = (B,)
    _want(u_sample, "u_sample", one, f32, dev)
    _want(n_accept, "n_accept", one, i32, dev)
    ts = _want(tokens, "tokens", (B, rows), i32, dev)
    nd = 0
    if n_draft is not None:
        _want(n_draft, "n_draft", one, i32, dev)
        nd = n_draft.data_ptr()
    # (the stride of a dimension of size 1 says nothing)
    ld_draft, ld_u, ld_tokens = (ds[0], us[0], ts[0]) if B > 1 else (T, T, rows)
    call = _pack_verify(p.data_ptr(), ps[0], ps[1], qa, qs[0], qs[1], da, ld_draft, nd, ua, ld_u,
                        u_sample.data_ptr(), n_accept.data_ptr(), tokens.data_ptr(), ld_tokens, B, T, V)
    _check(lib().spike_proj_verify(call, _stream(stream)), "spike_proj_verify")
