"""Thin binding over the C ABI of ``liblrsa.so`` (declared in ``include/lrsa.h``).

Argument marshalling only: torch supplies device memory and streams, every step of the path
runs in the library's CUDA kernels.  There is no fallback: if the shared library is missing
the import of any entry point raises.

A call runs on `stream`, by default the current one, and the caller orders that stream behind what made the
inputs.  Results and workspaces that the caller does not give are made in the memory of that stream.  A device-side wait that
runs out (LRSA_ERR_TIMEOUT) is told by lrsa_workspace_status on the workspace of the call: give one where that matters.
"""
from __future__ import annotations

import ctypes
import importlib.machinery
import importlib.util
import os
from dataclasses import dataclass

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "liblrsa.so")
CALL_PATH = os.path.join(_HERE, "_lrsa_call" + importlib.machinery.EXTENSION_SUFFIXES[0])

STATUS = {0: "LRSA_OK", 1: "LRSA_ERR_INVALID_ARG", 2: "LRSA_ERR_UNSUPPORTED",
          3: "LRSA_ERR_WORKSPACE_TOO_SMALL", 4: "LRSA_ERR_CUDA", 5: "LRSA_ERR_TIMEOUT"}


class LrsaError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {STATUS.get(status, status)} ({status_string(status)})")


class lrsa_params_t(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in
                ("batch", "n_q_heads", "n_kv_heads", "seq_len", "head_dim", "chunk", "lag", "top_k",
                 "n_sink", "n_dense_prev", "std_ddof")] + [("softmax_scale", ctypes.c_float),
                                                           ("n_seqs", ctypes.c_int32),
                                                           ("cu_seqlens", ctypes.POINTER(ctypes.c_int32)),
                                                           ("o_residual", ctypes.c_void_p)]


class lrsa_store_t(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("list_type", "block", "keep", "reserved")] + \
               [(n, ctypes.c_void_p) for n in ("k_list", "v_list", "k_scale", "v_scale", "k_recent", "v_recent", "weight", "idx")]


class lrsa_rope_t(ctypes.Structure):
    _fields_ = [("cos", ctypes.c_void_p), ("sin", ctypes.c_void_p)] + \
               [(n, ctypes.c_int32) for n in ("n_pos", "dim", "interleaved", "reserved")]


class lrsa_paged_t(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("page", "n_pages", "n_seqs", "table_width")] + \
               [(n, ctypes.c_void_p) for n in ("k_pages", "v_pages", "table", "n_tokens")]


class lrsa_rows_t(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("head_stride", ctypes.c_int64), ("token_stride", ctypes.c_int64)]


@dataclass(frozen=True)
class Params:
    """Mirror of ``lrsa_params_t`` (Section 3.2: sink size S, lag L, kept tokens K = r*L)."""
    batch: int
    n_q_heads: int
    n_kv_heads: int
    seq_len: int
    head_dim: int
    lag: int
    top_k: int
    n_sink: int
    chunk: int = 0            # 0 -> lag
    n_dense_prev: int = 1
    std_ddof: int = 1
    softmax_scale: float = 0.0
    cu_seqlens: tuple = ()    # packed batch: boundaries (0, ..., seq_len) of the sequences on the token axis

    __slots__ = ("_struct", "__dict__", "__weakref__")   # the C struct lies beside the fields, not among them

    def c(self, o_residual=None) -> lrsa_params_t:
        """The C struct; `o_residual`: a bf16 tensor shaped like O (or None), see lrsa_attn_fwd."""
        cp = lrsa_params_t(self.batch, self.n_q_heads, self.n_kv_heads, self.seq_len, self.head_dim,
                           self.chunk or self.lag, self.lag, self.top_k, self.n_sink,
                           self.n_dense_prev, self.std_ddof, self.softmax_scale, 0, None,
                           None if o_residual is None else o_residual.data_ptr())
        if self.cu_seqlens:
            arr = (ctypes.c_int32 * len(self.cu_seqlens))(*self.cu_seqlens)
            cp.n_seqs = len(self.cu_seqlens) - 1
            cp.cu_seqlens = ctypes.cast(arr, ctypes.POINTER(ctypes.c_int32))
            cp._keepalive = arr          # the host array lives as long as the struct
        return cp

    def struct(self) -> lrsa_params_t:
        """The C struct of a call without a residual (the library only reads it), built once per object: building it on every
        call took a third of a decode step's host time.  Boundaries in a list may change and are read each time.  The
        caller holds on to the struct while it uses its address."""
        try:
            return self._struct
        except AttributeError:
            cp = self.c()
            if type(self.cu_seqlens) is tuple:
                object.__setattr__(self, "_struct", cp)
            return cp

    def ref(self, o_residual=None):
        """The C struct by reference, for a call (the reference keeps it alive)."""
        return ctypes.byref(self.struct() if o_residual is None else self.c(o_residual))

    def __getstate__(self):
        return dict(self.__dict__)   # without the struct, which holds addresses of this process

    @staticmethod
    def from_workload(w, **kw) -> "Params":
        return Params(w.B, w.Hq, w.Hkv, w.N, w.d, w.L, w.K, w.S, **kw)


_lib = None
_call = None   # the module of csrc/pycall.c, the short calls without ctypes, or what stands for it


def lib() -> ctypes.CDLL:
    """Loads the CUDA library; raises if it has not been built."""
    global _lib, _call
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError(f"{LIB_PATH} is missing: run `python -c 'import __graft_entry__ as g; g.build()'` "
                              "(there is no CPU fallback)")
        L = ctypes.CDLL(LIB_PATH)
        vp, sz, i32p, fp = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p, ctypes.c_void_p
        pp = ctypes.POINTER(lrsa_params_t)
        L.lrsa_num_sel_windows.argtypes = [pp, ctypes.POINTER(ctypes.c_int32)]
        L.lrsa_workspace_bytes.argtypes = [pp] + [ctypes.POINTER(sz)] * 3
        L.lrsa_score_select.argtypes = [pp, vp, vp, i32p, fp, vp, sz, vp]
        L.lrsa_score_select_static.argtypes = [pp, vp, vp, i32p, fp, vp]
        L.lrsa_score_select_static.restype = ctypes.c_int
        L.lrsa_attn_fwd.argtypes = [pp, vp, vp, vp, i32p, vp, fp, vp, sz, vp]
        L.lrsa_attn_bwd.argtypes = [pp, vp, vp, vp, vp, vp, fp, i32p, vp, vp, vp, vp, sz, vp]
        i32 = ctypes.c_int32
        L.lrsa_cache_bytes.argtypes = [pp, ctypes.POINTER(sz), ctypes.POINTER(sz)]
        L.lrsa_cache_append.argtypes = [pp, vp, sz, vp, vp, i32, i32, vp, sz, vp]
        L.lrsa_cache_kept.argtypes = [pp, vp, ctypes.POINTER(ctypes.c_void_p), ctypes.POINTER(i32)]
        L.lrsa_attn_decode.argtypes = [pp, vp, sz, vp, i32, vp, fp, vp, sz, vp]
        for name in ("lrsa_cache_bytes", "lrsa_cache_append", "lrsa_cache_kept", "lrsa_attn_decode"):
            getattr(L, name).restype = ctypes.c_int
        sp = ctypes.POINTER(lrsa_store_t)
        L.lrsa_attn_weights.argtypes = [pp, vp, vp, fp, fp, vp, sz, vp]
        L.lrsa_weight_select.argtypes = [pp, fp, i32p, vp]
        L.lrsa_store_shape.argtypes = [pp, sp, ctypes.POINTER(i32), ctypes.POINTER(i32), ctypes.POINTER(sz)]
        L.lrsa_store_append.argtypes = [pp, sp, vp, vp, fp, i32, i32, vp, sz, vp]
        L.lrsa_store_decode.argtypes = [pp, sp, vp, i32, vp, fp, vp, sz, vp]
        L.lrsa_store_rows.argtypes = [pp, sp, i32, fp, fp, vp]
        for name in ("lrsa_attn_weights", "lrsa_weight_select", "lrsa_store_shape", "lrsa_store_append", "lrsa_store_decode",
                     "lrsa_store_rows"):
            getattr(L, name).restype = ctypes.c_int
        rp, gp, wp = ctypes.POINTER(lrsa_rope_t), ctypes.POINTER(lrsa_paged_t), ctypes.POINTER(lrsa_rows_t)
        L.lrsa_rotate.argtypes = [pp, vp, vp, vp, vp, rp, i32p, i32, vp]
        L.lrsa_paged_shape.argtypes = [pp, i32, i32, i32, i32, ctypes.POINTER(i32), ctypes.POINTER(i32), ctypes.POINTER(sz)]
        L.lrsa_paged_append.argtypes = [pp, gp, wp, wp, i32, vp, i32, vp, rp, vp, vp, sz, vp]
        L.lrsa_paged_attend.argtypes = [pp, gp, wp, wp, wp, vp, i32, i32, vp, rp, wp, fp, vp, sz, vp]
        for name in ("lrsa_rotate", "lrsa_paged_shape", "lrsa_paged_append", "lrsa_paged_attend"):
            getattr(L, name).restype = ctypes.c_int
        L.lrsa_workspace_status.argtypes = L.lrsa_paged_status.argtypes = [vp, vp]
        L.lrsa_paged_status.restype = ctypes.c_int
        L.lrsa_score_select_static_status.argtypes = [vp]
        L.lrsa_score_select_static_status.restype = ctypes.c_int
        L.lrsa_status_string.argtypes = [ctypes.c_int]
        L.lrsa_status_string.restype = ctypes.c_char_p
        L.lrsa_last_launch_count.argtypes = []
        L.lrsa_debug_set_impl.argtypes = [ctypes.c_int]
        L.lrsa_debug_set_wait_limit.argtypes = [ctypes.c_int]
        L.lrsa_debug_set_wait_limit.restype = ctypes.c_int
        for name in ("lrsa_num_sel_windows", "lrsa_workspace_bytes", "lrsa_score_select", "lrsa_attn_fwd",
                     "lrsa_attn_bwd", "lrsa_workspace_status", "lrsa_last_launch_count", "lrsa_debug_set_impl"):
            getattr(L, name).restype = ctypes.c_int
        _call = _token_calls(L)
        _lib = L
    return _lib


class _CtypesCalls:
    """The helper module's calls where there is none for this interpreter (about 1 us a call more)."""

    def __init__(self, L):
        at = ctypes.POINTER(lrsa_params_t)
        for name in ("cache_append", "attn_decode", "attn_weights", "weight_select"):
            setattr(self, name, lambda params, *args, f=getattr(L, "lrsa_" + name): f(ctypes.cast(params, at), *args))
        for name in ("store_append", "store_decode", "store_rows"):    # eleven arguments make a store
            setattr(self, name, lambda params, *args, f=getattr(L, "lrsa_" + name):
                    f(ctypes.cast(params, at), ctypes.byref(lrsa_store_t(*args[:3], 0, *args[3:11])), *args[11:]))

        def rope(cos, sin, *rest):
            return ctypes.byref(lrsa_rope_t(cos, sin, *rest, 0)) if cos else None

        def rows(*args):
            return ctypes.byref(lrsa_rows_t(*args))

        # the orders of csrc/pycall.c: eight values make a paged cache, three make rows, five a rope
        self.rotate = lambda params, q, k, qo, ko, *args: L.lrsa_rotate(
            ctypes.cast(params, at), q, k, qo, ko, rope(*args[:5]), *args[5:])
        self.paged_append = lambda params, *a: L.lrsa_paged_append(
            ctypes.cast(params, at), ctypes.byref(lrsa_paged_t(*a[:8])), rows(*a[8:11]), rows(*a[11:14]), *a[14:18], rope(*a[18:23]), *a[23:])
        self.paged_attend = lambda params, *a: L.lrsa_paged_attend(
            ctypes.cast(params, at), ctypes.byref(lrsa_paged_t(*a[:8])), rows(*a[8:11]), rows(*a[11:14]), rows(*a[14:17]), *a[17:21],
            rope(*a[21:26]), rows(*a[26:29]), *a[29:])


def _token_calls(L):
    spec = importlib.util.spec_from_file_location("_lrsa_call", CALL_PATH)
    try:
        if spec is None:
            raise ImportError(CALL_PATH)
        call = importlib.util.module_from_spec(spec)
        spec.loader.exec_module(call)
        return call
    except (ImportError, OSError):
        return _CtypesCalls(L)


def status_string(status: int) -> str:
    return lib().lrsa_status_string(int(status)).decode()


def _check(status: int, where: str):
    if status != 0:
        raise LrsaError(status, where)


_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device   # (a tensor on a GPU is in hand)


def _p(t):
    return None if t is None else t.data_ptr()


def _stream(stream):
    if stream is not None:
        return stream.cuda_stream
    if _raw_stream is not None:    # the handle without a Stream object around it (0.1 us instead of 3.2)
        return _raw_stream(torch.cuda.current_device())
    return torch.cuda.current_stream().cuda_stream


def lrsa_num_sel_windows(params: Params) -> int:
    out = ctypes.c_int32(0)
    _check(lib().lrsa_num_sel_windows(params.ref(), ctypes.byref(out)), "lrsa_num_sel_windows")
    return out.value


def lrsa_workspace_bytes(params: Params):
    a, b, c = ctypes.c_size_t(0), ctypes.c_size_t(0), ctypes.c_size_t(0)
    _check(lib().lrsa_workspace_bytes(params.ref(), ctypes.byref(a), ctypes.byref(b), ctypes.byref(c)),
           "lrsa_workspace_bytes")
    return a.value, b.value, c.value


def new_workspace(nbytes: int, device="cuda") -> torch.Tensor:
    return torch.empty(max(nbytes, 256), dtype=torch.uint8, device=device)


def _cleared_workspace(nbytes: int, device) -> torch.Tensor:
    """A workspace with a header of zeros, as lrsa_paged_status wants it."""
    ws = new_workspace(nbytes, device)
    ws[:256].zero_()
    return ws


def _made(stream, near, make, *args, **kw):
    """make(*args, **kw), a tensor beside `near` that a call on `stream` makes for itself or returns, in memory of that stream.
    The allocator orders the users of a block by the stream it was asked for on: a block of the current stream may still be in
    use there when a call on another stream starts to write it, and a temporary that the call drops may be another tensor of
    the current stream before the kernel has run."""
    if stream is None or not near.is_cuda:
        return make(*args, **kw)
    here = torch.cuda.current_stream()
    if not isinstance(stream, torch.cuda.Stream):     # another library's
        stream = torch.cuda.ExternalStream(stream.cuda_stream)
    with torch.cuda.stream(stream):
        t = make(*args, **kw)
    t.record_stream(here)     # where the caller will use it, and drop it
    return t


def lrsa_score_select(params: Params, K, V, idx=None, score=None, workspace=None, stream=None,
                      want_score: bool = False):
    """Eq. 4-8 + top-K.  Returns (idx int32 [B,Hkv,W_sel,K], score or None)."""
    wsel = lrsa_num_sel_windows(params)
    if idx is None:
        idx = _made(stream, K, torch.empty, (params.batch, params.n_kv_heads, wsel, params.top_k), dtype=torch.int32,
                    device=K.device)
    if score is None and want_score:
        score = _made(stream, K, torch.empty, (params.batch, params.n_kv_heads, wsel, params.lag), dtype=torch.float32,
                      device=K.device)
    if workspace is None:
        workspace = _made(stream, K, new_workspace, lrsa_workspace_bytes(params)[0], K.device)
    _check(lib().lrsa_score_select(params.ref(), _p(K), _p(V), _p(idx), _p(score), _p(workspace),
                                   workspace.numel(), _stream(stream)), "lrsa_score_select")
    return idx, score


STATIC_SCRATCH_BYTES = 4 << 20


def lrsa_score_select_static(params: Params, K, V, idx, score=None, stream=None):
    """lrsa_score_select for callers that cannot provide or allocate scratch memory: the library's
    own fixed device array (STATIC_SCRATCH_BYTES) is used, so nothing is allocated here either -
    `idx` (and `score`, if wanted) must be passed in.  Problems that need more scratch raise
    LRSA_ERR_WORKSPACE_TOO_SMALL.  Calls that may overlap on the GPU must be serialised."""
    _check(lib().lrsa_score_select_static(params.ref(), _p(K), _p(V), _p(idx), _p(score), _stream(stream)),
           "lrsa_score_select_static")
    return idx, score


def lrsa_score_select_static_status(stream=None) -> int:
    """Status of the last lrsa_score_select_static call on the current device (0 = ok, 5 = a bounded
    device-side wait expired).  Synchronises the stream."""
    return lib().lrsa_score_select_static_status(_stream(stream))


def lrsa_attn_fwd(params: Params, Q, K, V, idx, O=None, LSE=None, workspace=None, stream=None, o_residual=None):
    """Eq. 3 under the chunked mask.  Returns (O bf16 [B,Hq,N,d], LSE fp32 [B,Hq,N]).  `o_residual` (bf16,
    shaped like O, optional) receives what the bf16 O cannot hold; lrsa_attn_bwd takes it to form dK more accurately."""
    if O is None:
        O = _made(stream, Q, torch.empty_like, Q)
    if LSE is None:
        LSE = _made(stream, Q, Q.new_empty, Q.shape[:3], dtype=torch.float32)
    if workspace is None:
        workspace = _made(stream, Q, new_workspace, lrsa_workspace_bytes(params)[1], Q.device)
    _check(lib().lrsa_attn_fwd(params.ref(o_residual), _p(Q), _p(K), _p(V), _p(idx), _p(O), _p(LSE), _p(workspace),
                               workspace.numel(), _stream(stream)), "lrsa_attn_fwd")
    return O, LSE


def lrsa_attn_bwd(params: Params, Q, K, V, O, dO, LSE, idx, dQ=None, dK=None, dV=None, workspace=None,
                  stream=None, o_residual=None):
    """Gradient of Eq. 3 with the mask constant.  Returns (dQ, dK, dV) in bf16."""
    if dQ is None:
        dQ = _made(stream, Q, torch.empty_like, Q)
    if dK is None:
        dK = _made(stream, Q, torch.empty_like, K)
    if dV is None:
        dV = _made(stream, Q, torch.empty_like, V)
    if workspace is None:
        workspace = _made(stream, Q, new_workspace, lrsa_workspace_bytes(params)[2], Q.device)
    _check(lib().lrsa_attn_bwd(params.ref(o_residual), _p(Q), _p(K), _p(V), _p(O), _p(dO), _p(LSE), _p(idx), _p(dQ),
                               _p(dK), _p(dV), _p(workspace), workspace.numel(), _stream(stream)), "lrsa_attn_bwd")
    return dQ, dK, dV


def _device(where, name, t) -> int:
    """The index of the current device, on which `t` has to be."""
    dev = t.get_device()      # -1: not a GPU's
    if dev < 0 or dev != _current_device():
        raise LrsaError(1, f"{where}: {name} must be on the current device, got {t.device}")
    return dev


def _expect(where, name, t, shape, dtype, dev):
    """Raises LRSA_ERR_INVALID_ARG unless `t` is a contiguous tensor of this shape and type on device `dev`."""
    if t.dtype is not dtype or t.shape != shape or not t.is_contiguous() or t.get_device() != dev:
        raise LrsaError(1, f"{where}: {name} must be a contiguous {dtype} tensor of shape {tuple(shape)} on cuda:{dev}, got "
                           f"{t.dtype} {tuple(t.shape)} on {t.device}{'' if t.is_contiguous() else ' (strided)'}")


def _stream_of(stream, dev):
    if stream is None and _raw_stream is not None:
        return _raw_stream(dev)
    return _stream(stream)


def _calls():
    if _call is None:
        lib()
    return _call


def lrsa_attn_weights(params: Params, Q, K, LSE, weight=None, workspace=None, stream=None):
    """The attention weight that every position gathers from the queries that see it uncompressed: fp32 [B,Hkv,N], summed
    over the query heads of a group.  `LSE`: that of lrsa_attn_fwd on the same Q and K.  The status of the call stays in the
    `workspace` that the caller gives (256 bytes, lrsa_workspace_status)."""
    p, where, call = params, "lrsa_attn_weights", _calls()
    dev = _device(where, "Q", Q)
    _expect(where, "Q", Q, (p.batch, p.n_q_heads, p.seq_len, p.head_dim), torch.bfloat16, dev)
    _expect(where, "K", K, (p.batch, p.n_kv_heads, p.seq_len, p.head_dim), torch.bfloat16, dev)
    _expect(where, "LSE", LSE, (p.batch, p.n_q_heads, p.seq_len), torch.float32, dev)
    if weight is None:
        weight = _made(stream, Q, torch.empty, (p.batch, p.n_kv_heads, p.seq_len), dtype=torch.float32, device=Q.device)
    else:
        _expect(where, "weight", weight, (p.batch, p.n_kv_heads, p.seq_len), torch.float32, dev)
    if workspace is None:
        workspace = _made(stream, Q, new_workspace, 256, Q.device)
    else:
        _device(where, "workspace", workspace)
    cp = p.struct()
    status = call.attn_weights(ctypes.addressof(cp), Q.data_ptr(), K.data_ptr(), LSE.data_ptr(), weight.data_ptr(),
                               workspace.data_ptr(), workspace.numel(), _stream_of(stream, dev))
    if status:
        _check(status, where)
    return weight


def lrsa_weight_select(params: Params, weight, idx=None, stream=None):
    """The top_k heaviest positions of every scored window: idx int32 [B,Hkv,W_sel,K], for lrsa_attn_fwd and lrsa_attn_bwd in
    the place of lrsa_score_select's."""
    p, where, call = params, "lrsa_weight_select", _calls()
    dev = _device(where, "weight", weight)
    _expect(where, "weight", weight, (p.batch, p.n_kv_heads, p.seq_len), torch.float32, dev)
    n = lrsa_num_sel_windows(p) if p.cu_seqlens or p.lag < 1 else max((p.seq_len - p.n_sink) // p.lag - 1, 0)
    shape = (p.batch, p.n_kv_heads, n, p.top_k)
    if idx is None:
        idx = _made(stream, weight, torch.empty, shape, dtype=torch.int32, device=weight.device)
    else:
        _expect(where, "idx", idx, shape, torch.int32, dev)
    cp = p.struct()
    status = call.weight_select(ctypes.addressof(cp), weight.data_ptr(), idx.data_ptr(), _stream_of(stream, dev))
    if status:
        _check(status, where)
    return idx


def lrsa_workspace_status(workspace, stream=None) -> int:
    return lib().lrsa_workspace_status(_p(workspace), _stream(stream))


def lrsa_last_launch_count() -> int:
    return lib().lrsa_last_launch_count()


def lrsa_debug_set_wait_limit(polls: int):
    """Test hook: polls granted to the long-window scoring kernel's wait (negative: give up at once, 0: default)."""
    _check(lib().lrsa_debug_set_wait_limit(int(polls)), "lrsa_debug_set_wait_limit")


def lrsa_debug_set_impl(impl: int):
    _check(lib().lrsa_debug_set_impl(int(impl)), "lrsa_debug_set_impl")


class KVCache:
    """Condensed KV cache of one layer for inference (Section 3.2): owns the device buffer and the token
    count; every operation runs in the library's kernels."""

    _lse = None   # what an lse looks like (2 us less of host time per token than its shape); none in a cache saved without it

    def __init__(self, params: Params, device="cuda"):
        self.params = params
        a, b = ctypes.c_size_t(0), ctypes.c_size_t(0)
        _check(lib().lrsa_cache_bytes(params.ref(), ctypes.byref(a), ctypes.byref(b)), "lrsa_cache_bytes")
        self.buf = torch.zeros(a.value, dtype=torch.uint8, device=device)
        self.ws = new_workspace(b.value, device)
        self.n_tokens = 0
        self._lse = torch.empty((params.batch, params.n_q_heads), dtype=torch.float32, device=device)

    def append(self, k_new, v_new, stream=None):
        """k_new, v_new: bf16 [B, Hkv, n_new, d] (contiguous)."""
        n_new = k_new.shape[2]
        buf, ws = self.buf, self.ws
        cp = self.params.struct()
        if _call is None:      # a cache that came from another process
            lib()
        status = _call.cache_append(ctypes.addressof(cp), buf.data_ptr(), buf.numel(), _p(k_new), _p(v_new),
                                    self.n_tokens, n_new, ws.data_ptr(), ws.numel(), _stream(stream))
        if status:
            _check(status, "lrsa_cache_append")
        self.n_tokens += n_new

    def decode(self, q, o=None, lse=None, stream=None):
        """q: bf16 [B, Hq, d], the query of the last token in the cache.  Returns (o, lse)."""
        if o is None:
            o = torch.empty_like(q) if stream is None else _made(stream, q, torch.empty_like, q)
        if lse is None:
            like = self._lse
            if like is None:
                lse = _made(stream, q, q.new_empty, q.shape[:2], dtype=torch.float32)
            else:
                lse = torch.empty_like(like) if stream is None else _made(stream, q, torch.empty_like, like)
        buf, ws = self.buf, self.ws
        cp = self.params.struct()
        if _call is None:
            lib()
        status = _call.attn_decode(ctypes.addressof(cp), buf.data_ptr(), buf.numel(), _p(q), self.n_tokens,
                                   o.data_ptr(), lse.data_ptr(), ws.data_ptr(), ws.numel(), _stream(stream))
        if status:
            _check(status, "lrsa_attn_decode")
        return o, lse

    def kept(self):
        """int32 [B, Hkv, w_cap, top_k] view of the kept positions (windows compressed so far are valid)."""
        ptr, wcap = ctypes.c_void_p(0), ctypes.c_int32(0)
        _check(lib().lrsa_cache_kept(self.params.ref(), _p(self.buf), ctypes.byref(ptr), ctypes.byref(wcap)),
               "lrsa_cache_kept")
        off = ptr.value - self.buf.data_ptr()
        n = self.params.batch * self.params.n_kv_heads * wcap.value * self.params.top_k
        return self.buf[off:off + 4 * n].view(torch.int32).view(self.params.batch, self.params.n_kv_heads, wcap.value,
                                                                 self.params.top_k)

    def windows_compressed(self) -> int:
        p = self.params
        if self.n_tokens <= p.n_sink:
            return 0
        return max((self.n_tokens - 1 - p.n_sink) // p.lag - 1, 0)

    def status(self, stream=None) -> int:
        return lrsa_workspace_status(self.ws, stream)


class KVStore:
    """Condensed KV cache of one layer as plain tensors (see lrsa_store_t in the C header), for inference.  `dtype` of the
    kept rows: torch.bfloat16, torch.float8_e4m3fn or torch.int8, 8 bits with one scale per `block` rows and head.  `keep`: the rule
    by which a window is cut, "lag" (lrsa_score_select's) or "weight" (the attention weight its tokens have gathered: what
    they entered with, and what decode adds).  The tensors may be read and written between calls, or replaced by others of
    the same shape, type and device: anything else is refused by the next call.  Two stores share nothing.  (bf16 by "lag" is
    what KVCache holds, which takes 3 to 8 % less time for a token.)"""

    TYPES = {torch.bfloat16: 0, torch.float8_e4m3fn: 1, torch.int8: 2}
    RULES = {"lag": 0, "weight": 1}
    _TENSORS = ("k_list", "v_list", "k_scale", "v_scale", "k_recent", "v_recent", "weight", "idx")
    _checked = None   # when the tensors were last looked at: addresses, and aliases so that no other memory can be there

    def __init__(self, params: Params, dtype=torch.float8_e4m3fn, block: int = 64, keep: str = "weight", device="cuda"):
        if dtype not in self.TYPES or keep not in self.RULES:
            raise LrsaError(1, f"KVStore: dtype {dtype}, keep {keep!r}")
        self.params, self.dtype, self.block, self.keep = params, dtype, block, keep
        self._type, self._rule = self.TYPES[dtype], self.RULES[keep]
        self.n_tokens = 0
        want, ws = self._layout()
        for name in self._TENSORS:
            shape, kind = want[name]
            setattr(self, name, None if shape is None else torch.zeros(shape, dtype=kind, device=device))
        self.ws = new_workspace(ws, device)
        self._lse = torch.empty((params.batch, params.n_q_heads), dtype=torch.float32, device=device)   # what an lse looks like
        self._q_shape = torch.Size((params.batch, params.n_q_heads, params.head_dim))

    def _layout(self):
        """({tensor: (shape or None, type)}, bytes of workspace) as the library has them."""
        p, block = self.params, self.block
        st = lrsa_store_t(self._type, block, self._rule, 0)
        wcap, rows, ws = ctypes.c_int32(0), ctypes.c_int32(0), ctypes.c_size_t(0)
        _check(lib().lrsa_store_shape(p.ref(), ctypes.byref(st), ctypes.byref(wcap), ctypes.byref(rows), ctypes.byref(ws)),
               "lrsa_store_shape")
        self.rows_per_window = rows.value
        heads, n = (p.batch, p.n_kv_heads), wcap.value * rows.value
        kept = (heads + (n, p.head_dim), self.dtype)
        scale = (None if self.dtype == torch.bfloat16 else heads + (n // block,), torch.float32)
        recent = (heads + (p.n_sink + 2 * p.lag, p.head_dim), torch.bfloat16)
        return {"k_list": kept, "v_list": kept, "k_scale": scale, "v_scale": scale, "k_recent": recent, "v_recent": recent,
                "weight": (heads + (2 * p.lag,) if self.keep == "weight" else None, torch.float32),
                "idx": (heads + (wcap.value, p.top_k), torch.int32)}, ws.value

    def __setattr__(self, name, value):
        object.__setattr__(self, name, value)
        if name != "n_tokens":
            object.__setattr__(self, "_checked", None)

    def __getstate__(self):
        return {k: v for k, v in self.__dict__.items() if k != "_checked"}   # (addresses of this process)

    def _look(self, where):
        """Raises LRSA_ERR_INVALID_ARG unless the store's tensors are what its kernels read and write."""
        p, dev = self.params, self._lse.get_device()
        if (self.TYPES.get(self.dtype), self.RULES.get(self.keep)) != (self._type, self._rule) or \
                self._q_shape != (p.batch, p.n_q_heads, p.head_dim):
            raise LrsaError(1, f"{where}: dtype, rule, heads and batch of a store are those that it was made with")
        want, held = dict(self._layout()[0], ws=(tuple(self.ws.shape), torch.uint8)), []
        for name, (shape, kind) in want.items():
            t = getattr(self, name)
            if shape is None and t is None:
                continue
            if shape is None or not isinstance(t, torch.Tensor) or t.device != self._lse.device:
                what = "None" if shape is None else f"a tensor on {self._lse.device}"
                raise LrsaError(1, f"{where}: {name} of the store must be {what}")
            _expect(where, name + " of the store", t, shape, kind, dev)
            if t.untyped_storage().nbytes() < (t.storage_offset() + t.numel()) * t.element_size():
                raise LrsaError(1, f"{where}: {name} of the store has lost its memory")
            held.append(t.detach())
        object.__setattr__(self, "_checked", (None, None, held))

    def _device(self, where, name, t) -> int:
        dev = _device(where, name, t)
        if self._lse.get_device() != dev:
            raise LrsaError(1, f"{where}: the store is on {self._lse.device}, {name} on {t.device}")
        return dev

    def _parts(self, where, ws):
        """The store as the calls of csrc/pycall.c take it: type, block, rule, addresses.  The tensors are looked at when one
        has been replaced, or lies elsewhere than it did (that takes 21 us, the comparison 0.4).  ws: address of the
        workspace."""
        if self._checked is None:
            self._look(where)
        seen, scale_k, scale_v, weight = self._checked, self.k_scale, self.v_scale, self.weight
        parts = (self._type, self.block, self._rule, self.k_list.data_ptr(), self.v_list.data_ptr(),
                 None if scale_k is None else scale_k.data_ptr(), None if scale_v is None else scale_v.data_ptr(),
                 self.k_recent.data_ptr(), self.v_recent.data_ptr(), None if weight is None else weight.data_ptr(),
                 self.idx.data_ptr())
        if parts != seen[0] or ws != seen[1]:
            self._look(where)
            object.__setattr__(self, "_checked", (parts, ws, self._checked[2]))
        return parts

    def append(self, k_new, v_new, w_new=None, stream=None):
        """k_new, v_new: bf16 [B, Hkv, n_new, d].  w_new (keep="weight"): fp32 [B, Hkv, n_new], the weight that the tokens enter
        with (lrsa_attn_weights of a prompt); none: zero, unless the call compresses a window of its own tokens."""
        p, where, call = self.params, "lrsa_store_append", _calls()
        n_new = k_new.shape[2] if k_new.dim() == 4 else 0
        shape = (p.batch, p.n_kv_heads, n_new, p.head_dim)
        dev = self._device(where, "k_new", k_new)
        _expect(where, "k_new", k_new, shape, torch.bfloat16, dev)
        _expect(where, "v_new", v_new, shape, torch.bfloat16, dev)
        if w_new is not None:
            _expect(where, "w_new", w_new, shape[:3], torch.float32, dev)
        cp, ws = p.struct(), self.ws
        at = ws.data_ptr()
        status = call.store_append(ctypes.addressof(cp), *self._parts(where, at), k_new.data_ptr(), v_new.data_ptr(), _p(w_new),
                                   self.n_tokens, n_new, at, ws.numel(), _stream_of(stream, dev))
        if status:
            _check(status, where)
        self.n_tokens += n_new

    def decode(self, q, o=None, lse=None, stream=None):
        """q: bf16 [B, Hq, d], the query of the last token in the store.  Returns (o, lse); with keep="weight" the weights of
        the ring's tokens grow by those of the query."""
        where, call, like = "lrsa_store_decode", _call or _calls(), self._lse
        dev = self._device(where, "q", q)
        _expect(where, "q", q, self._q_shape, torch.bfloat16, dev)
        if o is None:
            o = torch.empty_like(q) if stream is None else _made(stream, q, torch.empty_like, q)
        else:
            _expect(where, "o", o, self._q_shape, torch.bfloat16, dev)
        if lse is None:
            lse = torch.empty_like(like) if stream is None else _made(stream, q, torch.empty_like, like)
        else:
            _expect(where, "lse", lse, like.shape, torch.float32, dev)
        cp, ws = self.params.struct(), self.ws
        at = ws.data_ptr()
        status = call.store_decode(ctypes.addressof(cp), *self._parts(where, at), q.data_ptr(), self.n_tokens, o.data_ptr(),
                                   lse.data_ptr(), at, ws.numel(), _stream_of(stream, dev))
        if status:
            _check(status, where)
        return o, lse

    def rows(self, k=None, v=None, stream=None):
        """What the kept rows of the windows compressed so far stand for: (k, v), fp32 [B, Hkv, windows * top_k, d]."""
        p, n, where, call = self.params, self.windows_compressed(), "lrsa_store_rows", _calls()
        shape = (p.batch, p.n_kv_heads, n * p.top_k, p.head_dim)
        dev = self._device(where, "the store", self._lse)
        if k is None:
            k = _made(stream, self._lse, torch.empty, shape, dtype=torch.float32, device=self._lse.device)
        else:
            _expect(where, "k", k, shape, torch.float32, dev)
        if v is None:
            v = _made(stream, k, torch.empty_like, k)
        else:
            _expect(where, "v", v, shape, torch.float32, dev)
        cp = p.struct()
        status = call.store_rows(ctypes.addressof(cp), *self._parts(where, self.ws.data_ptr()), n, k.data_ptr(), v.data_ptr(),
                                 _stream_of(stream, dev))
        if status:
            _check(status, where)
        return k, v

    def windows_compressed(self) -> int:
        p = self.params
        if self.n_tokens <= p.n_sink:
            return 0
        return max((self.n_tokens - 1 - p.n_sink) // p.lag - 1, 0)

    def status(self, stream=None) -> int:
        return lrsa_workspace_status(self.ws, stream)


class Rope:
    """The angles of a position rotation: cos, sin fp32 [positions, pairs], whatever base or scaling they were made with.  The first
    2 * pairs channels of a row are rotated, pairs (i, i + pairs), or neighbours (2i, 2i + 1) where `interleaved`.  The tables may be written
    between calls, or replaced by others (both: longer ones for a longer context); the next call takes them.  A captured call goes on with
    the memory that it was captured with."""

    _args = None     # what csrc/pycall.c takes of the tables, as they were when they were last looked at

    def __init__(self, cos, sin, interleaved: bool = False):
        self.cos, self.sin, self.interleaved = cos, sin, interleaved
        self._look("Rope")

    def __setattr__(self, name, value):
        object.__setattr__(self, name, value.detach() if isinstance(value, torch.Tensor) else value)
        object.__setattr__(self, "_args", None)
        object.__setattr__(self, "_held", None)

    def _look(self, where):
        """Raises LRSA_ERR_INVALID_ARG unless the tables are what the kernels read."""
        cos, sin = self.cos, self.sin
        for name, t in (("cos", cos), ("sin", sin)):
            if not isinstance(t, torch.Tensor) or t.dtype is not torch.float32 or t.dim() != 2 or not t.is_contiguous() or \
                    t.shape != cos.shape or t.device != cos.device or t.data_ptr() % 16:
                raise LrsaError(1, f"{where}: {name} of a rope must be a contiguous, 16-byte aligned float32 tensor [positions, pairs], "
                                   "the same for both")
            if t.untyped_storage().nbytes() < (t.storage_offset() + t.numel()) * t.element_size():
                raise LrsaError(1, f"{where}: {name} of the rope has lost its memory")
        if cos.shape[0] < 1 or cos.shape[1] < 8 or cos.shape[1] % 8:
            raise LrsaError(1, f"{where}: {cos.shape[1]} pairs of {cos.shape[0]} positions (pairs: a multiple of 8)")
        args = cos.data_ptr(), sin.data_ptr(), cos.shape[0], 2 * cos.shape[1], int(bool(self.interleaved))
        # (while the aliases are held no other memory can be at these addresses)
        for name, value in (("_dev", cos.get_device()), ("_numel", cos.numel()), ("_held", (cos.detach(), sin.detach())), ("_args", args)):
            object.__setattr__(self, name, value)
        return args

    @staticmethod
    def of_base(base: float, dim: int, n_positions: int, interleaved: bool = False, device="cuda") -> "Rope":
        """The usual table: pair i of `dim` channels turns by base ** (-2i / dim) a position.  Angles in 64 bits."""
        f = float(base) ** (-torch.arange(0, dim, 2, dtype=torch.float64) / dim)
        angle = torch.arange(n_positions, dtype=torch.float64)[:, None] * f
        return Rope(angle.cos().float().to(device), angle.sin().float().to(device), interleaved)

    def __getstate__(self):
        return {"cos": self.cos, "sin": self.sin, "interleaved": self.interleaved}

    def __setstate__(self, state):
        self.__init__(**state)


_NO_ROPE = (None, None, 0, 0, 0)


def _rope_args(where, rope, dev):
    if rope is None:
        return _NO_ROPE
    args = rope._args
    if args is None or rope.cos.data_ptr() != args[0] or rope.sin.data_ptr() != args[1] or rope.cos.numel() != rope._numel:
        args = rope._look(where)
    if rope._dev != dev:
        raise LrsaError(1, f"{where}: the rope is on {rope.cos.device}")
    return args


def lrsa_rotate(params: Params, Q, K, rope: Rope, positions=None, inverse: bool = False, Q_out=None, K_out=None, stream=None):
    """Position rotation of Q [B,Hq,N,d] and K [B,Hkv,N,d] (either may be None), in front of lrsa_score_select and lrsa_attn_fwd;
    inverse: its gradient, behind lrsa_attn_bwd.  positions: int32 [N]; none: a token's index in its sequence.  Q_out, K_out may be
    Q, K themselves.  Returns (Q_out, K_out)."""
    p, where, call = params, "lrsa_rotate", _call or _calls()
    first = Q if Q is not None else K
    if first is None:
        raise LrsaError(1, f"{where}: neither Q nor K")
    dev = _device(where, "Q" if Q is not None else "K", first)
    q_at, q_to, Q_out = _turned(where, "Q", Q, Q_out, (p.batch, p.n_q_heads, p.seq_len, p.head_dim), dev, stream)
    k_at, k_to, K_out = _turned(where, "K", K, K_out, (p.batch, p.n_kv_heads, p.seq_len, p.head_dim), dev, stream)
    if positions is not None:
        _expect(where, "positions", positions, (p.seq_len,), torch.int32, dev)
    cp = p.struct()
    status = call.rotate(ctypes.addressof(cp), q_at, k_at, q_to, k_to, *_rope_args(where, rope, dev), _p(positions), int(inverse),
                         _stream_of(stream, dev))
    if status:
        _check(status, where)
    return Q_out, K_out


def _turned(where, name, x, y, shape, dev, stream):
    """(address of x, address of y, y) of a tensor to be rotated; y is made where there is none."""
    if x is None:
        if y is not None:
            raise LrsaError(1, f"{where}: {name}_out without {name}")
        return None, None, None
    if x.dtype is not torch.bfloat16 or x.shape != shape or not x.is_contiguous() or x.get_device() != dev:
        _expect(where, name, x, shape, torch.bfloat16, dev)
    if y is None:
        y = torch.empty_like(x) if stream is None else _made(stream, x, torch.empty_like, x)
    elif y is not x:
        _expect(where, name + "_out", y, shape, torch.bfloat16, dev)
    return x.data_ptr(), y.data_ptr(), y


class _Space:
    """A workspace, and those that it has outgrown (a captured call may hold their addresses)."""

    def __init__(self, ws):
        self.ws, self.old = ws, []


class PagedCache:
    """Condensed KV cache of one layer for sequences of different lengths, in pages (lrsa_paged_* in the C header): k_pages and
    v_pages, bf16 [n_pages, Hkv, page, d], which may be replaced by others of that shape, type and device.  What the layers of a
    model share is the caller's, on the device: the page table (int32 [sequences, table_width]), the tokens in the cache (n_tokens, int32
    [sequences]) and where the new tokens of a sequence begin (cu_new, int32 [sequences + 1]).  Neither call changes them, so a step is
    attend (and append) for every layer, then n_tokens += the new tokens.  Counts and page numbers that cannot be used are told by status(),
    until it has been asked.
    The calls of a cache share its workspace, so they run one after the other, captured ones too; different caches share nothing, unless one is
    made `beside` another: then that one's workspace, its status and this rule are those of both (the layers of a model, whose calls run
    one after the other anyway; the attention of trees takes 40 MB at d = 128, a prompt of 32K tokens 34)."""

    MOST_NEW = 128   # new tokens of a sequence in an attend
    _seen = None     # where the pages were when they were last looked at,
    _held = None     # and aliases of them

    def __init__(self, params: Params, n_pages: int, page: int = 64, device="cuda", beside: "PagedCache | None" = None):
        self.params, self.page, self.n_pages = params, page, n_pages
        width, cap = ctypes.c_int32(0), ctypes.c_int32(0)
        _check(lib().lrsa_paged_shape(params.ref(), page, 0, 0, 0, ctypes.byref(width), ctypes.byref(cap), None), "lrsa_paged_shape")
        if n_pages < 1:
            raise LrsaError(1, f"PagedCache: {n_pages} pages")
        self.table_width, self.w_cap = width.value, cap.value
        self._shape = torch.Size((n_pages, params.n_kv_heads, page, params.head_dim))
        self.k_pages = torch.zeros(self._shape, dtype=torch.bfloat16, device=device)
        self.v_pages = torch.zeros(self._shape, dtype=torch.bfloat16, device=device)
        self._need = {}
        if beside is None:
            self._space = _Space(_cleared_workspace(self.workspace_bytes(1, 1, 1), device))
        elif not isinstance(beside, PagedCache) or beside.ws.device != self.k_pages.device:
            raise LrsaError(1, f"PagedCache: beside a cache on {self.k_pages.device}, got {getattr(getattr(beside, 'ws', None), 'device', beside)}")
        else:
            self._space = beside._space

    @property
    def ws(self):
        return self._space.ws

    @ws.setter
    def ws(self, ws):
        self._space.ws = ws

    @property
    def _old(self):
        return self._space.old

    def workspace_bytes(self, n_seqs: int, n_new: int, max_new: int) -> int:
        """What an attend of n_new tokens of n_seqs sequences, at most max_new each, takes; max_new = 0: an append."""
        out = ctypes.c_size_t(0)
        _check(lib().lrsa_paged_shape(self.params.ref(), self.page, n_seqs, n_new, max_new, None, None, ctypes.byref(out)), "lrsa_paged_shape")
        return out.value

    def _workspace(self, near, stream, *sizes):
        """The workspace, at least as large as a call of these sizes needs.  One that was outgrown stays where it is: a captured
        call may hold its address.  (The next is twice as large at least: all that were outgrown take no more than it does.)"""
        need = self._need.get(sizes)
        if need is None:
            if len(self._need) > 4096:
                self._need.clear()
            need = self._need[sizes] = self.workspace_bytes(*sizes)
        if self.ws.numel() < need:
            self._old.append(self.ws)
            self.ws = _made(stream, near, _cleared_workspace, max(need, 2 * self.ws.numel()), near.device)
        return self.ws

    def columns(self, n_tokens: int):
        """Columns of the page table that a sequence of n_tokens has reached: those that need a page."""
        p, size = self.params, self.page
        sinks, ring, kept = (-(-x // size) for x in (p.n_sink, p.lag, p.top_k))
        rest = max(n_tokens - p.n_sink, 0)
        cols = list(range(-(-min(n_tokens, p.n_sink) // size)))
        for g in range(2):
            cols += range(sinks + g * ring, sinks + g * ring - (-min(max(rest - g * p.lag, 0), p.lag) // size))
        first = sinks + 2 * ring
        return cols + list(range(first, first + max(rest // p.lag - 1, 0) * kept))

    def room(self, n_tokens):
        """How many tokens from n_tokens on (int32, on the device or the host) see in one attend what they would see one by one.  From there on
        a window more is condensed, and a deeper draft has seen it whole: a server that accepts at most so many drafts, which it can tell on the
        device, gets what single tokens give."""
        p = self.params
        return p.n_sink + (((n_tokens - p.n_sink) // p.lag - 1).clamp(min=0) + 2) * p.lag - n_tokens

    def _pages(self, where, name, first, table, n_tokens, cu_new):
        """(device, what csrc/pycall.c takes of the cache), when everything is what the kernels read and write.  The pages are looked at
        when they have been replaced, or lie elsewhere than they did."""
        dev = _device(where, name, first)
        if self._seen is None:
            self._look(where, dev)
        at_k, at_v = self.k_pages.data_ptr(), self.v_pages.data_ptr()
        if self._seen != (at_k, at_v, dev):
            self._look(where, dev)
            object.__setattr__(self, "_seen", (at_k, at_v, dev))
        shape, i32 = table.shape, torch.int32
        n = shape[0] if len(shape) == 2 else 0
        if table.dtype is not i32 or shape != (n, self.table_width) or not table.is_contiguous() or table.get_device() != dev:
            _expect(where, "table", table, (n, self.table_width), i32, dev)
        if n_tokens.dtype is not i32 or n_tokens.shape != (n,) or not n_tokens.is_contiguous() or n_tokens.get_device() != dev:
            _expect(where, "n_tokens", n_tokens, (n,), i32, dev)
        if cu_new.dtype is not i32 or cu_new.shape != (n + 1,) or not cu_new.is_contiguous() or cu_new.get_device() != dev:
            _expect(where, "cu_new", cu_new, (n + 1,), i32, dev)
        return dev, (self.page, self.n_pages, n, self.table_width, at_k, at_v, table.data_ptr(), n_tokens.data_ptr())

    def __setattr__(self, name, value):
        object.__setattr__(self, name, value)
        object.__setattr__(self, "_seen", None)
        if name in ("k_pages", "v_pages"):
            object.__setattr__(self, "_held", None)   # (the caller may want the room of the old ones)

    def __getstate__(self):
        return {k: v for k, v in self.__dict__.items() if k not in ("_seen", "_held")}   # (addresses of this process)

    def __setstate__(self, state):
        state = dict(state)
        if "_space" not in state:      # saved before caches could share one
            state["_space"] = _Space(_cleared_workspace(state["ws"].numel(), state["ws"].device))
        self.__dict__.update((k, v) for k, v in state.items() if k not in ("ws", "_old"))

    def _look(self, where, dev):
        """Raises LRSA_ERR_INVALID_ARG unless the pages are what the kernels read and write."""
        for name, t in (("k_pages", self.k_pages), ("v_pages", self.v_pages)):
            if not isinstance(t, torch.Tensor) or t.device != self.ws.device:
                raise LrsaError(1, f"{where}: {name} of the cache must be a tensor on {self.ws.device}")
            _expect(where, name + " of the cache", t, self._shape, torch.bfloat16, dev)
            if t.untyped_storage().nbytes() < (t.storage_offset() + t.numel()) * t.element_size():
                raise LrsaError(1, f"{where}: {name} of the cache has lost its memory")
        if self.ws.get_device() != dev:
            raise LrsaError(1, f"{where}: the workspace of the cache is on {self.ws.device}")
        # aliases: while they are held no other memory can be at these addresses
        object.__setattr__(self, "_held", (self.k_pages.detach(), self.v_pages.detach()))

    @staticmethod
    def _rows(where, name, t, shape, dev):
        """(address, strides) of rows [heads, n, d] with any strides between heads and tokens."""
        if t.dtype is not torch.bfloat16 or t.shape != shape or t.get_device() != dev:
            raise LrsaError(1, f"{where}: {name} must be a bfloat16 tensor of shape {shape} on cuda:{dev}, got {t.dtype} {tuple(t.shape)} on "
                               f"{t.device}")
        head, token, channel = t.stride()
        at = t.data_ptr()
        if channel != 1 or (head | token) & 7 or at & 15:
            head, token = head if shape[0] > 1 else 0, token if shape[1] > 1 else 0    # (of one head or token a stride is never used)
            if channel != 1 or (head | token) & 7 or at & 15:
                raise LrsaError(1, f"{where}: the rows of {name} must be contiguous and 16-byte aligned, got strides {t.stride()}")
        return at, head, token

    def append(self, k_new, v_new, table, n_tokens, cu_new, rows=None, rope=None, kept=None, stream=None):
        """The new tokens enter the cache: k_new, v_new bf16 [Hkv, tokens, d] with any strides, K rotated on the way unless rope is
        None.  rows (int32): new token i is row rows[i] of k_new and v_new (the accepted ones of drafts).  kept (int32 [sequences, Hkv,
        w_cap, top_k]) receives the kept positions of the windows that are cut."""
        p, where, call = self.params, "lrsa_paged_append", _call or _calls()
        dev, pages = self._pages(where, "k_new", k_new, table, n_tokens, cu_new)
        n_rows = k_new.shape[1] if k_new.dim() == 3 else 0
        shape = (p.n_kv_heads, n_rows, p.head_dim)
        k, v = self._rows(where, "k_new", k_new, shape, dev), self._rows(where, "v_new", v_new, shape, dev)
        n_new = n_rows
        if rows is not None:
            n_new = rows.shape[0] if rows.dim() == 1 else -1
            _expect(where, "rows", rows, (n_new,), torch.int32, dev)
        if kept is not None:
            _expect(where, "kept", kept, (pages[2], p.n_kv_heads, self.w_cap, p.top_k), torch.int32, dev)
        cp, ws = p.struct(), self._workspace(k_new, stream, pages[2], n_new, 0)
        status = call.paged_append(ctypes.addressof(cp), *pages, *k, *v, n_rows, cu_new.data_ptr(), n_new, _p(rows),
                                   *_rope_args(where, rope, dev), _p(kept), ws.data_ptr(), ws.numel(), _stream_of(stream, dev))
        if status:
            _check(status, where)

    def attend(self, q, k, v, table, n_tokens, cu_new, parent=None, rope=None, max_new=None, o=None, lse=None, stream=None):
        """Attention of every sequence's next token, or of a tree of drafted ones, over the cache: q bf16 [Hq, tokens, d], k, v bf16
        [Hkv, tokens, d] with any strides, not in the cache, rotated on the way unless rope is None.  parent (int32 [tokens]): which
        token of its sequence each one continues, -1: the cache; none: the one in front of it.  max_new: the most tokens of a
        sequence (at most 128); fewer than 17 rows, heads of a group times max_new, take the kernel for few.  Without it any sequence may
        have all of them: a step of single tokens says max_new=1, or it is taken for a tree (sixteen sequences with seven heads to a group: 112
        rows, three launches for two and 40 MB of workspace for 5).  Returns (o [Hq, tokens, d], lse fp32 [Hq, tokens]); o lies in memory as q
        does, token by token or head by head.  (Rows of a sequence that status() tells of may hold anything in an o that the call made.)"""
        p, where, call = self.params, "lrsa_paged_attend", _call or _calls()
        dev, pages = self._pages(where, "q", q, table, n_tokens, cu_new)
        n = q.shape[1] if q.dim() == 3 else 0
        Hq, d = p.n_q_heads, p.head_dim
        shape, kv_shape = (Hq, n, d), (p.n_kv_heads, n, d)
        qa, ka, va = self._rows(where, "q", q, shape, dev), self._rows(where, "k", k, kv_shape, dev), self._rows(where, "v", v, kv_shape, dev)
        if parent is not None:
            _expect(where, "parent", parent, (n,), torch.int32, dev)
        if o is None:
            dense = qa[1:] == (d, Hq * d) or qa[1:] == (n * d, d)
            if dense and stream is None:
                o = torch.empty_like(q)
            elif n > 1 and qa[2] > qa[1]:     # token by token
                o = _made(stream, q, torch.empty, (n, Hq, d), dtype=q.dtype, device=q.device).transpose(0, 1)
            else:
                o = _made(stream, q, torch.empty, shape, dtype=q.dtype, device=q.device)
            oa = (o.data_ptr(),) + o.stride()[:2]
        else:
            oa = self._rows(where, "o", o, shape, dev)
            if (Hq > 1 and oa[1] < d) or (n > 1 and oa[2] < d):
                raise LrsaError(1, f"{where}: rows of o overlap, strides {o.stride()}")
        if lse is None:
            lse = torch.empty((Hq, n), dtype=torch.float32, device=q.device) if stream is None else \
                _made(stream, q, torch.empty, (Hq, n), dtype=torch.float32, device=q.device)
        else:
            _expect(where, "lse", lse, (Hq, n), torch.float32, dev)
        if max_new is None:
            max_new = max(1, min(n, self.MOST_NEW))
        cp, ws = p.struct(), self._workspace(q, stream, pages[2], n, max_new)
        status = call.paged_attend(ctypes.addressof(cp), *pages, *qa, *ka, *va, cu_new.data_ptr(), n, max_new, _p(parent),
                                   *_rope_args(where, rope, dev), *oa, lse.data_ptr(), ws.data_ptr(), ws.numel(), _stream_of(stream, dev))
        if status:
            _check(status, where)
        return o, lse

    def status(self, stream=None) -> int:
        """What the calls of this cache have found since this was last asked, in whichever workspace they ran, replays of captured ones too: 0, 1
        (counts, page numbers, rows or parents that cannot be used) or 5 (a bounded wait ran out).  Synchronises the stream; calls on others are
        done by then, or told the next time.  (A workspace that a call makes while it is captured starts anew with every replay.)"""
        at = _stream(stream)
        return max(lib().lrsa_paged_status(ws.data_ptr(), at) for ws in (*self._old, self.ws))
