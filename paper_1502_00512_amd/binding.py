"""Thin ctypes binding of include/rnnlm.h: argument marshalling only.

Every step of the path runs in the HIP library; PyTorch only owns device memory and
streams.  Function names mirror the C ABI.  Importing this module needs the built
librnnlm_hip.so next to it (see build.py) and raises if it is missing: there is no
fallback path.
"""
from __future__ import annotations

import ctypes as C
import os

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "librnnlm_hip.so")

RNNLM_FP32 = 0
RNNLM_BF16_FP32MASTER = 1
RNNLM_DTYPE_FP32, RNNLM_DTYPE_BF16 = 0, 1
RNNLM_EXCHANGE_AUTO, RNNLM_EXCHANGE_CHIP_WIDE, RNNLM_EXCHANGE_XCD_LOCAL = 0, 1, 2

SYMBOLS = [
    "rnnlm_workspace_bytes", "rnnlm_init", "rnnlm_free", "rnnlm_stream_chunk", "rnnlm_forward_logprob",
    "rnnlm_train_chunk", "rnnlm_grad_chunk", "rnnlm_perplexity", "rnnlm_reset_state",
    "rnnlm_sync_compute_copies", "rnnlm_check", "rnnlm_sort_segments", "rnnlm_status_string",
    "rnnlm_profile_enable", "rnnlm_profile_read", "rnnlm_set_barrier_spin_limit", "rnnlm_measure_peaks",
    "rnnlm_nce_train_chunk", "rnnlm_nce_grad_chunk", "rnnlm_forward_score",
    "rnnlm_train_chunk_rmsprop", "rnnlm_nce_train_chunk_rmsprop",
    "rnnlm_grad_chunk_compressed", "rnnlm_quantize_weights", "rnnlm_forward_score_shortlist",
    "rnnlm_set_recurrent_exchange", "rnnlm_sort_segments_static",
    "rnnlm_top_logits_workspace_bytes", "rnnlm_top_logits", "rnnlm_distill_loss", "rnnlm_verify_workspace_bytes",
    "rnnlm_verify_drafts", "rnnlm_forward_logits", "rnnlm_distill_train_chunk", "rnnlm_distill_grad_chunk",
    "rnnlm_distill_grad_chunk_compressed", "rnnlm_verify_chunk",
]
SIZES = ["rnnlm_workspace_bytes", "rnnlm_top_logits_workspace_bytes", "rnnlm_verify_workspace_bytes"]  # return bytes

STAGES = ["prep", "rnn_fwd", "out_fwd", "stats", "softmax_grad", "out_bwd_h", "rnn_bwd", "out_bwd_w", "rec_w", "emb", "reduce",
          "nce_score", "nce_grad", "nce_bwd_h", "nce_bwd_w", "nce_update", "rmsprop", "proj"]


class rnnlm_config(C.Structure):
    _fields_ = [("V", C.c_int32), ("H", C.c_int32), ("B", C.c_int32), ("T_max", C.c_int32),
                ("precision", C.c_int32), ("device", C.c_int32), ("K_max", C.c_int32), ("rmsprop", C.c_int32),
                ("P", C.c_int32)]


class rnnlm_rmsprop_state(C.Structure):
    _fields_ = [("rE", C.c_void_p), ("rU", C.c_void_p), ("rWo", C.c_void_p), ("rb", C.c_void_p)]


class rnnlm_buffers(C.Structure):
    _fields_ = [("E", C.c_void_p), ("U", C.c_void_p), ("Wo", C.c_void_p), ("b", C.c_void_p),
                ("h_state", C.c_void_p), ("workspace", C.c_void_p), ("workspace_bytes", C.c_size_t),
                ("A", C.c_void_p), ("C", C.c_void_p)]


class rnnlm_quantized(C.Structure):
    _fields_ = [("qE", C.c_void_p), ("sE", C.c_void_p), ("qA", C.c_void_p), ("sA", C.c_void_p),
                ("qU", C.c_void_p), ("sU", C.c_void_p), ("qC", C.c_void_p), ("sC", C.c_void_p)]


class rnnlm_distill(C.Structure):
    _fields_ = [("ids", C.c_void_p), ("vals", C.c_void_p), ("lse", C.c_void_p), ("weight", C.c_void_p), ("K", C.c_int32),
                ("tau", C.c_float), ("alpha", C.c_float), ("logits", C.c_void_p), ("ld", C.c_int64)]


class rnnlm_verify(C.Structure):
    _fields_ = [("draft", C.c_void_p), ("ld_draft", C.c_int64), ("lengths", C.c_void_p), ("u", C.c_void_p), ("tau", C.c_float),
                ("tau_draft", C.c_float), ("logits", C.c_void_p), ("ld", C.c_int64), ("workspace", C.c_void_p),
                ("workspace_bytes", C.c_size_t)]


class RnnlmError(RuntimeError):
    def __init__(self, status: int, what: str):
        super().__init__(f"{what}: {status_string(status)} ({status})")
        self.status = status


_lib = None


def load():
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is not built; run `python -m paper_1502_00512_amd.build` "
                          "(there is no fallback path)")
    lib = C.CDLL(LIB_PATH)
    vp, i32, i64 = C.c_void_p, C.c_int32, C.c_int64
    lib.rnnlm_workspace_bytes.argtypes = [C.POINTER(rnnlm_config)]
    lib.rnnlm_init.argtypes = [C.POINTER(rnnlm_config), C.POINTER(rnnlm_buffers), C.POINTER(vp)]
    lib.rnnlm_free.argtypes = [vp]
    lib.rnnlm_free.restype = None
    lib.rnnlm_stream_chunk.argtypes = [vp, vp, i64, i64, i32, vp, vp, vp]
    lib.rnnlm_forward_logprob.argtypes = [vp, vp, vp, i32, vp, vp]
    lib.rnnlm_train_chunk.argtypes = [vp, vp, vp, i32, C.c_float, vp, vp, vp]
    lib.rnnlm_grad_chunk.argtypes = [vp, vp, vp, i32, vp, vp, vp, vp, vp, vp]
    lib.rnnlm_perplexity.argtypes = [vp, vp, i64, i32, C.POINTER(C.c_double), C.POINTER(i64), vp]
    lib.rnnlm_reset_state.argtypes = [vp, vp]
    lib.rnnlm_sync_compute_copies.argtypes = [vp, vp]
    lib.rnnlm_check.argtypes = [vp, vp]
    lib.rnnlm_sort_segments.argtypes = [vp, vp, i32, vp, vp, vp, vp]
    lib.rnnlm_set_barrier_spin_limit.argtypes = [vp, C.c_uint32]
    lib.rnnlm_set_recurrent_exchange.argtypes = [vp, i32]
    lib.rnnlm_sort_segments_static.argtypes = [vp, i32, i32, i32, vp, vp, vp, vp, vp]
    lib.rnnlm_measure_peaks.argtypes = [vp, C.POINTER(C.c_double), C.POINTER(C.c_double), C.POINTER(C.c_double), vp]
    f32 = C.c_float
    lib.rnnlm_nce_train_chunk.argtypes = [vp, vp, vp, i32, vp, i32, vp, f32, f32, vp, vp, vp]
    lib.rnnlm_nce_grad_chunk.argtypes = [vp, vp, vp, i32, vp, i32, vp, f32, vp, vp, vp, vp, vp, vp]
    lib.rnnlm_train_chunk_rmsprop.argtypes = [vp, vp, vp, i32, f32, f32, f32, C.POINTER(rnnlm_rmsprop_state), vp, vp, vp]
    lib.rnnlm_nce_train_chunk_rmsprop.argtypes = [vp, vp, vp, i32, vp, i32, vp, f32, f32, f32, f32,
                                                  C.POINTER(rnnlm_rmsprop_state), vp, vp, vp]
    lib.rnnlm_forward_score.argtypes = [vp, vp, vp, i32, f32, vp, vp]
    lib.rnnlm_forward_score_shortlist.argtypes = [vp, vp, vp, i32, i32, f32, vp, vp]
    lib.rnnlm_grad_chunk_compressed.argtypes = [vp, vp, vp, i32, vp, vp, vp, vp, vp, vp, vp]
    lib.rnnlm_quantize_weights.argtypes = [vp, C.POINTER(rnnlm_quantized), vp]
    lib.rnnlm_top_logits_workspace_bytes.argtypes = [i64, i32, i32, i32]
    lib.rnnlm_top_logits.argtypes = [vp, i32, i64, i32, i64, i32, f32, vp, vp, vp, vp, C.c_size_t, vp]
    lib.rnnlm_distill_loss.argtypes = [vp, i32, i64, i32, i64, vp, vp, i32, vp, vp, vp, f32, f32, f32, vp, vp, vp, i64, vp, vp]
    lib.rnnlm_verify_workspace_bytes.argtypes = [i32, i32, i32]
    lib.rnnlm_verify_drafts.argtypes = [vp, i64, vp, i64, i32, i32, i32, i32, vp, vp, vp, f32, f32, vp, vp, vp, vp, C.c_size_t, vp]
    lib.rnnlm_forward_logits.argtypes = [vp, vp, i32, vp, i64, vp]
    lib.rnnlm_distill_train_chunk.argtypes = [vp, vp, vp, i32, C.POINTER(rnnlm_distill), f32, vp, vp, vp]
    lib.rnnlm_distill_grad_chunk.argtypes = [vp, vp, vp, i32, C.POINTER(rnnlm_distill), vp, vp, vp, vp, vp, vp]
    lib.rnnlm_distill_grad_chunk_compressed.argtypes = [vp, vp, vp, i32, C.POINTER(rnnlm_distill), vp, vp, vp, vp, vp, vp, vp]
    lib.rnnlm_verify_chunk.argtypes = [vp, vp, i32, C.POINTER(rnnlm_verify), vp, vp, vp]
    for name in SIZES:
        getattr(lib, name).restype = C.c_size_t
    lib.rnnlm_profile_enable.argtypes = [vp, C.c_uint32]
    lib.rnnlm_profile_read.argtypes = [vp, i32, C.POINTER(C.c_double), C.POINTER(i64)]
    lib.rnnlm_status_string.argtypes = [C.c_int]
    lib.rnnlm_status_string.restype = C.c_char_p
    for name in SYMBOLS:
        if name not in SIZES + ["rnnlm_free", "rnnlm_status_string"]:
            getattr(lib, name).restype = C.c_int
    _lib = lib
    return lib


def status_string(status: int) -> str:
    return load().rnnlm_status_string(int(status)).decode()


def _ok(rc: int, what: str):
    if rc != 0:
        raise RnnlmError(rc, what)


def _ptr(t):
    return None if t is None else C.c_void_p(t.data_ptr())


def _stream(stream):
    import torch
    s = torch.cuda.current_stream() if stream is None else stream
    return C.c_void_p(s.cuda_stream)


def rnnlm_workspace_bytes(V, H, B, T_max, precision, device=0, K_max=0, rmsprop=0, P=0) -> int:
    cfg = rnnlm_config(V, H, B, T_max, precision, device, K_max, rmsprop, P)
    return int(load().rnnlm_workspace_bytes(C.byref(cfg)))


def rnnlm_sort_segments_static(x, V: int, perm, seg_start, nseg, range_flag=None, stream=None):
    """The handle-free call: x int32[T][B] and the three outputs are device tensors the caller allocated."""
    _ok(load().rnnlm_sort_segments_static(_ptr(x), x.shape[0], x.shape[1], V, _ptr(perm), _ptr(seg_start), _ptr(nseg),
                                          _ptr(range_flag), _stream(stream)), "rnnlm_sort_segments_static")


# -- operators on arrays of logits: device tensors, no handle ------------------------------------------------
# (A call's checks are a good part of its time where its kernels take some 5 us: no message is formed unless it is raised.)
def _refuse(call: str, what: str):
    raise RnnlmError(-1, f"{call}: {what}")


def _rows(call, name, t, like=None):
    """(rows, V, elements from row to row, dtype) of a tensor [..., V] whose rows are evenly spaced and dense in V; like: a
    tensor whose device and type it has to share."""
    import torch
    dtype = t.dtype
    if not t.is_cuda or (dtype is not torch.float32 and dtype is not torch.bfloat16):
        _refuse(call, f"{name}: float32 or bfloat16 rows on a GPU are wanted")
    if like is not None and (dtype is not like.dtype or t.get_device() != like.get_device()):
        _refuse(call, f"{name}: another type or device than the other logits'")
    shape, stride = t.shape, t.stride()
    if len(shape) < 2 or (V := shape[-1]) < 1 or (stride[-1] != 1 and V > 1):
        _refuse(call, f"{name}: rows of neighbouring logits are wanted")
    rows, ld = 1, None
    for i in range(len(shape) - 2, -1, -1):
        n = shape[i]
        if n != 1:
            if ld is None:
                ld = stride[i]
            if stride[i] != ld * rows:
                _refuse(call, f"{name}: rows have to be evenly spaced")
            rows *= n
    if ld is None or rows == 0:
        ld = V
    elif ld < V:
        _refuse(call, f"{name}: rows overlap")
    return rows, V, ld, RNNLM_DTYPE_FP32 if dtype is torch.float32 else RNNLM_DTYPE_BF16


def _at(call, name, t, dtype, n, device, last=None):
    """Address of a contiguous tensor of n elements (its last dimension, if given) on that device; None of None."""
    if t is None:
        return None
    if t.dtype is not dtype or t.numel() != n or t.get_device() != device or not t.is_contiguous() or (last is not None and t.shape[-1] != last):
        _refuse(call, f"{name}: a contiguous {dtype} tensor of {n} elements on device {device} is wanted"
                + ("" if last is None else f", {last} in its last dimension"))
    return t.data_ptr()


def _scratch(call, t, device, nbytes):
    """(address, bytes, the tensor) of the workspace given, or of a new one of nbytes() bytes."""
    import torch
    if t is None:
        t = torch.empty(max(nbytes(), 1), dtype=torch.uint8, device=torch.device("cuda", device))
    elif t.get_device() != device or not t.is_contiguous():
        _refuse(call, "workspace: a contiguous tensor on the logits' device is wanted")
    return t.data_ptr(), t.nbytes, t


def _on(call, stream, device, f, *args):
    """f(*args) with `stream` the current one, so that what is allocated in there (scratch that is dropped when the call
    returns, above all) comes from this stream's pool: memory of another one's may still be at work there, or be again."""
    import torch
    if stream.device.index != device:
        _refuse(call, f"stream: one of device {device} is wanted")
    with torch.cuda.stream(stream):
        return f(*args)


def _launch(device, f, *args):
    """f(*args, the current stream of that device) with that device current."""
    import torch
    stream = torch.cuda.current_stream(device).cuda_stream
    if torch.cuda.current_device() == device:
        return f(*args, stream)
    with torch.cuda.device(device):
        return f(*args, stream)


def rnnlm_top_logits_workspace_bytes(rows: int, V: int, K: int, dtype: int) -> int:
    return int(load().rnnlm_top_logits_workspace_bytes(rows, V, K, dtype))


def rnnlm_top_logits(logits, K: int, tau: float = 1.0, ids=None, vals=None, lse=None, workspace=None, stream=None):
    """logits: float32 or bfloat16 [..., V], rows evenly spaced.  Returns (ids int32 [..., K], vals float32 [..., K],
    lse float32 [...]); tensors given for them, and a workspace, are used."""
    import torch
    call = "rnnlm_top_logits"
    rows, V, ld, dt = _rows(call, "logits", logits)
    if stream is not None:
        return _on(call, stream, logits.get_device(), rnnlm_top_logits, logits, K, tau, ids, vals, lse, workspace)
    dev, lead = logits.get_device(), logits.shape[:-1]
    if not 1 <= K <= V:
        _refuse(call, f"K = {K} of V = {V}")
    ids = torch.empty(*lead, K, dtype=torch.int32, device=logits.device) if ids is None else ids
    vals = torch.empty(*lead, K, dtype=torch.float32, device=logits.device) if vals is None else vals
    lse = torch.empty(lead, dtype=torch.float32, device=logits.device) if lse is None else lse
    at, nbytes, _keep = _scratch(call, workspace, dev, lambda: rnnlm_top_logits_workspace_bytes(rows, V, K, dt))
    _ok(_launch(dev, load().rnnlm_top_logits, logits.data_ptr(), dt, rows, V, ld, K, tau,
                _at(call, "ids", ids, torch.int32, rows * K, dev, K), _at(call, "vals", vals, torch.float32, rows * K, dev, K),
                _at(call, "lse", lse, torch.float32, rows, dev), at, nbytes), call)
    return ids, vals, lse


def rnnlm_distill_loss(logits, ids, vals, lse=None, y=None, weight=None, tau: float = 1.0, alpha: float = 1.0,
                       scale: float = 1.0, loss=None, dlogits=None, sum_loss=None, range_flag=None, stream=None):
    """logits: float32 or bfloat16 [..., V]; ids, vals [..., K]: the teacher's lists; lse [...]: the teacher's, or None.
    Returns loss float32 [...].  dlogits (a tensor like logits, or logits itself) receives the gradient; sum_loss float64 [1]."""
    import torch
    call, f32, i32 = "rnnlm_distill_loss", torch.float32, torch.int32
    rows, V, ld, dt = _rows(call, "logits", logits)
    if stream is not None:
        return _on(call, stream, logits.get_device(), rnnlm_distill_loss, logits, ids, vals, lse, y, weight, tau, alpha, scale, loss,
                   dlogits, sum_loss, range_flag)
    dev, K = logits.get_device(), ids.shape[-1]
    loss = torch.empty(logits.shape[:-1], dtype=f32, device=logits.device) if loss is None else loss
    z, dz, ldd = logits.data_ptr(), None, 0
    if dlogits is not None:
        if dlogits.shape != logits.shape:
            _refuse(call, "dlogits: the logits' shape is wanted")
        dz, ldd = dlogits.data_ptr(), _rows(call, "dlogits", dlogits, logits)[2]
        if dz == z and rows <= 1:  # in place (one row has no distance to the next)
            ldd = ld
    _ok(_launch(dev, load().rnnlm_distill_loss, z, dt, rows, V, ld, _at(call, "ids", ids, i32, rows * K, dev, K),
                _at(call, "vals", vals, f32, rows * K, dev, K), K, _at(call, "lse", lse, f32, rows, dev),
                _at(call, "y", y, i32, rows, dev), _at(call, "weight", weight, f32, rows, dev), tau, alpha, scale,
                _at(call, "loss", loss, f32, rows, dev), _at(call, "sum_loss", sum_loss, torch.float64, 1, dev), dz, ldd,
                _at(call, "range_flag", range_flag, i32, 1, dev)), call)
    return loss


def rnnlm_verify_workspace_bytes(K: int, B: int, V: int) -> int:
    return int(load().rnnlm_verify_workspace_bytes(K, B, V))


def rnnlm_verify_drafts(target, drafts, u, draft=None, lengths=None, tau: float = 1.0, tau_draft: float = 1.0, accepted=None,
                        tokens=None, workspace=None, range_flag=None, stream=None):
    """target: float32 or bfloat16 [K+1][B][V]; drafts int32 [K][B] (K = 0: None); u float32 [K+1][B]; draft [K][B][V] or None:
    drafts without probabilities; lengths int32 [B] or None.  Returns (accepted int32 [B], tokens int32 [K+1][B])."""
    import torch
    call, i32 = "rnnlm_verify_drafts", torch.int32
    rows, V, ld, dt = _rows(call, "target", target)
    if stream is not None:
        return _on(call, stream, target.get_device(), rnnlm_verify_drafts, target, drafts, u, draft, lengths, tau, tau_draft, accepted,
                   tokens, workspace, range_flag)
    if target.dim() != 3 or rows == 0:
        _refuse(call, "target: [K+1][B][V] is wanted")
    K, B, dev = target.shape[0] - 1, target.shape[1], target.get_device()
    q, ldd = None, 0
    if draft is not None and K > 0:
        if tuple(draft.shape) != (K, B, V):
            _refuse(call, f"draft: [{K}][{B}][{V}] is wanted")
        q, ldd = draft.data_ptr(), _rows(call, "draft", draft, target)[2]
    if drafts is None and K > 0:
        _refuse(call, "drafts are wanted")
    accepted = torch.empty(B, dtype=i32, device=target.device) if accepted is None else accepted
    tokens = torch.empty(K + 1, B, dtype=i32, device=target.device) if tokens is None else tokens
    at, nbytes, _keep = _scratch(call, workspace, dev, lambda: rnnlm_verify_workspace_bytes(K, B, V))
    _ok(_launch(dev, load().rnnlm_verify_drafts, target.data_ptr(), ld, q, ldd, dt, K, B, V,
                _at(call, "drafts", drafts, i32, K * B, dev, B) if K > 0 else None, _at(call, "lengths", lengths, i32, B, dev),
                _at(call, "u", u, torch.float32, rows, dev, B), tau, tau_draft, _at(call, "accepted", accepted, i32, B, dev),
                _at(call, "tokens", tokens, i32, rows, dev, B), _at(call, "range_flag", range_flag, i32, 1, dev), at, nbytes), call)
    return accepted, tokens


class Rnnlm:
    """Owns the torch tensors (masters, state, workspace) and the library handle.

    Plain architecture: E[V][H], U, Wo[V][H], b.  Compressed architecture (Sec. 5.4): pass Wo=None and
    A[H][P], C[P][H]; then E is the tied word matrix [V][P]."""

    def __init__(self, E, U, Wo, b, B: int, T_max: int, precision: int, device: int = 0, K_max: int = 0,
                 rmsprop: bool = False, r_init: float = 1.0, A=None, C_=None):
        import torch
        self.lib = load()
        dev = torch.device("cuda", device)
        f = lambda a: torch.as_tensor(a, dtype=torch.float32).contiguous().to(dev).clone()
        self.E, self.U, self.b = f(E), f(U), f(b)
        self.H = self.U.shape[0]
        self.V = self.E.shape[0]
        self.P = 0
        self.Wo = self.A = self.C = None
        if A is not None:
            assert Wo is None and C_ is not None
            self.A, self.C = f(A), f(C_)
            self.P = self.E.shape[1]
            assert self.A.shape == (self.H, self.P) and self.C.shape == (self.P, self.H)
        else:
            self.Wo = f(Wo)
            assert self.E.shape == (self.V, self.H) and self.Wo.shape == (self.V, self.H)
        self.B, self.T_max, self.precision, self.device = int(B), int(T_max), int(precision), dev
        assert self.U.shape == (self.H, self.H) and self.b.shape == (self.V,)
        self.h_state = torch.zeros(self.B, self.H, dtype=torch.float32, device=dev)
        self.K_max = int(K_max)
        cfg = rnnlm_config(self.V, self.H, self.B, self.T_max, self.precision, device, self.K_max, int(bool(rmsprop)),
                           self.P)
        if rmsprop:  # the caller-owned statistics, all starting at r_init
            fill = lambda *shp: torch.full(shp, float(r_init), dtype=torch.float32, device=dev)
            self.rE, self.rU, self.rWo, self.rb = fill(self.V), fill(self.H, self.H), fill(self.V), fill(self.V)
            self.rms_state = rnnlm_rmsprop_state(self.rE.data_ptr(), self.rU.data_ptr(), self.rWo.data_ptr(),
                                                 self.rb.data_ptr())
        nbytes = int(self.lib.rnnlm_workspace_bytes(C.byref(cfg)))
        if nbytes == 0:
            raise RnnlmError(-1, "rnnlm_workspace_bytes")
        self.workspace = torch.empty(nbytes, dtype=torch.uint8, device=dev)
        opt = lambda t: None if t is None else t.data_ptr()
        buf = rnnlm_buffers(self.E.data_ptr(), self.U.data_ptr(), opt(self.Wo), self.b.data_ptr(),
                            self.h_state.data_ptr(), self.workspace.data_ptr(), nbytes, opt(self.A), opt(self.C))
        self.handle = C.c_void_p()
        torch.cuda.synchronize(dev)
        _ok(self.lib.rnnlm_init(C.byref(cfg), C.byref(buf), C.byref(self.handle)), "rnnlm_init")

    def close(self):
        if getattr(self, "handle", None):
            import torch
            torch.cuda.synchronize(self.device)
            self.lib.rnnlm_free(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # -- the calls of the C ABI, same names ----------------------------------------------------
    def rnnlm_stream_chunk(self, tok, k: int, T: int, x=None, y=None, stream=None):
        import torch
        if stream is not None:
            return _on("rnnlm_stream_chunk", stream, self.device.index, self.rnnlm_stream_chunk, tok, k, T, x, y)
        if x is None:
            x = torch.empty(T, self.B, dtype=torch.int32, device=self.device)
            y = torch.empty(T, self.B, dtype=torch.int32, device=self.device)
        _ok(self.lib.rnnlm_stream_chunk(self.handle, _ptr(tok), tok.numel(), k, T, _ptr(x), _ptr(y), _stream(None)),
            "rnnlm_stream_chunk")
        return x, y

    def rnnlm_forward_logprob(self, x, y, logp=None, stream=None):
        import torch
        if stream is not None:
            return _on("rnnlm_forward_logprob", stream, self.device.index, self.rnnlm_forward_logprob, x, y, logp)
        T = x.shape[0]
        if logp is None:
            logp = torch.empty(T, self.B, dtype=torch.float32, device=self.device)
        _ok(self.lib.rnnlm_forward_logprob(self.handle, _ptr(x), _ptr(y), T, _ptr(logp), _stream(None)),
            "rnnlm_forward_logprob")
        return logp

    def rnnlm_train_chunk(self, x, y, lr: float, logp=None, sum_logp=None, stream=None):
        _ok(self.lib.rnnlm_train_chunk(self.handle, _ptr(x), _ptr(y), x.shape[0], lr, _ptr(logp), _ptr(sum_logp),
                                       _stream(stream)), "rnnlm_train_chunk")

    def rnnlm_grad_chunk(self, x, y, want_logp=True, stream=None):
        import torch
        if stream is not None:
            return _on("rnnlm_grad_chunk", stream, self.device.index, self.rnnlm_grad_chunk, x, y, want_logp)
        z = lambda *s: torch.empty(*s, dtype=torch.float32, device=self.device)
        dE, dU, dWo, db = z(self.V, self.H), z(self.H, self.H), z(self.V, self.H), z(self.V)
        logp = z(x.shape[0], self.B) if want_logp else None
        _ok(self.lib.rnnlm_grad_chunk(self.handle, _ptr(x), _ptr(y), x.shape[0], _ptr(dE), _ptr(dU), _ptr(dWo),
                                      _ptr(db), _ptr(logp), _stream(None)), "rnnlm_grad_chunk")
        return dict(gE=dE, gU=dU, gWo=dWo, gb=db, logp=logp)

    def rnnlm_grad_chunk_compressed(self, x, y, want_logp=True, stream=None):
        import torch
        if stream is not None:
            return _on("rnnlm_grad_chunk_compressed", stream, self.device.index, self.rnnlm_grad_chunk_compressed, x, y, want_logp)
        z = lambda *s: torch.empty(*s, dtype=torch.float32, device=self.device)
        dE, dA, dU, dC, db = z(self.V, self.P), z(self.H, self.P), z(self.H, self.H), z(self.P, self.H), z(self.V)
        logp = z(x.shape[0], self.B) if want_logp else None
        _ok(self.lib.rnnlm_grad_chunk_compressed(self.handle, _ptr(x), _ptr(y), x.shape[0], _ptr(dE), _ptr(dA),
                                                 _ptr(dU), _ptr(dC), _ptr(db), _ptr(logp), _stream(None)),
            "rnnlm_grad_chunk_compressed")
        return dict(gE=dE, gA=dA, gU=dU, gC=dC, gb=db, logp=logp)

    def rnnlm_quantize_weights(self, stream=None):
        """Returns dict name -> (codes int8 tensor, scale float tensor); the model then runs on the quantised values."""
        import torch
        if stream is not None:
            return _on("rnnlm_quantize_weights", stream, self.device.index, self.rnnlm_quantize_weights)
        out = {}
        ptrs = []
        for name, W in (("E", self.E), ("A", self.A), ("U", self.U), ("C", self.C)):
            q = torch.empty(W.shape, dtype=torch.int8, device=self.device)
            s = torch.empty(W.shape[0], dtype=torch.float32, device=self.device)
            out[name] = (q, s)
            ptrs += [q.data_ptr(), s.data_ptr()]
        qs = rnnlm_quantized(*ptrs)
        _ok(self.lib.rnnlm_quantize_weights(self.handle, C.byref(qs), _stream(None)), "rnnlm_quantize_weights")
        return out

    def rnnlm_perplexity(self, tok, T: int, stream=None):
        ppl = C.c_double(0.0)
        scored = C.c_int64(0)
        _ok(self.lib.rnnlm_perplexity(self.handle, _ptr(tok), tok.numel(), T, C.byref(ppl), C.byref(scored),
                                      _stream(stream)), "rnnlm_perplexity")
        return ppl.value, scored.value

    def rnnlm_train_chunk_rmsprop(self, x, y, lr: float, rho: float, eps: float, logp=None, sum_logp=None,
                                  stream=None):
        state = getattr(self, "rms_state", None)
        _ok(self.lib.rnnlm_train_chunk_rmsprop(self.handle, _ptr(x), _ptr(y), x.shape[0], lr, rho, eps,
                                               C.byref(state) if state is not None else None, _ptr(logp),
                                               _ptr(sum_logp), _stream(stream)), "rnnlm_train_chunk_rmsprop")

    def rnnlm_nce_train_chunk_rmsprop(self, x, y, noise, lnq, lnZ: float, lr: float, rho: float, eps: float, J=None,
                                      sum_J=None, stream=None):
        state = getattr(self, "rms_state", None)
        _ok(self.lib.rnnlm_nce_train_chunk_rmsprop(self.handle, _ptr(x), _ptr(y), x.shape[0], _ptr(noise),
                                                   noise.numel(), _ptr(lnq), lnZ, lr, rho, eps,
                                                   C.byref(state) if state is not None else None, _ptr(J),
                                                   _ptr(sum_J), _stream(stream)), "rnnlm_nce_train_chunk_rmsprop")

    def rnnlm_forward_score(self, x, y, lnZ: float = 0.0, score=None, stream=None):
        import torch
        if stream is not None:
            return _on("rnnlm_forward_score", stream, self.device.index, self.rnnlm_forward_score, x, y, lnZ, score)
        T = x.shape[0]
        if score is None:
            score = torch.empty(T, self.B, dtype=torch.float32, device=self.device)
        _ok(self.lib.rnnlm_forward_score(self.handle, _ptr(x), _ptr(y), T, lnZ, _ptr(score), _stream(None)),
            "rnnlm_forward_score")
        return score

    def rnnlm_forward_score_shortlist(self, x, cand, lnZ: float = 0.0, score=None, stream=None):
        import torch
        if stream is not None:
            return _on("rnnlm_forward_score_shortlist", stream, self.device.index, self.rnnlm_forward_score_shortlist, x, cand, lnZ, score)
        T, C_ = x.shape[0], cand.shape[2]
        if score is None:
            score = torch.empty(T, self.B, C_, dtype=torch.float32, device=self.device)
        _ok(self.lib.rnnlm_forward_score_shortlist(self.handle, _ptr(x), _ptr(cand), C_, T, lnZ, _ptr(score),
                                                   _stream(None)), "rnnlm_forward_score_shortlist")
        return score

    def rnnlm_nce_train_chunk(self, x, y, noise, lnq, lnZ: float, lr: float, J=None, sum_J=None, stream=None):
        _ok(self.lib.rnnlm_nce_train_chunk(self.handle, _ptr(x), _ptr(y), x.shape[0], _ptr(noise), noise.numel(),
                                           _ptr(lnq), lnZ, lr, _ptr(J), _ptr(sum_J), _stream(stream)),
            "rnnlm_nce_train_chunk")

    def rnnlm_nce_grad_chunk(self, x, y, noise, lnq, lnZ: float, want_J=True, stream=None):
        import torch
        if stream is not None:
            return _on("rnnlm_nce_grad_chunk", stream, self.device.index, self.rnnlm_nce_grad_chunk, x, y, noise, lnq, lnZ, want_J)
        z = lambda *s: torch.empty(*s, dtype=torch.float32, device=self.device)
        dE, dU, dWo, db = z(self.V, self.H), z(self.H, self.H), z(self.V, self.H), z(self.V)
        J = z(x.shape[0], self.B) if want_J else None
        _ok(self.lib.rnnlm_nce_grad_chunk(self.handle, _ptr(x), _ptr(y), x.shape[0], _ptr(noise), noise.numel(),
                                          _ptr(lnq), lnZ, _ptr(dE), _ptr(dU), _ptr(dWo), _ptr(db), _ptr(J),
                                          _stream(None)), "rnnlm_nce_grad_chunk")
        return dict(gE=dE, gU=dU, gWo=dWo, gb=db, J=J)

    # -- windows whose logits are the caller's -----------------------------------------------------
    def _logit_rows(self, call, T, logits):
        """A tensor [T][B][V] of the compute type (a new one if None) and the distance of its rows."""
        import torch
        dtype = torch.float32 if self.precision == RNNLM_FP32 else torch.bfloat16
        if logits is None:
            return torch.empty(T, self.B, self.V, dtype=dtype, device=self.device), self.V
        if tuple(logits.shape) != (T, self.B, self.V) or logits.dtype is not dtype or logits.get_device() != self.device.index:
            _refuse(call, f"logits: {dtype} [{T}][{self.B}][{self.V}] on {self.device} is wanted")
        return logits, _rows(call, "logits", logits)[2]

    def _window(self, call, x):
        import torch
        if x.dim() != 2:
            _refuse(call, f"x: [T][{self.B}] is wanted")
        return x.shape[0], _at(call, "x", x, torch.int32, x.shape[0] * self.B, self.device.index, self.B)

    def rnnlm_forward_logits(self, x, logits=None, stream=None):
        call = "rnnlm_forward_logits"
        if stream is not None:
            return _on(call, stream, self.device.index, self.rnnlm_forward_logits, x, logits)
        T, at = self._window(call, x)
        logits, ld = self._logit_rows(call, T, logits)
        _ok(_launch(self.device.index, self.lib.rnnlm_forward_logits, self.handle, at, T, logits.data_ptr(), ld), call)
        return logits

    def _distill(self, call, x, y, ids, vals, lse, weight, tau, alpha, logits, loss, sum_loss):
        import torch
        T, at = self._window(call, x)
        logits, ld = self._logit_rows(call, T, logits)
        n, K, dev, f32, i32 = T * self.B, ids.shape[-1], self.device.index, torch.float32, torch.int32
        d = rnnlm_distill(_at(call, "ids", ids, i32, n * K, dev, K), _at(call, "vals", vals, f32, n * K, dev, K),
                          _at(call, "lse", lse, f32, n, dev), _at(call, "weight", weight, f32, n, dev), K, tau, alpha,
                          logits.data_ptr(), ld)
        return (d, logits, T, at, _at(call, "y", y, i32, n, dev), _at(call, "loss", loss, f32, n, dev),
                _at(call, "sum_loss", sum_loss, torch.float64, 1, dev))

    def rnnlm_distill_train_chunk(self, x, y, ids, vals, lr: float, lse=None, weight=None, tau: float = 1.0, alpha: float = 1.0,
                                  logits=None, loss=None, sum_loss=None, stream=None):
        """ids, vals [T][B][K], lse [T][B] or None: the teacher's (rnnlm_top_logits of its rnnlm_forward_logits at the same tau)."""
        call = "rnnlm_distill_train_chunk"
        if stream is not None:
            return _on(call, stream, self.device.index, self.rnnlm_distill_train_chunk, x, y, ids, vals, lr, lse, weight, tau, alpha,
                       logits, loss, sum_loss)
        d, _keep, T, at, y_at, loss_at, sum_at = self._distill(call, x, y, ids, vals, lse, weight, tau, alpha, logits, loss, sum_loss)
        _ok(_launch(self.device.index, self.lib.rnnlm_distill_train_chunk, self.handle, at, y_at, T, C.byref(d), lr, loss_at, sum_at), call)

    def rnnlm_distill_grad_chunk(self, x, y, ids, vals, lse=None, weight=None, tau: float = 1.0, alpha: float = 1.0, logits=None,
                                 stream=None):
        import torch
        call = "rnnlm_distill_grad_chunk" + ("_compressed" if self.P else "")
        if stream is not None:
            return _on(call, stream, self.device.index, self.rnnlm_distill_grad_chunk, x, y, ids, vals, lse, weight, tau, alpha, logits)
        z = lambda *s: torch.empty(*s, dtype=torch.float32, device=self.device)
        loss = z(x.shape[0], self.B)
        d, _keep, T, at, y_at, loss_at, _ = self._distill(call, x, y, ids, vals, lse, weight, tau, alpha, logits, loss, None)
        if self.P:
            g = dict(gE=z(self.V, self.P), gA=z(self.H, self.P), gU=z(self.H, self.H), gC=z(self.P, self.H), gb=z(self.V))
        else:
            g = dict(gE=z(self.V, self.H), gU=z(self.H, self.H), gWo=z(self.V, self.H), gb=z(self.V))
        _ok(_launch(self.device.index, getattr(self.lib, call), self.handle, at, y_at, T, C.byref(d), *map(_ptr, g.values()), loss_at), call)
        return dict(loss=loss, **g)

    def rnnlm_verify_chunk(self, x, u, draft=None, lengths=None, tau: float = 1.0, tau_draft: float = 1.0, logits=None, accepted=None,
                           tokens=None, workspace=None, stream=None):
        """x int32 [K+1][B]: the word not read yet, then the drafts.  Returns (accepted [B], tokens [K+1][B])."""
        import torch
        call, i32, B, dev = "rnnlm_verify_chunk", torch.int32, self.B, self.device.index
        if stream is not None:
            return _on(call, stream, dev, self.rnnlm_verify_chunk, x, u, draft, lengths, tau, tau_draft, logits, accepted, tokens,
                       workspace)
        T, x_at = self._window(call, x)
        logits, ld = self._logit_rows(call, T, logits)
        ldd = self._logit_rows(call, T - 1, draft)[1] if draft is not None and T > 1 else 0
        accepted = torch.empty(B, dtype=i32, device=self.device) if accepted is None else accepted
        tokens = torch.empty(T, B, dtype=i32, device=self.device) if tokens is None else tokens
        at, nbytes, _keep = _scratch(call, workspace, dev, lambda: rnnlm_verify_workspace_bytes(T - 1, B, self.V))
        v = rnnlm_verify(draft.data_ptr() if ldd else None, ldd, _at(call, "lengths", lengths, i32, B, dev),
                         _at(call, "u", u, torch.float32, T * B, dev, B), tau, tau_draft, logits.data_ptr(), ld, at, nbytes)
        _ok(_launch(dev, self.lib.rnnlm_verify_chunk, self.handle, x_at, T - 1, C.byref(v), _at(call, "accepted", accepted, i32, B, dev),
                    _at(call, "tokens", tokens, i32, T * B, dev, B)), call)
        return accepted, tokens

    def rnnlm_reset_state(self, stream=None):
        _ok(self.lib.rnnlm_reset_state(self.handle, _stream(stream)), "rnnlm_reset_state")

    def rnnlm_sync_compute_copies(self, stream=None):
        _ok(self.lib.rnnlm_sync_compute_copies(self.handle, _stream(stream)), "rnnlm_sync_compute_copies")

    def rnnlm_check(self, stream=None):
        _ok(self.lib.rnnlm_check(self.handle, _stream(stream)), "rnnlm_check")

    def rnnlm_set_barrier_spin_limit(self, polls: int):
        _ok(self.lib.rnnlm_set_barrier_spin_limit(self.handle, polls), "rnnlm_set_barrier_spin_limit")

    def rnnlm_set_recurrent_exchange(self, mode: int):
        _ok(self.lib.rnnlm_set_recurrent_exchange(self.handle, mode), "rnnlm_set_recurrent_exchange")

    def rnnlm_measure_peaks(self, stream=None):
        r, c, g = C.c_double(0), C.c_double(0), C.c_double(0)
        _ok(self.lib.rnnlm_measure_peaks(self.handle, C.byref(r), C.byref(c), C.byref(g), _stream(stream)),
            "rnnlm_measure_peaks")
        return dict(mfma_bf16_random_tflops=r.value, mfma_bf16_constant_tflops=c.value, copy_gbs=g.value)

    def rnnlm_profile_enable(self, stage_mask: int):
        _ok(self.lib.rnnlm_profile_enable(self.handle, stage_mask), "rnnlm_profile_enable")

    def rnnlm_profile_read(self, stage: int):
        ms = C.c_double(0.0)
        n = C.c_int64(0)
        _ok(self.lib.rnnlm_profile_read(self.handle, stage, C.byref(ms), C.byref(n)), "rnnlm_profile_read")
        return ms.value, n.value

    def rnnlm_sort_segments(self, x, stream=None):
        import torch
        if stream is not None:
            return _on("rnnlm_sort_segments", stream, self.device.index, self.rnnlm_sort_segments, x)
        M = x.numel()
        perm = torch.empty(M, dtype=torch.int32, device=self.device)
        seg = torch.empty(M + 1, dtype=torch.int32, device=self.device)
        nseg = torch.zeros(1, dtype=torch.int32, device=self.device)
        _ok(self.lib.rnnlm_sort_segments(self.handle, _ptr(x), x.shape[0], _ptr(perm), _ptr(seg), _ptr(nseg),
                                         _stream(None)), "rnnlm_sort_segments")
        n = int(nseg.item())
        return perm, seg[:n + 1]
