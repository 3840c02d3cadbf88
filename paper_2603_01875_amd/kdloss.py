"""ctypes binding of libkdloss (see include/kdloss.h for the contract).

Argument marshalling only: every step of the computation runs in the HIP
kernels of the shared library.  torch is used to own device memory and to name
the stream.  There is no fallback: if the library has not been built, loading
fails with an error that says how to build it.
"""
from __future__ import annotations

import ctypes
import os

FKL, RKL, JSD, TVD, SKEW_FKL, SKEW_RKL, AKL = 0, 1, 2, 3, 4, 5, 6
BF16, F32 = 0, 1
W_HV, W_VH = 0, 1
I32, I64 = 0, 1
TAIL_RENORM, TAIL_REST, TAIL_DROP = 0, 1, 2
TOPK_MAX = 1024

KD_OK = 0
STATUS_NAMES = {0: "KD_OK", 1: "KD_ERR_NULL", 2: "KD_ERR_SHAPE", 3: "KD_ERR_ALIGN", 4: "KD_ERR_PARAM",
                5: "KD_ERR_WORKSPACE", 6: "KD_ERR_UNSUPPORTED", 7: "KD_ERR_LAUNCH", 8: "KD_ERR_TOO_LARGE"}
STATIC_SCRATCH_BYTES = 128 << 20

# KDLOSS_LIBRARY names another build of the library (measurement builds for the profiles); default: the
# product build next to the sources
_LIB_PATH = os.environ.get("KDLOSS_LIBRARY") or os.path.join(os.path.dirname(os.path.abspath(__file__)), "csrc",
                                                             "libkdloss.so")
_lib = None


class KdLossParams(ctypes.Structure):
    _fields_ = [("T", ctypes.c_int64), ("H_t", ctypes.c_int64), ("H_s", ctypes.c_int64), ("V", ctypes.c_int64),
                ("in_dtype", ctypes.c_int32), ("grad_dtype", ctypes.c_int32), ("w_layout", ctypes.c_int32),
                ("kind", ctypes.c_int32), ("tau", ctypes.c_float), ("beta", ctypes.c_float),
                ("accumulate_grad_W", ctypes.c_int32), ("flags", ctypes.c_int32),
                ("teacher_scale", ctypes.c_float), ("vocab_chunk", ctypes.c_int32),
                ("loss_scale", ctypes.c_float), ("reserved", ctypes.c_int32)]


class KdCeParams(ctypes.Structure):
    """kd_ce_params of the C header."""
    _fields_ = [("T", ctypes.c_int64), ("H", ctypes.c_int64), ("V", ctypes.c_int64),
                ("in_dtype", ctypes.c_int32), ("grad_dtype", ctypes.c_int32), ("w_layout", ctypes.c_int32),
                ("index_dtype", ctypes.c_int32), ("label_smoothing", ctypes.c_float), ("z_loss", ctypes.c_float),
                ("loss_scale", ctypes.c_float), ("accumulate_grad_W", ctypes.c_int32), ("vocab_chunk", ctypes.c_int32),
                ("reserved", ctypes.c_int32)]


class KdTopkParams(ctypes.Structure):
    """kd_topk_params of the C header."""
    _fields_ = [("T", ctypes.c_int64), ("H", ctypes.c_int64), ("V", ctypes.c_int64), ("K", ctypes.c_int32),
                ("in_dtype", ctypes.c_int32), ("grad_dtype", ctypes.c_int32), ("w_layout", ctypes.c_int32),
                ("index_dtype", ctypes.c_int32), ("top_dtype", ctypes.c_int32), ("tail", ctypes.c_int32),
                ("tau", ctypes.c_float), ("loss_scale", ctypes.c_float), ("accumulate_grad_W", ctypes.c_int32),
                ("flags", ctypes.c_int32), ("vocab_chunk", ctypes.c_int32), ("reserved", ctypes.c_int32 * 2)]


class KdLossError(RuntimeError):
    def __init__(self, status):
        self.status = int(status)
        msg = lib().kd_status_string(self.status).decode()
        super().__init__(f"{STATUS_NAMES.get(self.status, self.status)}: {msg}")


def lib():
    """The loaded shared library (loads on first use; never falls back to anything else)."""
    global _lib
    if _lib is None:
        if not os.path.exists(_LIB_PATH):
            raise RuntimeError(f"{_LIB_PATH} is missing: build it with "
                               "`python -c 'import __graft_entry__ as g; g.build()'` "
                               "or paper_2603_01875_amd/csrc/build.sh")
        # The tensors handed to the library and the streams it launches on belong to torch's HIP runtime
        # (the wheel carries its own copy).  Import torch first, so that this library's HIP calls bind to
        # that same runtime; loaded before torch it would bring up a second one, which knows neither the
        # streams nor, on a box that admits one runtime per process, the device.
        import torch  # noqa: F401
        L = ctypes.CDLL(_LIB_PATH)
        P = ctypes.POINTER(KdLossParams)
        vp = ctypes.c_void_p
        L.kd_loss_workspace_size.argtypes = [P, ctypes.POINTER(ctypes.c_size_t)]
        L.kd_loss_workspace_size.restype = ctypes.c_int
        L.kd_loss_plan_info.argtypes = [P, ctypes.POINTER(ctypes.c_int64), ctypes.POINTER(ctypes.c_int64)]
        L.kd_loss_plan_info.restype = ctypes.c_int
        L.kd_loss_plan_loop.argtypes = [P, ctypes.POINTER(ctypes.c_int32)]
        L.kd_loss_plan_loop.restype = ctypes.c_int
        L.kd_loss_plan_grad_h.argtypes = [P, ctypes.POINTER(ctypes.c_int32), ctypes.POINTER(ctypes.c_int32)]
        L.kd_loss_plan_grad_h.restype = ctypes.c_int
        L.kd_loss_fwd_bwd.argtypes = [P, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, ctypes.c_size_t, vp]
        L.kd_loss_fwd_bwd.restype = ctypes.c_int
        L.kd_loss_fwd_bwd_static.argtypes = [P, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp]
        L.kd_loss_fwd_bwd_static.restype = ctypes.c_int
        L.kd_loss_fwd.argtypes = [P, vp, vp, vp, vp, vp, vp, vp, vp, ctypes.c_size_t, vp]
        L.kd_loss_fwd.restype = ctypes.c_int
        L.kd_loss_workspace_size_multi.argtypes = [P, ctypes.c_int, ctypes.POINTER(ctypes.c_int64),
                                                   ctypes.POINTER(ctypes.c_size_t)]
        L.kd_loss_workspace_size_multi.restype = ctypes.c_int
        L.kd_loss_fwd_bwd_multi.argtypes = [P, ctypes.c_int, ctypes.POINTER(vp), ctypes.POINTER(vp),
                                            ctypes.POINTER(ctypes.c_int64), ctypes.POINTER(ctypes.c_float),
                                            ctypes.POINTER(ctypes.c_float),
                                            vp, vp, vp, vp, vp, vp, vp, vp, ctypes.c_size_t, vp]
        L.kd_loss_fwd_bwd_multi.restype = ctypes.c_int
        C, Q = ctypes.POINTER(KdCeParams), ctypes.POINTER(KdTopkParams)
        for size, params in ((L.kd_ce_workspace_size, C), (L.kd_topk_workspace_size, Q)):
            size.argtypes = [params, ctypes.POINTER(ctypes.c_size_t)]
            size.restype = ctypes.c_int
        L.kd_ce_fwd.argtypes = [C] + [vp] * 7 + [ctypes.c_size_t, vp]
        L.kd_ce_fwd_bwd.argtypes = [C] + [vp] * 9 + [ctypes.c_size_t, vp]
        L.kd_topk_fwd.argtypes = [Q] + [vp] * 9 + [ctypes.c_size_t, vp]
        L.kd_topk_fwd_bwd.argtypes = [Q] + [vp] * 11 + [ctypes.c_size_t, vp]
        for call in (L.kd_ce_fwd, L.kd_ce_fwd_bwd, L.kd_topk_fwd, L.kd_topk_fwd_bwd):
            call.restype = ctypes.c_int
        L.kd_quantize_e4m3.argtypes = [vp, ctypes.c_int32, ctypes.c_int64, ctypes.c_float, vp, vp]
        L.kd_quantize_e4m3.restype = ctypes.c_int
        L.kd_loss_profile_clock.argtypes = [vp]
        L.kd_loss_profile_clock.restype = ctypes.c_int
        L.kd_probe_mfma_rate.argtypes = [vp, ctypes.c_int, vp, vp]
        L.kd_probe_mfma_rate.restype = ctypes.c_int
        L.kd_loss_profile_hook.argtypes = [ctypes.c_int, ctypes.POINTER(ctypes.c_void_p), ctypes.c_int]
        L.kd_loss_profile_hook.restype = ctypes.c_int
        L.kd_loss_profile_count.argtypes = []
        L.kd_loss_profile_count.restype = ctypes.c_int
        L.kd_build_info.argtypes = []
        L.kd_build_info.restype = ctypes.c_char_p
        L.kd_build_ablation.argtypes = []
        L.kd_build_ablation.restype = ctypes.c_int
        L.kd_status_string.argtypes = [ctypes.c_int]
        L.kd_status_string.restype = ctypes.c_char_p
        _lib = L
    return _lib


FLAG_TAU2 = 1
FLAG_TEACHER_FP8 = 2

def make_params(T, H_t, H_s, V, kind=FKL, tau=1.0, beta=0.5, in_dtype=BF16, grad_dtype=None,
                w_layout=W_VH, accumulate_grad_W=False, flags=0, teacher_scale=0.0, vocab_chunk=0,
                loss_scale=1.0):
    if grad_dtype is None:
        grad_dtype = in_dtype
    return KdLossParams(int(T), int(H_t), int(H_s), int(V), int(in_dtype), int(grad_dtype), int(w_layout),
                        int(kind), float(tau), float(beta), int(bool(accumulate_grad_W)), int(flags),
                        float(teacher_scale), int(vocab_chunk), float(loss_scale), 0)


def quantize_e4m3(x, scale, out=None):
    """e4m3 codes (uint8 tensor of x's shape) of x / scale; x is a contiguous bf16 or fp32 CUDA tensor."""
    import torch
    if not (isinstance(x, torch.Tensor) and x.is_cuda and x.is_contiguous()
            and x.dtype in (torch.bfloat16, torch.float32)):
        raise ValueError("x must be a contiguous bfloat16 or float32 CUDA (HIP) tensor")
    if out is None:
        out = torch.empty(x.shape, dtype=torch.uint8, device=x.device)
    elif not (out.is_cuda and out.device == x.device and out.is_contiguous() and out.dtype == torch.uint8
              and out.numel() == x.numel()):
        raise ValueError("out must be a contiguous uint8 tensor of x's size on x's device")
    st = lib().kd_quantize_e4m3(_ptr(x), BF16 if x.dtype == torch.bfloat16 else F32, x.numel(), float(scale),
                                _ptr(out), ctypes.c_void_p(torch.cuda.current_stream().cuda_stream))
    if st != KD_OK:
        raise KdLossError(st)
    return out


def kd_loss_workspace_size(params) -> int:
    """Workspace bytes of a call with this parameter block (KdLossParams, KdCeParams or KdTopkParams)."""
    n = ctypes.c_size_t(0)
    for block, query in ((KdLossParams, lib().kd_loss_workspace_size), (KdCeParams, lib().kd_ce_workspace_size),
                         (KdTopkParams, lib().kd_topk_workspace_size)):
        if isinstance(params, block):
            break
    else:
        raise TypeError(f"params must be a KdLossParams, KdCeParams or KdTopkParams, got {type(params).__name__}")
    st = query(ctypes.byref(params), ctypes.byref(n))
    if st != KD_OK:
        raise KdLossError(st)
    return int(n.value)


def kd_loss_plan_info(params: KdLossParams):
    vc, nl = ctypes.c_int64(0), ctypes.c_int64(0)
    st = lib().kd_loss_plan_info(ctypes.byref(params), ctypes.byref(vc), ctypes.byref(nl))
    if st != KD_OK:
        raise KdLossError(st)
    return int(vc.value), int(nl.value)


def kd_loss_plan_loop(params: KdLossParams):
    """0: the eight-wave loop makes the logit tiles of such a call; 1: the strip loop."""
    loop = ctypes.c_int32(0)
    st = lib().kd_loss_plan_loop(ctypes.byref(params), ctypes.byref(loop))
    if st != KD_OK:
        raise KdLossError(st)
    return int(loop.value)


def kd_loss_plan_grad_h(params: KdLossParams):
    """(hidden rows of a tile of the grad_h_s product, parts that it splits the vocabulary into) for such a call."""
    rows, parts = ctypes.c_int32(0), ctypes.c_int32(0)
    st = lib().kd_loss_plan_grad_h(ctypes.byref(params), ctypes.byref(rows), ctypes.byref(parts))
    if st != KD_OK:
        raise KdLossError(st)
    return int(rows.value), int(parts.value)


PROF_STATS, PROF_ROWS, PROF_GRAD, PROF_GEMM_GRAD_W, PROF_GEMM_GRAD_H = range(5)


class KernelTimer:
    """Brackets every launch of one kernel family with HIP events (kd_loss_profile_hook).

    with KernelTimer(PROF_STATS, max_launches) as kt: ...calls...; then kt.durations_ms()
    after a device synchronisation.
    """

    def __init__(self, which, max_launches):
        import torch
        self.which = which
        self.events = [torch.cuda.Event(enable_timing=True) for _ in range(2 * max_launches)]
        for e in self.events:
            e.record()                      # materialise the underlying hipEvent_t
        self.arr = (ctypes.c_void_p * len(self.events))(*[e.cuda_event for e in self.events])
        self.count = 0

    def __enter__(self):
        st = lib().kd_loss_profile_hook(self.which, self.arr, len(self.events))
        if st != KD_OK:
            raise KdLossError(st)
        return self

    def __exit__(self, *exc):
        self.count = lib().kd_loss_profile_count()
        lib().kd_loss_profile_hook(-1, None, 0)

    def durations_ms(self):
        return [self.events[2 * i].elapsed_time(self.events[2 * i + 1]) for i in range(self.count)]


PROBE_FLOP_PER_ITER = 256.0 * 8 * 8 * 2 * 32 * 32 * 16


class ShaderClock:
    """with ShaderClock() as sc: <library calls>; sc.ghz() is the shader clock that workgroup 0 of the last
    statistics kernel (or MFMA probe) saw: cycles of its main loop over 100 MHz reference ticks."""

    def __enter__(self):
        import torch
        self.buf = torch.zeros(2, dtype=torch.int64, device="cuda")
        st = lib().kd_loss_profile_clock(_ptr(self.buf))
        if st != KD_OK:
            raise KdLossError(st)
        return self

    def __exit__(self, *exc):
        lib().kd_loss_profile_clock(None)

    def ghz(self):
        c, r = [int(x) for x in self.buf.cpu()]
        return c / r * 0.1 if r > 0 else float("nan")


def probe_mfma_rate(iters=20000, repeats=3):
    """TFLOP/s of an MFMA-only loop on random bf16 operands (best of `repeats`): the matrix-pipe
    ceiling of this GPU at the clock it holds under that load."""
    import torch
    ops = torch.randn(64 * 1024, device="cuda", dtype=torch.float32).to(torch.bfloat16)
    sink = torch.empty(256 * 512, device="cuda", dtype=torch.float32)
    s = torch.cuda.current_stream().cuda_stream
    best = 0.0
    for _ in range(repeats + 1):                 # first launch warms up
        e0, e1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        e0.record()
        st = lib().kd_probe_mfma_rate(_ptr(ops), int(iters), _ptr(sink), ctypes.c_void_p(s))
        if st != KD_OK:
            raise KdLossError(st)
        e1.record()
        torch.cuda.synchronize()
        best = max(best, PROBE_FLOP_PER_ITER * iters / (e0.elapsed_time(e1) * 1e-3) / 1e12)
    return best


def _ptr(t):
    return ctypes.c_void_p(0 if t is None else t.data_ptr())


def _nbytes(t):
    return t.numel() * t.element_size()


def check_operands(h_t, W_t, h_s, W_s, mask=None, w_layout=W_VH, flags=0, grad_dtype=None, grad_W_s=None,
                   workspace=None, require_cuda=True):
    """Host-side checks of the tensors handed to the convenience wrappers.  The C ABI sees only addresses, so
    a wrong dtype, shape, device or a non-contiguous tensor would become an out-of-bounds device access:
    everything the library cannot see is checked here, and a ValueError is raised before any call.
    Returns (T, H_t, H_s, V, in_dtype, grad_dtype)."""
    import torch
    names = ("h_t", "W_t", "h_s", "W_s")
    ts = (h_t, W_t, h_s, W_s)
    for n, t in zip(names, ts):
        if not isinstance(t, torch.Tensor):
            raise ValueError(f"{n} must be a torch tensor")
        if t.dim() != 2:
            raise ValueError(f"{n} must be 2-dimensional, got shape {tuple(t.shape)}")
        if not t.is_contiguous():
            raise ValueError(f"{n} must be contiguous")
        if require_cuda and not t.is_cuda:
            raise ValueError(f"{n} must be a CUDA (HIP) tensor")
        if t.device != h_s.device:
            raise ValueError(f"{n} is on {t.device}, h_s on {h_s.device}")
    if w_layout not in (W_HV, W_VH):
        raise ValueError("unknown w_layout")
    if h_s.dtype not in (torch.bfloat16, torch.float32):
        raise ValueError(f"h_s must be bfloat16 or float32, got {h_s.dtype}")
    if W_s.dtype != h_s.dtype:
        raise ValueError(f"W_s is {W_s.dtype}, h_s is {h_s.dtype}")
    want_t = torch.uint8 if (flags & FLAG_TEACHER_FP8) else h_s.dtype
    for n, t in (("h_t", h_t), ("W_t", W_t)):
        if t.dtype != want_t:
            raise ValueError(f"{n} must be {want_t} here, got {t.dtype}")
    in_dtype = BF16 if h_s.dtype == torch.bfloat16 else F32
    T, H_t = h_t.shape
    if h_s.shape[0] != T:
        raise ValueError(f"h_s has {h_s.shape[0]} rows, h_t has {T}")
    H_s = h_s.shape[1]
    V = W_t.shape[0] if w_layout == W_VH else W_t.shape[1]
    want_Wt = (V, H_t) if w_layout == W_VH else (H_t, V)
    want_Ws = (V, H_s) if w_layout == W_VH else (H_s, V)
    if tuple(W_t.shape) != want_Wt:
        raise ValueError(f"W_t has shape {tuple(W_t.shape)}, expected {want_Wt} for this layout")
    if tuple(W_s.shape) != want_Ws:
        raise ValueError(f"W_s has shape {tuple(W_s.shape)}, expected {want_Ws} for this layout")
    if mask is not None:
        if not isinstance(mask, torch.Tensor) or mask.numel() != T or mask.element_size() != 1:
            raise ValueError("mask must be a tensor of T one-byte elements (uint8 or bool)")
        if not mask.is_contiguous() or mask.device != h_s.device:
            raise ValueError("mask must be contiguous and on the operands' device")
    if grad_dtype is None:
        grad_dtype = in_dtype
    if grad_dtype not in (BF16, F32):
        raise ValueError("unknown grad_dtype")
    if grad_W_s is not None:
        tdt = torch.bfloat16 if grad_dtype == BF16 else torch.float32
        if (not isinstance(grad_W_s, torch.Tensor) or tuple(grad_W_s.shape) != want_Ws or grad_W_s.dtype != tdt
                or not grad_W_s.is_contiguous() or grad_W_s.device != h_s.device):
            raise ValueError(f"grad_W_s must be a contiguous {tdt} tensor of shape {want_Ws} on the operands' device")
    if workspace is not None:
        if not isinstance(workspace, torch.Tensor) or not workspace.is_contiguous() or workspace.device != h_s.device:
            raise ValueError("workspace must be a contiguous tensor on the operands' device")
    return int(T), int(H_t), int(H_s), int(V), in_dtype, grad_dtype


def _check_raw(params, h_t, W_t, h_s, W_s, mask, loss, per_token_loss, grad_h_s, grad_W_s, workspace):
    """The thin calls take a prepared parameter block: check that every tensor holds what that block says
    the library will read or write (byte counts, contiguity, one device)."""
    es_in = 2 if params.in_dtype == BF16 else 4
    es_t = 1 if (params.flags & FLAG_TEACHER_FP8) else es_in
    es_g = 2 if params.grad_dtype == BF16 else 4
    T, H_t, H_s, V = params.T, params.H_t, params.H_s, params.V
    need = [("h_t", h_t, T * H_t * es_t), ("W_t", W_t, V * H_t * es_t), ("h_s", h_s, T * H_s * es_in),
            ("W_s", W_s, V * H_s * es_in), ("loss", loss, 4)]
    if mask is not None:
        need.append(("mask", mask, T))
    if per_token_loss is not None:
        need.append(("per_token_loss", per_token_loss, 4 * T))
    if grad_h_s is not None:
        need.append(("grad_h_s", grad_h_s, T * H_s * es_g))
    if grad_W_s is not None:
        need.append(("grad_W_s", grad_W_s, V * H_s * es_g))
    dev = h_s.device
    for n, t, nb in need:
        if not t.is_cuda or t.device != dev:
            raise ValueError(f"{n} must be a CUDA (HIP) tensor on {dev}")
        if not t.is_contiguous():
            raise ValueError(f"{n} must be contiguous")
        if _nbytes(t) != nb:
            raise ValueError(f"{n} holds {_nbytes(t)} bytes, the parameter block implies {nb}")
    if mask is not None and mask.element_size() != 1:
        raise ValueError("mask must have one-byte elements")
    if workspace is not None and (not workspace.is_cuda or workspace.device != dev or not workspace.is_contiguous()):
        raise ValueError("workspace must be a contiguous CUDA (HIP) tensor on the operands' device")


def kd_loss_fwd_bwd_raw(params, h_t, W_t, h_s, W_s, mask, loss, per_token_loss, grad_h_s, grad_W_s,
                        workspace, stream=None):
    """Thin call: all tensors are caller-allocated torch CUDA tensors (or None where allowed)."""
    import torch
    _check_raw(params, h_t, W_t, h_s, W_s, mask, loss, per_token_loss, grad_h_s, grad_W_s, workspace)
    s = torch.cuda.current_stream().cuda_stream if stream is None else stream
    st = lib().kd_loss_fwd_bwd(ctypes.byref(params), _ptr(h_t), _ptr(W_t), _ptr(h_s), _ptr(W_s), _ptr(mask),
                               _ptr(loss), _ptr(per_token_loss), _ptr(grad_h_s), _ptr(grad_W_s),
                               _ptr(workspace), ctypes.c_size_t(_nbytes(workspace)), ctypes.c_void_p(s))
    if st != KD_OK:
        raise KdLossError(st)


def kd_loss_fwd_bwd_static_raw(params, h_t, W_t, h_s, W_s, mask, loss, per_token_loss, grad_h_s, grad_W_s,
                               stream=None):
    """Thin call of the entry point that needs no workspace (the library's static scratch array)."""
    import torch
    _check_raw(params, h_t, W_t, h_s, W_s, mask, loss, per_token_loss, grad_h_s, grad_W_s, None)
    s = torch.cuda.current_stream().cuda_stream if stream is None else stream
    st = lib().kd_loss_fwd_bwd_static(ctypes.byref(params), _ptr(h_t), _ptr(W_t), _ptr(h_s), _ptr(W_s), _ptr(mask),
                                      _ptr(loss), _ptr(per_token_loss), _ptr(grad_h_s), _ptr(grad_W_s),
                                      ctypes.c_void_p(s))
    if st != KD_OK:
        raise KdLossError(st)


def kd_loss_fwd_raw(params, h_t, W_t, h_s, W_s, mask, loss, per_token_loss, workspace, stream=None):
    import torch
    _check_raw(params, h_t, W_t, h_s, W_s, mask, loss, per_token_loss, None, None, workspace)
    s = torch.cuda.current_stream().cuda_stream if stream is None else stream
    st = lib().kd_loss_fwd(ctypes.byref(params), _ptr(h_t), _ptr(W_t), _ptr(h_s), _ptr(W_s), _ptr(mask),
                           _ptr(loss), _ptr(per_token_loss), _ptr(workspace),
                           ctypes.c_size_t(_nbytes(workspace)), ctypes.c_void_p(s))
    if st != KD_OK:
        raise KdLossError(st)


def alloc_workspace(params, device="cuda"):
    import torch
    n = kd_loss_workspace_size(params)
    return torch.empty((n + 255) // 256 * 256, dtype=torch.uint8, device=device)


def kd_loss_fwd_bwd(h_t, W_t, h_s, W_s, mask=None, tau=1.0, kind=FKL, beta=0.5, w_layout=W_VH,
                    grad_dtype=None, workspace=None, grad_W_s=None, accumulate_grad_W=False,
                    want_per_token=True, flags=0, teacher_scale=0.0, vocab_chunk=0, loss_scale=1.0):
    """Convenience wrapper: allocates outputs (and the workspace unless given) and calls the library.

    h_t [T,H_t], h_s [T,H_s]; W_t, W_s in `w_layout` ([V,H] for W_VH).  Returns a dict of CUDA tensors.
    With FLAG_TEACHER_FP8, h_t and W_t are uint8 tensors of e4m3 codes and teacher_scale their joint scale.
    """
    import torch
    T, H_t, H_s, V, in_dtype, grad_dtype = check_operands(h_t, W_t, h_s, W_s, mask, w_layout, flags, grad_dtype,
                                                          grad_W_s, workspace)
    p = make_params(T, H_t, H_s, V, kind, tau, beta, in_dtype, grad_dtype, w_layout, accumulate_grad_W, flags,
                    teacher_scale, vocab_chunk, loss_scale)
    tdt = torch.bfloat16 if grad_dtype == BF16 else torch.float32
    dev = h_t.device
    if workspace is None:
        workspace = alloc_workspace(p, dev)
    loss = torch.empty(1, dtype=torch.float32, device=dev)
    ptl = torch.empty(T, dtype=torch.float32, device=dev) if want_per_token else None
    grad_h = torch.empty((T, H_s), dtype=tdt, device=dev)
    if grad_W_s is None:
        grad_W_s = torch.empty_like(W_s, dtype=tdt)
    kd_loss_fwd_bwd_raw(p, h_t, W_t, h_s, W_s, mask, loss, ptl, grad_h, grad_W_s, workspace)
    return dict(loss=loss, per_token_loss=ptl, grad_h_s=grad_h, grad_W_s=grad_W_s, workspace=workspace)


def kd_loss_fwd_bwd_multi(h_ts, W_ts, weights, h_s, W_s, mask=None, tau=1.0, kind=FKL, beta=0.5, flags=0,
                          grad_dtype=None, teacher_scales=None, w_layout=W_VH, vocab_chunk=0, loss_scale=1.0):
    """Multi-teacher call: lists of teacher hidden states / heads (in `w_layout`) and weights; with
    FLAG_TEACHER_FP8 the teacher tensors are e4m3 codes and teacher_scales their joint scales."""
    import torch
    n = len(h_ts)
    if n < 1 or len(W_ts) != n or len(weights) != n or (teacher_scales is not None and len(teacher_scales) != n):
        raise ValueError("h_ts, W_ts, weights (and teacher_scales) must have one entry per teacher")
    if (flags & FLAG_TEACHER_FP8) and teacher_scales is None:
        raise ValueError("FLAG_TEACHER_FP8 needs teacher_scales")
    for h_t, W_t in zip(h_ts, W_ts):
        T, _, H_s, V, in_dtype, grad_dtype = check_operands(h_t, W_t, h_s, W_s, mask, w_layout, flags, grad_dtype)
    p = make_params(T, h_ts[0].shape[1], H_s, V, kind, tau, beta, in_dtype, grad_dtype, w_layout, False, flags,
                    0.0, vocab_chunk, loss_scale)
    H_t = (ctypes.c_int64 * n)(*[int(h.shape[1]) for h in h_ts])
    nbytes = ctypes.c_size_t(0)
    st = lib().kd_loss_workspace_size_multi(ctypes.byref(p), n, H_t, ctypes.byref(nbytes))
    if st != KD_OK:
        raise KdLossError(st)
    dev = h_s.device
    ws = torch.empty((nbytes.value + 255) // 256 * 256, dtype=torch.uint8, device=dev)
    tdt = torch.bfloat16 if grad_dtype == BF16 else torch.float32
    loss = torch.empty(1, dtype=torch.float32, device=dev)
    ptl = torch.empty(T, dtype=torch.float32, device=dev)
    grad_h = torch.empty((T, H_s), dtype=tdt, device=dev)
    grad_W = torch.empty_like(W_s, dtype=tdt)
    hp = (ctypes.c_void_p * n)(*[h.data_ptr() for h in h_ts])
    wp = (ctypes.c_void_p * n)(*[w.data_ptr() for w in W_ts])
    wt = (ctypes.c_float * n)(*[float(w) for w in weights])
    sc = None if teacher_scales is None else (ctypes.c_float * n)(*[float(x) for x in teacher_scales])
    st = lib().kd_loss_fwd_bwd_multi(ctypes.byref(p), n, hp, wp, H_t, wt, sc, _ptr(h_s), _ptr(W_s), _ptr(mask),
                                     _ptr(loss), _ptr(ptl), _ptr(grad_h), _ptr(grad_W), _ptr(ws),
                                     ctypes.c_size_t(ws.numel()),
                                     ctypes.c_void_p(torch.cuda.current_stream().cuda_stream))
    if st != KD_OK:
        raise KdLossError(st)
    return dict(loss=loss, per_token_loss=ptl, grad_h_s=grad_h, grad_W_s=grad_W)


def kd_loss_fwd(h_t, W_t, h_s, W_s, mask=None, tau=1.0, kind=FKL, beta=0.5, w_layout=W_VH, workspace=None,
                flags=0, teacher_scale=0.0, loss_scale=1.0):
    import torch
    T, H_t, H_s, V, in_dtype, _ = check_operands(h_t, W_t, h_s, W_s, mask, w_layout, flags, None, None, workspace)
    p = make_params(T, H_t, H_s, V, kind, tau, beta, in_dtype, in_dtype, w_layout, False, flags, teacher_scale,
                    0, loss_scale)
    dev = h_t.device
    if workspace is None:
        workspace = alloc_workspace(p, dev)
    loss = torch.empty(1, dtype=torch.float32, device=dev)
    ptl = torch.empty(T, dtype=torch.float32, device=dev)
    kd_loss_fwd_raw(p, h_t, W_t, h_s, W_s, mask, loss, ptl, workspace)
    return dict(loss=loss, per_token_loss=ptl)


# ------------------------------------------------------------------------------------------------
# losses over one output head
# ------------------------------------------------------------------------------------------------
def make_ce_params(T, H, V, label_smoothing=0.0, z_loss=0.0, in_dtype=BF16, grad_dtype=None, w_layout=W_VH,
                   index_dtype=I64, accumulate_grad_W=False, vocab_chunk=0, loss_scale=1.0):
    return KdCeParams(int(T), int(H), int(V), int(in_dtype), int(in_dtype if grad_dtype is None else grad_dtype),
                      int(w_layout), int(index_dtype), float(label_smoothing), float(z_loss), float(loss_scale),
                      int(bool(accumulate_grad_W)), int(vocab_chunk), 0)


def make_topk_params(T, H, V, K, tau=1.0, tail=TAIL_RENORM, in_dtype=BF16, grad_dtype=None, w_layout=W_VH,
                     index_dtype=I64, top_dtype=F32, accumulate_grad_W=False, flags=0, vocab_chunk=0, loss_scale=1.0):
    return KdTopkParams(int(T), int(H), int(V), int(K), int(in_dtype),
                        int(in_dtype if grad_dtype is None else grad_dtype), int(w_layout), int(index_dtype),
                        int(top_dtype), int(tail), float(tau), float(loss_scale), int(bool(accumulate_grad_W)),
                        int(flags), int(vocab_chunk))


def _float_dtype(t, name):
    import torch
    if t.dtype not in (torch.bfloat16, torch.float32):
        raise ValueError(f"{name} must be bfloat16 or float32, got {t.dtype}")
    return BF16 if t.dtype == torch.bfloat16 else F32


def _index_dtype(t, name):
    import torch
    if t.dtype not in (torch.int32, torch.int64):
        raise ValueError(f"{name} must be int32 or int64, got {t.dtype}")
    return I32 if t.dtype == torch.int32 else I64


def _check_head(h, W, w_layout):
    """Hidden states and head of the one-head losses: (T, H, V, in_dtype)."""
    import torch
    for n, t in (("h", h), ("W", W)):
        if not isinstance(t, torch.Tensor) or t.dim() != 2:
            raise ValueError(f"{n} must be a 2-dimensional torch tensor")
    if w_layout not in (W_HV, W_VH):
        raise ValueError("unknown w_layout")
    in_dtype = _float_dtype(h, "h")
    if W.dtype != h.dtype:
        raise ValueError(f"W is {W.dtype}, h is {h.dtype}")
    T, H = h.shape
    V, H_w = W.shape if w_layout == W_VH else (W.shape[1], W.shape[0])
    if H_w != H:
        raise ValueError(f"W has shape {tuple(W.shape)}, expected {'[V, H]' if w_layout == W_VH else '[H, V]'} with H = {H}")
    return int(T), int(H), int(V), in_dtype


def _check_tensors(need, dev):
    """need: (name, tensor or None, dtypes, elements, may be None)."""
    for n, t, dtypes, count, optional in need:
        if t is None:
            if optional:
                continue
            raise ValueError(f"{n} is needed")
        if t.device != dev or not t.is_cuda:
            raise ValueError(f"{n} must be a CUDA (HIP) tensor on {dev}, got {t.device}")
        if not t.is_contiguous():
            raise ValueError(f"{n} must be contiguous")
        if t.dtype not in dtypes:
            raise ValueError(f"{n} must be {' or '.join(map(str, dtypes))} here, got {t.dtype}")
        if t.numel() != count:
            raise ValueError(f"{n} has {t.numel()} elements, expected {count}")


def _head_call(name, p, inputs, h, W, mask, loss, per_token_loss, grads, workspace, stream):
    """Checks what a call of the one-head losses is given against its parameter block and makes it.
    inputs: (name, tensor, dtypes, elements, optional) in front of h / behind W, with their place; grads: None or a pair."""
    import torch
    before, behind = inputs
    fdt = (torch.bfloat16 if p.in_dtype == BF16 else torch.float32,)
    gdt = (torch.bfloat16 if p.grad_dtype == BF16 else torch.float32,)
    T, H, V = p.T, p.H, p.V
    need = before + [("h", h, fdt, T * H, False), ("W", W, fdt, V * H, False)] + behind
    need += [("mask", mask, (torch.uint8, torch.bool), T, True), ("loss", loss, (torch.float32,), 1, False),
             ("per_token_loss", per_token_loss, (torch.float32,), T, True)]
    if grads is not None:
        need += [("grad_h", grads[0], gdt, T * H, True), ("grad_W", grads[1], gdt, V * H, True)]
    dev = h.device
    _check_tensors(need, dev)
    if workspace is None or not workspace.is_cuda or workspace.device != dev or not workspace.is_contiguous():
        raise ValueError("workspace must be a contiguous CUDA (HIP) tensor on the operands' device")
    args = [_ptr(t) for _, t, *_ in before] + [_ptr(h), _ptr(W)] + [_ptr(t) for _, t, *_ in behind]
    args += [_ptr(mask), _ptr(loss), _ptr(per_token_loss)] + ([] if grads is None else [_ptr(g) for g in grads])
    with torch.cuda.device(dev):                   # the launches go to the operands' device, whatever the current one is
        s = torch.cuda.current_stream().cuda_stream if stream is None else stream
        st = getattr(lib(), name)(ctypes.byref(p), *args, _ptr(workspace), ctypes.c_size_t(_nbytes(workspace)),
                                  ctypes.c_void_p(s))
    if st != KD_OK:
        raise KdLossError(st)


def _label_inputs(p, labels):
    import torch
    return [], [("labels", labels, (torch.int32 if p.index_dtype == I32 else torch.int64,), p.T, False)]


def _top_inputs(p, top_logits, top_index, lse):
    import torch
    return [("top_logits", top_logits, (torch.bfloat16 if p.top_dtype == BF16 else torch.float32,), p.T * p.K, False),
            ("top_index", top_index, (torch.int32 if p.index_dtype == I32 else torch.int64,), p.T * p.K, False),
            ("lse", lse, (torch.float32,), p.T, p.tail == TAIL_RENORM)], []


def kd_ce_fwd_raw(params, h, W, labels, mask, loss, per_token_loss, workspace, stream=None):
    """Thin call: all tensors are the caller's (mask and per_token_loss may be None)."""
    _head_call("kd_ce_fwd", params, _label_inputs(params, labels), h, W, mask, loss, per_token_loss, None, workspace, stream)


def kd_ce_fwd_bwd_raw(params, h, W, labels, mask, loss, per_token_loss, grad_h, grad_W, workspace, stream=None):
    """Thin call: all tensors are the caller's (mask, per_token_loss and one of the gradients may be None)."""
    _head_call("kd_ce_fwd_bwd", params, _label_inputs(params, labels), h, W, mask, loss, per_token_loss, (grad_h, grad_W),
               workspace, stream)


def kd_topk_fwd_raw(params, top_logits, top_index, lse, h_s, W_s, mask, loss, per_token_loss, workspace, stream=None):
    """Thin call: all tensors are the caller's (mask and per_token_loss may be None, lse with TAIL_RENORM)."""
    _head_call("kd_topk_fwd", params, _top_inputs(params, top_logits, top_index, lse), h_s, W_s, mask, loss, per_token_loss,
               None, workspace, stream)


def kd_topk_fwd_bwd_raw(params, top_logits, top_index, lse, h_s, W_s, mask, loss, per_token_loss, grad_h_s, grad_W_s,
                        workspace, stream=None):
    """Thin call: all tensors are the caller's (mask, per_token_loss and one of the gradients may be None, lse with
    TAIL_RENORM)."""
    _head_call("kd_topk_fwd_bwd", params, _top_inputs(params, top_logits, top_index, lse), h_s, W_s, mask, loss,
               per_token_loss, (grad_h_s, grad_W_s), workspace, stream)


def _head_outputs(p, h, W, workspace, grads, grad_W, want):
    """Outputs (and the workspace unless given) of a convenience call."""
    import torch
    dev = h.device
    if workspace is None:
        workspace = alloc_workspace(p, dev)
    loss = torch.empty(1, dtype=torch.float32, device=dev)
    ptl = torch.empty(p.T, dtype=torch.float32, device=dev)
    if not grads:
        return loss, ptl, None, None, workspace
    tdt = torch.bfloat16 if p.grad_dtype == BF16 else torch.float32
    grad_h = torch.empty(h.shape, dtype=tdt, device=dev) if want[0] else None
    if grad_W is None and want[1]:
        grad_W = torch.empty(W.shape, dtype=tdt, device=dev)
    return loss, ptl, grad_h, grad_W, workspace


def kd_ce_fwd_bwd(h, W, labels, mask=None, label_smoothing=0.0, z_loss=0.0, w_layout=W_VH, grad_dtype=None,
                  workspace=None, grad_W=None, accumulate_grad_W=False, vocab_chunk=0, loss_scale=1.0,
                  want_grad_h=True, want_grad_W=True):
    """Cross entropy of `labels` ([T] int32 or int64; negative: the token does not count) under softmax(h W), and its
    gradients.  h [T,H]; W in `w_layout`.  Allocates outputs (and the workspace unless given); returns a dict of tensors."""
    T, H, V, in_dtype = _check_head(h, W, w_layout)
    p = make_ce_params(T, H, V, label_smoothing, z_loss, in_dtype, grad_dtype, w_layout, _index_dtype(labels, "labels"),
                       accumulate_grad_W, vocab_chunk, loss_scale)
    if accumulate_grad_W and grad_W is None:
        raise ValueError("accumulate_grad_W needs the grad_W to add to")
    loss, ptl, gh, gW, ws = _head_outputs(p, h, W, workspace, True, grad_W, (want_grad_h, want_grad_W))
    kd_ce_fwd_bwd_raw(p, h, W, labels, mask, loss, ptl, gh, gW, ws)
    return dict(loss=loss, per_token_loss=ptl, grad_h=gh, grad_W=gW, workspace=ws)


def kd_ce_fwd(h, W, labels, mask=None, label_smoothing=0.0, z_loss=0.0, w_layout=W_VH, workspace=None, loss_scale=1.0):
    """The same without gradients."""
    T, H, V, in_dtype = _check_head(h, W, w_layout)
    p = make_ce_params(T, H, V, label_smoothing, z_loss, in_dtype, None, w_layout, _index_dtype(labels, "labels"),
                       loss_scale=loss_scale)
    loss, ptl, _, _, ws = _head_outputs(p, h, W, workspace, False, None, None)
    kd_ce_fwd_raw(p, h, W, labels, mask, loss, ptl, ws)
    return dict(loss=loss, per_token_loss=ptl)


def _check_top(T, top_logits, top_index):
    if top_index.dim() != 2 or top_index.shape[0] != T or top_logits.shape != top_index.shape:
        raise ValueError(f"top_logits and top_index must be [T, K] with T = {T}, got {tuple(top_logits.shape)} and "
                         f"{tuple(top_index.shape)}")
    return int(top_index.shape[1]), _float_dtype(top_logits, "top_logits"), _index_dtype(top_index, "top_index")


def kd_topk_fwd_bwd(top_logits, top_index, h_s, W_s, lse=None, mask=None, tau=1.0, tail=TAIL_RENORM, w_layout=W_VH,
                    grad_dtype=None, workspace=None, grad_W_s=None, accumulate_grad_W=False, flags=0, vocab_chunk=0,
                    loss_scale=1.0, want_grad_h=True, want_grad_W=True):
    """Divergence of softmax(h_s W_s / tau) from the teacher's top logits ([T,K], with their vocabulary rows top_index, as
    torch.topk returns them; negative rows are entries that are not there), and its gradients.  `tail` says what stands for
    the rest of the teacher's vocabulary; lse [T] is the teacher's log-sum-exp of its logits over tau (not with
    TAIL_RENORM).  Allocates outputs (and the workspace unless given); returns a dict of tensors."""
    T, H, V, in_dtype = _check_head(h_s, W_s, w_layout)
    K, top_dtype, index_dtype = _check_top(T, top_logits, top_index)
    p = make_topk_params(T, H, V, K, tau, tail, in_dtype, grad_dtype, w_layout, index_dtype, top_dtype, accumulate_grad_W,
                         flags, vocab_chunk, loss_scale)
    if accumulate_grad_W and grad_W_s is None:
        raise ValueError("accumulate_grad_W needs the grad_W_s to add to")
    loss, ptl, gh, gW, ws = _head_outputs(p, h_s, W_s, workspace, True, grad_W_s, (want_grad_h, want_grad_W))
    kd_topk_fwd_bwd_raw(p, top_logits, top_index, lse, h_s, W_s, mask, loss, ptl, gh, gW, ws)
    return dict(loss=loss, per_token_loss=ptl, grad_h_s=gh, grad_W_s=gW, workspace=ws)


def kd_topk_fwd(top_logits, top_index, h_s, W_s, lse=None, mask=None, tau=1.0, tail=TAIL_RENORM, w_layout=W_VH,
                workspace=None, flags=0, loss_scale=1.0):
    """The same without gradients."""
    T, H, V, in_dtype = _check_head(h_s, W_s, w_layout)
    K, top_dtype, index_dtype = _check_top(T, top_logits, top_index)
    p = make_topk_params(T, H, V, K, tau, tail, in_dtype, None, w_layout, index_dtype, top_dtype, flags=flags,
                         loss_scale=loss_scale)
    loss, ptl, _, _, ws = _head_outputs(p, h_s, W_s, workspace, False, None, None)
    kd_topk_fwd_raw(p, top_logits, top_index, lse, h_s, W_s, mask, loss, ptl, ws)
    return dict(loss=loss, per_token_loss=ptl)
