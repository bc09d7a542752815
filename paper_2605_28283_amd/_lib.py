"""ctypes binding of libprunepath.so -- argument marshalling only.

Every function has the name and argument order of the C entry point declared
in include/prunepath.h.  Array arguments may be torch tensors on the current
HIP device (their data pointer is passed; bf16 arrays may be typed bfloat16,
int16 or uint16) or raw integer device addresses.  A non-OK status raises
PrunePathError.  There is no fallback: if the shared library is missing the
import fails.
"""
import ctypes
import os

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libprunepath.so")

PP_OK = 0
PP_EINVAL = 1
PP_ENOMEM = 2
PP_EHIP = 3
PP_EUNSUPPORTED = 4
PP_ENOTCONVERGED = 5

PP_SELECT_NUCLEUS = 0
PP_SELECT_STRICT = 1
PP_SELECT_TOPK = 4
PP_SELECT_LTE = 8
PP_AGG_SUM = 0
PP_AGG_SIGMOID = 2

PP_SCORE_SOFTMAX = 0
PP_SCORE_SIGMOID = 1
PP_TOPK_RENORM = 2
PP_GROUP_TOP2 = 4
PP_GRAD_ADD = 8
PP_NORM_F32 = 1

PP_KERNEL_ROUTE = 0
PP_KERNEL_DISPATCH = 1
PP_KERNEL_GATEUP = 2
PP_KERNEL_DOWN = 3
PP_KERNEL_COUNT = 4

EXPORTED = ("prunepath_create", "prunepath_create_mlp", "prunepath_route", "prunepath_ffn_decode",
            "prunepath_ffn_prefill", "prunepath_destroy", "prunepath_status_string",
            "prunepath_profile_begin", "prunepath_profile_end", "prunepath_residual_rmsnorm",
            "prunepath_router_loss_workspace", "prunepath_router_loss",
            "prunepath_router_loss_noalloc",
            "prunepath_route_topk", "prunepath_route_topk_logits", "prunepath_route_topk_grad",
            "prunepath_ffn_decode_routed", "prunepath_ffn_prefill_routed",
            "prunepath_residual_layernorm", "prunepath_residual_layernorm_grad_workspace",
            "prunepath_residual_layernorm_grad",
            "prunepath_kmeans_workspace", "prunepath_balanced_kmeans")


class PrunePathError(RuntimeError):
    def __init__(self, status, where):
        self.status = status
        super().__init__("%s: %s (status %d)" % (where, _status_text(status), status))


_lib = None


def load():
    """Load the HIP library (raises OSError if it has not been built).

    torch is imported first: its wheel carries its own HIP runtime, which the
    process must share with the library.  Both runtimes have the soname
    libamdhip64.so.7, but torch asks for it by the unversioned name, so a
    library loaded before torch would bind to the system runtime and torch
    would then map its own: device memory from one runtime and kernel launches
    on the other fail."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise OSError("libprunepath.so not built: run __graft_entry__.build() "
                          "or python paper_2605_28283_amd/build.py")
        import torch  # noqa: F401  (maps torch's HIP runtime before the library's dependency)
        lib = ctypes.CDLL(LIB_PATH)
        P, I32, U32, F32 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_uint32, ctypes.c_float
        lib.prunepath_create.argtypes = [ctypes.POINTER(ctypes.c_void_p), I32, I32, I32, I32,
                                         P, P, P, P, P, P, U32, P]
        lib.prunepath_create.restype = ctypes.c_int
        lib.prunepath_create_mlp.argtypes = [ctypes.POINTER(ctypes.c_void_p), I32, I32, I32, I32,
                                             P, P, P, P, P, P, P, U32, P]
        lib.prunepath_create_mlp.restype = ctypes.c_int
        lib.prunepath_route.argtypes = [P, P, I32, F32, P, P, P, P, P]
        lib.prunepath_route.restype = ctypes.c_int
        for f in (lib.prunepath_ffn_decode, lib.prunepath_ffn_prefill):
            f.argtypes = [P, P, I32, F32, P, P, P, P, P]
            f.restype = ctypes.c_int
        lib.prunepath_destroy.argtypes = [P]
        lib.prunepath_destroy.restype = None
        lib.prunepath_profile_begin.argtypes = [P, I32]
        lib.prunepath_profile_begin.restype = ctypes.c_int
        lib.prunepath_profile_end.argtypes = [P, ctypes.POINTER(ctypes.c_double),
                                              ctypes.POINTER(ctypes.c_int32)]
        lib.prunepath_profile_end.restype = ctypes.c_int
        lib.prunepath_residual_rmsnorm.argtypes = [P, P, P, I32, I32, F32, P, P]
        lib.prunepath_residual_rmsnorm.restype = ctypes.c_int
        lib.prunepath_router_loss_workspace.argtypes = [I32, I32]
        lib.prunepath_router_loss_workspace.restype = ctypes.c_size_t
        lib.prunepath_router_loss.argtypes = [P, I32, I32, F32, F32, F32, F32, P, P, P, P]
        lib.prunepath_router_loss.restype = ctypes.c_int
        lib.prunepath_router_loss_noalloc.argtypes = [P, I32, I32, F32, F32, F32, F32, P, P, P]
        lib.prunepath_router_loss_noalloc.restype = ctypes.c_int
        lib.prunepath_route_topk.argtypes = [P, P, I32, P, I32, I32, I32, P, F32, U32, P, P, P, P]
        lib.prunepath_route_topk_logits.argtypes = [P, I32, I32, I32, I32, I32, P, F32, U32, P, P,
                                                    P]
        lib.prunepath_route_topk_grad.argtypes = [P, I32, I32, I32, P, P, F32, U32, P, P]
        lib.prunepath_ffn_decode_routed.argtypes = [P, P, I32, I32, P, P, P, P]
        lib.prunepath_ffn_prefill_routed.argtypes = [P, P, I32, I32, P, P, P, P]
        lib.prunepath_residual_layernorm.argtypes = [P, P, P, I32, I32, F32, P, P, P, P, U32, P]
        lib.prunepath_residual_layernorm_grad_workspace.argtypes = [I32, I32]
        lib.prunepath_residual_layernorm_grad_workspace.restype = ctypes.c_size_t
        lib.prunepath_residual_layernorm_grad.argtypes = [P, P, P, I32, I32, P, P, P, P, P, P, U32,
                                                          P]
        for f in (lib.prunepath_route_topk, lib.prunepath_route_topk_logits,
                  lib.prunepath_route_topk_grad, lib.prunepath_ffn_decode_routed,
                  lib.prunepath_ffn_prefill_routed, lib.prunepath_residual_layernorm,
                  lib.prunepath_residual_layernorm_grad):
            f.restype = ctypes.c_int
        lib.prunepath_kmeans_workspace.argtypes = [I32, I32, I32]
        lib.prunepath_kmeans_workspace.restype = ctypes.c_size_t
        lib.prunepath_balanced_kmeans.argtypes = [P, I32, I32, I32, P, I32, P, P, P, P, P, P, P,
                                                  P]
        lib.prunepath_balanced_kmeans.restype = ctypes.c_int
        lib.prunepath_status_string.argtypes = [ctypes.c_int]
        lib.prunepath_status_string.restype = ctypes.c_char_p
        _lib = lib
    return _lib


def _status_text(s):
    try:
        return load().prunepath_status_string(int(s)).decode()
    except OSError:
        return "unknown"


_KINDS = None


def _kinds():
    """The torch types that an argument of each kind may have."""
    global _KINDS
    if _KINDS is None:
        import torch
        _KINDS = {"bf16": {torch.bfloat16, torch.int16, torch.uint16}, "f32": {torch.float32},
                  "i32": {torch.int32}}
    return _KINDS


def _ptr(a, kind=None):
    """Device address of a tensor (checked) or an int; None -> NULL."""
    if a is None:
        return None
    if isinstance(a, int):
        return a
    if not a.is_cuda:
        raise ValueError("array arguments must live on the GPU")
    if not a.is_contiguous():
        raise ValueError("array arguments must be contiguous")
    want = _kinds().get(kind)
    if want is not None and a.dtype not in want:
        raise TypeError("expected %s array, got %s" % (kind, a.dtype))
    return a.data_ptr()


def _arg(a, kind, n, name, dev):
    """_ptr for the calls that also know how many elements they touch and on
    which device they run: one pass over a tensor's properties, the reasons
    only where one does not hold."""
    if a is None or isinstance(a, int):
        return a
    if (a.get_device() == dev and a.is_contiguous() and a.numel() >= n
            and (kind is None or a.dtype in (_KINDS or _kinds())[kind])):
        return a.data_ptr()
    _ptr(a, kind)  # raises for anything but the device and the size
    if a.get_device() != dev:
        raise ValueError("%s is on %s, the current device is cuda:%d" % (name, a.device, dev))
    raise ValueError("%s: %d elements, the call needs %d" % (name, a.numel(), n))


_dims = {}  # (d, E) of the handles made here: what the calls on them touch


def _sizes(handle):
    """(d, E) of a handle; zeros, which ask nothing of an array, for one made elsewhere."""
    return _dims.get(handle, (0, 0))


_current = None  # (current device's index, its current stream's handle by index)


def _current_calls():
    """torch's calls for the current device and stream: the ones that return
    plain numbers, where this torch has them (0.1 us; the stream's object
    takes 3)."""
    global _current
    if _current is None:
        import torch
        device = getattr(torch._C, "_cuda_getDevice", None)
        stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
        torch.cuda.current_device()  # initialises the device
        _current = (device or torch.cuda.current_device,
                    stream or (lambda i: torch.cuda.current_stream(i).cuda_stream))
    return _current


def _place(stream):
    """(current device's index, handle of `stream` or of the current one)."""
    device, raw = _current or _current_calls()
    i = device()
    return i, raw(i) if stream is None else _stream(stream)


def _stream(stream):
    if stream is None:
        device, raw = _current or _current_calls()
        return raw(device())
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


def _check(st, where):
    if st != PP_OK:
        raise PrunePathError(st, where)


def prunepath_status_string(status):
    return _status_text(status)


def prunepath_create(d, d_ff, E, max_tokens, W_r, W_gate, W_up, W_down, perm=None,
                     router_bias=None, flags=0, stream=None):
    """Returns an opaque handle (int)."""
    out = ctypes.c_void_p()
    st = load().prunepath_create(ctypes.byref(out), d, d_ff, E, max_tokens,
                                 _ptr(W_r, "bf16"), _ptr(W_gate, "bf16"), _ptr(W_up, "bf16"),
                                 _ptr(W_down, "bf16"), _ptr(perm, "i32"),
                                 _ptr(router_bias, "f32"), flags, _stream(stream))
    _check(st, "prunepath_create")
    _dims[out.value] = (d, E)
    return out.value


def prunepath_create_mlp(d, d_ff, E, max_tokens, W_r, W_fc, b_fc, W_proj, b_proj, perm=None,
                         router_bias=None, flags=0, stream=None):
    """Non-gated GELU MLP layer (b_fc / b_proj may be None).  Returns a handle."""
    out = ctypes.c_void_p()
    st = load().prunepath_create_mlp(ctypes.byref(out), d, d_ff, E, max_tokens,
                                     _ptr(W_r, "bf16"), _ptr(W_fc, "bf16"), _ptr(b_fc, "f32"),
                                     _ptr(W_proj, "bf16"), _ptr(b_proj, "f32"), _ptr(perm, "i32"),
                                     _ptr(router_bias, "f32"), flags, _stream(stream))
    _check(st, "prunepath_create_mlp")
    _dims[out.value] = (d, E)
    return out.value


def prunepath_route(handle, x, T, tau, inv_temp, expert_idx, count, gate_w=None, stream=None):
    st = load().prunepath_route(handle, _ptr(x, "bf16"), T, tau, _ptr(inv_temp, "f32"),
                                _ptr(expert_idx, "i32"), _ptr(count, "i32"),
                                _ptr(gate_w, "f32"), _stream(stream))
    _check(st, "prunepath_route")


def prunepath_ffn_decode(handle, x, T, tau, inv_temp, y, expert_idx=None, count=None,
                         stream=None):
    st = load().prunepath_ffn_decode(handle, _ptr(x, "bf16"), T, tau, _ptr(inv_temp, "f32"),
                                     _ptr(y, "f32"), _ptr(expert_idx, "i32"), _ptr(count, "i32"),
                                     _stream(stream))
    _check(st, "prunepath_ffn_decode")


def prunepath_ffn_prefill(handle, x, T, tau, inv_temp, y, expert_idx=None, count=None,
                          stream=None):
    st = load().prunepath_ffn_prefill(handle, _ptr(x, "bf16"), T, tau, _ptr(inv_temp, "f32"),
                                      _ptr(y, "f32"), _ptr(expert_idx, "i32"),
                                      _ptr(count, "i32"), _stream(stream))
    _check(st, "prunepath_ffn_prefill")


def prunepath_residual_rmsnorm(x, y, x_out, T, d, eps, u=None, stream=None):
    st = load().prunepath_residual_rmsnorm(_ptr(x, "f32"), _ptr(y, "f32"), _ptr(x_out, "f32"),
                                           T, d, eps, _ptr(u, "bf16"), _stream(stream))
    _check(st, "prunepath_residual_rmsnorm")


def prunepath_route_topk(handle, x, T, inv_temp, k, n_groups, top_groups, sel_bias, scale, flags,
                         expert_idx, gate_w, logits=None, stream=None):
    """k experts per token by the handle's router (include/prunepath.h has the rule)."""
    (v, stream), (d, E) = _place(stream), _sizes(handle)
    st = load().prunepath_route_topk(
        handle, _arg(x, "bf16", T * d, "x", v), T, _arg(inv_temp, "f32", T, "inv_temp", v), k,
        n_groups, top_groups, _arg(sel_bias, "f32", E, "sel_bias", v), scale, flags,
        _arg(expert_idx, "i32", T * k, "expert_idx", v), _arg(gate_w, "f32", T * k, "gate_w", v),
        _arg(logits, "f32", T * E, "logits", v), stream)
    _check(st, "prunepath_route_topk")


def prunepath_route_topk_logits(g, T, E, k, n_groups, top_groups, sel_bias, scale, flags,
                                expert_idx, gate_w, stream=None):
    """k experts per row of the logits g [T, E]."""
    v, stream = _place(stream)
    st = load().prunepath_route_topk_logits(
        _arg(g, "f32", T * E, "g", v), T, E, k, n_groups, top_groups,
        _arg(sel_bias, "f32", E, "sel_bias", v), scale, flags,
        _arg(expert_idx, "i32", T * k, "expert_idx", v), _arg(gate_w, "f32", T * k, "gate_w", v),
        stream)
    _check(st, "prunepath_route_topk_logits")


def prunepath_route_topk_grad(g, T, E, k, expert_idx, dgate_w, scale, flags, dg, stream=None):
    """dg = dL/dg of the rows' weights (added to dg with PP_GRAD_ADD)."""
    v, stream = _place(stream)
    st = load().prunepath_route_topk_grad(
        _arg(g, "f32", T * E, "g", v), T, E, k, _arg(expert_idx, "i32", T * k, "expert_idx", v),
        _arg(dgate_w, "f32", T * k, "dgate_w", v), scale, flags, _arg(dg, "f32", T * E, "dg", v),
        stream)
    _check(st, "prunepath_route_topk_grad")


def _ffn_routed(name, handle, x, T, k, expert_idx, gate_w, y, stream):
    (v, stream), (d, _) = _place(stream), _sizes(handle)
    st = getattr(load(), name)(handle, _arg(x, "bf16", T * d, "x", v), T, k,
                               _arg(expert_idx, "i32", T * k, "expert_idx", v),
                               _arg(gate_w, "f32", T * k, "gate_w", v),
                               _arg(y, "f32", T * d, "y", v), stream)
    _check(st, name)


def prunepath_ffn_decode_routed(handle, x, T, k, expert_idx, gate_w, y, stream=None):
    """y = the weighted sum of the given experts' outputs (gate_w None: weights 1)."""
    _ffn_routed("prunepath_ffn_decode_routed", handle, x, T, k, expert_idx, gate_w, y, stream)


def prunepath_ffn_prefill_routed(handle, x, T, k, expert_idx, gate_w, y, stream=None):
    """The same, organised for long batches."""
    _ffn_routed("prunepath_ffn_prefill_routed", handle, x, T, k, expert_idx, gate_w, y, stream)


def prunepath_residual_layernorm(x, y, x_out, T, d, eps, w, b, u, stats=None, flags=0,
                                 stream=None):
    """x_out = x + y, u = its layer norm (y, x_out, w, b, stats may be None)."""
    (v, stream), n = _place(stream), T * d
    st = load().prunepath_residual_layernorm(
        _arg(x, "f32", n, "x", v), _arg(y, "f32", n, "y", v), _arg(x_out, "f32", n, "x_out", v),
        T, d, eps, _arg(w, "f32", d, "w", v), _arg(b, "f32", d, "b", v),
        _arg(u, "f32" if flags & PP_NORM_F32 else "bf16", n, "u", v),
        _arg(stats, "f32", 2 * T, "stats", v), flags, stream)
    _check(st, "prunepath_residual_layernorm")


def prunepath_residual_layernorm_grad_workspace(T, d):
    """Workspace bytes prunepath_residual_layernorm_grad needs (0 for bad sizes)."""
    return int(load().prunepath_residual_layernorm_grad_workspace(T, d))


def prunepath_residual_layernorm_grad(x_out, du, dres, T, d, w, stats, dx, dw=None, db=None,
                                      workspace=None, flags=0, stream=None):
    """dx, and dw and db unless None (then without a workspace if both are)."""
    (v, stream), n, lib = _place(stream), T * d, load()
    ws = _arg(workspace, None, 0, "workspace", v)
    if (dw is not None or db is not None) and ws is not workspace:
        need = lib.prunepath_residual_layernorm_grad_workspace(T, d)
        if workspace.numel() * workspace.element_size() < need:
            raise ValueError("workspace: the call needs %d bytes" % need)
    st = lib.prunepath_residual_layernorm_grad(
        _arg(x_out, "f32", n, "x_out", v),
        _arg(du, "f32" if flags & PP_NORM_F32 else "bf16", n, "du", v),
        _arg(dres, "f32", n, "dres", v), T, d, _arg(w, "f32", d, "w", v),
        _arg(stats, "f32", 2 * T, "stats", v), _arg(dx, "f32", n, "dx", v),
        _arg(dw, "f32", d, "dw", v), _arg(db, "f32", d, "db", v), ws, flags, stream)
    _check(st, "prunepath_residual_layernorm_grad")


def prunepath_router_loss_workspace(B, E):
    """Workspace bytes prunepath_router_loss needs (0 for bad sizes)."""
    return int(load().prunepath_router_loss_workspace(B, E))


def prunepath_router_loss(g, B, E, eps, eta, lam, gamma, losses, dg, workspace, stream=None):
    """losses[4] = [L_ent, L_bal, L_gate, total] and dg = dL/dg (None: skipped)."""
    st = load().prunepath_router_loss(_ptr(g, "f32"), B, E, eps, eta, lam, gamma,
                                      _ptr(losses, "f32"), _ptr(dg, "f32"), _ptr(workspace),
                                      _stream(stream))
    _check(st, "prunepath_router_loss")


def prunepath_router_loss_noalloc(g, B, E, eps, eta, lam, gamma, losses, dg, stream=None):
    """prunepath_router_loss with the library's own device scratch (no
    workspace argument, nothing allocated)."""
    st = load().prunepath_router_loss_noalloc(_ptr(g, "f32"), B, E, eps, eta, lam, gamma,
                                              _ptr(losses, "f32"), _ptr(dg, "f32"),
                                              _stream(stream))
    _check(st, "prunepath_router_loss_noalloc")


def prunepath_kmeans_workspace(n, D, k):
    """Workspace bytes prunepath_balanced_kmeans needs (0 for bad sizes)."""
    return int(load().prunepath_kmeans_workspace(n, D, k))


def prunepath_balanced_kmeans(F, n, D, k, init_centroids, iters, assign, perm, centroids,
                              workspace, objective=None, prices=None, stream=None):
    """Balanced k-means of F's rows (blocks until done).  Returns the auction
    rounds of each iteration as a list."""
    rounds = (ctypes.c_int32 * iters)()
    st = load().prunepath_balanced_kmeans(
        _ptr(F, "bf16"), n, D, k, _ptr(init_centroids, "f32"), iters, _ptr(assign, "i32"),
        _ptr(perm, "i32"), _ptr(centroids, "f32"), _ptr(objective, "f32"), _ptr(prices, "f32"),
        ctypes.cast(rounds, ctypes.c_void_p), _ptr(workspace), _stream(stream))
    _check(st, "prunepath_balanced_kmeans")
    return list(rounds)


def prunepath_profile_begin(handle, capacity):
    _check(load().prunepath_profile_begin(handle, capacity), "prunepath_profile_begin")


def prunepath_profile_end(handle):
    """Returns (ms[PP_KERNEL_COUNT], launches[PP_KERNEL_COUNT]) as lists."""
    ms = (ctypes.c_double * PP_KERNEL_COUNT)()
    n = (ctypes.c_int32 * PP_KERNEL_COUNT)()
    _check(load().prunepath_profile_end(handle, ms, n), "prunepath_profile_end")
    return list(ms), list(n)


def prunepath_destroy(handle):
    if handle:
        _dims.pop(handle, None)
        load().prunepath_destroy(handle)
