"""ctypes binding of librn18.so: the C ABI of include/rn18.h and
include/rn18_ops.h under the same names.

Argument marshalling only: torch tensors provide device memory
(``data_ptr()``) and the HIP stream (``torch.cuda.current_stream()``); every
step of the computation runs in the library's HIP kernels. If the library is
not built, importing a function raises instead of falling back to anything.

Sizes and strides are the caller's. What a caller takes from torch in another
type than the library's (classes of torch.topk in int64, values and scales in
16 bits) is refused by the row operators, and a Worker refuses a teacher's
list or labels of other sizes than the batch's.
"""
import ctypes
import os

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "librn18.so")

RN18_OK, RN18_EINVAL, RN18_ELABEL, RN18_ENOMEM, RN18_EHIP, RN18_ENONFINITE = 0, -1, -2, -3, -4, -5
RN18_TINY, RN18_CIFAR, RN18_IMAGENET = 0, 1, 2
RN18_FP32, RN18_BF16, RN18_FP16 = 0, 1, 2
ARCH_IDS = {"tiny": RN18_TINY, "cifar": RN18_CIFAR, "imagenet": RN18_IMAGENET}
PREC_IDS = {"fp32": RN18_FP32, "bf16": RN18_BF16, "fp16": RN18_FP16}

# Every symbol the headers declare (checked by the CPU test suite).
EXPORTED = [
    "rn18_state_floats", "rn18_init", "rn18_workspace_bytes", "rn18_set_workspace", "rn18_train_step",
    "rn18_eval_logits", "ps_dual_merge", "ps_worker_delta", "rn18_sync_status", "rn18_get_momentum",
    "rn18_set_momentum", "rn18_set_dropout", "rn18_set_loss_scale", "rn18_get_loss_scale", "rn18_destroy",
    "rn18_last_error", "rn18_profile_enable",
    "rn18_profile_read",
    "rn18op_conv2d_fwd", "rn18op_conv2d_dgrad", "rn18op_conv2d_wgrad_workspace", "rn18op_conv2d_wgrad",
    "rn18op_maxpool_fwd", "rn18op_maxpool_bwd", "rn18_debug_set", "rn18_debug_copy",
    "rn18_debug_capture", "rn18op_round_bf16", "rn18op_conv2d_wgrad_noalloc_limit", "rn18op_conv2d_wgrad_noalloc",
    "rn18_train_step_distill", "rn18op_layernorm_fwd", "rn18op_layernorm_bwd_workspace", "rn18op_layernorm_bwd",
    "rn18op_topk_logits_workspace", "rn18op_topk_logits", "rn18op_distill_loss_workspace", "rn18op_distill_loss",
]


class Rn18Error(RuntimeError):
    def __init__(self, code, msg):
        super().__init__("rn18 error %d: %s" % (code, msg))
        self.code = code


class rn18_prof_rec(ctypes.Structure):
    _fields_ = [("cls", ctypes.c_int), ("layer", ctypes.c_int), ("tile", ctypes.c_int), ("pad_", ctypes.c_int),
                ("flops", ctypes.c_double), ("bytes", ctypes.c_double), ("ms", ctypes.c_double),
                ("kernel", ctypes.c_char * 104)]


K_NAMES = ["conv_fwd", "conv_dgrad", "conv_wgrad", "wgrad_reduce", "bn_stats", "bn_apply", "bn_bwd_reduce",
           "bn_bwd_apply", "maxpool", "avgpool", "head", "sgd", "prep"]


class rn18_config(ctypes.Structure):
    _fields_ = [("arch", ctypes.c_int), ("num_classes", ctypes.c_int), ("prec", ctypes.c_int),
                ("momentum", ctypes.c_float), ("weight_decay", ctypes.c_float), ("bn_eps", ctypes.c_float),
                ("bn_momentum", ctypes.c_float)]


_lib = None
_P = ctypes.c_void_p
_I = ctypes.c_int
_Z = ctypes.c_size_t
_F = ctypes.c_float
_L = ctypes.c_int64


def lib():
    """Load the HIP library; raise if it is not built (no fallback)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError("librn18.so is not built (run __graft_entry__.build()); there is no fallback path")
    L = ctypes.CDLL(LIB_PATH)
    sig = {
        "rn18_state_floats": (_Z, [ctypes.POINTER(rn18_config), ctypes.POINTER(_Z)]),
        "rn18_init": (_I, [ctypes.POINTER(rn18_config), ctypes.c_uint64, _P, _P, ctypes.POINTER(_P)]),
        "rn18_workspace_bytes": (_Z, [_P, _I, _I, _I]),
        "rn18_set_workspace": (_I, [_P, _P, _Z]),
        "rn18_train_step": (_I, [_P, _P, _P, _P, _I, _I, _I, _F, _P]),
        "rn18_eval_logits": (_I, [_P, _P, _P, _I, _I, _I, _P]),
        "ps_dual_merge": (_I, [_P, _P, _P, _Z, _F, _P]),
        "ps_worker_delta": (_I, [_P, _P, _P, _Z, _P]),
        "rn18_sync_status": (_I, [_P]),
        "rn18_get_momentum": (_I, [_P, _P]),
        "rn18_set_momentum": (_I, [_P, _P]),
        "rn18_set_dropout": (_I, [_P, _F, ctypes.c_uint64, ctypes.c_uint64]),
        "rn18_set_loss_scale": (_I, [_P, _F, ctypes.c_uint]),
        "rn18_get_loss_scale": (_I, [_P, ctypes.POINTER(_F), ctypes.POINTER(ctypes.c_uint64)]),
        "rn18_destroy": (None, [_P]),
        "rn18_last_error": (ctypes.c_char_p, []),
        "rn18op_conv2d_fwd": (_I, [_I, _P, _P, _P, _I, _I, _I, _I, _I, _I, _I, _I, _P]),
        "rn18op_conv2d_dgrad": (_I, [_I, _P, _P, _P, _I, _I, _I, _I, _I, _I, _I, _I, _P]),
        "rn18op_conv2d_wgrad_workspace": (_Z, [_I, _I, _I, _I, _I, _I, _I, _I, _I]),
        "rn18op_conv2d_wgrad": (_I, [_I, _P, _P, _P, _I, _I, _I, _I, _I, _I, _I, _I, _I, _P, _Z, _P]),
        "rn18op_conv2d_wgrad_noalloc_limit": (_Z, []),
        "rn18op_conv2d_wgrad_noalloc": (_I, [_I, _P, _P, _P, _I, _I, _I, _I, _I, _I, _I, _I, _I, _P]),
        "rn18op_maxpool_fwd": (_I, [_I, _P, _P, _P, _I, _I, _I, _I, _P]),
        "rn18op_maxpool_bwd": (_I, [_I, _P, _P, _P, _I, _I, _I, _I, _P]),
        "rn18op_round_bf16": (_I, [_P, _P, _Z, _P]),
        "rn18_train_step_distill": (_I, [_P, _P, _P, _P, _P, _P, _I, _F, _F, _I, _I, _I, _F, _P]),
        "rn18op_layernorm_fwd": (_I, [_I, _P, _P, _P, _P, _P, _P, _L, _I, _L, _L, _F, _P]),
        "rn18op_layernorm_bwd_workspace": (_Z, [_I, _L, _I]),
        "rn18op_layernorm_bwd": (_I, [_I, _P, _P, _P, _P, _P, _P, _P, _P, _L, _I, _L, _L, _L, _P, _Z, _P]),
        "rn18op_topk_logits_workspace": (_Z, [_I, _L, _I, _I]),
        "rn18op_topk_logits": (_I, [_I, _P, _P, _P, _L, _I, _L, _I, _P, _Z, _P]),
        "rn18op_distill_loss_workspace": (_Z, [_I, _L, _I, _I]),
        "rn18op_distill_loss": (_I, [_I, _P, _P, _P, _P, _P, _P, _P, _P, _L, _I, _L, _L, _I, _F, _F, _F, _P, _Z,
                                     _P]),
        "rn18_debug_set": (_I, [_P, _I, ctypes.c_long]),
        "rn18_profile_enable": (_I, [_P, _I]),
        "rn18_profile_read": (_I, [_P, ctypes.POINTER(rn18_prof_rec), _I, ctypes.POINTER(_I)]),
        "rn18_debug_copy": (_I, [_P, _I, _I, _I, _I, _I, _P, _Z]),
        "rn18_debug_capture": (_I, [_P, _I, _I, _P, _Z]),
    }
    for name, (res, args) in sig.items():
        f = getattr(L, name)
        f.restype = res
        f.argtypes = args
    _lib = L
    return L


def _check(code):
    if code != RN18_OK:
        raise Rn18Error(code, lib().rn18_last_error().decode())
    return code


def _ptr(t):
    return None if t is None else t.data_ptr()


class _Types(dict):
    """torch's type of a name, looked up once."""

    def __missing__(self, name):
        import torch
        t = self[name] = getattr(torch, name)
        return t


_types = _Types()


def _arr(t, kind, name, n=0):
    """The pointer of an array of type `kind` with n elements at least, or
    None. (0.1 us more than _ptr, with n 0.3.)"""
    if t is None:
        return None
    if t.dtype is _types[kind] and (not n or t.numel() >= n and t.is_contiguous()):
        return t.data_ptr()
    raise Rn18Error(RN18_EINVAL, "%s must be %s%s, not %s of shape %s and strides %s"
                    % (name, kind, ", %d elements one after the other" % n if n else "", t.dtype, tuple(t.shape),
                       t.stride()))


_current_handle = None   # the function that gives the handle of torch's current stream


def _stream(stream=None):
    """The HIP stream of `stream`, or torch's current one. torch is asked for
    its handle by device where it can be: 0.2 us in place of the 2.9 of a
    torch.cuda.Stream object (a layer norm of 64x512 fp32, one call after the
    other: 4.7 and 7.6 us)."""
    global _current_handle
    if stream is not None:
        return stream.cuda_stream
    if _current_handle is None:
        import torch
        by_device = getattr(torch._C, "_cuda_getCurrentRawStream", None)
        torch.cuda.current_device()   # (starts CUDA, which its own short form expects)
        device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
        _current_handle = (lambda: by_device(device())) if by_device else \
            (lambda: torch.cuda.current_stream().cuda_stream)
    return _current_handle()


def make_config(arch, num_classes, prec="fp32", momentum=0.9, weight_decay=5e-4, bn_eps=1e-5, bn_momentum=0.1):
    return rn18_config(ARCH_IDS[arch] if isinstance(arch, str) else arch, num_classes,
                       PREC_IDS[prec] if isinstance(prec, str) else prec, momentum, weight_decay, bn_eps,
                       bn_momentum)


# ------------------------------------------------------------------ C ABI, same names
def rn18_state_floats(cfg):
    p = _Z(0)
    total = lib().rn18_state_floats(ctypes.byref(cfg), ctypes.byref(p))
    if total == 0:
        raise Rn18Error(RN18_EINVAL, "invalid config")
    return total, p.value


def rn18_init(cfg, seed, state_out=None, stream=None):
    h = _P()
    _check(lib().rn18_init(ctypes.byref(cfg), ctypes.c_uint64(seed), _stream(stream), _ptr(state_out), ctypes.byref(h)))
    return h


def rn18_workspace_bytes(ctx, N, H, W):
    return lib().rn18_workspace_bytes(ctx, N, H, W)


def rn18_set_workspace(ctx, ws):
    _check(lib().rn18_set_workspace(ctx, _ptr(ws), ws.numel() * ws.element_size()))


def rn18_train_step(ctx, state, images, labels, N, H, W, lr, loss=None):
    return _check(lib().rn18_train_step(ctx, _ptr(state), _ptr(images), _ptr(labels), N, H, W, lr, _ptr(loss)))


def rn18_train_step_distill(ctx, state, images, labels, t_vals, t_idx, K, temperature, alpha, N, H, W, lr, loss=None):
    return _check(lib().rn18_train_step_distill(ctx, _ptr(state), _ptr(images), _arr(labels, "int32", "labels", N),
                                                _arr(t_vals, "float32", "t_vals", N * K),
                                                _arr(t_idx, "int32", "t_idx", N * K), K, temperature, alpha, N, H, W,
                                                lr, _ptr(loss)))


def rn18_eval_logits(ctx, state, images, N, H, W, logits):
    return _check(lib().rn18_eval_logits(ctx, _ptr(state), _ptr(images), N, H, W, _ptr(logits)))


def ps_dual_merge(state, g_small, g_large, n, factor, stream=None):
    return _check(lib().ps_dual_merge(_ptr(state), _ptr(g_small), _ptr(g_large), n, factor, _stream(stream)))


def ps_worker_delta(pulled, local, delta, n, stream=None):
    return _check(lib().ps_worker_delta(_ptr(pulled), _ptr(local), _ptr(delta), n, _stream(stream)))


def rn18_sync_status(ctx):
    return lib().rn18_sync_status(ctx)


def rn18_set_dropout(ctx, p, seed, step):
    return _check(lib().rn18_set_dropout(ctx, ctypes.c_float(p), ctypes.c_uint64(seed), ctypes.c_uint64(step)))


def rn18_set_loss_scale(ctx, scale, growth_interval=2000):
    return _check(lib().rn18_set_loss_scale(ctx, ctypes.c_float(scale), ctypes.c_uint(growth_interval)))


def rn18_get_loss_scale(ctx):
    """(scale, skipped steps) of an fp16 context."""
    sc, sk = _F(0.0), ctypes.c_uint64(0)
    _check(lib().rn18_get_loss_scale(ctx, ctypes.byref(sc), ctypes.byref(sk)))
    return sc.value, sk.value


def rn18_get_momentum(ctx, dst):
    return _check(lib().rn18_get_momentum(ctx, _ptr(dst)))


def rn18_set_momentum(ctx, src):
    return _check(lib().rn18_set_momentum(ctx, _ptr(src)))


def rn18_destroy(ctx):
    lib().rn18_destroy(ctx)


def rn18_profile_enable(ctx, on):
    return _check(lib().rn18_profile_enable(ctx, 1 if on else 0))


def rn18_profile_read(ctx, max_records=4096):
    """Profile records (kernel class, layer, tile, kernel name, flops, bytes, ms) in launch order."""
    buf = (rn18_prof_rec * max_records)()
    n = _I(0)
    _check(lib().rn18_profile_read(ctx, buf, max_records, ctypes.byref(n)))
    return [dict(cls=K_NAMES[r.cls], layer=r.layer, tile=r.tile, kernel=r.kernel.decode(), flops=r.flops,
                 bytes=r.bytes, ms=r.ms)
            for r in buf[:min(n.value, max_records)]]


def rn18_last_error():
    return lib().rn18_last_error().decode()


def rn18op_conv2d_fwd(prec, x, w, y, N, H, W, Cin, Cout, k, s, p, stream=None):
    return _check(lib().rn18op_conv2d_fwd(prec, _ptr(x), _ptr(w), _ptr(y), N, H, W, Cin, Cout, k, s, p, _stream(stream)))


def rn18op_conv2d_dgrad(prec, dy, w, dx, N, H, W, Cin, Cout, k, s, p, stream=None):
    return _check(lib().rn18op_conv2d_dgrad(prec, _ptr(dy), _ptr(w), _ptr(dx), N, H, W, Cin, Cout, k, s, p,
                                            _stream(stream)))


def rn18op_conv2d_wgrad_workspace(prec, N, H, W, Cin, Cout, k, s, p):
    return lib().rn18op_conv2d_wgrad_workspace(prec, N, H, W, Cin, Cout, k, s, p)


def rn18op_conv2d_wgrad(prec, dy, x, dw, N, H, W, Cin, cin_real, Cout, k, s, p, ws, stream=None):
    return _check(lib().rn18op_conv2d_wgrad(prec, _ptr(dy), _ptr(x), _ptr(dw), N, H, W, Cin, cin_real, Cout, k, s, p,
                                            _ptr(ws), ws.numel() * ws.element_size(), _stream(stream)))


def rn18op_conv2d_wgrad_noalloc_limit():
    return lib().rn18op_conv2d_wgrad_noalloc_limit()


def rn18op_conv2d_wgrad_noalloc(prec, dy, x, dw, N, H, W, Cin, cin_real, Cout, k, s, p, stream=None):
    return _check(lib().rn18op_conv2d_wgrad_noalloc(prec, _ptr(dy), _ptr(x), _ptr(dw), N, H, W, Cin, cin_real, Cout,
                                                    k, s, p, _stream(stream)))


def rn18op_maxpool_fwd(prec, x, y, arg, N, H, W, C, stream=None):
    return _check(lib().rn18op_maxpool_fwd(prec, _ptr(x), _ptr(y), _ptr(arg), N, H, W, C, _stream(stream)))


def rn18op_maxpool_bwd(prec, dy, arg, dx, N, H, W, C, stream=None):
    return _check(lib().rn18op_maxpool_bwd(prec, _ptr(dy), _ptr(arg), _ptr(dx), N, H, W, C, _stream(stream)))


def rn18op_round_bf16(x, y, n, stream=None):
    return _check(lib().rn18op_round_bf16(_ptr(x), _ptr(y), n, _stream(stream)))


def _ws(t):
    """(pointer, bytes) of a workspace tensor or None."""
    return (None, 0) if t is None else (_ptr(t), t.numel() * t.element_size())


def rn18op_layernorm_fwd(prec, x, gamma, beta, y, mean, rstd, R, D, ldx, ldy, eps=1e-5, stream=None):
    r = (_lib or lib()).rn18op_layernorm_fwd(prec, _ptr(x), _arr(gamma, "float32", "gamma"),
                                             _arr(beta, "float32", "beta"), _ptr(y), _ptr(mean), _ptr(rstd), R, D, ldx,
                                             ldy, eps, _stream(stream))
    return _check(r) if r else r


def rn18op_layernorm_bwd_workspace(prec, R, D):
    return lib().rn18op_layernorm_bwd_workspace(prec, R, D)


def rn18op_layernorm_bwd(prec, dy, x, gamma, mean, rstd, dx, dgamma, dbeta, R, D, lddy, ldx, lddx, ws=None,
                         stream=None):
    r = (_lib or lib()).rn18op_layernorm_bwd(prec, _ptr(dy), _ptr(x), _arr(gamma, "float32", "gamma"), _ptr(mean),
                                             _ptr(rstd), _ptr(dx), _arr(dgamma, "float32", "dgamma"),
                                             _arr(dbeta, "float32", "dbeta"), R, D, lddy, ldx, lddx, *_ws(ws),
                                             _stream(stream))
    return _check(r) if r else r


def rn18op_topk_logits_workspace(prec, R, C, K):
    return lib().rn18op_topk_logits_workspace(prec, R, C, K)


def rn18op_topk_logits(prec, z, vals, idx, R, C, ldz, K, ws=None, stream=None):
    r = (_lib or lib()).rn18op_topk_logits(prec, _ptr(z), _arr(vals, "float32", "vals"), _arr(idx, "int32", "idx"), R,
                                           C, ldz, K, *_ws(ws), _stream(stream))
    return _check(r) if r else r


def rn18op_distill_loss_workspace(prec, R, C, K):
    return lib().rn18op_distill_loss_workspace(prec, R, C, K)


def rn18op_distill_loss(prec, z, t_vals, t_idx, labels, row_weight, dz, row_loss, loss, R, C, ldz, lddz, K,
                        temperature, alpha, scale, ws=None, stream=None):
    n = R * K
    r = (_lib or lib()).rn18op_distill_loss(prec, _ptr(z), _arr(t_vals, "float32", "t_vals", n),
                                            _arr(t_idx, "int32", "t_idx", n), _arr(labels, "int32", "labels", R),
                                            _arr(row_weight, "float32", "row_weight", R), _ptr(dz), _ptr(row_loss),
                                            _ptr(loss), R, C, ldz, lddz, K, temperature, alpha, scale, *_ws(ws),
                                            _stream(stream))
    return _check(r) if r else r


DBG = dict(y=0, z1=1, out=2, gA=3, gB=4, gz=5, gy=6, gyd=7, grad=8, wf=9, wd=10, mean=11, rstd=12, zstem=13,
           parg=14)


RN18_DBG_STOP_BLOCKS, RN18_DBG_GATHER_CONFIG, RN18_DBG_WGRAD_CONFIG, RN18_DBG_CONV_CHUNK, RN18_DBG_SERIAL = 0, 1, 2, 3, 4
RN18_DBG_GATHER_SPLIT = 5


def rn18_debug_set(ctx, key, value):
    return _check(lib().rn18_debug_set(ctx, key, value))


CAP = dict(dy=0, dz1=1, dx=3, da_avg=4, da_pool=5)


def rn18_debug_capture(ctx, kind, index, dst):
    if dst is None:
        return _check(lib().rn18_debug_capture(ctx, 0, 0, None, 0))
    return _check(lib().rn18_debug_capture(ctx, CAP[kind] if isinstance(kind, str) else kind, index, _ptr(dst),
                                           dst.numel() * dst.element_size()))


def rn18_debug_copy(ctx, N, H, W, which, index, dst):
    return _check(lib().rn18_debug_copy(ctx, N, H, W, DBG[which] if isinstance(which, str) else which, index,
                                        _ptr(dst), dst.numel() * dst.element_size()))


# ------------------------------------------------------------------ thin owner of a context
class Worker:
    """One training context (a parameter-server worker): the library context
    plus a torch-allocated device workspace sized for the largest shape seen.
    Holds no state of its own beyond memory ownership.

    The context is bound to `stream` (torch's current stream at construction
    by default); the workspace is allocated on that stream, so torch's
    allocator hands a replaced workspace to later allocations only in that
    stream's order, after every step that used it."""

    def __init__(self, arch, num_classes, prec="fp32", seed=0, state=None, stream=None, **hyper):
        import torch
        self.cfg = make_config(arch, num_classes, prec, **hyper)
        self.n_state, self.n_trainable = rn18_state_floats(self.cfg)
        self.stream = stream if stream is not None else torch.cuda.current_stream()
        self.ctx = rn18_init(self.cfg, seed, state, stream=self.stream)
        self.ws = None
        self.torch = torch

    def _ensure(self, N, H, W):
        need = rn18_workspace_bytes(self.ctx, N, H, W)
        if need == 0:
            raise Rn18Error(RN18_EINVAL, rn18_last_error())
        if self.ws is None or self.ws.numel() < need:
            with self.torch.cuda.stream(self.stream):
                ws = self.torch.empty(need, dtype=self.torch.uint8, device="cuda")
            rn18_set_workspace(self.ctx, ws)
            self.ws = ws

    def train_step(self, state, images, labels, lr, loss=None):
        N, _, H, W = images.shape
        self._ensure(N, H, W)
        return rn18_train_step(self.ctx, state, images, labels, N, H, W, lr, loss)

    def train_step_distill(self, state, images, labels, t_vals, t_idx, temperature, alpha, lr, loss=None):
        """A step against a teacher's top logits: t_vals fp32 and t_idx int32
        [N][K], labels int32 [N] or None for alpha = 1, all contiguous and on
        the images' device."""
        N, _, H, W = images.shape
        K = t_vals.shape[-1]
        for t, kind, shape, name in ((t_vals, "float32", (N, K), "t_vals"), (t_idx, "int32", (N, K), "t_idx"),
                                     (labels, "int32", (N,), "labels")):
            if t is None:
                continue
            if tuple(t.shape) != shape or t.device != images.device:
                raise Rn18Error(RN18_EINVAL, "%s must be of shape %s on %s, not %s on %s"
                                % (name, shape, images.device, tuple(t.shape), t.device))
            _arr(t, kind, name, t.numel())
        self._ensure(N, H, W)
        return rn18_train_step_distill(self.ctx, state, images, labels, t_vals, t_idx, K, temperature, alpha, N, H, W,
                                       lr, loss)

    def eval_logits(self, state, images, logits):
        N, _, H, W = images.shape
        self._ensure(N, H, W)
        return rn18_eval_logits(self.ctx, state, images, N, H, W, logits)

    def sync_status(self):
        return rn18_sync_status(self.ctx)

    def close(self):
        if self.ctx:
            rn18_destroy(self.ctx)
            self.ctx = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
