"""ctypes binding of include/lp.h.  Same names as the C entry points; tensors are torch
tensors on the GPU (their data_ptr() is what crosses the ABI), the stream is torch's current
stream.  No arithmetic happens here, and there is no CPU fallback: if liblp.so is missing or
fails to load, every call raises."""
import ctypes
import os

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "liblp.so")
_lib = None

LP_ROUND_NEAREST_AWAY = 0
LP_ROUND_NEAREST_EVEN = 1
LP_ROUND_STOCHASTIC = 2
LP_RANGE_WORKSPACE_WORDS = 32
LP_F32, LP_BF16, LP_F16 = 0, 1, 2                                                                # lp_dtype
LP_ACT_NONE, LP_ACT_RELU, LP_ACT_SILU, LP_ACT_GELU_TANH = 0, 1, 2, 3                              # lp_actfn
LP_KERNEL_DIRECT, LP_KERNEL_PATCH, LP_KERNEL_FLAT, LP_KERNEL_ROWS = 0, 1, 2, 3   # lp_plan_info.kernel


class LpError(RuntimeError):
    def __init__(self, status, what):
        self.status = int(status)
        super().__init__("%s failed: status %d (%s)" % (what, status, lp_status_string(status)))


class QFmt(ctypes.Structure):
    """(n, m, f): n total bits, m integer bits including sign, f fraction bits."""
    _fields_ = [("n", ctypes.c_int32), ("m", ctypes.c_int32), ("f", ctypes.c_int32)]

    def __repr__(self):
        return "Q%d.%d(n=%d)" % (self.m, self.f, self.n)

    def astuple(self):
        return (self.n, self.m, self.f)


class PlanInfo(ctypes.Structure):
    _fields_ = [(k, ctypes.c_int32) for k in ("path", "limbs", "bn", "tile_rows", "tile_cols", "patch_rows",
                                               "patch_cols", "tiles_m", "tiles_n", "lds_bytes", "patch_pitch", "patch_pixel",
                                               "workgroups", "split", "items_per_die", "whole_items_per_die", "kernel")]

    def asdict(self):
        return {k: getattr(self, k) for k, _ in self._fields_}


class ZeroMap(ctypes.Structure):
    """Per-tile nonzero flags of a tensor and the tile geometry they were written in (lp_zero_map)."""
    _fields_ = [("flags_dev", ctypes.c_void_p)] + [(k, ctypes.c_int32) for k in ("tile_rows", "tile_cols", "tiles_c", "tiles_n",
                                                                             "bn", "scale")]


class ConvDesc(ctypes.Structure):
    _fields_ = [(k, ctypes.c_int32) for k in ("N", "H", "W", "Cin", "Cout", "R", "S", "stride", "pad", "pool")]


_SIGNATURES = {
    "lp_status_string": (ctypes.c_char_p, [ctypes.c_int]),
    "lp_range": (ctypes.c_int, [ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int, ctypes.c_double,
                                ctypes.POINTER(QFmt), ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p]),
    "lp_range_acc": (ctypes.c_int, [ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int, ctypes.c_int, ctypes.c_int,
                                    ctypes.c_double, ctypes.POINTER(QFmt), ctypes.c_void_p, ctypes.c_void_p,
                                    ctypes.c_void_p]),
    "lp_quantize": (ctypes.c_int, [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_size_t, QFmt, ctypes.c_int,
                                   ctypes.c_uint64, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p]),
    "lp_act": (ctypes.c_int, [ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int, QFmt, ctypes.c_int, ctypes.c_int,
                              ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p]),
    "lp_act_stochastic": (ctypes.c_int, [ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int, QFmt, ctypes.c_int,
                                         ctypes.c_uint64, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p,
                                         ctypes.c_void_p]),
    "lp_conv_packed_bytes": (ctypes.c_int, [ctypes.POINTER(ConvDesc), QFmt, QFmt, ctypes.POINTER(ctypes.c_size_t)]),
    "lp_conv_plan_info": (ctypes.c_int, [ctypes.POINTER(ConvDesc), QFmt, QFmt, ctypes.POINTER(PlanInfo)]),
    "lp_conv_pack_weights": (ctypes.c_int, [ctypes.POINTER(ConvDesc), QFmt, QFmt, ctypes.c_void_p, ctypes.c_void_p,
                                            ctypes.c_size_t, ctypes.c_void_p]),
    "lp_conv_pool_check": (ctypes.c_int, [ctypes.POINTER(ConvDesc), QFmt, QFmt, ctypes.c_int, QFmt, QFmt, ctypes.c_int,
                                          ctypes.c_int]),
    "lp_conv_workspace_bytes": (ctypes.c_int, [ctypes.POINTER(ConvDesc), QFmt, QFmt,
                                               ctypes.POINTER(ctypes.c_size_t)]),
    "lp_conv_fwd": (ctypes.c_int, [ctypes.POINTER(ConvDesc), ctypes.c_void_p, QFmt, ctypes.c_void_p, QFmt,
                                   ctypes.c_void_p, QFmt, ctypes.c_void_p, ctypes.c_void_p, QFmt, ctypes.c_int,
                                   ctypes.c_int, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_size_t,
                                   ctypes.c_void_p]),
    "lp_conv_fwd_zskip": (ctypes.c_int, [ctypes.POINTER(ConvDesc), ctypes.c_void_p, QFmt, ctypes.POINTER(ZeroMap),
                                         ctypes.c_void_p, QFmt, ctypes.c_void_p, QFmt, ctypes.c_void_p, QFmt, ctypes.c_int,
                                         ctypes.c_int, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p,
                                         ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p]),
    "lp_conv_fwd_static": (ctypes.c_int, [ctypes.POINTER(ConvDesc), ctypes.c_void_p, QFmt, ctypes.c_void_p, QFmt,
                                          ctypes.c_void_p, QFmt, ctypes.c_void_p, ctypes.c_void_p, QFmt, ctypes.c_int,
                                          ctypes.c_int, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p]),
    "lp_fc_packed_bytes": (ctypes.c_int, [ctypes.c_int, ctypes.c_int, ctypes.c_int, QFmt, QFmt,
                                          ctypes.POINTER(ctypes.c_size_t)]),
    "lp_fc_pack_weights": (ctypes.c_int, [ctypes.c_int, ctypes.c_int, ctypes.c_int, QFmt, QFmt, ctypes.c_void_p,
                                          ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p]),
    "lp_fc_workspace_bytes": (ctypes.c_int, [ctypes.c_int, ctypes.c_int, ctypes.c_int, QFmt, QFmt,
                                             ctypes.POINTER(ctypes.c_size_t)]),
    "lp_fc_fwd": (ctypes.c_int, [ctypes.c_int, ctypes.c_int, ctypes.c_int, ctypes.c_void_p, QFmt, ctypes.c_void_p,
                                 QFmt, ctypes.c_void_p, QFmt, ctypes.c_void_p, ctypes.c_void_p, QFmt, ctypes.c_int,
                                 ctypes.c_int, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_size_t,
                                 ctypes.c_void_p]),
    "lp_maxpool2x2": (ctypes.c_int, [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int, ctypes.c_int, ctypes.c_int,
                                     ctypes.c_int, ctypes.c_int, ctypes.c_void_p]),
    "lp_mx4_bytes": (ctypes.c_int, [ctypes.c_size_t, ctypes.c_size_t, ctypes.POINTER(ctypes.c_size_t),
                                    ctypes.POINTER(ctypes.c_size_t)]),
    "lp_ckpt8_bytes": (ctypes.c_int, [ctypes.c_size_t, ctypes.c_size_t, ctypes.POINTER(ctypes.c_size_t),
                                      ctypes.POINTER(ctypes.c_size_t)]),
    "lp_mx4_quantize": (ctypes.c_int, [ctypes.c_void_p, ctypes.c_int, ctypes.c_size_t, ctypes.c_size_t,
                                       ctypes.c_size_t, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int,
                                       ctypes.c_uint64, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p]),
    "lp_mx4_dequantize": (ctypes.c_int, [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_size_t,
                                         ctypes.c_void_p, ctypes.c_int, ctypes.c_size_t, ctypes.c_void_p]),
    "lp_mx4_fc_workspace_bytes": (ctypes.c_int, [ctypes.c_int, ctypes.c_int, ctypes.c_int,
                                                 ctypes.POINTER(ctypes.c_size_t)]),
    "lp_mx4_fc_fwd": (ctypes.c_int, [ctypes.c_int, ctypes.c_int, ctypes.c_int, ctypes.c_void_p, ctypes.c_int,
                                     ctypes.c_size_t, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p,
                                     ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int, ctypes.c_size_t, ctypes.c_int,
                                     ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p]),
    "lp_mx4_fc_dgrad_workspace_bytes": (ctypes.c_int, [ctypes.c_int, ctypes.c_int, ctypes.c_int,
                                                       ctypes.POINTER(ctypes.c_size_t)]),
    "lp_mx4_fc_dgrad": (ctypes.c_int, [ctypes.c_int, ctypes.c_int, ctypes.c_int, ctypes.c_void_p, ctypes.c_size_t,
                                       ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int,
                                       ctypes.c_size_t, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p]),
    "lp_ckpt8_save": (ctypes.c_int, [ctypes.c_void_p, ctypes.c_int, ctypes.c_size_t, ctypes.c_size_t, ctypes.c_size_t,
                                     ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int, ctypes.c_uint64, ctypes.c_int,
                                     ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p]),
    "lp_ckpt8_load": (ctypes.c_int, [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_size_t,
                                     ctypes.c_void_p, ctypes.c_int, ctypes.c_size_t, ctypes.c_void_p]),
    "lp_ckpt8_act_bwd": (ctypes.c_int, [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_size_t,
                                        ctypes.c_void_p, ctypes.c_int, ctypes.c_size_t, ctypes.c_int, ctypes.c_void_p,
                                        ctypes.c_size_t, ctypes.c_void_p]),
    "lp_ckpt8_fc_wgrad_workspace_bytes": (ctypes.c_int, [ctypes.c_int, ctypes.c_int, ctypes.c_int,
                                                         ctypes.POINTER(ctypes.c_size_t)]),
    "lp_ckpt8_fc_wgrad": (ctypes.c_int, [ctypes.c_int, ctypes.c_int, ctypes.c_int, ctypes.c_void_p, ctypes.c_size_t,
                                         ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int,
                                         ctypes.c_size_t, ctypes.c_void_p, ctypes.c_int, ctypes.c_void_p,
                                         ctypes.c_size_t, ctypes.c_void_p]),
}


def lib_path():
    return _LIB_PATH


def exported_symbols():
    return sorted(_SIGNATURES)


def load():
    """Load liblp.so (built beforehand by build.py); raises if it is not there."""
    global _lib
    if _lib is None:
        if not os.path.exists(_LIB_PATH):
            raise RuntimeError("liblp.so is not built: run `python -m paper_1711_04713_amd.build` "
                               "(there is no fallback path)")
        lib = ctypes.CDLL(_LIB_PATH)
        for name, (res, args) in _SIGNATURES.items():
            fn = getattr(lib, name)
            fn.restype = res
            fn.argtypes = args
        _lib = lib
    return _lib


def lp_status_string(status):
    return load().lp_status_string(int(status)).decode()


def _check(status, what):
    if status != 0:
        raise LpError(status, what)


def _ptr(t):
    return None if t is None else t.data_ptr()   # (c_void_p arguments take plain integers)


def _first_stream():
    import torch

    global _stream
    handle = torch.cuda.current_stream().cuda_stream   # initialises the GPU, or says why it cannot
    raw, device = getattr(torch._C, "_cuda_getCurrentRawStream", None), getattr(torch._C, "_cuda_getDevice", None)
    if raw is not None and device is not None:
        _stream = lambda: raw(device())
    return handle


# The handle of torch's current stream on the current device.  torch.cuda.current_stream() builds a Stream object for
# it on every call, 2.9 us of the 7 that an lp_quantize took to issue; from the second call on the handle is asked for directly, 0.2.
_stream = _first_stream


def _q(q):
    return q if isinstance(q, QFmt) else QFmt(*q)


def lp_range(x, n, loss_threshold=0.0, workspace=None):
    """x: float32 CUDA tensor.  Returns (QFmt, lost list with lost[m] for m=1..n)."""
    import torch

    ws = workspace if workspace is not None else torch.empty(LP_RANGE_WORKSPACE_WORDS, dtype=torch.int64, device=x.device)
    out = QFmt()
    lost = (ctypes.c_uint64 * (n + 1))()
    _check(load().lp_range(_ptr(x), x.numel(), n, loss_threshold, ctypes.byref(out), lost, _ptr(ws), _stream()),
           "lp_range")
    return out, list(lost)


def lp_range_acc(acc, f_acc, relu, n, loss_threshold=0.0, workspace=None):
    import torch

    ws = workspace if workspace is not None else torch.empty(LP_RANGE_WORKSPACE_WORDS, dtype=torch.int64, device=acc.device)
    out = QFmt()
    lost = (ctypes.c_uint64 * (n + 1))()
    _check(load().lp_range_acc(_ptr(acc), acc.numel(), f_acc, int(bool(relu)), n, loss_threshold, ctypes.byref(out),
                               lost, _ptr(ws), _stream()), "lp_range_acc")
    return out, list(lost)


def lp_quantize(x, codes, q, r=LP_ROUND_NEAREST_AWAY, seed=0, zero_count=None, sat_count=None):
    _check(load().lp_quantize(_ptr(x), _ptr(codes), x.numel(), _q(q), r, seed, _ptr(zero_count), _ptr(sat_count),
                              _stream()), "lp_quantize")


def lp_act(acc, f_acc, qy, relu, y_codes, r=LP_ROUND_NEAREST_AWAY, zero_count=None, sat_count=None):
    _check(load().lp_act(_ptr(acc), acc.numel(), f_acc, _q(qy), int(bool(relu)), r, _ptr(y_codes), _ptr(zero_count),
                         _ptr(sat_count), _stream()), "lp_act")


def lp_act_stochastic(acc, f_acc, qy, relu, seed, y_codes, zero_count=None, sat_count=None):
    _check(load().lp_act_stochastic(_ptr(acc), acc.numel(), f_acc, _q(qy), int(bool(relu)), seed, _ptr(y_codes),
                                    _ptr(zero_count), _ptr(sat_count), _stream()), "lp_act_stochastic")


def lp_conv_packed_bytes(desc, qx, qw):
    n = ctypes.c_size_t(0)
    _check(load().lp_conv_packed_bytes(ctypes.byref(desc), _q(qx), _q(qw), ctypes.byref(n)), "lp_conv_packed_bytes")
    return n.value


def lp_conv_plan_info(desc, qx, qw):
    out = PlanInfo()
    _check(load().lp_conv_plan_info(ctypes.byref(desc), _q(qx), _q(qw), ctypes.byref(out)), "lp_conv_plan_info")
    return out.asdict()


def lp_conv_pool_check(desc, qx, qw, qy, relu=True, r=LP_ROUND_NEAREST_AWAY, qb=None):
    """True if lp_conv_fwd takes this call with desc.pool = 1."""
    status = load().lp_conv_pool_check(ctypes.byref(desc), _q(qx), _q(qw), int(qb is not None),
                                       _q(qb) if qb is not None else QFmt(), _q(qy), int(bool(relu)), r)
    if status not in (0, 2):
        raise LpError(status, "lp_conv_pool_check")
    return status == 0


def lp_conv_pack_weights(desc, qx, qw, w_codes, packed):
    _check(load().lp_conv_pack_weights(ctypes.byref(desc), _q(qx), _q(qw), _ptr(w_codes), _ptr(packed),
                                       packed.numel() * packed.element_size(), _stream()), "lp_conv_pack_weights")


def lp_conv_workspace_bytes(desc, qx, qw):
    n = ctypes.c_size_t(0)
    _check(load().lp_conv_workspace_bytes(ctypes.byref(desc), _q(qx), _q(qw), ctypes.byref(n)),
           "lp_conv_workspace_bytes")
    return n.value


def lp_conv_fwd(desc, x_codes, qx, w_packed, qw, qy=None, y_codes=None, acc_out=None, relu=True,
                r=LP_ROUND_NEAREST_AWAY, bias_codes=None, qb=None, zero_count=None, workspace=None, sat_count=None):
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(load().lp_conv_fwd(ctypes.byref(desc), _ptr(x_codes), _q(qx), _ptr(w_packed), _q(qw), _ptr(bias_codes),
                              _q(qb) if qb is not None else QFmt(), _ptr(acc_out), _ptr(y_codes),
                              _q(qy) if qy is not None else QFmt(), int(bool(relu)), r, _ptr(zero_count),
                              _ptr(sat_count), _ptr(workspace), ws_bytes, _stream()), "lp_conv_fwd")


def zero_map(flags, producer_info, Wo, scale=1):
    """lp_zero_map for a tensor whose producer (plan info producer_info, output width Wo) wrote `flags`;
    scale = 2 when the tensor was 2x2-pooled after the flags were taken."""
    return ZeroMap(flags.data_ptr(), producer_info["tile_rows"], producer_info["tile_cols"],
                   (Wo + producer_info["tile_cols"] - 1) // producer_info["tile_cols"], producer_info["tiles_n"],
                   producer_info["bn"], scale)


def lp_conv_fwd_zskip(desc, x_codes, qx, x_map, w_packed, qw, qy, y_codes, relu=True, r=LP_ROUND_NEAREST_AWAY,
                      bias_codes=None, qb=None, zero_count=None, sat_count=None, y_flags=None, skipped=None,
                      workspace=None):
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(load().lp_conv_fwd_zskip(ctypes.byref(desc), _ptr(x_codes), _q(qx), ctypes.byref(x_map) if x_map is not None else None,
                                    _ptr(w_packed), _q(qw), _ptr(bias_codes), _q(qb) if qb is not None else QFmt(),
                                    _ptr(y_codes), _q(qy), int(bool(relu)), r, _ptr(zero_count), _ptr(sat_count),
                                    _ptr(y_flags), _ptr(skipped), _ptr(workspace), ws_bytes, _stream()),
           "lp_conv_fwd_zskip")


LP_STATIC_WORKSPACE_BYTES = 64 << 20


def lp_conv_fwd_static(desc, x_codes, qx, w_packed, qw, qy=None, y_codes=None, acc_out=None, relu=True,
                       r=LP_ROUND_NEAREST_AWAY, bias_codes=None, qb=None, zero_count=None, sat_count=None):
    _check(load().lp_conv_fwd_static(ctypes.byref(desc), _ptr(x_codes), _q(qx), _ptr(w_packed), _q(qw),
                                     _ptr(bias_codes), _q(qb) if qb is not None else QFmt(), _ptr(acc_out),
                                     _ptr(y_codes), _q(qy) if qy is not None else QFmt(), int(bool(relu)), r,
                                     _ptr(zero_count), _ptr(sat_count), _stream()), "lp_conv_fwd_static")


def lp_fc_packed_bytes(M, K, Nout, qx, qw):
    n = ctypes.c_size_t(0)
    _check(load().lp_fc_packed_bytes(M, K, Nout, _q(qx), _q(qw), ctypes.byref(n)), "lp_fc_packed_bytes")
    return n.value


def lp_fc_pack_weights(M, K, Nout, qx, qw, w_codes, packed):
    _check(load().lp_fc_pack_weights(M, K, Nout, _q(qx), _q(qw), _ptr(w_codes), _ptr(packed),
                                     packed.numel() * packed.element_size(), _stream()), "lp_fc_pack_weights")


def lp_fc_workspace_bytes(M, K, Nout, qx, qw):
    n = ctypes.c_size_t(0)
    _check(load().lp_fc_workspace_bytes(M, K, Nout, _q(qx), _q(qw), ctypes.byref(n)), "lp_fc_workspace_bytes")
    return n.value


def lp_fc_fwd(M, K, Nout, x_codes, qx, w_packed, qw, qy=None, y_codes=None, acc_out=None, relu=True,
              r=LP_ROUND_NEAREST_AWAY, bias_codes=None, qb=None, zero_count=None, workspace=None, sat_count=None):
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(load().lp_fc_fwd(M, K, Nout, _ptr(x_codes), _q(qx), _ptr(w_packed), _q(qw), _ptr(bias_codes),
                            _q(qb) if qb is not None else QFmt(), _ptr(acc_out), _ptr(y_codes),
                            _q(qy) if qy is not None else QFmt(), int(bool(relu)), r, _ptr(zero_count),
                            _ptr(sat_count), _ptr(workspace), ws_bytes, _stream()), "lp_fc_fwd")


def lp_maxpool2x2(x_codes, y_codes, N, H, W, C, n_bits):
    _check(load().lp_maxpool2x2(_ptr(x_codes), _ptr(y_codes), N, H, W, C, n_bits, _stream()), "lp_maxpool2x2")


# ------------------------------------------------------------- microscaled formats (float tensors: 2-d, unit column stride)

_dtypes = {}


def _first_device():
    import torch

    global _device
    _dtypes.update({torch.float32: LP_F32, torch.bfloat16: LP_BF16, torch.float16: LP_F16})
    if not torch.cuda.is_available():
        return None                            # no tensor is there
    device = torch.cuda.current_device()      # initialises the GPU
    _device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
    return device


_device = _first_device


def _dtype(t):
    """lp_dtype of a tensor; -1, which every call refuses, where there is none."""
    return _dtypes.get(t.dtype, -1)


def _refuse(what, why):
    raise ValueError("%s: %s" % (what, why))


# What the C entry points cannot see for themselves: where the tensors are, their own sizes and strides.

# Tensors have to be on the current GPU, whose stream the call goes to.

def _counter(t, device, what, name):
    """Address of an integer of 64 bits, the tensor's first (None: a null pointer)."""
    if t is None:
        return None
    if t.element_size() != 8 or t.is_floating_point() or t.is_complex() or not t.numel():
        _refuse(what, "%s is not an integer of 64 bits" % name)
    if t.get_device() != device:
        _refuse(what, "%s is not on the current GPU" % name)
    return t.data_ptr()


def _rows(t, rows, cols, device, what, name):
    """Address and row stride of a float tensor [rows][cols]."""
    if t.shape == (rows, cols) and t.get_device() == device:
        ld, step = t.stride()
        if step == 1 or cols <= 1:
            return t.data_ptr(), ld if rows > 1 else cols or 1
    elif t.shape == (rows, cols):
        _refuse(what, "%s is not on the current GPU" % name)
    _refuse(what, "%s is not a [%d][%d] tensor with unit column stride" % (name, rows, cols))


def _dense(t, nbytes, device, what, name):
    """Address of nbytes of dense memory."""
    if t.nbytes != nbytes or not t.is_contiguous():
        _refuse(what, "%s does not hold %d dense bytes" % (name, nbytes))
    if t.get_device() != device:
        _refuse(what, "%s is not on the current GPU" % name)
    return t.data_ptr()


def _blocks(codes, scales, blocks, size, device, what, name):
    """Addresses of a microscaled tensor's codes and scales."""
    if (codes.nbytes == size * blocks and scales.nbytes == blocks and codes.is_contiguous() and scales.is_contiguous()
            and codes.get_device() == device == scales.get_device()):
        return codes.data_ptr(), scales.data_ptr()
    return _dense(codes, size * blocks, device, what, name + "'s codes"), _dense(scales, blocks, device, what, name + "'s scales")


def _mx4(codes, scales, rows, cols, device, what, name):
    return _blocks(codes, scales, rows * ((cols + 255) // 256 * 8), 16, device, what, name)


def _ckpt8(codes, scales, rows, cols, device, what, name):
    return _blocks(codes, scales, rows * ((cols + 31) // 32), 32, device, what, name)


def _vector(t, n, device, what, name):
    """Address of n dense float32 (None: a null pointer)."""
    if t is None:
        return None
    if _dtype(t) != LP_F32:
        _refuse(what, "%s is not float32" % name)
    return _dense(t, 4 * n, device, what, name)


def _workspace(t, device, what):
    """Address and bytes of a workspace."""
    return (None, 0) if t is None else (_dense(t, t.nbytes, device, what, "workspace"), t.nbytes)


def _bf16(t, what, name):
    if _dtype(t) != LP_BF16:
        _refuse(what, "%s is not bfloat16" % name)


# Sizes as the C calls take them.  One that their type does not hold becomes its largest number, which every call refuses: ctypes
# would cut it off.

def _ints(*sizes):
    return tuple(min(max(n, -1), 0x7fffffff) for n in sizes)


def _size(n):
    return n if 0 <= n < 1 << 64 else (1 << 64) - 1


def _two_sizes(what, rows, cols):
    a, b = ctypes.c_size_t(0), ctypes.c_size_t(0)
    _check(getattr(load(), what)(_size(rows), _size(cols), ctypes.byref(a), ctypes.byref(b)), what)
    return a.value, b.value


def _fc_workspace_bytes(what, M, K, Nout):
    n = ctypes.c_size_t(0)
    if (M | K | Nout) >> 31:
        M, K, Nout = _ints(M, K, Nout)
    _check(getattr(load(), what)(M, K, Nout, ctypes.byref(n)), what)
    return n.value


def lp_mx4_bytes(rows, cols):
    """(codes, scales) bytes of an mx4 tensor."""
    return _two_sizes("lp_mx4_bytes", rows, cols)


def lp_ckpt8_bytes(rows, cols):
    """(codes, scales) bytes of a ckpt8 tensor."""
    return _two_sizes("lp_ckpt8_bytes", rows, cols)


def lp_mx4_quantize(x, codes, scales, r=LP_ROUND_NEAREST_EVEN, seed=0, zero_count=None, sat_count=None):
    """x: [rows][cols] float32, bfloat16 or float16."""
    what, device = "lp_mx4_quantize", _device()
    rows, cols = x.shape
    px, ldx = _rows(x, rows, cols, device, what, "x")
    pc, ps = _mx4(codes, scales, rows, cols, device, what, "x")
    pz, psat = _counter(zero_count, device, what, "zero_count"), _counter(sat_count, device, what, "sat_count")
    _check(load().lp_mx4_quantize(px, _dtype(x), rows, cols, ldx, pc, ps, r, seed, pz, psat, _stream()), what)


def lp_mx4_dequantize(codes, scales, y):
    what, device = "lp_mx4_dequantize", _device()
    rows, cols = y.shape
    py, ldy = _rows(y, rows, cols, device, what, "y")
    pc, ps = _mx4(codes, scales, rows, cols, device, what, "y")
    _check(load().lp_mx4_dequantize(pc, ps, rows, cols, py, _dtype(y), ldy, _stream()), what)


def lp_mx4_fc_workspace_bytes(M, K, Nout):
    return _fc_workspace_bytes("lp_mx4_fc_workspace_bytes", M, K, Nout)


def lp_mx4_fc_fwd(M, K, Nout, x, w_codes, w_scales, y, x_scales=None, bias=None, act=LP_ACT_NONE, workspace=None):
    """x: floats [M][K], or the codes of an mx4 tensor whose scales are x_scales.  bias: float32 [Nout]."""
    what, device = "lp_mx4_fc_fwd", _device()
    if x_scales is None:
        (px, ldx), pxs, xt = _rows(x, M, K, device, what, "x"), None, _dtype(x)
    else:
        (px, pxs), ldx, xt = _mx4(x, x_scales, M, K, device, what, "x"), 0, LP_F32
    py, ldy = _rows(y, M, Nout, device, what, "y")
    pc, ps = _mx4(w_codes, w_scales, Nout, K, device, what, "w")
    pb = _vector(bias, Nout, device, what, "bias")
    pw, nw = _workspace(workspace, device, what)
    if (M | K | Nout) >> 31:
        M, K, Nout = _ints(M, K, Nout)
    _check(load().lp_mx4_fc_fwd(M, K, Nout, px, xt, ldx, pxs, pc, ps, pb, py, _dtype(y), ldy, act, pw, nw, _stream()), what)


def lp_mx4_fc_dgrad_workspace_bytes(M, K, Nout):
    return _fc_workspace_bytes("lp_mx4_fc_dgrad_workspace_bytes", M, K, Nout)


def lp_mx4_fc_dgrad(M, K, Nout, dy, w_codes, w_scales, dx, workspace=None):
    """dy: bfloat16 [M][Nout]; dx: bfloat16 or float32 [M][K]."""
    what, device = "lp_mx4_fc_dgrad", _device()
    _bf16(dy, what, "dy")
    pdy, lddy = _rows(dy, M, Nout, device, what, "dy")
    pdx, lddx = _rows(dx, M, K, device, what, "dx")
    pc, ps = _mx4(w_codes, w_scales, Nout, K, device, what, "w")
    pw, nw = _workspace(workspace, device, what)
    if (M | K | Nout) >> 31:
        M, K, Nout = _ints(M, K, Nout)
    _check(load().lp_mx4_fc_dgrad(M, K, Nout, pdy, lddy, pc, ps, pdx, _dtype(dx), lddx, pw, nw, _stream()), what)


def lp_ckpt8_save(x, codes, scales, act=LP_ACT_NONE, y=None, r=LP_ROUND_NEAREST_EVEN, seed=0):
    """Keeps x in codes and scales; y (nullable, of x's type; may be x) receives act(x)."""
    what, device = "lp_ckpt8_save", _device()
    rows, cols = x.shape
    px, ldx = _rows(x, rows, cols, device, what, "x")
    py, ldy = None, 0
    if y is not None:
        if y.dtype != x.dtype:
            _refuse(what, "y is not of x's type")
        py, ldy = _rows(y, rows, cols, device, what, "y")
    pc, ps = _ckpt8(codes, scales, rows, cols, device, what, "x")
    _check(load().lp_ckpt8_save(px, _dtype(x), rows, cols, ldx, pc, ps, r, seed, act, py, ldy, _stream()), what)


def lp_ckpt8_load(codes, scales, y):
    what, device = "lp_ckpt8_load", _device()
    rows, cols = y.shape
    py, ldy = _rows(y, rows, cols, device, what, "y")
    pc, ps = _ckpt8(codes, scales, rows, cols, device, what, "y")
    _check(load().lp_ckpt8_load(pc, ps, rows, cols, py, _dtype(y), ldy, _stream()), what)


def lp_ckpt8_act_bwd(codes, scales, dy, dx, act):
    """dx = dy * act'(kept value); dx may be dy."""
    what, device = "lp_ckpt8_act_bwd", _device()
    rows, cols = dy.shape
    if dx.dtype != dy.dtype:
        _refuse(what, "dx is not of dy's type")
    pdy, lddy = _rows(dy, rows, cols, device, what, "dy")
    pdx, lddx = _rows(dx, rows, cols, device, what, "dx")
    pc, ps = _ckpt8(codes, scales, rows, cols, device, what, "dy")
    _check(load().lp_ckpt8_act_bwd(pc, ps, rows, cols, pdy, _dtype(dy), lddy, act, pdx, lddx, _stream()), what)


def lp_ckpt8_fc_wgrad_workspace_bytes(M, K, Nout):
    return _fc_workspace_bytes("lp_ckpt8_fc_wgrad_workspace_bytes", M, K, Nout)


def lp_ckpt8_fc_wgrad(M, K, Nout, dy, x_codes, x_scales, dw, dbias=None, accumulate=False, workspace=None):
    """dy: bfloat16 [M][Nout]; dw: bfloat16 or float32 [Nout][K]; dbias: float32 [Nout]."""
    what, device = "lp_ckpt8_fc_wgrad", _device()
    _bf16(dy, what, "dy")
    pdy, lddy = _rows(dy, M, Nout, device, what, "dy")
    pdw, lddw = _rows(dw, Nout, K, device, what, "dw")
    pc, ps = _ckpt8(x_codes, x_scales, M, K, device, what, "x")
    pb = _vector(dbias, Nout, device, what, "dbias")
    pw, nw = _workspace(workspace, device, what)
    if (M | K | Nout) >> 31:
        M, K, Nout = _ints(M, K, Nout)
    _check(load().lp_ckpt8_fc_wgrad(M, K, Nout, pdy, lddy, pc, ps, pdw, _dtype(dw), lddw, pb, int(bool(accumulate)), pw, nw, _stream()), what)
