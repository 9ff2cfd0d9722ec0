"""ctypes binding of libftpipe.so: argument marshalling only, one function per C entry point,
same names.  Device buffers are torch tensors (torch provides device memory and streams);
every step of the path runs inside the library's kernels.

There is no fallback: importing this module without the built library raises.
"""
import ctypes as C
import os

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.environ.get("FTPIPE_LIB") or os.path.join(_HERE, "libftpipe.so")       # FTPIPE_LIB: another build of the library (measurement variants)
if not os.path.exists(LIB_PATH):
    raise ImportError(f"{LIB_PATH} is missing: build it with `python -m paper_2110_02781_b200.build`")
lib = C.CDLL(LIB_PATH)

OK = 0
STATUS = {0: "FTP_OK", 1: "FTP_EINVAL", 2: "FTP_ERANGE", 3: "FTP_ENOMEM", 4: "FTP_ECUDA", 5: "FTP_ESTATE",
          6: "FTP_ETIMEOUT", 7: "FTP_EUNSUPPORTED"}
T_WEIGHTS, T_GRADS, T_MOMENTUM, T_STATE = 0, 1, 2, 3
FP32, BF16 = 0, 1
ACT_NONE, ACT_RELU, ACT_RELU6, ACT_GELU, ACT_SILU = 0, 1, 2, 3, 4
STASH_NONE, STASH_FULL, STASH_8BIT = 0, 1, 2
NORM_NONE, NORM_RMS, NORM_LAYER = 0, 1, 2


class LayerDesc(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("unit", "kind", "cin", "cout", "k", "stride", "pad", "act", "has_bias",
                                          "residual_src")]


class ModelCfg(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("batch", "in_c", "in_h", "in_w", "n_classes", "precision", "max_stages")] + \
               [(n, C.c_float) for n in ("lr", "momentum", "weight_decay", "bn_eps", "bn_momentum")]


class TraceRec(C.Structure):
    _fields_ = [("kernel", C.c_int32), ("unit", C.c_int32), ("op", C.c_int32), ("backward", C.c_int32),
                ("ms", C.c_float), ("bytes", C.c_double), ("flops", C.c_double)]


class TrainState(C.Structure):
    _fields_ = [("committed_forward_id", C.c_int64), ("committed_backward_id", C.c_int64), ("status", C.c_int32),
                ("learning_rate", C.c_float), ("epoch_number", C.c_int64), ("batch_number", C.c_int64)]


class FfnDesc(C.Structure):
    _fields_ = [("rows", C.c_int64)] + [(n, C.c_int32) for n in ("cin", "cout", "precision", "act", "stash", "x_8bit", "dw_f32",
                                                                 "unaligned")] + \
               [(n, C.c_int64) for n in ("ldx", "ldw", "ldy", "ldr", "lddx", "lddw")]


class JoinDesc(C.Structure):
    _fields_ = [("rows", C.c_int64)] + [(n, C.c_int32) for n in ("cols", "precision", "post", "pre")] + \
               [(n, C.c_float) for n in ("eps", "alpha", "beta")] + [("site", C.c_int32), ("dropout", C.c_double)] + \
               [(n, C.c_int64) for n in ("row0", "gate_rows", "ldu", "ldx", "lds", "ldy", "ldg", "lddu", "ldds", "lddx", "lddg")]


class RecurrenceDesc(C.Structure):
    _fields_ = [(n, C.c_int64) for n in ("seqs", "len", "rows")] + [(n, C.c_int32) for n in ("cols", "precision", "act", "coupled")] + \
               [(n, C.c_int64) for n in ("ldf", "ldv", "ldo", "ldy", "lddf", "lddv", "lddo")]


PROBE_NORMAL, PROBE_RESTARTED, PROBE_SILENT = 0, 1, 2
ACTION_RESTART_BATCH, ACTION_RESEND_STATE, ACTION_REDISTRIBUTE = 0, 1, 2


class FtpError(RuntimeError):
    def __init__(self, status, text):
        super().__init__(f"{STATUS.get(status, status)}: {text}")
        self.status = status


_vp, _i32, _i64, _sz, _f32 = C.c_void_p, C.c_int32, C.c_int64, C.c_size_t, C.c_float
_P = C.POINTER
_SIGS = {
    "ftp_workspace_bytes": [_P(LayerDesc), _i32, _P(ModelCfg), _P(_sz), _P(_sz)],
    "ftp_build_model": [_P(LayerDesc), _i32, _P(ModelCfg), _vp, _sz, _vp, _sz, _P(_vp)],
    "ftp_num_units": [_vp, _P(_i32)],
    "ftp_unit_param_span": [_vp, _i32, _P(_i64), _P(_i64)],
    "ftp_unit_state_span": [_vp, _i32, _P(_i64), _P(_i64)],
    "ftp_unit_output_shape": [_vp, _i32, _P(_i32), _P(_i64)],
    "ftp_set_tensor": [_vp, _i32, _i32, _vp, _i64, _i32, _vp],
    "ftp_get_tensor": [_vp, _i32, _i32, _vp, _i64, _i32, _vp],
    "ftp_run_stage_forward": [_vp, _i32, _i32, _vp, _vp, _vp, _vp, _vp],
    "ftp_run_stage_backward": [_vp, _i32, _i32, _vp, _vp, _vp],
    "ftp_get_logits": [_vp, _vp, _i32, _vp],
    "ftp_sgd_step": [_vp, _i32, _i32, _f32, _vp, _vp, _vp],
    "ftp_train_step": [_vp, _vp, _vp, _i32, _f32, _P(_f32), _vp],
    "ftp_profile_layers": [_vp, _i32, _vp, _vp, _P(C.c_double), _P(C.c_double), _P(_i64), _vp],
    "ftp_estimate_capacity": [_P(C.c_double), _i32, _P(_i32), _i32, _P(C.c_double), _P(C.c_double)],
    "ftp_choose_partition": [_P(C.c_double), _i32, _P(C.c_double), _i32, _P(C.c_double), _P(C.c_double), _P(_i32),
                             _P(C.c_double)],
    "ftp_redistribution_plan": [_P(_i32), _i32, _P(_i32), _i32, _i32, _i32, _i32, _P(_i32), _P(_i32)],
    "ftp_stage_timing_enable": [_vp, _i32],
    "ftp_stage_times": [_vp, _P(C.c_double), _P(_i32)],
    "ftp_recovery_plan": [_P(_i32), _i32, _P(_i32), _i32, _P(_i32), _i32, _P(_i32), _P(_i32)],
    "ftp_recover": [_vp, _vp, _i32, _vp, _sz, _P(_i32), _i32, _P(_i32), _vp],
    "ftp_set_partition": [_vp, _P(_i32), _i32, _P(_i32), _vp],
    "ftp_get_partition": [_vp, _P(_i32), _P(_i32)],
    "ftp_snapshot_weights": [_vp, _i32, _vp, _sz, _i32, _P(_sz), _vp],
    "ftp_state_init": [_P(TrainState), _f32, _i64, _i64],
    "ftp_state_forward_done": [_P(TrainState), _i64],
    "ftp_state_backward_done": [_P(TrainState), _i64],
    "ftp_state_timer_expired": [_P(TrainState), _i64, _P(_i32)],
    "ftp_state_may_forward": [_P(TrainState), _i64, _P(_i32)],
    "ftp_state_reset": [_P(TrainState), _i64, _P(_i64)],
    "ftp_classify_probe": [_P(_i32), _i32, _P(_i32), _P(_i32), _P(_i32), _P(_i32)],
    "ftp_async_stage_order": [_i32, _i32, _i32, _P(_i32), _P(_i32)],
    "ftp_async_version_trace": [_i32, _i32, _i32, _i32, _P(_i64), _P(_i64), _P(_i32)],
    "ftp_sync_units": [_vp, _vp, _i32, _i32, _i32, _vp],
    "ftp_sgd_step_from": [_vp, _vp, _i32, _i32, _f32, _vp],
    "ftp_aggregate_weights": [_vp, _P(_vp), _i32, _i32, _i32, _vp],
    "ftp_measure_bandwidth": [_vp, _vp, _sz, _i32, _P(C.c_double), _P(C.c_double), _vp],
    "ftp_check_guards": [_vp, _P(_i32), _P(_i64), _vp],
    "ftp_check_device_status": [_vp, _vp],
    "ftp_debug_set_device_status": [_vp, _i32, _vp],
    "ftp_trace_enable": [_vp, _i32],
    "ftp_trace_read": [_vp, _P(TraceRec), _i32, _P(_i32)],
    "ftp_launch_count": [_vp, _P(_i64)],
    "ftp_linear_workspace_bytes": [_P(FfnDesc), _i32, _P(_sz)],
    "ftp_gated_workspace_bytes": [_P(FfnDesc), _i32, _P(_sz)],
    "ftp_linear_forward": [_P(FfnDesc), _vp, _vp, _vp, _vp, _vp, _vp, _vp, _sz, _vp],
    "ftp_linear_backward": [_P(FfnDesc), _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _sz, _vp],
    "ftp_gated_forward": [_P(FfnDesc), _vp, _vp, _vp, _vp, _vp, _vp, _sz, _vp],
    "ftp_gated_backward": [_P(FfnDesc), _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _sz, _vp],
    "ftp_checkpoint_bytes": [_i64, _i32, _i32, _P(_sz)],
    "ftp_checkpoint_pack": [_vp, _i64, _i32, _i64, _i32, _vp, _i32, _vp],
    "ftp_checkpoint_unpack": [_vp, _i32, _i64, _i32, _i32, _vp, _i64, _vp],
    "ftp_check_op_status": [_vp],
    "ftp_dropout": [_vp, _vp, _i64, _i32, _i64, _i64, _i32, C.c_double, _vp, _i32, _i64, _vp],
    "ftp_join_workspace_bytes": [_P(JoinDesc), _P(_sz)],
    "ftp_join_forward": [_P(JoinDesc)] + [_vp] * 12,
    "ftp_join_backward": [_P(JoinDesc)] + [_vp] * 18 + [_sz, _vp],
    "ftp_recurrence_states": [_P(RecurrenceDesc), _P(_i64)],
    "ftp_recurrence_forward": [_P(RecurrenceDesc)] + [_vp] * 9,
    "ftp_recurrence_backward": [_P(RecurrenceDesc)] + [_vp] * 12,
    "ftp_logprob_forward": [_vp, _i64, _i32, _i64, _i32, _f32] + [_vp] * 6 + [_i32, _vp],
    "ftp_logprob_backward": [_vp, _i64, _i32, _i64, _i32, _f32] + [_vp] * 6 + [_i64, _vp],
    "ftp_conv_wgrad_static": [_vp, _vp, _vp, _i32, _i32, _i32, _i32, _i32, _i32, _i32, _i32, _vp],
}
for _name, _args in _SIGS.items():
    _f = getattr(lib, _name)
    _f.argtypes, _f.restype = _args, C.c_int
lib.ftp_destroy_model.argtypes, lib.ftp_destroy_model.restype = [_vp], None
lib.ftp_last_error.argtypes, lib.ftp_last_error.restype = [], C.c_char_p
lib.ftp_kernel_name.argtypes, lib.ftp_kernel_name.restype = [_i32], C.c_char_p
lib.ftp_is_repartition_iter.argtypes, lib.ftp_is_repartition_iter.restype = [_i64, _i64, _i64], _i32
lib.ftp_is_replication_iter.argtypes, lib.ftp_is_replication_iter.restype = [_i64, _i64], _i32


def _check(status):
    if status != OK:
        raise FtpError(status, lib.ftp_last_error().decode())


def _ptr(t):
    """Address of a torch tensor / numpy array / raw int, or NULL."""
    if t is None:
        return None
    if isinstance(t, int):
        return t
    if isinstance(t, np.ndarray):
        return t.ctypes.data
    return t.data_ptr()


def _stream(stream):
    if stream is None:
        import torch
        return torch.cuda.current_stream().cuda_stream
    return stream if isinstance(stream, int) else stream.cuda_stream


def _dbl(a):
    a = np.ascontiguousarray(a, dtype=np.float64)
    return a, a.ctypes.data_as(_P(C.c_double))


def _i32arr(a):
    a = np.ascontiguousarray(a, dtype=np.int32)
    return a, a.ctypes.data_as(_P(_i32))


def layer_array(layers):
    arr = (LayerDesc * len(layers))()
    for i, l in enumerate(layers):
        arr[i] = LayerDesc(*[int(v) for v in l])
    return arr


def model_cfg(cfg):
    return ModelCfg(cfg["batch"], cfg["in_c"], cfg["in_h"], cfg["in_w"], cfg["n_classes"], cfg["precision"],
                    cfg["max_stages"], cfg["lr"], cfg["momentum"], cfg["weight_decay"], cfg["bn_eps"], cfg["bn_momentum"])


# ---- pure host functions (usable without a GPU) ------------------------------------------------
def ftp_estimate_capacity(layer_times, points, stage_times):
    lt, plt = _dbl(layer_times)
    pts, ppts = _i32arr(points)
    stt, pst = _dbl(stage_times)
    out = np.zeros(len(pts) - 1, np.float64)
    _check(lib.ftp_estimate_capacity(plt, len(lt), ppts, len(pts) - 1, pst, out.ctypes.data_as(_P(C.c_double))))
    return out.tolist()


def ftp_choose_partition(layer_times, capacities, out_bytes=None, bandwidth=None):
    lt, plt = _dbl(layer_times)
    cp, pcp = _dbl(capacities)
    ob = bw = pob = pbw = None
    if out_bytes is not None:
        ob, pob = _dbl(out_bytes)
    if bandwidth is not None:
        bw, pbw = _dbl(bandwidth)
    pts = np.zeros(len(cp) + 1, np.int32)
    bott = C.c_double()
    _check(lib.ftp_choose_partition(plt, len(lt), pcp, len(cp), pob, pbw, pts.ctypes.data_as(_P(_i32)), C.byref(bott)))
    return pts.tolist(), bott.value


def ftp_redistribution_plan(p_new, p_cur, i_cur, i_new, i_fail=-1):
    pn, ppn = _i32arr(p_new)
    pc, ppc = _i32arr(p_cur)
    if not (0 <= i_new < len(pn) - 1):
        raise FtpError(2, "i_new out of range")
    owners = np.full(max(int(pn[i_new + 1] - pn[i_new]), 1), -7, np.int32)
    nloc = _i32()
    _check(lib.ftp_redistribution_plan(ppn, len(pn) - 1, ppc, len(pc) - 1, i_fail, i_cur, i_new,
                                       owners.ctypes.data_as(_P(_i32)), C.byref(nloc)))
    return owners[:int(pn[i_new + 1] - pn[i_new])].tolist(), nloc.value


SRC_LOCAL, SRC_STAGE, SRC_REPLICA, SRC_CENTRAL = 0, 1, 2, 3


class FailedStage(C.Structure):
    _fields_ = [("stage", _i32), ("replica_is_host", _i32), ("replica", _vp), ("replica_bytes", _sz)]


def ftp_recovery_plan(p_cur, failed, p_new):
    """Per unit: (kind, index) as ftp_recovery_plan in include/ftpipe.h defines them."""
    pc, ppc = _i32arr(p_cur)
    pn, ppn = _i32arr(p_new)
    fl, pfl = _i32arr(failed)
    L = int(pc[-1])
    kind, index = np.full(max(L, 1), -7, np.int32), np.full(max(L, 1), -7, np.int32)
    _check(lib.ftp_recovery_plan(ppc, len(pc) - 1, pfl, len(fl), ppn, len(pn) - 1, kind.ctypes.data_as(_P(_i32)),
                                 index.ctypes.data_as(_P(_i32))))
    return kind[:L].tolist(), index[:L].tolist()


def ftp_state_init(learning_rate, epoch_number, batch_number):
    st = TrainState()
    _check(lib.ftp_state_init(C.byref(st), learning_rate, epoch_number, batch_number))
    return st


def ftp_state_forward_done(st, batch_id):
    _check(lib.ftp_state_forward_done(C.byref(st), batch_id))


def ftp_state_backward_done(st, batch_id):
    _check(lib.ftp_state_backward_done(C.byref(st), batch_id))


def ftp_state_timer_expired(st, batch_id):
    t = _i32()
    _check(lib.ftp_state_timer_expired(C.byref(st), batch_id, C.byref(t)))
    return bool(t.value)


def ftp_state_may_forward(st, batch_id):
    a = _i32()
    _check(lib.ftp_state_may_forward(C.byref(st), batch_id, C.byref(a)))
    return bool(a.value)


def ftp_state_reset(st, batch_id):
    r = _i64()
    _check(lib.ftp_state_reset(C.byref(st), batch_id, C.byref(r)))
    return r.value


def ftp_classify_probe(responses):
    n = len(responses)
    r = (_i32 * n)(*responses)
    failed = (_i32 * n)()
    action, nf, rw = _i32(), _i32(), _i32()
    _check(lib.ftp_classify_probe(r, n, C.byref(action), failed, C.byref(nf), C.byref(rw)))
    return action.value, list(failed[:nf.value]), (rw.value if rw.value >= 0 else None)


def ftp_is_repartition_iter(it, first=10, period=100):
    return bool(lib.ftp_is_repartition_iter(it, first, period))


def ftp_is_replication_iter(it, period):
    return bool(lib.ftp_is_replication_iter(it, period))


SYNC_WEIGHTS, SYNC_MOMENTUM, SYNC_STATE = 1, 2, 4


def ftp_async_stage_order(n_stages, stage, n_batches):
    isb, bat = (_i32 * (2 * n_batches + 1))(), (_i32 * (2 * n_batches + 1))()
    _check(lib.ftp_async_stage_order(n_stages, stage, n_batches, isb, bat))
    return [("B" if isb[e] else "F", bat[e]) for e in range(2 * n_batches)]


def ftp_async_version_trace(n_stages, stage, n_batches, k=1):
    fv, av, ag = (_i64 * max(n_batches, 1))(), (_i64 * max(n_batches, 1))(), (_i32 * max(n_batches, 1))()
    _check(lib.ftp_async_version_trace(n_stages, stage, n_batches, k, fv, av, ag))
    return list(fv[:n_batches]), list(av[:n_batches]), [b for b in range(n_batches) if ag[b]]


def ftp_sync_units(dst, src, a, b, what, stream=None):
    _check(lib.ftp_sync_units(dst.h, src.h, a, b, what, _stream(stream)))


def ftp_sgd_step_from(dst, grads, a, b, lr, stream=None):
    _check(lib.ftp_sgd_step_from(dst.h, grads.h, a, b, lr, _stream(stream)))


def ftp_aggregate_weights(dst, srcs, a, b, stream=None):
    arr = (_vp * len(srcs))(*[m.h for m in srcs])
    _check(lib.ftp_aggregate_weights(dst.h, arr, len(srcs), a, b, _stream(stream)))


def ftp_workspace_bytes(layers, cfg):
    d, p = _sz(), _sz()
    _check(lib.ftp_workspace_bytes(layer_array(layers), len(layers), C.byref(model_cfg(cfg)), C.byref(d), C.byref(p)))
    return d.value, p.value


def ftp_conv_wgrad_static(x, dy, dw, k, stride, pad, stream=None):
    """Weight gradient of a dense k x k convolution without any workspace argument, for callers that
    may not allocate device memory: x (n, h, w, cin), dy (n, ho, wo, cout) and dw (k, k, cin, cout)
    are float32 CUDA tensors the caller already owns.  See include/ftpipe.h for the limits."""
    import torch
    def bad(why):
        raise FtpError(1, "conv_wgrad_static: " + why)
    for name, t in (("x", x), ("dy", dy), ("dw", dw)):
        if not (isinstance(t, torch.Tensor) and t.is_cuda and t.dtype == torch.float32 and t.is_contiguous()):
            bad(f"{name} must be a contiguous float32 CUDA tensor")
        if t.device != x.device:
            bad("x, dy and dw must live on one device")
    if x.device.index != torch.cuda.current_device():
        bad("the tensors' device must be the current device")
    if x.dim() != 4 or dy.dim() != 4 or k < 1 or stride < 1 or pad < 0:
        bad("x and dy must be 4-D (n, h, w, c); k, stride >= 1, pad >= 0")
    n, h, w, cin = x.shape
    if h + 2 * pad < k or w + 2 * pad < k:
        bad("kernel larger than the padded input")
    ho, wo = (h + 2 * pad - k) // stride + 1, (w + 2 * pad - k) // stride + 1
    if tuple(dy.shape[:3]) != (n, ho, wo):
        bad(f"dy must be ({n}, {ho}, {wo}, cout), got {tuple(dy.shape)}")
    if tuple(dw.shape) != (k, k, cin, dy.shape[3]):
        bad(f"dw must be ({k}, {k}, {cin}, {dy.shape[3]}), got {tuple(dw.shape)}")
    _check(lib.ftp_conv_wgrad_static(_ptr(x), _ptr(dy), _ptr(dw), n, h, w, cin, dy.shape[3], k, stride, pad,
                                     _stream(stream)))


# ---- feed-forward operators ----------------------------------------------------------------------
# Tensors are CUDA tensors of the current device: tokens x channels (leading dimensions are flattened), rows without gaps
# inside, the same gap between all rows.  An 8-bit image is a contiguous uint8 tensor of ftp_checkpoint_bytes bytes.
# `ws`: a uint8 tensor used as the workspace; without one the binding takes it from torch's allocator, on the stream of
# the call.
def _bad(who, why):
    raise FtpError(1, f"{who}: {why}")


torch = _device = _raw_current = None


def _load_torch():
    """torch is loaded with the first operator call."""
    global torch, _device, _raw_current
    import torch as module
    module.cuda.init()
    torch, _device, _raw_current = module, module._C._cuda_getDevice, module._C._cuda_getCurrentRawStream


def _current():
    """Index of the current CUDA device."""
    if torch is None:
        _load_torch()
    return _device()


def _raw_stream(stream, cur):
    if stream is None:
        return _raw_current(cur)
    return stream if isinstance(stream, int) else stream.cuda_stream


def _rows(who, name, t, cols, dtype, cur):
    """(rows, elements between rows) of t seen as rows x cols; checks type, device and layout."""
    if t.dtype is not dtype:
        _bad(who, f"{name} must be {dtype}, got {t.dtype}")
    if t.get_device() != cur:
        _bad(who, f"{name} must live on the current CUDA device")
    if t.dim() == 2:
        rows, c = t.shape
        s0, s1 = t.stride()
        if c == cols:
            if s1 != 1 and cols > 1:
                _bad(who, f"{name}: a row must be contiguous")
            if rows <= 1:
                return rows, cols
            if s0 < cols:
                _bad(who, f"{name}: rows overlap")
            return rows, s0
    if t.dim() < 1 or cols < 1 or t.shape[-1] != cols:
        _bad(who, f"{name} must have {cols} columns, got {tuple(t.shape)}")
    if not t.is_contiguous():
        _bad(who, f"{name}: only a two-dimensional tensor may have gaps between its rows")
    return t.numel() // cols, cols


def _same_rows(who, name, t, rows, cols, dtype, cur):
    """Elements between the rows of t, which has to be rows x cols."""
    r, ld = _rows(who, name, t, cols, dtype, cur)
    if r != rows:
        _bad(who, f"{name} must have {rows} rows, got {r}")
    return ld


def _precision(who, t):
    if t.dtype is torch.bfloat16:
        return BF16
    if t.dtype is torch.float32:
        return FP32
    _bad(who, f"tensors are float32 or bfloat16, got {t.dtype}")


def _vector(who, name, t, n, cur):
    if t.get_device() != cur or t.dtype is not torch.float32 or not t.is_contiguous() or t.numel() != n:
        _bad(who, f"{name} must be {n} contiguous float32 values on the current CUDA device")
    return t.data_ptr()


def _is_image(t):
    return t.dtype is torch.uint8


def _image(who, name, t, rows, cols, parts, cur):
    if t.get_device() != cur or not _is_image(t) or not t.is_contiguous():
        _bad(who, f"{name}: an 8-bit image is a contiguous uint8 tensor on the current CUDA device")
    pitch = (cols + 31) // 32 * 32
    need = parts * ((rows * (pitch + pitch // 32) + 255) // 256 * 256)
    if t.numel() < need:
        _bad(who, f"{name}: an image of {rows} x {cols} ({parts} parts) takes {need} bytes, got {t.numel()}")


def _kept(who, stash, rows, cols, parts, dtype, cur):
    """Form of the kept values from the tensor's type: STASH_*."""
    if stash is None:
        return STASH_NONE
    if _is_image(stash):
        _image(who, "stash", stash, rows, cols, parts, cur)
        return STASH_8BIT
    if stash.dtype is not dtype or stash.get_device() != cur or not stash.is_contiguous() or stash.numel() != parts * rows * cols:
        _bad(who, f"stash must be a contiguous {dtype} tensor of {parts} x {rows} x {cols} values, or an 8-bit image")
    return STASH_FULL


def _addr(t):
    return None if t is None else t.data_ptr()


# What a call's checks depend on (device, types, shapes, gaps, alignment, options: nothing of an address but whether it
# lies on 16 bytes, nothing of the values) -> its descriptor and workspace size, so that a call like an earlier one is not
# checked again
_PLANS = {}


def _sig(t):
    return None if t is None else (t.dtype, t.get_device(), t.shape, t.stride())


def _plan(key, size_of, backward, *fields):
    d, n = FfnDesc(*fields), _sz()
    _check(size_of(C.byref(d), backward, C.byref(n)))
    if len(_PLANS) >= 4096:
        _PLANS.clear()
    p = _PLANS[key] = (C.byref(d), n.value)
    return p


_NO_WS = (None, 0, None)


def _workspace(who, need, ws, stream, cur):
    """(address, bytes, tensor to keep alive until the launches are queued)."""
    if ws is None:
        if stream is None:
            ws = torch.empty(need, dtype=torch.uint8, device="cuda")
        else:
            with torch.cuda.stream(torch.cuda.ExternalStream(stream) if isinstance(stream, int) else stream):
                ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    elif ws.get_device() != cur or not ws.is_contiguous():
        _bad(who, "ws must be a contiguous tensor on the current CUDA device")
    return ws.data_ptr(), ws.numel() * ws.element_size(), ws


def ftp_checkpoint_bytes(rows, cols, parts=1):
    n = _sz()
    _check(lib.ftp_checkpoint_bytes(rows, cols, parts, C.byref(n)))
    return n.value


def _plan_checkpoint(key, cur, who, name, x, image, part):
    cols = x.shape[-1] if x.dim() else 0
    prec = _precision(who, x)
    rows, ld = _rows(who, name, x, cols, x.dtype, cur)
    _image(who, "image", image, rows, cols, part + 1, cur)
    if len(_PLANS) >= 4096:
        _PLANS.clear()
    p = _PLANS[key] = (rows, cols, ld, prec)
    return p


def ftp_checkpoint_pack(x, image, part=0, stream=None):
    """8-bit image of x (tokens x channels) into part `part` of `image`; see include/ftpipe.h for the format."""
    cur = _current()
    key = (4, cur, part, x.dtype, x.get_device(), x.shape, x.stride(), _sig(image))
    rows, cols, ld, prec = _PLANS.get(key) or _plan_checkpoint(key, cur, "checkpoint_pack", "x", x, image, part)
    st = lib.ftp_checkpoint_pack(x.data_ptr(), rows, cols, ld, prec, image.data_ptr(), part, _raw_stream(stream, cur))
    if st:
        _check(st)


def ftp_checkpoint_unpack(image, out, part=0, stream=None):
    """The values of part `part` of an 8-bit image into out (tokens x channels)."""
    cur = _current()
    key = (5, cur, part, out.dtype, out.get_device(), out.shape, out.stride(), _sig(image))
    rows, cols, ld, prec = _PLANS.get(key) or _plan_checkpoint(key, cur, "checkpoint_unpack", "out", out, image, part)
    st = lib.ftp_checkpoint_unpack(image.data_ptr(), part, rows, cols, prec, out.data_ptr(), ld, _raw_stream(stream, cur))
    if st:
        _check(st)


def _weight(who, w, dtype, cur):
    """cin, cout, elements between rows of a weight matrix [cin][cout]."""
    if w.dim() != 2:
        _bad(who, "a weight matrix is [cin][cout]")
    cin, cout = w.shape
    return cin, cout, _rows(who, "w", w, cout, dtype, cur)[1]


def _weight_pair(who, a, b, dtype, cur):
    cin, cout, ld = _weight(who, a, dtype, cur)
    if _weight(who, b, dtype, cur) != (cin, cout, ld):
        _bad(who, "both weight matrices must have one shape and one gap between rows")
    return cin, cout, ld


def _plan_linear_forward(key, cur, x, w, y, bias, residual, act, stash, off):
    who, dt = "linear_forward", x.dtype
    prec = _precision(who, x)
    cin, cout, ldw = _weight(who, w, dt, cur)
    rows, ldx = _rows(who, "x", x, cin, dt, cur)
    ldy = _same_rows(who, "y", y, rows, cout, dt, cur)
    ldr = 0 if residual is None else _same_rows(who, "residual", residual, rows, cout, dt, cur)
    kind = _kept(who, stash, rows, cout, 1, dt, cur)
    if bias is not None:
        _vector(who, "bias", bias, cout, cur)
    return _plan(key, lib.ftp_linear_workspace_bytes, 0, rows, cin, cout, prec, act, kind, 0, 0, int(off), ldx, ldw, ldy, ldr, 0, 0)


def ftp_linear_forward(x, w, y, bias=None, residual=None, act=ACT_NONE, stash=None, ws=None, stream=None):
    """y = act(x w + bias) + residual.  stash: keeps x w + bias, in a tensor like y or as an 8-bit image (uint8)."""
    cur = _current()
    px, pw = x.data_ptr(), w.data_ptr()
    off = (px | pw) & 15 != 0
    key = (0, cur, act, off, x.dtype, x.get_device(), x.shape, x.stride(), w.dtype, w.get_device(), w.shape, w.stride(), y.dtype, y.get_device(), y.shape,
           y.stride(), _sig(bias), _sig(residual), _sig(stash))
    d, need = _PLANS.get(key) or _plan_linear_forward(key, cur, x, w, y, bias, residual, act, stash, off)
    pws, nws, keep = _workspace("linear_forward", need, ws, stream, cur) if need else _NO_WS
    st = lib.ftp_linear_forward(d, px, pw, _addr(bias), _addr(residual), y.data_ptr(), _addr(stash), pws, nws, _raw_stream(stream, cur))
    if st:
        _check(st)


def _ffn_input(who, x, rows, cin, dtype, cur):
    """(is an image, elements between rows) of a backward pass's x."""
    if x is None:
        return 0, 0
    if _is_image(x):
        _image(who, "x", x, rows, cin, 1, cur)
        return 1, 0
    return 0, _same_rows(who, "x", x, rows, cin, dtype, cur)


def _ffn_dx(who, dx, dx_addend, rows, cin, dtype, cur):
    return (0 if dx is None else _same_rows(who, "dx", dx, rows, cin, dtype, cur),
            0 if dx_addend is None else _same_rows(who, "dx_addend", dx_addend, rows, cin, dtype, cur))


def _ffn_dw(who, dw, cin, cout, dtype, cur):
    """(elements between rows, gradients are float although the tensors are bf16)."""
    if dw is None:
        return 0, 0
    f32 = dw.dtype is torch.float32
    return _same_rows(who, "dw", dw, cin, cout, torch.float32 if f32 else dtype, cur), int(f32 and dtype is torch.bfloat16)


def _plan_linear_backward(key, cur, x, w, dy, dx, dw, dbias, act, stash, dx_addend, off):
    who, dt = "linear_backward", dy.dtype
    prec = _precision(who, dy)
    cin, cout, ldw = _weight(who, w, dt, cur)
    rows, ldy = _rows(who, "dy", dy, cout, dt, cur)
    x8, ldx = _ffn_input(who, x, rows, cin, dt, cur)
    lddx, ldr = _ffn_dx(who, dx, dx_addend, rows, cin, dt, cur)
    lddw, f32 = _ffn_dw(who, dw, cin, cout, dt, cur)
    kind = _kept(who, stash, rows, cout, 1, dt, cur)
    if dbias is not None:
        _vector(who, "dbias", dbias, cout, cur)
    return _plan(key, lib.ftp_linear_workspace_bytes, 1, rows, cin, cout, prec, act, kind, x8, f32, int(off), ldx, ldw, ldy, ldr, lddx, lddw)


def ftp_linear_backward(x, w, dy, dx=None, dw=None, dbias=None, act=ACT_NONE, stash=None, dx_addend=None, ws=None, stream=None):
    """Gradients of ftp_linear_forward from dy: dx = dz w^T + dx_addend, dw = x^T dz, dbias = column sums of
    dz = dy act'(stash).  x: the input, or its 8-bit image; dw: x's type or float32.  Each output may be left out."""
    cur = _current()
    px, pw, pdy = _addr(x), w.data_ptr(), dy.data_ptr()
    off = ((px or 0) | pw | pdy) & 15 != 0
    key = (1, cur, act, off, _sig(x), w.dtype, w.get_device(), w.shape, w.stride(), dy.dtype, dy.get_device(), dy.shape, dy.stride(), _sig(dx), _sig(dw),
           _sig(dbias), _sig(stash), _sig(dx_addend))
    d, need = _PLANS.get(key) or _plan_linear_backward(key, cur, x, w, dy, dx, dw, dbias, act, stash, dx_addend, off)
    pws, nws, keep = _workspace("linear_backward", need, ws, stream, cur) if need else _NO_WS
    st = lib.ftp_linear_backward(d, px, pw, _addr(stash), pdy, _addr(dx_addend), _addr(dx), _addr(dw), _addr(dbias), pws, nws, _raw_stream(stream, cur))
    if st:
        _check(st)


def _plan_gated_forward(key, cur, x, w_gate, w_up, h, act, stash, off):
    who, dt = "gated_forward", x.dtype
    prec = _precision(who, x)
    cin, cout, ldw = _weight_pair(who, w_gate, w_up, dt, cur)
    rows, ldx = _rows(who, "x", x, cin, dt, cur)
    ldy = 0 if h is None else _same_rows(who, "h", h, rows, cout, dt, cur)
    kind = _kept(who, stash, rows, cout, 2, dt, cur)
    return _plan(key, lib.ftp_gated_workspace_bytes, 0, rows, cin, cout, prec, act, kind, 0, 0, int(off), ldx, ldw, ldy, 0, 0, 0)


def ftp_gated_forward(x, w_gate, w_up, h=None, act=ACT_SILU, stash=None, ws=None, stream=None):
    """h = act(x w_gate) * (x w_up).  stash: keeps both products, in a tensor (2, rows, cout) or as an 8-bit image of two
    parts (uint8)."""
    cur = _current()
    px, pg, pu = x.data_ptr(), w_gate.data_ptr(), w_up.data_ptr()
    off = (px | pg | pu) & 15 != 0
    key = (2, cur, act, off, x.dtype, x.get_device(), x.shape, x.stride(), w_gate.dtype, w_gate.get_device(), w_gate.shape, w_gate.stride(), _sig(w_up), _sig(h),
           _sig(stash))
    d, need = _PLANS.get(key) or _plan_gated_forward(key, cur, x, w_gate, w_up, h, act, stash, off)
    pws, nws, keep = _workspace("gated_forward", need, ws, stream, cur) if need else _NO_WS
    st = lib.ftp_gated_forward(d, px, pg, pu, _addr(h), _addr(stash), pws, nws, _raw_stream(stream, cur))
    if st:
        _check(st)


def _plan_gated_backward(key, cur, x, w_gate, w_up, dh, dx, dw_gate, dw_up, act, stash, dx_addend, off):
    who, dt = "gated_backward", dh.dtype
    prec = _precision(who, dh)
    if (dw_gate is None) != (dw_up is None):
        _bad(who, "both weight gradients or neither")
    cin, cout, ldw = _weight_pair(who, w_gate, w_up, dt, cur)
    rows, ldy = _rows(who, "dh", dh, cout, dt, cur)
    x8, ldx = _ffn_input(who, x, rows, cin, dt, cur)
    lddx, ldr = _ffn_dx(who, dx, dx_addend, rows, cin, dt, cur)
    lddw, f32 = _ffn_dw(who, dw_gate, cin, cout, dt, cur)
    if dw_up is not None and _ffn_dw(who, dw_up, cin, cout, dt, cur) != (lddw, f32):
        _bad(who, "both weight gradients must have one type and one gap between rows")
    kind = _kept(who, stash, rows, cout, 2, dt, cur)
    return _plan(key, lib.ftp_gated_workspace_bytes, 1, rows, cin, cout, prec, act, kind, x8, f32, int(off), ldx, ldw, ldy, ldr, lddx, lddw)


def ftp_gated_backward(x, w_gate, w_up, dh, dx=None, dw_gate=None, dw_up=None, act=ACT_SILU, stash=None, dx_addend=None, ws=None, stream=None):
    """Gradients of ftp_gated_forward from dh.  x: the input, or its 8-bit image; stash: what the forward pass kept (None:
    both products are computed again from x); dw_gate, dw_up: x's type or float32.  dx or the pair may be left out."""
    cur = _current()
    px, pg, pu = _addr(x), w_gate.data_ptr(), w_up.data_ptr()
    off = ((px or 0) | pg | pu) & 15 != 0
    key = (3, cur, act, off, _sig(x), w_gate.dtype, w_gate.get_device(), w_gate.shape, w_gate.stride(), _sig(w_up), dh.dtype, dh.get_device(), dh.shape,
           dh.stride(), _sig(dx), _sig(dw_gate), _sig(dw_up), _sig(stash), _sig(dx_addend))
    d, need = _PLANS.get(key) or _plan_gated_backward(key, cur, x, w_gate, w_up, dh, dx, dw_gate, dw_up, act, stash, dx_addend, off)
    pws, nws, keep = _workspace("gated_backward", need, ws, stream, cur) if need else _NO_WS
    st = lib.ftp_gated_backward(d, px, pg, pu, _addr(stash), dh.data_ptr(), _addr(dx_addend), _addr(dx), _addr(dw_gate), _addr(dw_up), pws, nws,
                                _raw_stream(stream, cur))
    if st:
        _check(st)


def ftp_check_op_status(stream=None):
    """Waits for the stream; raises FtpError if a bounded wait of an operator's kernel ran out since the last check."""
    _check(lib.ftp_check_op_status(_stream(stream)))


# ---- operators around the feed-forward products --------------------------------------------------
def _remember(key, plan):
    if len(_PLANS) >= 4096:
        _PLANS.clear()
    _PLANS[key] = plan
    return plan


def _words(who, rng, dropout, cur):
    """The generator's two words (int64: key, step) on the device."""
    if rng is None:
        if dropout:
            _bad(who, "dropout without the generator's words")
        return
    if rng.get_device() != cur or rng.dtype is not torch.int64 or not rng.is_contiguous() or rng.numel() != 2:
        _bad(who, "rng must be two contiguous int64 words (key, step) on the current CUDA device")


def _floats(who, name, t, n, cur):
    if t is not None:
        _vector(who, name, t, n, cur)


def _plan_dropout(key, cur, x, y, dropout, rng):
    who, cols = "dropout", x.shape[-1] if x.dim() else 0
    prec = _precision(who, x)
    rows, ldx = _rows(who, "x", x, cols, x.dtype, cur)
    ldy = _same_rows(who, "y", y, rows, cols, x.dtype, cur)
    _words(who, rng, dropout, cur)
    return _remember(key, (rows, cols, ldx, ldy, prec))


def ftp_dropout(x, y, dropout, rng, site=0, row0=0, stream=None):
    """y = x with elements dropped at the rate `dropout`, the others divided by what stays; the same call on dy gives the
    gradient.  rng: int64 tensor (key, step) in device memory; site: which dropout of a step; row0: number of x's first row."""
    cur = _current()
    key = (6, cur, dropout != 0, _sig(x), _sig(y), _sig(rng))
    rows, cols, ldx, ldy, prec = _PLANS.get(key) or _plan_dropout(key, cur, x, y, dropout, rng)
    st = lib.ftp_dropout(x.data_ptr(), y.data_ptr(), rows, cols, ldx, ldy, prec, dropout, _addr(rng), site, row0, _raw_stream(stream, cur))
    if st:
        _check(st)


def _gate(who, name, gate, gate_rows, rows, cols, dt, cur):
    """Elements between rows of a gate or its gradient (0: a vector)."""
    if gate is None:
        return 0
    if gate_rows < 0:
        _bad(who, "gate_rows must not be negative")
    if gate_rows == 0:
        _vector(who, name, gate, cols, cur)
        return 0
    return _same_rows(who, name, gate, -(-rows // gate_rows), cols, dt, cur)


def _plan_join_forward(key, cur, u, x, s, y, post, pre, w_post, b_post, w_pre, b_pre, gate, gate_rows, alpha, beta, eps, dropout, rng, site, row0, stats):
    who, one = "join_forward", u if u is not None else x
    if one is None:
        _bad(who, "u or x is needed")
    dt, prec, cols = one.dtype, _precision(who, one), one.shape[-1] if one.dim() else 0
    rows = _rows(who, "u" if u is not None else "x", one, cols, dt, cur)[0]
    ldu, ldx, lds, ldy = (0 if t is None else _same_rows(who, n, t, rows, cols, dt, cur) for n, t in (("u", u), ("x", x), ("s", s), ("y", y)))
    for n, t in (("w_post", w_post), ("b_post", b_post), ("w_pre", w_pre), ("b_pre", b_pre)):
        _floats(who, n, t, cols, cur)
    _floats(who, "stats", stats, 4 * rows, cur)
    _words(who, rng, dropout, cur)
    ldg = _gate(who, "gate", gate, gate_rows, rows, cols, dt, cur)
    d = JoinDesc(rows, cols, prec, post, pre, eps, alpha, beta, site, dropout, row0, gate_rows, ldu, ldx, lds, ldy, ldg, 0, 0, 0, 0)
    return _remember(key, (C.byref(d), 0))


def ftp_join_forward(u, x, s, y=None, post=NORM_RMS, pre=NORM_RMS, w_post=None, b_post=None, w_pre=None, b_pre=None, gate=None, gate_rows=0, alpha=1.0,
                     beta=1.0, eps=1e-6, dropout=0.0, rng=None, site=0, row0=0, stats=None, stream=None):
    """s = alpha x + beta gate drop(post(u)), y = pre(s).  u None: y = pre(x) alone (s None).  gate: a float vector, or with
    gate_rows a tensor like u with a row for every gate_rows tokens.  stats: float32, (4, rows), for the backward pass.  dropout, rng,
    site, row0: as in ftp_dropout."""
    cur = _current()
    key = (7, cur, post, pre, gate_rows, alpha, beta, eps, dropout, site, row0, _sig(u), _sig(x), _sig(s), _sig(y), _sig(w_post), _sig(b_post), _sig(w_pre),
           _sig(b_pre), _sig(gate), _sig(rng), _sig(stats))
    d, _ = _PLANS.get(key) or _plan_join_forward(key, cur, u, x, s, y, post, pre, w_post, b_post, w_pre, b_pre, gate, gate_rows, alpha, beta, eps, dropout, rng,
                                                 site, row0, stats)
    st = lib.ftp_join_forward(d, _addr(u), _addr(x), _addr(w_post), _addr(b_post), _addr(gate), _addr(w_pre), _addr(b_pre), _addr(rng), _addr(s), _addr(y),
                              _addr(stats), _raw_stream(stream, cur))
    if st:
        _check(st)


def _plan_join_backward(key, cur, u, s, dy, ds, stats, du, dx, dw_post, db_post, dw_pre, db_pre, dgate, post, pre, w_post, b_post, w_pre, gate, gate_rows, alpha,
                        beta, dropout, rng, site, row0):
    who, one = "join_backward", dy if dy is not None else ds
    if one is None:
        _bad(who, "no gradient comes in")
    dt, prec, cols = one.dtype, _precision(who, one), one.shape[-1] if one.dim() else 0
    rows = _rows(who, "dy" if dy is not None else "ds", one, cols, dt, cur)[0]
    ldu, lds, ldy, ldds, lddu, lddx = (0 if t is None else _same_rows(who, n, t, rows, cols, dt, cur)
                                       for n, t in (("u", u), ("s", s), ("dy", dy), ("ds", ds), ("du", du), ("dx", dx)))
    for n, t in (("w_post", w_post), ("b_post", b_post), ("w_pre", w_pre), ("dw_post", dw_post), ("db_post", db_post), ("dw_pre", dw_pre), ("db_pre", db_pre)):
        _floats(who, n, t, cols, cur)
    _floats(who, "stats", stats, 4 * rows, cur)
    _words(who, rng, dropout, cur)
    ldg = _gate(who, "gate", gate, gate_rows, rows, cols, dt, cur)
    lddg = _gate(who, "dgate", dgate, gate_rows, rows, cols, dt, cur)
    d, n = JoinDesc(rows, cols, prec, post, pre, 0.0, alpha, beta, site, dropout, row0, gate_rows, ldu, 0, lds, ldy, ldg, lddu, ldds, lddx, lddg), _sz()
    _check(lib.ftp_join_workspace_bytes(C.byref(d), C.byref(n)))
    return _remember(key, (C.byref(d), n.value))


def ftp_join_backward(u, s, dy, ds, stats, du=None, dx=None, dw_post=None, db_post=None, dw_pre=None, db_pre=None, dgate=None, post=NORM_RMS, pre=NORM_RMS,
                      w_post=None, b_post=None, w_pre=None, gate=None, gate_rows=0, alpha=1.0, beta=1.0, dropout=0.0, rng=None, site=0, row0=0, ws=None,
                      stream=None):
    """Gradients of ftp_join_forward from dy and ds, with its other arguments (s: x where u was None).  Each output may be left out."""
    cur = _current()
    key = (8, cur, post, pre, gate_rows, alpha, beta, dropout, site, row0, _sig(u), _sig(s), _sig(dy), _sig(ds), _sig(stats), _sig(du), _sig(dx), _sig(dw_post),
           _sig(db_post), _sig(dw_pre), _sig(db_pre), _sig(dgate), _sig(w_post), _sig(b_post), _sig(w_pre), _sig(gate), _sig(rng))
    d, need = _PLANS.get(key) or _plan_join_backward(key, cur, u, s, dy, ds, stats, du, dx, dw_post, db_post, dw_pre, db_pre, dgate, post, pre, w_post, b_post, w_pre,
                                                     gate, gate_rows, alpha, beta, dropout, rng, site, row0)
    pws, nws, keep = _workspace("join_backward", need, ws, stream, cur) if need else _NO_WS
    st = lib.ftp_join_backward(d, _addr(u), _addr(s), _addr(w_post), _addr(b_post), _addr(gate), _addr(w_pre), _addr(stats), _addr(rng), _addr(dy), _addr(ds),
                               _addr(du), _addr(dx), _addr(dw_post), _addr(db_post), _addr(dw_pre), _addr(db_pre), _addr(dgate), pws, nws,
                               _raw_stream(stream, cur))
    if st:
        _check(st)


def _steps(who, name, t, shape, dt, cur):
    """Elements between the steps of t, whose shape must be `shape`: (rows, cols), or (seqs, len, cols) with one gap throughout."""
    if tuple(t.shape) != tuple(shape):
        _bad(who, f"{name} must be {tuple(shape)}, got {tuple(t.shape)}")
    if t.dim() == 3 and not t.is_contiguous():
        if t.dtype is not dt or t.get_device() != cur:
            _bad(who, f"{name} must be {dt} on the current CUDA device")
        b, n, c = t.shape
        s0, s1, s2 = t.stride()
        if n == 1:
            s1 = s0                                                  # a step each: the sequences' gap is the steps'
        if (s2 != 1 and c > 1) or s1 < c or (b > 1 and s0 != n * s1):
            _bad(who, f"{name}: steps must be contiguous inside and the same gap apart throughout")
        return s1
    return _rows(who, name, t, shape[-1], dt, cur)[1]


def _recurrence_desc(who, cur, f, act, coupled, offsets, max_len, named, states, vectors):
    """Descriptor from f's shape; named: (name, tensor) in the order of the descriptor's pitches."""
    if f.dim() not in (2, 3):
        _bad(who, "f is (steps, channels) or (sequences, steps, channels)")
    dt, prec = f.dtype, _precision(who, f)
    cols = f.shape[-1]
    if offsets is None:
        seqs, n, rows = (f.shape[0], f.shape[1], 0) if f.dim() == 3 else (1, f.shape[0], 0)
    else:
        if f.dim() != 2:
            _bad(who, "with offsets f is (rows, channels)")
        if offsets.get_device() != cur or offsets.dtype is not torch.int32 or not offsets.is_contiguous() or offsets.dim() != 1 or offsets.numel() < 1:
            _bad(who, "offsets must be a contiguous int32 vector of sequences + 1 values on the current CUDA device")
        seqs, rows = offsets.numel() - 1, f.shape[0]
        n = rows if max_len is None else min(max_len, rows)
    pitches = [0 if t is None else _steps(who, name, t, f.shape, dt, cur) for name, t in named]
    d = RecurrenceDesc(seqs, n, rows, cols, prec, act, int(coupled), *pitches)
    for name, t in vectors:
        _floats(who, name, t, seqs * cols, cur)
    if states is not None:
        need = _i64()
        _check(lib.ftp_recurrence_states(C.byref(d), C.byref(need)))
        if states.get_device() != cur or states.dtype is not torch.float32 or not states.is_contiguous() or states.numel() < need.value * cols:
            _bad(who, f"states must be contiguous float32 of {need.value} x {cols} values on the current CUDA device")
    return d


def ftp_recurrence_states(rows, seqs):
    """Rows of the tensor of kept states for `rows` steps in all of `seqs` sequences."""
    d, n = RecurrenceDesc(seqs, 0, rows, 1, 0, 0, 0), _i64()
    _check(lib.ftp_recurrence_states(C.byref(d), C.byref(n)))
    return n.value


def ftp_recurrence_forward(f, v, y, o=None, h0=None, h1=None, states=None, act=ACT_SILU, coupled=True, offsets=None, max_len=None, stream=None):
    """h_t = a_t h_(t-1) + (1 - a_t) v_t (coupled, else + v_t), a = sigmoid(f), y = act(o) h (o None: y = h).  f, v, o, y: (sequences,
    steps, channels), or (rows, channels): one sequence, or those that offsets (int32, sequences + 1) cut out of the rows, max_len
    steps at most.  h0, h1: float32 states (sequences, channels) before and behind, which may be one tensor; states: float32
    (ftp_recurrence_states(rows, sequences), channels), kept for the backward pass."""
    cur = _current()
    if o is None:
        act = ACT_NONE
    key = (9, cur, act, bool(coupled), max_len, _sig(f), _sig(v), _sig(y), _sig(o), _sig(h0), _sig(h1), _sig(states), _sig(offsets))
    d = _PLANS.get(key) or _remember(key, C.byref(_recurrence_desc("recurrence_forward", cur, f, act, coupled, offsets, max_len, (
        ("f", f), ("v", v), ("o", o), ("y", y)), states, (("h0", h0), ("h1", h1)))))
    st = lib.ftp_recurrence_forward(d, f.data_ptr(), v.data_ptr(), _addr(o), _addr(h0), _addr(offsets), y.data_ptr(), _addr(h1), _addr(states),
                                    _raw_stream(stream, cur))
    if st:
        _check(st)


def ftp_recurrence_backward(f, v, dy, states, df, dv, o=None, do=None, dh1=None, dh0=None, act=ACT_SILU, coupled=True, offsets=None, max_len=None, stream=None):
    """Gradients of ftp_recurrence_forward from dy and dh1 (of h1), with its other arguments and the states it kept.  dh0 may be dh1."""
    cur = _current()
    if o is None:
        act = ACT_NONE
    key = (10, cur, act, bool(coupled), max_len, _sig(f), _sig(v), _sig(dy), _sig(states), _sig(df), _sig(dv), _sig(o), _sig(do), _sig(dh1), _sig(dh0),
           _sig(offsets))
    d = _PLANS.get(key) or _remember(key, C.byref(_recurrence_desc("recurrence_backward", cur, f, act, coupled, offsets, max_len, (
        ("f", f), ("v", v), ("o", o), ("dy", dy), ("df", df), ("dv", dv), ("do", do)), states, (("dh1", dh1), ("dh0", dh0)))))
    st = lib.ftp_recurrence_backward(d, f.data_ptr(), v.data_ptr(), _addr(o), states.data_ptr(), _addr(offsets), dy.data_ptr(), _addr(dh1), df.data_ptr(),
                                     dv.data_ptr(), _addr(do), _addr(dh0), _raw_stream(stream, cur))
    if st:
        _check(st)


def _integers(who, name, t, n, cur):
    if t is not None and (t.get_device() != cur or t.dtype is not torch.int32 or not t.is_contiguous() or t.numel() != n):
        _bad(who, f"{name} must be {n} contiguous int32 values on the current CUDA device")


def _plan_logprob_forward(key, cur, logits, targets, logp, entropy, lse, top, top_logp):
    who, vocab = "logprob_forward", logits.shape[-1] if logits.dim() else 0
    prec = _precision(who, logits)
    rows, ld = _rows(who, "logits", logits, vocab, logits.dtype, cur)
    k = 0 if top is None else top.shape[-1] if top.dim() else 0
    if top is not None and k < 1:
        _bad(who, "top must be rows x k")
    _integers(who, "targets", targets, rows, cur)
    _integers(who, "top", top, rows * k, cur)
    for n, t, size in (("logp", logp, rows), ("entropy", entropy, rows), ("lse", lse, 2 * rows), ("top_logp", top_logp, rows * k)):
        _floats(who, n, t, size, cur)
    return _remember(key, (rows, vocab, ld, prec, k))


def ftp_logprob_forward(logits, targets, logp=None, entropy=None, lse=None, top=None, top_logp=None, scale=1.0, stream=None):
    """Log probabilities of the tokens `targets` (int32) under scale * logits (rows x vocab), the rows' entropies, the likeliest
    tokens (top: int32, rows x k) with their log probabilities, and lse (rows x 2) for the backward pass; all float32, each may be left out."""
    cur = _current()
    key = (11, cur, _sig(logits), _sig(targets), _sig(logp), _sig(entropy), _sig(lse), _sig(top), _sig(top_logp))
    rows, vocab, ld, prec, k = _PLANS.get(key) or _plan_logprob_forward(key, cur, logits, targets, logp, entropy, lse, top, top_logp)
    st = lib.ftp_logprob_forward(logits.data_ptr(), rows, vocab, ld, prec, scale, _addr(targets), _addr(logp), _addr(entropy), _addr(lse), _addr(top),
                                 _addr(top_logp), k, _raw_stream(stream, cur))
    if st:
        _check(st)


def _plan_logprob_backward(key, cur, logits, targets, lse, dlogp, dlogits, entropy, dentropy):
    who, vocab = "logprob_backward", logits.shape[-1] if logits.dim() else 0
    prec = _precision(who, logits)
    rows, ld = _rows(who, "logits", logits, vocab, logits.dtype, cur)
    ldd = _same_rows(who, "dlogits", dlogits, rows, vocab, logits.dtype, cur)
    _integers(who, "targets", targets, rows, cur)
    for n, t, size in (("lse", lse, 2 * rows), ("dlogp", dlogp, rows), ("entropy", entropy, rows), ("dentropy", dentropy, rows)):
        _floats(who, n, t, size, cur)
    return _remember(key, (rows, vocab, ld, prec, ldd))


def ftp_logprob_backward(logits, targets, lse, dlogp, dlogits, entropy=None, dentropy=None, scale=1.0, stream=None):
    """Gradient of the logits from dlogp and dentropy (each may be None) with what ftp_logprob_forward left; dlogits may be logits."""
    cur = _current()
    key = (12, cur, _sig(logits), _sig(targets), _sig(lse), _sig(dlogp), _sig(dlogits), _sig(entropy), _sig(dentropy))
    rows, vocab, ld, prec, ldd = _PLANS.get(key) or _plan_logprob_backward(key, cur, logits, targets, lse, dlogp, dlogits, entropy, dentropy)
    st = lib.ftp_logprob_backward(logits.data_ptr(), rows, vocab, ld, prec, scale, _addr(targets), _addr(lse), _addr(entropy), _addr(dlogp), _addr(dentropy),
                                  dlogits.data_ptr(), ldd, _raw_stream(stream, cur))
    if st:
        _check(st)


def ftp_kernel_name(k):
    return lib.ftp_kernel_name(k).decode()


# ---- the model -----------------------------------------------------------------------------------
class Model:
    """Owns the workspaces (torch device memory + pinned host memory) and the ftp_model handle.
    Methods are the C entry points with the handle bound."""

    def __init__(self, layers, cfg, device="cuda:0"):
        import torch
        self.torch = torch
        self.layers, self.cfg = list(layers), dict(cfg)
        self.device = torch.device(device)
        dev_bytes, pin_bytes = ftp_workspace_bytes(layers, cfg)
        self.dev_ws = torch.empty(dev_bytes + 256, dtype=torch.uint8, device=self.device)
        self.pin_ws = torch.empty(max(pin_bytes, 256), dtype=torch.uint8).pin_memory()
        base = (self.dev_ws.data_ptr() + 255) // 256 * 256
        h = _vp()
        with torch.cuda.device(self.device):
            _check(lib.ftp_build_model(layer_array(layers), len(layers), C.byref(model_cfg(cfg)), base, dev_bytes,
                                       self.pin_ws.data_ptr(), self.pin_ws.numel(), C.byref(h)))
        self.h = h
        n = _i32()
        _check(lib.ftp_num_units(self.h, C.byref(n)))
        self.L = n.value
        self.act_dtype = torch.bfloat16 if cfg["precision"] == BF16 else torch.float32

    def close(self):
        if getattr(self, "h", None) and lib is not None:        # lib is None while the interpreter shuts down
            lib.ftp_destroy_model(self.h)
            self.h = None

    __del__ = close

    def ftp_unit_param_span(self, unit):
        o, c = _i64(), _i64()
        _check(lib.ftp_unit_param_span(self.h, unit, C.byref(o), C.byref(c)))
        return o.value, c.value

    def ftp_unit_state_span(self, unit):
        o, c = _i64(), _i64()
        _check(lib.ftp_unit_state_span(self.h, unit, C.byref(o), C.byref(c)))
        return o.value, c.value

    def ftp_unit_output_shape(self, unit):
        shp = (_i32 * 4)()
        b = _i64()
        _check(lib.ftp_unit_output_shape(self.h, unit, shp, C.byref(b)))
        return tuple(shp), b.value

    def ftp_set_tensor(self, which, unit, src, stream=None):
        """src: float32 numpy array (host) or torch CUDA tensor (device)."""
        dev = not isinstance(src, np.ndarray)
        if not dev:
            src = np.ascontiguousarray(src, dtype=np.float32)
        n = src.size if not dev else src.numel()
        _check(lib.ftp_set_tensor(self.h, which, unit, _ptr(src), n, int(dev), _stream(stream)))

    def ftp_get_tensor(self, which, unit, stream=None):
        """Returns a float32 numpy array (host copy)."""
        n = self.ftp_unit_state_span(unit)[1] if which == T_STATE else self.ftp_unit_param_span(unit)[1]
        out = np.empty(n, np.float32)
        _check(lib.ftp_get_tensor(self.h, which, unit, _ptr(out), n, 0, _stream(stream)))
        return out

    def ftp_run_stage_forward(self, a, b, act_in, act_out=None, labels=None, loss_out=None, stream=None):
        _check(lib.ftp_run_stage_forward(self.h, a, b, _ptr(act_in), _ptr(act_out), _ptr(labels), _ptr(loss_out),
                                         _stream(stream)))

    def ftp_run_stage_backward(self, a, b, grad_out=None, grad_in=None, stream=None):
        _check(lib.ftp_run_stage_backward(self.h, a, b, _ptr(grad_out), _ptr(grad_in), _stream(stream)))

    def ftp_get_logits(self, stream=None):
        out = np.empty((self.cfg["batch"], self.cfg["n_classes"]), np.float32)
        _check(lib.ftp_get_logits(self.h, _ptr(out), 0, _stream(stream)))
        return out

    def ftp_sgd_step(self, a, b, lr, snap_dev=None, snap_host=None, stream=None):
        _check(lib.ftp_sgd_step(self.h, a, b, lr, _ptr(snap_dev), _ptr(snap_host), _stream(stream)))

    def ftp_train_step(self, x, labels, lr, inputs_on_host=False, want_loss=True, stream=None, loss_pinned=None):
        """loss_pinned: a pinned float32 host tensor of one element that receives the loss instead of the return value --
        the form to use while the step is captured into a CUDA graph (the copy becomes a node of the graph)."""
        if loss_pinned is not None:
            if loss_pinned.is_cuda or not loss_pinned.is_pinned() or loss_pinned.numel() < 1 or loss_pinned.element_size() != 4:
                raise ValueError("loss_pinned must be a pinned float32 host tensor")
            _check(lib.ftp_train_step(self.h, _ptr(x), _ptr(labels), int(inputs_on_host), lr,
                                      C.cast(loss_pinned.data_ptr(), _P(_f32)), _stream(stream)))
            return None
        loss = _f32()
        _check(lib.ftp_train_step(self.h, _ptr(x), _ptr(labels), int(inputs_on_host), lr,
                                  C.byref(loss) if want_loss else None, _stream(stream)))
        return loss.value if want_loss else None

    def ftp_stage_timing_enable(self, on):
        _check(lib.ftp_stage_timing_enable(self.h, int(on)))

    def ftp_stage_times(self):
        """Forward + backward device seconds of every stage in the last timed ftp_train_step."""
        t = (C.c_double * self.cfg["max_stages"])()
        n = _i32()
        _check(lib.ftp_stage_times(self.h, t, C.byref(n)))
        return list(t[:n.value])

    def ftp_profile_layers(self, reps, sample_in, labels, stream=None):
        f, b = np.zeros(self.L), np.zeros(self.L)
        ob = np.zeros(self.L, np.int64)
        _check(lib.ftp_profile_layers(self.h, reps, _ptr(sample_in), _ptr(labels), f.ctypes.data_as(_P(C.c_double)),
                                      b.ctypes.data_as(_P(C.c_double)), ob.ctypes.data_as(_P(_i64)), _stream(stream)))
        return f, b, ob

    def ftp_set_partition(self, points, stream=None):
        pts, pp = _i32arr(points)
        moved = _i32()
        _check(lib.ftp_set_partition(self.h, pp, len(pts) - 1, C.byref(moved), _stream(stream)))
        return moved.value

    def ftp_recover(self, failed, p_new, central=None, stream=None):
        """failed: {stage: chain replica tensor (device, or host for the last stage) or None}; central: the global
        replica (host tensor, all units in canonical order) or None.  Returns (from stages, from replicas, from central)."""
        recs = (FailedStage * max(len(failed), 1))()
        for k, (stage, rep) in enumerate(sorted(failed.items())):
            recs[k].stage = stage
            recs[k].replica_is_host = int(rep is not None and not rep.is_cuda)
            recs[k].replica = _ptr(rep)
            recs[k].replica_bytes = 0 if rep is None else rep.numel() * rep.element_size()
        pts, pp = _i32arr(p_new)
        counts = (_i32 * 3)()
        _check(lib.ftp_recover(self.h, recs, len(failed), _ptr(central), 0 if central is None else central.numel() * central.element_size(),
                               pp, len(pts) - 1, counts, _stream(stream)))
        return tuple(counts)

    def ftp_get_partition(self):
        pts = (_i32 * (self.cfg["max_stages"] + 1))()
        n = _i32()
        _check(lib.ftp_get_partition(self.h, pts, C.byref(n)))
        return list(pts[:n.value + 1])

    def ftp_snapshot_weights(self, stage, dst, stream=None):
        """dst: torch tensor, device or pinned host (float32)."""
        w = _sz()
        _check(lib.ftp_snapshot_weights(self.h, stage, _ptr(dst), dst.numel() * dst.element_size(),
                                        int(not dst.is_cuda), C.byref(w), _stream(stream)))
        return w.value

    def ftp_measure_bandwidth(self, pinned_host=None, nbytes=64 << 20, reps=5, stream=None):
        """(device-to-device, device-to-pinned-host) copy bandwidth in bytes per second."""
        a, b = C.c_double(), C.c_double()
        _check(lib.ftp_measure_bandwidth(self.h, _ptr(pinned_host), nbytes, reps, C.byref(a), C.byref(b), _stream(stream)))
        return a.value, b.value

    def ftp_check_guards(self, stream=None):
        """Number of guard zones checked; raises FtpError (with .bad_offset) if one was overwritten."""
        n, bad = _i32(), _i64()
        st = lib.ftp_check_guards(self.h, C.byref(n), C.byref(bad), _stream(stream))
        if st != OK:
            e = FtpError(st, lib.ftp_last_error().decode())
            e.bad_offset = bad.value
            raise e
        return n.value

    def ftp_check_device_status(self, stream=None):
        _check(lib.ftp_check_device_status(self.h, _stream(stream)))

    def ftp_debug_set_device_status(self, code, stream=None):
        _check(lib.ftp_debug_set_device_status(self.h, int(code), _stream(stream)))

    def ftp_trace_enable(self, on):
        _check(lib.ftp_trace_enable(self.h, int(on)))

    def ftp_trace_read(self, max_records=65536):
        buf = (TraceRec * max_records)()
        n = _i32()
        _check(lib.ftp_trace_read(self.h, buf, max_records, C.byref(n)))
        return [dict(kernel=ftp_kernel_name(r.kernel), unit=r.unit, op=r.op, backward=r.backward, ms=r.ms,
                     bytes=r.bytes, flops=r.flops) for r in buf[:min(n.value, max_records)]]

    def ftp_launch_count(self):
        n = _i64()
        _check(lib.ftp_launch_count(self.h, C.byref(n)))
        return n.value

    # -- marshalling helpers (no arithmetic) --
    def load_params(self, per_op_params, per_op_state=None):
        """Scatter per-op float32 arrays (canonical order) into the unit tensors."""
        for u in range(self.L):
            parts = [a.reshape(-1) for l, arrs in zip(self.layers, per_op_params) if l.unit == u for a in arrs]
            if parts:
                self.ftp_set_tensor(T_WEIGHTS, u, np.concatenate(parts).astype(np.float32))
            if per_op_state is not None:
                parts = [a.reshape(-1) for l, arrs in zip(self.layers, per_op_state) if l.unit == u for a in arrs]
                if parts:
                    self.ftp_set_tensor(T_STATE, u, np.concatenate(parts).astype(np.float32))


__all__ = ["Model", "FtpError", "LayerDesc", "ModelCfg", "TraceRec", "ftp_estimate_capacity", "ftp_choose_partition",
           "ftp_redistribution_plan", "ftp_recovery_plan", "FailedStage", "SRC_LOCAL", "SRC_STAGE", "SRC_REPLICA", "SRC_CENTRAL", "ftp_workspace_bytes", "ftp_kernel_name", "ftp_conv_wgrad_static", "layer_array", "model_cfg", "lib",
           "T_WEIGHTS", "T_GRADS", "T_MOMENTUM", "T_STATE", "FP32", "BF16", "LIB_PATH"]
