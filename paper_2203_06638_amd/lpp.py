"""Python binding of liblpp.so (argument marshalling only).

Every step of the LPP-SGD hot path runs in the HIP library; this module only
converts Python/torch arguments to the C ABI of include/lpp.h and raises
LppError on a non-zero status.  torch provides device memory and streams.
The library must have been built (paper_2203_06638_amd/build.py); there is
no fallback of any kind.
"""
from __future__ import annotations

import ctypes as C
import os

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "liblpp.so")
_LIB = None

CONV, BN, RELU, ADD, MAXPOOL, GAP, LINEAR, CONCAT, RMSNORM, GROUPNORM = range(10)
FP32, BF16 = 0, 1
SEQUENTIAL, ASYNC = 0, 1
ACT8 = 0x100
ACT_NONE, ACT_RELU, ACT_SILU = range(3)
OK, EINVAL, ENOMEM, EHIP, ESTATE, EUNSUPPORTED = 0, -1, -2, -3, -4, -5
STATUS = {0: "LPP_OK", -1: "LPP_EINVAL", -2: "LPP_ENOMEM", -3: "LPP_EHIP", -4: "LPP_ESTATE", -5: "LPP_EUNSUPPORTED"}


class LppError(RuntimeError):
    def __init__(self, code, msg):
        super().__init__("%s: %s" % (STATUS.get(code, code), msg))
        self.code = code


class Layer(C.Structure):
    _fields_ = [("op", C.c_int), ("in0", C.c_int), ("in1", C.c_int), ("cin", C.c_int), ("cout", C.c_int),
                ("k", C.c_int), ("stride", C.c_int), ("pad", C.c_int), ("bias", C.c_int), ("block", C.c_int)]


class ModelDesc(C.Structure):
    _fields_ = [("n_layers", C.c_int), ("layers", C.POINTER(Layer)), ("in_c", C.c_int), ("in_h", C.c_int),
                ("in_w", C.c_int), ("n_classes", C.c_int), ("batch", C.c_int), ("dtype", C.c_int),
                ("momentum", C.c_float), ("weight_decay", C.c_float), ("bn_eps", C.c_float)]


class Options(C.Structure):
    _fields_ = [("mode", C.c_int), ("worker_streams", C.POINTER(C.c_void_p)), ("avg_stream", C.c_void_p),
                ("unfused", C.c_int), ("no_graphs", C.c_int)]


class Batch(C.Structure):
    _fields_ = [("images", C.c_void_p), ("labels", C.c_void_p), ("n", C.c_int)]


class Teacher(C.Structure):
    _fields_ = [("values", C.c_void_p), ("index", C.c_void_p), ("rest", C.c_void_p), ("k", C.c_int),
                ("alpha", C.c_float), ("temperature", C.c_float)]


class TraceStep(C.Structure):
    _fields_ = [("worker", C.c_int), ("replica", C.c_int), ("partition", C.c_int), ("counter", C.c_long),
                ("t", C.c_ulonglong * 4)]


class TraceAvg(C.Structure):
    _fields_ = [("index", C.c_long), ("n_replicas", C.c_int), ("counter_min", C.c_long), ("t", C.c_ulonglong * 2)]


class SnapConv(C.Structure):
    _fields_ = [("src", C.c_long), ("cout", C.c_int), ("cin", C.c_int), ("cin_p", C.c_int), ("kh", C.c_int),
                ("kw", C.c_int), ("dst_f", C.c_long), ("dst_d", C.c_long)]


class RmsNormArgs(C.Structure):
    _fields_ = [("x", C.c_void_p), ("res", C.c_void_p), ("h", C.c_void_p), ("y", C.c_void_p), ("q", C.c_void_p),
                ("ldx", C.c_long), ("ldres", C.c_long), ("ldh", C.c_long), ("ldy", C.c_long), ("gamma", C.c_void_p),
                ("rstd", C.c_void_p), ("rows", C.c_long), ("cols", C.c_int), ("dtype", C.c_int), ("eps", C.c_float),
                ("keep_sign", C.c_int)]


class RmsNormBwdArgs(C.Structure):
    _fields_ = [("dy", C.c_void_p), ("h", C.c_void_p), ("q", C.c_void_p), ("dres", C.c_void_p), ("dx", C.c_void_p),
                ("lddy", C.c_long), ("ldh", C.c_long), ("lddres", C.c_long), ("lddx", C.c_long),
                ("gamma", C.c_void_p), ("rstd", C.c_void_p), ("dgamma", C.c_void_p), ("ws", C.c_void_p),
                ("ws_floats", C.c_long), ("rows", C.c_long), ("cols", C.c_int), ("dtype", C.c_int)]


class GroupNormArgs(C.Structure):
    _fields_ = [("x", C.c_void_p), ("y", C.c_void_p), ("ldx", C.c_long), ("ldy", C.c_long), ("gamma", C.c_void_p),
                ("beta", C.c_void_p), ("mean", C.c_void_p), ("rstd", C.c_void_p), ("ws", C.c_void_p),
                ("ws_floats", C.c_long), ("images", C.c_long), ("pixels", C.c_long), ("channels", C.c_int),
                ("groups", C.c_int), ("dtype", C.c_int), ("act", C.c_int), ("eps", C.c_float)]


class GroupNormBwdArgs(C.Structure):
    _fields_ = [("dy", C.c_void_p), ("x", C.c_void_p), ("dres", C.c_void_p), ("dx", C.c_void_p), ("lddy", C.c_long),
                ("ldx", C.c_long), ("lddres", C.c_long), ("lddx", C.c_long), ("gamma", C.c_void_p),
                ("beta", C.c_void_p), ("mean", C.c_void_p), ("rstd", C.c_void_p), ("dgamma", C.c_void_p),
                ("dbeta", C.c_void_p), ("ws", C.c_void_p), ("ws_floats", C.c_long), ("images", C.c_long),
                ("pixels", C.c_long), ("channels", C.c_int), ("groups", C.c_int), ("dtype", C.c_int),
                ("act", C.c_int)]


class TopLogitsArgs(C.Structure):
    _fields_ = [("z", C.c_void_p), ("ldz", C.c_long), ("rows", C.c_long), ("classes", C.c_int), ("k", C.c_int),
                ("dtype", C.c_int), ("temperature", C.c_float), ("values", C.c_void_p), ("index", C.c_void_p),
                ("rest", C.c_void_p), ("ws", C.c_void_p), ("ws_floats", C.c_long)]


class DistillArgs(C.Structure):
    _fields_ = [("z", C.c_void_p), ("dz", C.c_void_p), ("ldz", C.c_long), ("lddz", C.c_long), ("rows", C.c_long),
                ("classes", C.c_int), ("k", C.c_int), ("dtype", C.c_int), ("values", C.c_void_p),
                ("index", C.c_void_p), ("rest", C.c_void_p), ("labels", C.c_void_p), ("weight", C.c_void_p),
                ("loss", C.c_void_p), ("alpha", C.c_float), ("temperature", C.c_float), ("scale", C.c_float),
                ("ws", C.c_void_p), ("ws_floats", C.c_long)]


class ModelInfo(C.Structure):
    _fields_ = [("d", C.c_long), ("P", C.c_int), ("block_lo", C.c_long * 65), ("block_hi", C.c_long * 65),
                ("fwd_flops", C.c_double), ("bwd_flops", C.c_double * 65)]


def lib():
    global _LIB
    if _LIB is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError("liblpp.so is not built (run paper_2203_06638_amd/build.py); there is no fallback")
        L = C.CDLL(LIB_PATH)
        ctx = C.c_void_p
        fp = C.POINTER(C.c_float)
        sig = {
            "lpp_describe": ([C.POINTER(ModelDesc), C.c_int, C.POINTER(ModelInfo)], C.c_int),
            "lpp_init": ([C.POINTER(ModelDesc), C.c_int, C.c_int, C.POINTER(Options), C.POINTER(ctx)], C.c_int),
            "lpp_step": ([ctx, C.c_int, C.POINTER(Batch), C.c_int, C.c_float], C.c_int),
            "lpp_step_distill": ([ctx, C.c_int, C.POINTER(Batch), C.POINTER(Teacher), C.c_int, C.c_float], C.c_int),
            "lpp_top_logits": ([ctx, C.c_int, C.c_int, C.c_float, C.c_void_p, C.c_void_p, C.c_void_p], C.c_int),
            "lpp_average": ([ctx, C.POINTER(C.c_int), C.c_int], C.c_int),
            "lpp_set_params": ([ctx, C.c_int, fp, C.c_long], C.c_int),
            "lpp_get_params": ([ctx, C.c_int, fp, C.c_long], C.c_int),
            "lpp_get_grad": ([ctx, C.c_int, fp, C.c_long], C.c_int),
            "lpp_get_momentum": ([ctx, C.c_int, fp, C.c_long], C.c_int),
            "lpp_set_momentum": ([ctx, C.c_int, fp, C.c_long], C.c_int),
            "lpp_get_loss": ([ctx, C.c_int, fp], C.c_int),
            "lpp_get_logits": ([ctx, C.c_int, fp, C.c_long], C.c_int),
            "lpp_get_activation": ([ctx, C.c_int, C.c_int, fp, C.c_long], C.c_int),
            "lpp_get_activation_grad": ([ctx, C.c_int, C.c_int, fp, C.c_long], C.c_int),
            "lpp_num_params": ([ctx], C.c_long),
            "lpp_workspace_bytes": ([ctx], C.c_long),
            "lpp_block_range": ([ctx, C.c_int, C.POINTER(C.c_long), C.POINTER(C.c_long)], C.c_int),
            "lpp_counter": ([ctx, C.c_int], C.c_long),
            "lpp_sync": ([ctx], C.c_int),
            "lpp_destroy": ([ctx], C.c_int),
            "lpp_last_error": ([], C.c_char_p),
            "lpp_timer_enable": ([ctx, C.c_char_p], C.c_int),
            "lpp_timer_read": ([ctx, C.POINTER(C.c_double), C.POINTER(C.c_long), C.POINTER(C.c_double)], C.c_int),
            "lpp_trace_enable": ([ctx, C.c_long], C.c_int),
            "lpp_trace_read": ([ctx, C.POINTER(TraceStep), C.c_long, C.POINTER(C.c_long), C.POINTER(TraceAvg), C.c_long,
                                C.POINTER(C.c_long)], C.c_int),
            "lpp_trace_clock_khz": ([ctx], C.c_long),
            "lpp_kernel_sgd_update": ([C.c_void_p, C.c_void_p, C.c_void_p, C.c_long, C.c_float, C.c_float,
                                       C.c_float, C.c_void_p], C.c_int),
            "lpp_kernel_average": ([C.POINTER(C.c_void_p), C.c_int, C.c_long, C.c_void_p], C.c_int),
            "lpp_snapshot_plan_create": ([C.POINTER(SnapConv), C.c_int, C.c_long, C.c_int, C.c_long,
                                          C.POINTER(C.c_void_p)], C.c_int),
            "lpp_kernel_snapshot": ([C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p], C.c_int),
            "lpp_snapshot_plan_destroy": ([C.c_void_p], C.c_int),
            "lpp_kernel_snapshot_noalloc": ([C.POINTER(SnapConv), C.c_int, C.c_long, C.c_int, C.c_long, C.c_void_p,
                                             C.c_void_p, C.c_void_p, C.c_void_p], C.c_int),
            "lpp_act8_bytes": ([C.c_long, C.c_int], C.c_long),
            "lpp_kernel_act8_pack": ([C.c_void_p, C.c_int, C.c_long, C.c_int, C.c_long, C.c_int, C.c_void_p,
                                      C.c_void_p], C.c_int),
            "lpp_kernel_act8_unpack": ([C.c_void_p, C.c_long, C.c_int, C.c_void_p, C.c_int, C.c_long, C.c_void_p],
                                       C.c_int),
            "lpp_act8_wgrad_ws": ([C.c_long, C.c_int, C.c_int], C.c_long),
            "lpp_kernel_act8_wgrad": ([C.c_void_p, C.c_int, C.c_long, C.c_int, C.c_long, C.c_void_p, C.c_int,
                                       C.c_void_p, C.c_void_p, C.c_long, C.c_void_p], C.c_int),
            "lpp_kernel_rmsnorm": ([C.POINTER(RmsNormArgs), C.c_void_p], C.c_int),
            "lpp_rmsnorm_bwd_ws": ([C.c_long, C.c_int], C.c_long),
            "lpp_kernel_rmsnorm_bwd": ([C.POINTER(RmsNormBwdArgs), C.c_void_p], C.c_int),
            "lpp_groupnorm_ws": ([C.c_long, C.c_long, C.c_int, C.c_int], C.c_long),
            "lpp_kernel_groupnorm": ([C.POINTER(GroupNormArgs), C.c_void_p], C.c_int),
            "lpp_groupnorm_bwd_ws": ([C.c_long, C.c_long, C.c_int, C.c_int], C.c_long),
            "lpp_kernel_groupnorm_bwd": ([C.POINTER(GroupNormBwdArgs), C.c_void_p], C.c_int),
            "lpp_top_logits_ws": ([C.c_long, C.c_int, C.c_int], C.c_long),
            "lpp_kernel_top_logits": ([C.POINTER(TopLogitsArgs), C.c_void_p], C.c_int),
            "lpp_distill_ws": ([C.c_long, C.c_int], C.c_long),
            "lpp_kernel_distill": ([C.POINTER(DistillArgs), C.c_void_p], C.c_int),
        }
        for name, (args, res) in sig.items():
            f = getattr(L, name)
            f.argtypes = args
            f.restype = res
        _LIB = L
    return _LIB


def _check(rc):
    if rc != 0:
        raise LppError(rc, lib().lpp_last_error().decode())


def _fptr(a):
    return a.ctypes.data_as(C.POINTER(C.c_float))


def make_desc(model, batch, dtype=FP32, momentum=0.0, weight_decay=0.0, bn_eps=1e-5):
    """ModelDesc for a models.Model; the returned object keeps its layer
    array alive."""
    arr = (Layer * len(model.layers))(*[Layer(*rec) for rec in model.layers])
    c, h, w = model.in_shape
    desc = ModelDesc(len(model.layers), arr, c, h, w, model.n_classes, batch, dtype, momentum, weight_decay, bn_eps)
    desc._keep = arr
    return desc


def describe(model, batch=1, **kw):
    info = ModelInfo()
    desc = make_desc(model, batch, **kw)
    _check(lib().lpp_describe(C.byref(desc), model.P, C.byref(info)))
    return info


def _stream_handle(s):
    if s is None:
        return None
    return C.c_void_p(s.cuda_stream if hasattr(s, "cuda_stream") else int(s))


class Context:
    """One lpp_ctx: K replicas x P workers of `model` on the current device."""

    def __init__(self, model, K, batch, mode=SEQUENTIAL, dtype=FP32, momentum=0.0, weight_decay=0.0,
                 bn_eps=1e-5, streams=None, avg_stream=None, unfused=False, graphs=True, act8=False):
        """act8: activations are kept for the backward pass in 8 bits."""
        self.model = model
        self.K, self.P, self.batch = K, model.P, batch
        self._desc = make_desc(model, batch, dtype, momentum, weight_decay, bn_eps)
        opt = Options(mode | (ACT8 if act8 else 0), None, None, int(unfused), int(not graphs))
        if streams is not None:
            assert len(streams) == K * model.P
            self._streams = (C.c_void_p * len(streams))(*[_stream_handle(s).value for s in streams])
            opt.worker_streams = C.cast(self._streams, C.POINTER(C.c_void_p))
        if avg_stream is not None:
            opt.avg_stream = _stream_handle(avg_stream)
        self._ctx = C.c_void_p()
        _check(lib().lpp_init(C.byref(self._desc), K, model.P, C.byref(opt), C.byref(self._ctx)))
        self.d = int(lib().lpp_num_params(self._ctx))

    # -- the three calls of the method --
    def step(self, worker, images, labels, partition, lr):
        """images: device float32 NCHW tensor; labels: device int32 tensor."""
        b = Batch(images.data_ptr(), labels.data_ptr(), images.shape[0])
        _check(lib().lpp_step(self._ctx, worker, C.byref(b), partition, lr))

    def step_distill(self, worker, images, labels, values, index, partition, lr, rest=None, alpha=0.9, temperature=1.0):
        """A step whose loss is alpha parts distillation from a teacher's list (values,
        index [batch][k], rest [batch]: device tensors, see top_logits); labels None: from the
        list alone."""
        dev = _current_device(images)
        vp, ip, k = _list(values, index, self.batch, dev)
        rp = _floats(rest, self.batch, "rest", dev) if rest is not None else None
        lp = None if labels is None else _ints(labels, self.batch, "labels", dev)
        b = Batch(images.data_ptr(), lp, images.shape[0])
        t = Teacher(vp, ip, rp, k, alpha, temperature)
        _check(lib().lpp_step_distill(self._ctx, worker, C.byref(b), C.byref(t), partition, lr))

    def top_logits(self, worker, values, index, rest=None, temperature=1.0):
        """The k largest logits of each image of the worker's last step into values, index
        [batch][k], and the log weight of the others into rest [batch] (device tensors)."""
        dev = _current_device(values)
        vp, ip, k = _list(values, index, self.batch, dev)
        rp = _floats(rest, self.batch, "rest", dev) if rest is not None else None
        _check(lib().lpp_top_logits(self._ctx, worker, k, temperature, vp, ip, rp))

    def average(self, replicas=None):
        if replicas is None:
            _check(lib().lpp_average(self._ctx, None, 0))
        else:
            arr = (C.c_int * len(replicas))(*replicas)
            _check(lib().lpp_average(self._ctx, arr, len(replicas)))

    # -- accessors --
    def set_params(self, x, replica=-1):
        x = np.ascontiguousarray(x, np.float32)
        assert x.shape == (self.d,)
        _check(lib().lpp_set_params(self._ctx, replica, _fptr(x), self.d))

    def get_params(self, replica=0):
        out = np.empty(self.d, np.float32)
        _check(lib().lpp_get_params(self._ctx, replica, _fptr(out), self.d))
        return out

    def get_grad(self, worker):
        out = np.empty(self.d, np.float32)
        _check(lib().lpp_get_grad(self._ctx, worker, _fptr(out), self.d))
        return out

    def get_momentum(self, worker):
        out = np.empty(self.d, np.float32)
        _check(lib().lpp_get_momentum(self._ctx, worker, _fptr(out), self.d))
        return out

    def set_momentum(self, worker, m):
        m = np.ascontiguousarray(m, np.float32)
        _check(lib().lpp_set_momentum(self._ctx, worker, _fptr(m), self.d))

    def get_loss(self, worker):
        out = np.zeros(1, np.float32)
        _check(lib().lpp_get_loss(self._ctx, worker, _fptr(out)))
        return float(out[0])

    def get_logits(self, worker):
        out = np.empty((self.batch, self.model.n_classes), np.float32)
        _check(lib().lpp_get_logits(self._ctx, worker, _fptr(out), out.size))
        return out

    def get_activation(self, worker, layer, shape):
        out = np.empty((self.batch,) + tuple(shape), np.float32)
        _check(lib().lpp_get_activation(self._ctx, worker, layer, _fptr(out), out.size))
        return out

    def get_activation_grad(self, worker, layer, shape):
        out = np.empty((self.batch,) + tuple(shape), np.float32)
        _check(lib().lpp_get_activation_grad(self._ctx, worker, layer, _fptr(out), out.size))
        return out

    def block_range(self, i):
        lo, hi = C.c_long(), C.c_long()
        _check(lib().lpp_block_range(self._ctx, i, C.byref(lo), C.byref(hi)))
        return lo.value, hi.value

    def workspace_bytes(self):
        """Device memory of each worker."""
        return int(lib().lpp_workspace_bytes(self._ctx))

    def counter(self, replica):
        return int(lib().lpp_counter(self._ctx, replica))

    def sync(self):
        _check(lib().lpp_sync(self._ctx))

    def timer_enable(self, family):
        _check(lib().lpp_timer_enable(self._ctx, family.encode() if family else None))

    def timer_read(self):
        ms, n, work = C.c_double(), C.c_long(), C.c_double()
        _check(lib().lpp_timer_read(self._ctx, C.byref(ms), C.byref(n), C.byref(work)))
        return ms.value, n.value, work.value

    def trace_enable(self, capacity):
        _check(lib().lpp_trace_enable(self._ctx, capacity))

    def trace_read(self):
        """(steps, rounds, clock_khz): lists of dicts in issue order."""
        ns, na = C.c_long(), C.c_long()
        _check(lib().lpp_trace_read(self._ctx, None, 0, C.byref(ns), None, 0, C.byref(na)))
        st = (TraceStep * max(1, ns.value))()
        av = (TraceAvg * max(1, na.value))()
        _check(lib().lpp_trace_read(self._ctx, st, ns.value, C.byref(ns), av, na.value, C.byref(na)))
        steps = [dict(worker=r.worker, replica=r.replica, partition=r.partition, counter=r.counter, t=list(r.t))
                 for r in st[:ns.value]]
        rounds = [dict(index=r.index, n_replicas=r.n_replicas, counter_min=r.counter_min, t=list(r.t))
                  for r in av[:na.value]]
        return steps, rounds, int(lib().lpp_trace_clock_khz(self._ctx))

    def close(self):
        if self._ctx:
            _check(lib().lpp_destroy(self._ctx))
            self._ctx = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def __enter__(self):
        return self

    def __exit__(self, *a):
        self.close()


def kernel_sgd_update(x, m, g, lr, mu=0.0, wd=0.0, stream=None):
    """In-place block update on whole device tensors x, m (or None), g."""
    _check(lib().lpp_kernel_sgd_update(x.data_ptr(), m.data_ptr() if m is not None else None, g.data_ptr(),
                                       x.numel(), lr, mu, wd, _stream_handle(stream)))


def kernel_average(reps, stream=None):
    """In-place averaging round over a list of equally sized device tensors."""
    arr = (C.c_void_p * len(reps))(*[r.data_ptr() for r in reps])
    _check(lib().lpp_kernel_average(arr, len(reps), reps[0].numel(), _stream_handle(stream)))


def _snap_convs(convs):
    """host array of lpp_snap_conv from (src, cout, cin, cin_p, kh, kw, dst_f, dst_d) tuples"""
    return (SnapConv * max(1, len(convs)))(*[SnapConv(*c) for c in convs])


class SnapshotPlan:
    """lpp_snapshot_plan_create / lpp_kernel_snapshot / lpp_snapshot_plan_destroy.
    convs: (src, cout, cin, cin_p, kh, kw, dst_f, dst_d) tuples sorted by src."""

    def __init__(self, convs, d, dtype, wbuf_elems):
        arr = _snap_convs(convs)
        self._p = C.c_void_p()
        _check(lib().lpp_snapshot_plan_create(arr, len(convs), d, dtype, wbuf_elems, C.byref(self._p)))

    def run(self, x, v, wbuf, stream=None):
        """x, v: device float32 tensors of d floats; wbuf: device tensor of
        wbuf_elems float32 (FP32) or 16-bit (BF16) elements."""
        _check(lib().lpp_kernel_snapshot(self._p, x.data_ptr(), v.data_ptr(), wbuf.data_ptr(),
                                         _stream_handle(stream)))

    def close(self):
        if self._p:
            _check(lib().lpp_snapshot_plan_destroy(self._p))
            self._p = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def kernel_snapshot_noalloc(convs, d, dtype, wbuf_elems, x, v, wbuf, stream=None):
    """lpp_kernel_snapshot_noalloc on device tensors (see SnapshotPlan.run)."""
    arr = _snap_convs(convs)
    _check(lib().lpp_kernel_snapshot_noalloc(arr, len(convs), d, dtype, wbuf_elems, x.data_ptr(), v.data_ptr(),
                                             wbuf.data_ptr(), _stream_handle(stream)))


# -- 8-bit activation checkpoints, norms, top logits and distillation on device tensors (include/lpp.h) --
# Matrices are 2-D float32 or bfloat16 tensors on the current device whose rows are
# contiguous (any row distance); checkpoints are 1-D contiguous uint8 tensors of
# act8_bytes(rows, cols) bytes; gamma, rstd, gradients of parameters and
# workspaces are contiguous float32 tensors.  Buffers are checked and nothing
# is allocated; tensors used on a stream other than the one they were
# allocated on must outlive the call's work.  stream=None is the default (NULL)
# stream, as in every call here, not torch's current one: inside
# torch.cuda.stream(s), and to be captured, calls need stream=s.

_TORCH = None     # torch, on first use
_DTYPES = {}      # torch dtype: lpp dtype


def _current_device(t):
    """The current device; t, the first argument of a call, is a tensor on one."""
    global _TORCH
    if _TORCH is None:
        import torch
        _DTYPES.update({torch.float32: FP32, torch.bfloat16: BF16})
        _TORCH = torch
    if not isinstance(t, _TORCH.Tensor) or not t.is_cuda:
        raise LppError(EINVAL, "expected a tensor on the current device")
    return _TORCH.cuda.current_device()


def _matrix(t, what, dev, like=None):
    """(pointer, row distance, dtype, shape) of a 2-D tensor; like: the shape and dtype
    that it must have."""
    dt, s, st = _DTYPES.get(t.dtype), t.shape, t.stride()
    if dt is None or len(s) != 2 or t.get_device() != dev:
        raise LppError(EINVAL, what + " must be a 2-D float32 or bfloat16 tensor on the current device")
    rows, cols = s
    ld = st[0] if rows > 1 else cols
    if cols > 1 and st[1] != 1 or ld < cols or cols > 1 << 24:
        raise LppError(EINVAL, what + " must have contiguous rows, of at most 2^24 columns, that do not overlap")
    if like is not None and (s, dt) != like:
        raise LppError(EINVAL, what + " must have the other matrices' shape and type")
    return t.data_ptr(), ld, dt, s


def _floats(t, n, what, dev):
    if t.dtype != _TORCH.float32 or not t.is_contiguous() or t.numel() < n or t.get_device() != dev:
        raise LppError(EINVAL, "%s must be a contiguous float32 tensor of at least %d elements on the current device"
                       % (what, n))
    return t.data_ptr()


def _act8(q, rows, cols, dev):
    if q.dtype != _TORCH.uint8 or not q.is_contiguous() or q.numel() != act8_bytes(rows, cols) or q.get_device() != dev:
        raise LppError(EINVAL, "q must be a contiguous uint8 tensor of act8_bytes(rows, cols) elements on the current "
                               "device")
    return q.data_ptr()


def _need(ok, what):
    if not ok:
        raise LppError(EINVAL, what)


def act8_bytes(rows, cols):
    """Bytes of the 8-bit checkpoint of a [rows][cols] matrix."""
    n = lib().lpp_act8_bytes(rows, cols) if cols <= 1 << 24 else -1
    _need(n >= 0, "rows must be at least 0, cols at least 1, and the matrix under 2^40 elements")
    return n


def kernel_act8_pack(x, q, keep_sign=False, stream=None):
    """q = the 8-bit checkpoint of x (keep_sign: nonzero values stay nonzero)."""
    dev = _current_device(x)
    p, ld, dt, (rows, cols) = _matrix(x, "x", dev)
    _check(lib().lpp_kernel_act8_pack(p, dt, rows, cols, ld, int(keep_sign), _act8(q, rows, cols, dev),
                                      _stream_handle(stream)))


def kernel_act8_unpack(q, x, stream=None):
    """x = the values of checkpoint q."""
    dev = _current_device(x)
    p, ld, dt, (rows, cols) = _matrix(x, "x", dev)
    _check(lib().lpp_kernel_act8_unpack(_act8(q, rows, cols, dev), rows, cols, p, dt, ld, _stream_handle(stream)))


def act8_wgrad_ws(rows, cout, cin):
    """Floats of the workspace of kernel_act8_wgrad."""
    n = lib().lpp_act8_wgrad_ws(rows, cout, cin) if max(cout, cin) <= 1 << 24 else -1
    _need(n >= 0, "bad sizes")
    return n


def kernel_act8_wgrad(dy, q, dw, ws=None, stream=None):
    """dw [cout][cin] = dy^T X, dy [rows][cout], q the checkpoint of X [rows][cin];
    ws: act8_wgrad_ws(rows, cout, cin) floats (None where that is 0)."""
    dev = _current_device(dy)
    p, ld, dt, (rows, cout) = _matrix(dy, "dy", dev)
    _need(dw.dim() == 2 and dw.shape[0] == cout, "dw must be [cout][cin]")
    cin = dw.shape[1]
    wp, wn = (_floats(ws, 0, "ws", dev), ws.numel()) if ws is not None else (None, 0)
    _check(lib().lpp_kernel_act8_wgrad(p, dt, rows, cout, ld, _act8(q, rows, cin, dev), cin,
                                       _floats(dw, cout * cin, "dw", dev), wp, wn, _stream_handle(stream)))


def kernel_rmsnorm(x, gamma, rstd=None, eps=1e-5, res=None, h=None, y=None, q=None, keep_sign=False, stream=None):
    """RMS norm of x (+ res) over the columns into y and / or its checkpoint q;
    h: the sum x + res; rstd [rows]."""
    dev = _current_device(x)
    xp, ldx, dt, shape = _matrix(x, "x", dev)
    rows, cols = shape
    like = (shape, dt)
    rp = hp = yp = qp = sp = None
    ldr = ldh = ldy = 0
    if res is not None:
        rp, ldr = _matrix(res, "res", dev, like)[:2]
    if h is not None:
        hp, ldh = _matrix(h, "h", dev, like)[:2]
    if y is not None:
        yp, ldy = _matrix(y, "y", dev, like)[:2]
    if q is not None:
        qp = _act8(q, rows, cols, dev)
    if rstd is not None:
        sp = _floats(rstd, rows, "rstd", dev)
    a = RmsNormArgs(xp, rp, hp, yp, qp, ldx, ldr, ldh, ldy, _floats(gamma, cols, "gamma", dev), sp, rows, cols, dt, eps,
                    int(keep_sign))
    _check(lib().lpp_kernel_rmsnorm(C.byref(a), _stream_handle(stream)))


def rmsnorm_bwd_ws(rows, cols):
    """Floats of the workspace of kernel_rmsnorm_bwd."""
    n = lib().lpp_rmsnorm_bwd_ws(rows, cols) if cols <= 1 << 24 else -1
    _need(n >= 0, "bad sizes")
    return n


def kernel_rmsnorm_bwd(dy, gamma, rstd, dx=None, dgamma=None, ws=None, h=None, q=None, dres=None, stream=None):
    """Gradient of kernel_rmsnorm from its h (x where there was no residual) or from
    h's checkpoint q: dx (+ dres) and dgamma (with ws: rmsnorm_bwd_ws(rows, cols) floats)."""
    dev = _current_device(dy)
    yp, ldy, dt, shape = _matrix(dy, "dy", dev)
    rows, cols = shape
    like = (shape, dt)
    hp = qp = rp = xp = gp = wp = None
    ldh = ldr = ldx = wn = 0
    if h is not None:
        hp, ldh = _matrix(h, "h", dev, like)[:2]
    if q is not None:
        qp = _act8(q, rows, cols, dev)
    if dres is not None:
        rp, ldr = _matrix(dres, "dres", dev, like)[:2]
    if dx is not None:
        xp, ldx = _matrix(dx, "dx", dev, like)[:2]
    if dgamma is not None:
        gp = _floats(dgamma, cols, "dgamma", dev)
    if ws is not None:
        wp, wn = _floats(ws, 0, "ws", dev), ws.numel()
    a = RmsNormBwdArgs(yp, hp, qp, rp, xp, ldy, ldh, ldr, ldx, _floats(gamma, cols, "gamma", dev),
                       _floats(rstd, rows, "rstd", dev), gp, wp, wn, rows, cols, dt)
    _check(lib().lpp_kernel_rmsnorm_bwd(C.byref(a), _stream_handle(stream)))


def _groups(f, images, pixels, channels, groups):
    n = f(images, pixels, channels, groups) if max(channels, groups) <= 1 << 24 else -1
    _need(n >= 0, "images must be at least 0, pixels and channels at least 1, groups must divide channels, and the "
                  "matrix be under 2^40 elements")
    return n


def groupnorm_ws(images, pixels, channels, groups):
    """Floats of the workspace of kernel_groupnorm."""
    return _groups(lib().lpp_groupnorm_ws, images, pixels, channels, groups)


def groupnorm_bwd_ws(images, pixels, channels, groups):
    """Floats of the workspace of kernel_groupnorm_bwd."""
    return _groups(lib().lpp_groupnorm_bwd_ws, images, pixels, channels, groups)


def _pixels(rows, images, channels, groups):
    """Pixels of an image."""
    _need(images >= 0 and (rows % images == 0 and rows >= images if images else rows == 0),
          "the rows must be images * pixels")
    _need(1 <= groups <= channels and channels % groups == 0, "groups must divide the channels")
    return rows // images if images else 1


def kernel_groupnorm(x, images, groups, gamma, beta, y, mean=None, rstd=None, ws=None, eps=1e-5, act=ACT_NONE,
                     stream=None):
    """y = act(group norm of x): x [images * pixels][channels]; mean, rstd [images][groups];
    ws: groupnorm_ws(images, pixels, channels, groups) floats (None where that is 0)."""
    dev = _current_device(x)
    xp, ldx, dt, shape = _matrix(x, "x", dev)
    rows, ch = shape
    pixels = _pixels(rows, images, ch, groups)
    yp, ldy = _matrix(y, "y", dev, (shape, dt))[:2]
    mp = _floats(mean, images * groups, "mean", dev) if mean is not None else None
    rp = _floats(rstd, images * groups, "rstd", dev) if rstd is not None else None
    wp, wn = (_floats(ws, 0, "ws", dev), ws.numel()) if ws is not None else (None, 0)
    a = GroupNormArgs(xp, yp, ldx, ldy, _floats(gamma, ch, "gamma", dev), _floats(beta, ch, "beta", dev), mp, rp, wp, wn,
                      images, pixels, ch, groups, dt, act, eps)
    _check(lib().lpp_kernel_groupnorm(C.byref(a), _stream_handle(stream)))


def kernel_groupnorm_bwd(dy, x, images, groups, gamma, beta, mean, rstd, dx=None, dgamma=None, dbeta=None, ws=None,
                         dres=None, act=ACT_NONE, stream=None):
    """Gradient of kernel_groupnorm from its x, mean and rstd: dx (+ dres), dgamma and dbeta;
    ws: groupnorm_bwd_ws(images, pixels, channels, groups) floats (None where that is 0)."""
    dev = _current_device(dy)
    yp, ldy, dt, shape = _matrix(dy, "dy", dev)
    rows, ch = shape
    pixels = _pixels(rows, images, ch, groups)
    like = (shape, dt)
    xp, ldx = _matrix(x, "x", dev, like)[:2]
    ep = dp = gp = bp = wp = None
    lde = ldd = wn = 0
    if dres is not None:
        ep, lde = _matrix(dres, "dres", dev, like)[:2]
    if dx is not None:
        dp, ldd = _matrix(dx, "dx", dev, like)[:2]
    if dgamma is not None:
        gp = _floats(dgamma, ch, "dgamma", dev)
    if dbeta is not None:
        bp = _floats(dbeta, ch, "dbeta", dev)
    if ws is not None:
        wp, wn = _floats(ws, 0, "ws", dev), ws.numel()
    a = GroupNormBwdArgs(yp, xp, ep, dp, ldy, ldx, lde, ldd, _floats(gamma, ch, "gamma", dev),
                         _floats(beta, ch, "beta", dev), _floats(mean, images * groups, "mean", dev),
                         _floats(rstd, images * groups, "rstd", dev), gp, bp, wp, wn, images, pixels, ch, groups, dt, act)
    _check(lib().lpp_kernel_groupnorm_bwd(C.byref(a), _stream_handle(stream)))


def _ints(t, n, what, dev):
    if t.dtype != _TORCH.int32 or not t.is_contiguous() or t.numel() < n or t.get_device() != dev:
        raise LppError(EINVAL, "%s must be a contiguous int32 tensor of at least %d elements on the current device"
                       % (what, n))
    return t.data_ptr()


def _list(values, index, rows, dev):
    """(pointers, k) of a teacher's list."""
    _need(values.dim() == 2 and values.shape[0] == rows and index.shape == values.shape and values.shape[1] <= 1 << 24,
          "values and index must be [rows][k]")
    return _floats(values, 0, "values", dev), _ints(index, 0, "index", dev), values.shape[1]


def top_logits_ws(rows, classes, k):
    """Floats of the workspace of kernel_top_logits."""
    n = lib().lpp_top_logits_ws(rows, classes, k) if max(classes, k) <= 1 << 24 else -1
    _need(n >= 0, "rows must be at least 0, k in [1, min(classes, 128)], at most 2^24 classes, and the matrix under "
                  "2^40 elements")
    return n


def kernel_top_logits(z, values, index, rest=None, temperature=1.0, ws=None, stream=None):
    """The k largest logits of each row of z [rows][classes] into values and index
    [rows][k], and the log of the sum of exp(z / temperature) over the others into rest [rows];
    ws: top_logits_ws(rows, classes, k) floats (None where that is 0)."""
    dev = _current_device(z)
    p, ld, dt, (rows, classes) = _matrix(z, "z", dev)
    vp, ip, k = _list(values, index, rows, dev)
    rp = _floats(rest, rows, "rest", dev) if rest is not None else None
    wp, wn = (_floats(ws, 0, "ws", dev), ws.numel()) if ws is not None else (None, 0)
    a = TopLogitsArgs(p, ld, rows, classes, k, dt, temperature, vp, ip, rp, wp, wn)
    _check(lib().lpp_kernel_top_logits(C.byref(a), _stream_handle(stream)))


def distill_ws(rows, classes):
    """Floats of the workspace of kernel_distill."""
    n = lib().lpp_distill_ws(rows, classes) if classes <= 1 << 24 else -1
    _need(n >= 0, "rows must be at least 0, classes in [1, 2^24], and the matrix under 2^40 elements")
    return n


def kernel_distill(z, values, index, loss, dz=None, rest=None, labels=None, weight=None, alpha=1.0, temperature=1.0,
                   scale=1.0, ws=None, stream=None):
    """The loss [rows] of logits z [rows][classes] against a teacher's list values, index [rows][k]
    and rest [rows] (share alpha) and labels [rows], and dz = scale times its gradient;
    ws: distill_ws(rows, classes) floats (None where that is 0)."""
    dev = _current_device(z)
    p, ld, dt, shape = _matrix(z, "z", dev)
    rows, classes = shape
    vp, ip, k = _list(values, index, rows, dev)
    dp = ep = lp = hp = wp = None
    ldd = wn = 0
    if dz is not None:
        dp, ldd = _matrix(dz, "dz", dev, (shape, dt))[:2]
    if rest is not None:
        ep = _floats(rest, rows, "rest", dev)
    if labels is not None:
        lp = _ints(labels, rows, "labels", dev)
    if weight is not None:
        hp = _floats(weight, rows, "weight", dev)
    if ws is not None:
        wp, wn = _floats(ws, 0, "ws", dev), ws.numel()
    a = DistillArgs(p, dp, ld, ldd, rows, classes, k, dt, vp, ip, ep, lp, hp, _floats(loss, rows, "loss", dev), alpha,
                    temperature, scale, wp, wn)
    _check(lib().lpp_kernel_distill(C.byref(a), _stream_handle(stream)))
