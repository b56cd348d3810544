"""Thin ctypes binding over libmuxmatch.so: argument marshalling only.

Every step of the scheduling round runs inside the library's HIP kernels;
torch is used here for device buffers and the stream handle, nothing else.
There is no CPU fallback: if the shared library is missing, importing this
module raises.
"""
import ctypes as C
import os
import struct

import torch

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libmuxmatch.so")

INFEASIBLE = -2147483648
OK, ERR_ARG, ERR_SHAPE, ERR_HIP, ERR_NOT_CONVERGED, ERR_CERT, ERR_RANGE = 0, -1, -2, -3, -4, -5, -6
FALLBACK_TEAMS, FALLBACK_SEARCHES = 1, 2

EXPORTS = ["mf_create", "mf_destroy", "mf_score_pairs", "mf_solve_assignment",
           "mf_check_certificate", "mf_check_certificate_noalloc", "mf_schedule_round", "mf_schedule_round_update", "mf_score_pairs_typed",
           "mf_schedule_round_typed", "mf_set_option", "mf_last_timings", "mf_measure_ceilings",
           "mf_predictor_loss", "mf_predictor_loss_work", "mf_predict_pairs", "mf_layer_norm", "mf_layer_norm_grad",
           "mf_layer_norm_grad_work", "mf_dropout", "mf_strerror", "mf_last_hip_error"]

TIMING_NAMES = ["projections_ms", "pair_scoring_ms", "bulk_bid_ms", "bulk_bid_launches",
                "prepare_ms", "duals_ms", "certificate_ms", "auction_ms", "bulk_bid_bytes",
                "pairs_evaluated_fraction", "list_launches", "lists_made", "list_sides_left", "lists_by_column"]


class Predictor(C.Structure):
    _fields_ = [("F", C.c_int32), ("H", C.c_int32), ("scale", C.c_float),
                ("mem_feature", C.c_int32), ("mem_limit", C.c_float),
                ("d_W1", C.c_void_p), ("d_b1", C.c_void_p), ("d_W2", C.c_void_p),
                ("d_b2", C.c_void_p), ("d_W3", C.c_void_p), ("d_b3", C.c_void_p),
                ("d_W1sm", C.c_void_p), ("sm_on_feature", C.c_int32), ("sm_off_feature", C.c_int32),
                ("d_W3_slow", C.c_void_p), ("d_b3_slow", C.c_void_p), ("slow_limit", C.c_float),
                ("d_ln_w", C.c_void_p), ("d_ln_b", C.c_void_p), ("ln_eps", C.c_float)]


class DropoutRule(C.Structure):
    _fields_ = [("p", C.c_float), ("seed", C.c_uint64), ("step", C.c_uint64), ("d_step", C.c_void_p)]


class Samples(C.Structure):
    _fields_ = [("d_on", C.c_void_p), ("d_off", C.c_void_p), ("d_target", C.c_void_p), ("d_target_slow", C.c_void_p),
                ("count", C.c_int64)]


# members of mf_gradients, the names their parameters have in a predictor's dictionary, and their sizes: so many times F, H, 1, H * H and F * H
PARAMETERS = (("d_W1", "W1", (0, 0, 0, 0, 2)), ("d_b1", "b1", (0, 1, 0, 0, 0)), ("d_W2", "W2", (0, 0, 0, 1, 0)),
              ("d_b2", "b2", (0, 1, 0, 0, 0)), ("d_W3", "W3", (0, 1, 0, 0, 0)), ("d_b3", "b3", (0, 0, 1, 0, 0)),
              ("d_W1sm", "W1sm", (0, 1, 0, 0, 0)), ("d_W3_slow", "W3slow", (0, 1, 0, 0, 0)), ("d_b3_slow", "b3slow", (0, 0, 1, 0, 0)),
              ("d_ln_w", "ln_w", (2, 0, 0, 0, 0)), ("d_ln_b", "ln_b", (2, 0, 0, 0, 0)))


class Gradients(C.Structure):
    _fields_ = [(member, C.c_void_p) for member, _, _ in PARAMETERS]


# The same three as bytes, which take a third of the time to make.
DROPOUT_RULE, SAMPLES, GRADIENTS = struct.Struct("@fQQP"), struct.Struct("@PPPPq"), struct.Struct("@11P")
assert (DROPOUT_RULE.size, SAMPLES.size, GRADIENTS.size) == (C.sizeof(DropoutRule), C.sizeof(Samples), C.sizeof(Gradients))

LAYER_TYPES = {torch.float32: 0, torch.float16: 1, torch.bfloat16: 2}


class Result(C.Structure):
    _fields_ = [("primal", C.c_int64), ("dual", C.c_int64), ("K", C.c_int64),
                ("min_reduced_cost", C.c_int64), ("rounds", C.c_int64), ("bids", C.c_int64),
                ("bytes_scanned", C.c_int64), ("chain_bids", C.c_int64), ("chain_depth", C.c_int64),
                ("chain_retries", C.c_int64), ("team_bids", C.c_int64), ("path_steps", C.c_int64),
                ("path_scans", C.c_int64),
                ("matched", C.c_int32), ("phases", C.c_int32),
                ("cert_ok", C.c_int32), ("status", C.c_int32), ("ms_solve", C.c_float),
                ("ms_certify", C.c_float), ("fallbacks", C.c_int32)]

    def as_dict(self):
        return {k: getattr(self, k) for k, _ in self._fields_}


class Certificate(C.Structure):
    _fields_ = [("primal", C.c_int64), ("dual", C.c_int64), ("K", C.c_int64), ("min_reduced_cost", C.c_int64),
                ("matched", C.c_int32), ("flags", C.c_int32), ("cert_ok", C.c_int32), ("reserved", C.c_int32)]


NOALLOC_MAX_COLS = 65536


def load_library():
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is missing: build it with `python paper_2303_13803_amd/build.py` "
                          "(there is no CPU fallback)")
    lib = C.CDLL(LIB_PATH)
    vp, i32, i64 = C.c_void_p, C.c_int, C.c_int64
    lib.mf_create.argtypes = [C.POINTER(vp), i32, vp, i32, i32]
    lib.mf_destroy.argtypes = [vp]
    lib.mf_score_pairs.argtypes = [vp, C.POINTER(Predictor), vp, i32, vp, i32, vp, i64, vp]
    lib.mf_solve_assignment.argtypes = [vp, vp, i32, i32, i64, vp, vp, vp, C.POINTER(Result)]
    lib.mf_check_certificate.argtypes = [vp, vp, i32, i32, i64, vp, vp, vp, i64, C.POINTER(Result)]
    lib.mf_check_certificate_noalloc.argtypes = [vp, vp, i32, i32, i64, vp, vp, vp, i64, vp]
    lib.mf_schedule_round.argtypes = [vp, C.POINTER(Predictor), vp, i32, vp, i32, vp, i64, vp, vp, vp,
                                      C.POINTER(Result)]
    lib.mf_schedule_round_update.argtypes = [vp, C.POINTER(Predictor), vp, i32, vp, i32, vp, i32, vp, i32, vp, i64,
                                             vp, vp, vp, C.POINTER(Result)]
    lib.mf_score_pairs_typed.argtypes = [vp, C.POINTER(Predictor), i32, vp, vp, i32, vp, i32, vp, i64, vp]
    lib.mf_schedule_round_typed.argtypes = [vp, C.POINTER(Predictor), i32, vp, vp, i32, vp, i32, vp, i64, vp, vp, vp,
                                            C.POINTER(Result)]
    lib.mf_measure_ceilings.argtypes = [vp, vp, i64, C.POINTER(C.c_float * 8)]
    pred, f32 = C.POINTER(Predictor), C.c_float
    lib.mf_predictor_loss.argtypes = [vp, pred, vp, i32, vp, i32, vp, vp, f32,
                                      vp, vp, vp, vp, vp, i64]
    lib.mf_predictor_loss_work.argtypes = [vp, pred, i64]
    lib.mf_predict_pairs.argtypes = [vp, pred, vp, i32, vp, i32, vp, vp, i64, vp, vp]
    lib.mf_layer_norm.argtypes = [vp, i32, vp, i64, i64, i64, vp, vp, f32, vp, i64]
    lib.mf_layer_norm_grad.argtypes = [vp, i32, vp, i64, i64, i64, vp, i64, vp, f32, vp, i64, vp, vp, vp, i64]
    lib.mf_layer_norm_grad_work.argtypes = [vp, i64, i64]
    lib.mf_dropout.argtypes = [vp, i32, vp, i64, i64, i64, vp, i32, vp, i64]
    lib.mf_set_option.argtypes = [vp, C.c_char_p, i64]
    lib.mf_last_timings.argtypes = [vp, C.POINTER(C.c_float * 16)]
    lib.mf_strerror.argtypes = [i32]
    lib.mf_strerror.restype = C.c_char_p
    lib.mf_last_hip_error.argtypes = [vp]
    lib.mf_last_hip_error.restype = C.c_char_p
    for name in EXPORTS:
        if name not in ("mf_strerror", "mf_last_hip_error"):
            getattr(lib, name).restype = i64 if name.endswith("_work") else i32
    return lib


_lib = load_library()


class MuxmatchError(RuntimeError):
    def __init__(self, code, detail=""):
        self.code = code
        super().__init__(f"muxmatch error {code}: {_lib.mf_strerror(code).decode()} {detail}".strip())


def _ptr(t, dtype):
    if t is None:
        return None
    if not t.is_cuda or t.dtype != dtype or not t.is_contiguous():
        raise TypeError(f"expected a contiguous device tensor of {dtype}")
    return t.data_ptr()


class Context:
    """Owns the library's scratch for problems up to max_n x max_m on one device."""

    def __init__(self, max_n, max_m, device=0, stream=None):
        self.device = int(device)
        self.stream = stream if stream is not None else torch.cuda.current_stream(self.device)
        handle = C.c_void_p()
        rc = _lib.mf_create(C.byref(handle), self.device, C.c_void_p(self.stream.cuda_stream),
                            int(max_n), int(max_m))
        if rc != OK:
            raise MuxmatchError(rc)
        self._h = handle
        self._keep = None

    def close(self):
        if getattr(self, "_h", None):
            _lib.mf_destroy(self._h)
            self._h = None

    __del__ = close

    def _check(self, rc, allow=()):
        if rc != OK and rc not in allow:
            detail = _lib.mf_last_hip_error(self._h).decode() if rc == ERR_HIP else ""
            raise MuxmatchError(rc, detail)
        return rc

    # Calls of the layers and of fits may be two microseconds on the device, and every look at a tensor's attribute is a tenth of one or more: each is looked
    # at once, and what is wrong with a tensor is found out after it has been refused.
    def _flat(self, t, dtype, count, what):
        """Pointer of a contiguous tensor of `count` values on this context's device."""
        try:
            if t.dtype is dtype and t.get_device() == self.device and t.is_contiguous() and t.numel() == count:
                return t.data_ptr()
            fits = t.dtype == dtype and t.get_device() == self.device and t.is_contiguous()
        except AttributeError:
            fits = False
        if not fits:
            raise TypeError(f"{what}: expected a contiguous tensor of {dtype} on device {self.device}")
        raise ValueError(f"{what}: expected {count} values, got {t.numel()}")

    def _rows(self, t, kind, shape, what):
        """(pointer, pitch) of a matrix of this type and shape whose rows may lie apart but whose values lie side by side."""
        try:
            if t.get_device() != self.device:
                raise TypeError(f"{what}: expected a tensor on device {self.device}")
            if t.dtype is not kind or t.shape != shape:
                raise ValueError(f"{what}: expected a matrix of the input's shape and type")
        except AttributeError:
            raise TypeError(f"{what}: expected a tensor on device {self.device}") from None
        return t.data_ptr(), self._pitch(t, shape, what)

    def _pitch(self, t, shape, what):
        pitch, step = t.stride()
        rows, width = shape
        if rows < 2:
            pitch = max(width, 1)
        if (step != 1 and width > 1) or pitch < width:
            raise ValueError(f"{what}: the values of a row have to lie side by side, rows must not overlap")
        return pitch

    def _matrix(self, t, what):
        """Type, its number, shape, pointer and pitch of a matrix."""
        if not isinstance(t, torch.Tensor) or t.dtype not in LAYER_TYPES or t.dim() != 2:
            raise TypeError(f"{what}: expected a float32, float16 or bfloat16 matrix")
        if t.get_device() != self.device:
            raise TypeError(f"{what}: expected a tensor on device {self.device}")
        kind, shape = t.dtype, t.shape
        return kind, LAYER_TYPES[kind], shape, t.data_ptr(), self._pitch(t, shape, what)

    def _work(self, work, needed, *args):
        """The caller's scratch (the call itself looks at its size), or needed(*args) bytes from torch's allocator, in the order of this
        context's stream."""
        if work is None:
            size = needed(*args)
            with torch.cuda.stream(self.stream):
                return torch.empty(max(size, 16), dtype=torch.uint8, device=f"cuda:{self.device}")
        if not isinstance(work, torch.Tensor) or work.dtype != torch.uint8 or work.get_device() != self.device or not work.is_contiguous():
            raise TypeError(f"work: expected a contiguous tensor of torch.uint8 on device {self.device}")
        return work

    def _dropout(self, p, seed, step=0):
        """An mf_dropout_rule."""
        if isinstance(step, torch.Tensor):
            return DROPOUT_RULE.pack(float(p), int(seed) & (2 ** 64 - 1), 0, self._flat(step, torch.int64, 1, "step"))
        return DROPOUT_RULE.pack(float(p), int(seed) & (2 ** 64 - 1), int(step) & (2 ** 64 - 1), 0)

    def layer_norm(self, x, weight, bias, y, eps=1e-5):
        """y = layer norm of the rows of x (float32, float16 or bfloat16; weight and bias float32).  y may be x."""
        kind, number, shape, px, ldx = self._matrix(x, "x")
        py, ldy = self._rows(y, kind, shape, "y")
        rows, width = shape
        self._check(_lib.mf_layer_norm(self._h, number, px, rows, width, ldx,
                                       self._flat(weight, torch.float32, width, "weight"),
                                       self._flat(bias, torch.float32, width, "bias"), float(eps), py, ldy))

    def layer_norm_grad_work(self, rows, width):
        """Bytes of scratch layer_norm_grad needs."""
        needed = _lib.mf_layer_norm_grad_work(self._h, int(rows), int(width))
        if needed < 0:
            raise MuxmatchError(int(needed))
        return int(needed)

    def layer_norm_grad(self, x, dy, weight, dx, dweight, dbias, eps=1e-5, work=None):
        """dx, dweight and dbias of layer_norm from dy.  dx may be x or dy."""
        kind, number, shape, px, ldx = self._matrix(x, "x")
        pdy, lddy = self._rows(dy, kind, shape, "dy")
        pdx, lddx = self._rows(dx, kind, shape, "dx")
        rows, width = shape
        work = self._work(work, self.layer_norm_grad_work, rows, width)
        f32 = torch.float32
        self._check(_lib.mf_layer_norm_grad(self._h, number, px, rows, width, ldx, pdy, lddy,
                                            self._flat(weight, f32, width, "weight"), float(eps), pdx, lddx, self._flat(dweight, f32, width, "dweight"),
                                            self._flat(dbias, f32, width, "dbias"), work.data_ptr(), work.numel()))

    def dropout(self, x, y, p, seed, step=0, layer=0):
        """y = dropout of x, the mask made from (seed, step, layer, element); on a gradient, the backward pass.
        step: a number, or an int64 tensor of one value on the device.  y may be x."""
        if not 0 <= layer < 65536:                          # (would reach the library without its upper bits)
            raise MuxmatchError(ERR_ARG, "layer")
        kind, number, shape, px, ldx = self._matrix(x, "x")
        py, ldy = self._rows(y, kind, shape, "y")
        rows, width = shape
        self._check(_lib.mf_dropout(self._h, number, px, rows, width, ldx, self._dropout(p, seed, step), int(layer), py, ldy))

    def _side(self, x, F, what):
        """Pointer and rows of a side's features, [rows, F]."""
        shape = x.shape if isinstance(x, torch.Tensor) else ()
        if len(shape) != 2 or shape[1] != F:
            raise ValueError(f"{what}: expected a matrix of {F} features a workload")
        rows = shape[0]
        if rows > 0x7fffffff:                               # (would reach the library without its upper bits)
            raise ValueError(f"{what}: expected fewer than 2^31 workloads")
        return self._flat(x, torch.float32, rows * F, what), rows

    def predictor_loss_work(self, pred, count):
        """Bytes of scratch predictor_loss needs."""
        needed = _lib.mf_predictor_loss_work(self._h, C.byref(pred), int(count))
        if needed < 0:
            raise MuxmatchError(int(needed))
        return int(needed)

    def predictor_loss(self, pred, x_on, x_off, on, off, target, loss, grads=None, target_slow=None, dropout=None,
                       scale=None, sigma=None, sigma_slow=None, work=None):
        """loss[0] = scale * sum of squared errors of the predictions for the pairs (on[s], off[s]), and in `grads`, a
        dictionary of tensors shaped like the predictor's parameters, its gradients.  on, off: int32, out of range
        (-1) for samples that only fill the batch; target: float32, NaN where not measured.  dropout: (p, seed) or
        (p, seed, step).  scale: 1 / number of samples if not given."""
        count, F, H, flat, f32, i32 = on.numel() if isinstance(on, torch.Tensor) else 0, pred.F, pred.H, self._flat, torch.float32, torch.int32
        p_on, n = self._side(x_on, F, "x_on")
        p_off, m = self._side(x_off, F, "x_off")
        samples = SAMPLES.pack(flat(on, i32, count, "on"), flat(off, i32, count, "off"), flat(target, f32, count, "target"),
                               0 if target_slow is None else flat(target_slow, f32, count, "target_slow"), count)
        if grads is not None:
            grads = GRADIENTS.pack(*[0 if getattr(pred, member) is None else flat(grads[name], f32, columns * F + units * H + ones + squares * H * H + both * F * H, name)
                                     for member, name, (columns, units, ones, squares, both) in PARAMETERS])
        work = self._work(work, self.predictor_loss_work, pred, count)
        self._check(_lib.mf_predictor_loss(
            self._h, C.byref(pred), p_on, n, p_off, m, samples, None if dropout is None else self._dropout(*dropout),
            1.0 / max(count, 1) if scale is None else float(scale), grads, flat(loss, f32, 1, "loss"), None if sigma is None else flat(sigma, f32, count, "sigma"),
            None if sigma_slow is None else flat(sigma_slow, f32, count, "sigma_slow"), work.data_ptr(), work.numel()))

    def predict_pairs(self, pred, x_on, x_off, on, off, sigma, sigma_slow=None):
        """sigma[s] (and sigma_slow[s]) = what the predictor says of the pair (on[s], off[s])."""
        count, F = on.numel() if isinstance(on, torch.Tensor) else 0, pred.F
        p_on, n = self._side(x_on, F, "x_on")
        p_off, m = self._side(x_off, F, "x_off")
        self._check(_lib.mf_predict_pairs(
            self._h, C.byref(pred), p_on, n, p_off, m, self._flat(on, torch.int32, count, "on"), self._flat(off, torch.int32, count, "off"), count,
            self._flat(sigma, torch.float32, count, "sigma"), None if sigma_slow is None else self._flat(sigma_slow, torch.float32, count, "sigma_slow")))

    def predictor(self, params, scale, mem_feature=0, mem_limit=1.0, sm=None, slow_limit=None, norm_eps=None):
        """params: dict of float32 device tensors W1 [H,2F], b1, W2 [H,H], b2, W3 [H], b3 [1];
        with sm = (online feature, offline feature) also W1sm [H], the weights of the
        pair-dependent SM input; with slow_limit also W3slow [H], b3slow [1], the second output
        unit that predicts the online workload's slowdown (pairs above slow_limit are infeasible);
        with norm_eps also ln_w [2F], ln_b [2F], weight and bias of the layer norm of the features."""
        H = params["b1"].numel()
        F = params["W1"].shape[1] // 2
        there = {"d_W1sm": sm, "d_W3_slow": slow_limit, "d_b3_slow": slow_limit, "d_ln_w": norm_eps, "d_ln_b": norm_eps}
        p = Predictor(F, H, float(scale), int(mem_feature), float(mem_limit))
        for member, name, (columns, units, ones, squares, both) in PARAMETERS:
            if there.get(member, params) is not None:
                setattr(p, member, self._flat(params[name], torch.float32, columns * F + units * H + ones + squares * H * H + both * F * H, name))
        if sm is not None:
            p.sm_on_feature, p.sm_off_feature = int(sm[0]), int(sm[1])
        if slow_limit is not None:
            p.slow_limit = float(slow_limit)
        if norm_eps is not None:
            p.ln_eps = float(norm_eps)
        p._keep = params
        return p

    def set_option(self, name, value):
        self._check(_lib.mf_set_option(self._h, name.encode(), int(value)))

    def score_pairs(self, pred, x_on, x_off, W, sigma=None):
        n, m = x_on.shape[0], x_off.shape[0]
        self._check(_lib.mf_score_pairs(self._h, C.byref(pred), _ptr(x_on, torch.float32), n,
                                        _ptr(x_off, torch.float32), m, _ptr(W, torch.int32),
                                        W.stride(0), _ptr(sigma, torch.float32)))

    def solve_assignment(self, W, n, m, row2col, u, v, allow_cert_failure=False):
        res = Result()
        rc = _lib.mf_solve_assignment(self._h, _ptr(W, torch.int32), n, m, W.stride(0),
                                      _ptr(row2col, torch.int32), _ptr(u, torch.int64),
                                      _ptr(v, torch.int64), C.byref(res))
        self._check(rc, allow=(ERR_CERT,) if allow_cert_failure else ())
        return res

    def check_certificate(self, W, n, m, row2col, u, v, K):
        res = Result()
        self._check(_lib.mf_check_certificate(self._h, _ptr(W, torch.int32), n, m, W.stride(0),
                                              _ptr(row2col, torch.int32), _ptr(u, torch.int64),
                                              _ptr(v, torch.int64), int(K), C.byref(res)))
        return res

    def schedule_round(self, pred, x_on, x_off, W, row2col, u, v):
        n, m = x_on.shape[0], x_off.shape[0]
        res = Result()
        self._check(_lib.mf_schedule_round(self._h, C.byref(pred), _ptr(x_on, torch.float32), n,
                                           _ptr(x_off, torch.float32), m, _ptr(W, torch.int32),
                                           W.stride(0), _ptr(row2col, torch.int32),
                                           _ptr(u, torch.int64), _ptr(v, torch.int64), C.byref(res)))
        return res

    def schedule_round_update(self, pred, x_on, x_off, changed_on, changed_off, W, row2col, u, v):
        n, m = x_on.shape[0], x_off.shape[0]
        res = Result()
        self._check(_lib.mf_schedule_round_update(
            self._h, C.byref(pred), _ptr(x_on, torch.float32), n, _ptr(x_off, torch.float32), m,
            _ptr(changed_on, torch.int32) if changed_on is not None and changed_on.numel() else None,
            0 if changed_on is None else changed_on.numel(),
            _ptr(changed_off, torch.int32) if changed_off is not None and changed_off.numel() else None,
            0 if changed_off is None else changed_off.numel(),
            _ptr(W, torch.int32), W.stride(0), _ptr(row2col, torch.int32), _ptr(u, torch.int64),
            _ptr(v, torch.int64), C.byref(res)))
        return res

    def score_pairs_typed(self, preds, type_on, x_on, x_off, W, sigma=None):
        """preds: list of predictors, one per GPU type; type_on: int32 device tensor [n]."""
        n, m = x_on.shape[0], x_off.shape[0]
        arr = (Predictor * len(preds))(*preds)
        self._check(_lib.mf_score_pairs_typed(self._h, arr, len(preds), _ptr(type_on, torch.int32),
                                              _ptr(x_on, torch.float32), n, _ptr(x_off, torch.float32), m,
                                              _ptr(W, torch.int32), W.stride(0), _ptr(sigma, torch.float32)))

    def schedule_round_typed(self, preds, type_on, x_on, x_off, W, row2col, u, v):
        n, m = x_on.shape[0], x_off.shape[0]
        arr = (Predictor * len(preds))(*preds)
        res = Result()
        self._check(_lib.mf_schedule_round_typed(
            self._h, arr, len(preds), _ptr(type_on, torch.int32), _ptr(x_on, torch.float32), n,
            _ptr(x_off, torch.float32), m, _ptr(W, torch.int32), W.stride(0), _ptr(row2col, torch.int32),
            _ptr(u, torch.int64), _ptr(v, torch.int64), C.byref(res)))
        return res

    def measure_ceilings(self, buffer=None):
        """Measured fp32 and fp16 MFMA rates (TFLOP/s) and, with a device tensor, streaming read rate (GB/s)."""
        arr = (C.c_float * 8)()
        nbytes = 0 if buffer is None else buffer.numel() * buffer.element_size()
        self._check(_lib.mf_measure_ceilings(self._h, None if buffer is None else buffer.data_ptr(), nbytes,
                                             C.byref(arr)))
        return {"mfma_f32_tflops": float(arr[0]), "read_gbps": float(arr[2]), "mfma_f16_tflops": float(arr[4])}

    def last_timings(self):
        arr = (C.c_float * 16)()
        self._check(_lib.mf_last_timings(self._h, C.byref(arr)))
        return {name: float(arr[i]) for i, name in enumerate(TIMING_NAMES)}


def check_certificate_noalloc(W, n, m, row2col, u, v, K, out, stream=None):
    """mf_check_certificate_noalloc on the current device: `out` is a uint8 device tensor of
    ctypes.sizeof(Certificate) bytes that receives the result once `stream` gets there
    (read it with read_certificate after synchronising).  Returns the call's status code."""
    if not out.is_cuda or out.dtype != torch.uint8 or out.numel() < C.sizeof(Certificate) or not out.is_contiguous():
        raise TypeError("out: a contiguous uint8 device tensor of at least sizeof(Certificate) bytes")
    s = stream if stream is not None else torch.cuda.current_stream()
    return _lib.mf_check_certificate_noalloc(C.c_void_p(s.cuda_stream), _ptr(W, torch.int32), int(n), int(m),
                                             W.stride(0), _ptr(row2col, torch.int32), _ptr(u, torch.int64),
                                             _ptr(v, torch.int64), int(K), out.data_ptr())


def read_certificate(out):
    """The Certificate a finished mf_check_certificate_noalloc left in `out` (copies it to the host)."""
    return Certificate.from_buffer_copy(out.cpu().numpy().tobytes()[:C.sizeof(Certificate)])


def strerror(code):
    return _lib.mf_strerror(int(code)).decode()


def raw_library():
    return _lib
