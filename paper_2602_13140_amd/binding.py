"""Thin ctypes binding over libqsv.so with the C ABI's names.

Argument marshalling only: every step of the path runs in the HIP kernels.  torch is used for
device memory and the current stream; there is no CPU fallback, and a missing library is an
error, not a reason to compute elsewhere.
"""
import ctypes
import os

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libqsv.so")

QSV_OK, QSV_ERR_INVALID_ARG, QSV_ERR_UNSUPPORTED, QSV_ERR_ZERO_NORM, QSV_ERR_WORKSPACE, QSV_ERR_HIP = range(6)
QSV_RX, QSV_RY, QSV_RZ = 1, 2, 3
QSV_ENT_NONE, QSV_ENT_CNOT_RING, QSV_ENT_CZ_LADDER = 0, 1, 2
(QSV_M_PROBS, QSV_M_EXPZ_ALL, QSV_M_EXPZ_ONE, QSV_M_MARGINAL, QSV_M_PROJECT_ZERO, QSV_M_FIDELITY,
 QSV_M_SAMPLE) = range(1, 8)


class qsv_circuit(ctypes.Structure):
    _fields_ = [("n_layers", ctypes.c_int32), ("reupload", ctypes.c_int32),
                ("n_rot", ctypes.c_int32), ("rot", ctypes.c_int32 * 3),
                ("entangler", ctypes.c_int32)]


class qsv_measure_req(ctypes.Structure):
    _fields_ = [("kind", ctypes.c_int32), ("qubit", ctypes.c_int32), ("mask", ctypes.c_uint64),
                ("renormalise", ctypes.c_int32), ("reserved", ctypes.c_int32),
                ("x_dev", ctypes.c_void_p), ("dim", ctypes.c_int64),
                ("uniforms_dev", ctypes.c_void_p), ("shots", ctypes.c_int64),
                ("out_dev", ctypes.c_void_p)]


class qsv_loss(ctypes.Structure):
    _fields_ = [("kind", ctypes.c_int32), ("reserved", ctypes.c_int32), ("mask", ctypes.c_uint64),
                ("targets_dev", ctypes.c_void_p)]


QSV_LOSS_TRASH, QSV_LOSS_MSE_Z = 1, 2
QSV_S_F32, QSV_S_F16, QSV_S_BF16, QSV_S_PROBS, QSV_S_STATE = range(1, 6)


class qsv_sample_req(ctypes.Structure):
    _fields_ = [("kind", ctypes.c_int32), ("reserved", ctypes.c_int32), ("scores_dev", ctypes.c_void_p),
                ("rows", ctypes.c_int64), ("cols", ctypes.c_int64), ("row_stride", ctypes.c_int64),
                ("temperature_dev", ctypes.c_void_p), ("top_k_dev", ctypes.c_void_p),
                ("top_p_dev", ctypes.c_void_p), ("min_p_dev", ctypes.c_void_p),
                ("uniforms_dev", ctypes.c_void_p), ("shots", ctypes.c_int64), ("out_dev", ctypes.c_void_p),
                ("logp_dev", ctypes.c_void_p), ("kept_dev", ctypes.c_void_p)]


class qsv_teacher(ctypes.Structure):
    _fields_ = [("n_top", ctypes.c_int32), ("reserved", ctypes.c_int32), ("top_idx_dev", ctypes.c_void_p),
                ("top_logits_dev", ctypes.c_void_p), ("top_lse_dev", ctypes.c_void_p), ("temperature", ctypes.c_double)]


class qsv_distill_req(ctypes.Structure):
    _fields_ = [("kind", ctypes.c_int32), ("have_stats", ctypes.c_int32), ("scores_dev", ctypes.c_void_p),
                ("rows", ctypes.c_int64), ("cols", ctypes.c_int64), ("row_stride", ctypes.c_int64),
                ("loss_dev", ctypes.c_void_p), ("stats_dev", ctypes.c_void_p), ("grad_loss_dev", ctypes.c_void_p),
                ("grad_dev", ctypes.c_void_p), ("grad_stride", ctypes.c_int64)]


class qsv_adjust_req(ctypes.Structure):
    _fields_ = [("kind", ctypes.c_int32), ("n_entries", ctypes.c_int32), ("scores_dev", ctypes.c_void_p),
                ("rows", ctypes.c_int64), ("cols", ctypes.c_int64), ("row_stride", ctypes.c_int64),
                ("out_dev", ctypes.c_void_p), ("out_stride", ctypes.c_int64),
                ("prior_dev", ctypes.c_void_p), ("n_prior", ctypes.c_int64), ("prior_stride", ctypes.c_int64),
                ("prior_len_dev", ctypes.c_void_p), ("prompt_len_dev", ctypes.c_void_p),
                ("repetition_dev", ctypes.c_void_p), ("frequency_dev", ctypes.c_void_p), ("presence_dev", ctypes.c_void_p),
                ("bias_dev", ctypes.c_void_p), ("entry_idx_dev", ctypes.c_void_p), ("entry_bias_dev", ctypes.c_void_p),
                ("masks_dev", ctypes.c_void_p), ("n_masks", ctypes.c_int64), ("mask_stride", ctypes.c_int64),
                ("mask_of_dev", ctypes.c_void_p)]


class qsv_adjust_grad_req(ctypes.Structure):
    _fields_ = [("grad_out_dev", ctypes.c_void_p), ("grad_out_stride", ctypes.c_int64), ("grad_dev", ctypes.c_void_p),
                ("grad_stride", ctypes.c_int64), ("grad_bias_dev", ctypes.c_void_p), ("grad_entry_dev", ctypes.c_void_p)]


class qsv_tensor(ctypes.Structure):
    _fields_ = [("kind", ctypes.c_int32), ("reserved", ctypes.c_int32), ("data_dev", ctypes.c_void_p),
                ("rows", ctypes.c_int64), ("cols", ctypes.c_int64), ("row_stride", ctypes.c_int64)]


class qsv_adam_tensor(ctypes.Structure):
    _fields_ = [("kind", ctypes.c_int32), ("reserved", ctypes.c_int32), ("param_dev", ctypes.c_void_p),
                ("grad_dev", ctypes.c_void_p), ("m_dev", ctypes.c_void_p), ("v_dev", ctypes.c_void_p), ("count", ctypes.c_int64)]


class QsvError(RuntimeError):
    def __init__(self, status, message):
        super().__init__("qsv status %d: %s" % (status, message))
        self.status = status


_lib = None


def load():
    """Loads libqsv.so (built in-tree by build.py).  Raises if it is missing."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise FileNotFoundError(
            "%s not found: build it with `python -m paper_2602_13140_amd.build` "
            "(there is no fallback path)" % LIB_PATH)
    import torch  # noqa: F401  (first: the library then takes the HIP runtime that torch brings; with one of its own it finds no device)
    L = ctypes.CDLL(LIB_PATH)
    vp, i32, i64 = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64
    L.qsv_num_params.restype = i64
    L.qsv_num_params.argtypes = [ctypes.POINTER(qsv_circuit), i32]
    L.qsv_workspace_bytes.restype = ctypes.c_size_t
    L.qsv_workspace_bytes.argtypes = [i32, i32]
    L.qsv_grad_workspace_bytes.restype = ctypes.c_size_t
    L.qsv_grad_workspace_bytes.argtypes = [i32, i32, ctypes.POINTER(qsv_circuit)]
    L.qsv_create.restype = i32
    L.qsv_create.argtypes = [ctypes.POINTER(vp), i32, i32, i32, vp, vp, vp, ctypes.c_size_t]
    L.qsv_destroy.restype = None
    L.qsv_destroy.argtypes = [vp]
    L.qsv_last_error.restype = ctypes.c_char_p
    L.qsv_last_error.argtypes = [vp]
    L.qsv_amp_encode.restype = i32
    L.qsv_amp_encode.argtypes = [vp, vp, i64, vp]
    L.qsv_apply_layers.restype = i32
    L.qsv_apply_layers.argtypes = [vp, ctypes.POINTER(qsv_circuit), vp, vp, i32]
    L.qsv_measure.restype = i32
    L.qsv_measure.argtypes = [vp, ctypes.POINTER(qsv_measure_req)]
    L.qsv_forward_small.restype = i32
    L.qsv_forward_small.argtypes = [vp, vp, i64, ctypes.POINTER(qsv_circuit), vp, vp, i32, i32, vp, vp]
    L.qsv_measure_static.restype = i32
    L.qsv_measure_static.argtypes = [vp, ctypes.POINTER(qsv_measure_req)]
    L.qsv_param_shift_grad.restype = i32
    L.qsv_param_shift_grad.argtypes = [vp, ctypes.POINTER(qsv_circuit), vp, i64, vp, vp, ctypes.c_int32,
                                       vp, vp, vp, vp]
    L.qsv_adjoint_grad.restype = i32
    L.qsv_adjoint_grad.argtypes = [vp, ctypes.POINTER(qsv_circuit), vp, i64, vp, vp, ctypes.c_int32,
                                       vp, vp, vp, vp]
    L.qsv_loss_grad.restype = i32
    L.qsv_loss_grad.argtypes = [vp, ctypes.POINTER(qsv_circuit), vp, i64, vp, vp, ctypes.POINTER(qsv_loss),
                                vp, vp, vp, vp]
    L.qsv_sgd_step.restype = i32
    L.qsv_sgd_step.argtypes = [vp, vp, vp, i64, ctypes.c_double]
    L.qsv_adam_step.restype = i32
    L.qsv_adam_step.argtypes = [vp, vp, vp, vp, vp, i64, i64, ctypes.c_double, ctypes.c_double,
                                ctypes.c_double, ctypes.c_double]
    L.qsv_reset_fidelity.restype = i32
    L.qsv_reset_fidelity.argtypes = [vp, ctypes.POINTER(qsv_circuit), vp, vp, ctypes.c_uint64, vp, i64, vp]
    L.qsv_shot_expz.restype = i32
    L.qsv_shot_expz.argtypes = [vp, vp, i64, vp]
    L.qsv_distill_workspace_bytes.restype = ctypes.c_size_t
    L.qsv_distill_workspace_bytes.argtypes = [i64, i64]
    L.qsv_distill.restype = i32
    L.qsv_distill.argtypes = [vp, ctypes.POINTER(qsv_distill_req), ctypes.POINTER(qsv_teacher)]
    L.qsv_distill_grad_workspace_bytes.restype = ctypes.c_size_t
    L.qsv_distill_grad_workspace_bytes.argtypes = [i32, i32, ctypes.POINTER(qsv_circuit)]
    L.qsv_distill_grad.restype = i32
    L.qsv_distill_grad.argtypes = [vp, ctypes.POINTER(qsv_circuit), vp, i64, vp, vp, ctypes.POINTER(qsv_teacher),
                                   vp, vp, vp, vp]
    L.qsv_sample_workspace_bytes.restype = ctypes.c_size_t
    L.qsv_sample_workspace_bytes.argtypes = [i64, i64]
    L.qsv_sample.restype = i32
    L.qsv_sample.argtypes = [vp, ctypes.POINTER(qsv_sample_req)]
    L.qsv_adjust.restype = i32
    L.qsv_adjust.argtypes = [vp, ctypes.POINTER(qsv_adjust_req)]
    L.qsv_adjust_grad_workspace_bytes.restype = ctypes.c_size_t
    L.qsv_adjust_grad_workspace_bytes.argtypes = [i64, i64]
    L.qsv_adjust_grad.restype = i32
    L.qsv_adjust_grad.argtypes = [vp, ctypes.POINTER(qsv_adjust_req), ctypes.POINTER(qsv_adjust_grad_req)]
    L.qsv_clip_grads.restype = i32
    L.qsv_clip_grads.argtypes = [vp, vp, vp, i64, ctypes.c_double, vp]
    L.qsv_adam_clipped.restype = i32
    L.qsv_adam_clipped.argtypes = [vp, vp, i64, i64, ctypes.c_double, ctypes.c_double, ctypes.c_double, ctypes.c_double,
                                   ctypes.c_double, vp]
    L.qsv_pauli_expect.restype = i32
    L.qsv_pauli_expect.argtypes = [vp, ctypes.c_uint64, ctypes.c_uint64, ctypes.c_uint64, vp]
    L.qsv_plan_describe.restype = i64
    L.qsv_plan_describe.argtypes = [ctypes.POINTER(qsv_circuit), i32, i32, i32, i32, ctypes.c_char_p, i64]
    L.qsv_probe_pass.restype = i32
    L.qsv_probe_pass.argtypes = [vp, i32, i32, i32]
    L.qsv_set_option.restype = i32
    L.qsv_set_option.argtypes = [vp, ctypes.c_char_p, i64]
    _lib = L
    return L


def make_circuit(n_layers, rot, entangler, reupload=0):
    c = qsv_circuit()
    c.n_layers = int(n_layers)
    c.reupload = int(reupload)
    c.n_rot = len(rot)
    for i, r in enumerate(rot):
        c.rot[i] = int(r)
    c.entangler = int(entangler)
    return c


def circuit_from_spec(spec):
    """spec: workloads.CircuitSpec."""
    return make_circuit(spec.n_layers, spec.rot, spec.entangler, spec.reupload)


def qsv_num_params(circ, n):
    return int(load().qsv_num_params(ctypes.byref(circ), n))


def qsv_workspace_bytes(n, batch):
    return int(load().qsv_workspace_bytes(n, batch))


def qsv_grad_workspace_bytes(n, batch, circ):
    return int(load().qsv_grad_workspace_bytes(n, batch, ctypes.byref(circ)))


def qsv_sample_workspace_bytes(rows, cols):
    return int(load().qsv_sample_workspace_bytes(rows, cols))


def qsv_distill_workspace_bytes(rows, cols):
    return int(load().qsv_distill_workspace_bytes(rows, cols))


def qsv_distill_grad_workspace_bytes(n, batch, circ):
    return int(load().qsv_distill_grad_workspace_bytes(n, batch, ctypes.byref(circ)))


def qsv_adjust_grad_workspace_bytes(rows, cols):
    return int(load().qsv_adjust_grad_workspace_bytes(rows, cols))


def qsv_plan_describe(circ, n, batch=1, inverse=0, tile_log2=0):
    L = load()
    need = L.qsv_plan_describe(ctypes.byref(circ), n, batch, inverse, tile_log2, None, 0)
    if need < 0:
        raise ValueError("bad circuit descriptor")
    buf = ctypes.create_string_buffer(need + 1)
    L.qsv_plan_describe(ctypes.byref(circ), n, batch, inverse, tile_log2, buf, need + 1)
    return buf.value.decode()


def _ptr(t):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


_TYPE_OF = {QSV_S_F32: "float32", QSV_S_F16: "float16", QSV_S_BF16: "bfloat16", QSV_S_PROBS: "float32"}
_dtypes = {}


def _dtype(name):
    if not _dtypes:
        import torch
        _dtypes.update((n, getattr(torch, n)) for n in ("float16", "bfloat16", "float32", "float64", "int32", "int64"))
    return _dtypes[name]


def _need(ok, what):
    if not ok:
        raise QsvError(QSV_ERR_INVALID_ARG, what)


def _rows(t, kind, dev, what):
    """Rows of scores: [rows][cols] of the kind's type, values of a row next to each other, any row stride."""
    _need(kind in _TYPE_OF, "unknown kind of scores")
    if not (t is not None and t.get_device() == dev and t.dim() == 2 and t.dtype is _dtype(_TYPE_OF[kind])
            and (t.shape[1] == 1 or t.stride(1) == 1)):
        _need(False, "%s must be rows of %s on cuda:%d, the values of a row next to each other" % (what, _TYPE_OF[kind], dev))
    return t


def _flat(t, dtype, dev, what, *shape):
    """The address of a contiguous tensor of this type and shape; None stays None."""
    if t is None:
        return None
    if not (t.dtype is _dtype(dtype) and t.get_device() == dev and t.is_contiguous() and t.shape == shape):
        _need(False, "%s must be a contiguous tensor of %s %s on cuda:%d" % (what, dtype, list(shape), dev))
    return t.data_ptr()


def _room(t, dtype, dev, what, count):
    """The address of a contiguous tensor of this type, of `count` values or more; None stays None."""
    if t is None:
        return None
    if not (t.dtype is _dtype(dtype) and t.get_device() == dev and t.is_contiguous() and t.numel() >= count):
        _need(False, "%s must be a contiguous tensor of %d values of %s on cuda:%d" % (what, count, dtype, dev))
    return t.data_ptr()


def _teacher(rows, top_idx, top_logits, temperature, top_lse, dev):
    _need(top_idx is not None and top_idx.dim() == 2, "top_idx must be [rows][n_top]")
    top = top_idx.shape[1]
    return qsv_teacher(top, 0, _flat(top_idx, "int32", dev, "top_idx", rows, top),
                       _flat(top_logits, "float32", dev, "top_logits", rows, top),
                       _flat(top_lse, "float32", dev, "top_lse", rows), float(temperature))


def _grid(t, dtype, dev, what):
    """(address, rows, columns, row stride) of rows whose values lie next to each other."""
    shape, stride = t.shape, t.stride()
    if not (t.dtype is dtype and t.get_device() == dev and len(shape) == 2 and (stride[1] == 1 or shape[1] < 2)):
        _need(False, "%s must be rows of %s on cuda:%d, the values of a row next to each other" % (what, str(dtype)[6:], dev))
    return t.data_ptr(), shape[0], shape[1], stride[0]


def _each(t, dtype, dev, shape, what):
    if t.dtype is dtype and t.get_device() == dev and t.shape == shape and t.is_contiguous():
        return t.data_ptr()
    _need(False, "%s must be a contiguous tensor of %s %s on cuda:%d" % (what, str(dtype)[6:], list(shape), dev))


def _score_type(kind):
    if kind not in (QSV_S_F32, QSV_S_F16, QSV_S_BF16):
        _need(False, "kind must be one of the three types of scores")
    return _dtype(_TYPE_OF[kind])


def _adjustment(r, d, rows, prior, prior_len, prompt_len, repetition, frequency, presence, entry_idx, masks, mask_of):
    """The part of a request that qsv_adjust and its backward pass share; rows of whole numbers may lie further apart."""
    i32, f32, each = _dtype("int32"), _dtype("float32"), (rows,)
    if prior is not None:
        r.prior_dev, n, r.n_prior, r.prior_stride = _grid(prior, i32, d, "prior")
        if n != rows:
            _need(False, "prior must have the scores' rows")
    if entry_idx is not None:
        if entry_idx.dim() != 2:
            _need(False, "entry_idx must be [rows][n_entries]")
        r.n_entries = n = entry_idx.shape[1]
        r.entry_idx_dev = _each(entry_idx, i32, d, (rows, n), "entry_idx")
    if masks is not None:
        r.masks_dev, r.n_masks, words, r.mask_stride = _grid(masks, i32, d, "masks")
        if words < (r.cols + 31) // 32:
            _need(False, "masks must have a bit for each outcome")
    elif mask_of is not None:
        _need(False, "mask_of without masks")
    if prior_len is not None:
        r.prior_len_dev = _each(prior_len, i32, d, each, "prior_len")
    if prompt_len is not None:
        r.prompt_len_dev = _each(prompt_len, i32, d, each, "prompt_len")
    if repetition is not None:
        r.repetition_dev = _each(repetition, f32, d, each, "repetition")
    if frequency is not None:
        r.frequency_dev = _each(frequency, f32, d, each, "frequency")
    if presence is not None:
        r.presence_dev = _each(presence, f32, d, each, "presence")
    if mask_of is not None:
        r.mask_of_dev = _each(mask_of, i32, d, each, "mask_of")


def _kinds():
    """The kinds of scores by their types."""
    return {_dtype(_TYPE_OF[kind]): kind for kind in (QSV_S_F32, QSV_S_F16, QSV_S_BF16)}


class TensorList:
    """Tensors as qsv_clip_grads takes them, laid out once: contiguous ones of any shape, or rows (of two dimensions) further apart.
    Holds their memory as it is now: a tensor that is given other memory later (t.data = ..., gradients that are allocated anew) needs
    another list, which takes about 0.6 us a tensor."""

    def __init__(self, tensors):
        tensors, kinds = list(tensors), _kinds()
        self.at = (qsv_tensor * max(1, len(tensors)))()
        for e, t in zip(self.at, tensors):
            shape = t.shape
            rows, cols = shape if len(shape) == 2 else (1, t.numel())
            step = cols
            if not t.is_contiguous():
                if len(shape) != 2 or not ((cols < 2 or t.stride(1) == 1) and (rows < 2 or t.stride(0) >= cols)):
                    _need(False, "tensors must be contiguous, or rows whose values lie next to each other")
                step = t.stride(0)
            kind = kinds.get(t.dtype)
            if kind is None:
                _need(False, "tensors must be float32, float16 or bfloat16")
            e.kind, e.data_dev, e.rows, e.cols, e.row_stride = kind, t.data_ptr() or None, rows, cols, step
        self.held = [t.untyped_storage() for t in tensors]
        self.devices = {t.get_device() for t in tensors}

    def __len__(self):
        return len(self.held)


class AdamList:
    """Parameters, gradients and moments as qsv_adam_clipped takes them, laid out once (about 1.5 us a parameter).  Holds their memory as
    it is now, as TensorList."""

    def __init__(self, params, grads, m, v):
        lists = [list(x) for x in (params, grads, m, v)]
        self.n = n = len(lists[0])
        _need(all(len(x) == n for x in lists), "params, grads, m and v must be as many")
        kinds, f32 = _kinds(), _dtype("float32")
        self.at = (qsv_adam_tensor * max(1, n))()
        for e, p, g, a, b in zip(self.at, *lists):
            if not (p.dtype is f32 and a.dtype is f32 and b.dtype is f32):
                _need(False, "params, m and v must be float32")
            shape = p.shape
            if not (p.is_contiguous() and g.is_contiguous() and a.is_contiguous() and b.is_contiguous()
                    and g.shape == shape and a.shape == shape and b.shape == shape):
                _need(False, "params, grads, m and v must be contiguous, of one shape")
            kind = kinds.get(g.dtype)
            if kind is None:
                _need(False, "tensors must be float32, float16 or bfloat16")
            e.kind, e.count = kind, p.numel()
            e.param_dev, e.grad_dev, e.m_dev, e.v_dev = p.data_ptr() or None, g.data_ptr() or None, a.data_ptr() or None, b.data_ptr() or None
        self.held = [t.untyped_storage() for x in lists for t in x]
        self.devices = {t.get_device() for x in lists for t in x}

    def __len__(self):
        return self.n


class Context:
    """Owns a qsv_ctx plus the torch tensors that back its state and workspace."""

    def __init__(self, n, batch, device=0, ws_bytes=None):
        import torch
        if not torch.cuda.is_available():
            raise RuntimeError("qsv needs a GPU: torch.cuda.is_available() is False")
        self.L = load()
        self.n, self.batch = n, batch
        self.dev = torch.device("cuda", device)
        self.state = torch.zeros((batch, 1 << n, 2), dtype=torch.float32, device=self.dev)
        need = qsv_workspace_bytes(n, batch)
        ws_bytes = need if ws_bytes is None else ws_bytes
        self.ws = torch.empty(ws_bytes + 256, dtype=torch.uint8, device=self.dev)
        off = (-self.ws.data_ptr()) % 256
        self.stream = torch.cuda.current_stream(self.dev)
        h = ctypes.c_void_p()
        st = self.L.qsv_create(ctypes.byref(h), n, batch, device,
                               ctypes.c_void_p(self.stream.cuda_stream),
                               ctypes.c_void_p(self.state.data_ptr()),
                               ctypes.c_void_p(self.ws.data_ptr() + off), ws_bytes)
        if st != QSV_OK:
            raise QsvError(st, self.L.qsv_last_error(None).decode())
        self.h = h

    def close(self):
        if getattr(self, "h", None):
            self.L.qsv_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _check(self, st):
        if st != QSV_OK:
            raise QsvError(st, self.L.qsv_last_error(self.h).decode())

    def qsv_set_option(self, name, value):
        self._check(self.L.qsv_set_option(self.h, name.encode(), int(value)))

    def qsv_probe_pass(self, low_bits, window_start, transposes=0):
        self._check(self.L.qsv_probe_pass(self.h, low_bits, window_start, transposes))

    def qsv_amp_encode(self, x, norm_out=None):
        assert x.is_cuda and x.dtype.is_floating_point and x.is_contiguous() and x.shape[0] == self.batch
        self._check(self.L.qsv_amp_encode(self.h, _ptr(x), x.shape[1], _ptr(norm_out)))

    def qsv_apply_layers(self, circ, params, feats=None, inverse=0):
        self._check(self.L.qsv_apply_layers(self.h, ctypes.byref(circ), _ptr(params), _ptr(feats),
                                            int(inverse)))

    def qsv_forward_small(self, x, circ, params, feats, decode, kind, out, norm_out=None):
        assert x.is_cuda and x.is_contiguous() and x.shape[0] == self.batch and out.is_cuda and out.is_contiguous()
        self._check(self.L.qsv_forward_small(self.h, _ptr(x), x.shape[1], ctypes.byref(circ), _ptr(params),
                                             _ptr(feats), int(decode), int(kind), _ptr(out), _ptr(norm_out)))

    def qsv_measure_static(self, kind, out, **kw):
        self.qsv_measure(kind, out, entry=self.L.qsv_measure_static, **kw)

    def qsv_measure(self, kind, out, qubit=0, mask=0, renormalise=0, x=None, uniforms=None, entry=None):
        r = qsv_measure_req()
        r.kind, r.qubit, r.mask, r.renormalise, r.reserved = kind, qubit, mask, int(renormalise), 0
        r.x_dev = x.data_ptr() if x is not None else None
        r.dim = x.shape[1] if x is not None else 0
        r.uniforms_dev = uniforms.data_ptr() if uniforms is not None else None
        r.shots = uniforms.shape[1] if uniforms is not None else 0
        r.out_dev = out.data_ptr()
        self._check((entry or self.L.qsv_measure)(self.h, ctypes.byref(r)))

    def qsv_loss_grad(self, circ, x, params, feats, kind, loss, grad, mean_loss=None, mean_grad=None,
                      mask=0, targets=None):
        spec = qsv_loss(kind, 0, mask, None if targets is None else targets.data_ptr())
        self._check(self.L.qsv_loss_grad(self.h, ctypes.byref(circ), _ptr(x), x.shape[1], _ptr(params),
                                         _ptr(feats), ctypes.byref(spec), _ptr(loss), _ptr(grad),
                                         _ptr(mean_loss), _ptr(mean_grad)))

    def qsv_distill(self, kind, scores, top_idx, top_logits, temperature=1.0, top_lse=None, loss=None, stats=None,
                    have_stats=0, grad_loss=None, grad=None):
        d = self.dev.index
        s = _rows(scores, kind, d, "scores")
        r = qsv_distill_req()
        r.kind, r.have_stats, r.scores_dev, r.row_stride = kind, have_stats, s.data_ptr(), s.stride(0)
        r.rows, r.cols = s.shape
        r.loss_dev, r.stats_dev = _flat(loss, "float32", d, "loss", r.rows), _flat(stats, "float32", d, "stats", r.rows, 2)
        r.grad_loss_dev = _flat(grad_loss, "float32", d, "grad_loss", r.rows)
        if grad is not None:
            _need(_rows(grad, kind, d, "grad").shape == s.shape, "grad must have the shape of the scores")
            r.grad_dev, r.grad_stride = grad.data_ptr(), grad.stride(0)
        t = _teacher(r.rows, top_idx, top_logits, temperature, top_lse, d)
        self._check(self.L.qsv_distill(self.h, ctypes.byref(r), ctypes.byref(t)))

    def qsv_distill_grad(self, circ, x, params, feats, top_idx, top_logits, loss, grad, mean_loss=None, mean_grad=None,
                         temperature=1.0, top_lse=None):
        d, B, P = self.dev.index, self.batch, max(0, qsv_num_params(circ, self.n))       # (a bad circuit is the library's to refuse)
        t = _teacher(B, top_idx, top_logits, temperature, top_lse, d)
        _need(x is not None and x.dim() == 2, "x must be [batch][dim]")
        at = (_room(x, "float32", d, "x", B * x.shape[1]), x.shape[1], _room(params, "float32", d, "params", P),
              _room(feats, "float32", d, "feats", B * self.n) if circ.reupload else None)
        out = (_room(loss, "float32", d, "loss", B), _room(grad, "float32", d, "grad", B * P),
               _room(mean_loss, "float32", d, "mean_loss", 1), _room(mean_grad, "float32", d, "mean_grad", P))
        self._check(self.L.qsv_distill_grad(self.h, ctypes.byref(circ), *at, ctypes.byref(t), *out))

    def qsv_reset_fidelity(self, circ, params, feats, mask, x, out):
        self._check(self.L.qsv_reset_fidelity(self.h, ctypes.byref(circ), _ptr(params), _ptr(feats), mask,
                                              _ptr(x), x.shape[1], _ptr(out)))

    def qsv_shot_expz(self, samples, out):
        self._check(self.L.qsv_shot_expz(self.h, _ptr(samples), samples.shape[1], _ptr(out)))

    def qsv_sample(self, kind, out, uniforms, scores=None, temperature=None, top_k=None, top_p=None, min_p=None,
                   logp=None, kept=None):
        r, d = qsv_sample_req(), self.dev.index
        r.kind = kind
        if kind == QSV_S_STATE:
            _need(scores is None, "scores must be None for the context's state")
            r.rows, r.cols = self.batch, 1 << self.n
        else:
            s = _rows(scores, kind, d, "scores")
            r.scores_dev, r.rows, r.cols, r.row_stride = s.data_ptr(), s.shape[0], s.shape[1], s.stride(0)
        _need(uniforms is not None and uniforms.dim() == 2, "uniforms must be [rows][shots]")
        r.shots = uniforms.shape[1]
        r.temperature_dev = _flat(temperature, "float32", d, "temperature", r.rows)
        r.top_k_dev = _flat(top_k, "int32", d, "top_k", r.rows)
        r.top_p_dev = _flat(top_p, "float32", d, "top_p", r.rows)
        r.min_p_dev = _flat(min_p, "float32", d, "min_p", r.rows)
        r.uniforms_dev = _flat(uniforms, "float64", d, "uniforms", r.rows, r.shots)
        r.out_dev = _flat(out, "int64", d, "out", r.rows, r.shots)
        r.logp_dev = _flat(logp, "float32", d, "logp", r.rows, r.shots)
        r.kept_dev = _flat(kept, "int32", d, "kept", r.rows)
        self._check(self.L.qsv_sample(self.h, ctypes.byref(r)))

    def qsv_adjust(self, kind, scores, out=None, prior=None, prior_len=None, prompt_len=None, repetition=None, frequency=None,
                   presence=None, bias=None, entry_idx=None, entry_bias=None, masks=None, mask_of=None):
        """out None: over the scores."""
        r, d, dtype = qsv_adjust_req(), self.dev.index, _score_type(kind)
        r.kind = kind
        _need(scores is not None, "scores must be given")
        at, rows, cols, stride = _grid(scores, dtype, d, "scores")
        r.scores_dev, r.rows, r.cols, r.row_stride = at, rows, cols, stride
        if out is not None:
            at, n, m, stride = _grid(out, dtype, d, "out")
            if n != rows or m != cols:
                _need(False, "out must have the shape of the scores")
        r.out_dev, r.out_stride = at, stride
        _adjustment(r, d, rows, prior, prior_len, prompt_len, repetition, frequency, presence, entry_idx, masks, mask_of)
        if bias is not None:
            r.bias_dev = _each(bias, _dtype("float32"), d, (cols,), "bias")
        if entry_bias is not None and entry_idx is not None:
            r.entry_bias_dev = _each(entry_bias, _dtype("float32"), d, (rows, r.n_entries), "entry_bias")
        elif entry_bias is not None or entry_idx is not None:
            _need(False, "entry_idx and entry_bias go together")
        self._check(self.L.qsv_adjust(self.h, ctypes.byref(r)))

    def qsv_adjust_grad(self, kind, grad_out, grad=None, scores=None, grad_bias=None, grad_entry=None, prior=None, prior_len=None,
                        prompt_len=None, repetition=None, frequency=None, presence=None, entry_idx=None, masks=None, mask_of=None):
        """grad may be grad_out; None: the gradients of the biases alone."""
        r, b, d, dtype = qsv_adjust_req(), qsv_adjust_grad_req(), self.dev.index, _score_type(kind)
        r.kind = kind
        _need(grad_out is not None, "grad_out must be given")
        b.grad_out_dev, rows, cols, b.grad_out_stride = _grid(grad_out, dtype, d, "grad_out")
        r.rows, r.cols = rows, cols
        if scores is not None:
            r.scores_dev, n, m, r.row_stride = _grid(scores, dtype, d, "scores")
            if n != rows or m != cols:
                _need(False, "scores must have the shape of grad_out")
        if grad is not None:
            b.grad_dev, n, m, b.grad_stride = _grid(grad, dtype, d, "grad")
            if n != rows or m != cols:
                _need(False, "grad must have the shape of grad_out")
        _adjustment(r, d, rows, prior, prior_len, prompt_len, repetition, frequency, presence, entry_idx, masks, mask_of)
        if grad_bias is not None:
            b.grad_bias_dev = _each(grad_bias, _dtype("float32"), d, (cols,), "grad_bias")
        if grad_entry is not None:
            b.grad_entry_dev = _each(grad_entry, _dtype("float32"), d, (rows, r.n_entries), "grad_entry")
        self._check(self.L.qsv_adjust_grad(self.h, ctypes.byref(r), ctypes.byref(b)))

    def _list(self, tensors, cls):
        got = tensors if isinstance(tensors, cls) else cls(tensors)
        _need(got.devices <= {self.dev.index}, "tensors must be on cuda:%d" % self.dev.index)
        return got

    def qsv_clip_grads(self, grads, max_norm, norm=None, out=None):
        """grads, out: tensors, or a TensorList of them; out None: over the gradients."""
        g = self._list(grads, TensorList)
        o = None if out is None else self._list(out, TensorList)
        _need(o is None or len(o) == len(g), "out must be as many as grads")
        at = _flat(norm, "float32", self.dev.index, "norm", 1)
        self._check(self.L.qsv_clip_grads(self.h, g.at, None if o is None else o.at, len(g), max_norm, at))

    def qsv_adam_clipped(self, tensors, t, lr, max_norm, beta1=0.9, beta2=0.999, eps=1e-8, norm=None):
        """tensors: an AdamList."""
        _need(isinstance(tensors, AdamList), "tensors must be an AdamList")
        a = self._list(tensors, AdamList)
        at = _flat(norm, "float32", self.dev.index, "norm", 1)
        self._check(self.L.qsv_adam_clipped(self.h, a.at, len(a), t, lr, beta1, beta2, eps, max_norm, at))

    def qsv_pauli_expect(self, out, xmask=0, ymask=0, zmask=0):
        self._check(self.L.qsv_pauli_expect(self.h, xmask, ymask, zmask, _ptr(out)))

    def qsv_sgd_step(self, params, grad, lr):
        self._check(self.L.qsv_sgd_step(self.h, _ptr(params), _ptr(grad), params.numel(), lr))

    def qsv_adam_step(self, params, grad, m, v, t, lr, beta1=0.9, beta2=0.999, eps=1e-8):
        self._check(self.L.qsv_adam_step(self.h, _ptr(params), _ptr(grad), _ptr(m), _ptr(v), params.numel(),
                                         t, lr, beta1, beta2, eps))

    def qsv_adjoint_grad(self, circ, x, params, feats, obs_qubit, loss, grad, mean_loss=None,
                         mean_grad=None):
        self._check(self.L.qsv_adjoint_grad(self.h, ctypes.byref(circ), _ptr(x), x.shape[1],
                                            _ptr(params), _ptr(feats), obs_qubit, _ptr(loss),
                                            _ptr(grad), _ptr(mean_loss), _ptr(mean_grad)))

    def qsv_param_shift_grad(self, circ, x, params, feats, obs_qubit, loss, grad, mean_loss=None,
                             mean_grad=None):
        self._check(self.L.qsv_param_shift_grad(self.h, ctypes.byref(circ), _ptr(x), x.shape[1],
                                                _ptr(params), _ptr(feats), obs_qubit, _ptr(loss),
                                                _ptr(grad), _ptr(mean_loss), _ptr(mean_grad)))
