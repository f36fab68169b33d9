"""ctypes binding of the operators around the convolution layer (include/bltrain.h).

Layer norm, group norm, the gated recurrence, log probabilities and the AdamW and
orthogonalised steps, as plans like ``blconv.Plan``: argument marshalling only, every compute step runs in the HIP kernels of
libblconv.so on the GPU that holds the tensors, all of them on one, and on that
GPU's current stream (or the one given).  Buffers are the caller's;
``workspace()`` and ``state()`` make those whose size a plan sets.
"""
from __future__ import annotations

import ctypes
import itertools

import torch

from . import blconv
from .blconv import BlError, _check  # noqa: F401  (BlError: what these calls raise)

BL_F32, BL_BF16, BL_F16 = 0, 1, 2
BL_CHANNELS_LAST, BL_CHANNELS_FIRST = 0, 1
BL_ACT_NONE, BL_ACT_RELU, BL_ACT_SILU = 0, 1, 2
BL_GATE_SIGMOID, BL_GATE_EXP = 0, 1

EXPORTED = (
    "bl_norm_plan_create", "bl_norm_plan_destroy", "bl_norm_workspace_size", "bl_norm_forward", "bl_norm_backward",
    "bl_logprob_plan_create", "bl_logprob_plan_destroy", "bl_logprob_workspace_size", "bl_logprob_forward",
    "bl_logprob_backward", "bl_adamw_plan_create", "bl_adamw_plan_destroy", "bl_adamw_state_size",
    "bl_adamw_state_layout", "bl_adamw_step", "bl_adamw_get_moments", "bl_adamw_set_moments",
    "bl_group_norm_plan_create", "bl_group_norm_plan_destroy", "bl_group_norm_workspace_size",
    "bl_group_norm_forward", "bl_group_norm_backward", "bl_recurrence_plan_create", "bl_recurrence_plan_destroy",
    "bl_recurrence_workspace_size", "bl_recurrence_states_size", "bl_recurrence_forward", "bl_recurrence_backward",
    "bl_muon_plan_create", "bl_muon_plan_destroy", "bl_muon_state_size", "bl_muon_workspace_size", "bl_muon_step",
    "bl_muon_orthogonalize",
)

_P, _I, _L, _D, _S = ctypes.c_void_p, ctypes.c_int, ctypes.c_longlong, ctypes.c_double, ctypes.c_size_t


class NormDesc(ctypes.Structure):
    _fields_ = [("outer", _L), ("size", _L), ("inner", _L), ("dtype", _I), ("wdtype", _I), ("eps", _D),
                ("x_stride", _L), ("y_stride", _L)]


class LogProbDesc(ctypes.Structure):
    _fields_ = [("rows", _L), ("classes", _L), ("top", _I), ("dtype", _I), ("stride", _L), ("grad_stride", _L)]


class AdamWDesc(ctypes.Structure):
    _fields_ = [("count", _I), ("sizes", ctypes.POINTER(_L)), ("decay", ctypes.POINTER(ctypes.c_ubyte)),
                ("param_dtype", _I), ("grad_dtype", _I), ("bits", _I)]


class AdamWArgs(ctypes.Structure):
    _fields_ = [("lr", _D), ("beta1", _D), ("beta2", _D), ("eps", _D), ("weight_decay", _D), ("step", _L),
                ("seed", ctypes.c_uint), ("grad_scale", _P), ("live", _P)]


class GroupNormDesc(ctypes.Structure):
    _fields_ = [("batch", _L), ("sites", _L), ("channels", _L), ("groups", _L), ("layout", _I), ("act", _I),
                ("dtype", _I), ("wdtype", _I), ("eps", _D), ("x_stride", _L), ("y_stride", _L)]


class RecurrenceDesc(ctypes.Structure):
    _fields_ = [("outer", _L), ("length", _L), ("inner", _L), ("gate", _I), ("dtype", _I), ("in_outer", _L),
                ("in_step", _L), ("out_outer", _L), ("out_step", _L)]


class MuonDesc(ctypes.Structure):
    _fields_ = [("count", _I), ("rows", ctypes.POINTER(_L)), ("cols", ctypes.POINTER(_L)),
                ("decay", ctypes.POINTER(ctypes.c_ubyte)), ("scale", ctypes.POINTER(_D)), ("steps", _I),
                ("coef", ctypes.POINTER(_D)), ("param_dtype", _I), ("grad_dtype", _I)]


class MuonArgs(ctypes.Structure):
    _fields_ = [("lr", _D), ("momentum", _D), ("eps", _D), ("weight_decay", _D), ("nesterov", _I), ("step", _L),
                ("seed", ctypes.c_uint), ("grad_scale", _P), ("live", _P)]


_lib = None


def load():
    """libblconv.so with this module's calls declared."""
    global _lib
    if _lib is not None:
        return _lib
    lib = blconv.load()
    pp = ctypes.POINTER(_P)
    lib.bl_norm_plan_create.argtypes = [pp, ctypes.POINTER(NormDesc)]
    lib.bl_norm_workspace_size.argtypes = [_P, ctypes.POINTER(_S)]
    lib.bl_norm_forward.argtypes = [_P] * 8
    lib.bl_norm_backward.argtypes = [_P] * 10
    lib.bl_logprob_plan_create.argtypes = [pp, ctypes.POINTER(LogProbDesc)]
    lib.bl_logprob_workspace_size.argtypes = [_P, ctypes.POINTER(_S)]
    lib.bl_logprob_forward.argtypes = [_P] * 9
    lib.bl_logprob_backward.argtypes = [_P] * 8
    lib.bl_adamw_plan_create.argtypes = [pp, ctypes.POINTER(AdamWDesc)]
    lib.bl_adamw_state_size.argtypes = [_P, ctypes.POINTER(_S), ctypes.POINTER(_L), ctypes.POINTER(_L)]
    lib.bl_adamw_state_layout.argtypes = [_P] + [ctypes.POINTER(_S)] * 4
    lib.bl_adamw_step.argtypes = [_P, _P, _P, _P, ctypes.POINTER(AdamWArgs), _P]
    lib.bl_adamw_get_moments.argtypes = [_P] * 5
    lib.bl_adamw_set_moments.argtypes = [_P] * 5
    lib.bl_group_norm_plan_create.argtypes = [pp, ctypes.POINTER(GroupNormDesc)]
    lib.bl_group_norm_workspace_size.argtypes = [_P, ctypes.POINTER(_S)]
    lib.bl_group_norm_forward.argtypes = [_P] * 8
    lib.bl_group_norm_backward.argtypes = [_P] * 11
    lib.bl_recurrence_plan_create.argtypes = [pp, ctypes.POINTER(RecurrenceDesc)]
    lib.bl_recurrence_workspace_size.argtypes = [_P, ctypes.POINTER(_S)]
    lib.bl_recurrence_states_size.argtypes = [_P, ctypes.POINTER(_L)]
    lib.bl_recurrence_forward.argtypes = [_P] * 10
    lib.bl_recurrence_backward.argtypes = [_P] * 12
    lib.bl_muon_plan_create.argtypes = [pp, ctypes.POINTER(MuonDesc)]
    lib.bl_muon_state_size.argtypes = [_P, ctypes.POINTER(_S), ctypes.POINTER(_L), ctypes.POINTER(_L)]
    lib.bl_muon_workspace_size.argtypes = [_P, ctypes.POINTER(_S)]
    lib.bl_muon_step.argtypes = [_P, _P, _P, _P, _P, ctypes.POINTER(MuonArgs), _P]
    lib.bl_muon_orthogonalize.argtypes = [_P, _P, _P, _P, _D, _P]
    for name in ("bl_norm_plan_destroy", "bl_logprob_plan_destroy", "bl_adamw_plan_destroy",
                 "bl_group_norm_plan_destroy", "bl_recurrence_plan_destroy", "bl_muon_plan_destroy"):
        getattr(lib, name).argtypes = [_P]
    for name in EXPORTED:
        getattr(lib, name)  # every declared symbol must be exported
    _lib = lib
    return lib


_DTYPES = {torch.float32: BL_F32, torch.bfloat16: BL_BF16, torch.float16: BL_F16}


def _dtype_code(dtype, name):
    code = _DTYPES.get(dtype)
    if code is None:
        raise ValueError(f"{name} must be torch.float32, torch.bfloat16 or torch.float16, not {dtype}")
    return code


def _gpu(t, name):
    """Number of the GPU that holds tensor t."""
    device = t.get_device()
    if device < 0:
        raise ValueError(f"{name} must be a tensor on the GPU")
    return device


def _stream(stream, device):
    """The HIP stream: the given one, or the current one of the GPU."""
    if stream is None:
        return torch._C._cuda_getCurrentRawStream(device)
    if stream.device_index != device:
        raise ValueError(f"the stream is not one of the tensors' GPU {device}")
    return stream.cuda_stream


def _run(call, function, device, *args):
    """One call of the library, whose launches go to the current GPU."""
    if torch._C._cuda_getDevice() == device:
        code = function(*args)
    else:
        with torch.cuda.device(device):
            code = function(*args)
    _check(call, code)


def _flat(t, dtype, numel, name, device):
    """Device pointer of a contiguous tensor of `numel` elements, whatever its shape."""
    if t is None:
        return None
    if t.get_device() != device or t.dtype != dtype or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous {dtype} tensor on GPU {device}, as the others")
    if t.numel() != numel:
        raise ValueError(f"{name} has {t.numel()} elements, expected {numel}")
    return t.data_ptr()


def _sliced(t, dtype, outer, length, stride, name, device):
    """Device pointer of `outer` contiguous slices of `length` elements whose
    starts are `stride` apart: a contiguous tensor where stride = length, else
    one whose first axis has that stride."""
    if t.get_device() != device or t.dtype != dtype:
        raise ValueError(f"{name} must be a {dtype} tensor on GPU {device}, as the others")
    if t.numel() != outer * length:
        raise ValueError(f"{name} has {t.numel()} elements, expected {outer * length}")
    if stride == length or outer <= 1:
        if not t.is_contiguous():
            raise ValueError(f"{name} must be contiguous")
    elif t.dim() < 2 or t.shape[0] != outer or t.stride(0) != stride or not t[0].is_contiguous():
        raise ValueError(f"{name} must have {outer} contiguous slices, {stride} elements apart")
    return t.data_ptr()


class _Plan:
    _destroy = ""

    def __del__(self):
        h = getattr(self, "_h", None)
        if h is not None and h.value:
            getattr(self._lib, self._destroy)(h)
            self._h = None

    def workspace(self, device="cuda"):
        return torch.empty(self.workspace_bytes, dtype=torch.uint8, device=device)

    def _ws(self, ws, device):
        if self.workspace_bytes == 0:
            return None
        if ws is None or ws.get_device() != device or not ws.is_contiguous() or ws.nbytes < self.workspace_bytes:
            raise ValueError("workspace must be a contiguous tensor of at least workspace_bytes bytes on the tensors' GPU")
        return ws.data_ptr()


class NormPlan(_Plan):
    """Layer norm over the middle axis of [outer][size][inner].

    Rows: ``NormPlan(rows, features)``; the channels at each position of the
    convolution layer's maps: ``NormPlan(N, C, L)`` or ``NormPlan(N, C, H * W)``;
    whole samples: ``NormPlan(N, C * H * W)``.  Tensors may have any shape of
    that many elements.  ``x_stride`` and ``y_stride`` (elements between outer
    slices, 0: dense) are those of x and dx, and of y and dy.
    """

    _destroy = "bl_norm_plan_destroy"

    def __init__(self, outer, size, inner=1, dtype=None, wdtype=None, eps=1e-5, x_stride=0, y_stride=0):
        self._lib = load()
        self.dtype = torch.float32 if dtype is None else dtype
        self.wdtype = torch.float32 if wdtype is None else wdtype
        d = NormDesc(outer, size, inner, _dtype_code(self.dtype, "dtype"), _dtype_code(self.wdtype, "wdtype"),
                     float(eps), x_stride, y_stride)
        self._h = _P()
        _check("bl_norm_plan_create", self._lib.bl_norm_plan_create(ctypes.byref(self._h), ctypes.byref(d)))
        self.outer, self.size, self.inner = outer, size, inner
        self.x_stride, self.y_stride = x_stride or size * inner, y_stride or size * inner
        n = _S()
        _check("bl_norm_workspace_size", self._lib.bl_norm_workspace_size(self._h, ctypes.byref(n)))
        self.workspace_bytes = n.value

    def stats_shape(self):
        return (2, self.outer, self.inner)

    def _x(self, t, name, device):
        return _sliced(t, self.dtype, self.outer, self.size * self.inner, self.x_stride, name, device)

    def _y(self, t, name, device):
        return _sliced(t, self.dtype, self.outer, self.size * self.inner, self.y_stride, name, device)

    def _w(self, t, name, device):
        return _flat(t, self.wdtype, self.size, name, device)

    def _stats(self, t, device):
        return _flat(t, torch.float32, 2 * self.outer * self.inner, "stats", device)

    def forward(self, x, weight, bias, y, stats, ws, stream=None):
        """y, and mean and 1 / deviation in `stats` (None: not wanted); weight
        None: 1, bias None: 0."""
        on = _gpu(x, "x")
        _run("bl_norm_forward", self._lib.bl_norm_forward, on,
             self._h, self._x(x, "x", on), self._w(weight, "weight", on), self._w(bias, "bias", on),
             self._y(y, "y", on), self._stats(stats, on), self._ws(ws, on), _stream(stream, on))

    def backward(self, dy, x, weight, stats, dx, dweight, dbias, ws, stream=None):
        """dx, and the gradients of weight and bias (None: not wanted)."""
        on = _gpu(x, "x")
        _run("bl_norm_backward", self._lib.bl_norm_backward, on,
             self._h, self._y(dy, "dy", on), self._x(x, "x", on), self._w(weight, "weight", on),
             self._stats(stats, on), self._x(dx, "dx", on), self._w(dweight, "dweight", on),
             self._w(dbias, "dbias", on), self._ws(ws, on), _stream(stream, on))


class GroupNormPlan(_Plan):
    """Group norm with an activation (None, "relu" or "silu") of [batch][sites][channels]
    (channels_last) or [batch][channels][sites], the convolution layer's maps with
    L or H * W sites.  Tensors may have any shape of that many elements.
    ``x_stride`` and ``y_stride`` (elements between samples, 0: dense) are those of
    x and dx, and of y and dy.
    """

    _destroy = "bl_group_norm_plan_destroy"
    _acts = {None: BL_ACT_NONE, "none": BL_ACT_NONE, "relu": BL_ACT_RELU, "silu": BL_ACT_SILU}

    def __init__(self, batch, sites, channels, groups, channels_last=False, act=None, dtype=None, wdtype=None, eps=1e-5,
                 x_stride=0, y_stride=0):
        self._lib = load()
        if act not in self._acts:
            raise ValueError(f"act must be None, 'relu' or 'silu', not {act!r}")
        self.dtype = torch.float32 if dtype is None else dtype
        self.wdtype = torch.float32 if wdtype is None else wdtype
        d = GroupNormDesc(batch, sites, channels, groups, BL_CHANNELS_LAST if channels_last else BL_CHANNELS_FIRST,
                          self._acts[act], _dtype_code(self.dtype, "dtype"), _dtype_code(self.wdtype, "wdtype"),
                          float(eps), x_stride, y_stride)
        self._h = _P()
        _check("bl_group_norm_plan_create", self._lib.bl_group_norm_plan_create(ctypes.byref(self._h), ctypes.byref(d)))
        self.batch, self.sites, self.channels, self.groups = batch, sites, channels, groups
        self.x_stride, self.y_stride = x_stride or sites * channels, y_stride or sites * channels
        n = _S()
        _check("bl_group_norm_workspace_size", self._lib.bl_group_norm_workspace_size(self._h, ctypes.byref(n)))
        self.workspace_bytes = n.value

    def stats_shape(self):
        return (2, self.batch, self.groups)

    def _x(self, t, name, device):
        return _sliced(t, self.dtype, self.batch, self.sites * self.channels, self.x_stride, name, device)

    def _y(self, t, name, device):
        return _sliced(t, self.dtype, self.batch, self.sites * self.channels, self.y_stride, name, device)

    def _w(self, t, name, device):
        return _flat(t, self.wdtype, self.channels, name, device)

    def _stats(self, t, device):
        return _flat(t, torch.float32, 2 * self.batch * self.groups, "stats", device)

    def forward(self, x, weight, bias, y, stats, ws, stream=None):
        """y, and mean and 1 / deviation of the groups in `stats` (None: not
        wanted); weight None: 1, bias None: 0."""
        on = _gpu(x, "x")
        _run("bl_group_norm_forward", self._lib.bl_group_norm_forward, on,
             self._h, self._x(x, "x", on), self._w(weight, "weight", on), self._w(bias, "bias", on),
             self._y(y, "y", on), self._stats(stats, on), self._ws(ws, on), _stream(stream, on))

    def backward(self, dy, x, weight, bias, stats, dx, dweight, dbias, ws, stream=None):
        """dx, and the gradients of weight and bias (None: not wanted)."""
        on = _gpu(x, "x")
        _run("bl_group_norm_backward", self._lib.bl_group_norm_backward, on,
             self._h, self._y(dy, "dy", on), self._x(x, "x", on), self._w(weight, "weight", on),
             self._w(bias, "bias", on), self._stats(stats, on), self._x(dx, "dx", on),
             self._w(dweight, "dweight", on), self._w(dbias, "dbias", on), self._ws(ws, on), _stream(stream, on))


class RecurrencePlan(_Plan):
    """h_t = a_t h_(t-1) + b_t along the middle axis of [outer][length][inner], with
    a = sigmoid(gate), b = (1 - a) x (gate="sigmoid") or a = exp(gate), b = x
    (gate="exp").

    Tokens: ``RecurrencePlan(N, tokens, channels)``; the samples of the convolution
    layer's maps: ``RecurrencePlan(N * C, L)``.  Tensors are [outer, length, inner],
    or of any shape where they are contiguous and dense.  ``in_strides`` and
    ``out_strides`` are the elements between two outer entries and two steps (0:
    dense) of gate, x and their gradients, and of y and dy.
    """

    _destroy = "bl_recurrence_plan_destroy"
    _gates = {"sigmoid": BL_GATE_SIGMOID, "exp": BL_GATE_EXP}

    def __init__(self, outer, length, inner=1, gate="sigmoid", dtype=None, in_strides=(0, 0), out_strides=(0, 0)):
        self._lib = load()
        if gate not in self._gates:
            raise ValueError(f"gate must be 'sigmoid' or 'exp', not {gate!r}")
        self.dtype = torch.float32 if dtype is None else dtype
        d = RecurrenceDesc(outer, length, inner, self._gates[gate], _dtype_code(self.dtype, "dtype"), *in_strides,
                           *out_strides)
        self._h = _P()
        _check("bl_recurrence_plan_create", self._lib.bl_recurrence_plan_create(ctypes.byref(self._h), ctypes.byref(d)))
        self.outer, self.length, self.inner = outer, length, inner

        def strides(given):
            step = given[1] or inner
            return given[0] or length * step, step
        self.in_strides, self.out_strides = strides(in_strides), strides(out_strides)
        n, m = _S(), _L()
        _check("bl_recurrence_workspace_size", self._lib.bl_recurrence_workspace_size(self._h, ctypes.byref(n)))
        _check("bl_recurrence_states_size", self._lib.bl_recurrence_states_size(self._h, ctypes.byref(m)))
        self.workspace_bytes, self.states_elements = n.value, m.value

    def states(self, device="cuda"):
        """What forward() leaves for backward()."""
        return torch.empty(self.states_elements, device=device)

    def _steps(self, t, strides, name, device):
        if t.get_device() != device or t.dtype != self.dtype:
            raise ValueError(f"{name} must be a {self.dtype} tensor on GPU {device}, as the others")
        shape = (self.outer, self.length, self.inner)
        if t.numel() != self.outer * self.length * self.inner:
            raise ValueError(f"{name} has {t.numel()} elements, expected {self.outer * self.length * self.inner}")
        if t.numel() == 0:
            return t.data_ptr()
        dense = strides == (self.length * self.inner, self.inner) or t.numel() == self.inner
        if dense and t.is_contiguous():
            return t.data_ptr()
        if t.shape != shape or any(n > 1 and s != want for n, s, want in zip(shape, t.stride(), (*strides, 1))):
            raise ValueError(f"{name} must be {shape} with strides {(*strides, 1)}, "
                             f"not {tuple(t.shape)} with {t.stride()}")
        return t.data_ptr()

    def _in(self, t, name, device):
        return self._steps(t, self.in_strides, name, device)

    def _out(self, t, name, device):
        return self._steps(t, self.out_strides, name, device)

    def _state(self, t, name, device):
        return _flat(t, torch.float32, self.outer * self.inner, name, device)

    def _resets(self, t, device):
        if t is not None and t.dtype == torch.bool:
            t = t.view(torch.uint8)
        return _flat(t, torch.uint8, self.outer * self.length, "resets", device)

    def _saved(self, t, device):
        return _flat(t, torch.float32, self.states_elements, "states", device)

    def forward(self, gate, x, y, ws, h0=None, last=None, resets=None, states=None, stream=None):
        """y = h of every step; `last`: the last one in float32; `states`: what
        backward() needs (both None: not wanted); h0 None: 0.  resets: bytes or
        truth values [outer][length], the steps at which the state is dropped."""
        on = _gpu(x, "x")
        _run("bl_recurrence_forward", self._lib.bl_recurrence_forward, on,
             self._h, self._in(gate, "gate", on), self._in(x, "x", on), self._resets(resets, on),
             self._state(h0, "h0", on), self._out(y, "y", on), self._state(last, "last", on),
             self._saved(states, on), self._ws(ws, on), _stream(stream, on))

    def backward(self, gate, x, dy, states, dgate, dx, ws, dlast=None, dh0=None, resets=None, stream=None):
        """dgate, dx and dh0 (None: not wanted) from dy and dlast (None: 0)."""
        on = _gpu(x, "x")
        _run("bl_recurrence_backward", self._lib.bl_recurrence_backward, on,
             self._h, self._in(gate, "gate", on), self._in(x, "x", on), self._resets(resets, on),
             self._saved(states, on), self._out(dy, "dy", on), self._state(dlast, "dlast", on),
             self._in(dgate, "dgate", on), self._in(dx, "dx", on), self._state(dh0, "dh0", on), self._ws(ws, on),
             _stream(stream, on))


class LogProbPlan(_Plan):
    """Log probabilities of given classes, entropies and the `top` likeliest
    classes of rows of logits, and the logits' gradient."""

    _destroy = "bl_logprob_plan_destroy"

    def __init__(self, rows, classes, top=0, dtype=None, stride=0, grad_stride=0):
        self._lib = load()
        self.dtype = torch.float32 if dtype is None else dtype
        d = LogProbDesc(rows, classes, top, _dtype_code(self.dtype, "dtype"), stride, grad_stride)
        self._h = _P()
        _check("bl_logprob_plan_create", self._lib.bl_logprob_plan_create(ctypes.byref(self._h), ctypes.byref(d)))
        self.rows, self.classes, self.top = rows, classes, top
        self.stride, self.grad_stride = stride or classes, grad_stride or classes
        n = _S()
        _check("bl_logprob_workspace_size", self._lib.bl_logprob_workspace_size(self._h, ctypes.byref(n)))
        self.workspace_bytes = n.value

    def forward(self, logits, targets, logp, stats, top_logp, top_index, ws, stream=None):
        """logp [rows], stats [3][rows] (largest logit, log of the sum of
        exponentials over it, entropy), top_logp and top_index [rows][top]."""
        on, n = _gpu(logits, "logits"), self.rows
        _run("bl_logprob_forward", self._lib.bl_logprob_forward, on,
             self._h, _sliced(logits, self.dtype, n, self.classes, self.stride, "logits", on),
             _flat(targets, torch.int64, n, "targets", on), _flat(logp, torch.float32, n, "logp", on),
             _flat(stats, torch.float32, 3 * n, "stats", on),
             _flat(top_logp, torch.float32, n * self.top, "top_logp", on),
             _flat(top_index, torch.int64, n * self.top, "top_index", on), self._ws(ws, on), _stream(stream, on))

    def backward(self, logits, targets, stats, g_logp, g_entropy, dlogits, stream=None):
        """The logits' gradient from those of logp and of the entropy (None: 0)."""
        on, n = _gpu(logits, "logits"), self.rows
        _run("bl_logprob_backward", self._lib.bl_logprob_backward, on,
             self._h, _sliced(logits, self.dtype, n, self.classes, self.stride, "logits", on),
             _flat(targets, torch.int64, n, "targets", on), _flat(stats, torch.float32, 3 * n, "stats", on),
             _flat(g_logp, torch.float32, n, "g_logp", on), _flat(g_entropy, torch.float32, n, "g_entropy", on),
             _sliced(dlogits, self.dtype, n, self.classes, self.grad_stride, "dlogits", on), _stream(stream, on))


class StepTensors:
    """The parameters and gradients that an optimiser's step goes over: the tensors,
    which it keeps alive, and the list of their addresses, taken once (a tensor
    that is given other storage has to be bound again)."""

    def __init__(self, plan, params, grads):
        if len(params) != len(plan.sizes) or len(grads) != len(plan.sizes):
            raise ValueError(f"expected {len(plan.sizes)} parameters and gradients")
        self.plan, self.params, self.grads = plan, list(params), list(grads)
        there = [t for t in self.params + self.grads if t is not None]  # (None: of an empty tensor)
        self.on = _gpu(there[0], "a parameter") if there else None
        ptrs = _P * len(plan.sizes)
        self._p = ptrs(*[_flat(t, plan.param_dtype, n, f"parameter {i}", self.on)
                         for i, (t, n) in enumerate(zip(params, plan.sizes))])
        self._g = ptrs(*[_flat(t, plan.grad_dtype, n, f"gradient {i}", self.on)
                         for i, (t, n) in enumerate(zip(grads, plan.sizes))])


AdamWTensors = StepTensors


class AdamWPlan(_Plan):
    """One AdamW step over tensors of the given sizes; `bits`: 32 or 8 for the
    moments; `decay`: for each tensor whether weight decay applies (None: to all)."""

    _destroy = "bl_adamw_plan_destroy"
    workspace_bytes = 0

    def __init__(self, sizes, param_dtype=None, grad_dtype=None, bits=32, decay=None):
        self._lib = load()
        self.sizes, self.bits = [int(n) for n in sizes], bits
        self.param_dtype = torch.float32 if param_dtype is None else param_dtype
        self.grad_dtype = torch.float32 if grad_dtype is None else grad_dtype
        count = len(self.sizes)
        if decay is not None and len(decay) != count:
            raise ValueError("decay must have a value for each tensor")
        d = AdamWDesc(count, (_L * count)(*self.sizes),
                      None if decay is None else (ctypes.c_ubyte * count)(*[bool(x) for x in decay]),
                      _dtype_code(self.param_dtype, "param_dtype"), _dtype_code(self.grad_dtype, "grad_dtype"), bits)
        self._h = _P()
        _check("bl_adamw_plan_create", self._lib.bl_adamw_plan_create(ctypes.byref(self._h), ctypes.byref(d)))
        n, total, start = _S(), _L(), (_L * count)()
        _check("bl_adamw_state_size", self._lib.bl_adamw_state_size(self._h, ctypes.byref(n), ctypes.byref(total),
                                                                    start))
        self.state_bytes, self.total, self.starts = n.value, total.value, list(start)

    def state(self, device="cuda"):
        """A new state: moments of zero."""
        return torch.zeros(self.state_bytes, dtype=torch.uint8, device=device)

    def _state(self, state):
        if not state.is_contiguous() or state.nbytes != self.state_bytes:
            raise ValueError("state must be a contiguous GPU tensor of state_bytes bytes")
        return state.data_ptr()

    def bind(self, params, grads):
        """The list of tensors that step() takes: contiguous, of the plan's sizes and types."""
        return StepTensors(self, params, grads)

    def step(self, tensors, state, lr=1e-3, betas=(0.9, 0.999), eps=1e-8, weight_decay=1e-2, step=1, grad_scale=None,
             seed=0, live=None, stream=None):
        """One step, in place.  `grad_scale`: a float32 GPU tensor of one element
        that gradients are multiplied by.  `live`: a float64 GPU tensor (lr, step)
        that is read in the place of those two when the kernels run."""
        if tensors.plan is not self:
            raise ValueError("the tensors were bound to another plan")
        on = _gpu(state, "state")
        if tensors.on not in (None, on):
            raise ValueError("the state and the tensors must be on one GPU")
        a = AdamWArgs(lr, betas[0], betas[1], eps, weight_decay, step, seed & 0xFFFFFFFF,
                      _flat(grad_scale, torch.float32, 1, "grad_scale", on),
                      _flat(live, torch.float64, 2, "live", on))
        _run("bl_adamw_step", self._lib.bl_adamw_step, on, self._h, tensors._p, tensors._g, self._state(state),
             ctypes.byref(a), _stream(stream, on))

    def moments(self, state, m=None, v=None, stream=None):
        """(m, v), [total] each, tensor i's at starts[i]: of 32 bits as views of
        the state, of 8 bits as their values in new bfloat16 tensors (or those given)."""
        if self.bits == 32 and m is None and v is None:
            both = state.view(torch.float32)
            return both[:self.total], both[self.total:]
        dtype, on = torch.float32 if self.bits == 32 else torch.bfloat16, _gpu(state, "state")
        with torch.cuda.stream(stream):  # (None: the current one) memory of the stream that writes it
            m = torch.empty(self.total, dtype=dtype, device=state.device) if m is None else m
            v = torch.empty(self.total, dtype=dtype, device=state.device) if v is None else v
        _run("bl_adamw_get_moments", self._lib.bl_adamw_get_moments, on, self._h, self._state(state),
             _flat(m, dtype, self.total, "m", on), _flat(v, dtype, self.total, "v", on), _stream(stream, on))
        return m, v

    def load_moments(self, state, m, v, stream=None):
        """Sets the moments from values (converted to float32) in the layout of
        moments(), 0 between the tensors."""
        on = _gpu(state, "state")
        with torch.cuda.stream(stream):
            m, v = m.float(), v.float()
        _run("bl_adamw_set_moments", self._lib.bl_adamw_set_moments, on, self._h, self._state(state),
             _flat(m, torch.float32, self.total, "m", on), _flat(v, torch.float32, self.total, "v", on),
             _stream(stream, on))


class MuonPlan(_Plan):
    """One step of the Muon optimiser over matrices of the given shapes (rows,
    columns): momentum, orthogonalised by Newton-Schulz products.  `decay`: for each
    matrix whether weight decay applies (None: to all); `scales`: its factor on the
    learning rate (None: sqrt(max(1, rows / columns))); `coefficients`: (a, b, c) of
    each product step (None: the usual ones, five times)."""

    _destroy = "bl_muon_plan_destroy"

    def __init__(self, shapes, param_dtype=None, grad_dtype=None, decay=None, scales=None, coefficients=None):
        self._lib = load()
        self.shapes = [(int(r), int(c)) for r, c in shapes]
        self.sizes = [r * c for r, c in self.shapes]
        self.param_dtype = torch.float32 if param_dtype is None else param_dtype
        self.grad_dtype = torch.float32 if grad_dtype is None else grad_dtype
        count = len(self.shapes)
        for name, given in (("decay", decay), ("scales", scales)):
            if given is not None and len(given) != count:
                raise ValueError(f"{name} must have a value for each matrix")
        flat = None if coefficients is None else [float(v) for step in coefficients for v in step]
        if flat is not None and len(flat) != 3 * len(coefficients):
            raise ValueError("coefficients must be three values for each step")
        d = MuonDesc(count, (_L * count)(*[r for r, _ in self.shapes]), (_L * count)(*[c for _, c in self.shapes]),
                     None if decay is None else (ctypes.c_ubyte * count)(*[bool(x) for x in decay]),
                     None if scales is None else (_D * count)(*[float(x) for x in scales]),
                     5 if flat is None else len(coefficients), None if flat is None else (_D * len(flat))(*flat),
                     _dtype_code(self.param_dtype, "param_dtype"), _dtype_code(self.grad_dtype, "grad_dtype"))
        self._h = _P()
        _check("bl_muon_plan_create", self._lib.bl_muon_plan_create(ctypes.byref(self._h), ctypes.byref(d)))
        n, total, start, m = _S(), _L(), (_L * count)(), _S()
        _check("bl_muon_state_size", self._lib.bl_muon_state_size(self._h, ctypes.byref(n), ctypes.byref(total), start))
        _check("bl_muon_workspace_size", self._lib.bl_muon_workspace_size(self._h, ctypes.byref(m)))
        self.state_bytes, self.total, self.starts, self.workspace_bytes = n.value, total.value, list(start), m.value

    def state(self, device="cuda"):
        """A new state: momentum of zero."""
        return torch.zeros(self.state_bytes, dtype=torch.uint8, device=device)

    def _state(self, state):
        if not state.is_contiguous() or state.nbytes != self.state_bytes:
            raise ValueError("state must be a contiguous GPU tensor of state_bytes bytes")
        return state.data_ptr()

    def momentum(self, state):
        """The momentum [total] as a view of the state, matrix i's at starts[i]."""
        self._state(state)
        return state.view(torch.float32)

    def bind(self, params, grads):
        """The list of matrices that step() and orthogonalize() take: contiguous, of the
        plan's sizes and types.  No two parameters share memory, nor does one with
        another's gradient."""
        tensors = StepTensors(self, params, grads)

        def places(of):
            return sorted((t.data_ptr(), t.data_ptr() + t.nbytes, i) for i, t in enumerate(of) if t is not None and t.nbytes)
        own = places(tensors.params)
        for (_, end, i), (start, _, j) in zip(own, own[1:]):
            if start < end:
                raise ValueError(f"parameters {i} and {j} share memory")
        at = 0
        for start, end, i in places(tensors.grads):
            while at < len(own) and own[at][1] <= start:
                at += 1
            # (of two that it reaches into one is another's)
            if any(j != i for _, _, j in itertools.takewhile(lambda q: q[0] < end, own[at:at + 2])):
                raise ValueError(f"gradient {i} shares memory with another matrix's parameter")
        return tensors

    def _bound(self, tensors):
        if tensors.plan is not self:
            raise ValueError("the matrices were bound to another plan")
        return tensors.on

    def step(self, tensors, state, ws, lr=0.02, momentum=0.95, nesterov=True, weight_decay=0.0, eps=1e-7, step=1,
             grad_scale=None, seed=0, live=None, stream=None):
        """One step, in place.  `grad_scale`: a float32 GPU tensor of one element
        that gradients are multiplied by.  `live`: a float64 GPU tensor (lr, step)
        that is read in the place of those two when the kernels run."""
        on = _gpu(state, "state")
        if self._bound(tensors) not in (None, on):
            raise ValueError("the state and the matrices must be on one GPU")
        a = MuonArgs(lr, momentum, eps, weight_decay, bool(nesterov), step, seed & 0xFFFFFFFF,
                     _flat(grad_scale, torch.float32, 1, "grad_scale", on), _flat(live, torch.float64, 2, "live", on))
        _run("bl_muon_step", self._lib.bl_muon_step, on, self._h, tensors._p, tensors._g, self._state(state),
             self._ws(ws, on), ctypes.byref(a), _stream(stream, on))

    def orthogonalize(self, tensors, ws, eps=1e-7, stream=None):
        """The orthogonalised gradients, in the place of the parameters of bind()."""
        on = self._bound(tensors)
        if on is None:
            return
        _run("bl_muon_orthogonalize", self._lib.bl_muon_orthogonalize, on, self._h, tensors._p, tensors._g,
             self._ws(ws, on), eps, _stream(stream, on))
