"""Python binding of the layers of a recurrent language model (include/zo_layers.h):
linear attention with a decay for each head, layer norm and AdamW.

Argument marshalling only: every computation runs in the library's HIP
kernels, on the current torch stream unless one is passed (which then serves as the
current one: the caller makes it wait for what it needs). Outputs and
workspaces are allocated by torch, for the call's stream, when they are not given. Errors: ValueError
for arguments that do not fit together, zo.ZoError for what the library refuses. torch's autograd does not see
the calls: inputs that require gradients are taken under torch.no_grad() only (ValueError otherwise), and gradients
are those of the backward functions.

    layer_norm, layer_norm_backward
    linear_attention, linear_attention_backward, linear_attention_step
    AdamW (step, moments)
"""
from __future__ import annotations

import ctypes as C
import struct
from operator import attrgetter

import torch

from . import zo
from .zo import _beside, _record

MAX_DIM = 256   # ZO_LINATTN_MAX_DIM
BLOCK = 256     # ZO_ADAMW_BLOCK
_DTYPES = {torch.float32: zo.FP32, torch.bfloat16: zo.BF16}


# zo_linattn and zo_heads, packed (a call passes five of them; ctypes structures take several times as long to fill)
_SHAPE = struct.Struct("=7if")   # batch, length, q_heads, kv_heads, key_dim, value_dim, dtype, scale
_HEADS = struct.Struct("=Q3q")   # data, batch_stride, position_stride, head_stride


class _Tensor(C.Structure):  # zo_adamw_tensor
    _fields_ = [("param", C.c_void_p), ("grad", C.c_void_p), ("n", C.c_int64), ("state_offset", C.c_int64),
                ("weight_decay", C.c_double), ("pdtype", C.c_int32), ("gdtype", C.c_int32)]


class _AdamWConfig(C.Structure):  # zo_adamw_config
    _fields_ = [("lr", C.c_double), ("beta1", C.c_double), ("beta2", C.c_double), ("eps", C.c_double),
                ("step", C.c_int64), ("state_bits", C.c_int32)]


_lib = None


def lib():
    """The loaded library with the layers' signatures; raises if it has not been built."""
    global _lib
    if _lib is None:
        L = zo.lib()
        vp, shape, heads, i32, i64 = C.c_void_p, C.c_char_p, C.c_char_p, C.c_int32, C.c_int64
        L.zo_linear_attention_workspace_bytes.argtypes = [shape, i32]
        L.zo_linear_attention_workspace_bytes.restype = C.c_size_t
        L.zo_linear_attention.argtypes = [shape] + [heads] * 4 + [vp] * 5 + [C.c_size_t, vp]
        L.zo_linear_attention_backward.argtypes = [shape] + [heads] * 7 + [vp] * 6 + [C.c_size_t, vp]
        L.zo_linear_attention_step.argtypes = [shape] + [heads] * 4 + [vp, vp, i32, vp, vp]
        L.zo_layer_norm.argtypes = [i32, i32, i64, i64, vp, i64, vp, vp, C.c_float, vp, i64, vp, vp, vp]
        L.zo_layer_norm_workspace_bytes.argtypes = [i64, i64]
        L.zo_layer_norm_workspace_bytes.restype = C.c_size_t
        L.zo_layer_norm_backward.argtypes = [i32, i32, i64, i64, vp, i64, vp, i64, vp, vp, vp, vp, i64, vp, vp, vp,
                                             C.c_size_t, vp]
        L.zo_adamw.argtypes = [C.POINTER(_AdamWConfig), C.POINTER(_Tensor), i32, vp, vp, vp, vp, vp, vp, vp]
        L.zo_adamw_moments.argtypes = [i64] + [vp] * 7
        for f in ("zo_linear_attention", "zo_linear_attention_backward", "zo_linear_attention_step", "zo_layer_norm",
                  "zo_layer_norm_backward", "zo_adamw", "zo_adamw_moments"):
            getattr(L, f).restype = C.c_int
        _lib = L
    return _lib


def _check(st: int):
    if st:
        zo._check(st)


_current_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(like: torch.Tensor):
    """torch's current raw stream on like's device."""
    if _current_stream is not None:
        return _current_stream(like.get_device())
    return torch.cuda.current_stream(like.device).cuda_stream


def _device(t: torch.Tensor, name: str, dtype=None, like: torch.Tensor | None = None):
    if not isinstance(t, torch.Tensor) or t.get_device() < 0:
        raise ValueError(f"{name} must be a device tensor")
    if dtype is None:
        if t.dtype not in _DTYPES:
            raise ValueError(f"{name} must be float32 or bfloat16, got {t.dtype}")
    elif t.dtype is not dtype:
        raise ValueError(f"{name} must be {dtype}, got {t.dtype}")
    if like is not None and t.get_device() != like.get_device():
        raise ValueError(f"{name} is on {t.device}, not on {like.device}")


_recording = torch.is_grad_enabled


def _refuse_gradients():
    """For a call whose inputs require gradients while torch records: its outputs would silently carry none."""
    raise ValueError("inputs that require gradients: torch's autograd does not see the layers' calls; call them under "
                     "torch.no_grad() and their backward functions for the gradients")


def _flat(t: torch.Tensor | None, name: str, dtype, shape, like: torch.Tensor):
    """The address of a contiguous tensor of a given shape, or None."""
    if t is None:
        return None
    if not isinstance(t, torch.Tensor) or t.dtype is not dtype or t.get_device() != like.get_device():
        _device(t, name, dtype, like)
    if t.shape != shape:
        raise ValueError(f"{name} must be {list(shape)}, got {list(t.shape)}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t.data_ptr()


# ---- linear attention ----

def _heads(t: torch.Tensor, name: str, shape, like: torch.Tensor) -> bytes:
    """zo_heads of a tensor of a given shape, like's type and device."""
    if not isinstance(t, torch.Tensor) or t.dtype is not like.dtype or t.get_device() != like.get_device():
        raise ValueError(f"{name} must be a {like.dtype} tensor on {like.device}")
    if t.shape != shape:
        raise ValueError(f"{name} must be {list(shape)}, got {list(t.shape)}")
    st = t.stride()
    if st[-1] != 1 and shape[-1] != 1:
        raise ValueError(f"the values of a head must be contiguous in {name}")
    return _HEADS.pack(t.data_ptr(), st[0], st[1] if len(st) == 4 else 0, st[-2])


def _sizes(q, k, v, dims: int, scale):
    """(B, T, Hq, Hkv, Dk, Dv, zo_linattn, q's, k's and v's zo_heads) of tensors [B, T, heads, dim], or
    [B, heads, dim]."""
    _device(q, "q")
    qs, ks, vs = q.shape, k.shape, v.shape
    if not len(qs) == len(ks) == len(vs) == dims:
        raise ValueError(f"q, k and v must have {dims} dimensions")
    B, T = qs[0], qs[1] if dims == 4 else 1
    Hq, Dk, Hkv, Dv = qs[-2], qs[-1], vs[-2], vs[-1]
    if Hkv < 1 or Hq % Hkv:
        raise ValueError(f"{Hq} query heads are no multiple of {Hkv} key/value heads")
    lead = (B, T) if dims == 4 else (B,)
    return (B, T, Hq, Hkv, Dk, Dv,
            _SHAPE.pack(B, T, Hq, Hkv, Dk, Dv, _DTYPES[q.dtype], Dk ** -0.5 if scale is None else scale),
            _heads(q, "q", qs, q), _heads(k, "k", (*lead, Hkv, Dk), q), _heads(v, "v", (*lead, Hkv, Dv), q))


def _new_heads(like: torch.Tensor, *shape):
    """A new contiguous tensor [B, T, heads, dim] (or [B, heads, dim]) of like's type, and its zo_heads."""
    t = like.new_empty(shape)
    H, D = shape[-2:]
    return t, _HEADS.pack(t.data_ptr(), (shape[1] if len(shape) == 4 else 1) * H * D, H * D, D)


def _workspace(given: torch.Tensor | None, need: int, like: torch.Tensor):
    """(tensor or None, its address, its bytes)."""
    if given is None:
        if need == 0:
            return None, None, 0
        given = torch.empty(need, dtype=torch.uint8, device=like.device)
    else:
        _device(given, "workspace", torch.uint8, like)
        if not given.is_contiguous():
            raise ValueError("workspace must be contiguous")
    return given, given.data_ptr(), given.numel()


def linear_attention_workspace_bytes(B: int, T: int, q_heads: int, kv_heads: int, key_dim: int, value_dim: int,
                                     dtype=torch.float32, backward: bool = False) -> int:
    s = _SHAPE.pack(B, T, q_heads, kv_heads, key_dim, value_dim, _DTYPES[dtype], 1.0)
    return int(lib().zo_linear_attention_workspace_bytes(s, int(backward)))


def linear_attention(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, log_decay: torch.Tensor,
                     scale: float | None = None, initial_state: torch.Tensor | None = None,
                     lengths: torch.Tensor | None = None, return_state: bool = False,
                     out: torch.Tensor | None = None, final_state: torch.Tensor | None = None,
                     workspace: torch.Tensor | None = None, stream=None):
    """Returns (o, final state or None), asynchronously.

    q [B, T, Hq, Dk], k [B, T, Hkv, Dk], v [B, T, Hkv, Dv] fp32 or bf16, any strides with
    contiguous heads; log_decay fp32 [Hkv]; scale defaults to Dk ** -0.5; states fp32
    [B, Hkv, Dk, Dv]; lengths int32 [B] or None (all T). The final state is returned with
    return_state, or written into final_state (if that overlaps initial_state, its values are copied first).
    out may lie in any strides, but shares no memory with q, k and v."""
    if stream is not None:
        return _beside(stream, linear_attention, q, k, v, log_decay, scale, initial_state, lengths, return_state, out,
                       final_state, workspace)
    L = lib()
    B, T, Hq, Hkv, Dk, Dv, s, hq, hk, hv = _sizes(q, k, v, 4, scale)
    if _recording() and (q.requires_grad or k.requires_grad or v.requires_grad
                         or getattr(initial_state, "requires_grad", False)):
        _refuse_gradients()
    states = (B, Hkv, Dk, Dv)
    o, ho = _new_heads(q, B, T, Hq, Dv) if out is None else (out, _heads(out, "out", (B, T, Hq, Dv), q))
    f32 = torch.float32
    if final_state is None:
        if return_state:
            final_state = torch.empty(states, dtype=f32, device=q.device)
    elif initial_state is not None and abs(final_state.data_ptr() - initial_state.data_ptr()) < 4 * B * Hkv * Dk * Dv:
        # (shared, or in part) the kernels read the one while they write the other
        initial_state = initial_state.clone()
    ws, wp, wn = _workspace(workspace, L.zo_linear_attention_workspace_bytes(s, 0), q)
    _check(L.zo_linear_attention(
        s, hq, hk, hv, ho, _flat(log_decay, "log_decay", f32, (Hkv,), q),
        _flat(lengths, "lengths", torch.int32, (B,), q), _flat(initial_state, "initial_state", f32, states, q),
        _flat(final_state, "final_state", f32, states, q), wp, wn, _stream(q)))
    return o, final_state


def linear_attention_backward(do: torch.Tensor, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor,
                              log_decay: torch.Tensor, scale: float | None = None,
                              initial_state: torch.Tensor | None = None, lengths: torch.Tensor | None = None,
                              dfinal_state: torch.Tensor | None = None, return_dinitial: bool | None = None,
                              dq: torch.Tensor | None = None, dk: torch.Tensor | None = None,
                              dv: torch.Tensor | None = None, workspace: torch.Tensor | None = None, stream=None):
    """Returns (dq, dk, dv, dinitial_state or None) for the output's gradient do
    [B, T, Hq, Dv] and the final state's dfinal_state (None: zeros), asynchronously.
    The initial state's gradient is computed when one was given, or as return_dinitial says.
    dq, dk and dv (slices of one buffer, if wanted) share no memory with the inputs."""
    if stream is not None:
        return _beside(stream, linear_attention_backward, do, q, k, v, log_decay, scale, initial_state, lengths,
                       dfinal_state, return_dinitial, dq, dk, dv, workspace)
    L = lib()
    B, T, Hq, Hkv, Dk, Dv, s, hq, hk, hv = _sizes(q, k, v, 4, scale)
    states = (B, Hkv, Dk, Dv)
    dq, hdq = _new_heads(q, B, T, Hq, Dk) if dq is None else (dq, _heads(dq, "dq", (B, T, Hq, Dk), q))
    dk, hdk = _new_heads(q, B, T, Hkv, Dk) if dk is None else (dk, _heads(dk, "dk", (B, T, Hkv, Dk), q))
    dv, hdv = _new_heads(q, B, T, Hkv, Dv) if dv is None else (dv, _heads(dv, "dv", (B, T, Hkv, Dv), q))
    if return_dinitial is None:
        return_dinitial = initial_state is not None
    f32 = torch.float32
    dinitial = torch.empty(states, dtype=f32, device=q.device) if return_dinitial else None
    ws, wp, wn = _workspace(workspace, L.zo_linear_attention_workspace_bytes(s, 1), q)
    _check(L.zo_linear_attention_backward(
        s, _heads(do, "do", (B, T, Hq, Dv), q), hq, hk, hv, hdq, hdk, hdv,
        _flat(log_decay, "log_decay", f32, (Hkv,), q), _flat(lengths, "lengths", torch.int32, (B,), q),
        _flat(initial_state, "initial_state", f32, states, q), _flat(dfinal_state, "dfinal_state", f32, states, q),
        _flat(dinitial, "dinitial", f32, states, q), wp, wn, _stream(q)))
    return dq, dk, dv, dinitial


def linear_attention_step(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, log_decay: torch.Tensor,
                          state: torch.Tensor, scale: float | None = None, slots: torch.Tensor | None = None,
                          out: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """One token for each of B sequences: q [B, Hq, Dk], k [B, Hkv, Dk], v [B, Hkv, Dv] -> o
    [B, Hq, Dv] (asynchronous); state fp32 [n, Hkv, Dk, Dv] is updated in place. slots (int32
    [B], no two alike) names each sequence's state in it, -1 a sequence without one (its
    output is zero); None: sequence b's is state[b]. out shares no memory with q, k and v."""
    if stream is not None:
        return _beside(stream, linear_attention_step, q, k, v, log_decay, state, scale, slots, out)
    L = lib()
    B, _, Hq, Hkv, Dk, Dv, s, hq, hk, hv = _sizes(q, k, v, 3, scale)
    if _recording() and (q.requires_grad or k.requires_grad or v.requires_grad
                         or getattr(state, "requires_grad", False)):
        _refuse_gradients()
    n = state.shape[0]
    if n > 0x7fffffff:
        raise ValueError("state must hold fewer than 2^31 states")
    o, ho = _new_heads(q, B, Hq, Dv) if out is None else (out, _heads(out, "out", (B, Hq, Dv), q))
    _check(L.zo_linear_attention_step(
        s, hq, hk, hv, ho, _flat(log_decay, "log_decay", torch.float32, (Hkv,), q),
        _flat(state, "state", torch.float32, (n, Hkv, Dk, Dv), q), n, _flat(slots, "slots", torch.int32, (B,), q),
        _stream(q)))
    return o


# ---- layer norm ----

def _rows(t: torch.Tensor, name: str, shape=None, like: torch.Tensor | None = None):
    """(rows, D, stride between rows) of [..., D], whose rows must lie at equal distances."""
    _device(t, name, None if like is None else like.dtype, like)
    if shape is not None and t.shape != shape:
        raise ValueError(f"{name} must be {list(shape)}, got {list(t.shape)}")
    if t.dim() < 1 or t.shape[-1] < 1:
        raise ValueError(f"{name} must be [..., D] with D >= 1")
    D = t.shape[-1]
    if t.is_contiguous():
        return t.numel() // D, D, D
    if t.stride(-1) != 1 and D != 1:
        raise ValueError(f"the rows of {name} must be contiguous")
    try:
        flat = t.view(-1, D)
    except RuntimeError:
        raise ValueError(f"the rows of {name} must lie at equal distances") from None
    return flat.shape[0], D, flat.stride(0)


def _norm_params(weight, bias, D, like):
    w = weight if weight is not None else bias
    wtype = like.dtype if w is None else w.dtype
    if wtype not in _DTYPES:
        raise ValueError(f"weight and bias must be float32 or bfloat16, got {wtype}")
    return (_DTYPES[wtype], _flat(weight, "weight", wtype, (D,), like), _flat(bias, "bias", wtype, (D,), like))


def layer_norm(x: torch.Tensor, weight: torch.Tensor | None = None, bias: torch.Tensor | None = None,
               eps: float = 1e-5, out: torch.Tensor | None = None, stream=None):
    """Layer norm over the last dimension: returns (y, mean, rstd), asynchronously; y of x's
    type and shape (out, which may be x, or a new tensor), mean and rstd fp32 [rows] for the
    backward pass. weight and bias [D], fp32 or bf16, or None."""
    if stream is not None:
        return _beside(stream, layer_norm, x, weight, bias, eps, out)
    L = lib()
    rows, D, xs = _rows(x, "x")
    wtype, w, b = _norm_params(weight, bias, D, x)
    if _recording() and (x.requires_grad or (weight is not None and weight.requires_grad)
                         or (bias is not None and bias.requires_grad)):
        _refuse_gradients()
    dev = x.device
    y = torch.empty(x.shape, dtype=x.dtype, device=dev) if out is None else out
    ys = D if out is None else _rows(y, "out", x.shape, x)[2]
    mean = torch.empty(rows, dtype=torch.float32, device=dev)
    rstd = torch.empty(rows, dtype=torch.float32, device=dev)
    _check(L.zo_layer_norm(_DTYPES[x.dtype], wtype, rows, D, x.data_ptr(), xs, w, b, eps, y.data_ptr(), ys,
                           mean.data_ptr(), rstd.data_ptr(), _stream(x)))
    return y, mean, rstd


def layer_norm_workspace_bytes(rows: int, D: int) -> int:
    return int(lib().zo_layer_norm_workspace_bytes(rows, D))


def layer_norm_backward(dy: torch.Tensor, x: torch.Tensor, weight: torch.Tensor | None, mean: torch.Tensor,
                        rstd: torch.Tensor, out: torch.Tensor | None = None, workspace: torch.Tensor | None = None,
                        stream=None):
    """Returns (dx, dweight, dbias), asynchronously: dx of x's type and shape (out, which may
    be dy or x, or a new tensor), dweight and dbias fp32 [D], summed in a fixed order."""
    if stream is not None:
        return _beside(stream, layer_norm_backward, dy, x, weight, mean, rstd, out, workspace)
    L = lib()
    rows, D, xs = _rows(x, "x")
    dys = _rows(dy, "dy", x.shape, x)[2]
    wtype, w, _ = _norm_params(weight, None, D, x)
    mp = _flat(mean, "mean", torch.float32, (rows,), x)
    rp = _flat(rstd, "rstd", torch.float32, (rows,), x)
    dev = x.device
    dx = torch.empty(x.shape, dtype=x.dtype, device=dev) if out is None else out
    dxs = D if out is None else _rows(dx, "out", x.shape, x)[2]
    dw = torch.empty(D, dtype=torch.float32, device=dev)
    db = torch.empty(D, dtype=torch.float32, device=dev)
    ws, wp, wn = _workspace(workspace, L.zo_layer_norm_workspace_bytes(rows, D), x)
    _check(L.zo_layer_norm_backward(_DTYPES[x.dtype], wtype, rows, D, dy.data_ptr(), dys, x.data_ptr(), xs, w, mp, rp,
                                    dx.data_ptr(), dxs, dw.data_ptr(), db.data_ptr(), wp, wn, _stream(x)))
    return dx, dw, db


# ---- AdamW ----

_shape_of, _dtype_of = attrgetter("shape"), attrgetter("dtype")
_device_of, _contiguous, _address = torch.Tensor.get_device, torch.Tensor.is_contiguous, torch.Tensor.data_ptr


class AdamW:
    """AdamW over a list of parameter tensors, all in one launch for up to 64 of them.

    params: contiguous device tensors, fp32 or bf16, updated in place, that share no memory (a tied tensor
    is given once, with the sum of its gradients). bf16 values are rounded to nearest, which loses
    changes under 2^-9 of them: where those count, keep fp32 parameters and cast them. weight_decay: one
    number, or one for each tensor. state_bits: 32 (m and v fp32) or 8 (m int8 and v uint8
    codes with m_scale and v_scale, the largest values of blocks of 256: see
    zo_layers.h). The moments of tensor i begin at offsets[i] of the flat m and v and take
    whole blocks. step_count is the number of steps done; a checkpoint is step_count, m, v
    and the scales, to be copied back into the same buffers (m.copy_(...)). A step captured
    into a HIP graph replays with the learning rate and the bias corrections of its capture."""

    def __init__(self, params, lr: float = 1e-3, betas=(0.9, 0.999), eps: float = 1e-8, weight_decay=0.0,
                 state_bits: int = 32):
        self.params = list(params)
        if not self.params:
            raise ValueError("no parameters")
        if state_bits not in (32, 8):
            raise ValueError("state_bits must be 32 or 8")
        first = self.params[0]
        for i, p in enumerate(self.params):
            _device(p, f"params[{i}]", None, first)
            if not p.is_contiguous():
                raise ValueError(f"params[{i}] must be contiguous")
        ends = sorted((p.data_ptr(), p.data_ptr() + p.numel() * p.element_size(), i)
                      for i, p in enumerate(self.params) if p.numel())
        for a, b in zip(ends, ends[1:]):
            if b[0] < a[1]:
                raise ValueError(f"params[{a[2]}] and params[{b[2]}] share memory: a tied tensor is given once")
        decay = list(weight_decay) if isinstance(weight_decay, (list, tuple)) else [weight_decay] * len(self.params)
        if len(decay) != len(self.params):
            raise ValueError(f"{len(decay)} weight decays for {len(self.params)} tensors")
        self.lr, self.betas, self.eps, self._bits, self.step_count = lr, tuple(betas), eps, state_bits, 0
        self.offsets, at = [], 0
        for p in self.params:
            self.offsets.append(at)
            at += (p.numel() + BLOCK - 1) // BLOCK * BLOCK
        dev = first.device
        self._m_scale = self._v_scale = None
        if state_bits == 8:
            self._m = torch.zeros(at, dtype=torch.int8, device=dev)
            self._v = torch.zeros(at, dtype=torch.uint8, device=dev)
            self._m_scale = torch.zeros(at // BLOCK, dtype=torch.float32, device=dev)
            self._v_scale = torch.zeros(at // BLOCK, dtype=torch.float32, device=dev)
        else:
            self._m = torch.zeros(at, dtype=torch.float32, device=dev)
            self._v = torch.zeros(at, dtype=torch.float32, device=dev)
        self._leaves = [p for p in self.params if p.requires_grad]
        self._shapes = [p.shape for p in self.params]
        self._dtypes = [p.dtype for p in self.params]
        self._devices = [first.get_device()] * len(self.params)
        self._table = (_Tensor * len(self.params))(
            *(_Tensor(p.data_ptr(), None, p.numel(), o, float(d), _DTYPES[p.dtype], zo.FP32)
              for p, o, d in zip(self.params, self.offsets, decay)))

    # the kernels trust the buffers' types and sizes: they can be written into, not exchanged
    state_bits = property(lambda self: self._bits)
    m = property(lambda self: self._m)
    v = property(lambda self: self._v)
    m_scale = property(lambda self: self._m_scale)
    v_scale = property(lambda self: self._v_scale)

    def step(self, grads, grad_scale: torch.Tensor | None = None, skipped: torch.Tensor | None = None, stream=None):
        """One step (asynchronous) with one contiguous fp32 or bf16 gradient for each tensor.
        grad_scale (device fp32 [1]) multiplies them; if it is not finite the step changes
        nothing, and skipped (device int32 [1]) is set to 1, else to 0. step_count goes up
        either way, and with it the bias corrections; who reads skipped may take the step off again."""
        grads = list(grads)
        if stream is not None:
            _beside(stream, self.step, grads, grad_scale, skipped)
            return _record(stream, (self.params, self._m, self._v, self._m_scale, self._v_scale))
        if len(grads) != len(self.params):
            raise ValueError(f"{len(grads)} gradients for {len(self.params)} tensors")
        like, params = self._m, self.params
        # whole lists at a time: a check of each tensor in turn takes a third longer
        if (list(map(_shape_of, params)) != self._shapes or list(map(_dtype_of, params)) != self._dtypes
                or list(map(_device_of, params)) != self._devices or not all(map(_contiguous, params))):
            raise ValueError("a parameter's type, shape, layout or device is not what it was when AdamW was made")
        kinds = list(map(_DTYPES.get, map(_dtype_of, grads)))
        if (list(map(_shape_of, grads)) != self._shapes or None in kinds
                or list(map(_device_of, grads)) != self._devices or not all(map(_contiguous, grads))):
            for i, (g, shape) in enumerate(zip(grads, self._shapes)):
                if g.shape != shape or g.dtype not in _DTYPES or g.device != like.device or not g.is_contiguous():
                    raise ValueError(f"gradients must be contiguous fp32 or bf16 tensors of their parameters' shapes on "
                                     f"{like.device}: grads[{i}] is {g.dtype} {list(g.shape)} on {g.device} for "
                                     f"{list(shape)}")
        for t, p, g, kind in zip(self._table, map(_address, params), map(_address, grads), kinds):
            t.param, t.grad, t.gdtype = p, g, kind
        gs = _flat(grad_scale, "grad_scale", torch.float32, (1,), like)
        sk = _flat(skipped, "skipped", torch.int32, (1,), like)
        cfg = _AdamWConfig(self.lr, self.betas[0], self.betas[1], self.eps, self.step_count + 1, self._bits)
        eight = self._bits == 8
        _check(lib().zo_adamw(C.byref(cfg), self._table, len(grads), like.data_ptr(), self._v.data_ptr(),
                              self._m_scale.data_ptr() if eight else None,
                              self._v_scale.data_ptr() if eight else None,
                              gs, sk, _stream(like)))
        self.step_count += 1
        if self._leaves:  # what torch has recorded on them is about the values before
            torch.autograd.graph.increment_version(self._leaves)

    def moments(self, stream=None):
        """The flat fp32 (m, v): the buffers themselves (32 bits), or the values that the codes stand for."""
        if self._bits == 32:
            return self.m, self.v
        if stream is not None:
            _record(stream, (self._m, self._v, self._m_scale, self._v_scale))
            return _beside(stream, self.moments)
        m = torch.empty(self.m.numel(), dtype=torch.float32, device=self.m.device)
        v = torch.empty_like(m)
        _check(lib().zo_adamw_moments(m.numel(), self.m.data_ptr(), self.v.data_ptr(), self.m_scale.data_ptr(),
                                      self.v_scale.data_ptr(), m.data_ptr(), v.data_ptr(), _stream(m)))
        return m, v
