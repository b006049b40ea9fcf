"""The operators around a language-model layer's attention: layer norm, rotary
positions and causal linear attention with a decay per head.

They share the attention calls' layout, ``[n, heads, N, d]``, but take any
strides on the first three axes (``project_qkv``'s results, token-major tensors,
slices of a wider projection); ``layer_norm`` takes rows of any shape in front that
one stride steps along.  Like the other calls they run on the current
stream or on ``stream``, raise ``ValueError`` for tensors that do not fit and
``NystraError`` for what the C ABI refuses, and have no CPU path.

The calls record no autograd graph: each forward call has its backward call
beside it, for use inside a ``torch.autograd.Function`` or a training loop of
one's own.  Inputs that require gradients are refused while grad mode is on, and
inputs with forward-mode tangents always, rather than silently cut off.

A result is allocated on the stream that the call runs on.  An input of another
stream's is not recorded on it (``Tensor.record_stream`` does that): as with torch's
own calls, it has to be there when the call runs, and to stay until it has.
"""
from __future__ import annotations

import ctypes
import functools
import math

import torch
from torch.autograd import forward_ad

from .binding import _DTYPE_CODE, NYSTRA_OK, NystraError, _stream_ptr, lib

ROTARY_LAYOUTS = {"half": 0, "interleaved": 1}
LINEAR_MAX_D, ROTARY_MAX_D = 128, 256
_INT_MAX = 2 ** 31 - 1


# What a call checks of its tensors' shapes, strides and dtypes, and derives from them alone, is kept by
# those (`_sig`) and not worked out again: the `_*_plan` functions.  A refusal is not kept.
_plan = functools.lru_cache(maxsize=4096)


def _sig(t):
    return None if t is None else (t.shape, t.stride(), t.dtype)


def _array(strides):
    """Strides as the C ABI takes them; the calls only read them."""
    return (ctypes.c_longlong * len(strides))(*strides)


def _recorded(t) -> bool:
    """Whether autograd would record a graph for t, or carry a tangent of it along."""
    if t.requires_grad and torch.is_grad_enabled():
        return True
    # (a Function's forward method is called with tangents that are its jvp method's to carry on)
    return (forward_ad._current_level >= 0 and torch._C._is_fwd_grad_enabled()
            and forward_ad.unpack_dual(t).tangent is not None)


def _tensors(*ts):
    """Checks that hold for every tensor of a call: one CUDA device, no gradients to record."""
    device = ts[0].get_device()
    for t in ts:
        if t is None:
            continue
        if t.get_device() != device or not t.is_cuda:
            raise ValueError("tensors must be on one CUDA device (no CPU path)")
        if _recorded(t):
            raise ValueError("an input requires gradients or has a tangent, and these calls record no autograd graph: "
                             "call under torch.no_grad() or in an autograd.Function, with the *_backward call for its "
                             "gradient")


def _dtype(*sigs) -> int:
    kind = sigs[0][2]
    if any(t is not None and t[2] != kind for t in sigs):
        raise ValueError("tensors must share their dtype")
    if kind not in _DTYPE_CODE:
        raise ValueError(f"unsupported dtype {kind}")
    return _DTYPE_CODE[kind]


def _dense(shape, stride) -> bool:
    step = 1
    for size, st in zip(reversed(shape), reversed(stride)):
        if size != 1 and st != step:
            return 0 in shape
        step *= size
    return True


def _shaped(name, t, shape, kind=None):
    """A strided tensor of the given shape (features adjacent); with `kind` a contiguous one of that dtype."""
    if tuple(t[0]) != shape:
        raise ValueError(f"{name} must be {list(shape)}")
    if kind is not None and (t[2] != kind or not _dense(t[0], t[1])):
        raise ValueError(f"{name} must be contiguous, of {kind}")
    if kind is None and t[1][-1] != 1 and shape[-1] > 1 and 0 not in shape:
        raise ValueError(f"{name}: features (the last axis) must be adjacent")


def _sizes_fit(**sizes):
    """The C entries take these as 32-bit integers, and ctypes would cut a larger one off without a word."""
    for name, size in sizes.items():
        if size > _INT_MAX:
            raise ValueError(f"{name} = {size}: at most {_INT_MAX}")


def _on(x, stream, call):
    """``call(stream address)`` with x's device and the stream current, for allocations as well as for the launch."""
    device = x.get_device()
    if stream is None and device == torch.cuda.current_device():
        return call(torch._C._cuda_getCurrentRawStream(device))
    with torch.cuda.device(device):
        if stream is None:
            return call(torch._C._cuda_getCurrentRawStream(device))
        s = stream if isinstance(stream, torch.cuda.Stream) else torch.cuda.ExternalStream(_stream_ptr(stream))
        if s.device_index != device:
            raise ValueError("the stream must be of the tensors' device")
        with torch.cuda.stream(s):
            return call(s.cuda_stream)


def _empty_like(t):
    """Contiguous, whatever t is; cheaper than by its shape where t is contiguous."""
    return torch.empty_like(t) if t.is_contiguous() else torch.empty(t.shape, dtype=t.dtype, device=t.device)


def _empty(shape, like, dtype=None):
    return torch.empty(shape, dtype=like.dtype if dtype is None else dtype, device=like.device)


def _raise(rc: int, where: str):
    if rc != NYSTRA_OK:
        raise NystraError(int(rc), where)


def _ptr(t) -> int | None:
    return None if t is None else t.data_ptr()


def _result(shape, like, need):
    """A result and a workspace of ``need`` bytes for the call that fills it: (result, workspace, its address).

    Outside a stream capture the workspace is the allocator's, free again in
    stream order.  A captured graph goes on using it after the call, and who began the
    capture cannot be told (only the allocator's own captures keep such memory), so
    there it lies behind the result in one storage."""
    if not need:
        return _empty(shape, like), None, None
    if not torch.cuda.is_current_stream_capturing():
        ws = _empty(need, like, torch.uint8)
        return _empty(shape, like), ws, ws.data_ptr()
    size = -(-math.prod(shape) * like.element_size() // 512) * 512
    both = _empty(size + need, like, torch.uint8)
    return _empty(0, like).set_(both.untyped_storage(), 0, shape), None, both.data_ptr() + size


# ------------------------------------------------------------------ layer norm
def _rows(shape, stride):
    """(rows, stride between rows) of a tensor whose leading axes step evenly."""
    if len(shape) < 1:
        raise ValueError("expected at least one axis")
    C, rows = shape[-1], math.prod(shape[:-1])
    if C > 1 and rows and stride[-1] != 1:
        raise ValueError("features (the last axis) must be adjacent")
    step = None
    reach = 1  # rows that the axes behind this one hold
    for size, st in zip(reversed(shape[:-1]), reversed(stride[:-1])):
        if size == 1 or not rows:
            continue
        if step is None:
            step = st
        elif st != step * reach:
            raise ValueError("the axes in front of the features must step evenly (one row stride)")
        reach *= size
    return rows, C if step is None else step


@_plan
def _norm_plan(x, weight, bias, out, dy):
    """(dtype codes of x and of the parameters, rows, C, row strides of x, out, dy, bytes of the backward workspace)."""
    dt = _dtype(x, out, dy)
    C = x[0][-1] if len(x[0]) else 0
    _sizes_fit(C=C)
    kind = None
    for p in (weight, bias):
        if p is None:
            continue
        if len(p[0]) != 1 or p[0][0] != C or not _dense(p[0], p[1]):
            raise ValueError(f"weight and bias must be contiguous, of {C} values")
        if p[2] not in (torch.float32, x[2]) or (kind is not None and p[2] != kind):
            raise ValueError("weight and bias must share a dtype: fp32, or the input's")
        kind = p[2]
    rows, xs = _rows(x[0], x[1])
    strides = []
    for name, t in (("out", out), ("dy", dy)):
        if t is not None and t[0] != x[0]:
            raise ValueError(f"{name} must have x's shape")
        strides.append(C if t is None else _rows(t[0], t[1])[1])
    need = lib().nystra_layer_norm_workspace(rows, C)
    if need < 0:
        raise NystraError(int(need), "nystra_layer_norm_workspace")
    return dt, _DTYPE_CODE[x[2] if kind is None else kind], rows, C, xs, *strides, need


def layer_norm(x: torch.Tensor, weight: torch.Tensor | None = None, bias: torch.Tensor | None = None,
               eps: float = 1e-5, out: torch.Tensor | None = None, return_stats: bool = False, stream=None):
    """Layer norm over the last axis of ``x`` ``[..., C]`` with optional ``weight``
    and ``bias`` ``[C]`` (fp32, or x's dtype).  ``out`` may be ``x`` itself.  With
    ``return_stats``: ``(y, mean, rstd)``, the two fp32 per row (NaN where C is 0),
    which ``layer_norm_backward`` reads."""
    _tensors(x, weight, bias, out)
    dt, wdt, rows, C, xs, ys, _, _ = _norm_plan(_sig(x), _sig(weight), _sig(bias), _sig(out), None)

    def call(st):
        y = _empty_like(x) if out is None else out
        mean = rstd = None
        if return_stats:
            mean = _empty(x.shape[:-1], x, torch.float32)
            rstd = torch.empty_like(mean)
            if not C:  # the C entry writes nothing where rows have no values, whose mean is no number
                mean.fill_(math.nan)
                rstd.fill_(math.nan)
        _raise(lib().nystra_layer_norm(x.data_ptr(), xs, _ptr(weight), _ptr(bias), y.data_ptr(), ys, _ptr(mean),
                                       _ptr(rstd), rows, C, eps, dt, wdt, st), "nystra_layer_norm")
        return (y, mean, rstd) if return_stats else y

    return _on(x, stream, call)


def layer_norm_backward(dy: torch.Tensor, x: torch.Tensor, mean: torch.Tensor, rstd: torch.Tensor,
                        weight: torch.Tensor | None = None, stream=None, bias: torch.Tensor | None = None):
    """Gradients of ``layer_norm``: ``(dx, dweight, dbias)`` from the output's
    gradient, the input and the saved statistics.  Without ``weight`` the last two
    are None, but for ``dbias`` where ``bias`` is given (which is else not needed)."""
    _tensors(dy, x, mean, rstd, weight, bias)
    dt, wdt, rows, C, xs, _, ds, need = _norm_plan(_sig(x), _sig(weight), _sig(bias), None, _sig(dy))
    for t in (mean, rstd):
        if t.shape != x.shape[:-1] or t.dtype != torch.float32 or not t.is_contiguous():
            raise ValueError("mean and rstd must be contiguous fp32 tensors of x's shape without the last axis")

    def call(st):
        dx = _empty_like(x)
        dw = db = ws = wp = None
        if weight is not None:
            both, ws, wp = _result((2, C), weight, need)
            dw, db = both.unbind(0)
        elif bias is not None:
            db, ws, wp = _result((C,), bias, need)
        _raise(lib().nystra_layer_norm_backward(dy.data_ptr(), ds, x.data_ptr(), xs, mean.data_ptr(), rstd.data_ptr(),
                                                _ptr(weight), dx.data_ptr(), C, _ptr(dw), _ptr(db), rows, C, dt, wdt,
                                                wp, need, st), "nystra_layer_norm_backward")
        return dx, dw, db

    return _on(x, stream, call)


# ------------------------------------------------------------------ rotary positions
def rotary_frequencies(rotary_dim: int, base: float = 10000.0, scaling: str = "none", factor: float = 1.0,
                       original_length: int | None = None, beta_fast: float = 32.0, beta_slow: float = 1.0,
                       device="cuda"):
    """``(inv_freq, amplitude)`` for ``rotary``: radians per position of each of the
    ``rotary_dim / 2`` pairs (fp64), ``base^(-2 i / rotary_dim)``, changed for
    contexts ``factor`` times longer than trained:

    - "none": as trained;
    - "linear": positions divided by ``factor`` (position interpolation, arXiv 2306.15595);
    - "ntk": the base grows by ``factor^(r / (r - 2))``, so that the slowest pair is
      interpolated by ``factor`` and the fastest not at all;
    - "yarn" (arXiv 2309.00071): pairs that turn fewer than ``beta_slow`` times over
      ``original_length`` are interpolated, those of more than ``beta_fast`` turns
      are not, with a linear ramp between, and queries and keys grow by
      ``0.1 ln(factor) + 1``.
    """
    if rotary_dim < 0 or rotary_dim % 2 or rotary_dim > ROTARY_MAX_D:
        raise ValueError(f"rotary_dim must be even, 0..{ROTARY_MAX_D}")
    if not (base > 1 and math.isfinite(base)) or not (factor >= 1 and math.isfinite(factor)):
        raise ValueError("base must be above 1 and factor at least 1")
    i = torch.arange(rotary_dim // 2, dtype=torch.float64)
    amplitude = 1.0
    if scaling == "ntk" and rotary_dim > 2:
        base = base * factor ** (rotary_dim / (rotary_dim - 2))
    inv = torch.exp(-math.log(base) * 2 * i / max(rotary_dim, 1))
    if scaling == "linear":
        inv = inv / factor
    elif scaling == "yarn":
        if original_length is None or original_length < 1 or not beta_fast > beta_slow > 0:
            raise ValueError("yarn needs original_length >= 1 and beta_fast > beta_slow > 0")

        def pair_of(turns):  # the (fractional) pair that turns so often over the original length
            return rotary_dim * math.log(original_length / (turns * 2 * math.pi)) / (2 * math.log(base))

        lo = max(math.floor(pair_of(beta_fast)), 0)
        hi = min(math.ceil(pair_of(beta_slow)), rotary_dim - 1)
        ramp = ((i - lo) / max(hi - lo, 0.001)).clamp(0, 1)
        inv = inv * (1 - ramp) + inv / factor * ramp
        amplitude = 0.1 * math.log(factor) + 1.0
    elif scaling not in ("none", "ntk"):
        raise ValueError(f"unknown scaling {scaling!r}")
    return inv.to(device), amplitude


@_plan
def _rotary_plan(q, k, inv_freq, positions, out_q, out_k, layout):
    """(per tensor its strides, its result's and its heads; the C call's sizes)."""
    dt = _dtype(q, k, out_q, out_k)
    for t in (q,) if k is None else (q, k):
        if len(t[0]) != 4:
            raise ValueError("expected [n, heads, N, d]")
    n, _, N, d = q[0]
    rows = []
    for name, t, o in (("q", q, out_q), ("k", k, out_k)):
        if t is None:
            continue
        h = t[0][1]
        _shaped(name, t, (n, h, N, d))
        if o is not None:
            _shaped("out", o, (n, h, N, d))
        rows.append((_array(t[1][:3]), _array(o[1][:3] if o is not None else (h * N * d, N * d, d)), h))
    if len(inv_freq[0]) != 1:
        raise ValueError("inv_freq must have one axis")
    _shaped("inv_freq", inv_freq, tuple(inv_freq[0]), torch.float64)
    _sizes_fit(n=n, heads=max(x[2] for x in rows), N=N, d=d, rotary_dim=2 * inv_freq[0][0])
    if layout not in ROTARY_LAYOUTS:
        raise ValueError(f"unknown layout {layout!r}")
    bits = step = 0
    if positions is not None:
        shape, stride, kind = positions
        if kind not in (torch.int64, torch.int32):
            raise ValueError("positions must be int64 or int32")
        if tuple(shape) not in ((N,), (n, N)):
            raise ValueError(f"positions must be [{N}] or [{n}, {N}]")
        if N > 1 and stride[-1] != 1:
            raise ValueError("a sequence's positions must be adjacent")
        bits, step = (64 if kind == torch.int64 else 32), (stride[0] if len(shape) == 2 else 0)
    return rows, 2 * inv_freq[0][0], bits, step, n, N, d, ROTARY_LAYOUTS[layout], dt


def _rotary(q, k, inv_freq, positions, layout, amplitude, inverse, outs, stream):
    _tensors(q, k, inv_freq, positions, *outs)
    rows, r, bits, step, n, N, d, lay, dt = _rotary_plan(_sig(q), _sig(k), _sig(inv_freq), _sig(positions),
                                                         _sig(outs[0]), _sig(outs[1]), layout)

    def call(st):
        res, args = [], []
        for t, o, (ts, os, heads) in zip((q, k), outs, rows):
            o = _empty_like(t) if o is None else o
            res.append(o)
            args += [t.data_ptr(), ts, o.data_ptr(), os, heads]
        if k is None:
            args += [None, None, None, None, 0]
        _raise(lib().nystra_rotary(*args, inv_freq.data_ptr(), r, _ptr(positions), bits, step, amplitude, n, N, d, lay,
                                   int(bool(inverse)), dt, st), "nystra_rotary")
        return res

    return _on(q, stream, call)


def rotary(x: torch.Tensor, inv_freq: torch.Tensor, positions: torch.Tensor | None = None, layout: str = "half",
           amplitude: float = 1.0, inverse: bool = False, out: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """Rotary positions of ``x`` ``[n, heads, N, d]``: the first ``2 len(inv_freq)``
    features turn by ``positions * inv_freq`` (fp64, see ``rotary_frequencies``), the
    rest is copied.  ``positions``: int64 or int32 ``[N]`` or ``[n, N]``, None for
    0..N-1.  ``layout`` pairs feature i with ``i + r/2`` ("half") or 2i with 2i + 1
    ("interleaved").  ``inverse`` turns back, which is also the gradient: of
    ``y = rotary(x)``, ``dx = rotary(dy, inverse=True)``.  ``out`` may be ``x``."""
    return _rotary(x, None, inv_freq, positions, layout, amplitude, inverse, (out, None), stream)[0]


def rotary_qk(q: torch.Tensor, k: torch.Tensor, inv_freq: torch.Tensor, positions: torch.Tensor | None = None,
              layout: str = "half", amplitude: float = 1.0, inverse: bool = False, out=None, stream=None):
    """``rotary`` of queries and keys in one launch: ``(q', k')``.  Their numbers of
    heads may differ.  ``out`` may give the two results; ``(q, k)`` turns them in place,
    where they may be slices of one buffer but share no elements."""
    return tuple(_rotary(q, k, inv_freq, positions, layout, amplitude, inverse, (None, None) if out is None else out,
                         stream))


# ------------------------------------------------------------------ linear attention
def _sizes(q, v, axes):
    if len(q[0]) != axes or len(v[0]) != axes:
        raise ValueError("expected q, k [n, heads, N, d_k] and v [n, heads, N, d_v]" if axes == 4 else
                         "expected q, k [n, heads, d_k] and v [n, heads, d_v]")
    dk, dv = q[0][-1], v[0][-1]
    if not (1 <= dk <= LINEAR_MAX_D and 1 <= dv <= LINEAR_MAX_D):
        raise ValueError(f"d_k and d_v must lie in 1..{LINEAR_MAX_D}")
    _sizes_fit(**dict(zip(("n", "heads", "N"), q[0][:-1])))
    return tuple(q[0][:-1]), dk, dv


@_plan
def _linear_plan(q, k, v, dout, log_decay, state, lengths, dstate, out, backward):
    """(dtype code, n, heads, N, d_k, d_v, workspace bytes, strides of q, k, v, dout and of results as wide as q and v)."""
    dt = _dtype(q, k, v, dout, out)
    lead, dk, dv = _sizes(q, v, 4)
    n, h, N = lead
    for name, t, d in (("q", q, dk), ("k", k, dk), ("v", v, dv), ("dout", dout, dv), ("out", out, dv)):
        if t is not None:
            _shaped(name, t, lead + (d,))
    for name, t in (("state", state), ("dstate", dstate)):
        if t is not None:
            _shaped(name, t, (n, h, dk, dv), torch.float32)
    _shaped("log_decay", log_decay, (h,), torch.float32)
    if lengths is not None:
        _shaped("lengths", lengths, (n,), torch.int32)
    need = lib().nystra_linear_attention_workspace(n, h, N, dk, dv, dt, backward)
    if need < 0:
        raise NystraError(int(need), "nystra_linear_attention_workspace")
    strides = [None if t is None else _array(t[1][:3]) for t in (q, k, v, dout, out)]
    return (dt, n, h, N, dk, dv, need, *strides, _array((h * N * dk, N * dk, dk)), _array((h * N * dv, N * dv, dv)))


@_plan
def _step_plan(q, k, v, log_decay, state, state_out, out):
    dt = _dtype(q, k, v, out)
    lead, dk, dv = _sizes(q, v, 3)
    n, h = lead
    for name, t, d in (("q", q, dk), ("k", k, dk), ("v", v, dv), ("out", out, dv)):
        if t is not None:
            _shaped(name, t, lead + (d,))
    _shaped("state", state, (n, h, dk, dv), torch.float32)
    _shaped("state_out", state_out, (n, h, dk, dv), torch.float32)
    _shaped("log_decay", log_decay, (h,), torch.float32)
    return (dt, n, h, dk, dv, *(_array(t[1][:2]) for t in (q, k, v)), _array((h * dv, dv) if out is None else out[1][:2]))


def linear_attention(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, log_decay: torch.Tensor,
                     state: torch.Tensor | None = None, lengths: torch.Tensor | None = None,
                     scale: float | None = None, out: torch.Tensor | None = None, return_state: bool = False,
                     stream=None):
    """Causal linear attention with a decay ``exp(log_decay[h])`` per head (fp32
    ``[heads]``, not above 0): ``S_t = gamma S_{t-1} + k_t v_t^T``,
    ``out_t = scale q_t^T S_t`` with ``scale`` 1/sqrt(d_k) by default.

    ``q, k`` ``[n, heads, N, d_k]``, ``v`` ``[n, heads, N, d_v]``; ``state``
    ``[n, heads, d_k, d_v]`` fp32 is S_0 (zeros by default); ``lengths`` int32 ``[n]``:
    tokens of each sequence of a padded batch, whose rows behind come out zero.
    Returns ``out``, with ``return_state`` ``(out, state)`` behind each sequence's last
    token, for ``linear_attention_step`` or the next call.

    Values have to be finite (behind ``lengths`` anything may lie): one that is not makes
    the results of its 64 tokens and of all later ones of its sequence and head undefined.
    In 16 bits the masked scores and the state that meets the queries are rounded on the
    way, but for the scores of a sequence's first 64 tokens where no state enters it; and the
    state that is returned is summed more exactly than one that is only read on the way, so
    results with and without ``return_state`` may differ by roundings.

    In a stream capture with ``out`` given the call has no place for a workspace and
    does not split long sequences."""
    _tensors(q, k, v, log_decay, state, lengths, out)
    dt, n, h, N, dk, dv, need, qs, ks, vs, _, os, _, wide = _linear_plan(
        _sig(q), _sig(k), _sig(v), None, _sig(log_decay), _sig(state), _sig(lengths), None, _sig(out), 0)

    def call(st):
        ws = wp = None
        if out is None:
            o, ws, wp = _result((n, h, N, dv), q, need)
        else:
            o = out
            if need and not torch.cuda.is_current_stream_capturing():
                ws = _empty(need, q, torch.uint8)
                wp = ws.data_ptr()
        last = _empty((n, h, dk, dv), q, torch.float32) if return_state else None
        _raise(lib().nystra_linear_attention(
            q.data_ptr(), qs, k.data_ptr(), ks, v.data_ptr(), vs, o.data_ptr(), wide if out is None else os,
            log_decay.data_ptr(), _ptr(lengths), _ptr(state), _ptr(last), dk ** -0.5 if scale is None else scale, n, h,
            N, dk, dv, dt, wp, need, st), "nystra_linear_attention")
        return (o, last) if return_state else o

    return _on(q, stream, call)


def linear_attention_backward(dout: torch.Tensor, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor,
                              log_decay: torch.Tensor, state: torch.Tensor | None = None,
                              lengths: torch.Tensor | None = None, dstate: torch.Tensor | None = None,
                              scale: float | None = None, stream=None):
    """Gradients of ``linear_attention``: ``(dq, dk, dv, dstate_in)`` from the
    output's gradient and, where the final state was used, ``dstate``, its gradient.
    ``dstate_in``, the gradient of ``state``, is None where ``state`` is.  The decay
    has none: it is a constant of the head."""
    _tensors(dout, q, k, v, log_decay, state, lengths, dstate)
    dt, n, h, N, dk, dv, need, qs, ks, vs, ds, _, kwide, vwide = _linear_plan(
        _sig(q), _sig(k), _sig(v), _sig(dout), _sig(log_decay), _sig(state), _sig(lengths), _sig(dstate), None, 1)

    def call(st):
        gq, ws, wp = _result((n, h, N, dk), q, need)
        gk, gv = _empty((n, h, N, dk), q), _empty((n, h, N, dv), q)
        first = torch.empty_like(state) if state is not None else None
        _raise(lib().nystra_linear_attention_backward(
            dout.data_ptr(), ds, q.data_ptr(), qs, k.data_ptr(), ks, v.data_ptr(), vs, log_decay.data_ptr(),
            _ptr(lengths), _ptr(state), _ptr(dstate), gq.data_ptr(), kwide, gk.data_ptr(), kwide, gv.data_ptr(), vwide,
            _ptr(first), dk ** -0.5 if scale is None else scale, n, h, N, dk, dv, dt, wp, need, st),
            "nystra_linear_attention_backward")
        return gq, gk, gv, first

    return _on(q, stream, call)


def linear_attention_step(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, log_decay: torch.Tensor,
                          state: torch.Tensor, scale: float | None = None, out: torch.Tensor | None = None,
                          state_out: torch.Tensor | None = None, stream=None):
    """One token of ``linear_attention`` for each sequence: ``q, k`` ``[n, heads, d_k]``,
    ``v`` ``[n, heads, d_v]``, ``state`` ``[n, heads, d_k, d_v]`` fp32.  Returns
    ``(out, state)``: ``state`` is updated in place, or left as it was and the new
    one written to ``state_out``."""
    state_out = state if state_out is None else state_out
    _tensors(q, k, v, log_decay, state, out, state_out)
    dt, n, h, dk, dv, qs, ks, vs, os = _step_plan(_sig(q), _sig(k), _sig(v), _sig(log_decay), _sig(state),
                                                  _sig(state_out), _sig(out))

    def call(st):
        o = _empty((n, h, dv), q) if out is None else out
        _raise(lib().nystra_linear_attention_step(
            q.data_ptr(), qs, k.data_ptr(), ks, v.data_ptr(), vs, o.data_ptr(), os, log_decay.data_ptr(),
            state.data_ptr(), state_out.data_ptr(), dk ** -0.5 if scale is None else scale, n, h, dk, dv, dt, st),
            "nystra_linear_attention_step")
        return o, state_out

    return _on(q, stream, call)
