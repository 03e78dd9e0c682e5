"""Training-step operators around the optimizer step, on torch tensors.

Between a model's loss and the gradients of its hidden matrices:

* ``qk_norm_rope``: norms of the query and key heads and the rotation of their
  positions (``Rotary``; positions of one or several axes), and its backward pass;
* ``attention``: causal (or full) attention over packed sequences of different
  lengths with grouped heads, with a sliding window where the plan has one, and its
  backward pass;
* 8-bit activation checkpoints: ``checkpoint_pack`` / ``checkpoint_unpack``,
  ``checkpoint_act`` (an MLP's activation and the checkpoints its backward pass
  needs, in one pass), ``checkpoint_act_grad`` and ``checkpoint_weight_grad``
  (the gradients that read them), and the layers made of them:
  ``checkpointed_linear`` and ``checkpointed_mlp``;
* ``grad_norm`` and ``clip_grads``: the norm of all gradients together, and the
  gradients scaled down to a limit, for the optimizer step.

Every operator runs in the gfx950 kernels of libnormpre.so on the current
stream of its tensors' device, in bf16 or fp32; there is no fallback.  The
``*_forward``, ``*_backward`` and ``checkpoint_*`` functions are the kernels'
calls and record nothing for autograd; ``qk_norm_rope``, ``attention``,
``checkpointed_linear`` and ``checkpointed_mlp`` are differentiable.
"""
from __future__ import annotations

import ctypes
import math
import struct
from array import array
from typing import Iterable, NamedTuple, Sequence

import torch

from . import normpre as N

GROUP = N.NORMPRE_CHECKPOINT_GROUP
_DTYPES = {torch.float32: N.NORMPRE_DTYPE_F32, torch.bfloat16: N.NORMPRE_DTYPE_BF16}
_ACTS = {"none": N.NORMPRE_ACT_NONE, "gelu": N.NORMPRE_ACT_GELU, "swiglu": N.NORMPRE_ACT_SWIGLU}
_LAYOUTS = {"io": N.NORMPRE_WEIGHT_INNER_OUTER, "oi": N.NORMPRE_WEIGHT_OUTER_INNER}


def _dtype(x: torch.Tensor) -> int:
    if x.dtype not in _DTYPES:
        raise TypeError(f"expected a bfloat16 or float32 tensor, got {x.dtype}")
    return _DTYPES[x.dtype]


def _same(first: torch.Tensor, *others: torch.Tensor) -> int:
    """Operands of one call share device and type; the device's index."""
    if not first.is_cuda:
        raise ValueError("expected tensors on a GPU")
    at, dtype = first.get_device(), first.dtype
    for x in others:
        if x.get_device() != at or x.dtype != dtype:
            raise ValueError(f"operands differ: {x.dtype} on {x.device}, {dtype} on {first.device}")
    return at


def _elsewhere(at: int) -> bool:
    """Whether `at` is not the current device: the calls below then start over with
    it current, so that allocations and launches go there."""
    return at != torch.cuda.current_device()


def _stream(at: int) -> ctypes.c_void_p:
    return ctypes.c_void_p(torch._C._cuda_getCurrentRawStream(at))


# ------------------------------------------------------------- attention ---
class AttentionPlan:
    """How a packed batch is worked through: made once per batch from its
    sequence lengths (zero-length ones allowed), used by every layer.

    Sequence i holds ``lens[i]`` consecutive tokens, one sequence after the
    other; ``causal``: token t sees the tokens up to itself in its sequence.
    ``window``: of these, the last ``window`` alone, itself among them, and the first
    ``sinks`` tokens of its sequence, which stay visible.
    """

    def __init__(self, lens: Sequence[int], causal: bool = True, device="cuda", window: int | None = None,
                 sinks: int = 0):
        self.lens = [int(n) for n in lens]
        self.causal = bool(causal)
        self.window, self.sinks = None if window is None else int(window), int(sinks)
        self.bounds = None                           # of plans with a window
        if self.window is None:
            if self.sinks:
                raise ValueError("sinks are the first tokens before a window")
        elif not self.causal:
            raise ValueError("a window is causal")
        elif self.window < 1 or self.sinks < 0:
            raise ValueError(f"a window of {window} tokens and {sinks} first ones")
        self.tokens = sum(self.lens)
        # Where every query sees all keys before it, no window is looked at.
        if self.window is None or self.window + self.sinks >= max(self.lens, default=0):
            plan = N.normpre_attention_plan(self.lens, self.causal)
            self.num_tiles = plan.shape[1]
        else:
            plan, self.num_tiles, self.bounds = N.normpre_window_attention_plan(self.lens, self.window, self.sinks)
        self.data = torch.from_numpy(plan).to(device)


def _rows(x: torch.Tensor) -> torch.Tensor:
    """[tokens, heads, dim] with the feature stride the kernels take."""
    if x.dim() != 3:
        raise ValueError(f"expected a tensor [tokens, heads, dim], got {tuple(x.shape)}")
    return x if x.stride(2) == 1 or x.shape[2] == 1 else x.contiguous()


def _fresh(x: torch.Tensor) -> torch.Tensor:
    """A contiguous tensor like x (2 us of host work less than by its shape)."""
    return torch.empty_like(x, memory_format=torch.contiguous_format)


# normpre_attention (include/normpre.h) in one piece: filling a ctypes structure
# field by field takes as long as the launch itself.
_ARGS = struct.Struct("=5if3q" + "Q2q" * 4 + "Q" + "Q2q" * 4 + "Qq")
_NONE = (0, 0, 0)


def _heads(x: torch.Tensor):
    st = x.stride()
    return x.data_ptr(), st[0], st[1]


def _attention_args(q, k, v, plan: AttentionPlan, scale):
    """(device index, the fields up to v); checks the operands."""
    tokens, heads, dim = q.shape
    ks = k.shape
    if v.shape != ks or ks[0] != tokens or ks[2] != dim or tokens != plan.tokens:
        raise ValueError(f"expected q [tokens, heads, dim] and k, v [tokens, kv_heads, dim] of {plan.tokens} tokens, "
                         f"got {tuple(q.shape)}, {tuple(k.shape)}, {tuple(v.shape)}")
    at, data = _same(q, k, v), plan.data
    if data.get_device() != at:
        raise ValueError("the plan lies on another device")
    return at, (_dtype(q), heads, ks[1], dim, int(plan.causal), scale if scale is not None else 1.0 / math.sqrt(dim) if dim else 0.0,
                tokens, data.data_ptr(), plan.num_tiles, *_heads(q), *_heads(k), *_heads(v))


def attention_forward(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, plan: AttentionPlan,
                      scale: float | None = None):
    """(out [tokens, heads, dim], lse fp32 [heads, tokens]) of attention over a
    packed batch; q [tokens, heads, dim], k and v [tokens, kv_heads, dim], query
    head h reading key head h * kv_heads // heads; scale 1 / sqrt(dim) if None.
    Any strides; views of one projection's output need no copy."""
    q, k, v = _rows(q), _rows(k), _rows(v)
    at, args = _attention_args(q, k, v, plan, scale)
    if _elsewhere(at):
        with torch.cuda.device(at):
            return attention_forward(q, k, v, plan, scale)
    tokens, heads, dim = q.shape
    out = _fresh(q)
    lse = q.new_empty((heads, tokens), dtype=torch.float32)
    block = _ARGS.pack(*args, out.data_ptr(), heads * dim, dim, lse.data_ptr(), *_NONE * 4, 0, 0)
    if plan.bounds is None:
        N.normpre_attention_forward(N.normpre_attention.from_buffer_copy(block), _stream(at))
    else:
        N.normpre_window_attention_forward(N.normpre_attention.from_buffer_copy(block), plan.bounds, _stream(at))
    return out, lse


def attention_backward(dout: torch.Tensor, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, out: torch.Tensor,
                       lse: torch.Tensor, plan: AttentionPlan, scale: float | None = None):
    """(dq, dk, dv) from the gradient of ``attention_forward``'s output and what
    that call took and returned."""
    if out.shape != q.shape or dout.shape != q.shape:
        raise ValueError("q, out and dout have one shape")
    q, k, v, out, dout = _rows(q), _rows(k), _rows(v), _rows(out), _rows(dout)
    at, args = _attention_args(q, k, v, plan, scale)
    _same(q, out, dout)
    if lse.shape != (q.shape[1], q.shape[0]) or lse.dtype != torch.float32 or not lse.is_contiguous() \
            or lse.get_device() != at:
        raise ValueError("lse is attention_forward's")
    if _elsewhere(at):
        with torch.cuda.device(at):
            return attention_backward(dout, q, k, v, out, lse, plan, scale)
    dq, dk, dv = _fresh(q), _fresh(k), _fresh(v)
    block = N.normpre_attention.from_buffer_copy(_ARGS.pack(
        *args, *_heads(out), lse.data_ptr(), *_heads(dout), *_heads(dq), *_heads(dk), *_heads(dv), 0, 0))
    bounds = plan.bounds
    block.workspace_bytes = (N.normpre_attention_workspace(block) if bounds is None
                             else N.normpre_window_attention_workspace(block, bounds))
    work = lse.new_empty(block.workspace_bytes, dtype=torch.uint8)
    block.workspace = work.data_ptr()
    if bounds is None:
        N.normpre_attention_backward(block, _stream(at))
    else:
        N.normpre_window_attention_backward(block, bounds, _stream(at))
    return dq, dk, dv


class _Attention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, plan, scale):
        out, lse = attention_forward(q, k, v, plan, scale)
        ctx.save_for_backward(q, k, v, out, lse)
        ctx.plan, ctx.scale = plan, scale
        return out

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dout):
        q, k, v, out, lse = ctx.saved_tensors
        return *attention_backward(dout, q, k, v, out, lse, ctx.plan, ctx.scale), None, None


def attention(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, plan: AttentionPlan,
              scale: float | None = None) -> torch.Tensor:
    """Differentiable ``attention_forward``; returns out alone."""
    return _Attention.apply(q, k, v, plan, scale)


# -------------------------------------------------------------- rotation ---
class Rotary:
    """How heads turn with their positions: made once, used by every layer.

    freqs: radians a step of each turning pair of features (finite numbers, kept in
    64 bits); the first 2 * len(freqs) features of a head turn, the others stay.
    Angles (position * frequency) are off by 2^-51 of their size at most, for up to 2^51,
    and their cos and sin by another 5 2^-24 (fp32).
    axes: the axis of positions that each pair turns by (default: all by the
    first); num_axes: how many axes positions have, where there are more than the
    highest of these.  adjacent: pair i is features (2i, 2i + 1); else (i, i + len(freqs)).
    """

    def __init__(self, freqs: Sequence[float], axes: Sequence[int] | None = None, adjacent: bool = False,
                 device="cuda", num_axes: int | None = None):
        freqs = [float(f) for f in freqs]
        if not all(map(math.isfinite, freqs)):
            raise ValueError("a frequency is not finite")
        self.pairs, self.adjacent = len(freqs), bool(adjacent)
        axes = [0] * len(freqs) if axes is None else [int(a) for a in axes]
        if len(axes) != len(freqs) or any(a < 0 for a in axes):
            raise ValueError("axes names an axis, 0 or above, for each frequency")
        named = max(axes, default=0) + 1
        self.num_axes = named if num_axes is None else int(num_axes)
        if self.num_axes < named:
            raise ValueError(f"axis {named - 1} of {num_axes}")
        self.freqs = torch.tensor(freqs, dtype=torch.float64, device=device)
        self.axes = None if named == 1 else torch.tensor(axes, dtype=torch.int32, device=device)

    @staticmethod
    def geometric(rotated: int, base: float = 10000.0) -> list[float]:
        """Frequencies base^(-2i / rotated) of `rotated` / 2 pairs."""
        if rotated < 0 or rotated % 2:
            raise ValueError(f"{rotated} features do not make pairs")
        return [base ** (-2 * i / rotated) for i in range(rotated // 2)]


# normpre_qk_rope (include/normpre.h) in one piece, as for attention.
_ROPE = struct.Struct("=10idq" + "3Qq" + "2Q" + "Q2q" * 6 + "2Q" + "Qq")


def _norm_weight(w: torch.Tensor, dim: int, at: int) -> int:
    if w.shape != (dim,) or w.get_device() != at or not w.is_contiguous():
        raise ValueError(f"a weight is a contiguous [{dim}] tensor on cuda:{at}, got {tuple(w.shape)} on {w.device}")
    return _dtype(w)


def _rope_args(q, k, positions, rotary: Rotary | None, norm, q_weight, k_weight, eps):
    """(device index, the fields up to k_weight); checks the operands."""
    tokens, heads, dim = q.shape
    ks = k.shape
    if ks[0] != tokens or ks[2] != dim:
        raise ValueError(f"expected q [tokens, heads, dim] and k [tokens, kv_heads, dim], got {tuple(q.shape)}, {tuple(ks)}")
    at = _same(q, k)
    kind = qw = kw = 0
    if q_weight is not None:
        kind, qw = _norm_weight(q_weight, dim, at), q_weight.data_ptr()
    if k_weight is not None:
        other, kw = _norm_weight(k_weight, dim, at), k_weight.data_ptr()
        if q_weight is not None and other != kind:
            raise ValueError("the weights have one type")
        kind = other
    if (qw or kw) and not norm:
        raise ValueError("weights are the norm's")
    if rotary is None:
        return at, (_dtype(q), heads, ks[1], dim, 0, 0, int(bool(norm)), kind, 1, 4, float(eps), tokens, 0, 0, 0, 0, qw, kw)
    axes = rotary.num_axes
    if positions is None or positions.dtype not in (torch.int32, torch.int64) or positions.get_device() != at \
            or not (positions.shape == (axes, tokens) or (axes == 1 and positions.shape == (tokens,))):
        raise ValueError(f"positions are int32 or int64 [{axes}, {tokens}] on {q.device}")
    if rotary.freqs.get_device() != at:
        raise ValueError("the rotary lies on another device")
    return at, (_dtype(q), heads, ks[1], dim, rotary.pairs, int(rotary.adjacent), int(bool(norm)), kind, axes,
                positions.element_size(), float(eps), tokens, rotary.freqs.data_ptr(),
                0 if rotary.axes is None else rotary.axes.data_ptr(), positions.data_ptr(),
                positions.stride(0) if axes > 1 else 0, qw, kw)


def _positions(positions: torch.Tensor | None) -> torch.Tensor | None:
    """Positions with adjacent tokens."""
    return positions if positions is None or positions.dim() not in (1, 2) or positions.stride(-1) == 1 else positions.contiguous()


def qk_norm_rope_forward(q: torch.Tensor, k: torch.Tensor, positions: torch.Tensor | None, rotary: Rotary | None, *,
                         norm: bool = True, q_weight: torch.Tensor | None = None,
                         k_weight: torch.Tensor | None = None, eps: float = 1e-6):
    """(q, k) with their heads normed, x / sqrt(mean x^2 + eps) times the weight
    [dim] if there is one (``norm``), and turned by ``rotary`` (None: not turned)
    at ``positions``, int32 or int64 [tokens], or [axes, tokens] of several axes
    (the rotary's ``num_axes``).
    q [tokens, heads, dim], k [tokens, kv_heads, dim], dim up to 256, any strides;
    weights fp32 or bf16."""
    q, k, positions = _rows(q), _rows(k), _positions(positions)
    at, args = _rope_args(q, k, positions, rotary, norm, q_weight, k_weight, eps)
    if _elsewhere(at):
        with torch.cuda.device(at):
            return qk_norm_rope_forward(q, k, positions, rotary, norm=norm, q_weight=q_weight, k_weight=k_weight, eps=eps)
    q_out, k_out = _fresh(q), _fresh(k)
    block = _ROPE.pack(*args, *_heads(q), *_heads(k), *_heads(q_out), *_heads(k_out), *_NONE * 2, 0, 0, 0, 0)
    N.normpre_qk_rope_forward(N.normpre_qk_rope.from_buffer_copy(block), _stream(at))
    return q_out, k_out


def qk_norm_rope_backward(dq_out: torch.Tensor, dk_out: torch.Tensor, q: torch.Tensor, k: torch.Tensor,
                          positions: torch.Tensor | None, rotary: Rotary | None, *, norm: bool = True,
                          q_weight: torch.Tensor | None = None, k_weight: torch.Tensor | None = None,
                          eps: float = 1e-6):
    """(dq, dk, dq_weight, dk_weight) from the gradients of ``qk_norm_rope_forward``'s
    outputs and what that call took (without ``norm`` the shapes of q and k alone); the
    weights' in fp32, None where there is no weight."""
    if dq_out.shape != q.shape or dk_out.shape != k.shape:
        raise ValueError("gradients have the shapes of q and k")
    q, k, dq_out, dk_out, positions = _rows(q), _rows(k), _rows(dq_out), _rows(dk_out), _positions(positions)
    at, args = _rope_args(q, k, positions, rotary, norm, q_weight, k_weight, eps)
    _same(q, dq_out, dk_out)
    if _elsewhere(at):
        with torch.cuda.device(at):
            return qk_norm_rope_backward(dq_out, dk_out, q, k, positions, rotary, norm=norm, q_weight=q_weight,
                                         k_weight=k_weight, eps=eps)
    dq, dk = _fresh(q), _fresh(k)
    dwq = dwk = None
    ends = (0, 0, 0, 0)
    if q_weight is not None or k_weight is not None:
        dim = q.shape[2]
        work = q.new_empty(1024 * dim, dtype=torch.float32)      # the bound: the size itself is not worth a call
        dwq = None if q_weight is None else work.new_empty(dim)
        dwk = None if k_weight is None else work.new_empty(dim)
        ends = (0 if dwq is None else dwq.data_ptr(), 0 if dwk is None else dwk.data_ptr(), work.data_ptr(), 4096 * dim)
    N.normpre_qk_rope_backward(N.normpre_qk_rope.from_buffer_copy(_ROPE.pack(
        *args, *_heads(q), *_heads(k), *_heads(dq_out), *_heads(dk_out), *_heads(dq), *_heads(dk), *ends)), _stream(at))
    return dq, dk, dwq, dwk


class _QkNormRope(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, positions, rotary, norm, q_weight, k_weight, eps):
        # Without norms the gradients need nothing of q and k.
        ctx.save_for_backward(q if norm else None, k if norm else None, positions, q_weight, k_weight)
        ctx.rotary, ctx.how = rotary, {"norm": norm, "eps": eps}
        return qk_norm_rope_forward(q, k, positions, rotary, norm=norm, q_weight=q_weight, k_weight=k_weight, eps=eps)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dq_out, dk_out):
        q, k, positions, *weights = ctx.saved_tensors
        if q is None:
            q, k = dq_out, dk_out
        dq, dk, *dw = qk_norm_rope_backward(dq_out, dk_out, q, k, positions, ctx.rotary, q_weight=weights[0],
                                            k_weight=weights[1], **ctx.how)
        dwq, dwk = (d if d is None else d.to(w.dtype) for d, w in zip(dw, weights))
        return dq, dk, None, None, None, dwq, dwk, None


def qk_norm_rope(q: torch.Tensor, k: torch.Tensor, positions: torch.Tensor | None, rotary: Rotary | None, *,
                 norm: bool = True, q_weight: torch.Tensor | None = None, k_weight: torch.Tensor | None = None,
                 eps: float = 1e-6) -> tuple[torch.Tensor, torch.Tensor]:
    """Differentiable ``qk_norm_rope_forward``, with respect to q, k and the weights."""
    return _QkNormRope.apply(q, k, positions, rotary, norm, q_weight, k_weight, eps)


# ----------------------------------------------------------- checkpoints ---
class Checkpoint(NamedTuple):
    """An activation [rows, cols] in 8 bits: codes int8 [rows, cols rounded up
    to 64], one exponent int8 for each 64 of them; value = code * 2^exponent."""
    codes: torch.Tensor
    exps: torch.Tensor
    cols: int


def _matrix(x: torch.Tensor) -> torch.Tensor:
    """2-D, rows of adjacent features."""
    if x.dim() != 2:
        raise ValueError(f"expected a matrix [tokens, features], got {tuple(x.shape)}")
    st = x.stride()
    return x if (st[1] == 1 or x.shape[1] == 1) and st[0] >= x.shape[1] else x.contiguous()


def _new_checkpoint(x: torch.Tensor) -> Checkpoint:
    rows, cols = x.shape
    groups = -(-cols // GROUP)
    return Checkpoint(x.new_empty((rows, groups * GROUP), dtype=torch.int8),
                      x.new_empty((rows, groups), dtype=torch.int8), cols)


def _held(c: Checkpoint, rows: int | None = None):
    codes, exps = c.codes, c.exps
    groups = -(-c.cols // GROUP)
    if not (codes.dtype == exps.dtype == torch.int8 and codes.dim() == 2 and codes.shape[1] == groups * GROUP
            and exps.shape == (codes.shape[0], groups) and codes.is_contiguous() and exps.is_contiguous()
            and codes.is_cuda and codes.get_device() == exps.get_device() and rows in (None, codes.shape[0])):
        raise ValueError("not a checkpoint of this shape on a GPU")
    return codes.data_ptr(), exps.data_ptr()


def _ld(x: torch.Tensor) -> int:
    return max(x.stride(0), x.shape[1])


_NOTHING = (None, 0)


def _row_args(x: torch.Tensor | None):
    return _NOTHING if x is None else (x.data_ptr(), _ld(x))


def _held_args(c: Checkpoint | None):
    return (None, None) if c is None else (c.codes.data_ptr(), c.exps.data_ptr())


def checkpoint_pack(x: torch.Tensor) -> Checkpoint:
    """The 8-bit checkpoint of x [tokens, features]."""
    x = _matrix(x)
    at = _same(x)
    if _elsewhere(at):
        with torch.cuda.device(at):
            return checkpoint_pack(x)
    c = _new_checkpoint(x)
    N.normpre_checkpoint_pack(N.NORMPRE_ACT_NONE, _dtype(x), *x.shape, *_row_args(x), *_NOTHING, *_NOTHING,
                              *_held_args(c), None, None, None, None, _stream(at))
    return c


def checkpoint_unpack(c: Checkpoint, dtype: torch.dtype = torch.bfloat16) -> torch.Tensor:
    """The values a checkpoint stands for (exact in bf16 and fp32)."""
    held, at = _held(c), c.codes.get_device()
    if _elsewhere(at):
        with torch.cuda.device(at):
            return checkpoint_unpack(c, dtype)
    rows, cols = c.codes.shape[0], c.cols
    out = c.codes.new_empty((rows, cols), dtype=dtype)
    N.normpre_checkpoint_unpack(_dtype(out), rows, cols, *held, out.data_ptr(), cols, _stream(at))
    return out


def checkpoint_act(act: str, u: torch.Tensor, up: torch.Tensor | None = None):
    """(h, checkpoint of u, checkpoint of up or None, checkpoint of h):
    ``"gelu"`` (tanh form) of u, or ``"swiglu"``: h = u logistic(u) up."""
    if act not in ("gelu", "swiglu") or (act == "swiglu") != (up is not None):
        raise ValueError("act is 'gelu' with u, or 'swiglu' with u and up")
    u = _matrix(u)
    at = _same(u)
    if up is not None:
        up = _matrix(up)
        _same(u, up)
        if up.shape != u.shape:
            raise ValueError("u and up have one shape")
    if _elsewhere(at):
        with torch.cuda.device(at):
            return checkpoint_act(act, u, up)
    rows, cols = u.shape
    h = u.new_empty((rows, cols))
    cu, ch = _new_checkpoint(u), _new_checkpoint(u)
    cup = None if up is None else _new_checkpoint(u)
    N.normpre_checkpoint_pack(_ACTS[act], _dtype(u), rows, cols, *_row_args(u), *_row_args(up), h.data_ptr(), cols,
                              *_held_args(cu), *_held_args(cup), *_held_args(ch), _stream(at))
    return h, cu, cup, ch


def checkpoint_act_grad(act: str, dh: torch.Tensor, cu: Checkpoint, cup: Checkpoint | None = None):
    """(du, dup or None) from dh and the checkpoints ``checkpoint_act`` made."""
    if act not in ("gelu", "swiglu") or (act == "swiglu") != (cup is not None):
        raise ValueError("act is 'gelu' with u's checkpoint, or 'swiglu' with those of u and up")
    dh = _matrix(dh)
    at = _same(dh)
    rows, cols = dh.shape
    for c in (cu, cup):
        if c is not None and (c.cols != cols or c.codes.get_device() != at):
            raise ValueError("the checkpoint is of another activation")
    hu = _held(cu, rows)
    hup = (None, None) if cup is None else _held(cup, rows)
    if _elsewhere(at):
        with torch.cuda.device(at):
            return checkpoint_act_grad(act, dh, cu, cup)
    du = dh.new_empty((rows, cols))
    dup = None if cup is None else dh.new_empty((rows, cols))
    N.normpre_checkpoint_act_grad(_ACTS[act], _dtype(dh), rows, cols, *_row_args(dh), *hu, *hup, du.data_ptr(), cols,
                                  None if dup is None else dup.data_ptr(), cols, _stream(at))
    return du, dup


def checkpoint_weight_grad(c: Checkpoint, dy: torch.Tensor, layout: str = "oi", out: torch.Tensor | None = None,
                           accumulate: bool = False) -> torch.Tensor:
    """fp32 weight gradient of a linear layer from the checkpoint of its input
    and the gradient dy [tokens, outer] of its output: [outer, inner] for
    layout "oi" (y = x W^T), [inner, outer] for "io" (y = x W).  ``out``: where
    to put it, added to what is there with ``accumulate``."""
    if layout not in _LAYOUTS:
        raise ValueError("layout is 'io' or 'oi'")
    if accumulate and out is None:
        raise ValueError("accumulate needs out")
    dy = _matrix(dy)
    at = _same(dy)
    tokens, outer = dy.shape
    held = _held(c, tokens)
    if c.codes.get_device() != at:
        raise ValueError("the checkpoint lies on another device")
    shape = (c.cols, outer) if layout == "io" else (outer, c.cols)
    if out is not None and (out.shape != shape or out.dtype != torch.float32 or out.device != dy.device
                            or (out.stride(1) != 1 and shape[1] > 1) or (out.stride(0) < shape[1] and shape[0] > 1)):
        raise ValueError(f"out is a row-major float32 {shape} matrix on {dy.device}")
    if _elsewhere(at):
        with torch.cuda.device(at):
            return checkpoint_weight_grad(c, dy, layout, out, accumulate)
    if out is None:
        out = dy.new_empty(shape, dtype=torch.float32)
    dt = _dtype(dy)
    need = N.normpre_checkpoint_weight_grad_workspace(dt, tokens, c.cols, outer)
    ws = dy.new_empty(need, dtype=torch.uint8) if need else None
    N.normpre_checkpoint_weight_grad(dt, _LAYOUTS[layout], accumulate, tokens, c.cols, outer, *held, *_row_args(dy),
                                     *_row_args(out), None if ws is None else ws.data_ptr(), need, _stream(at))
    return out


def _plain_types(backward):
    """A backward pass whose products run in their operands' types, also where it is
    called under autocast."""
    def call(*args):
        with torch.autocast("cuda", enabled=False):
            return backward(*args)
    return staticmethod(torch.autograd.function.once_differentiable(call))


def _times(x: torch.Tensor, w: torch.Tensor, layout: str) -> torch.Tensor:
    return x @ (w if layout == "io" else w.t())


def _back(dy: torch.Tensor, w: torch.Tensor, layout: str) -> torch.Tensor:
    return dy @ (w.t() if layout == "io" else w)


class _Linear(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, layout, keep):
        w = weight.to(x.dtype)
        y = _times(x, w, layout)
        if bias is not None:
            y += bias.to(y.dtype)
        ctx.layout, ctx.bias, ctx.cols = layout, None if bias is None else bias.dtype, x.shape[1]
        c = checkpoint_pack(x) if keep else None
        ctx.save_for_backward(weight, *(() if c is None else (c.codes, c.exps)))
        return y

    @_plain_types
    def backward(ctx, dy):
        weight, *held = ctx.saved_tensors
        dx = _back(dy, weight.to(dy.dtype), ctx.layout) if ctx.needs_input_grad[0] else None
        dw = None
        if held:
            dw = checkpoint_weight_grad(Checkpoint(*held, ctx.cols), dy, ctx.layout).to(weight.dtype)
        db = dy.sum(0, dtype=torch.float32).to(ctx.bias) if ctx.needs_input_grad[2] else None
        return dx, dw, db, None, None


def _trained(*weights: torch.Tensor | None) -> bool:
    """Whether a weight gradient may be asked for later, so that x is kept for it
    (inside an autograd function's forward pass the grad mode is always off)."""
    return torch.is_grad_enabled() and any(w is not None and w.requires_grad for w in weights)


def _check_layer(x: torch.Tensor, layout: str):
    if layout not in _LAYOUTS:
        raise ValueError("layout is 'io' or 'oi'")
    if x.dim() != 2:
        raise ValueError(f"expected x [tokens, inner], got {tuple(x.shape)}")
    _same(x)
    _dtype(x)


def checkpointed_linear(x: torch.Tensor, weight: torch.Tensor, bias: torch.Tensor | None = None,
                        layout: str = "oi") -> torch.Tensor:
    """A linear layer on x [tokens, inner] that keeps x in 8 bits for its weight
    gradient.  The products run in x's type, also under autocast (forward and
    backward); weights and their gradients may be fp32.  layout: "oi" for y = x W^T, "io" for y = x W."""
    _check_layer(x, layout)
    with torch.autocast("cuda", enabled=False):
        return _Linear.apply(x, weight, bias, layout, _trained(weight))


class _Mlp(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, act, layout, w_in, b_in, w_up, w_out, b_out, keep):
        u = _times(x, w_in.to(x.dtype), layout)
        if b_in is not None:
            u += b_in.to(u.dtype)
        up = None if w_up is None else _times(x, w_up.to(x.dtype), layout)
        h, cu, cup, ch = checkpoint_act(act, u, up)
        y = _times(h, w_out.to(h.dtype), layout)
        if b_out is not None:
            y += b_out.to(y.dtype)
        cx = checkpoint_pack(x) if keep else Checkpoint(None, None, 0)
        ctx.act, ctx.layout, ctx.cols = act, layout, (x.shape[1], u.shape[1])
        ctx.bias = tuple(None if b is None else b.dtype for b in (b_in, b_out))
        held = [cx, cu, ch] + ([] if cup is None else [cup])
        ctx.save_for_backward(w_in, w_up, w_out, *(t for c in held for t in (c.codes, c.exps)))
        return y

    @_plain_types
    def backward(ctx, dy):
        w_in, w_up, w_out, *held = ctx.saved_tensors
        inner, mid = ctx.cols
        cx, cu, ch = (Checkpoint(*held[2 * i:2 * i + 2], c) for i, c in enumerate((inner, mid, mid)))
        cup = Checkpoint(*held[6:8], mid) if w_up is not None else None
        need = ctx.needs_input_grad
        dh = _back(dy, w_out.to(dy.dtype), ctx.layout)
        du, dup = checkpoint_act_grad(ctx.act, dh, cu, cup)
        d_out = checkpoint_weight_grad(ch, dy, ctx.layout).to(w_out.dtype) if need[6] else None
        d_in = checkpoint_weight_grad(cx, du, ctx.layout).to(w_in.dtype) if need[3] else None
        d_up = checkpoint_weight_grad(cx, dup, ctx.layout).to(w_up.dtype) if need[5] else None
        dx = None
        if need[0]:
            dx = _back(du, w_in.to(du.dtype), ctx.layout)
            if dup is not None:
                dx += _back(dup, w_up.to(dup.dtype), ctx.layout)
        b_in = du.sum(0, dtype=torch.float32).to(ctx.bias[0]) if need[4] else None
        b_out = dy.sum(0, dtype=torch.float32).to(ctx.bias[1]) if need[7] else None
        return dx, None, None, d_in, b_in, d_up, d_out, b_out, None


def checkpointed_mlp(x: torch.Tensor, w_in: torch.Tensor, w_out: torch.Tensor, *, act: str = "gelu",
                     w_up: torch.Tensor | None = None, b_in: torch.Tensor | None = None,
                     b_out: torch.Tensor | None = None, layout: str = "oi") -> torch.Tensor:
    """An MLP on x [tokens, inner] that keeps nothing but 8-bit checkpoints for
    its backward pass: of x, of the activation's inputs and of its output.
    "gelu": gelu(x W_in + b_in) W_out + b_out; "swiglu": (silu(x W_in) * (x W_up))
    W_out.  layout as in ``checkpointed_linear``, of all three matrices."""
    if act not in ("gelu", "swiglu") or (act == "swiglu") != (w_up is not None):
        raise ValueError("act is 'gelu', or 'swiglu' with w_up")
    _check_layer(x, layout)
    with torch.autocast("cuda", enabled=False):
        return _Mlp.apply(x, act, layout, w_in, b_in, w_up, w_out, b_out, _trained(w_in, w_up))


# ------------------------------------------------------------- gradients ---
def _dense(x: torch.Tensor) -> bool:
    """Whether x's elements fill a piece of memory, each place once."""
    if x.is_contiguous():
        return True
    expected = 1
    for stride, size in sorted((st, n) for st, n in zip(x.stride(), x.shape) if n != 1):
        if stride != expected:
            return False
        expected *= size
    return True


def _grad_list(grads: Iterable[torch.Tensor]) -> list[torch.Tensor]:
    return [grads] if isinstance(grads, torch.Tensor) else list(grads)


def _grad_entries(grads, outs) -> tuple[int, array]:
    """(device index, the C ABI's list of gradients).  Hundreds of tensors a step: a
    pass over them for each thing that is asked of them."""
    at = grads[0].get_device()
    if at < 0:
        raise ValueError("expected tensors on a GPU")
    kinds, places, sizes = [_DTYPES.get(g.dtype) for g in grads], [g.data_ptr() for g in grads], [g.numel() for g in grads]
    devices = {g.get_device() for g in grads}
    to, into = kinds, places
    if outs is not grads:
        to, into = [_DTYPES.get(o.dtype) for o in outs], [o.data_ptr() for o in outs]
        devices |= {o.get_device() for o in outs}
    if devices != {at}:
        raise ValueError("gradients lie on different devices")
    if None in kinds or None in to:
        raise TypeError("expected bfloat16 or float32 gradients")
    return at, array("Q", [x for e in zip(places, into, sizes, [a | b << 32 for a, b in zip(kinds, to)]) for x in e])


def _grad_workspace(like: torch.Tensor):
    return like.new_empty((), dtype=torch.float32), like.new_empty(N.NORMPRE_GRAD_WORKSPACE_BYTES, dtype=torch.uint8)


def grad_norm(grads: Iterable[torch.Tensor] | torch.Tensor) -> torch.Tensor:
    """The 2-norm of all gradients together, as an fp32 tensor of no dimensions on
    their device (0 on the CPU for an empty list); does not wait for the GPU.
    Gradients in bf16 and fp32, mixed or not, of any strides (those that do not
    fill a piece of memory are copied)."""
    grads = [g if _dense(g) else g.contiguous() for g in _grad_list(grads)]
    if not grads:
        return torch.zeros(())
    at, block = _grad_entries(grads, grads)
    if _elsewhere(at):
        with torch.cuda.device(at):
            return grad_norm(grads)
    norm, work = _grad_workspace(grads[0])
    N.normpre_grad_norm(len(grads), block.buffer_info()[0], norm.data_ptr(), work.data_ptr(), work.numel(), _stream(at))
    return norm


def _in_one_order(grads, outs):
    """(gradients, outputs, pairs to copy afterwards), each gradient's elements in its
    output's order in memory."""
    sources, targets, back = [], [], []
    for g, o in zip(grads, outs):
        if not _dense(o) and any(st == 0 and n > 1 for st, n in zip(o.stride(), o.shape)):
            raise ValueError("an output's elements share memory")
        if _dense(g) and (g.stride() == o.stride() or (g.is_contiguous() and o.is_contiguous())):
            sources.append(g)
            targets.append(o)
            continue
        sources.append(g.contiguous())
        targets.append(o if o.is_contiguous() else torch.empty_like(o, memory_format=torch.contiguous_format))
        if not o.is_contiguous():
            back.append((o, targets[-1]))
    return sources, targets, back


def clip_grads(grads: Iterable[torch.Tensor] | torch.Tensor, max_norm: float,
               out: Iterable[torch.Tensor] | torch.Tensor | None = None) -> torch.Tensor:
    """Scales the gradients by max_norm / norm where their norm (``grad_norm``, which
    is returned) exceeds max_norm: in place, or into ``out``, tensors of the same
    shapes, bf16 or fp32, which are written in any case (bf16 gradients for an
    optimizer that takes fp32 ones).  Autograd takes either for a write in place,
    whatever the norm.  Does not wait for the GPU.  NaN or infinite gradients follow
    the formula: a norm of NaN makes every gradient NaN, an infinite one 0 or, where it
    was infinite, NaN."""
    grads = _grad_list(grads)
    if not max_norm >= 0:
        raise ValueError(f"max_norm is {max_norm}")
    outs = grads if out is None else _grad_list(out)
    if len(outs) != len(grads) or any(o.shape != g.shape for g, o in zip(grads, outs)):
        raise ValueError("out has the gradients' number and shapes")
    if not grads:
        return torch.zeros(())
    sources, targets, back = grads, outs, []
    if not (all(g.is_contiguous() for g in grads) and (out is None or all(o.is_contiguous() for o in outs))):
        sources, targets, back = _in_one_order(grads, outs)
    at, block = _grad_entries(sources, targets)
    if _elsewhere(at):
        with torch.cuda.device(at):
            return clip_grads(grads, max_norm, None if out is None else outs)    # out may be used up
    norm, work = _grad_workspace(grads[0])
    N.normpre_grad_clip(len(grads), block.buffer_info()[0], float(max_norm), norm.data_ptr(), work.data_ptr(),
                        work.numel(), _stream(at))
    torch.autograd.graph.increment_version(outs)     # a backward pass that kept them has to notice
    with torch.no_grad():
        for o, t in back:
            o.copy_(t)
    return norm
