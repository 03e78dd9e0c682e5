"""Training-step operators around the optimizer step, on torch tensors.

Between a model's loss and the gradients of its hidden matrices:

* ``attention``: causal (or full) attention over packed sequences of different
  lengths with grouped heads, and its backward pass;
* 8-bit activation checkpoints: ``checkpoint_pack`` / ``checkpoint_unpack``,
  ``checkpoint_act`` (an MLP's activation and the checkpoints its backward pass
  needs, in one pass), ``checkpoint_act_grad`` and ``checkpoint_weight_grad``
  (the gradients that read them), and the layers made of them:
  ``checkpointed_linear`` and ``checkpointed_mlp``.

Every operator runs in the gfx950 kernels of libnormpre.so on the current
stream of its tensors' device, in bf16 or fp32; there is no fallback.  The
``*_forward``, ``*_backward`` and ``checkpoint_*`` functions are the kernels'
calls and record nothing for autograd; ``attention``, ``checkpointed_linear``
and ``checkpointed_mlp`` are differentiable.
"""
from __future__ import annotations

import math
from typing import NamedTuple, Sequence

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


def _same(first: torch.Tensor, **others) -> None:
    """Operands of one call share device and type."""
    if first.device.type != "cuda":
        raise ValueError("expected tensors on a GPU")
    for name, x in others.items():
        if x.device != first.device or x.dtype != first.dtype:
            raise ValueError(f"{name} is {x.dtype} on {x.device}, expected {first.dtype} on {first.device}")


# ------------------------------------------------------------- attention ---
class AttentionPlan:
    """How a packed batch is worked through: made once per batch from its
    sequence lengths (zero-length ones allowed), used by every layer.

    Sequence i holds ``lens[i]`` consecutive tokens, one sequence after the
    other; ``causal``: token t sees the tokens up to itself in its sequence.
    """

    def __init__(self, lens: Sequence[int], causal: bool = True, device="cuda"):
        self.lens = [int(n) for n in lens]
        self.causal = bool(causal)
        plan = N.normpre_attention_plan(self.lens, self.causal)
        self.tokens = sum(self.lens)
        self.num_tiles = plan.shape[1]
        self.data = torch.from_numpy(plan).to(device)


def _rows(x: torch.Tensor) -> torch.Tensor:
    """[tokens, heads, dim] with the feature stride the kernels take."""
    return x if x.stride(2) == 1 or x.shape[2] == 1 else x.contiguous()


def _heads(x: torch.Tensor) -> N.normpre_heads:
    return N.normpre_heads(x.data_ptr(), x.stride(0), x.stride(1))


def _attention_args(q, k, v, plan: AttentionPlan, scale) -> N.normpre_attention:
    if q.dim() != 3 or k.dim() != 3 or v.shape != k.shape:
        raise ValueError("expected q [tokens, heads, dim] and k, v [tokens, kv_heads, dim]")
    _same(q, k=k, v=v)
    if q.shape[0] != plan.tokens or k.shape[0] != plan.tokens or k.shape[2] != q.shape[2]:
        raise ValueError(f"q {tuple(q.shape)} and k {tuple(k.shape)} do not fit a plan of {plan.tokens} tokens")
    if plan.data.device != q.device:
        raise ValueError("the plan lies on another device")
    return N.normpre_attention(
        dtype=_dtype(q), heads=q.shape[1], kv_heads=k.shape[1], head_dim=q.shape[2], causal=int(plan.causal),
        scale=1.0 / math.sqrt(q.shape[2]) if scale is None else float(scale), tokens=plan.tokens,
        plan=plan.data.data_ptr(), num_tiles=plan.num_tiles, q=_heads(q), k=_heads(k), v=_heads(v))


def attention_forward(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, plan: AttentionPlan,
                      scale: float | None = None):
    """(out [tokens, heads, dim], lse fp32 [heads, tokens]) of attention over a
    packed batch; q [tokens, heads, dim], k and v [tokens, kv_heads, dim], query
    head h reading key head h * kv_heads // heads; scale 1 / sqrt(dim) if None.
    Any strides; views of one projection's output need no copy."""
    q, k, v = _rows(q), _rows(k), _rows(v)
    a = _attention_args(q, k, v, plan, scale)
    with torch.cuda.device(q.device):
        out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
        lse = torch.empty((q.shape[1], q.shape[0]), dtype=torch.float32, device=q.device)
        a.out, a.lse = _heads(out), lse.data_ptr()
        N.normpre_attention_forward(a)
    return out, lse


def attention_backward(dout: torch.Tensor, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, out: torch.Tensor,
                       lse: torch.Tensor, plan: AttentionPlan, scale: float | None = None):
    """(dq, dk, dv) from the gradient of ``attention_forward``'s output and what
    that call took and returned."""
    q, k, v, out, dout = _rows(q), _rows(k), _rows(v), _rows(out), _rows(dout)
    a = _attention_args(q, k, v, plan, scale)
    _same(q, out=out, dout=dout)
    if out.shape != q.shape or dout.shape != q.shape:
        raise ValueError("out and dout have q's shape")
    if lse.shape != (q.shape[1], q.shape[0]) or lse.dtype != torch.float32 or not lse.is_contiguous() \
            or lse.device != q.device:
        raise ValueError("lse is attention_forward's")
    with torch.cuda.device(q.device):
        dq, dk, dv = (torch.empty(x.shape, dtype=x.dtype, device=x.device) for x in (q, k, v))
        delta = torch.empty_like(lse)
        a.out, a.lse, a.dout, a.workspace = _heads(out), lse.data_ptr(), _heads(dout), delta.data_ptr()
        a.dq, a.dk, a.dv = _heads(dq), _heads(dk), _heads(dv)
        N.normpre_attention_backward(a)
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
    return x if (x.stride(1) == 1 or x.shape[1] == 1) and x.stride(0) >= x.shape[1] else x.contiguous()


def _new_checkpoint(x: torch.Tensor) -> Checkpoint:
    rows, cols = x.shape
    pitch = -(-cols // GROUP) * GROUP
    return Checkpoint(torch.empty((rows, pitch), dtype=torch.int8, device=x.device),
                      torch.empty((rows, pitch // GROUP), dtype=torch.int8, device=x.device), cols)


def _held(c: Checkpoint, rows: int | None = None):
    pitch = -(-c.cols // GROUP) * GROUP
    ok = (c.codes.dtype == torch.int8 and c.exps.dtype == torch.int8 and c.codes.is_contiguous()
          and c.exps.is_contiguous() and c.codes.device == c.exps.device and c.codes.device.type == "cuda"
          and c.codes.dim() == 2 and c.codes.shape[1] == pitch
          and c.exps.shape == (c.codes.shape[0], pitch // GROUP) and rows in (None, c.codes.shape[0]))
    if not ok:
        raise ValueError("not a checkpoint of this shape")
    return c.codes.data_ptr(), c.exps.data_ptr()


def _ld(x: torch.Tensor) -> int:
    return max(x.stride(0), x.shape[1])


def checkpoint_pack(x: torch.Tensor) -> Checkpoint:
    """The 8-bit checkpoint of x [tokens, features]."""
    x = _matrix(x)
    _same(x)
    with torch.cuda.device(x.device):
        c = _new_checkpoint(x)
        N.normpre_checkpoint_pack(N.NORMPRE_ACT_NONE, _dtype(x), *x.shape, x.data_ptr(), _ld(x), None, 0, None, 0,
                                  *_held(c), None, None, None, None)
    return c


def checkpoint_unpack(c: Checkpoint, dtype: torch.dtype = torch.bfloat16) -> torch.Tensor:
    """The values a checkpoint stands for (exact in bf16 and fp32)."""
    held = _held(c)
    with torch.cuda.device(c.codes.device):
        out = torch.empty((c.codes.shape[0], c.cols), dtype=dtype, device=c.codes.device)
        N.normpre_checkpoint_unpack(_dtype(out), *out.shape, *held, out.data_ptr(), _ld(out))
    return out


def checkpoint_act(act: str, u: torch.Tensor, up: torch.Tensor | None = None):
    """(h, checkpoint of u, checkpoint of up or None, checkpoint of h):
    ``"gelu"`` (tanh form) of u, or ``"swiglu"``: h = u logistic(u) up."""
    if act not in ("gelu", "swiglu") or (act == "swiglu") != (up is not None):
        raise ValueError("act is 'gelu' with u, or 'swiglu' with u and up")
    u = _matrix(u)
    _same(u)
    if up is not None:
        up = _matrix(up)
        _same(u, up=up)
        if up.shape != u.shape:
            raise ValueError("u and up have one shape")
    with torch.cuda.device(u.device):
        h = torch.empty(u.shape, dtype=u.dtype, device=u.device)
        cu, ch = _new_checkpoint(u), _new_checkpoint(u)
        cup = None if up is None else _new_checkpoint(u)
        N.normpre_checkpoint_pack(_ACTS[act], _dtype(u), *u.shape, u.data_ptr(), _ld(u),
                                  None if up is None else up.data_ptr(), 0 if up is None else _ld(up),
                                  h.data_ptr(), _ld(h), *_held(cu), *((None, None) if cup is None else _held(cup)),
                                  *_held(ch))
    return h, cu, cup, ch


def checkpoint_act_grad(act: str, dh: torch.Tensor, cu: Checkpoint, cup: Checkpoint | None = None):
    """(du, dup or None) from dh and the checkpoints ``checkpoint_act`` made."""
    if act not in ("gelu", "swiglu") or (act == "swiglu") != (cup is not None):
        raise ValueError("act is 'gelu' with u's checkpoint, or 'swiglu' with those of u and up")
    dh = _matrix(dh)
    _same(dh)
    for c in (cu, cup):
        if c is not None and (c.cols != dh.shape[1] or c.codes.device != dh.device):
            raise ValueError("the checkpoint is of another activation")
    hu = _held(cu, dh.shape[0])
    hup = (None, None) if cup is None else _held(cup, dh.shape[0])
    with torch.cuda.device(dh.device):
        du = torch.empty(dh.shape, dtype=dh.dtype, device=dh.device)
        dup = None if cup is None else torch.empty_like(du)
        N.normpre_checkpoint_act_grad(_ACTS[act], _dtype(dh), *dh.shape, dh.data_ptr(), _ld(dh), *hu, *hup,
                                      du.data_ptr(), _ld(du), None if dup is None else dup.data_ptr(), _ld(du))
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
    _same(dy)
    tokens, outer = dy.shape
    held = _held(c, tokens)
    if c.codes.device != dy.device:
        raise ValueError("the checkpoint lies on another device")
    shape = (c.cols, outer) if layout == "io" else (outer, c.cols)
    with torch.cuda.device(dy.device):
        if out is None:
            out = torch.empty(shape, dtype=torch.float32, device=dy.device)
        elif (tuple(out.shape) != shape or out.dtype != torch.float32 or out.device != dy.device
              or (out.stride(1) != 1 and shape[1] > 1) or (out.stride(0) < shape[1] and shape[0] > 1)):
            raise ValueError(f"out is a row-major float32 {shape} matrix on {dy.device}")
        dt = _dtype(dy)
        need = N.normpre_checkpoint_weight_grad_workspace(dt, tokens, c.cols, outer)
        ws = torch.empty(need, dtype=torch.uint8, device=dy.device) if need else None
        N.normpre_checkpoint_weight_grad(dt, _LAYOUTS[layout], accumulate, tokens, c.cols, outer, *held,
                                         dy.data_ptr(), _ld(dy), out.data_ptr(), _ld(out),
                                         None if ws is None else ws.data_ptr(), need)
    return out


def _times(x: torch.Tensor, w: torch.Tensor, layout: str) -> torch.Tensor:
    return x @ (w if layout == "io" else w.t())


def _back(dy: torch.Tensor, w: torch.Tensor, layout: str) -> torch.Tensor:
    return dy @ (w.t() if layout == "io" else w)


class _Linear(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, layout):
        w = weight.to(x.dtype)
        y = _times(x, w, layout)
        if bias is not None:
            y += bias.to(y.dtype)
        ctx.layout, ctx.bias, ctx.cols = layout, bias is not None, x.shape[1]
        c = checkpoint_pack(x) if ctx.needs_input_grad[1] else None
        ctx.save_for_backward(weight, *(() if c is None else (c.codes, c.exps)))
        return y

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy):
        weight, *held = ctx.saved_tensors
        dx = _back(dy, weight.to(dy.dtype), ctx.layout) if ctx.needs_input_grad[0] else None
        dw = None
        if held:
            dw = checkpoint_weight_grad(Checkpoint(*held, ctx.cols), dy, ctx.layout).to(weight.dtype)
        db = dy.sum(0, dtype=torch.float32).to(weight.dtype) if ctx.bias and ctx.needs_input_grad[2] else None
        return dx, dw, db, None


def checkpointed_linear(x: torch.Tensor, weight: torch.Tensor, bias: torch.Tensor | None = None,
                        layout: str = "oi") -> torch.Tensor:
    """A linear layer on x [tokens, inner] that keeps x in 8 bits for its weight
    gradient.  The product runs in x's type; weights and their gradients may be
    fp32.  layout: "oi" for y = x W^T, "io" for y = x W."""
    if layout not in _LAYOUTS:
        raise ValueError("layout is 'io' or 'oi'")
    return _Linear.apply(x, weight, bias, layout)


class _Mlp(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, act, layout, w_in, b_in, w_up, w_out, b_out):
        u = _times(x, w_in.to(x.dtype), layout)
        if b_in is not None:
            u += b_in.to(u.dtype)
        up = None if w_up is None else _times(x, w_up.to(x.dtype), layout)
        h, cu, cup, ch = checkpoint_act(act, u, up)
        y = _times(h, w_out.to(h.dtype), layout)
        if b_out is not None:
            y += b_out.to(y.dtype)
        cx = checkpoint_pack(x)
        ctx.act, ctx.layout, ctx.cols = act, layout, (x.shape[1], u.shape[1])
        ctx.bias = b_in is not None, b_out is not None
        held = [cx, cu, ch] + ([] if cup is None else [cup])
        ctx.save_for_backward(w_in, w_up, w_out, *(t for c in held for t in (c.codes, c.exps)))
        return y

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy):
        w_in, w_up, w_out, *held = ctx.saved_tensors
        inner, mid = ctx.cols
        cx, cu, ch = (Checkpoint(*held[2 * i:2 * i + 2], c) for i, c in enumerate((inner, mid, mid)))
        cup = Checkpoint(*held[6:8], mid) if w_up is not None else None
        dh = _back(dy, w_out.to(dy.dtype), ctx.layout)
        d_out = checkpoint_weight_grad(ch, dy, ctx.layout).to(w_out.dtype)
        du, dup = checkpoint_act_grad(ctx.act, dh, cu, cup)
        d_in = checkpoint_weight_grad(cx, du, ctx.layout).to(w_in.dtype)
        dx, d_up = _back(du, w_in.to(du.dtype), ctx.layout), None
        if dup is not None:
            d_up = checkpoint_weight_grad(cx, dup, ctx.layout).to(w_up.dtype)
            dx += _back(dup, w_up.to(dup.dtype), ctx.layout)
        b_in = du.sum(0, dtype=torch.float32).to(w_in.dtype) if ctx.bias[0] else None
        b_out = dy.sum(0, dtype=torch.float32).to(w_out.dtype) if ctx.bias[1] else None
        return dx, None, None, d_in, b_in, d_up, d_out, b_out


def checkpointed_mlp(x: torch.Tensor, w_in: torch.Tensor, w_out: torch.Tensor, *, act: str = "gelu",
                     w_up: torch.Tensor | None = None, b_in: torch.Tensor | None = None,
                     b_out: torch.Tensor | None = None, layout: str = "oi") -> torch.Tensor:
    """An MLP on x [tokens, inner] that keeps nothing but 8-bit checkpoints for
    its backward pass: of x, of the activation's inputs and of its output.
    "gelu": gelu(x W_in + b_in) W_out + b_out; "swiglu": (silu(x W_in) * (x W_up))
    W_out.  layout as in ``checkpointed_linear``, of all three matrices."""
    if act not in ("gelu", "swiglu") or (act == "swiglu") != (w_up is not None):
        raise ValueError("act is 'gelu', or 'swiglu' with w_up")
    if layout not in _LAYOUTS:
        raise ValueError("layout is 'io' or 'oi'")
    return _Mlp.apply(x, act, layout, w_in, b_in, w_up, w_out, b_out)
