"""End-to-end GPT-2 Small training steps on synthetic tokens.

Random-initialized GPT-2 Small (12 layers, width 768; no checkpoint, no
dataset: uniform random token ids), forward + backward + optimizer step.  The
48 hidden attention/MLP matrices are stepped by the NormPre library through
``NormPreOptimizer``; embeddings, layer norms and biases by AdamW (App. A.1).
The optimizer step is timed between device synchronizations, as in the
paper's efficiency tables (Sec. 4.2); the model runs in fp32.

Prints one JSON line: fwd+bwd and optimizer milliseconds per step (with
``--clip`` the optimizer's include the clipping of the gradients), the
optimizer's share of the step, tokens/s, and the descent alignment of the
last step (App. A.3: mean over the hidden matrices of the cosine between the
gradient and the update direction, weight decay excluded).

    python -m paper_2609_36692_amd.e2e_gpt2 --optimizer normpre-g --batch 4

With ``--train-ops`` the blocks' attention and MLP run on the operators of
``train_ops``: documents of different lengths packed into one sequence of
batch * seq tokens, and activations kept in 8 bits for the backward pass, in
fp32 or (``--dtype bf16``) in bf16 with fp32 parameters.  Attention weights have
no dropout there.

    python -m paper_2609_36692_amd.e2e_gpt2 --train-ops --dtype bf16 --batch 16 --documents 24
"""
from __future__ import annotations

import argparse
import inspect
import json
import time
import types

import torch

HIDDEN_SUFFIXES = ("attn.c_attn.weight", "attn.c_proj.weight", "mlp.c_fc.weight", "mlp.c_proj.weight")
# Arguments of a GPT2Model that its blocks need not know of.
HONOURED = ("input_ids", "inputs_embeds", "position_ids", "token_type_ids", "output_hidden_states", "return_dict")


def build(seq):
    from transformers import GPT2Config, GPT2LMHeadModel
    torch.manual_seed(1337)
    cfg = GPT2Config(n_layer=12, n_embd=768, n_head=12, n_positions=seq, vocab_size=50257)
    return GPT2LMHeadModel(cfg)


class Packing:
    """The packed batch that the blocks of a model work on: ``set`` before each
    forward pass."""

    def __init__(self, device):
        self.device = device
        self.plan = None

    def set(self, lens):
        """Makes the plan; returns (position ids [1, tokens], mask of the tokens
        that no token of their document precedes [1, tokens])."""
        from .train_ops import AttentionPlan
        self.plan = AttentionPlan(lens, causal=True, device=self.device)
        pos = torch.cat([torch.arange(n) for n in lens])[None]
        return pos.to(self.device), (pos == 0).to(self.device)


def use_train_ops(model, packing: Packing, dtype=torch.float32):
    """Runs the attention and the MLP of every block of a GPT2LMHeadModel on the
    operators of ``train_ops`` (parameters stay where they are).  Which token sees
    which is the packing's plan alone, nothing is cached between calls, and attention
    weights have no dropout: a call with an argument that would change any of it
    (a mask, a cache, attention weights asked for) raises ValueError."""
    from . import train_ops as T
    cfg = model.config
    if cfg.activation_function not in ("gelu_new", "gelu_pytorch_tanh") or cfg.add_cross_attention:
        raise ValueError("expected blocks with the tanh form of GELU and without cross-attention")

    def check(module, args, kwargs):
        given = inspect.signature(module.forward).bind(*args, **kwargs).arguments
        given |= given.pop("kwargs", {})
        for name, value in given.items():
            if name not in HONOURED and value is not None and value is not False:
                raise ValueError(f"blocks on the training-step operators take no {name}")
        if packing.plan is None:
            raise ValueError("set the packing's lengths before a forward pass")
        if "use_cache" in given and "use_cache" not in kwargs:       # as a positional argument
            return None
        return args, kwargs | {"use_cache": False}

    def attention(self, hidden_states, *args, **kwargs):     # the rest: checked above, or the model's own
        x = hidden_states.flatten(0, 1).to(dtype)
        qkv = T.checkpointed_linear(x, self.c_attn.weight, self.c_attn.bias, layout="io")
        q, k, v = (t.unflatten(1, (-1, self.head_dim)) for t in qkv.split(self.split_size, dim=1))
        out = T.attention(q, k, v, packing.plan, self.scaling)
        out = T.checkpointed_linear(out.flatten(1), self.c_proj.weight, self.c_proj.bias, layout="io")
        return self.resid_dropout(out.view(hidden_states.shape)), None

    def mlp(self, hidden_states):
        x = hidden_states.flatten(0, 1).to(dtype)
        out = T.checkpointed_mlp(x, self.c_fc.weight, self.c_proj.weight, act="gelu", b_in=self.c_fc.bias,
                                 b_out=self.c_proj.bias, layout="io")
        return self.dropout(out.view(hidden_states.shape))

    for block in model.transformer.h:
        block.attn.forward = types.MethodType(attention, block.attn)
        block.mlp.forward = types.MethodType(mlp, block.mlp)
    model.transformer.register_forward_pre_hook(check, with_kwargs=True)


def document_lengths(total, count, longest, gen):
    """`count` or more random lengths from 1 to `longest` with the sum `total`."""
    if not 1 <= count <= total:
        raise ValueError(f"{count} documents of {total} tokens")
    cuts = torch.randperm(total - 1, generator=gen)[:count - 1] + 1
    ends = sorted(set(cuts.tolist()) | set(range(longest, total, longest)) | {total})
    return [b - a for a, b in zip([0] + ends[:-1], ends)]


def make_optimizer(name, model, lr, wd, clip=None):
    hidden = [p for n, p in model.named_parameters() if n.endswith(HIDDEN_SUFFIXES)]
    hidden_ids = {id(p) for p in hidden}
    others = [p for p in model.parameters() if id(p) not in hidden_ids]
    if name == "adamw":
        return torch.optim.AdamW(model.parameters(), lr=lr, betas=(0.9, 0.95), weight_decay=wd), hidden
    from .optim import NormPreOptimizer
    variant = {"normpre-g": "G", "normpre-l": "L", "muon": "MUON", "normalize-only": "NORM"}[name]
    groups = [{"params": hidden, "normpre": True, "lr": lr, "weight_decay": wd},
              {"params": others, "normpre": False, "lr": lr, "weight_decay": wd}]
    return NormPreOptimizer(groups, lr=lr, variant=variant, weight_decay=wd, max_grad_norm=clip), hidden


def main(argv=None):
    ap = argparse.ArgumentParser()
    ap.add_argument("--optimizer", default="normpre-g",
                    choices=["normpre-g", "normpre-l", "muon", "normalize-only", "adamw"])
    ap.add_argument("--batch", type=int, default=4)
    ap.add_argument("--seq", type=int, default=1024)
    ap.add_argument("--steps", type=int, default=10)
    ap.add_argument("--warmup", type=int, default=3)
    ap.add_argument("--lr", type=float, default=6e-4)
    ap.add_argument("--weight-decay", type=float, default=0.1)
    ap.add_argument("--clip", type=float, help="largest norm of the gradients (not with adamw)")
    ap.add_argument("--train-ops", action="store_true", help="blocks on the operators of train_ops, packed documents")
    ap.add_argument("--documents", type=int, help="documents of a packed batch (default: the batch size)")
    ap.add_argument("--dtype", default="fp32", choices=["fp32", "bf16"], help="activations, with --train-ops")
    a = ap.parse_args(argv)
    if a.clip is not None and a.optimizer == "adamw":
        ap.error("--clip is the NormPre optimizers'")
    if not torch.cuda.is_available():
        raise SystemExit("needs a GPU")
    dev = torch.device("cuda:0")
    model = build(a.seq).to(dev)
    dtype = torch.bfloat16 if a.dtype == "bf16" else torch.float32
    if a.train_ops:
        packing = Packing(dev)
        use_train_ops(model, packing, dtype)
        host_gen = torch.Generator()
        host_gen.manual_seed(1337)
    elif a.documents is not None or dtype != torch.float32:
        ap.error("--documents and --dtype need --train-ops")
    opt, hidden = make_optimizer(a.optimizer, model, a.lr, a.weight_decay, a.clip)
    gen = torch.Generator(device=dev)
    gen.manual_seed(1337)
    fb_ms, op_ms = [], []
    align = None
    for it in range(a.warmup + a.steps):
        tokens = torch.randint(0, 50257, (a.batch, a.seq), generator=gen, device=dev)
        if a.train_ops:
            lens = document_lengths(a.batch * a.seq, a.batch if a.documents is None else a.documents, a.seq,
                                    host_gen)
        torch.cuda.synchronize()
        t0 = time.perf_counter()
        if a.train_ops:
            # One row of all documents; no token is the target of another document's.
            tokens = tokens.view(1, -1)
            pos, start = packing.set(lens)
            with torch.autocast("cuda", torch.bfloat16, enabled=dtype == torch.bfloat16):
                loss = model(tokens, position_ids=pos, labels=tokens.masked_fill(start, -100)).loss
        else:
            loss = model(tokens, labels=tokens).loss
        loss.backward()
        torch.cuda.synchronize()
        t1 = time.perf_counter()
        last = it == a.warmup + a.steps - 1
        if last:
            before = [(p.detach().clone(), p.grad.detach().clone()) for p in hidden]
        opt.step()
        torch.cuda.synchronize()
        t2 = time.perf_counter()
        if last:
            # App. A descent alignment, computed by the library's kernels.
            from . import normpre as N
            actx = N.normpre_init(dev.index or 0)
            try:
                _, align = N.normpre_descent_alignment(actx, [b[1] for b in before], [b[0] for b in before],
                                                       [p.detach() for p in hidden], a.lr, a.weight_decay)
            finally:
                N.normpre_destroy(actx)
        opt.zero_grad(set_to_none=True)
        if it >= a.warmup:
            fb_ms.append(1e3 * (t1 - t0))
            op_ms.append(1e3 * (t2 - t1))
    fb = sum(fb_ms) / len(fb_ms)
    op = sum(op_ms) / len(op_ms)
    out = {"metric": "GPT-2 Small end-to-end step (synthetic tokens, random init, %s)"
                     % (a.dtype + ", packed documents, 8-bit checkpoints" if a.train_ops else "fp32"),
           "optimizer": a.optimizer, "batch": a.batch, "seq_len": a.seq, "steps": a.steps,
           "fwd_bwd_ms": round(fb, 3), "optimizer_ms": round(op, 3), "step_ms": round(fb + op, 3),
           "optimizer_share": round(op / (fb + op), 4),
           "tokens_per_s": round(a.batch * a.seq / ((fb + op) / 1e3), 1),
           "descent_alignment_last_step": None if align is None else round(align, 4),
           **({"grad_norm_last_step": round(float(opt.grad_norm), 4)} if a.clip is not None else {}),
           **({"peak_memory_gib": round(torch.cuda.max_memory_allocated() / 2 ** 30, 2)} if a.train_ops else {}),
           "final_loss": round(float(loss.detach()), 4)}
    print(json.dumps(out), flush=True)


if __name__ == "__main__":
    main()
