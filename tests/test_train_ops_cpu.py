"""Training-step operators without a GPU: the plan of a packed batch, and the
refusals of the C ABI, which come before anything is launched."""
import ctypes
import os

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2609_36692_amd import normpre as N  # noqa: E402

INVALID, UNSUPPORTED = N.NORMPRE_ERR_INVALID_ARG, N.NORMPRE_ERR_UNSUPPORTED


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not os.path.exists(N.LIB_PATH):
        from paper_2609_36692_amd import _build
        _build.build_library()
    return N.load_library()


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("lens", [[], [0], [1], [128], [129], [300, 0, 1, 128, 1000], [5] * 40])
def test_plan_covers_every_row_once_by_falling_work(lens, causal):
    plan = N.normpre_attention_plan(lens, causal)
    starts = np.cumsum([0] + lens)
    for side in range(2):
        rows = np.zeros(sum(lens), int)
        work = []
        for start, n, tile, zero in plan[side].tolist():
            i = [j for j, s in enumerate(starts[:-1]) if s == start and lens[j] == n][0]
            assert zero == 0 and n > 0 and 0 <= 128 * tile < n
            end = min(n, 128 * (tile + 1))
            rows[starts[i] + 128 * tile:starts[i] + end] += 1
            work.append(n if not causal else end if side == 0 else n - 128 * tile)
        assert (rows == 1).all()
        assert work == sorted(work, reverse=True)


def test_plan_refusals(lib):
    tiles = ctypes.c_int64()
    one = (ctypes.c_int64 * 2)(1, -1)
    assert lib.normpre_attention_plan_tiles(2, one, ctypes.byref(tiles)) == INVALID
    assert "negative" in N.normpre_last_error()
    assert lib.normpre_attention_plan_tiles(1, None, ctypes.byref(tiles)) == INVALID
    assert lib.normpre_attention_plan_tiles(-1, one, ctypes.byref(tiles)) == INVALID
    assert lib.normpre_attention_plan_tiles(1, one, None) == INVALID
    big = (ctypes.c_int64 * 2)(2 ** 31 - 1, 1)
    assert lib.normpre_attention_plan_tiles(2, big, ctypes.byref(tiles)) == UNSUPPORTED
    assert lib.normpre_attention_plan_tiles(1, (ctypes.c_int64 * 1)(2 ** 62), ctypes.byref(tiles)) == UNSUPPORTED
    buf = (ctypes.c_int32 * 8)()
    ok = (ctypes.c_int64 * 1)(100)
    assert lib.normpre_attention_plan(1, ok, 1, buf, 7) == INVALID
    assert lib.normpre_attention_plan(1, ok, 2, buf, 8) == INVALID
    assert lib.normpre_attention_plan(1, ok, 1, None, 8) == INVALID
    assert lib.normpre_attention_plan(1, ok, 1, buf, 8) == 0


def _block(**over):
    """A valid argument block on pointers that nothing may touch."""
    at = 1 << 40
    rows = lambda i, h: N.normpre_heads(at + (i << 30), h * 64, 64)  # noqa: E731
    a = N.normpre_attention(dtype=1, heads=4, kv_heads=2, head_dim=64, causal=1, scale=0.125, tokens=100, plan=at,
                            num_tiles=1, q=rows(1, 4), k=rows(2, 2), v=rows(3, 2), out=rows(4, 4), lse=at + (5 << 30),
                            dout=rows(6, 4), dq=rows(7, 4), dk=rows(8, 2), dv=rows(9, 2), workspace=at + (10 << 30), workspace_bytes=1 << 30)
    for k, v in over.items():
        setattr(a, k, v)
    return a


H = N.normpre_heads
P = 1 << 40


@pytest.mark.parametrize("both,over,code", [
    (True, {"dtype": 2}, INVALID), (True, {"dtype": -1}, INVALID),
    (True, {"heads": 0}, INVALID), (True, {"kv_heads": 0}, INVALID), (True, {"kv_heads": 3}, INVALID),
    (True, {"head_dim": 0}, INVALID), (True, {"head_dim": 129}, UNSUPPORTED),
    (True, {"causal": 2}, INVALID), (True, {"scale": float("inf")}, INVALID), (True, {"scale": float("nan")}, INVALID),
    (True, {"tokens": -1}, INVALID), (True, {"tokens": 1 << 31}, UNSUPPORTED), (True, {"tokens": 129}, INVALID),
    (True, {"num_tiles": 0}, INVALID), (True, {"num_tiles": 101}, INVALID), (True, {"num_tiles": -1}, INVALID),
    (True, {"plan": None}, INVALID), (True, {"plan": P + 4}, INVALID), (True, {"lse": None}, INVALID),
    (True, {"lse": P + 2}, INVALID), (True, {"q": H(None, 256, 64)}, INVALID), (True, {"k": H(P + 1, 128, 64)}, INVALID),
    (True, {"v": H(P, -128, 64)}, INVALID), (True, {"q": H(P, 1 << 41, 64)}, UNSUPPORTED),
    (True, {"out": H(None, 256, 64)}, INVALID),
    (False, {"dout": H(None, 256, 64)}, INVALID), (False, {"dq": H(P, 255, 64)}, INVALID),
    (False, {"dk": H(P, 0, 64)}, INVALID), (False, {"dv": H(P, 128, 63)}, INVALID),
    (False, {"workspace": None}, INVALID), (False, {"workspace": P + 4}, INVALID),
    (False, {"workspace_bytes": 4 * 2 * 4 * 100 - 1}, INVALID),
    (True, {"tokens": 2 ** 31 - 1, "num_tiles": 2 ** 31 - 1}, UNSUPPORTED),
])
def test_attention_refusals(lib, both, over, code):
    a = _block(**over)
    calls = [lib.normpre_attention_backward] + ([lib.normpre_attention_forward] if both else [])
    for call in calls:
        assert call(ctypes.byref(a), None) == code
        assert N.normpre_last_error()


def test_attention_forward_output_must_not_overlap(lib):
    for out in (H(P, 0, 64), H(P, 256, 0), H(P, 255, 64), H(P, 64, 64)):
        assert lib.normpre_attention_forward(ctypes.byref(_block(out=out)), None) == INVALID
        assert "overlap" in N.normpre_last_error()


def test_attention_overlap_of_far_rows(lib):
    # (tokens - 1) * stride past 64 bits: heads 32 elements apart overlap all the same.
    sizes = dict(heads=2, kv_heads=2, tokens=(1 << 23) + 1, num_tiles=(1 << 16) + 1, workspace_bytes=1 << 62)
    for name in ("out", "dq", "dk", "dv"):
        a = _block(**sizes, **{name: H(P, 1 << 40, 32)})
        call = lib.normpre_attention_forward if name == "out" else lib.normpre_attention_backward
        assert call(ctypes.byref(a), None) == INVALID, name
        assert "overlap" in N.normpre_last_error()


def test_attention_null_block_and_empty_batch(lib):
    assert lib.normpre_attention_forward(None, None) == INVALID
    empty = _block(tokens=0, num_tiles=0, q=H(None, 0, 0), plan=None)
    assert lib.normpre_attention_forward(ctypes.byref(empty), None) == 0
    assert lib.normpre_attention_backward(ctypes.byref(empty), None) == 0


def test_attention_workspace(lib):
    a = _block()
    size = ctypes.c_int64()
    assert lib.normpre_attention_workspace(ctypes.byref(a), ctypes.byref(size)) == 0
    assert size.value >= 4 * 2 * 4 * 100
    a.workspace_bytes = size.value - 1
    assert lib.normpre_attention_backward(ctypes.byref(a), None) == INVALID
    assert lib.normpre_attention_workspace(ctypes.byref(a), None) == INVALID
    assert lib.normpre_attention_workspace(None, ctypes.byref(size)) == INVALID
    a.head_dim = 0
    assert lib.normpre_attention_workspace(ctypes.byref(a), ctypes.byref(size)) == INVALID


def test_checkpoint_refusals(lib):
    pack = lambda act=1, dt=1, rows=4, cols=70, u=P, ldu=70, up=P, ldup=70, h=P, ldh=70, cu=P, eu=P, cup=P, eup=P, \
        ch=P, eh=P: lib.normpre_checkpoint_pack(act, dt, rows, cols, u, ldu, up, ldup, h, ldh, cu, eu, cup, eup,  # noqa: E731
                                                ch, eh, None)
    for bad in ({"act": 3}, {"act": -1}, {"dt": 2}, {"rows": -1}, {"cols": 0}, {"u": None}, {"u": P + 1},
                {"ldu": 69}, {"cu": None}, {"eu": None}, {"cu": P + 8}, {"h": None}, {"ldh": 69}, {"ch": None},
                {"act": 2, "up": None}, {"act": 2, "ldup": 3}, {"act": 2, "cup": None}, {"act": 2, "eup": None}):
        assert pack(**bad) == INVALID, bad
        assert N.normpre_last_error()
    assert pack(rows=1 << 40) == UNSUPPORTED
    assert pack(cols=(1 << 40) + 1, ldu=1 << 62) == UNSUPPORTED
    assert pack(ldu=1 << 41) == UNSUPPORTED
    assert pack(rows=0, u=None, cu=None) == 0

    unpack = lambda dt=1, rows=4, cols=70, c=P, e=P, out=P, ld=70: \
        lib.normpre_checkpoint_unpack(dt, rows, cols, c, e, out, ld, None)  # noqa: E731
    for bad in ({"dt": 5}, {"rows": -1}, {"cols": -1}, {"c": None}, {"c": P + 1}, {"e": None}, {"out": None},
                {"ld": 69}):
        assert unpack(**bad) == INVALID, bad
    assert unpack(rows=0, out=None) == 0

    grad = lambda act=1, dt=1, rows=4, cols=70, dh=P, ldh=70, cu=P, eu=P, cup=P, eup=P, du=P, ldu=70, dup=P, \
        ldup=70: lib.normpre_checkpoint_act_grad(act, dt, rows, cols, dh, ldh, cu, eu, cup, eup, du, ldu, dup,  # noqa: E731
                                                 ldup, None)
    for bad in ({"act": 0}, {"act": 3}, {"dt": 2}, {"rows": -2}, {"cols": 0}, {"dh": None}, {"cu": P + 4},
                {"du": None}, {"ldu": 1}, {"act": 2, "cup": None}, {"act": 2, "dup": None}, {"act": 2, "ldup": 0}):
        assert grad(**bad) == INVALID, bad
    assert grad(rows=0, du=None) == 0


def test_weight_grad_refusals(lib):
    need = N.normpre_checkpoint_weight_grad_workspace(1, 4096, 128, 128)
    assert need > 0 and need % (4 * 128 * 128) == 0
    call = lambda dt=1, layout=0, acc=0, t=4096, i=128, o=128, c=P, e=P, dy=P, ldy=128, dw=P, ldw=128, ws=P, \
        n=need: lib.normpre_checkpoint_weight_grad(dt, layout, acc, t, i, o, c, e, dy, ldy, dw, ldw, ws, n, None)  # noqa: E731
    for bad in ({"dt": 2}, {"layout": 2}, {"layout": -1}, {"acc": 2}, {"t": -1}, {"i": 0}, {"o": 0}, {"c": None},
                {"c": P + 1}, {"e": None}, {"dy": None}, {"dy": P + 1}, {"ldy": 127}, {"dw": None}, {"dw": P + 2},
                {"ldw": 127}, {"ws": None}, {"ws": P + 8}, {"n": need - 1}):
        assert call(**bad) == INVALID, bad
        assert N.normpre_last_error()
    assert call(t=1 << 31, i=1, o=1) == UNSUPPORTED
    assert call(i=1 << 31, ldw=1 << 31, o=1, t=1) == UNSUPPORTED
    size = ctypes.c_int64()
    assert lib.normpre_checkpoint_weight_grad_workspace(1, 4096, 128, 128, None) == INVALID
    assert lib.normpre_checkpoint_weight_grad_workspace(7, 4096, 128, 128, ctypes.byref(size)) == INVALID
    assert lib.normpre_checkpoint_weight_grad_workspace(1, 1, 128, 128, ctypes.byref(size)) == 0 and size.value == 0


def test_front_end_needs_a_gpu_tensor():
    from paper_2609_36692_amd import train_ops as T
    x = torch.randn(4, 64)
    for call in (lambda: T.checkpoint_pack(x), lambda: T.checkpoint_act("gelu", x),
                 lambda: T.attention_forward(x[:, None], x[:, None], x[:, None], T.AttentionPlan([4], device="cpu"))):
        with pytest.raises(ValueError):
            call()


def _small_gpt2(**over):
    transformers = pytest.importorskip("transformers")
    cfg = dict(n_layer=1, n_embd=64, n_head=1, n_positions=32, vocab_size=50, bos_token_id=0, eos_token_id=0)
    return transformers.GPT2LMHeadModel(transformers.GPT2Config(**cfg | over))


def test_patched_model_refuses_what_its_blocks_would_ignore():
    from paper_2609_36692_amd import e2e_gpt2 as E
    model, packing = _small_gpt2(), E.Packing("cpu")
    E.use_train_ops(model, packing)
    tokens = torch.zeros(1, 4, dtype=torch.long)
    with pytest.raises(ValueError, match="lengths"):
        model(tokens)
    packing.set([3, 1])
    mask = torch.tensor([[1, 1, 0, 0]])
    for name, value in {"attention_mask": mask, "past_key_values": object(), "use_cache": True, "output_attentions": True,
                        "encoder_hidden_states": torch.zeros(1, 4, 64), "head_mask": torch.ones(1)}.items():
        with pytest.raises(ValueError, match=name):
            model(tokens, **{name: value})
    with pytest.raises(ValueError, match="past_key_values|attention_mask|use_cache"):
        model.generate(tokens, max_new_tokens=1)
    # What it honours comes as far as the first kernel's check of its device.
    with pytest.raises(ValueError, match="GPU"):
        model(tokens, position_ids=torch.tensor([[0, 1, 2, 0]]), labels=tokens, attention_mask=None, use_cache=False)


def test_models_that_the_operators_do_not_compute_are_refused():
    from paper_2609_36692_amd import e2e_gpt2 as E
    for over in ({"activation_function": "relu"}, {"activation_function": "gelu"}, {"add_cross_attention": True}):
        with pytest.raises(ValueError):
            E.use_train_ops(_small_gpt2(**over), E.Packing("cpu"))


def test_front_end_refusals_of_shapes():
    from paper_2609_36692_amd import train_ops as T
    plan = T.AttentionPlan([4], device="cpu")
    q, flat = torch.randn(4, 2, 64), torch.randn(4, 128)
    for args in ((flat, q, q), (q, flat, q), (q, q, flat), (q[0, 0], q, q)):
        with pytest.raises(ValueError, match="tokens, heads, dim"):
            T.attention_forward(*args, plan)
    with pytest.raises(ValueError):
        T.attention_backward(q, q, flat, q, q, torch.zeros(2, 4), plan)
    # Layers, also with nothing to train: no result from anything but the kernels.
    w = torch.randn(64, 128)
    with pytest.raises(ValueError, match="GPU"):
        T.checkpointed_linear(flat, w)
    with pytest.raises(ValueError, match="GPU"):
        T.checkpointed_mlp(flat, w, w.t())
    with pytest.raises(ValueError, match="tokens, inner"):
        T.checkpointed_linear(flat[None], w)
    with pytest.raises(ValueError, match="tokens, inner"):
        T.checkpointed_mlp(flat[None], w, w.t())
    with pytest.raises(ValueError, match="layout"):
        T.checkpointed_linear(flat, w, layout="xy")


@pytest.mark.parametrize("total,count,longest", [(1, 1, 1), (8, 8, 8), (64, 60, 16), (4096, 24, 1024), (100, 1, 30)])
def test_document_lengths(total, count, longest):
    from paper_2609_36692_amd import e2e_gpt2 as E
    gen = torch.Generator().manual_seed(5)
    for _ in range(20):
        lens = E.document_lengths(total, count, longest, gen)
        assert sum(lens) == total and len(lens) >= count and 1 <= min(lens) and max(lens) <= longest
    for bad in (0, -1, total + 1):
        with pytest.raises(ValueError):
            E.document_lengths(total, bad, longest, gen)
