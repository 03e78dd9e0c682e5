"""Attention with a window without a GPU: its plans, and the refusals of the C ABI, which come
before anything is launched."""
import ctypes
import os

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2609_36692_amd import normpre as N  # noqa: E402
from paper_2609_36692_amd import train_ops as T  # noqa: E402

INVALID, UNSUPPORTED = N.NORMPRE_ERR_INVALID_ARG, N.NORMPRE_ERR_UNSUPPORTED
P = 1 << 40                                          # pointers that nothing may touch
H, W = N.normpre_heads, N.normpre_window


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not os.path.exists(N.LIB_PATH):
        from paper_2609_36692_amd import _build
        _build.build_library()
    return N.load_library()


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (100, 4), (128, 200), (5000, 3), (1 << 40, 1 << 40), (7, 128)])
@pytest.mark.parametrize("lens", [[], [0], [1], [129], [300, 0, 1, 128, 4000], [2000] * 40, [70000]])
def test_plan(lens, window, sinks):
    plan, tiles, b = N.normpre_window_attention_plan(lens, window, sinks)
    starts, zero = np.cumsum([0] + lens), {}
    for side in range(2):
        rows, work = np.zeros(sum(lens), int), []
        for start, n, tile, mark in plan[4 * tiles * side:4 * tiles * (side + 1)].reshape(-1, 4).tolist():
            i = [j for j, s in enumerate(starts[:-1]) if s == start and lens[j] == n][0]
            first, end = 128 * tile, min(n, 128 * (tile + 1))
            assert n > 0 and 0 <= first < n
            rows[starts[i] + first:starts[i] + end] += 1
            lo = max(0, first - window + 1)
            work.append(end - lo + min(sinks, lo) if side == 0 else min(n - first, window + 127))
            assert mark == 0 if side == 0 or first >= sinks or n - first <= window else mark > 0
            if mark:
                zero[mark - 1] = (start, n, tile)
        assert (rows == 1).all() and work == sorted(work, reverse=True)
    # Sinks and their pieces: every slot once.
    at = 8 * tiles
    sink = plan[at:at + 8 * b.sink_tiles].reshape(-1, 8).tolist()
    pieces = plan[at + 8 * b.sink_tiles:].reshape(-1, 4).tolist()
    assert len(pieces) == b.sink_pieces <= b.sink_tiles + 512
    assert zero == {i: tuple(s[:3]) for i, s in enumerate(sink)}
    slots = sorted([s[3] + s[4] for s in sink] + [p[2] for p in pieces])
    assert slots == list(range(b.sink_tiles + b.sink_pieces))
    by = {}
    for s, piece, slot, _ in pieces:
        assert slot == sink[s][3] + piece
        by.setdefault(s, []).append(piece)
    assert all(sorted(by[i]) == list(range(s[4])) and s[4] >= 1 for i, s in enumerate(sink))


def test_front_end_takes_a_window_only_where_it_hides_something():
    assert T.AttentionPlan([10, 50], device="cpu", window=50).bounds is None
    assert T.AttentionPlan([10, 50], device="cpu", window=40, sinks=10).bounds is None
    p = T.AttentionPlan([10, 50], device="cpu", window=40, sinks=9)
    assert (p.bounds.window, p.bounds.sinks, p.bounds.sink_tiles, p.bounds.sink_pieces) == (40, 9, 1, 1)
    assert T.AttentionPlan([], device="cpu", window=1).bounds is None
    for args in ({"window": 0}, {"window": 3, "sinks": -1}, {"sinks": 1}, {"window": 3, "causal": False}):
        with pytest.raises(ValueError):
            T.AttentionPlan([5], device="cpu", **args)


def test_plan_refusals(lib):
    n = ctypes.c_int64()
    ok = (ctypes.c_int64 * 2)(300, 100)
    sizes = lib.normpre_window_attention_plan_sizes
    for w in (W(0, 0), W(-5, 0), W(1, -1)):
        assert sizes(2, ok, w, n) == INVALID
    assert sizes(2, ok, None, n) == INVALID and sizes(2, ok, W(5, 5), None) == INVALID
    assert sizes(2, None, W(5, 5), n) == INVALID and sizes(-1, ok, W(5, 5), n) == INVALID
    assert sizes(2, (ctypes.c_int64 * 2)(1, -1), W(5, 5), n) == INVALID
    assert sizes(2, (ctypes.c_int64 * 2)(2 ** 31 - 1, 1), W(5, 5), n) == UNSUPPORTED
    w = W(5, 5)
    assert sizes(2, ok, w, n) == 0 and (n.value, w.sink_tiles, w.sink_pieces) == (4, 2, 3)
    buf = (ctypes.c_int32 * 100)()
    plan = lib.normpre_window_attention_plan
    need = 8 * 4 + 8 * 2 + 4 * 3
    assert plan(2, ok, w, buf, need) == 0
    assert plan(2, ok, w, buf, need - 1) == INVALID and plan(2, ok, w, None, need) == INVALID
    assert plan(2, ok, W(5, 5, 1, 1), buf, need) == INVALID and plan(2, ok, W(0, 5, 2, 3), buf, need) == INVALID
    assert plan(2, ok, None, buf, need) == INVALID
    assert plan(1, ok, w, buf, need) == INVALID      # another batch's


def _block(**over):
    rows = lambda i, h: H(P + (i << 30), h * 64, 64)  # noqa: E731
    a = N.normpre_attention(dtype=1, heads=4, kv_heads=2, head_dim=64, causal=1, scale=0.125, tokens=300, plan=P,
                            num_tiles=3, q=rows(1, 4), k=rows(2, 2), v=rows(3, 2), out=rows(4, 4), lse=P, dout=rows(6, 4),
                            dq=rows(7, 4), dk=rows(8, 2), dv=rows(9, 2), workspace=P, workspace_bytes=1 << 30)
    for k, v in over.items():
        setattr(a, k, v)
    return a


@pytest.mark.parametrize("over,window,code", [
    ({}, (0, 0, 0, 0), INVALID), ({}, (5, -1, 0, 0), INVALID), ({}, (5, 1, -1, 0), INVALID), ({}, (5, 1, 4, 4), INVALID),
    ({}, (5, 1, 1, 0), INVALID), ({}, (5, 1, 1, 514), INVALID), ({}, (5, 1, 0, 1), INVALID), ({}, (5, 0, 1, 1), INVALID),
    ({"causal": 0}, (5, 1, 1, 1), INVALID), ({"heads": 0}, (5, 1, 1, 1), INVALID), ({"head_dim": 129}, (5, 1, 1, 1), UNSUPPORTED),
    ({"q": H(None, 256, 64)}, (5, 1, 1, 1), INVALID), ({"plan": None}, (5, 1, 1, 1), INVALID), ({"lse": P + 2}, (5, 1, 1, 1), INVALID),
    ({"tokens": 385}, (5, 1, 1, 1), INVALID), ({"scale": float("nan")}, (5, 1, 1, 1), INVALID),
    ({"heads": 1 << 15, "kv_heads": 1 << 15, "tokens": 300}, (5, 1, 3, 400), UNSUPPORTED),
])
def test_refusals(lib, over, window, code):
    a, w = _block(**over), W(*window)
    for call in (lib.normpre_window_attention_forward, lib.normpre_window_attention_backward):
        assert call(ctypes.byref(a), ctypes.byref(w), None) == code
        assert N.normpre_last_error()
    n = ctypes.c_int64()
    if not set(over) & {"q", "plan", "lse"}:
        assert lib.normpre_window_attention_workspace(a, w, n) == code


def test_backward_refusals_and_workspace(lib):
    w, n = W(5, 1, 1, 1), ctypes.c_int64()
    assert lib.normpre_window_attention_workspace(_block(), w, n) == 0
    need = n.value
    # Statistics, four shares of dk and dv, and the sums of two slots of 32 rows, four shares each.
    assert need == 4 * (2 * 4 * 300 + 2 * 4 * 2 * 300 * 64 + 2 * 4 * 2 * 2 * 32 * 64)
    assert lib.normpre_window_attention_workspace(_block(), None, n) == INVALID
    assert lib.normpre_window_attention_workspace(None, w, n) == INVALID
    assert lib.normpre_window_attention_workspace(_block(), w, None) == INVALID
    call = lib.normpre_window_attention_backward
    for over in ({"workspace_bytes": need - 1}, {"workspace": None}, {"workspace": P + 4}, {"dq": H(P, 255, 64)},
                 {"dk": H(P, 0, 64)}, {"dv": H(None, 128, 64)}, {"dout": H(P, -1, 64)}):
        assert call(ctypes.byref(_block(**over)), w, None) == INVALID
    empty = _block(tokens=0, num_tiles=0, plan=None)
    assert call(ctypes.byref(empty), W(5, 1, 0, 0), None) == 0
    assert lib.normpre_window_attention_forward(ctypes.byref(empty), W(5, 1, 0, 0), None) == 0
    assert lib.normpre_window_attention_forward(ctypes.byref(_block(out=H(P, 0, 64))), w, None) == INVALID
