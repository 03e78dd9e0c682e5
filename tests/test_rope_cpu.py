"""Norms and rotation of query and key heads without a GPU: refusals of the C ABI, which come
before anything is launched, and the front end's plan of a rotation."""
import ctypes
import os

import pytest

torch = pytest.importorskip("torch")

from paper_2609_36692_amd import normpre as N  # noqa: E402
from paper_2609_36692_amd import train_ops as T  # noqa: E402

INVALID, UNSUPPORTED = N.NORMPRE_ERR_INVALID_ARG, N.NORMPRE_ERR_UNSUPPORTED
P = 1 << 40                                          # pointers that nothing may touch
H = N.normpre_heads


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not os.path.exists(N.LIB_PATH):
        from paper_2609_36692_amd import _build
        _build.build_library()
    return N.load_library()


def _block(**over):
    rows = lambda i, h: H(P + (i << 30), h * 64, 64)  # noqa: E731
    a = N.normpre_qk_rope(dtype=1, heads=4, kv_heads=2, head_dim=64, pairs=32, adjacent=0, norm=1, weight_dtype=0,
                          num_axes=1, position_bytes=4, eps=1e-6, tokens=100, freqs=P, axes=None, positions=P,
                          position_stride=0, q_weight=P, k_weight=P, q=rows(1, 4), k=rows(2, 2), q_out=rows(3, 4),
                          k_out=rows(4, 2), dq=rows(5, 4), dk=rows(6, 2), dq_weight=P, dk_weight=P, workspace=P,
                          workspace_bytes=1 << 30)
    for k, v in over.items():
        setattr(a, k, v)
    return a


@pytest.mark.parametrize("both,over,code", [
    (True, {"dtype": 2}, INVALID), (True, {"heads": 0}, INVALID), (True, {"kv_heads": -1}, INVALID),
    (True, {"heads": (1 << 16) + 1}, UNSUPPORTED), (True, {"head_dim": 0}, INVALID), (True, {"head_dim": 257}, UNSUPPORTED),
    (True, {"pairs": -1}, INVALID), (True, {"pairs": 33}, INVALID), (True, {"adjacent": 2}, INVALID),
    (True, {"norm": 2}, INVALID), (True, {"weight_dtype": 7}, INVALID), (True, {"eps": -1e-9}, INVALID),
    (True, {"eps": float("nan")}, INVALID), (True, {"eps": float("inf")}, INVALID), (True, {"tokens": -1}, INVALID),
    (True, {"tokens": 1 << 31}, UNSUPPORTED), (True, {"freqs": None}, INVALID), (True, {"freqs": P + 4}, INVALID),
    (True, {"axes": P + 2}, INVALID), (True, {"num_axes": 0}, INVALID), (True, {"num_axes": 257}, UNSUPPORTED), (True, {"position_bytes": 2}, INVALID),
    (True, {"positions": None}, INVALID), (True, {"positions": P + 4, "position_bytes": 8}, INVALID),
    (True, {"position_stride": -1}, INVALID), (True, {"position_stride": 1 << 41}, UNSUPPORTED),
    (True, {"q": H(None, 256, 64)}, INVALID), (True, {"k": H(P + 1, 128, 64)}, INVALID), (True, {"k": H(P, -1, 64)}, INVALID),
    (True, {"q": H(P, 1 << 41, 64)}, UNSUPPORTED), (True, {"q_out": H(None, 256, 64)}, INVALID),
    (True, {"q_weight": P + 2}, INVALID), (True, {"k_weight": P + 1, "weight_dtype": 1}, INVALID),
    (False, {"dq": H(P, 255, 64)}, INVALID), (False, {"dk": H(P, 0, 64)}, INVALID), (False, {"dk": H(None, 128, 64)}, INVALID),
    (False, {"dq_weight": P + 2}, INVALID), (False, {"workspace": None}, INVALID), (False, {"workspace": P + 8}, INVALID),
    (False, {"workspace_bytes": 100}, INVALID),
])
def test_refusals(lib, both, over, code):
    a = _block(**over)
    for call in [lib.normpre_qk_rope_backward] + ([lib.normpre_qk_rope_forward] if both else []):
        assert call(ctypes.byref(a), None) == code
        assert N.normpre_last_error()


def test_forward_outputs_must_not_overlap(lib):
    for name in ("q_out", "k_out"):
        for rows in (H(P, 0, 64), H(P, 256, 0), H(P, 64, 64), H(P, 127, 64)):
            assert lib.normpre_qk_rope_forward(ctypes.byref(_block(**{name: rows})), None) == INVALID
            assert "overlap" in N.normpre_last_error()


def test_workspace_and_empty_batch(lib):
    n = ctypes.c_int64(-1)
    assert lib.normpre_qk_rope_workspace(None, ctypes.byref(n)) == INVALID
    assert lib.normpre_qk_rope_workspace(ctypes.byref(_block()), None) == INVALID
    assert lib.normpre_qk_rope_forward(None, None) == INVALID
    for over, need in (({}, True), ({"norm": 0}, False), ({"dq_weight": None, "dk_weight": None}, False),
                       ({"dk_weight": None}, True), ({"tokens": 0}, False), ({"tokens": (1 << 31) - 1}, True)):
        assert lib.normpre_qk_rope_workspace(ctypes.byref(_block(**over)), ctypes.byref(n)) == 0
        assert (n.value > 0) == need and n.value % (4 * 2 * 64) == 0 and n.value <= 1024 * 2 * 64 * 4
    # Nothing to read or write: nothing is asked for.
    empty = _block(tokens=0, freqs=None, positions=None, q=H(None, 0, 0), q_out=H(None, 0, 0), workspace=None)
    assert lib.normpre_qk_rope_forward(ctypes.byref(empty), None) == 0
    empty.dq_weight = empty.dk_weight = None
    assert lib.normpre_qk_rope_backward(ctypes.byref(empty), None) == 0


def test_layout_matches_the_front_end():
    assert ctypes.sizeof(N.normpre_qk_rope) == T._ROPE.size
    a = N.normpre_qk_rope.from_buffer_copy(T._ROPE.pack(*range(10), 0.5, *range(11, 40)))
    assert (a.dtype, a.position_bytes, a.eps, a.tokens, a.freqs, a.position_stride) == (0, 9, 0.5, 11, 12, 15)
    assert (a.k_weight, a.q.data, a.k_out.head_stride, a.dk.data, a.dk_weight, a.workspace_bytes) == (17, 18, 29, 33, 37, 39)


def test_rotary():
    r = T.Rotary([1.0, 0.25], device="cpu")
    assert (r.pairs, r.num_axes, r.axes, r.adjacent) == (2, 1, None, False) and r.freqs.dtype == torch.float64
    r = T.Rotary([1.0, 0.25, 0.5], [0, 2, 1], True, "cpu")
    assert r.num_axes == 3 and r.axes.tolist() == [0, 2, 1] and r.axes.dtype == torch.int32 and r.adjacent
    assert T.Rotary([], device="cpu").pairs == 0
    assert T.Rotary.geometric(4, 100.0) == [1.0, 0.1]
    assert T.Rotary.geometric(0) == []
    for bad in (lambda: T.Rotary([1.0, float("inf")], device="cpu"), lambda: T.Rotary([float("nan")], device="cpu"),
                lambda: T.Rotary([1.0], [0, 1], device="cpu"), lambda: T.Rotary([1.0], [-1], device="cpu"),
                lambda: T.Rotary.geometric(5), lambda: T.Rotary.geometric(-2)):
        with pytest.raises(ValueError):
            bad()
