"""The gradient norm and clipping without a GPU: refusals of the C ABI, which come
before anything is launched, and of the front end."""
import ctypes
import os

import pytest

torch = pytest.importorskip("torch")

from paper_2609_36692_amd import normpre as N  # noqa: E402
from paper_2609_36692_amd import train_ops as T  # noqa: E402

INVALID, UNSUPPORTED = N.NORMPRE_ERR_INVALID_ARG, N.NORMPRE_ERR_UNSUPPORTED
P = 1 << 40                                          # pointers that nothing may touch
WS = N.NORMPRE_GRAD_WORKSPACE_BYTES


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not os.path.exists(N.LIB_PATH):
        from paper_2609_36692_amd import _build
        _build.build_library()
    return N.load_library()


def _list(*entries):
    return (N.normpre_grad * max(1, len(entries)))(*[N.normpre_grad(*e) for e in entries])


GOOD = (P, P, 100, 0, 0)


@pytest.mark.parametrize("both,entries,code", [
    (True, [(P, P, 100, 2, 0)], INVALID), (True, [GOOD, (P + 4096, P + 4096, -1, 0, 0)], INVALID),
    (True, [(None, P, 100, 0, 0)], INVALID), (True, [(P + 2, P + 2, 100, 0, 0)], INVALID),
    (True, [(P + 1, P + 1, 100, 1, 1)], INVALID), (True, [(P, P, (1 << 40) + 1, 0, 0)], UNSUPPORTED),
    (True, [(P, P, 1 << 40, 0, 0), (P >> 1, P >> 1, 1, 0, 0)], UNSUPPORTED),
    (False, [(P, P, 100, 0, -1)], INVALID), (False, [(P, None, 100, 0, 0)], INVALID), (False, [(P, P + 2, 100, 1, 0)], INVALID),
    # Outputs on each other, on another's gradient, on a part of their own, in place with another type.
    (False, [GOOD, (P + 4096, P + 396, 100, 0, 0)], INVALID), (False, [GOOD, GOOD], INVALID),
    (False, [(P, P + 4096, 2000, 0, 0)], INVALID), (False, [(P, P, 100, 1, 0)], INVALID), (False, [(P, P, 100, 0, 1)], INVALID),
    (False, [(P, P + 8192, 100, 0, 0), (P + 8192 + 396, P, 100, 0, 0)], INVALID),
    (False, [(P, P + 4, 100, 0, 0)], INVALID),
    (False, [GOOD, (P + 400, P + 400, 100, 0, 0), (P + 396, P + 8192, 2, 0, 0)], INVALID),
])
def test_refusals_of_entries(lib, both, entries, code):
    arr = _list(*entries)
    assert lib.normpre_grad_clip(len(entries), arr, 1.0, P, P, WS, None) == code
    assert N.normpre_last_error()
    if both:
        assert lib.normpre_grad_norm(len(entries), arr, P, P, WS, None) == code


@pytest.mark.parametrize("over,code", [
    ({"num": -1}, INVALID), ({"num": (1 << 20) + 1}, UNSUPPORTED), ({"list": None}, INVALID), ({"norm": None}, INVALID),
    ({"norm": P + 2}, INVALID), ({"work": None}, INVALID), ({"work": P + 8}, INVALID), ({"bytes": WS - 1}, INVALID),
    ({"max": -1.0}, INVALID), ({"max": float("nan")}, INVALID),
])
def test_refusals_of_arguments(lib, over, code):
    a = {"num": 1, "list": _list(GOOD), "norm": P, "work": P, "bytes": WS, "max": 1.0} | over
    assert lib.normpre_grad_clip(a["num"], a["list"], a["max"], a["norm"], a["work"], a["bytes"], None) == code
    assert N.normpre_last_error()
    if "max" not in over:
        assert lib.normpre_grad_norm(a["num"], a["list"], a["norm"], a["work"], a["bytes"], None) == code


def test_struct_layout():
    assert ctypes.sizeof(N.normpre_grad) == 32 and N.normpre_grad.dtype.offset == 24


def test_front_end_refusals():
    x = torch.zeros(4)
    with pytest.raises(ValueError, match="GPU"):
        T.clip_grads([x], 1.0)
    with pytest.raises(ValueError, match="GPU"):
        T.grad_norm(x)
    with pytest.raises(ValueError, match="max_norm"):
        T.clip_grads([x], -1.0)
    with pytest.raises(ValueError, match="max_norm"):
        T.clip_grads([x], float("nan"))
    with pytest.raises(ValueError, match="shapes"):
        T.clip_grads([x], 1.0, out=[])
    with pytest.raises(ValueError, match="shapes"):
        T.clip_grads([x], 1.0, out=[torch.zeros(2, 2)])
    with pytest.raises(ValueError, match="share"):
        T.clip_grads([torch.zeros(1).expand(4)], 1.0)
    assert float(T.grad_norm([])) == 0.0 and float(T.clip_grads([], 1.0)) == 0.0


@pytest.mark.parametrize("x,dense", [
    (torch.zeros(3, 4), True), (torch.zeros(3, 4).t(), True), (torch.zeros(3, 4)[:, ::2], False),
    (torch.zeros(2, 3, 4).permute(2, 0, 1), True), (torch.zeros(3, 1).expand(3, 4), False), (torch.zeros(0, 3), True),
    (torch.zeros(()), True), (torch.zeros(3, 4)[:, :3], False), (torch.zeros(5, 1)[:, 0], True), (torch.zeros(6)[::2], False),
])
def test_dense(x, dense):
    assert T._dense(x) == dense


def test_optimizer_refusals():
    from paper_2609_36692_amd import e2e_gpt2 as E
    from paper_2609_36692_amd.optim import NormPreOptimizer
    m = torch.nn.Linear(8, 16)
    for limit in (-1.0, float("nan")):
        with pytest.raises(ValueError, match="max_grad_norm"):
            NormPreOptimizer(m.parameters(), max_grad_norm=limit)
    with pytest.raises(SystemExit):
        E.main(["--optimizer", "adamw", "--clip", "1.0"])
