"""Calls of clip_grads in the ways that a program makes them: outputs from a generator on another
device than the current one."""
import contextlib
from array import array

import pytest

torch = pytest.importorskip("torch")

from paper_2609_36692_amd import train_ops as T  # noqa: E402


def _elsewhere_at_first(monkeypatch):
    """As where the tensors' device is not the current one: the call starts over, once."""
    answers = iter([True, False])
    monkeypatch.setattr(T, "_elsewhere", lambda at: next(answers))


@pytest.mark.parametrize("kind", [list, iter, lambda x: (t for t in x)], ids=["list", "iterator", "generator"])
def test_outputs_survive_the_change_of_device(monkeypatch, kind):
    # Without a GPU: what reaches the kernels' list after the call has started over.
    grads, outs = [torch.ones(3), torch.ones(2, 4)], [torch.zeros(3), torch.zeros(2, 4)]
    seen = []
    _elsewhere_at_first(monkeypatch)
    monkeypatch.setattr(T, "_grad_entries", lambda g, o: seen.append((list(g), list(o))) or (0, array("Q", [0])))
    monkeypatch.setattr(T, "_grad_workspace", lambda like: (torch.zeros(()), torch.zeros(1)))
    monkeypatch.setattr(T, "_stream", lambda at: None)
    monkeypatch.setattr(T.N, "normpre_grad_clip", lambda *a: None)
    monkeypatch.setattr(torch.cuda, "device", lambda at: contextlib.nullcontext())
    T.clip_grads(kind(grads), 1.0, out=kind(outs))
    assert len(seen) == 2
    for g, o in seen:
        assert all(a is b for a, b in zip(g, grads)) and all(a is b for a, b in zip(o, outs)) and len(g) == len(o) == 2


@pytest.mark.gpu
def test_outputs_from_a_generator(monkeypatch):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    dev = torch.device("cuda:0")
    grads = [torch.full((100,), 3.0, device=dev), torch.full((44,), 4.0, device=dev)]
    outs = [torch.zeros_like(g) for g in grads]
    _elsewhere_at_first(monkeypatch)
    norm = T.clip_grads((g for g in grads), 1.0, out=(o for o in outs))
    assert abs(float(norm) - (900.0 + 704.0) ** 0.5) < 1e-4
    for g, o in zip(grads, outs):
        # One rounding of the factor's product, and 2^-40 for the factor.
        assert float((o.double() * (900.0 + 704.0) ** 0.5 / g.double() - 1.0).abs().max()) <= 2.0 ** -24 + 2.0 ** -40
