"""Calls of clip_grads in the ways that a program makes them: outputs from a generator on another
device than the current one, and gradients that a graph still holds."""
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


@pytest.mark.gpu
@pytest.mark.parametrize("limit", [0.1, 1e9])        # scaled, and left as they are
def test_writes_are_seen_by_autograd(limit):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    dev = torch.device("cuda:0")
    grads = [torch.ones(5, device=dev), torch.ones(4, 6, device=dev)[:, ::2], torch.ones(3, 4, device=dev, dtype=torch.bfloat16).t()]
    outs = [torch.zeros(5, device=dev), torch.zeros(4, 3, device=dev), torch.zeros(8, 3, device=dev)[::2]]
    before = [x._version for x in grads + outs]
    T.grad_norm(grads)
    assert [x._version for x in grads + outs] == before
    T.clip_grads(grads, limit, out=outs)
    assert [x._version for x in grads] == before[:3] and all(x._version > v for x, v in zip(outs, before[3:]))
    T.clip_grads(grads, limit)
    assert all(x._version > v for x, v in zip(grads, before))
    with torch.inference_mode():                     # tensors without a version
        x = torch.full((7,), 2.0, device=dev)
        T.clip_grads([x], limit)


@pytest.mark.gpu
def test_a_gradient_that_was_kept_and_clipped_is_refused():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    w = torch.tensor([1.0, 2.0, 3.0], device="cuda:0", requires_grad=True)
    g, = torch.autograd.grad((w ** 3).sum(), w, create_graph=True)
    penalty = (g * g).sum()                          # keeps g
    T.clip_grads([g], 0.5)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        penalty.backward()
