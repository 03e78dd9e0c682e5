"""Norms and rotation of query and key heads on the GPU against 64-bit references, with the
bounds of tests/rope_util.py."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

import rope_util as R  # noqa: E402
from paper_2609_36692_amd import train_ops as T  # noqa: E402

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
KIND = {BF16: "bf16", F32: "f32"}
EPS = 1e-6


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return torch.device("cuda:0")


def _gen(dev, seed):
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    return g


def _f64(x):
    return None if x is None else np.asarray(x.detach().double().cpu())


def _inputs(dev, t, hq, hk, d, dtype, seed=1):
    g = _gen(dev, seed)
    q, dq = (torch.randn(t, hq, d, generator=g, device=dev).to(dtype) for _ in range(2))
    k, dk = (torch.randn(t, hk, d, generator=g, device=dev).to(dtype) for _ in range(2))
    wq, wk = (1.0 + 0.3 * torch.randn(d, generator=g, device=dev) for _ in range(2))
    return q, k, dq, dk, wq, wk


def _check(q, k, dq, dk, positions, rotary, norm, wq, wk, eps=EPS, axes=None, freqs=()):
    """Both calls against the references; returns what they made."""
    args = {"norm": norm, "q_weight": wq, "k_weight": wk, "eps": eps}
    out = T.qk_norm_rope_forward(q, k, positions, rotary, **args)
    grads = T.qk_norm_rope_backward(dq, dk, q, k, positions, rotary, **args)
    pos = None if positions is None else positions.cpu().numpy().reshape(-1, q.shape[0])
    for i, (n, x, g, w) in enumerate((("q", q, dq, wq), ("k", k, dk, wk))):
        want = R.reference(_f64(x), _f64(w), pos, freqs, axes, rotary is not None and rotary.adjacent, norm, eps,
                           KIND[q.dtype], _f64(g))
        assert out[i].dtype == grads[i].dtype == q.dtype
        R.assert_close(n, out[i], want["y"])
        R.assert_close("d" + n, grads[i], want["dx"])
        if w is None:
            assert grads[2 + i] is None
        else:
            assert grads[2 + i].dtype == F32
            R.assert_close("dw" + n, grads[2 + i], want["dw"])
    return out + grads


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("adjacent", [False, True])
@pytest.mark.parametrize("t,hq,hk,d,pairs", [
    (1, 1, 1, 64, 32), (7, 12, 12, 64, 32), (33, 16, 8, 128, 64), (5, 3, 2, 80, 40), (9, 6, 2, 96, 48), (4, 5, 1, 51, 25),
    (3, 1, 1, 1, 0), (3, 2, 1, 2, 1), (6, 2, 3, 7, 2), (5, 4, 4, 256, 128), (2, 3, 1, 255, 127), (8, 2, 2, 64, 16),
    (8, 2, 2, 64, 0), (8, 2, 2, 64, 5), (5, 2, 1, 128, 8), (5, 1, 2, 24, 8), (5, 1, 1, 8, 4), (70, 1, 1, 130, 65),
    (3, 40, 33, 72, 36),
])
@pytest.mark.parametrize("norm", [True, False])
def test_matches_reference(dev, dtype, t, hq, hk, d, pairs, adjacent, norm):
    print(f"rope {dtype} {t} {hq}/{hk}x{d} pairs {pairs} {adjacent} {norm}", flush=True)
    q, k, dq, dk, wq, wk = _inputs(dev, t, hq, hk, d, dtype)
    freqs = T.Rotary.geometric(2 * pairs)
    pos = torch.randint(0, 5000, (t,), generator=_gen(dev, 2), device=dev, dtype=torch.int32)
    rotary = T.Rotary(freqs, adjacent=adjacent, device=dev)
    _check(q, k, dq, dk, pos, rotary, norm, wq if norm else None, wk if norm else None, freqs=freqs)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("t", [300, 5000])
@pytest.mark.parametrize("d,pairs", [(64, 32), (128, 64), (80, 40), (51, 20)])
def test_larger_batches(dev, dtype, t, d, pairs):
    q, k, dq, dk, wq, wk = _inputs(dev, t, 6, 2, d, dtype, seed=5)
    freqs = T.Rotary.geometric(2 * pairs, 1e6)
    pos = torch.arange(t, device=dev, dtype=torch.int64)
    _check(q, k, dq, dk, pos, T.Rotary(freqs, device=dev), True, wq, wk, freqs=freqs)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("norm", [True, False])
def test_axes(dev, dtype, norm):
    t, d = 60, 128
    q, k, dq, dk, wq, wk = _inputs(dev, t, 4, 2, d, dtype)
    freqs = T.Rotary.geometric(d)
    at = torch.arange(t)
    for axes in ([0] * 16 + [1] * 24 + [2] * 24, [i % 3 for i in range(64)], [2] * 64, [0, 1] * 32, [0] * 64):
        n = max(axes) + 1
        pos = torch.stack([at // 20, at // 5 % 4, at % 5])[:n].to(torch.int32).to(dev)
        for adjacent in (False, True):
            rotary = T.Rotary(freqs, axes, adjacent, dev)
            assert rotary.num_axes == n
            first = _check(q, k, dq, dk, pos, rotary, norm, wq if norm else None, wk if norm else None, axes=axes, freqs=freqs)
            # The same positions in 64 bits, and with other strides.
            wide = torch.empty(t, n, device=dev, dtype=torch.int64).t().copy_(pos)
            again = T.qk_norm_rope_forward(q, k, wide, rotary, norm=norm, q_weight=wq if norm else None,
                                           k_weight=wk if norm else None)
            assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_far_and_negative_positions(dev, dtype):
    q, k, dq, dk, wq, wk = _inputs(dev, 8, 2, 1, 64, dtype)
    freqs = T.Rotary.geometric(64)
    rotary = T.Rotary(freqs, device=dev)
    pos = [0, -1, -12345, 1 << 20, (1 << 31) - 1, -(1 << 31), 123456789, 3]
    _check(q, k, dq, dk, torch.tensor(pos, device=dev, dtype=torch.int32), rotary, True, wq, wk, freqs=freqs)
    pos[3:5] = [1 << 40, (1 << 50) + 3]
    _check(q, k, dq, dk, torch.tensor(pos, device=dev), rotary, True, wq, wk, freqs=freqs)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_norm_alone_and_weights(dev, dtype):
    q, k, dq, dk, wq, wk = _inputs(dev, 50, 3, 2, 96, dtype)
    _check(q, k, dq, dk, None, None, True, wq, wk)
    _check(q, k, dq, dk, None, None, True, None, None)
    _check(q, k, dq, dk, None, None, True, wq, None)
    _check(q, k, dq, dk, None, None, True, None, wk)
    _check(q, k, dq, dk, None, None, True, wq.bfloat16(), wk.bfloat16())
    _check(q, k, dq, dk, None, None, False, None, None)
    _check(q, k, dq, dk, None, None, True, wq, wk, eps=0.0)
    _check(q, k, dq, dk, None, None, True, wq, wk, eps=0.5)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("scale,eps", [(1e-30, 0.0), (1e-20, 1e-6), (1e18, 1e-6), (1e30, 1e-6)])
def test_norm_of_very_small_and_large_rows(dev, dtype, scale, eps):
    q, k, dq, dk, wq, wk = _inputs(dev, 20, 3, 2, 64, F32)
    q, k, dq, dk = ((s * x).to(dtype) for s, x in ((scale, q), (scale, k), (1.0, dq), (1.0, dk)))
    freqs = T.Rotary.geometric(64)
    pos = torch.arange(20, device=dev, dtype=torch.int32)
    _check(q, k, dq, dk, pos, T.Rotary(freqs, device=dev), True, wq, wk, eps=eps, freqs=freqs)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("layout", ["fused", "heads_first", "offset", "wide", "repeated"])
def test_strides(dev, dtype, layout):
    t, hq, hk, d = 37, 4, 2, 64
    q, k, dq, dk, wq, wk = _inputs(dev, t, hq, hk, d, dtype)
    freqs = T.Rotary.geometric(d)
    rotary, pos = T.Rotary(freqs, device=dev), torch.arange(t, device=dev, dtype=torch.int32)
    args = {"q_weight": wq, "k_weight": wk}
    want = T.qk_norm_rope_forward(q, k, pos, rotary, **args) + T.qk_norm_rope_backward(dq, dk, q, k, pos, rotary, **args)

    def other(x):
        if layout == "fused":
            buf = torch.full((t, x.shape[1] + 3, d), 9.0, device=dev, dtype=dtype)
            buf[:, 1:-2] = x
            return buf[:, 1:-2]
        if layout == "heads_first":
            return x.transpose(0, 1).contiguous().transpose(0, 1)
        if layout == "offset":                       # rows that start on any element
            buf = torch.full((t * x.shape[1] * (d + 3) + 1,), 9.0, device=dev, dtype=dtype)
            v = buf[1:].view(t, x.shape[1], d + 3)[..., :d]
            return v.copy_(x)
        if layout == "wide":                         # features apart: copied by the front end
            buf = torch.zeros(t, x.shape[1], 2 * d, device=dev, dtype=dtype)
            buf[..., ::2] = x
            return buf[..., ::2]
        return x
    if layout == "repeated":                         # one head for all
        q1, k1 = q[:, :1].expand(t, hq, d), k[:1].expand(t, hk, d)
        got = T.qk_norm_rope_forward(q1, k1, pos, rotary, **args)
        full = T.qk_norm_rope_forward(q1.contiguous(), k1.contiguous(), pos, rotary, **args)
        assert all(torch.equal(a, b) for a, b in zip(got, full))
        return
    x = [other(y) for y in (q, k, dq, dk)]
    got = T.qk_norm_rope_forward(x[0], x[1], pos, rotary, **args) + \
        T.qk_norm_rope_backward(x[2], x[3], x[0], x[1], pos, rotary, **args)
    assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d,pairs", [(64, 16), (51, 11)])
def test_nonfinite_stays_in_its_row(dev, dtype, d, pairs):
    t, h = 9, 3
    q, k, dq, dk, wq, wk = _inputs(dev, t, h, h, d, dtype)
    freqs = T.Rotary.geometric(2 * pairs)
    rotary, pos = T.Rotary(freqs, device=dev), torch.arange(t, device=dev, dtype=torch.int32)
    for value in (float("nan"), float("inf"), float("-inf")):
        for f in (0, pairs, 2 * pairs, d - 1):
            bad = q.clone()
            bad[4, 1, f] = value
            # Norm: every feature of the row is 0 or not finite; none of another row changes.
            clean = T.qk_norm_rope_forward(q, k, pos, rotary, q_weight=wq, k_weight=wk)
            out = T.qk_norm_rope_forward(bad, k, pos, rotary, q_weight=wq, k_weight=wk)
            rest = torch.ones(t, h, dtype=torch.bool, device=dev)
            rest[4, 1] = False
            assert torch.equal(out[0][rest], clean[0][rest]) and torch.equal(out[1], clean[1])
            row = out[0][4, 1]
            assert not torch.isfinite(row).all() and ((row == 0) | ~torch.isfinite(row)).all()
            # Rotation alone: the pair, or the feature that does not turn, and no other.
            out = T.qk_norm_rope_forward(bad, k, pos, rotary, norm=False)
            clean = T.qk_norm_rope_forward(q, k, pos, rotary, norm=False)
            touched = {f} if f >= 2 * pairs else {f % pairs, f % pairs + pairs}
            same = torch.ones(t, h, d, dtype=torch.bool, device=dev)
            same[4, 1, list(touched)] = False
            assert torch.equal(out[0][same], clean[0][same]) and not torch.isfinite(out[0][4, 1, f])
            # Backward, the gradient of one place.
            g = dq.clone()
            g[4, 1, f] = value
            grads = T.qk_norm_rope_backward(g, dk, q, k, pos, rotary, q_weight=wq, k_weight=wk)
            clean = T.qk_norm_rope_backward(dq, dk, q, k, pos, rotary, q_weight=wq, k_weight=wk)
            assert torch.equal(grads[0][rest], clean[0][rest]) and torch.equal(grads[1], clean[1])
            assert torch.equal(grads[3], clean[3]) and not torch.isfinite(grads[0][4, 1]).any()
            same = torch.ones(d, dtype=torch.bool, device=dev)
            same[list(touched)] = False
            assert torch.equal(grads[2][same], clean[2][same]) and not torch.isfinite(grads[2][f])


def test_rows_of_zeros(dev):
    q = torch.zeros(3, 2, 64, device=dev)
    out = T.qk_norm_rope_forward(q, q, None, None)
    assert not out[0].any()
    out = T.qk_norm_rope_forward(q, q, None, None, eps=0.0)
    assert torch.isnan(out[0]).all()                 # 0 / 0


def test_no_tokens(dev):
    q, w = torch.zeros(0, 2, 64, device=dev), torch.ones(64, device=dev)
    rotary, pos = T.Rotary(T.Rotary.geometric(64), device=dev), torch.zeros(0, dtype=torch.int32, device=dev)
    assert T.qk_norm_rope_forward(q, q, pos, rotary)[0].shape == (0, 2, 64)
    grads = T.qk_norm_rope_backward(q, q, q, q, pos, rotary, q_weight=w, k_weight=w)
    assert grads[0].shape == (0, 2, 64) and not grads[2].any() and not grads[3].any()


def test_is_inverse_and_reproducible(dev):
    # Turned there and back: the rotation's transpose, by the backward pass.
    q, k, *_ = _inputs(dev, 1000, 4, 2, 128, F32)
    rotary, pos = T.Rotary(T.Rotary.geometric(128), device=dev), torch.arange(1000, device=dev, dtype=torch.int32)
    a = T.qk_norm_rope_forward(q, k, pos, rotary, norm=False)
    b = T.qk_norm_rope_backward(a[0], a[1], q, k, pos, rotary, norm=False)
    assert (b[0] - q).abs().max() < 20 * R.U * q.abs().max() * 2
    w = torch.rand(128, device=dev)
    runs = [T.qk_norm_rope_backward(q, k, q, k, pos, rotary, q_weight=w, k_weight=w) for _ in range(3)]
    assert all(torch.equal(x, y) for r in runs[1:] for x, y in zip(runs[0], r))


@pytest.mark.parametrize("adjacent", [False, True])
def test_gradient_against_differences(dev, adjacent):
    """(f(x + h v) - f(x - h v)) / 2h in fp32: h^2 f''' / 6 and u |f| / h are both near 1e-5 of f's size."""
    t, hq, hk, d = 6, 2, 1, 10
    g = _gen(dev, 4)
    freqs, axes = T.Rotary.geometric(8), [0, 1, 1, 0]
    rotary = T.Rotary(freqs, axes, adjacent, dev)
    pos = torch.randint(0, 50, (2, t), generator=g, device=dev)
    x = [torch.randn(*s, generator=g, device=dev, requires_grad=True) for s in ((t, hq, d), (t, hk, d), (d,), (d,))]
    c = [torch.randn(*s, generator=g, device=dev) for s in ((t, hq, d), (t, hk, d))]

    def f(v):
        q, k = T.qk_norm_rope(v[0], v[1], pos, rotary, q_weight=v[2], k_weight=v[3])
        return (q.double() * c[0]).sum() + (k.double() * c[1]).sum()
    f(x).backward()
    h = 1e-2
    for i in range(4):
        v = torch.randn(*x[i].shape, generator=g, device=dev)
        with torch.no_grad():
            up, down = ([x[j] + s * h * v if j == i else x[j] for j in range(4)] for s in (1, -1))
            diff = float((f(up) - f(down)) / (2 * h))
        got = float((x[i].grad.double() * v).sum())
        size = float((x[i].grad.double() * v).abs().sum())
        print(f"{i}: {got:.6f} {diff:.6f} of {size:.3f}")
        assert abs(got - diff) <= 2e-3 * size


def test_autograd_matches_calls(dev):
    q, k, dq, dk, wq, wk = _inputs(dev, 40, 4, 2, 64, BF16)
    rotary, pos = T.Rotary(T.Rotary.geometric(64), device=dev), torch.arange(40, device=dev)
    leaves = [x.clone().requires_grad_() for x in (q, k, wq, wk.bfloat16())]
    out = T.qk_norm_rope(leaves[0], leaves[1], pos, rotary, q_weight=leaves[2], k_weight=leaves[3].float())
    torch.autograd.backward(out, (dq, dk))
    want = T.qk_norm_rope_backward(dq, dk, q, k, pos, rotary, q_weight=wq, k_weight=wk.bfloat16().float())
    for x, y in zip(leaves, want):
        assert x.grad.dtype == x.dtype and torch.equal(x.grad, y.to(x.dtype))
    # Without norms: nothing of q and k is kept.
    x = [q.clone().requires_grad_(), k.clone().requires_grad_()]
    out = T.qk_norm_rope(x[0], x[1], pos, rotary, norm=False)
    assert all(t is None or t.dtype == torch.int64 for t in out[0].grad_fn.saved_tensors)
    torch.autograd.backward(out, (dq, dk))
    turned = T.qk_norm_rope_backward(dq, dk, q, k, pos, rotary, norm=False)
    assert torch.equal(x[0].grad, turned[0]) and torch.equal(x[1].grad, turned[1])
    # One output unused; frozen weights.
    x = q.clone().requires_grad_()
    T.qk_norm_rope(x, k, pos, rotary, q_weight=wq, k_weight=wk)[0].backward(dq)
    assert torch.equal(x.grad, want[0])


def test_offsets_past_32_bits(dev):
    # The last token's heads begin behind 2^32 elements of a view.
    t, d = 5, 64
    buf = torch.zeros((1 << 30) * 4 + 4096, device=dev, dtype=BF16)
    q = buf.as_strided((t, 2, d), (1 << 30, 64, 1))
    g = _gen(dev, 3)
    q.copy_(torch.randn(t, 2, d, generator=g, device=dev))
    rotary, pos = T.Rotary(T.Rotary.geometric(d), device=dev), torch.arange(t, device=dev)
    got = T.qk_norm_rope_forward(q, q, pos, rotary)
    want = T.qk_norm_rope_forward(q.contiguous(), q.contiguous(), pos, rotary)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_side_stream_and_graph(dev):
    q, k, dq, dk, wq, wk = _inputs(dev, 700, 4, 2, 128, BF16)
    rotary, pos = T.Rotary(T.Rotary.geometric(128), device=dev), torch.arange(700, device=dev)
    args = {"q_weight": wq, "k_weight": wk}

    def both():
        return T.qk_norm_rope_forward(q, k, pos, rotary, **args) + T.qk_norm_rope_backward(dq, dk, q, k, pos, rotary, **args)
    want = both()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = both()
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = both()
    for i in range(3):
        q.neg_()
        pos.add_(i)
        want = both()
        for x in got:
            x.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_refusals(dev):
    q, k, dq, dk, wq, wk = _inputs(dev, 10, 4, 2, 64, BF16)
    rotary, pos = T.Rotary(T.Rotary.geometric(64), device=dev), torch.arange(10, device=dev)
    two = T.Rotary([1.0, 0.5], [0, 1], device=dev)
    call = T.qk_norm_rope_forward
    for bad in (lambda: call(q, k[:5], pos, rotary), lambda: call(q, k[..., :32], pos, rotary),
                lambda: call(q, k.float(), pos, rotary), lambda: call(q, k.cpu(), pos, rotary), lambda: call(q[0], k, pos, rotary),
                lambda: call(q, k, pos[:5], rotary), lambda: call(q, k, pos.float(), rotary), lambda: call(q, k, pos.cpu(), rotary),
                lambda: call(q, k, None, rotary), lambda: call(q, k, pos, two), lambda: call(q, k, pos.expand(3, 10), two),
                lambda: call(q, k, pos, rotary, q_weight=wq[:32]), lambda: call(q, k, pos, rotary, q_weight=wq.cpu()),
                lambda: call(q, k, pos, rotary, q_weight=wq, k_weight=wk.bfloat16()),
                lambda: call(q, k, pos, rotary, norm=False, q_weight=wq), lambda: call(q, k, pos, rotary, q_weight=wq.expand(2, 64)),
                lambda: call(q, k, pos, T.Rotary([1.0], device="cpu")),
                lambda: T.qk_norm_rope_backward(dq[:5], dk, q, k, pos, rotary),
                lambda: T.qk_norm_rope_backward(dq.float(), dk, q, k, pos, rotary)):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(TypeError):
        call(q.half(), k.half(), pos, rotary)
    with pytest.raises(TypeError):
        call(q, k, pos, rotary, q_weight=wq.double())
    for bad in (lambda: call(q[..., :62], k[..., :62], pos, rotary), lambda: call(q, k, pos, rotary, eps=-1.0),
                lambda: call(q, k, pos, rotary, eps=float("nan")), lambda: call(q[:, :0], k, pos, rotary),
                lambda: call(q.repeat(1, 1, 5), k.repeat(1, 1, 5), pos, rotary)):
        with pytest.raises(RuntimeError):
            bad()
