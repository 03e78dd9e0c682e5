"""The gradient norm and clipping on the GPU against sums in 64 bits.

Bounds: the kernels sum squares in 64 bits and round the norm to fp32 once, so it is off by
half a step (2^-24 of it; 2^-40 more covers the order of up to 2^28 sums of 2^-53 steps); the
factor is held in 64 bits, and its product rounded once to fp32 (2^-24), for bf16 once more
(2^-8); below the normal numbers half a step of the type is absolute."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2609_36692_amd import train_ops as T  # noqa: E402

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return torch.device("cuda:0")


def _make(dev, sizes, dtypes, seed=1, scale=1.0):
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    return [(scale * torch.randn(n, generator=g, device=dev)).to(dtypes[i % len(dtypes)]) for i, n in enumerate(sizes)]


def _f64(x):
    return np.asarray(x.detach().double().cpu())


def _norm(grads):
    return math.sqrt(math.fsum(float((_f64(g) ** 2).sum()) for g in grads))


def _check_norm(got, want):
    assert got.dtype == F32 and got.dim() == 0
    if want >= 2.0 ** 128:                           # past fp32's range: rounds to infinity
        assert float(got) == math.inf
        return
    assert abs(float(got) - want) <= (2.0 ** -24 + 2.0 ** -40) * want + 2.0 ** -150, (float(got), want)


def _check_scaled(got, grad, c):
    want = _f64(grad) * c
    tol = np.abs(want) * (2.0 ** -24 + 2.0 ** -40 + (2.0 ** -8 * (1 + 2.0 ** -20) if got.dtype == BF16 else 0.0)) \
        + (2.0 ** -133 if got.dtype == BF16 else 2.0 ** -149)
    off = np.abs(_f64(got) - want) - tol
    assert got.shape == grad.shape and (off <= 0).all(), off.max()


def _factor(norm, limit):
    return 1.0 if norm <= limit else limit / norm


SIZES = {
    "one": [(1,)],
    "odd": [(1,), (77,), (333, 65), (129,), (1000, 3), (2049,)],
    "borders": [(8191,), (8192,), (8193,), (16384,), (7,), (255, 257)],
    "many": [(n % 37 + 1,) for n in range(1000)],
    "lists": [(100,)] * 152 + [(9000,)] * 153,
    "empty": [(0,), (5,), (0, 3), (), (4,)],
    "large": [(3000, 2111), (5,), (4096, 4096)],
}


@pytest.mark.parametrize("types", [[F32], [BF16], [F32, BF16]], ids=["f32", "bf16", "mixed"])
@pytest.mark.parametrize("which", SIZES)
def test_norm_and_clip(dev, which, types):
    print(f"grads {which} {types}", flush=True)
    grads = _make(dev, SIZES[which], types)
    want = _norm(grads)
    _check_norm(T.grad_norm(grads), want)
    for limit in (0.3 * want, 2.0 * want):
        c = _factor(want, limit)
        before = [g.clone() for g in grads]
        # Into tensors of either type.
        for kind in (F32, BF16):
            out = [torch.full_like(g, 7.0, dtype=kind) for g in grads]
            _check_norm(T.clip_grads(grads, limit, out=out), want)
            for g, o, b in zip(grads, out, before):
                assert torch.equal(g, b)
                _check_scaled(o, g, c)
        # In place.
        mine = [g.clone() for g in grads]
        _check_norm(T.clip_grads(mine, limit), want)
        for g, m in zip(grads, mine):
            _check_scaled(m, g, c)
            assert c != 1.0 or torch.equal(m, g)


def test_limits(dev):
    grads = _make(dev, [(3, 5)], [F32])
    want = _norm(grads)
    for limit, c in ((math.inf, 1.0), (0.0, 0.0), (1e-300, 1e-300 / want)):
        mine = [grads[0].clone()]
        T.clip_grads(mine, limit)
        _check_scaled(mine[0], grads[0], c)
    zero = [torch.zeros(9, device=dev)]
    for limit in (0.0, 1.0):
        assert float(T.clip_grads(zero, limit)) == 0.0 and not zero[0].any()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("scale", [1e-38, 1e-30, 1e25, 1e37])
def test_squares_past_the_range_of_fp32(dev, dtype, scale):
    grads = _make(dev, [(5000,), (33, 7)], [dtype], scale=scale)
    want = _norm(grads)
    limit = want / 3
    out = [torch.empty_like(g) for g in grads]
    _check_norm(T.clip_grads(grads, limit, out=out), want)
    for g, o in zip(grads, out):
        _check_scaled(o, g, limit / want)


def test_norm_past_the_range_of_fp32(dev):
    grads = [torch.full((10000,), 3e38, device=dev)]
    norm = T.clip_grads(grads, 1.0)
    assert float(norm) == math.inf
    assert np.allclose(_f64(grads[0]), 0.01, rtol=2.0 ** -23)


def test_nonfinite(dev):
    for where in (0, 1):
        grads = _make(dev, [(100,), (9000,)], [F32, BF16])
        grads[where][7] = math.nan
        assert math.isnan(float(T.grad_norm(grads)))
        assert math.isnan(float(T.clip_grads(grads, 1.0)))
        assert all(torch.isnan(g).all() for g in grads)
        grads = _make(dev, [(100,), (9000,)], [F32, BF16])
        grads[where][7] = -math.inf
        assert float(T.clip_grads(grads, 1.0)) == math.inf
        for i, g in enumerate(grads):
            bad = torch.isnan(g)
            assert bad.sum() == (i == where) and not torch.where(bad, 0.0, g).any()
    # No limit: as they are.
    grads = [torch.tensor([1.0, math.inf], device=dev)]
    assert float(T.clip_grads(grads, math.inf)) == math.inf and grads[0].tolist() == [1.0, math.inf]


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_strides_and_alignment(dev, dtype):
    buf = _make(dev, [(40000,)], [dtype], seed=3)[0]
    inside = buf.clone()
    grads = [inside[1:8195], inside[8195:8196], inside[9001:17193].view(64, 128).t(), inside[20000:20600].view(20, 30)[:, ::2],
             inside[30000:30060].view(3, 4, 5).permute(2, 0, 1)]
    want = _norm(grads)
    _check_norm(T.grad_norm(grads), want)
    before = [g.clone() for g in grads]
    norm = T.clip_grads(grads, 0.5)
    _check_norm(norm, want)
    for g, b in zip(grads, before):
        _check_scaled(g, b, _factor(want, 0.5))
    # Nothing else has been written.
    touched = torch.zeros_like(buf, dtype=torch.bool)
    for g in (touched[1:8196], touched[9001:17193], touched[20000:20600].view(20, 30)[:, ::2], touched[30000:30060]):
        g.fill_(True)
    assert torch.equal(inside[~touched], buf[~touched])
    # Gradients and outputs of different strides.
    g = _make(dev, [(50, 70)], [dtype])[0]
    for out in (torch.empty(70, 50, device=dev, dtype=dtype).t(), torch.empty(50, 140, device=dev, dtype=dtype)[:, ::2],
                torch.empty(50 * 70 + 1, device=dev, dtype=F32)[1:].view(50, 70)):
        for x in (g, g.t().contiguous().t()):
            T.clip_grads([x], 1.0, out=[out])
            _check_scaled(out, g, 1.0 / _norm([g]))


def test_one_tensor_and_iterators(dev):
    g = _make(dev, [(50,)], [F32])[0]
    _check_norm(T.grad_norm(g), _norm([g]))
    _check_norm(T.grad_norm(x for x in (g, g)), _norm([g, g]))
    mine = g.clone()
    _check_norm(T.clip_grads(mine, 1.0), _norm([g]))
    _check_scaled(mine, g, 1.0 / _norm([g]))


def test_refusals(dev):
    g = torch.ones(100, device=dev)
    with pytest.raises(RuntimeError, match="overlap"):
        T.clip_grads([g, g], 1.0)
    with pytest.raises(RuntimeError, match="overlap"):
        T.clip_grads([g[:60], g[40:]], 1.0)
    with pytest.raises(RuntimeError, match="overlap"):
        T.clip_grads([g[:60].bfloat16(), g[60:]], 1.0, out=[g[40:], torch.empty(40, device=dev)])
    with pytest.raises(TypeError):
        T.clip_grads([g.half()], 1.0)
    with pytest.raises(TypeError):
        T.clip_grads([g], 1.0, out=[g.double()])
    with pytest.raises(ValueError):
        T.clip_grads([g, torch.ones(3)], 1.0)
    assert (g == 1).all()


def test_is_reproducible_on_side_streams_and_in_a_graph(dev):
    grads = _make(dev, [(3000, 2111), (5,), (129, 7)], [F32, BF16])
    out = [torch.empty_like(g, dtype=F32) for g in grads]
    norm = T.clip_grads(grads, 1.0, out=out)
    first = [norm.clone()] + [o.clone() for o in out]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for o in out:
            o.zero_()
        again = [T.clip_grads(grads, 1.0, out=out)] + out
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(first, again))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        norm = T.clip_grads(grads, 1.0, out=out)
    for k in range(4):
        scale = 2.0 ** k                             # exact in either type: the norm scales, the result stays
        for g in grads:
            g.mul_(2.0 if k else 1.0)
        for o in out:
            o.fill_(3.0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(norm, first[0] * scale)
        assert all(torch.equal(a, b) for a, b in zip(first[1:], out))
        eager = T.grad_norm(grads)
        assert torch.equal(eager, norm)


def test_offsets_past_32_bits(dev):
    # 2^32 + 100 elements of one tensor: pieces of 2^29.
    n = (1 << 32) + 100
    g = torch.zeros(n, device=dev, dtype=BF16)
    at = [0, (1 << 29) - 1, 1 << 29, (1 << 31) + 5, (1 << 32) - 1, 1 << 32, n - 1]
    for i, p in enumerate(at):
        g[p] = float(i + 1)
    want = math.sqrt(sum((i + 1) ** 2 for i in range(len(at))))
    _check_norm(T.clip_grads(g, 2.0), want)
    got = torch.stack([g[p] for p in at])
    _check_scaled(got, torch.arange(1, len(at) + 1, device=dev, dtype=F32), 2.0 / want)
    assert int(torch.count_nonzero(g)) == len(at)


def test_optimizer_clips_before_its_step(dev):
    from paper_2609_36692_amd.optim import NormPreOptimizer
    torch.manual_seed(3)
    m = torch.nn.Sequential(torch.nn.Linear(96, 192), torch.nn.GELU(), torch.nn.Linear(192, 64)).to(dev)
    opt = NormPreOptimizer(m.parameters(), lr=1e-3, adamw_lr=1e-3, max_grad_norm=0.25)
    (100.0 * m(torch.randn(32, 96, device=dev)).square().mean()).backward()
    before = [p.grad.clone() for p in m.parameters()]
    want = _norm(before)
    assert want > 0.25
    opt.step()
    _check_norm(opt.grad_norm, want)
    for p, g in zip(m.parameters(), before):
        _check_scaled(p.grad, g, 0.25 / want)
        if p.dim() == 2:                             # M = mu 0 + G
            assert torch.equal(opt.state[p]["momentum"], p.grad)
    # Below the limit gradients stay as they are.
    opt.zero_grad()
    (1e-6 * m(torch.randn(32, 96, device=dev)).square().mean()).backward()
    before = [p.grad.clone() for p in m.parameters()]
    opt.step()
    assert float(opt.grad_norm) < 0.25
    assert all(torch.equal(p.grad, g) for p, g in zip(m.parameters(), before))
    opt.close()


def test_command_line_clips(dev, capsys):
    pytest.importorskip("transformers")
    import json
    from paper_2609_36692_amd import e2e_gpt2 as E
    E.main(["--batch", "1", "--seq", "128", "--steps", "1", "--warmup", "1", "--clip", "0.5"])
    out = json.loads(capsys.readouterr().out.strip().splitlines()[-1])
    assert out["grad_norm_last_step"] > 0.0
