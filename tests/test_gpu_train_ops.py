"""Training-step operators on the GPU against 64-bit references: packed
attention and its backward pass, 8-bit activation checkpoints and the gradients
that read them.  Bounds: tests/train_ops_util.py."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2609_36692_amd import normpre as N  # noqa: E402
from paper_2609_36692_amd import train_ops as T  # noqa: E402
from train_ops_util import (H, U, act_grad_reference, act_reference, assert_within, attention_reference,  # noqa: E402
                            decode_reference, encode_reference)

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return torch.device("cuda:0")


def _gen(dev, seed):
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    return g


def _qkv(dev, seed, t, hq, hk, d, dtype):
    g = _gen(dev, seed)
    return [torch.randn(t, h, d, generator=g, device=dev).to(dtype) for h in (hq, hk, hk, hq)]


def _check(q, k, v, dout, lens, causal, scale=None):
    c = 1.0 / math.sqrt(q.shape[2]) if scale is None else scale
    plan = T.AttentionPlan(lens, causal, q.device)
    out, lse = T.attention_forward(q, k, v, plan, scale)
    dq, dk, dv = T.attention_backward(dout, q, k, v, out, lse, plan, scale)
    want, tol = attention_reference(q, k, v, lens, causal, c, dout)
    r = 1 if q.dtype == BF16 else 0
    for name, got in (("out", out), ("lse", lse), ("dq", dq), ("dk", dk), ("dv", dv)):
        assert got.dtype == (F32 if name == "lse" else q.dtype)
        assert_within(name, got, want[name], tol[name][r])
    return out, lse, dq, dk, dv


# ------------------------------------------------------------- attention ---
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("lens,hq,hk,d,causal", [
    ([1], 1, 1, 64, True),
    ([1, 2, 3, 31, 32, 33], 2, 1, 64, True),
    ([63, 64, 65, 0, 1], 3, 3, 64, True),
    ([127, 128, 129], 4, 2, 128, True),
    ([257], 2, 1, 128, True),
    ([100, 130], 2, 2, 128, False),
    ([5, 300], 1, 1, 64, False),
    ([40, 70], 8, 2, 40, True),
    ([150], 3, 1, 7, True),
    ([33, 66], 2, 1, 96, True),
    ([50], 5, 1, 1, True),
    ([90], 2, 2, 127, False),
])
def test_attention_matches_reference(dev, dtype, lens, hq, hk, d, causal):
    print(f"attention {dtype} {lens} {hq}/{hk}x{d} causal={causal}", flush=True)
    q, k, v, dout = _qkv(dev, 1 + sum(lens), sum(lens), hq, hk, d, dtype)
    _check(q, k, v, dout, lens, causal)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("crowd", [0, 250, 400, 600, 1100])
@pytest.mark.parametrize("nonfinite", [False, True])
def test_attention_in_a_crowd(dev, dtype, d, crowd, nonfinite):
    # How blocks share their work goes by the size of the batch: the same long
    # sequences alone and among ever more one-token ones.
    lens = [1] * (crowd // 2) + [300, 129] + [1] * (crowd - crowd // 2)
    q, k, v, dout = _qkv(dev, 25, sum(lens), 1, 1, d, dtype)
    if nonfinite:
        at = crowd // 2 + 200
        v[at, 0, 5] = float("inf")
        k[at + 20, 0, 2] = float("nan")
        dout[at + 40, 0, 1] = float("-inf")
    _check(q, k, v, dout, lens, True)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("scale", [0.0, -0.3, 2.0])
def test_attention_scales(dev, dtype, scale):
    q, k, v, dout = _qkv(dev, 5, 97, 2, 1, 64, dtype)
    _check(q, k, v, dout, [60, 37], True, scale)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("layout", ["fused", "head_major", "odd_stride", "misaligned", "expanded", "feature_major"])
def test_attention_strides(dev, dtype, layout):
    lens, hq, hk, d = [70, 1, 60], 4, 2, 64
    t = sum(lens)
    q, k, v, dout = _qkv(dev, 11, t, hq, hk, d, dtype)
    if layout == "fused":
        buf = torch.cat([x.flatten(1) for x in (q, k, v)], 1)
        q, k, v = (x.unflatten(1, (-1, d)) for x in buf.split([hq * d, hk * d, hk * d], 1))
    elif layout == "head_major":
        q, k, v, dout = (x.transpose(0, 1).contiguous().transpose(0, 1) for x in (q, k, v, dout))
    elif layout == "odd_stride":
        q, k, v, dout = (torch.nn.functional.pad(x, (0, 3))[:, :, :d] for x in (q, k, v, dout))
    elif layout == "misaligned":
        q, k, v, dout = (torch.nn.functional.pad(x.flatten(), (1, 0))[1:].view(x.shape) for x in (q, k, v, dout))
    elif layout == "expanded":
        k, v = (x[:, :1].expand(t, hk, d) for x in (k, v))
    else:
        q, k, v, dout = (x.transpose(1, 2).contiguous().transpose(1, 2) for x in (q, k, v, dout))
    _check(q, k, v, dout, lens, True)


def test_attention_extreme_scores(dev):
    # Scores of hundreds: a row's weights fall on one or two keys.
    q, k, v, dout = _qkv(dev, 21, 140, 2, 2, 64, F32)
    _check(8 * q, 8 * k, v, dout, [140], True)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_attention_with_one_dominating_score(dev, dtype):
    # Small whole numbers, so every score is exact; each row has nearly all weight on
    # one key, and the gradients of its scores almost vanish.  The bounds allow for
    # the rounding of out in delta; where delta is summed from the scores (blocks
    # of up to 128 keys) dq must do without: an error of 2 H (its operand's and its own
    # rounding; the terms of a row's sum are few) of the norm.  fp32: what a weight
    # lacks to 1 is 5e-3 or more, so u of out is at most some 1e-4 of the norm.
    n, d = 600, 64
    g = _gen(dev, 28)
    k = torch.randint(-1, 2, (n, 1, d), generator=g, device=dev).to(dtype)
    at = (torch.rand(n, generator=g, device=dev) * (torch.arange(n, device=dev) + 1)).long()
    v, dout = (torch.randn(n, 1, d, generator=g, device=dev).to(dtype) for _ in range(2))
    dq = _check(2 * k[at], k, v, dout, [n], True)[2]
    want = attention_reference(2 * k[at], k, v, [n], True, 1 / math.sqrt(d), dout)[0]["dq"]
    end = 128 if dtype == BF16 else n
    off = np.linalg.norm(dq.double().cpu().numpy()[:end] - want[:end]) / np.linalg.norm(want[:end])
    assert off <= (2 * H if dtype == BF16 else 1e-3)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("fq,fk,fv,fdout", [(2.0 ** 50, 2.0 ** -50, 2.0 ** -60, 2.0 ** 30),
                                            (2.0 ** -45, 2.0 ** 45, 2.0 ** 60, 2.0 ** -70)])
def test_attention_fp32_magnitudes(dev, d, fq, fk, fv, fdout):
    # All 24 digits of an operand count, whatever its size.
    q, k, v, dout = _qkv(dev, 23, 190, 2, 1, d, F32)
    _check(fq * q, fk * k, fv * v, fdout * dout, [150, 40], True)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d", [64, 128])
def test_attention_of_the_largest_values(dev, dtype, d):
    # A mean of values near the end of the range, of one sign or both, is in range.
    lens = [300, 40]
    q, k, v, _ = _qkv(dev, 26, sum(lens), 2, 1, d, dtype)
    v = (3e38 * torch.sign(v)).to(dtype)
    v[:300, :, 3] = 3e38
    out, _ = T.attention_forward(q, k, v, T.AttentionPlan(lens, True, dev))
    want, tol = attention_reference(q, k, v, lens, True, 1 / math.sqrt(d))
    assert_within("out", out, want["out"], tol["out"][1 if dtype == BF16 else 0])


def test_attention_fp32_products(dev):
    # One token a sequence, one feature: the log-sum-exp is the product q k.  The
    # split may leave out 8 u of it, the sum of the terms' products may cut off 2 u,
    # the exponent's rounding is taken back by the logarithm to 1 u, and their sum
    # rounds.  Among the operands some whose upper 16 bits fall short of them by
    # the most.
    n = 4096
    g = _gen(dev, 24)
    q, k = (torch.randn(n, 1, 1, generator=g, device=dev) for _ in range(2))
    q[:8] = k[:8] = torch.tensor(0x3f80ffff, dtype=torch.int32).view(F32).item()
    _, lse = T.attention_forward(q, k, k, T.AttentionPlan([1] * n, True, dev), 1.0)
    want = (q.double() * k.double()).flatten()
    assert ((lse[0].double() - want).abs() <= 12 * U * want.abs()).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_attention_long_rows(dev, dtype):
    # A sequence of many tiles.
    lens, hq, hk, d = [1500, 37], 2, 1, 64
    q, k, v, dout = _qkv(dev, 31, sum(lens), hq, hk, d, dtype)
    _check(q, k, v, dout, lens, True)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("value", [float("inf"), float("-inf"), float("nan")])
@pytest.mark.parametrize("where", ["q", "k", "v", "dout"])
def test_attention_nonfinite_stays_with_rows_that_see_it(dev, dtype, d, value, where):
    # In the middle of a diagonal tile of the second sequence, one head.
    lens, hq, hk = [50, 150, 40], 2, 1
    x = dict(zip(("q", "k", "v", "dout"), _qkv(dev, 41, sum(lens), hq, hk, d, dtype)))
    at = 50 + 77
    x[where][at, 0, 3] = value
    out, lse, dq, dk, dv = _check(**x, lens=lens, causal=True)
    # No row before it in its sequence and no other sequence is touched.
    others = torch.tensor([i for i in range(sum(lens)) if i < 50 or i >= 200], device=dev)
    before = torch.arange(50, at, device=dev)
    for y in (out, dq):
        assert torch.isfinite(y[others]).all() and torch.isfinite(y[before]).all()
    for y in (dk, dv):
        assert torch.isfinite(y[others]).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d", [40, 72, 96])
@pytest.mark.parametrize("value", [float("inf"), float("-inf"), float("nan")])
@pytest.mark.parametrize("where", ["q", "k", "v", "dout"])
@pytest.mark.parametrize("sign", [1, -1])
def test_attention_nonfinite_in_the_last_features(dev, dtype, d, value, where, sign):
    # Heads that fill their tiles in part.  An infinite key makes the scores of all
    # queries, of one sign there, +inf or -inf: a weight of zero in the second case.
    lens, hq, hk = [50, 150, 40], 2, 1
    x = dict(zip(("q", "k", "v", "dout"), _qkv(dev, 43, sum(lens), hq, hk, d, dtype)))
    x[where][50 + 77, 0, d - 1] = value
    if where == "k":
        x["q"][:, :, d - 1] = sign * x["q"][:, :, d - 1].abs().clamp(min=0.01)
    _check(**x, lens=lens, causal=True)


@pytest.mark.parametrize("dtype,hq,hk,d,crowd", [(BF16, 4, 2, 64, 0), (BF16, 2, 2, 128, 300), (F32, 2, 1, 64, 0),
                                                 (F32, 2, 1, 128, 600), (BF16, 2, 1, 96, 0)])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("where", ["q", "k", "v", "dout"])
@pytest.mark.parametrize("values", ["nan", "inf", "both", "all", "last", "first"])
def test_attention_nonfinite_in_long_sequences(dev, dtype, hq, hk, d, causal, crowd, where, values):
    # Rows far behind a value that is not finite, rows beside it, whole operands, the
    # ends of a sequence; batches whose keys' queries are shared out and not.
    lens = [203, 70] + [1] * crowd
    x = dict(zip(("q", "k", "v", "dout"), _qkv(dev, 45, sum(lens), hq, hk, d, dtype)))
    y, nan, inf = x[where], float("nan"), float("inf")
    if values == "all":
        y[:203] = nan
    elif values in ("last", "first"):
        y[202 if values == "last" else 0, 0, 1] = inf
        y[272 if values == "last" else 203, 0, d - 1] = nan
    else:
        if values != "inf":
            y[60, 0, 3] = nan
        if values != "nan":
            y[75, -1, 2], y[230, 0, 4] = inf, -inf
    _check(**x, lens=lens, causal=causal)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("where", ["one k", "all q", "all k", "all v", "all dout"])
def test_attention_nan_costs_no_second_pass(dev, dtype, where):
    # Results that are NaN by the formula are not computed again: 25 times the time
    # of finite operands is far above what the search for them takes, and far below
    # that of a second, scalar pass (100 to 500 times).
    n = 4096
    q, k, v, dout = _qkv(dev, 46, n, 4, 4, 64, dtype)
    plan = T.AttentionPlan([n], True, dev)

    def least():
        times = []
        for _ in range(5):
            ends = [torch.cuda.Event(enable_timing=True) for _ in range(3)]
            ends[0].record()
            out, lse = T.attention_forward(q, k, v, plan)
            ends[1].record()
            grads = T.attention_backward(dout, q, k, v, out, lse, plan)
            ends[2].record()
            ends[2].synchronize()
            times.append([a.elapsed_time(b) for a, b in zip(ends, ends[1:])])
        return [min(t) for t in zip(*times)], (out, *grads)

    finite, _ = least()
    count, name = where.split()
    x = {"q": q, "k": k, "v": v, "dout": dout}[name]
    x[n // 2 if count == "one" else slice(None)] = float("nan")
    got, (out, dq, dk, dv) = least()
    print(f"finite {finite} ms, {where} NaN {got} ms")
    assert got[0] <= 25 * finite[0] and got[1] <= 25 * finite[1]
    first = n // 2 if count == "one" else 0
    assert torch.isnan(dq[first:]).all() and torch.isnan(dk[first:]).all()
    assert torch.isnan(out[first:]).all() or name == "dout"


def test_attention_all_scores_minus_infinity(dev):
    # Formula of a row whose scores are all -inf: 0 / 0.
    q = torch.ones(4, 1, 64, device=dev)
    k = torch.full((4, 1, 64), float("-inf"), device=dev)
    v = torch.ones(4, 1, 64, device=dev)
    out, _ = T.attention_forward(q, k, v, T.AttentionPlan([4], True, dev))
    assert torch.isnan(out).all()


def test_attention_empty_batch(dev):
    for lens in ([], [0], [0, 0, 0]):
        plan = T.AttentionPlan(lens, True, dev)
        q = torch.empty(0, 4, 64, device=dev, dtype=BF16, requires_grad=True)
        k = torch.empty(0, 2, 64, device=dev, dtype=BF16, requires_grad=True)
        out = T.attention(q, k, k, plan)
        assert out.shape == q.shape
        out.sum().backward()
        assert q.grad.shape == q.shape


def test_attention_offsets_past_32_bits(dev):
    # Rows 24 MB apart: element offsets reach 2.5e9.
    lens, hq, hk, d, pitch = [130, 70], 2, 1, 64, 12_500_000
    t = sum(lens)
    q, k, v, dout = _qkv(dev, 51, t, hq, hk, d, BF16)
    want = _check(q, k, v, dout, lens, True)
    buf = torch.empty(t * pitch, dtype=BF16, device=dev)
    far, at = [], 0
    for x in (q, k, v, dout):
        y = buf.as_strided(x.shape, (pitch, d, 1), at)
        y.copy_(x)
        far.append(y)
        at += x.shape[1] * d
    plan = T.AttentionPlan(lens, True, dev)
    out, lse = T.attention_forward(*far[:3], plan)
    got = (out, lse, *T.attention_backward(far[3], *far[:3], out, lse, plan))
    for a, b in zip(got, want):
        assert torch.equal(a, b)


def test_attention_is_reproducible(dev):
    lens = [300, 17, 211]
    q, k, v, dout = _qkv(dev, 61, sum(lens), 8, 2, 128, BF16)
    plan = T.AttentionPlan(lens, True, dev)
    runs = []
    for _ in range(3):
        out, lse = T.attention_forward(q, k, v, plan)
        runs.append((out, lse, *T.attention_backward(dout, q, k, v, out, lse, plan)))
    for r in runs[1:]:
        assert all(torch.equal(a, b) for a, b in zip(r, runs[0]))


def test_attention_of_a_packed_batch_equals_its_sequences(dev):
    lens = [40, 129, 7]
    q, k, v, _ = _qkv(dev, 71, sum(lens), 4, 4, 64, BF16)
    out, lse = T.attention_forward(q, k, v, T.AttentionPlan(lens, True, dev))
    at = 0
    for n in lens:
        s = slice(at, at + n)
        o, l = T.attention_forward(q[s], k[s], v[s], T.AttentionPlan([n], True, dev))
        assert torch.equal(o, out[s]) and torch.equal(l, lse[:, s])
        at += n


def test_attention_gradient_against_differences(dev):
    # d/dt of sum(w * out) along random directions, by central differences of the
    # fp32 forward kernel (the loss summed in fp64).  Step 2^-7: the third
    # derivative's term is below step^2 * |direction|^3-ish = 1e-3 of the slope
    # here, the rounding of the outputs (1e-6 of them) over the step 2e-4.
    lens = [37, 70]
    q, k, v, w = _qkv(dev, 81, sum(lens), 4, 2, 64, F32)
    plan = T.AttentionPlan(lens, True, dev)
    xs = [x.requires_grad_() for x in (q, k, v)]
    (w * T.attention(*xs, plan)).sum().backward()
    g = _gen(dev, 82)
    step = 2.0 ** -7
    for i in range(3):
        r = torch.randn(xs[i].shape, generator=g, device=dev)
        ends = []
        for sign in (1, -1):
            moved = [x.detach() + (sign * step * r if j == i else 0) for j, x in enumerate(xs)]
            ends.append((w.double() * T.attention_forward(*moved, plan)[0].double()).sum().item())
        slope = (ends[0] - ends[1]) / (2 * step)
        want = (xs[i].grad.double() * r.double()).sum().item()
        scale = (xs[i].grad.double().norm() * r.double().norm()).item() / math.sqrt(r.numel())
        assert abs(slope - want) <= 3e-3 * max(abs(want), scale), (i, slope, want)


def test_attention_autograd_matches_calls(dev):
    lens = [90, 45]
    q, k, v, dout = _qkv(dev, 91, sum(lens), 4, 2, 64, BF16)
    plan = T.AttentionPlan(lens, True, dev)
    out, lse = T.attention_forward(q, k, v, plan)
    want = T.attention_backward(dout, q, k, v, out, lse, plan)
    xs = [x.clone().requires_grad_() for x in (q, k, v)]
    y = T.attention(*xs, plan)
    assert torch.equal(y, out)
    y.backward(dout)
    for x, g in zip(xs, want):
        assert torch.equal(x.grad, g)


# ----------------------------------------------------------- checkpoints ---
def _activations(dev, seed, rows, cols, dtype):
    g = _gen(dev, seed)
    x = torch.randn(rows, cols, generator=g, device=dev) * torch.exp(torch.randn(cols, generator=g, device=dev))
    return x.to(dtype)


def _special(dev, dtype):
    """Rows of one group each, and one of two groups of which the second is short."""
    rows = [[0.0], [1e-45], [2.0 ** -126], [2.0 ** -140, -(2.0 ** -127)], [127.0, 63.5, 0.5, -0.5, 1.5, 2.5],
            [127.5, 1.0], [127.49999, -127.4], [1.0, 2.0 ** -8, 2.0 ** -9], [3.3895314e38, 1.0],
            [-3.3895314e38, 3.0e38], [float("nan"), 1.0], [float("inf"), 1.0], [-float("inf"), float("nan")],
            [255.0, 1.0, 3.0, 5.0], [-128.0, 64.0]]
    x = torch.zeros(len(rows), 70)
    for i, r in enumerate(rows):
        x[i, :len(r)] = torch.tensor(r)
        x[i, 66] = i - 7.25
    return x.to(device=dev, dtype=dtype)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 64), (3, 65), (7, 127), (5, 128), (130, 200), (33, 1000)])
def test_pack_matches_definition(dev, dtype, rows, cols):
    x = _activations(dev, 3 + rows + cols, rows, cols, dtype)
    c = T.checkpoint_pack(x)
    codes, exps = encode_reference(x)
    assert np.array_equal(c.codes.cpu().numpy(), codes)
    assert np.array_equal(c.exps.cpu().numpy(), exps)
    want = decode_reference(codes, exps, cols)
    for out in (BF16, F32):
        y = T.checkpoint_unpack(c, out)
        assert y.dtype == out and np.array_equal(y.double().cpu().numpy(), want)
    # Half a step at most, and a step is at most amax / 63.
    top = np.repeat(np.abs(np.pad(x.double().cpu().numpy(), ((0, 0), (0, -cols % 64)))).reshape(rows, -1, 64)
                    .max(2), 64, axis=1)[:, :cols]
    assert (np.abs(x.double().cpu().numpy() - want) <= top / 126).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_pack_special_groups(dev, dtype):
    x = _special(dev, dtype)
    c = T.checkpoint_pack(x)
    codes, exps = encode_reference(x)
    assert np.array_equal(c.codes.cpu().numpy(), codes)
    assert np.array_equal(c.exps.cpu().numpy(), exps)
    for out in (BF16, F32):
        y = T.checkpoint_unpack(c, out).double().cpu().numpy()
        want = decode_reference(codes, exps, x.shape[1])
        assert np.array_equal(np.isnan(y), np.isnan(want)) and np.array_equal(y[~np.isnan(y)], want[~np.isnan(want)])


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("how", ["strided", "odd_stride", "misaligned", "transposed", "expanded"])
def test_pack_strides(dev, dtype, how):
    x = _activations(dev, 9, 50, 150, dtype)
    if how == "strided":
        y = torch.zeros(50, 400, dtype=dtype, device=dev)[:, 40:190]
    elif how == "odd_stride":
        y = torch.zeros(50, 153, dtype=dtype, device=dev)[:, :150]
    elif how == "misaligned":
        y = torch.zeros(50 * 150 + 1, dtype=dtype, device=dev)[1:].view(50, 150)
    elif how == "transposed":
        y = torch.zeros(150, 50, dtype=dtype, device=dev).t()
    else:
        x = x[:1].expand(50, 150)
        y = x
    if how != "expanded":
        y.copy_(x)
    a, b = T.checkpoint_pack(x.contiguous()), T.checkpoint_pack(y)
    assert torch.equal(a.codes, b.codes) and torch.equal(a.exps, b.exps)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("act", ["gelu", "swiglu"])
@pytest.mark.parametrize("rows,cols", [(1, 3), (4, 64), (37, 130), (64, 777)])
def test_act_and_its_checkpoints(dev, dtype, act, rows, cols):
    u = _activations(dev, 17, rows, cols, dtype)
    up = _activations(dev, 18, rows, cols, dtype) if act == "swiglu" else None
    h, cu, cup, ch = T.checkpoint_act(act, u, up)
    ud = u.double().cpu().numpy()
    want = act_reference(act, ud, None if up is None else up.double().cpu().numpy())
    # The logistic function's argument is off by 4 u relative, so the result by
    # |z| 4 u + 8 u relative; then the rounding to the type.
    z = np.abs(1.6 * (np.abs(ud) + 0.045 * np.abs(ud) ** 3)) if act == "gelu" else np.abs(ud)
    half = H if dtype == BF16 else 0.0
    assert_within("h", h, want, np.abs(want) * ((4 * z + 8) * U + half) + 1e-38)
    for c, x in ((cu, u), (cup, up), (ch, h)):
        if x is None:
            assert c is None
            continue
        codes, exps = encode_reference(x)
        assert np.array_equal(c.codes.cpu().numpy(), codes) and np.array_equal(c.exps.cpu().numpy(), exps)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("act", ["gelu", "swiglu"])
@pytest.mark.parametrize("rows,cols", [(1, 3), (4, 64), (37, 130), (64, 777)])
def test_act_grad(dev, dtype, act, rows, cols):
    cu = T.checkpoint_pack(_activations(dev, 27, rows, cols, dtype))
    cup = T.checkpoint_pack(_activations(dev, 28, rows, cols, dtype)) if act == "swiglu" else None
    dh = _activations(dev, 29, rows, cols, dtype)
    u = decode_reference(cu.codes, cu.exps, cols)
    up = None if cup is None else decode_reference(cup.codes, cup.exps, cols)
    d = dh.double().cpu().numpy()
    du, dup = T.checkpoint_act_grad(act, dh, cu, cup)
    want, want_up = act_grad_reference(act, d, u, up)
    half = H if dtype == BF16 else 0.0
    # Terms of the sum in the derivative, each off by (4 |z| + 16) u relative; the
    # second factor |u z'| is at most |z| of a cubic, 3 times it.
    z = np.abs(1.6 * (np.abs(u) + 0.045 * np.abs(u) ** 3)) if act == "gelu" else np.abs(u)
    mag = np.abs(d) * (1 + 3 * z) * (1.0 if up is None else np.abs(up))
    assert_within("du", du, want, (4 * z + 16) * U * mag + half * np.abs(want) + 1e-38)
    if cup is not None:
        assert_within("dup", dup, want_up, (4 * z + 16) * U * np.abs(d * u) + half * np.abs(want_up) + 1e-38)


@pytest.mark.parametrize("act", ["gelu", "swiglu"])
def test_act_far_out(dev, act):
    # Far from zero the derivative is 0 or 1 (times up), whatever the formula's
    # terms do on the way.
    big = torch.tensor([1e3, 1e8, 1e20, 1e37], device=dev)
    u = torch.stack([big, -big])[:, :, None].expand(2, 4, 64).reshape(2, 256)
    cu = T.checkpoint_pack(u)
    cup = T.checkpoint_pack(torch.ones(2, 256, device=dev)) if act == "swiglu" else None
    du, _ = T.checkpoint_act_grad(act, torch.ones(2, 256, device=dev), cu, cup)
    assert torch.equal(du, torch.tensor([[1.0], [0.0]], device=dev).expand(2, 256))
    h = T.checkpoint_act(act, u, None if cup is None else torch.ones(2, 256, device=dev))[0]
    assert torch.equal(h, u.clamp(min=0))


@pytest.mark.parametrize("act", ["gelu", "swiglu"])
def test_act_grad_against_differences(dev, act):
    # Central differences of the activation at the held values, in 64 bits: step
    # 2^-12, third derivatives below 4 here, so the error is below 4 2^-24 / 6,
    # plus that of the kernel's fp32 result.
    cu = T.checkpoint_pack(torch.linspace(-6, 6, 320, device=dev).view(5, 64))
    cup = T.checkpoint_pack(torch.linspace(3, -2, 320, device=dev).view(5, 64)) if act == "swiglu" else None
    u = decode_reference(cu.codes, cu.exps, 64)
    up = None if cup is None else decode_reference(cup.codes, cup.exps, 64)
    dh = torch.ones(5, 64, device=dev)
    du, dup = T.checkpoint_act_grad(act, dh, cu, cup)
    s = 2.0 ** -12
    slope = (act_reference(act, u + s, up) - act_reference(act, u - s, up)) / (2 * s)
    assert np.abs(du.double().cpu().numpy() - slope).max() <= 4e-6
    if dup is not None:
        slope = (act_reference(act, u, up + s) - act_reference(act, u, up - s)) / (2 * s)
        assert np.abs(dup.double().cpu().numpy() - slope).max() <= 4e-6


def _weight_bound(x, d, tokens):
    """Every product is exact: only the sums round."""
    return (tokens + 8) * U * (np.abs(x).T @ np.abs(d)) + 1e-38


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("layout", ["io", "oi"])
@pytest.mark.parametrize("tokens,inner,outer", [
    (1, 1, 1), (2, 64, 64), (31, 65, 129), (64, 128, 128), (100, 257, 100), (700, 130, 300), (1100, 70, 33),
    (4099, 200, 136),
])
def test_weight_grad(dev, dtype, layout, tokens, inner, outer):
    print(f"weight_grad {dtype} {layout} {tokens} {inner} {outer}", flush=True)
    c = T.checkpoint_pack(_activations(dev, 37, tokens, inner, dtype))
    dy = _activations(dev, 38, tokens, outer, dtype)
    x, d = decode_reference(c.codes, c.exps, inner), dy.double().cpu().numpy()
    want, tol = x.T @ d, _weight_bound(x, d, tokens)
    if layout == "oi":
        want, tol = want.T, tol.T
    got = T.checkpoint_weight_grad(c, dy, layout)
    assert_within("dw", got, want, tol)
    assert torch.equal(got, T.checkpoint_weight_grad(c, dy, layout))
    # Into a part of a larger matrix, added to what is there.
    big = torch.full((got.shape[0] + 2, got.shape[1] + 5), 3.0, device=dev)
    part = big[1:-1, 2:-3]
    T.checkpoint_weight_grad(c, dy, layout, out=part, accumulate=True)
    assert_within("accumulated", part, want + 3.0, tol + U * (np.abs(want) + 3.0) * 2)
    big[1:-1, 2:-3] = 3.0
    assert (big == 3.0).all()


@pytest.mark.parametrize("layout", ["io", "oi"])
@pytest.mark.parametrize("tokens,inner,outer", [
    (1, 2049, 3843), (33, 2048, 4096), (100, 4096, 2056), (161, 2049, 3843), (70, 33000, 3), (70, 33000, 250),
])
def test_weight_grad_of_large_matrices(dev, layout, tokens, inner, outer):
    # 128 tiles of 256 x 256 or more, the widths a multiple of the tile, of 8, or
    # odd.  fp64 on the GPU: the same numbers as the other tests' reference.
    print(f"weight_grad large {layout} {tokens} {inner} {outer}", flush=True)
    x = _activations(dev, 39, tokens, inner, BF16)
    if tokens == 100:
        x[7, 1030] = float("nan")
    c = T.checkpoint_pack(x)
    dy = _activations(dev, 40, tokens, outer, BF16)
    held, d = torch.from_numpy(decode_reference(c.codes, c.exps, inner)).to(dev), dy.double()
    want = held.T @ d if layout == "io" else d.T @ held
    tol = (tokens + 8) * U * (held.abs().T @ d.abs() if layout == "io" else d.abs().T @ held.abs()) + 1e-38
    got = T.checkpoint_weight_grad(c, dy, layout)
    assert torch.equal(torch.isfinite(got), torch.isfinite(want))
    fine = torch.isfinite(want)
    assert fine.all() or (~fine).sum() == 64 * outer
    assert ((got.double() - want).abs() <= tol)[fine].all()
    assert torch.equal(got.nan_to_num(7.0), T.checkpoint_weight_grad(c, dy, layout).nan_to_num(7.0))
    # Into a part of a larger matrix, added to what is there.
    big = torch.full((got.shape[0] + 2, got.shape[1] + 5), 3.0, device=dev)
    part = big[1:-1, 2:-3]
    T.checkpoint_weight_grad(c, dy, layout, out=part, accumulate=True)
    assert ((part.double() - want - 3.0).abs() <= tol + 2 * U * (want.abs() + 3.0))[fine].all()
    assert torch.equal(torch.isfinite(part), fine)
    big[1:-1, 2:-3] = 3.0
    assert (big == 3.0).all()


@pytest.mark.parametrize("how", ["strided", "odd_stride", "misaligned", "transposed"])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_weight_grad_strides(dev, dtype, how):
    c = T.checkpoint_pack(_activations(dev, 47, 90, 70, dtype))
    dy = _activations(dev, 48, 90, 150, dtype)
    y = {"strided": lambda: torch.zeros(90, 400, dtype=dtype, device=dev)[:, 40:190],
         "odd_stride": lambda: torch.zeros(90, 153, dtype=dtype, device=dev)[:, :150],
         "misaligned": lambda: torch.zeros(90 * 150 + 1, dtype=dtype, device=dev)[1:].view(90, 150),
         "transposed": lambda: torch.zeros(150, 90, dtype=dtype, device=dev).t()}[how]()
    y.copy_(dy)
    assert torch.equal(T.checkpoint_weight_grad(c, y), T.checkpoint_weight_grad(c, dy))


def test_weight_grad_of_no_tokens(dev):
    c = T.checkpoint_pack(torch.empty(0, 70, device=dev))
    dy = torch.empty(0, 30, device=dev)
    assert (T.checkpoint_weight_grad(c, dy, "io") == 0).all()
    out = torch.ones(30, 70, device=dev)
    T.checkpoint_weight_grad(c, dy, "oi", out=out, accumulate=True)
    assert (out == 1).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_weight_grad_nonfinite(dev, dtype):
    # A NaN in x reaches the 64 features of its group, an infinity in dy its column.
    x, dy = _activations(dev, 57, 40, 200, dtype), _activations(dev, 58, 40, 90, dtype)
    x[7, 70] = float("nan")
    dy[9, 5] = float("inf")
    c = T.checkpoint_pack(x)
    got = T.checkpoint_weight_grad(c, dy, "io").cpu()
    bad = torch.zeros(200, 90, dtype=torch.bool)
    bad[64:128] = True
    bad[:, 5] = True
    assert torch.equal(~torch.isfinite(got), bad)
    # Past the infinity only the sign of the code counts.
    held = torch.from_numpy(decode_reference(c.codes, c.exps, 200)[9])
    col = got[:, 5]
    keep = torch.ones(200, dtype=torch.bool)
    keep[64:128] = False
    assert torch.equal(col[keep & (held > 0)], torch.full_like(col[keep & (held > 0)], float("inf")))
    assert torch.equal(col[keep & (held < 0)], torch.full_like(col[keep & (held < 0)], float("-inf")))


def test_weight_grad_fp32_terms(dev):
    # One token: every product of a code and an fp32 value with all 24 bits set,
    # over the whole range of exponents, is within one rounding.
    g = _gen(dev, 67)
    x = torch.zeros(1, 64, device=dev)
    x[0, 0], x[0, 1] = 127.0, 1.0
    dy = torch.randn(1, 500, generator=g, device=dev) * 2.0 ** torch.linspace(-90, 110, 500, device=dev)
    got = T.checkpoint_weight_grad(T.checkpoint_pack(x), dy, "io").double()
    for i, c in ((0, 127.0), (1, 1.0)):
        want = c * dy[0].double()
        assert ((got[i] - want).abs() <= 3 * U * want.abs()).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("layout", ["io", "oi"])
def test_weight_grad_of_the_largest_values(dev, dtype, layout):
    # Magnitudes past 2^127 give a group the largest exponent, 121; dy makes the
    # products ordinary numbers.
    g = _gen(dev, 68)
    x = _activations(dev, 69, 40, 200, dtype)
    x[3:20, 64:128] = (3.3e38 * (2 * torch.rand(17, 64, generator=g, device=dev) - 1)).to(dtype)
    x[3:20, 70] = 3.3e38
    c = T.checkpoint_pack(x)
    assert (c.exps[3:20, 1] == 121).all()
    dy = (1e-25 * torch.randn(40, 90, generator=g, device=dev)).to(dtype)
    held, d = decode_reference(c.codes, c.exps, 200), dy.double().cpu().numpy()
    want, tol = held.T @ d, _weight_bound(held, d, 40)
    if layout == "oi":
        want, tol = want.T, tol.T
    assert_within("dw", T.checkpoint_weight_grad(c, dy, layout), want, tol)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("layout", ["io", "oi"])
@pytest.mark.parametrize("tokens", [33, 97, 129, 1025])
@pytest.mark.parametrize("outer,ld", [(1, 1), (2, 2), (3, 3), (6, 6), (3, 7), (9, 9)])
def test_weight_grad_of_narrow_rows(dev, dtype, layout, tokens, outer, ld):
    # Rows of dy shorter than the pieces that wider ones are read in, up to the very
    # end of their buffer.
    c = T.checkpoint_pack(_activations(dev, 70, tokens, 70, dtype))
    buf = torch.full(((tokens - 1) * ld + outer,), float("nan"), dtype=dtype, device=dev)
    dy = buf.as_strided((tokens, outer), (ld, 1))
    dy.copy_(_activations(dev, 71, tokens, outer, dtype))
    x, d = decode_reference(c.codes, c.exps, 70), dy.double().cpu().numpy()
    want, tol = x.T @ d, _weight_bound(x, d, tokens)
    if layout == "oi":
        want, tol = want.T, tol.T
    assert_within("dw", T.checkpoint_weight_grad(c, dy, layout), want, tol)


# ------------------------------------------------------------------ layers ---
@pytest.mark.parametrize("layout", ["io", "oi"])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_checkpointed_linear(dev, dtype, layout):
    g = _gen(dev, 77)
    x = torch.randn(130, 96, generator=g, device=dev).to(dtype).requires_grad_()
    w = (torch.randn(*((96, 200) if layout == "io" else (200, 96)), generator=g, device=dev) * 0.1).requires_grad_()
    b = torch.randn(200, generator=g, device=dev).requires_grad_()
    dy = torch.randn(130, 200, generator=g, device=dev).to(dtype)
    y = T.checkpointed_linear(x, w, b, layout)
    y.backward(dy)
    c = T.checkpoint_pack(x.detach())
    wt = w.detach().to(dtype)
    assert torch.equal(y, (x.detach() @ (wt if layout == "io" else wt.t())) + b.detach().to(dtype))
    assert torch.equal(w.grad, T.checkpoint_weight_grad(c, dy, layout))
    assert torch.equal(x.grad, dy @ (wt.t() if layout == "io" else wt))
    assert torch.equal(b.grad, dy.sum(0, dtype=F32))


@pytest.mark.parametrize("act", ["gelu", "swiglu"])
@pytest.mark.parametrize("layout", ["io", "oi"])
def test_checkpointed_mlp_against_formula(dev, act, layout):
    # fp32, against the formula in 64 bits with the held values in place of the
    # activations (that of h and the checkpoints come from the kernels' own h).
    g = _gen(dev, 87)
    t, n, m = 70, 64, 160
    shape = lambda a, b: (a, b) if layout == "io" else (b, a)  # noqa: E731
    x = torch.randn(t, n, generator=g, device=dev).requires_grad_()
    w1, w3 = ((torch.randn(*shape(n, m), generator=g, device=dev) * 0.1).requires_grad_() for _ in range(2))
    w2 = (torch.randn(*shape(m, n), generator=g, device=dev) * 0.1).requires_grad_()
    gated = act == "swiglu"
    b1, b2 = (None, None) if gated else (torch.randn(k, generator=g, device=dev).requires_grad_() for k in (m, n))
    dy = torch.randn(t, n, generator=g, device=dev)
    y = T.checkpointed_mlp(x, w1, w2, act=act, w_up=w3 if gated else None, b_in=b1, b_out=b2, layout=layout)
    y.backward(dy)
    D = lambda z: z.detach().double().cpu().numpy()  # noqa: E731
    W = lambda z: D(z) if layout == "io" else D(z).T  # noqa: E731
    u = D(x) @ W(w1) + (0 if gated else D(b1))
    up = D(x) @ W(w3) if gated else None
    h = act_reference(act, u, up)
    held = lambda z: decode_reference(*encode_reference(torch.from_numpy(z)), z.shape[1])  # noqa: E731
    dh = D(dy) @ W(w2).T
    du, dup = act_grad_reference(act, dh, held(u), held(up) if gated else None)
    want = {"dx": du @ W(w1).T + (dup @ W(w3).T if gated else 0), "w1": held(D(x)).T @ du, "w2": held(h).T @ D(dy)}
    got = {"dx": D(x.grad), "w1": W(w1.grad), "w2": W(w2.grad)}
    if gated:
        want["w3"], got["w3"] = held(D(x)).T @ dup, W(w3.grad)
    else:
        want |= {"b1": du.sum(0), "b2": D(dy).sum(0)}
        got |= {"b1": D(b1.grad), "b2": D(b2.grad)}
    np.testing.assert_allclose(D(y), h @ W(w2) + (0 if gated else D(b2)), rtol=0, atol=1e-5)
    for name in want:
        # A value beside a tie may round to the next code: at most a step of
        # amax / 63 at a few places; fp32 elsewhere.
        err = np.linalg.norm(got[name] - want[name]) / np.linalg.norm(want[name])
        assert err <= 1e-3, (name, err)


def test_checkpointed_layers_with_frozen_parts(dev):
    x = torch.randn(40, 64, device=dev)
    w1, w2 = torch.randn(128, 64, device=dev), torch.randn(64, 128, device=dev).requires_grad_()
    b = torch.randn(128, device=dev, dtype=torch.float64).requires_grad_()
    with torch.autocast("cuda", torch.bfloat16):
        y = T.checkpointed_mlp(T.checkpointed_linear(x, w1, b) @ w1, w1, w2)
    assert y.dtype == BF16
    y.float().sum().backward()
    assert w1.grad is None and w2.grad.shape == w2.shape and b.grad.dtype == torch.float64
    with torch.no_grad():
        assert torch.equal(T.checkpointed_linear(x, w1, layout="oi"), x @ w1.t())


@pytest.mark.parametrize("act", ["linear", "gelu", "swiglu"])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_checkpointed_layers_backward_under_autocast(dev, act, dtype):
    # The same gradients whether the backward pass is called under autocast or not.
    grads = []
    for inside in (False, True):
        g = _gen(dev, 79)
        x = torch.randn(70, 64, generator=g, device=dev).to(dtype).requires_grad_()
        w1, w3 = ((torch.randn(160, 64, generator=g, device=dev) * 0.1).requires_grad_() for _ in range(2))
        w2 = (torch.randn(64, 160, generator=g, device=dev) * 0.1).requires_grad_()
        with torch.autocast("cuda", BF16):
            if act == "linear":
                y = T.checkpointed_linear(x, w1)
            else:
                y = T.checkpointed_mlp(x, w1, w2, act=act, w_up=w3 if act == "swiglu" else None)
            dy = torch.randn(y.shape, generator=g, device=dev).to(dtype)
            if inside:
                y.backward(dy)
        if not inside:
            y.backward(dy)
        grads.append([t.grad for t in (x, w1, w2, w3) if t.grad is not None])
    assert len(grads[0]) == len(grads[1]) == {"linear": 2, "gelu": 3, "swiglu": 4}[act]
    for a, b in zip(*grads):
        assert torch.equal(a, b)


def test_checkpointed_layers_keep_x_for_training_only(dev, monkeypatch):
    packed = []
    pack = T.checkpoint_pack
    monkeypatch.setattr(T, "checkpoint_pack", lambda x: packed.append(x.shape) or pack(x))
    x = torch.randn(40, 64, device=dev)
    w1, w2, w3 = (torch.randn(128, 64, device=dev).requires_grad_() for _ in range(3))
    layers = [lambda a, b, c: T.checkpointed_linear(x, a), lambda a, b, c: T.checkpointed_mlp(x, a, b.t()),
              lambda a, b, c: T.checkpointed_mlp(x, a, b.t(), act="swiglu", w_up=c)]
    trained = [f(w1, w2, w3).detach() for f in layers]
    assert packed == [x.shape] * 3
    with torch.no_grad():
        for f, y in zip(layers, trained):
            assert torch.equal(f(w1, w2, w3), y)
    # Frozen in part: x is not needed for w_out's gradient.
    f1, f3 = w1.detach(), w3.detach()
    for f in layers[1:]:
        f(f1, w2, f3).sum().backward()
        assert w2.grad is not None
    assert packed == [x.shape] * 3
    T.checkpointed_mlp(x, f1, w2.t(), act="swiglu", w_up=w3).sum().backward()
    assert packed == [x.shape] * 4 and w3.grad is not None and w1.grad is None


def test_checkpointed_layers_keep_8_bits(dev):
    x = torch.randn(256, 128, device=dev).requires_grad_()
    w = torch.randn(512, 128, device=dev).requires_grad_()
    kept = []
    with torch.autograd.graph.saved_tensors_hooks(lambda t: kept.append(t) or t, lambda t: t):
        T.checkpointed_linear(x, w)
    kept = [t for t in kept if t.data_ptr() != w.data_ptr()]
    assert sum(t.numel() * t.element_size() for t in kept) == 256 * (128 + 2)


# ---------------------------------------------------- streams and graphs ---
def test_operators_on_a_side_stream(dev):
    s = torch.cuda.Stream()
    lens = [200, 56]
    with torch.cuda.stream(s):
        # Inputs made on the stream, used on it without a wait.
        torch.cuda._sleep(20_000_000)
        q, k, v, dout = _qkv(dev, 97, sum(lens), 4, 2, 64, BF16)
        plan = T.AttentionPlan(lens, True, dev)
        out, lse = T.attention_forward(q, k, v, plan)
        grads = T.attention_backward(dout, q, k, v, out, lse, plan)
        h, cu, _, ch = T.checkpoint_act("gelu", q.flatten(1))
        du, _ = T.checkpoint_act_grad("gelu", dout.flatten(1), cu)
        dw = T.checkpoint_weight_grad(ch, dout.flatten(1))
    s.synchronize()
    out2, lse2 = T.attention_forward(q, k, v, plan)
    assert torch.equal(out, out2)
    for a, b in zip(grads, T.attention_backward(dout, q, k, v, out2, lse2, plan)):
        assert torch.equal(a, b)
    h2, cu2, _, ch2 = T.checkpoint_act("gelu", q.flatten(1))
    assert torch.equal(h, h2)
    assert torch.equal(du, T.checkpoint_act_grad("gelu", dout.flatten(1), cu2)[0])
    assert torch.equal(dw, T.checkpoint_weight_grad(ch2, dout.flatten(1)))


def test_operators_in_a_graph(dev):
    lens = [200, 56, 700]
    q, k, v, dout = _qkv(dev, 107, sum(lens), 4, 2, 64, BF16)
    plan = T.AttentionPlan(lens, True, dev)

    def step():
        out, lse = T.attention_forward(q, k, v, plan)
        grads = T.attention_backward(dout, q, k, v, out, lse, plan)
        h, cu, cup, ch = T.checkpoint_act("swiglu", q.flatten(1), dout.flatten(1))
        du, dup = T.checkpoint_act_grad("swiglu", dout.flatten(1), cu, cup)
        return (out, *grads, h, du, dup, T.checkpoint_weight_grad(ch, out.flatten(1)))

    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        got = step()
    for r in range(3):
        q.mul_(-0.7).add_(0.01)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(got, step()):
            assert torch.equal(a, b), r


# ---------------------------------------------------------------- refusals ---
def test_refusals(dev):
    q, k, v, dout = _qkv(dev, 117, 20, 4, 2, 64, BF16)
    plan = T.AttentionPlan([20], True, dev)
    out, lse = T.attention_forward(q, k, v, plan)
    with pytest.raises(ValueError):
        T.attention_forward(q, k, v, T.AttentionPlan([19], True, dev))
    with pytest.raises(ValueError):
        T.attention_forward(q, k.float(), v, plan)
    with pytest.raises(ValueError):
        T.attention_forward(q, k[:, :, :32], v, plan)
    with pytest.raises(TypeError):
        T.attention_forward(q.half(), k.half(), v.half(), plan)
    with pytest.raises(N.NormPreError) as e:
        T.attention_forward(q[:, :3], k, v, plan)
    assert e.value.code == N.NORMPRE_ERR_INVALID_ARG
    with pytest.raises(N.NormPreError) as e:
        T.attention_forward(*(x.repeat(1, 1, 3) for x in (q, k, v)), plan)
    assert e.value.code == N.NORMPRE_ERR_UNSUPPORTED
    with pytest.raises(N.NormPreError):
        T.attention_forward(q, k, v, plan, float("nan"))
    with pytest.raises(ValueError):
        T.attention_backward(dout[:10], q, k, v, out, lse, plan)
    with pytest.raises(ValueError):
        T.attention_backward(dout, q, k, v, out, lse[:, :10], plan)
    with pytest.raises(N.NormPreError) as e:
        T.AttentionPlan([3, -1], True, dev)
    assert e.value.code == N.NORMPRE_ERR_INVALID_ARG
    with pytest.raises(ValueError):
        T.checkpoint_act("relu", q.flatten(1))
    c = T.checkpoint_pack(q.flatten(1))
    with pytest.raises(ValueError):
        T.checkpoint_weight_grad(c, dout.flatten(1)[:10])
    with pytest.raises(ValueError):
        T.checkpoint_weight_grad(c, dout.flatten(1), "xy")
    with pytest.raises(ValueError):
        T.checkpoint_weight_grad(c, dout.flatten(1), out=torch.empty(3, 3, device=dev))
    with pytest.raises(ValueError):
        T.checkpoint_act_grad("gelu", dout.flatten(1)[:, :100], c)
    with pytest.raises(ValueError):
        T.checkpoint_act_grad("swiglu", dout.flatten(1), c)
    with pytest.raises(ValueError):
        T.checkpoint_pack(q)
    with pytest.raises(TypeError):
        T.checkpoint_pack(q.flatten(1).half())
    with pytest.raises(TypeError):
        T.checkpoint_unpack(c, torch.float16)


def test_refusals_of_empty_heads_and_types(dev):
    plan = T.AttentionPlan([20], True, dev)
    empty = torch.empty(20, 2, 0, device=dev, dtype=BF16)
    with pytest.raises(N.NormPreError) as e:
        T.attention_forward(empty, empty, empty, plan)
    assert e.value.code == N.NORMPRE_ERR_INVALID_ARG
    x, w = torch.randn(20, 64, device=dev), torch.randn(32, 64, device=dev)
    with torch.no_grad(), pytest.raises(TypeError):
        T.checkpointed_linear(x.half(), w)
    with torch.no_grad(), pytest.raises(TypeError):
        T.checkpointed_mlp(x.double(), w, w.t())
