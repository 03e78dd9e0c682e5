"""Attention with a window on the GPU: of which kind results are where they are not finite.

Compared with the 64-bit references of tests/window_util.py: NaN, +inf and -inf each at their own places
in out and dv.  Not compared are lse (the reference has the infinite score itself where the kernels have the
NaN of the sum), and dq and dk (the difference of dp and delta, both infinite, is NaN or infinite by
the form in which delta is summed)."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2609_36692_amd import train_ops as T  # noqa: E402
from train_ops_util import assert_within  # noqa: E402
from window_util import window_reference  # noqa: E402

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
INF, NAN = math.inf, math.nan


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return torch.device("cuda:0")


def _qkv(dev, seed, t, hq, hk, d, dtype):
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    return [torch.randn(t, h, d, generator=g, device=dev).to(dtype) for h in (hq, hk, hk, hq)]


def assert_kind(name, got, want):
    got = np.asarray(got.detach().double().cpu())
    for kind, is_it in (("NaN", np.isnan), ("+inf", np.isposinf), ("-inf", np.isneginf)):
        other = np.argwhere(is_it(got) != is_it(want))
        assert not len(other), f"{name}: {len(other)} places differ in being {kind}, the first {other[0].tolist()}: " \
                               f"{got[tuple(other[0])]} for {want[tuple(other[0])]}"


def _check(x, lens, window, sinks, rows):
    q, k, v, dout = x
    plan = T.AttentionPlan(lens, device=q.device, window=window, sinks=sinks)
    assert plan.bounds is not None
    out, lse = T.attention_forward(q, k, v, plan)
    dv = T.attention_backward(dout, q, k, v, out, lse, plan)[2]
    want, tol = window_reference(q, k, v, lens, window, sinks, 1.0 / math.sqrt(q.shape[2]), dout, [0])
    r = 1 if q.dtype == BF16 else 0
    for name, got in (("out", out), ("dv", dv)):
        assert_kind(name, got[:rows], want[name][:rows])
        assert_within(name, got[:rows], want[name][:rows], tol[name][r][:rows])


# A first token's sum over its queries has two parts, those within its window and those past it.  Tiles on
# the border between them are in both, with the other part's queries masked.
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("crowd", [0, 1100])         # shares of the queries, or one
@pytest.mark.parametrize("window,sinks", [(70, 3), (70, 40), (33, 130), (96, 33)])
def test_dv_of_first_tokens_at_the_border_of_their_windows(dev, dtype, d, crowd, window, sinks):
    n = 300
    lens = [n] + [1] * crowd
    for place in sorted({window - 31, window - 1, window, window + 2, window + 31, window + 61, 64, 96, 127, 128, 130, 160, 299}):
        if place >= n:
            continue
        for value in (INF, -INF) if place == 64 else (INF,):
            x = _qkv(dev, 21, sum(lens), 2, 1, d, dtype)
            x[3][place, place % 2, d // 2] = value
            print(f"dout[{place}] = {value}", flush=True)
            _check(x, lens, window, sinks, n)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d", [64, 40])
@pytest.mark.parametrize("where", ["q", "k", "v", "dout"])
@pytest.mark.parametrize("value", [NAN, INF, -INF])
def test_kinds_everywhere(dev, dtype, d, where, value):
    for place in (0, 2, 3, 63, 64, 130, 192, 299):
        x = _qkv(dev, 22, 340, 2, 1, d, dtype)
        dict(zip(("q", "k", "v", "dout"), x))[where][place, 0, d // 2] = value
        print(f"{where}[{place}] = {value}", flush=True)
        _check(x, [300, 40], 70, 3, 300)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_infinities_of_both_signs(dev, dtype):
    x = _qkv(dev, 23, 300, 2, 1, 64, dtype)
    dout = x[3]
    dout[71, 0, 5], dout[200, 1, 5], dout[64, 1, 6], dout[90, 0, 7], dout[66, 0, 8] = INF, -INF, -INF, NAN, INF
    _check(x, [300], 70, 3, 300)
