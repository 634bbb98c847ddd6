"""Epilogues of products whose columns are split over a cluster: (N, M, K) with which a tile's sums are divided among 2, 4, 8 and 16 ranks, of 16, 32, 64 and 128 tokens, where a
rank has fewer (token, four rows) than a warp has lanes, more than the block has threads, and last rows that are not four. Bounds: tests/test_gpu_epilogue.py."""
import math

import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

from test_gpu_epilogue import BF16, F16, F32, b, check, gen, make  # noqa: F401

# ranks, tokens a tile, items a rank: 16, 16, 2; 4, 16, 8; 2, 16, 80; 4, 16, 128; 8, 16, 64; 2, 16, 256; 8, 32, 128; 2, 64, 528; 4, 64, 512; 4, 128, 800; 2, 128, 2048
SPLIT = [(1, 130, 16384), (1, 1024, 4096), (5, 1, 2048), (16, 7, 4096), (16, 130, 8192), (16, 2000, 2048), (32, 1000, 8192), (33, 1001, 2003), (64, 250, 4100), (100, 387, 16500),
         (300, 130, 8200)]


def even(M, gated):
    return M + M % 2 if gated else M


@pytest.mark.parametrize("act", [None, "relu", "silu", "gelu", "gelu_tanh"])
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("N,M,K", SPLIT)
@pytest.mark.parametrize("dtype", [F16, F32])
def test_activations(b, act, gated, N, M, K, dtype):  # noqa: F811
    x, w, kw = make(b, N, even(M, gated), K, BF16, N + M, F32, BF16, gated)
    y = b.mx4_linear(x, w, dtype=dtype, act=act, gated=gated, **kw)
    b.mx4_check()
    check(y, b.mx4_quantize(x).dequantize(), w.dequantize(), kw["bias"], act, gated, kw["residual"])


@pytest.mark.parametrize("bias", [None, F16, BF16, F32])
@pytest.mark.parametrize("residual", [None, F16, BF16, F32])
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("N,M,K", [(1, 130, 16384), (16, 2000, 2048), (33, 1001, 2003), (100, 387, 16500)])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_types(b, bias, residual, gated, N, M, K, dtype):  # noqa: F811
    x, w, kw = make(b, N, even(M, gated), K, F16, N, bias, residual, gated)
    y = b.mx4_linear(x, w, dtype=dtype, act="silu", gated=gated, **kw)
    b.mx4_check()
    check(y, b.mx4_quantize(x).dequantize(), w.dequantize(), kw["bias"], "silu", gated, kw["residual"])


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("N,M,K", SPLIT)
@pytest.mark.parametrize("pad", [0, 3])
def test_strides_and_in_place(b, gated, N, M, K, pad):  # noqa: F811
    """The residual is the output itself, rows apart; columns beside stay as they were."""
    M = even(M, gated)
    x, w, kw = make(b, N, M, K, BF16, M + pad, F32, None, gated)
    cols = M // 2 if gated else M
    rows = torch.randn(N, cols + 2 * pad, device="cuda", generator=gen(1)).to(BF16)
    keep, view = rows.clone(), rows[:, pad:pad + cols]
    apart = b.mx4_linear(x, w, act="silu", gated=gated, bias=kw["bias"], residual=keep[:, pad:pad + cols])
    got = b.mx4_linear(x, w, out=view, act="silu", gated=gated, bias=kw["bias"], residual=view)
    b.mx4_check()
    assert got is view and torch.equal(view, apart)
    assert torch.equal(rows[:, :pad], keep[:, :pad]) and torch.equal(rows[:, pad + cols:], keep[:, pad + cols:])
    check(apart, b.mx4_quantize(x).dequantize(), w.dequantize(), kw["bias"], "silu", gated, keep[:, pad:pad + cols])


@pytest.mark.parametrize("N,M,K", [(2, 254, 16400), (20, 1000, 8192), (100, 386, 16500), (1024, 5120, 64)])
def test_values_at_the_edges(b, N, M, K):  # noqa: F811
    """Large arguments of both signs; infinities and NaN stay in their places (the last: of pairs of SMs, which no other test has)."""
    x, w, _ = make(b, N, M, K, F32, N, spread=40.0)
    bias = torch.linspace(-300, 300, M, device="cuda")
    for act in ("silu", "gelu", "gelu_tanh", "relu"):
        for dtype in (BF16, F32):
            check(b.mx4_linear(x, w, dtype=dtype, act=act, bias=bias), b.mx4_quantize(x).dequantize(), w.dequantize(), bias, act, False, None)
    res = torch.zeros(N, M, device="cuda")
    res[1, 5], res[0, 7], res[1, 100] = math.inf, -math.inf, math.nan
    for r in (res, res.bfloat16()):
        y = b.mx4_linear(x, w, residual=r, act="relu")
        assert y[1, 5] == math.inf and y[0, 7] == -math.inf and bool(y[1, 100].isnan())
        same = torch.isfinite(res)
        assert torch.equal(y[same], b.mx4_linear(x, w, act="relu")[same])
    bias[3] = math.nan
    y = b.mx4_linear(x, w, act="relu", bias=bias)
    assert bool(y[:, 3].isnan().all()) and int(y.isnan().sum()) == N
    x[1, 3] = math.nan
    y = b.mx4_linear(x, w, act="relu", gated=True)
    assert bool(y[1].isnan().all()) and int(y.isnan().sum()) == M // 2
    b.mx4_check()


def test_graph_and_stream(b):  # noqa: F811
    """Bias and residual that the kernels just before write."""
    for N, M, K in SPLIT:
        x, w, kw = make(b, N, even(M, True), K, F16, N, F16, F16, True)
        w.freeze()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            r, bias = kw["residual"] * 2, kw["bias"] * 3
            r = b.mx4_linear(x, w, act="silu", gated=True, bias=bias, residual=r, out=r)
            z = b.mx4_linear(x, w, act="silu", gated=True, bias=bias, residual=r)
        for scale in (1.0, -3.0):
            base = kw["residual"].clone()
            kw["residual"].mul_(scale)
            graph.replay()
            torch.cuda.synchronize()
            want = b.mx4_linear(x, w, act="silu", gated=True, bias=kw["bias"] * 3, residual=kw["residual"] * 2)
            torch.cuda.synchronize()
            assert torch.equal(r, want)
            assert torch.equal(z, b.mx4_linear(x, w, act="silu", gated=True, bias=kw["bias"] * 3, residual=want))
            kw["residual"].copy_(base)
        st = torch.cuda.Stream()
        st.wait_stream(torch.cuda.current_stream())
        got = b.mx4_linear(x, w, act="silu", gated=True, stream=st.cuda_stream, **kw)
        st.synchronize()
        assert torch.equal(got, b.mx4_linear(x, w, act="silu", gated=True, **kw))
    b.mx4_check()
