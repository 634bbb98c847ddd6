"""What follows an MX4 product in its epilogue, on the GPU against the formulas in 64 bits. The kernel's error:
  * of a sum v of K exact products in fp32: K 2^-23 of the sum of magnitudes; with its bias z = v + bias: 2^-24 |z| more;
  * of f: its slope (at most 1.13) times that; and its own. silu and gelu_tanh are x sigma(t): the exponential's argument is off by a few roundings, at most
    2^-22 |t| (sigma changes by (1 - sigma) of that), exponential and reciprocal by 2^-22 each, products: |f| (2^-22 |t| (1 - sigma(t)) + 2^-20); below 2^-126
    a quotient is 0: 2^-126 |x|. gelu is x erfc(-x / sqrt 2) / 2: an argument off by 2^-23 changes erfc by (x^2 + 2) 2^-23 at most, the function is good to a few ulp:
    |f| ((x^2 + 2) 2^-22 + 2^-20);
  * of a gated product: f's error times |u|, u's times |f|, 2^-24 |f u|; of the residual's sum: 2^-24 of it;
then the result's rounding, eps / 2."""
import math

import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

F16, BF16, F32 = torch.float16, torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def b():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a CUDA device")
    from paper_2608_09291_b200 import binding
    torch.cuda.set_device(0)
    return binding


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def apply(z, ez, act):
    """f(z) and its bound."""
    if act is None:
        return z, ez
    if act == "relu":
        return z.clamp(min=0), ez
    if act == "gelu":
        f = 0.5 * z * torch.special.erfc(-z / math.sqrt(2))
        own = f.abs() * ((z * z + 2) * 2.0 ** -22 + 2.0 ** -20)
    else:
        t = z if act == "silu" else 2 * math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)
        s = torch.sigmoid(t)
        f = z * s
        own = f.abs() * (2.0 ** -22 * t.abs() * torch.sigmoid(-t) + 2.0 ** -20)
    return f, 1.13 * ez + own + 2.0 ** -126 * z.abs()


def check(y, xv, wv, bias, act, gated, residual):
    x, w, K = xv.double(), wv.double(), xv.shape[1]
    z, e = x @ w.t(), K * 2.0 ** -23 * (x.abs() @ w.abs().t())
    if bias is not None:
        z = z + bias.double()
        e = e + 2.0 ** -24 * z.abs()
    if gated:
        (f, ef), u, eu = apply(z[:, 0::2], e[:, 0::2], act), z[:, 1::2], e[:, 1::2]
        ref = f * u
        e = ef * u.abs() + (f.abs() + ef) * eu + 2.0 ** -24 * ref.abs()
    else:
        ref, e = apply(z, e, act)
    if residual is not None:
        ref = ref + residual.double()
        e = e + 2.0 ** -24 * ref.abs()
    lim = e + torch.finfo(y.dtype).eps / 2 * (ref.abs() + e) + torch.finfo(y.dtype).tiny
    d = (y.double() - ref).abs()
    assert y.shape == ref.shape and (d <= lim).all(), f"off by {float((d / lim).max()):.2f} bounds"


def make(b, N, M, K, x_type, seed, bias=None, residual=None, gated=False, spread=3.0):
    """Activations whose products are some units large; a weight; what an epilogue takes (types, or None)."""
    g = gen(seed)
    x = (torch.randn(N, K, device="cuda", generator=g) * spread).to(x_type)
    w = b.mx4_quantize(torch.randn(M, K, device="cuda", generator=g) / math.sqrt(K))
    kw = {"bias": None if bias is None else torch.randn(M, device="cuda", generator=g).to(bias),
          "residual": None if residual is None else torch.randn(N, M // 2 if gated else M, device="cuda", generator=g).to(residual)}
    return x, w, kw


@pytest.mark.parametrize("act", [None, "relu", "silu", "gelu", "gelu_tanh"])
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("N,M,K", [(1, 1024, 4096), (3, 258, 500), (16, 20000, 512), (40, 2000, 300), (65, 258, 100), (300, 2050, 256), (1300, 4100, 300)])
@pytest.mark.parametrize("dtype", [F16, F32])
def test_activations(b, act, gated, N, M, K, dtype):
    """Every way of cutting a product: columns split over a cluster, one block a tile, pairs of SMs that walk over tiles; ragged ends of each."""
    x, w, kw = make(b, N, M, K, BF16, N + M, F32, BF16, gated)
    y = b.mx4_linear(x, w, dtype=dtype, act=act, gated=gated, **kw)
    b.mx4_check()
    check(y, b.mx4_quantize(x).dequantize(), w.dequantize(), kw["bias"], act, gated, kw["residual"])


@pytest.mark.parametrize("bias", [None, F16, BF16, F32])
@pytest.mark.parametrize("residual", [None, F16, BF16, F32])
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("N,M", [(1, 512), (20, 19456), (1024, 5120)])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_types(b, bias, residual, gated, N, M, dtype):
    x, w, kw = make(b, N, M, 256, F16, N, bias, residual, gated)
    y = b.mx4_linear(x, w, dtype=dtype, act="silu", gated=gated, **kw)
    b.mx4_check()
    check(y, b.mx4_quantize(x).dequantize(), w.dequantize(), kw["bias"], "silu", gated, kw["residual"])


@pytest.mark.parametrize("N", [1, 2, 7, 16, 17, 32, 33, 64, 65, 128, 129, 257])
@pytest.mark.parametrize("M", [1, 7, 127, 129, 19001])
def test_odd_sizes(b, N, M):
    x, w, kw = make(b, N, M, 70, F16, N * M, BF16, F16)
    y = b.mx4_linear(x, w, act="gelu_tanh", **kw)
    check(y, b.mx4_quantize(x).dequantize(), w.dequantize(), kw["bias"], "gelu_tanh", False, kw["residual"])
    x, w, kw = make(b, N, M + M % 2, 70, F16, N * M + 1, BF16, F16, True)
    y = b.mx4_linear(x, w, act=None, gated=True, **kw)
    b.mx4_check()
    check(y, b.mx4_quantize(x).dequantize(), w.dequantize(), kw["bias"], None, True, kw["residual"])


@pytest.mark.parametrize("N,M,gated", [(5, 300, False), (33, 19200, True), (1200, 4096, False), (1200, 4096, True)])
@pytest.mark.parametrize("pad", [0, 3, 8])
def test_strides_and_in_place(b, N, M, gated, pad):
    """The residual is the output itself, rows apart; columns beside stay as they were."""
    x, w, kw = make(b, N, M, 256, BF16, M + pad, F32, None, gated)
    cols = M // 2 if gated else M
    rows = torch.randn(N, cols + 2 * pad, device="cuda", generator=gen(1)).to(BF16)
    keep, view = rows.clone(), rows[:, pad:pad + cols]
    apart = b.mx4_linear(x, w, act="silu", gated=gated, bias=kw["bias"], residual=keep[:, pad:pad + cols])
    got = b.mx4_linear(x, w, out=view, act="silu", gated=gated, bias=kw["bias"], residual=view)
    b.mx4_check()
    assert got is view and torch.equal(view, apart)
    assert torch.equal(rows[:, :pad], keep[:, :pad]) and torch.equal(rows[:, pad + cols:], keep[:, pad + cols:])
    check(apart, b.mx4_quantize(x).dequantize(), w.dequantize(), kw["bias"], "silu", gated, keep[:, pad:pad + cols])


def test_without_an_epilogue_nothing_changes(b):
    for N, M in ((1, 512), (50, 19456), (1024, 5120)):
        x, w, _ = make(b, N, M, 512, F16, N)
        y = b.mx4_linear(x, w, dtype=F32)
        assert torch.equal(y, b.mx4_linear(x, w, dtype=F32, bias=torch.zeros(M, device="cuda")))
        assert torch.equal(y, b.mx4_linear(x, w, dtype=F32, residual=torch.zeros(N, M, device="cuda")))
        q = b.mx4_quantize(x)
        kw = dict(dtype=F32, act="gelu", bias=torch.ones(M, device="cuda"))
        assert torch.equal(b.mx4_linear(q, w, **kw), b.mx4_linear(x, w.freeze(), **kw))


def test_values_at_the_edges(b):
    """Large arguments of both signs; infinities and NaN stay in their places."""
    for N, M in ((2, 256), (20, 19200), (300, 20480)):
        x, w, kw = make(b, N, M, 64, F32, N, None, None, spread=40.0)
        for act in ("silu", "gelu", "gelu_tanh", "relu"):
            bias = torch.linspace(-300, 300, M, device="cuda")
            for dtype in (BF16, F32):
                y = b.mx4_linear(x, w, dtype=dtype, act=act, bias=bias)
                check(y, b.mx4_quantize(x).dequantize(), w.dequantize(), bias, act, False, None)
        res = torch.zeros(N, M, device="cuda")
        res[1, 5], res[0, 7], res[1, 100] = math.inf, -math.inf, math.nan
        y = b.mx4_linear(x, w, residual=res, act="relu")
        assert y[1, 5] == math.inf and y[0, 7] == -math.inf and bool(y[1, 100].isnan())
        clean = b.mx4_linear(x, w, act="relu")
        same = torch.isfinite(res)
        assert torch.equal(y[same], clean[same])
        x[1, 3] = math.nan
        y = b.mx4_linear(x, w, act="relu", gated=True)
        assert bool(y[1].isnan().all()) and not bool(y[0].isnan().any())


def test_graph_and_stream(b):
    for N, M in ((1, 512), (40, 19456), (1024, 5120)):
        x, w, kw = make(b, N, M, 256, F16, N, F16, F16, True)
        w.freeze()
        want = b.mx4_linear(x, w, act="silu", gated=True, **kw)
        st = torch.cuda.Stream()
        st.wait_stream(torch.cuda.current_stream())
        got = b.mx4_linear(x, w, act="silu", gated=True, stream=st.cuda_stream, **kw)
        st.synchronize()
        assert torch.equal(got, want)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):   # a residual that the kernel before writes
            r = kw["residual"] * 2
            r = b.mx4_linear(x, w, act="silu", gated=True, bias=kw["bias"], residual=r, out=r)
        for scale in (1.0, -3.0):
            base = kw["residual"].clone()
            kw["residual"].mul_(scale)
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(r, b.mx4_linear(x, w, act="silu", gated=True, bias=kw["bias"], residual=kw["residual"] * 2))
            kw["residual"].copy_(base)
    b.mx4_check()


def test_refusals(b):
    x, w, kw = make(b, 5, 31, 64, F16, 0, F16, F16)
    even = b.mx4_quantize(torch.zeros(30, 64, device="cuda"))
    for a, k in ((w, dict(act="tanh")), (w, dict(act=3)), (w, dict(gated=True)), (w, dict(bias=torch.zeros(30, device="cuda"))), (w, dict(bias=torch.zeros(31))),
                 (w, dict(bias=torch.zeros(31, device="cuda").double())), (w, dict(bias=torch.zeros(1, 31, device="cuda"))), (w, dict(bias=torch.zeros(62, device="cuda")[::2])),
                 (w, dict(residual=torch.zeros(5, 30, device="cuda"))), (w, dict(residual=torch.zeros(4, 31, device="cuda"))), (w, dict(residual=torch.zeros(5, 31))),
                 (w, dict(residual=torch.zeros(31, 5, device="cuda").t())), (even, dict(gated=True, residual=torch.zeros(5, 30, device="cuda"))),
                 (even, dict(gated=True, out=torch.zeros(5, 30, device="cuda"))), (w, dict(residual=torch.zeros(5, 31, device="cuda").int()))):
        with pytest.raises(ValueError):
            b.mx4_linear(x, a, **k)
    none = x[:0]
    assert b.mx4_linear(none, even, gated=True, act="silu").shape == (0, 15)
