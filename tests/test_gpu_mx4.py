"""MX4 quantisation and product on the GPU against their definitions in 64 bits.

Codes and scale bytes are decided exactly and must be equal. Products of two E2M1 values with power-of-two scales are exact in fp32; a sum of K of
them in fp32, in any order, is off by at most K 2^-23 of the sum of magnitudes (K 2^-24 for rounded additions, twice that for ones that
cut off), and the result's one rounding by half a step of its type, eps / 2."""
import subprocess
import sys
from pathlib import Path

import numpy as np
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
ROOT = Path(__file__).resolve().parent.parent
GRID = np.array([0, .5, 1, 1.5, 2, 3, 4, 6])


@pytest.fixture(scope="module")
def b():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a CUDA device")
    from paper_2608_09291_b200 import binding
    torch.cuda.set_device(0)
    return binding


def ref_mx4(x):
    """(codes (rows, K), scale bytes, values) of float64 x by the definition."""
    rows, K = x.shape
    kb = -(-K // 32)
    pad = np.zeros((rows, kb * 32))
    pad[:, :K] = x
    blk = pad.reshape(rows, kb, 32)
    a = np.abs(blk).max(-1)
    bad = ~np.isfinite(a)
    e = np.where(a > 0, np.frexp(np.where(bad, 1, a))[1] - 1 - 2, -127).clip(-127, 127)
    m = np.abs(np.where(bad[..., None], 0, blk)) / 2.0 ** e[..., None]
    code = np.zeros(m.shape, int)
    for i in range(7):                     # over the border between two codes; on it, to the even one
        mid = (GRID[i] + GRID[i + 1]) / 2
        code = np.where((m > mid) | ((m == mid) & (i % 2 == 1)), i + 1, code)
    code = np.where(np.signbit(blk) & ~bad[..., None], code + 8, code)
    val = np.where(code >= 8, -1, 1) * GRID[code % 8] * 2.0 ** e[..., None]
    val = np.where(bad[..., None], np.nan, val)
    return code.reshape(rows, -1)[:, :K], np.where(bad, 255, e + 127).astype(np.uint8), val.reshape(rows, -1)[:, :K]


def unpack(codes, K):
    c = codes.cpu().numpy()
    return np.stack([c & 15, c >> 4], -1).reshape(c.shape[0], -1)[:, :K]


def draw(rows, K, dtype, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(rows, K, device="cuda", generator=g) * torch.exp2(torch.randint(-6, 7, (rows, 1), device="cuda", generator=g).float())
    return x.to(dtype)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,K", [(1, 1), (1, 31), (2, 33), (3, 256), (129, 257), (5, 1000), (130, 2049), (7, 4100)])
def test_quantize_is_exact(b, dtype, rows, K):
    x = draw(rows, K, dtype, rows + K)
    q = b.mx4_quantize(x)
    codes, scales = q.codes()
    rc, rs, rv = ref_mx4(x.double().cpu().numpy())
    assert np.array_equal(scales.cpu().numpy(), rs)
    got = unpack(codes, K)
    assert np.array_equal(got, rc)
    assert np.array_equal(q.dequantize().cpu().numpy(), rv.astype(np.float32))
    assert np.array_equal(q.dequantize(torch.bfloat16).double().cpu().numpy(), rv)       # 2 significant bits: bfloat16 holds them
    again = b.mx4_from_codes(codes, scales, K)
    assert again.frozen and torch.equal(again.dequantize(), q.dequantize())


def test_borders_and_special_values(b):
    """Every border between codes and its neighbours, signed; zero, subnormal, huge, infinite and NaN blocks."""
    mids = (GRID[:-1] + GRID[1:]) / 2
    near = np.concatenate([mids, np.nextafter(mids.astype(np.float32), 0), np.nextafter(mids.astype(np.float32), 9), [6, 5.99, 0, -0.0]])
    rows = []
    for e in (-120, -10, 0, 3, 100):
        v = np.concatenate([near, -near])[:31] * 2.0 ** e
        rows.append(np.concatenate([[4.0 * 2.0 ** e], v]))       # the largest magnitude fixes the scale at 2^e
        rows.append(np.concatenate([[7.9 * 2.0 ** e], v[::-1]]))
    x = np.zeros((len(rows) + 6, 64), np.float32)
    x[:len(rows), :32] = np.array(rows, dtype=np.float32)
    x[:len(rows), 32:] = x[:len(rows), :32][:, ::-1]
    x[-6, 5] = 2.0 ** -149                   # subnormal
    x[-5, 3] = np.float32(3e38)
    x[-4, 40] = np.inf
    x[-3, 2] = np.nan
    x[-2, 33] = -np.inf
    rc, rs, rv = ref_mx4(x.astype(np.float64))
    q = b.mx4_quantize(torch.from_numpy(x).cuda())
    codes, scales = q.codes()
    assert np.array_equal(scales.cpu().numpy(), rs)
    finite = np.isfinite(rv)
    assert np.array_equal(unpack(codes, 64)[finite], rc[finite])
    got = q.dequantize().cpu().numpy().astype(np.float64)
    assert np.array_equal(np.isnan(got), ~finite) and np.array_equal(got[finite], rv[finite])


@pytest.mark.parametrize("dtype,off,pad", [(torch.float16, 1, 7), (torch.bfloat16, 8, 24), (torch.float32, 4, 12), (torch.float32, 3, 0)])
def test_strided_rows(b, dtype, off, pad):
    full = draw(6, 500 + off + pad, dtype, 3)
    view = full[:, off:off + 500]
    want = b.mx4_quantize(view.contiguous())
    got = b.mx4_quantize(view)
    assert torch.equal(got.dequantize(), want.dequantize())
    out = torch.full((6, 600), 7.0, device="cuda", dtype=dtype)
    got.dequantize(out=out[:, off:off + 500])
    assert torch.equal(out[:, off:off + 500], want.dequantize(dtype)) and (out[:, :off] == 7).all() and (out[:, off + 500:] == 7).all()
    reused = b.mx4_quantize(view * 0.5, out=want)
    assert reused is want and torch.equal(want.dequantize(), b.mx4_quantize(view * 0.5).dequantize())


def check_product(y, xv, wv, K):
    x, w = xv.double(), wv.double()
    ref, mag = x @ w.t(), x.abs() @ w.abs().t()
    bound = K * 2.0 ** -23 * mag + (torch.finfo(y.dtype).eps / 2) * ref.abs() + torch.finfo(y.dtype).tiny
    d = (y.double() - ref).abs()
    # (a sum that may reach the type's largest number may become an infinity of its sign, as its conversion does: float16 from 65520 on)
    d[torch.isinf(y) & (y.double().sign() == ref.sign()) & (ref.abs() + bound >= torch.finfo(y.dtype).max)] = 0
    assert (d <= bound).all(), f"off by {float((d / bound).max()):.2f} bounds"


@pytest.mark.parametrize("N", [1, 2, 7, 8, 9, 16, 17, 32, 33, 64, 65, 128, 129, 300])
@pytest.mark.parametrize("M,K", [(1, 1), (128, 256), (130, 300), (1000, 2049), (4096, 1024)])
def test_product(b, N, M, K):
    x, w = draw(N, K, torch.bfloat16, N), b.mx4_quantize(draw(M, K, torch.float32, M + 1))
    y = b.mx4_linear(x, w, dtype=torch.float32)
    q = b.mx4_quantize(x)
    b.mx4_check()
    check_product(y, q.dequantize(), w.dequantize(), K)
    assert torch.equal(y, b.mx4_linear(q, w, dtype=torch.float32))           # quantised within the call or before it
    assert torch.equal(y, b.mx4_linear(x, w.freeze(), dtype=torch.float32))
    assert torch.equal(y, b.mx4_linear(x, w, dtype=torch.float32))           # the same every time


@pytest.mark.parametrize("N,M,K", [(1, 28672, 8192), (5, 11008, 4096), (16, 1024, 28672), (1, 128, 16384), (64, 8192, 28672), (128, 256, 8192), (700, 5120, 13824), (2048, 1408, 4096)])
def test_product_large(b, N, M, K):
    x, w = draw(N, K, torch.float16, 1), b.mx4_quantize(draw(M, K, torch.bfloat16, 2)).freeze()
    y = b.mx4_linear(x, w)
    b.mx4_check()
    assert y.dtype == torch.float16
    check_product(b.mx4_linear(x, w, dtype=torch.float32), b.mx4_quantize(x).dequantize(), w.dequantize(), K)
    assert torch.equal(y, b.mx4_linear(x, w, dtype=torch.float32).half())


@pytest.mark.parametrize("xt", [torch.float16, torch.bfloat16, torch.float32])
@pytest.mark.parametrize("yt", [torch.float16, torch.bfloat16, torch.float32])
@pytest.mark.parametrize("N", [1, 3, 40, 200])
def test_types_strides_and_out(b, xt, yt, N):
    M, K = 203, 517
    full = draw(N, K + 9, xt, 5)
    x = full[:, 3:3 + K]
    w = b.mx4_quantize(draw(M, K, torch.float32, 6))
    out = torch.full((N, M + 5), 3.0, device="cuda", dtype=yt)
    y = b.mx4_linear(x, w, out=out[:, 2:2 + M])
    b.mx4_check()
    check_product(y, b.mx4_quantize(x).dequantize(), w.dequantize(), K)
    assert (out[:, :2] == 3).all() and (out[:, 2 + M:] == 3).all()
    assert torch.equal(y, b.mx4_linear(x.contiguous(), w, dtype=yt))


# enough tiles for the pairs of SMs: an odd number of row tiles, one row or one token past a tile, none for a pair's second block, several tiles a pair
@pytest.mark.parametrize("N,M,K", [(200, 18945, 300), (129, 19072, 256), (1100, 4097, 2049), (512, 20000, 513), (1153, 4224, 33), (2048, 5120, 1600)])
@pytest.mark.parametrize("yt", [torch.float16, torch.float32])
def test_many_tokens(b, N, M, K, yt):
    x, w = draw(N, K, torch.float16, N), b.mx4_quantize(draw(M, K, torch.bfloat16, M))
    q = b.mx4_quantize(x)
    out = torch.full((N + 1, M + 3), 3.0, device="cuda", dtype=yt)
    y = b.mx4_linear(q, w, out=out[:N, 1:1 + M])
    b.mx4_check()
    check_product(y, q.dequantize(), w.dequantize(), K)
    assert (out[N] == 3).all() and (out[:, 0] == 3).all() and (out[:, 1 + M:] == 3).all()
    for _ in range(3):
        assert torch.equal(y, b.mx4_linear(x, w, dtype=yt))


def test_many_tokens_on_two_streams(b):
    """Products whose pairs of SMs share the GPU with each other and with a product of few tokens, back to back and captured."""
    w = b.mx4_quantize(draw(9728, 1024, torch.float32, 1)).freeze()
    x = [draw(n, 1024, torch.float16, n) for n in (512, 1024, 5)]
    want = [b.mx4_linear(t, w) for t in x]
    streams = [torch.cuda.Stream() for _ in x]
    torch.cuda.synchronize()
    got = []
    for _ in range(10):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got.append((i, b.mx4_linear(x[i], w)))
    torch.cuda.synchronize()
    b.mx4_check()
    assert all(torch.equal(y, want[i]) for i, y in got)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        y = [b.mx4_linear(t, w) for t in x]
    for _ in range(3):
        g.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, c) for a, c in zip(y, want))
    del g


def test_nan_stays_in_its_row_and_column(b):
    x, w = draw(20, 600, torch.float32, 7), draw(300, 600, torch.float32, 8)
    x[3, 599] = float("nan")
    w[250, 10] = float("inf")
    y = b.mx4_linear(x, b.mx4_quantize(w), dtype=torch.float32)
    nan = torch.isnan(y)
    assert nan[3].all() and nan[:, 250].all() and int(nan.sum()) == 300 + 20 - 1


def test_empty(b):
    w = b.mx4_quantize(draw(10, 40, torch.float32, 9))
    x = torch.empty(0, 40, device="cuda", dtype=torch.float16)
    assert b.mx4_linear(x, w).shape == (0, 10)
    q = b.mx4_quantize(x)
    assert (q.rows, q.K) == (0, 40) and q.dequantize().shape == (0, 40) and b.mx4_linear(q, w).shape == (0, 10)


def test_refusals(b):
    x, w = draw(4, 64, torch.float16, 1), b.mx4_quantize(draw(8, 64, torch.float32, 2))
    for bad in (x.t(), x[:, ::2], x.double(), x[0], x[:, :60]):
        with pytest.raises(ValueError):
            b.mx4_linear(bad, w)
    with pytest.raises(ValueError):
        b.mx4_linear(x, w, out=torch.empty(4, 9, device="cuda", dtype=torch.float16))
    with pytest.raises(ValueError):
        b.mx4_linear(x, w, dtype=torch.float64)
    with pytest.raises(ValueError):
        b.mx4_linear(b.mx4_quantize(x[:, :32]), w)
    with pytest.raises(ValueError):
        b.mx4_quantize(x, out=w)
    with pytest.raises(ValueError):
        b.mx4_quantize(w.dequantize(), out=b.mx4_from_codes(*w.codes(), 64))      # frozen
    with pytest.raises(ValueError):
        b.mx4_from_codes(torch.zeros(4, 30, device="cuda", dtype=torch.uint8), torch.zeros(4, 2, device="cuda", dtype=torch.uint8), 64)


def test_another_stream_and_graph(b):
    """On a stream that the caller names or has made current, and captured: new activations in the same place give the new product."""
    w = b.mx4_quantize(draw(512, 2048, torch.float32, 3)).freeze()
    for N in (1, 16, 100, 400):
        x = draw(N, 2048, torch.float16, N)
        want = b.mx4_linear(x, w)
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            a = b.mx4_linear(x, w)
        c = b.mx4_linear(x, w, stream=s.cuda_stream)
        s.synchronize()
        assert torch.equal(a, want) and torch.equal(c, want)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            y = b.mx4_linear(x, w)
            z = b.mx4_linear(b.mx4_quantize(x), w, dtype=torch.float32)
        for seed in (11, 12):
            x.copy_(draw(N, 2048, torch.float16, seed))
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(y, b.mx4_linear(x, w)) and torch.equal(z, b.mx4_linear(x, w, dtype=torch.float32))
        del g


def test_two_streams_at_once(b):
    w = [b.mx4_quantize(draw(1024, 4096, torch.float32, i)).freeze() for i in (1, 2)]
    x = [draw(n, 4096, torch.float16, n) for n in (3, 50)]
    want = [b.mx4_linear(x[i], w[i]) for i in (0, 1)]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(20):
        for i in (0, 1):
            with torch.cuda.stream(streams[i]):
                got[i].append(b.mx4_linear(x[i], w[i]))
    torch.cuda.synchronize()
    b.mx4_check()
    for i in (0, 1):
        assert all(torch.equal(y, want[i]) for y in got[i])


def test_beside_the_sparse_product(b):
    """Sparse and dense products in turn on one stream: each leaves the other's results as they are."""
    from paper_2608_09291_b200 import workloads
    W = workloads.make_weight(1024, 1024, 0.5, seed=1)
    s_w, _ = workloads.make_scales(1024, 1, seed=1)
    sw = b.SparseWeight(W, s_w, max_N=16)
    x = torch.from_numpy(workloads.make_x_f16(1024, 16, seed=2)).cuda()
    w = b.mx4_quantize(draw(1024, 1024, torch.float32, 4)).freeze()
    y0 = sw.spmm_requant(x, 16, b.absmax_f16(x))
    z0 = b.mx4_linear(y0, w)
    torch.cuda.synchronize()
    for _ in range(10):
        y = sw.spmm_requant(x, 16, b.absmax_f16(x))
        z = b.mx4_linear(y, w)
        assert torch.equal(y, y0) and torch.equal(z, z0)
    sw.check()
    b.mx4_check()
    sw.close()
