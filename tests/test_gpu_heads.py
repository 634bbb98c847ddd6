"""Norms and rotation of heads on the GPU against the formula in 64 bits. The kernel's error in fp32, relative to the values of a pair together:
  * of the norm: half of the sum of squares' (D terms, none negative: D 2^-24), its root and quotient, two products: (D / 2 + 6) 2^-24;
  * of a sine or cosine: the function's 2 ulp (2^-23), its argument's rounding (below 2^-24), the frequency's 53 bits times the position (2^-51 |p f|,
    the reference's own angle included);
  * of the turn: two products and a sum, 3 2^-24;
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


def reference(x, weight, pos, freq, axis, rotary, interleaved, eps):
    """(result, bound before the last rounding) in 64 bits."""
    D = x.shape[-1]
    y = x.double()
    if weight is not None:
        y = y / (y.square().mean(-1, keepdim=True) + eps).sqrt() * weight.double()
    rel = ((D / 2 + 6) * 2.0 ** -24 if weight is not None else 0.0)
    out, bound = y.clone(), y.abs() * rel
    for i in range(rotary // 2):
        a, c = (2 * i, 2 * i + 1) if interleaved else (i, i + rotary // 2)
        t = (pos[axis[i]].double() * freq[i])[:, None]
        out[..., a] = y[..., a] * t.cos() - y[..., c] * t.sin()
        out[..., c] = y[..., c] * t.cos() + y[..., a] * t.sin()
        e = (y[..., a].abs() + y[..., c].abs()) * (rel + 2.0 ** -23 + 2.0 ** -24 + 3 * 2.0 ** -24 + 2.0 ** -51 * t.abs())
        bound[..., a] = bound[..., c] = e
    return out, bound


def check(got, ref, bound):
    assert not torch.isnan(got).any()
    lim = bound + torch.finfo(got.dtype).eps / 2 * (ref.abs() + bound) + torch.finfo(got.dtype).tiny
    d = (got.double() - ref).abs()
    assert (d <= lim).all(), f"off by {float((d / lim).max()):.2f} bounds"


def run(b, N, Hq, Hk, D, dtype, rotary=None, axes=1, interleaved=False, norm=True, first=0, base=10000.0, seed=0, frequencies=None, eps=1e-6, place=None):
    g = gen(seed)
    r = rotary or D
    n = r // 2
    sections = None if axes == 1 else [n - (axes - 1) * (n // axes)] + [n // axes] * (axes - 1)
    rot = b.Rotary(D, base=base, rotary_dim=r, interleaved=interleaved, sections=sections, frequencies=frequencies)
    freq = frequencies or [base ** (-2 * i / r) for i in range(n)]
    axis = [0] * n if axes == 1 else [a for a, k in enumerate(sections) for _ in range(k)]
    qkv = (torch.randn(N, Hq + 2 * Hk, D, device="cuda", generator=g) * 3).to(dtype)
    q, k = qkv[:, :Hq], qkv[:, Hq:Hq + Hk] if Hk else None
    if place:
        q, k = place(q), place(k)
    qw, kw = ((1 + 0.3 * torch.randn(D, device="cuda", generator=g)).to(t) for t in (dtype, F32)) if norm else (None, None)
    pos = torch.stack([first + torch.arange(N, device="cuda") * (a + 1) for a in range(axes)]).int()
    before = [x.clone() for x in (q, k) if x is not None]
    got = b.qk_norm_rope(q, k, pos[0] if axes == 1 else pos, rot, qw, kw, eps=eps)
    for x, w, y, old in zip((q, k), (qw, kw), got, before):
        assert y.shape == x.shape and y.dtype == x.dtype and y.is_contiguous() and torch.equal(x, old)
        check(y, *reference(x, w, pos, freq, axis, r, interleaved, eps))
    if k is None:
        assert got[1] is None
    return q, k, pos, rot, qw, kw, got


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
@pytest.mark.parametrize("N", [1, 2, 33, 257])
@pytest.mark.parametrize("D", [64, 80, 96, 128, 192, 256])
def test_widths(b, dtype, N, D):
    run(b, N, 8, 2, D, dtype, seed=N + D)


@pytest.mark.parametrize("D,rotary", [(2, 2), (6, 4), (30, 30), (64, 2), (80, 32), (80, 40), (100, 50), (128, 8), (128, 66), (130, 128), (254, 254), (256, 16)])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype", [F16, F32])
def test_parts(b, D, rotary, interleaved, dtype):
    run(b, 19, 5, 3, D, dtype, rotary=rotary, interleaved=interleaved, seed=D)


@pytest.mark.parametrize("Hq,Hk", [(1, 0), (1, 1), (7, 1), (64, 8), (33, 0), (3, 5), (0, 3)])
@pytest.mark.parametrize("norm", [False, True])
def test_heads(b, Hq, Hk, norm):
    run(b, 40, Hq, Hk, 128, BF16, norm=norm, seed=Hq)


@pytest.mark.parametrize("axes", [2, 3, 4])
@pytest.mark.parametrize("interleaved", [False, True])
def test_axes(b, axes, interleaved):
    run(b, 100, 6, 2, 128, BF16, axes=axes, interleaved=interleaved, first=1000)
    run(b, 100, 6, 2, 80, F32, axes=axes, rotary=40, interleaved=interleaved, first=-7)


@pytest.mark.parametrize("first", [0, -1000, 131072, 1 << 24, (1 << 31) - 200, -(1 << 31)])
def test_far_positions(b, first):
    """fp32 shows the angle itself; the bound's 2^-51 |p f| is 2^-20 at most."""
    run(b, 64, 2, 1, 64, F32, first=first, norm=False)


def test_positions_with_gaps(b):
    """Rows of a longer tensor; an axis that is the same for all."""
    rot = b.Rotary(64, sections=[16, 16])
    x = torch.randn(10, 3, 64, device="cuda", generator=gen(1))
    wide = torch.randint(-50, 5000, (2, 25), device="cuda", dtype=torch.int32, generator=gen(2))
    got, _ = b.qk_norm_rope(x, None, wide[:, 3:13], rot)
    check(got, *reference(x, None, wide[:, 3:13], [10000.0 ** (-2 * i / 64) for i in range(32)], [0] * 16 + [1] * 16, 64, False, 0))
    same = wide[:1, :10].expand(2, 10)
    got, _ = b.qk_norm_rope(x, None, same, rot)
    assert torch.equal(got, b.qk_norm_rope(x, None, wide[0, :10], b.Rotary(64))[0])


def test_pairs_in_turn(b):
    """The axis of each pair; frequencies of the caller's, zero and negative among them."""
    f = [0.0, -0.5, 7.0, 1e-3] * 8
    axis = [0, 1, 2, 1] * 8
    rot = b.Rotary(64, frequencies=f, pair_axis=axis)
    x = torch.randn(30, 4, 64, device="cuda", generator=gen(3))
    pos = torch.randint(0, 4000, (3, 30), device="cuda", dtype=torch.int32, generator=gen(4))
    got, _ = b.qk_norm_rope(x, None, pos, rot)
    check(got, *reference(x, None, pos, f, axis, 64, False, 0))


@pytest.mark.parametrize("dtype", [F16, F32])
def test_strides(b, dtype):
    """Odd strides and addresses: no row is aligned; heads outermost."""
    def odd(x):
        if x is None:
            return None
        wide = torch.zeros(x.shape[0], x.shape[1], x.shape[2] + 3, device="cuda", dtype=x.dtype)
        wide[..., 1:1 + x.shape[2]] = x
        return wide[..., 1:1 + x.shape[2]]

    run(b, 21, 4, 2, 128, dtype, place=odd)
    run(b, 21, 4, 2, 64, dtype, place=lambda x: x.transpose(0, 1).contiguous().transpose(0, 1))
    run(b, 21, 4, 2, 64, dtype, place=lambda x: torch.cat([x, x[..., :4]], -1)[..., :64])   # 8-byte rows in 16 bits


def test_in_place_and_out(b):
    q, k, pos, rot, qw, kw, (y, z) = run(b, 50, 8, 2, 128, BF16)
    rows = torch.full((50, 12, 128), 7.0, device="cuda", dtype=BF16)
    out = b.qk_norm_rope(q, k, pos[0], rot, qw, kw, q_out=rows[:, 1:9], k_out=rows[:, 10:])
    assert torch.equal(out[0], y) and torch.equal(out[1], z) and out[0].data_ptr() == rows[:, 1:9].data_ptr()
    assert bool((rows[:, 0] == 7).all()) and bool((rows[:, 9] == 7).all())
    q2, k2 = q.clone(), k.clone()
    b.qk_norm_rope(q2, k2, pos[0], rot, qw, kw, q_out=q2, k_out=k2)
    assert torch.equal(q2, y) and torch.equal(k2, z)


def test_values_at_the_edges(b):
    """Heads of zeros stay zeros; a NaN or infinity stays in its head; without a norm it stays in its pair, and behind the rotated part in its place."""
    rot = b.Rotary(128, rotary_dim=64)
    x = torch.randn(3, 4, 128, device="cuda", generator=gen(5)).half()
    pos = torch.tensor([0, 5, 9], device="cuda", dtype=torch.int32)
    w = torch.ones(128, device="cuda")
    clean, _ = b.qk_norm_rope(x, None, pos, rot, w)
    bad = x.clone()
    bad[1, 2, 3], bad[2, 0] = math.inf, 0
    got, _ = b.qk_norm_rope(bad, None, pos, rot, w)
    keep = torch.ones(3, 4, dtype=torch.bool, device="cuda")
    keep[1, 2] = keep[2, 0] = False
    assert torch.equal(got[keep], clean[keep]) and bool(got[1, 2].isnan().any()) and bool((got[2, 0] == 0).all())
    plain, _ = b.qk_norm_rope(x, None, pos, rot)
    bad = x.clone()
    bad[1, 2, 3], bad[1, 3, 100] = math.nan, math.inf
    got, _ = b.qk_norm_rope(bad, None, pos, rot)
    diff = torch.zeros_like(x, dtype=torch.bool)
    diff[1, 2, 3] = diff[1, 2, 35] = diff[1, 3, 100] = True
    assert torch.equal(got[~diff], plain[~diff]) and bool(got[1, 2, [3, 35]].isnan().all()) and got[1, 3, 100] == math.inf


def test_nothing(b):
    rot = b.Rotary(64)
    none = torch.empty(0, 4, 64, device="cuda", dtype=F16)
    q, k = b.qk_norm_rope(none, none[:, :2], torch.empty(0, device="cuda", dtype=torch.int32), rot)
    assert q.shape == (0, 4, 64) and k.shape == (0, 2, 64)


def test_graph_and_stream(b):
    q, k, pos, rot, qw, kw, (y, z) = run(b, 9, 8, 2, 128, F16)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    got = b.qk_norm_rope(q, k, pos[0], rot, qw, kw, stream=st.cuda_stream)
    st.synchronize()
    assert torch.equal(got[0], y) and torch.equal(got[1], z)
    p = pos[0].clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a, c = b.qk_norm_rope(q, k, p, rot, qw, kw)
    for shift in (0, 100):
        p.copy_(pos[0] + shift)
        graph.replay()
        want = b.qk_norm_rope(q, k, pos[0] + shift, rot, qw, kw)
        torch.cuda.synchronize()
        assert torch.equal(a, want[0]) and torch.equal(c, want[1])


def test_refusals(b):
    rot = b.Rotary(64)
    q, k = torch.zeros(5, 4, 64, device="cuda", dtype=F16), torch.zeros(5, 2, 64, device="cuda", dtype=F16)
    pos = torch.zeros(5, device="cuda", dtype=torch.int32)
    for kw in (dict(q=q.double()), dict(q=q[0]), dict(q=q[..., :32]), dict(k=k.float()), dict(k=k[:4]), dict(positions=pos.long()), dict(positions=pos[:4]),
               dict(positions=pos.cpu()), dict(positions=pos.view(1, 5).expand(2, 5)), dict(q_weight=torch.zeros(32, device="cuda")), dict(k_weight=torch.zeros(64)),
               dict(q_out=q[:, :2]), dict(q_out=q.float()), dict(q=q.transpose(1, 2).contiguous().transpose(1, 2)), dict(rotary=b.Rotary(64, sections=[16, 16])),
               dict(k=None, k_out=k), dict(q=q.cpu())):
        a = dict(q=q, k=k, positions=pos, rotary=rot)
        a.update(kw)
        with pytest.raises(ValueError):
            b.qk_norm_rope(**a)
    with pytest.raises(b.UsError):
        b.qk_norm_rope(q, k, pos, rot, eps=-1.0)
