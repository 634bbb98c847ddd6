"""Entry points of the cache's blocks and of the heads' rotation on the host: refusals and sizes. No call here reaches a kernel."""
import ctypes
import math

import pytest

INVALID, TOO_SMALL = 1, 8
P = 1 << 20


@pytest.fixture(scope="module")
def b():
    from paper_2608_09291_b200 import binding
    return binding


@pytest.fixture()
def h(b):
    handle = b.us_kv_create(P, P, P, P, 100, 2, 64, 128)
    yield handle
    assert b._lib.us_kv_destroy(handle) == 0


def _fork(b, h, refs=P, seqs=True, parents=P, n=3, table=P, stride=10, lengths=P, keep=0, **kw):
    a = dict(block_table=P, table_stride=10, lengths=P, cu_tokens=None, n_seqs=3, table_width=10)
    a.update(kw)
    q = b.us_kv_seqs(**a)
    return b._lib.us_kv_fork(h, refs, ctypes.byref(q) if seqs else None, parents, n, table, stride, lengths, keep, None)


@pytest.mark.parametrize("kw", [dict(refs=None), dict(refs=P + 4), dict(seqs=False), dict(parents=None), dict(n=-1), dict(table=None), dict(stride=9), dict(lengths=None), dict(parents=P + 1),
                                dict(table=P + 2), dict(lengths=P + 3), dict(block_table=None), dict(n_seqs=-1), dict(table_width=0), dict(table_width=1 << 25), dict(table_stride=9)])
def test_fork_refuses(b, h, kw):
    assert _fork(b, h, **kw) == INVALID


def _extend(b, h, refs=P, table=P, stride=10, width=10, lengths=P, n=3, tokens=None, each=1, scratch=P, size=1 << 30):
    return b._lib.us_kv_extend(h, refs, table, stride, width, lengths, n, tokens, each, scratch, size, None)


@pytest.mark.parametrize("kw,st", [(dict(refs=None), INVALID), (dict(refs=P + 8), INVALID), (dict(table=None), INVALID), (dict(stride=9), INVALID), (dict(width=0), INVALID),
                                   (dict(lengths=None), INVALID), (dict(n=-1), INVALID), (dict(each=-1), INVALID), (dict(tokens=P + 2), INVALID), (dict(lengths=P + 1), INVALID),
                                   (dict(scratch=None), TOO_SMALL), (dict(scratch=P + 8), TOO_SMALL), (dict(size=100), TOO_SMALL)])
def test_extend_refuses(b, h, kw, st):
    assert _extend(b, h, **kw) == st


def test_other_refusals(b, h):
    lib = b._lib
    q = b.us_kv_seqs(block_table=P, table_stride=10, lengths=P, cu_tokens=None, n_seqs=3, table_width=10)
    assert lib.us_kv_release(h, None, ctypes.byref(q), None) == INVALID and lib.us_kv_release(h, P, None, None) == INVALID and lib.us_kv_release(None, P, ctypes.byref(q), None) == INVALID
    q = ctypes.byref(q)
    bad = ctypes.byref(b.us_kv_seqs(block_table=P, table_stride=9, lengths=P, cu_tokens=None, n_seqs=3, table_width=10))
    for a in ((None, q, 1, P, P, P, 1 << 30), (P + 4, q, 1, P, P, P, 1 << 30), (P, None, 1, P, P, P, 1 << 30), (P, q, -1, P, P, P, 1 << 30), (P, bad, 1, P, P, P, 1 << 30),
              (P, q, 1, None, P, P, 1 << 30), (P, q, 1, P, None, P, 1 << 30), (P, q, 1, P, P + 1, P, 1 << 30)):
        assert lib.us_kv_compact(h, *a, None) == INVALID
    for a in ((P, q, 1, P, P, None, 1 << 30), (P, None, 0, P, P, P, 800), (P, q, 1, P, P, P + 4, 1 << 30)):
        assert lib.us_kv_compact(h, *a, None) == TOO_SMALL
    assert lib.us_kv_remap(h, None, q, None) == INVALID and lib.us_kv_remap(h, P, bad, None) == INVALID and lib.us_kv_remap(h, P, None, None) == INVALID
    for a in ((None, P, 1), (P, None, 1), (P, P, -1), (P + 2, P, 1), (P, P, 1 << 31)):
        assert lib.us_kv_copy_blocks(h, *a, None) == INVALID
    assert lib.us_kv_copy_blocks(None, P, P, 1, None) == INVALID and lib.us_kv_copy_blocks(h, None, None, 0, None) == 0
    assert _fork(b, None) == INVALID and _extend(b, None) == INVALID and lib.us_kv_compact(None, P, None, 0, P, P, P, 1 << 30, None) == INVALID
    assert lib.us_kv_extend_scratch(None, 1) == -1 and lib.us_kv_extend_scratch(h, -1) == -1 and lib.us_kv_extend_scratch(h, 5) >= 4 * 5
    assert lib.us_kv_compact_scratch(None) == -1 and lib.us_kv_compact_scratch(h) >= 800
    assert "free blocks" in b.us_status_string(10)


def _rope(b, N=5, D=128, t=0, eps=1e-6, positions=P, axis_stride=5, rotary=True, q=True, k=True, rot=None, qh=None):
    r = dict(turns=P, axis=None, rotary_dim=128, axes=1, interleaved=0)
    r.update(rot or {})
    heads = dict(x=P, token_stride=1024, head_stride=128, out=P, out_token_stride=1024, out_head_stride=128, weight=P, weight_type=0, heads=8)
    a, c = b.us_heads(**{**heads, **(qh or {})}), b.us_heads(**heads)
    return b._lib.us_qk_norm_rope(ctypes.byref(b.us_rotary(**r)) if rotary else None, positions, axis_stride, N, D, t, ctypes.byref(a) if q else None,
                                  ctypes.byref(c) if k else None, eps, None)


@pytest.mark.parametrize("kw", [dict(rotary=False), dict(q=False), dict(N=-1), dict(N=1 << 31), dict(D=127), dict(D=258), dict(D=64), dict(D=0), dict(t=3), dict(t=-1), dict(eps=-1.0),
                                dict(eps=math.nan), dict(positions=None), dict(positions=P + 2), dict(rot=dict(turns=None)), dict(rot=dict(turns=P + 4)), dict(rot=dict(rotary_dim=0)),
                                dict(rot=dict(rotary_dim=3)), dict(rot=dict(rotary_dim=130)), dict(rot=dict(axes=0)), dict(rot=dict(axes=2)), dict(rot=dict(axes=256, axis=P)),
                                dict(rot=dict(axes=2, axis=P), axis_stride=-1), dict(qh=dict(x=None)), dict(qh=dict(out=None)), dict(qh=dict(x=P + 1)), dict(qh=dict(weight=P + 1)),
                                dict(qh=dict(weight_type=3)), dict(qh=dict(token_stride=127)), dict(qh=dict(out_head_stride=100)), dict(qh=dict(heads=-1)), dict(qh=dict(heads=70000)),
                                dict(qh=dict(head_stride=-128)), dict(t=2, qh=dict(out=P + 2))])
def test_heads_refuse(b, kw):
    assert _rope(b, **kw) == INVALID


def test_heads_nothing_to_do(b):
    assert _rope(b, N=0, positions=None, qh=dict(x=None, out=None)) == 0
    assert _rope(b, k=False, qh=dict(heads=0, x=None, out=None), positions=None) == 0


def test_rotary_tables(b):
    torch = pytest.importorskip("torch")
    r = b.Rotary(64, base=10000.0, device="cpu")
    turns = [int(x) % (1 << 64) for x in r.turns.tolist()]
    for i, t in enumerate(turns):   # the frequency's 53 bits
        assert abs(t / 2.0 ** 64 - 10000.0 ** (-2 * i / 64) / (2 * math.pi)) <= 2.0 ** -52
    assert r.pair_axis is None and r.axes == 1 and r.rotary_dim == 64
    s = b.Rotary(64, sections=[8, 12, 12], device="cpu")
    assert s.pair_axis.tolist() == [0] * 8 + [1] * 12 + [2] * 12 and s.axes == 3 and torch.equal(s.turns, r.turns)
    n = b.Rotary(8, frequencies=[0.0, -1.0, 1.0, 2 * math.pi * 3.25], device="cpu")
    v = [int(x) % (1 << 64) for x in n.turns.tolist()]
    assert v[0] == 0 and (v[1] + v[2]) % (1 << 64) == 0 and abs(v[3] / 2.0 ** 64 - 0.25) < 1e-14
    for kw in (dict(head_dim=63), dict(head_dim=258), dict(head_dim=0), dict(head_dim=64, rotary_dim=65), dict(head_dim=64, rotary_dim=66), dict(head_dim=64, rotary_dim=0),
               dict(head_dim=64, sections=[16, 15]), dict(head_dim=64, sections=[33, -1]), dict(head_dim=64, pair_axis=[0] * 31), dict(head_dim=64, pair_axis=[-1] + [0] * 31),
               dict(head_dim=64, sections=[16, 16], pair_axis=[0] * 32), dict(head_dim=64, frequencies=[1.0] * 31), dict(head_dim=64, frequencies=[math.inf] * 32)):
        with pytest.raises(ValueError):
            b.Rotary(device="cpu", **kw)


def _product(b, N=4, M=64, K=64, e=None, ldy=64, linear=True, y=P, **kw):
    a = dict(bias=P, residual=P, ldr=64, bias_type=0, residual_type=0, act=2, gated=0)
    a.update(kw)
    s = b.us_mx4_epilogue(**a)
    if linear:
        return b._lib.us_mx4_linear_epilogue(P, 0, K, N, P, M, K, ctypes.byref(s), y, 0, ldy, P, 1 << 40, 0, None)
    return b._lib.us_mx4_matmul_epilogue(P, N, P, M, K, ctypes.byref(s), y, 0, ldy, 0, None)


@pytest.mark.parametrize("linear", [False, True])
@pytest.mark.parametrize("kw", [dict(act=-1), dict(act=5), dict(bias_type=3), dict(bias=P + 1), dict(residual_type=-1), dict(residual=P + 1), dict(residual_type=2, residual=P + 2), dict(ldr=63),
                                dict(gated=1, M=63), dict(gated=1, ldr=31), dict(gated=1, ldy=31), dict(ldy=63), dict(y=None), dict(M=0), dict(N=-1)])
def test_epilogue_refuses(b, linear, kw):
    assert _product(b, linear=linear, **kw) == INVALID


def test_epilogue_nothing_to_do(b):
    assert _product(b, N=0, y=None) == 0 and _product(b, N=0, y=None, linear=False) == 0


def _shared(b, h, prefixes=True, seqs=True, N=3, Q=P, t=0, heads=8, qt=1024, scale=0.1, out=P, scratch=P, size=1 << 40, pre=None, **kw):
    a = dict(block_table=P, table_stride=10, lengths=P, cu_tokens=None, n_seqs=3, table_width=10)
    a.update(kw)
    c = dict(block_table=P, table_stride=10, lengths=P, cu_tokens=P, n_seqs=2, table_width=10)
    c.update(pre or {})
    s, p = ctypes.byref(b.us_kv_seqs(**a)) if seqs else None, ctypes.byref(b.us_kv_seqs(**c)) if prefixes else None
    return (b._lib.us_kv_shared_attention(h, p, s, N, Q, t, heads, qt, 128, scale, 1, out, 1024, 128, None, scratch, size, None),
            b._lib.us_kv_shared_attention_scratch(h, p, s, N, heads))


@pytest.mark.parametrize("kw", [dict(prefixes=False), dict(seqs=False), dict(pre=dict(cu_tokens=None)), dict(pre=dict(cu_tokens=P + 1)), dict(pre=dict(n_seqs=-1)), dict(pre=dict(block_table=None)),
                                dict(pre=dict(lengths=None)), dict(pre=dict(table_width=0)), dict(pre=dict(table_stride=3)), dict(pre=dict(table_width=1 << 25)), dict(n_seqs=4), dict(heads=7),
                                dict(heads=0), dict(block_table=None), dict(N=-1)])
def test_shared_attention_refuses(b, h, kw):
    assert _shared(b, h, **kw) == (INVALID, -1)


@pytest.mark.parametrize("kw,st", [(dict(Q=None), INVALID), (dict(out=None), INVALID), (dict(t=2), 4), (dict(t=5), INVALID), (dict(qt=100), INVALID), (dict(scale=math.nan), INVALID),
                                   (dict(scratch=None), TOO_SMALL), (dict(scratch=P + 4), TOO_SMALL), (dict(size=3 * 8 * 132 * 4), TOO_SMALL)])
def test_shared_attention_refuses_data(b, h, kw, st):
    got, need = _shared(b, h, **kw)
    assert got == st and need > 3 * 8 * 130 * 4


def test_shared_attention_nothing_to_do(b, h):
    assert _shared(b, h, N=0, n_seqs=0, block_table=None, lengths=None, Q=None, out=None, scratch=None, size=0) == (0, 0)
    assert _shared(b, None) == (INVALID, -1)
