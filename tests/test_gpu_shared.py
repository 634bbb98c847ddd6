"""Attention behind shared prefixes on the GPU against the softmax over prefix and own tokens in 64 bits.

The error is that of attention over one context of both (tests/test_gpu_kv.py): of the scores |ds| <= (D + 4) 2^-23 |scale| sum_d |q_d k_d|, p changes by e^(2 ds);
p's rounding to 11 bits, 2^-11 + 2^-19 of p |v|; what lies below the smallest normal fp16 number, 2^-31 127 max(p step) a token seen, of each of the two
parts, relative to the largest of its own; sums in fp32, at most 2^-23 of the magnitudes an addition, one in 16 tokens and 64 to join parts; the join of the two itself, four
roundings and an exponential each: 2^-20. Then the result's rounding, eps / 2."""
import math

import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

F16, BF16 = torch.float16, torch.bfloat16


@pytest.fixture(scope="module")
def b():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a CUDA device")
    from paper_2608_09291_b200 import binding
    torch.cuda.set_device(0)
    return binding


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def sums(v):
    return ints([0] + torch.tensor(v).cumsum(0).tolist())


def make(b, prefix, own, Hkv, D, T, seed, widths=(None, None), spread=0.5, rest=64.0):
    """A cache with these prefixes and own parts on blocks in any order; blocks of nobody hold NaN steps, unused table entries rubbish. rest: one over the own steps' size."""
    g = gen(seed)
    per = [-(-n // T) for n in prefix + own]
    blocks = sum(per) + 3
    order = torch.randperm(blocks, device="cuda", generator=g).int()
    steps = [torch.full((blocks, Hkv), float("nan"), device="cuda") for _ in range(2)]
    tables, at = [], 0
    for which, (lens, width) in enumerate(zip((prefix, own), widths)):
        t = torch.full((len(lens), max([1, width or 0] + [-(-n // T) for n in lens])), -7, dtype=torch.int32, device="cuda")
        for s, n in enumerate(lens):
            k = -(-n // T)
            t[s, :k] = order[at:at + k]
            for x in steps:
                x[order[at:at + k].long()] = torch.exp2((torch.rand(k, Hkv, device="cuda", generator=g) - 0.5) * 2 * spread) / (32 if which == 0 else rest)
            at += k
        tables.append(t)
    codes = [(torch.randn(blocks, Hkv, T, D, device="cuda", generator=g) * 32).round().clamp(-127, 127).to(torch.int8) for _ in range(2)]
    return b.KVCache(codes[0], codes[1], steps[0], steps[1]), tables[0], tables[1]


def values(cache, row, n):
    """K, V and V's steps of a row's first n tokens in 64 bits: (n, Hkv, D) twice, (n, Hkv)."""
    T = cache.block_tokens
    ids = row[:-(-n // T)].long()
    kv = [(c[ids].double() * st[ids].double()[..., None, None]).transpose(1, 2).flatten(0, 1)[:n]
          for c, st in ((cache.k_codes, cache.k_steps), (cache.v_codes, cache.v_steps))]
    return (*kv, cache.v_steps[ids].double().repeat_interleave(T, 0)[:n])


def reference(cache, ptable, prefix, group, table, own, new, q, scale, causal=True):
    """(out, bound before the last rounding, lse); group: of each sequence, or None."""
    Hq, D = q.shape[1:]
    outs, bounds, lses, at = [], [], [], 0
    for s, (L, n) in enumerate(zip(own, new)):
        x = q[at:at + n].double()
        at += n
        if L == 0 or n == 0:
            outs.append(torch.zeros_like(x)); bounds.append(torch.zeros_like(x)); lses.append(torch.full((n, Hq), -math.inf, device="cuda", dtype=torch.float64))
            continue
        P = 0 if group[s] is None else prefix[group[s]]
        parts = [values(cache, table[s], L)]
        if P:
            parts.insert(0, values(cache, ptable[group[s]], P))
        rep = Hq // cache.n_kv_heads
        k, v, step = (torch.cat(t).repeat_interleave(rep, 1) for t in zip(*parts))
        t, pos = torch.arange(P + L, device="cuda"), torch.arange(P + L - n, P + L, device="cuda")[:, None]
        seen = (t <= pos) if causal else torch.ones(n, P + L, dtype=torch.bool, device="cuda")
        a = (torch.einsum("nhd,lhd->hnl", x, k) * scale).masked_fill(~seen, -math.inf)
        mag = torch.einsum("nhd,lhd->hnl", x.abs(), k.abs()) * abs(scale)
        p = torch.softmax(a, -1)
        ds = (D + 4) * 2.0 ** -23 * mag.masked_fill(~seen, 0).amax(-1)
        rel = torch.expm1(2 * ds) + 2.0 ** -11 + 2.0 ** -19 + 2.0 ** -20 + 2 * ((P + L) / 16 + 64) * 2.0 ** -23
        low = 0
        for lo, hi in ((0, P), (P, P + L)):
            if hi > lo:
                low = low + 2.0 ** -31 * 127 * seen[:, lo:hi].sum(-1) * (p * step.t()[:, None])[..., lo:hi].amax(-1)
        outs.append(torch.einsum("hnl,lhd->nhd", p, v))
        bounds.append(rel.t()[..., None] * torch.einsum("hnl,lhd->nhd", p, v.abs()) + low.t()[..., None])
        lses.append(torch.logsumexp(a, -1).t())
    return torch.cat(outs), torch.cat(bounds), torch.cat(lses)


def check(got, ref, bound):
    assert not torch.isnan(got).any()
    lim = bound + torch.finfo(got.dtype).eps / 2 * (ref.abs() + bound) + torch.finfo(got.dtype).tiny
    d = (got.double() - ref).abs()
    assert (d <= lim).all(), f"off by {float((d / lim.clamp(min=1e-300)).max()):.2f} bounds"


def run(b, prefix, count, own, new, G, Hkv, D, T, dtype, seed=0, causal=True, scale=None, widths=(None, None), first=0, **kw):
    """first: sequences in front of the first group's."""
    cache, ptable, table = make(b, prefix, own, Hkv, D, T, seed, widths, **kw)
    group = [None] * first + [g for g, n in enumerate(count) for _ in range(n)]
    group += [None] * (len(own) - len(group))
    q = torch.randn(sum(new), G * Hkv, D, device="cuda", generator=gen(seed + 1)).to(dtype)
    lse = torch.full((sum(new), G * Hkv), 5.0, device="cuda")
    single = all(n == 1 for n in new)
    args = (q, ptable, ints(prefix), sums(count) + first, table, ints(own), None if single else sums(new))
    out = cache.shared_attention(*args, scale=scale, causal=causal, lse=lse)
    cache.check()
    ref, bound, rl = reference(cache, ptable, prefix, group, table, own, new, q, D ** -0.5 if scale is None else scale, causal)
    check(out, ref, bound)
    seen = torch.isfinite(rl)
    assert torch.equal(torch.isfinite(lse), seen)
    assert (lse.double() - rl)[seen].abs().le(1e-5 * (1 + rl[seen].abs()) + 1e-4).all()
    return cache, args, out, lse, (ref, bound)


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("D,T", [(128, 64), (64, 16), (128, 16), (64, 256)])
@pytest.mark.parametrize("G", [1, 4, 8, 9])
@pytest.mark.parametrize("P", [1, 16, 129, 1000])
def test_one_group(b, dtype, D, T, G, P):
    """Rows of the group below and above what one kernel takes."""
    run(b, [P], [5], [1, 7, 64, 65, 200], [1] * 5, G, 2, D, T, dtype, seed=P + G)


@pytest.mark.parametrize("G,Hkv", [(1, 4), (8, 2)])
@pytest.mark.parametrize("count,prefix", [([3, 1, 4], [300, 0, 17]), ([0, 8], [500, 130]), ([1] * 8, [1, 2, 64, 127, 128, 129, 255, 700]), ([2, 0, 0, 6], [40, 40, 40, 1]), ([8], [0])])
@pytest.mark.parametrize("wide", [None, 400])
def test_groups(b, G, Hkv, count, prefix, wide):
    """Empty prefixes and groups; tables that are wide enough for walks to be cut."""
    run(b, prefix, count, [3, 64, 1, 100, 17, 129, 500, 2], [1] * 8, G, Hkv, 128, 16, F16, seed=len(count), widths=(wide, wide))


@pytest.mark.parametrize("new", [[2, 1, 3, 1], [40, 1, 17, 5], [100, 60, 0, 70], [300, 1, 1, 200]])
@pytest.mark.parametrize("G", [1, 8])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("wide", [None, 300])
def test_several_new_tokens(b, new, G, causal, wide):
    run(b, [333, 90], [3, 1], [max(1, n) + 30 * i for i, n in enumerate(new)], new, G, 2, 128, 32, BF16, seed=sum(new), causal=causal, widths=(wide, wide))


@pytest.mark.parametrize("new", [1, 20, 150])
@pytest.mark.parametrize("D", [64, 128])
def test_sequences_without_a_prefix_and_padded_ones(b, new, D):
    """In front of the groups, behind them; sequences of length 0 with rows, in groups and not."""
    own = [200, 0, 210, 0, 300, 250, 0]
    run(b, [150, 70], [2, 2], own, [new] * 7, 4, 2, D, 16, F16, first=1, seed=new)


@pytest.mark.parametrize("P,S,G,Hkv,D", [(8192, 64, 8, 2, 128), (16000, 20, 1, 4, 64), (5000, 300, 2, 1, 128), (20000, 2, 4, 2, 128)])
def test_long_prefixes(b, P, S, G, Hkv, D):
    run(b, [P], [S], [1 + (37 * i) % 300 for i in range(S)], [1] * S, G, Hkv, D, 64, BF16, seed=2)


@pytest.mark.parametrize("scale", [0.0, -0.1, 1.0])
@pytest.mark.parametrize("new", [1, 40])
def test_scale(b, scale, new):
    run(b, [500], [3], [60, 50, 70], [new] * 3, 4, 2, 128, 64, F16, scale=scale, seed=new)


@pytest.mark.parametrize("new,S", [(1, 4), (1, 40), (50, 3)])
@pytest.mark.parametrize("rest", [64.0, 2.0 ** 25, 2.0 ** -14])
def test_parts_of_different_size(b, new, S, rest):
    """Own values 2^20 smaller or larger than the prefix's."""
    cache, args, out, lse, _ = run(b, [300], [S], [100] * S, [new] * S, 2, 2, 128, 16, BF16, seed=S, rest=32.0)
    k = cache.k_steps.clone()
    own = args[4].flatten().unique()
    own = own[own >= 0].long()
    cache.v_steps[own] *= 32 / rest
    q, ptable, _, _, table, _, cu = args
    got = cache.shared_attention(*args)
    cache.check()
    ref, bound, _ = reference(cache, ptable, [300], [0] * S, table, [100] * S, [new] * S, q, 128 ** -0.5)
    check(got, ref, bound)
    assert torch.equal(cache.k_steps.nan_to_num(0), k.nan_to_num(0))


@pytest.mark.parametrize("new", [1, 60])
def test_one_part_without_weight(b, new):
    """Scores of one of the parts lie far below the other's."""
    for which in (0, 1):
        cache, args, _, _, _ = run(b, [100], [2], [80, 90], [new] * 2, 1, 1, 64, 16, F16, seed=3)
        q, ptable, _, _, table, _, _ = args
        q[..., 0] = 4
        t = (ptable if which == 0 else table).flatten()
        ids = t[t >= 0].long()
        cache.k_codes[ids] = 0
        cache.k_codes[ids, :, :, 0] = -127
        cache.k_steps[ids] = 2.0
        got = cache.shared_attention(*args)
        ref, bound, _ = reference(cache, ptable, [100], [0, 0], table, [80, 90], [new] * 2, q, 64 ** -0.5)
        check(got, ref, bound)


@pytest.mark.parametrize("new,S", [(1, 4), (1, 50), (40, 6)])
@pytest.mark.parametrize("wide", [None, 200])
def test_nan_stays_in_its_rows(b, new, S, wide):
    half = S // 2
    cache, args, want, _, _ = run(b, [300, 200], [half, S - half], [130] * S, [new] * S, 4, 2, 128, 16, F16, seed=7, widths=(wide, wide))
    q, ptable, plen, cu_seqs, table, lengths, cu = args
    bad = q.clone()
    bad[1, 3, 7] = math.nan
    got = cache.shared_attention(bad, *args[1:])
    hit = torch.zeros(S * new, 8, dtype=torch.bool, device="cuda")
    hit[1, 3] = True
    assert torch.isnan(got[hit]).all() and torch.equal(got[~hit], want[~hit])
    cache.v_steps[table[S - 1, 2].long(), 0] = math.nan        # of one sequence's own tokens, seen by all its rows
    got = cache.shared_attention(*args)
    assert torch.equal(got[:(S - 1) * new], want[:(S - 1) * new]) and torch.isnan(got[(S - 1) * new:, :4]).all() and torch.equal(got[(S - 1) * new:, 4:], want[(S - 1) * new:, 4:])
    cache.v_steps[ptable[0, 3].long(), 1] = math.nan           # of a prefix: its group
    got = cache.shared_attention(*args)
    assert torch.isnan(got[:half * new, 4:]).all() and torch.equal(got[:half * new, :4], want[:half * new, :4])
    assert torch.equal(got[half * new:(S - 1) * new], want[half * new:(S - 1) * new])


def test_without_prefixes_it_is_attention(b):
    cache, args, out, _, (ref, bound) = run(b, [0], [3], [100, 5, 64], [1] * 3, 4, 2, 128, 64, F16)
    q, _, _, _, table, lengths, _ = args
    want = cache.attention(q, table, lengths)
    none = torch.zeros(0, 1, dtype=torch.int32, device="cuda")
    assert torch.equal(cache.shared_attention(q, none, ints([]), ints([0]), table, lengths), want)
    # (an empty prefix: the same sums, which another kernel may add in another order; each side is within the bound, and so they are within two of each other)
    check(want, ref, bound)
    check(out, ref, bound)


def test_after_a_fork(b):
    """One table of prompt and own tokens, cut into two views; each is as exact against both."""
    H, D, T = 2, 128, 64
    g = gen(5)
    cache = b.KVCache.new(64, H, D, T)
    pages = b.KVPages(cache)
    table, lengths = torch.zeros(1, 8, dtype=torch.int32, device="cuda"), ints([0])
    pages.extend(table, lengths, 3 * T + 20)
    cache.append(*(torch.randn(3 * T + 20, H, D, device="cuda", generator=g).half() for _ in range(2)), table, lengths, ints([0, 3 * T + 20]))
    table, lengths = pages.fork(table, lengths, ints([0] * 5))
    for _ in range(3):
        pages.extend(table, lengths)
        cache.append(*(torch.randn(5, H, D, device="cuda", generator=g).half() for _ in range(2)), table, lengths)
    q = torch.randn(5, 8, D, device="cuda", generator=g).half()
    out = cache.shared_attention(q, table[:1, :3], ints([3 * T]), ints([0, 5]), table[:, 3:], lengths - 3 * T)
    pages.check()
    ref, bound, _ = reference(cache, table[:, :3], [3 * T], [0] * 5, table[:, 3:], [23] * 5, [1] * 5, q, D ** -0.5)
    check(out, ref, bound)
    check(cache.attention(q, table, lengths), ref, bound)


def test_strides_and_out(b):
    cache, args, want, lse, _ = run(b, [200], [6], [70] * 6, [1] * 6, 8, 2, 128, 16, F16)
    q = args[0]
    wide = torch.full((6, 33, 131), 7.0, device="cuda", dtype=F16)
    wide[:, 1:17, 1:129] = q
    out = wide[:, 17:, 2:130]
    got = cache.shared_attention(wide[:, 1:17, 1:129], *args[1:], out=out)
    assert got is out and torch.equal(out, want) and bool((wide[:, 17:, :2] == 7).all()) and bool((wide[:, 17:, 130:] == 7).all())
    # rows behind the last sequence are left as they are
    more = torch.cat([q, q])
    out = torch.full_like(more, 3.0)
    l2 = torch.full((12, 16), 4.0, device="cuda")
    cache.shared_attention(more, *args[1:6], sums([1] * 6), out=out, lse=l2)
    cache.check()
    assert torch.equal(out[:6], want) and bool((out[6:] == 3).all()) and bool((l2[6:] == 4).all())


def test_graph_streams_and_two_calls(b):
    cache, args, want, _, _ = run(b, [900], [40], [70] * 40, [1] * 40, 8, 2, 128, 16, BF16)
    c2, a2, w2, _, _ = run(b, [400, 300], [2, 2], [70] * 4, [3] * 4, 1, 2, 64, 16, F16, seed=4)
    st = [torch.cuda.Stream() for _ in range(2)]
    graphs, outs = [], []
    for cache_, a_ in ((cache, args), (c2, a2)):
        q = a_[0].clone()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(cache_.shared_attention(q, *a_[1:]))
        graphs.append((graph, q))
    for k in (1.0, -0.5):
        for (graph, q), a_ in zip(graphs, (args, a2)):
            q.copy_(a_[0] * k)
        torch.cuda.synchronize()
        for s, (graph, _) in zip(st, graphs):
            with torch.cuda.stream(s):
                for _ in range(10):
                    graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(outs[0], cache.shared_attention(args[0] * k, *args[1:])) and torch.equal(outs[1], c2.shared_attention(a2[0] * k, *a2[1:]))
    got = []
    for _ in range(10):
        for s, cache_, a_ in ((st[0], cache, args), (st[1], c2, a2)):
            got.append(cache_.shared_attention(*a_, stream=s.cuda_stream))
    torch.cuda.synchronize()
    assert all(torch.equal(x, want) for x in got[0::2]) and all(torch.equal(x, w2) for x in got[1::2])
    cache.check()


@pytest.mark.parametrize("G", [1, 16])
def test_numbers_out_of_range(b, G):
    """They are reported, and nothing outside the arrays is touched; sequences that are right come out right where groups are."""
    cache, args, want, _, _ = run(b, [100, 90], [2, 2], [50] * 4, [1] * 4, G, 2, 128, 16, F16)
    q, ptable, plen, cu_seqs, table, lengths, _ = args
    broken = [cu_seqs.clone() for _ in range(3)]
    broken[0][1], broken[1][2], broken[2][0] = 9, 5, -3
    for cu in broken + [ints([2, 0, 4]), ints([4, 4, 0])]:
        out = torch.full_like(q, 3.0)
        cache.shared_attention(q, ptable, plen, cu, table, lengths, out=out)
        with pytest.raises(b.UsError):
            cache.check()
    cache.check()
    for plen2, ptable2 in ((ints([-1, 90]), ptable), (ints([100000, 90]), ptable), (plen, torch.cat([ptable[:1] * 0 + 10000, ptable[1:]]))):
        got = cache.shared_attention(q, ptable2.contiguous(), plen2, cu_seqs, table, lengths)
        with pytest.raises(b.UsError):
            cache.check()
        assert torch.equal(got[2:], want[2:])
    got = cache.shared_attention(q, ptable, plen, cu_seqs, table, ints([50, -2, 50, 100000]))
    with pytest.raises(b.UsError):
        cache.check()
    assert torch.equal(got[0], want[0]) and torch.equal(got[2], want[2]) and bool((got[1] == 0).all())
    assert torch.equal(cache.shared_attention(*args), want)
    cache.check()


def test_refusals(b):
    cache, args, want, _, _ = run(b, [100], [2], [50] * 2, [1] * 2, 2, 2, 128, 16, F16)
    q, ptable, plen, cu_seqs, table, lengths, _ = args
    for a in ((q.float(), ptable, plen, cu_seqs, table, lengths), (q[:, :3], ptable, plen, cu_seqs, table, lengths), (q, ptable.long(), plen, cu_seqs, table, lengths),
              (q, ptable, plen[:0], cu_seqs, table, lengths), (q, ptable, plen, cu_seqs[:1], table, lengths), (q, ptable, plen, None, table, lengths),
              (q, ptable, plen, cu_seqs.cpu(), table, lengths), (q, ptable, plen, cu_seqs, table[:1], lengths), (q[:1], ptable, plen, cu_seqs, table, lengths)):
        with pytest.raises(ValueError):
            cache.shared_attention(*a)
    assert cache.shared_attention(q[:0], ptable, plen, cu_seqs, table[:0], lengths[:0]).shape == (0, 4, 128)


@pytest.mark.parametrize("new,S,wide", [(1, 2, None), (1, 40, None), (1, 3, 12), (30, 4, None)])
def test_offsets_past_32_bits(b, new, S, wide):
    """Prefix and own tokens in blocks behind 4 GB of a pool; every kind of kernels; and copies to and from there."""
    T, Hkv, D = 256, 8, 128
    blocks = 17000                                      # 4.4e9 bytes of K
    codes = [torch.zeros(blocks, Hkv, T, D, dtype=torch.int8, device="cuda") for _ in range(2)]
    steps = [torch.full((blocks, Hkv), 1 / 32, device="cuda") for _ in range(2)]
    g = gen(1)
    far = blocks - 50
    for c in codes:
        c[far:] = (torch.randn(50, Hkv, T, D, device="cuda", generator=g) * 32).round().clamp(-127, 127).to(torch.int8)
    cache = b.KVCache(*codes, *steps)
    ptable, table = ints([[far, far + 1]]), torch.zeros(S, wide or 1, dtype=torch.int32, device="cuda")
    table[:, 0] = far + 2 + torch.arange(S, device="cuda").int()
    own = [new + 20] * S
    q = torch.randn(S * new, Hkv, D, device="cuda", generator=g).bfloat16()
    out = cache.shared_attention(q, ptable, ints([300]), ints([0, S]), table, ints(own), None if new == 1 else sums([new] * S))
    cache.check()
    ref, bound, _ = reference(cache, ptable, [300], [0] * S, table, own, [new] * S, q, D ** -0.5)
    check(out, ref, bound)
    cache.copy_blocks(ints([far, 3]), ints([1, far + 49]))
    cache.check()
    for c in codes:
        assert torch.equal(c[1], c[far]) and not c[far + 49].any()
