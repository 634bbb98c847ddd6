"""The 8-bit cache on the GPU against its definitions in 64 bits.

Append: steps (fp32) and codes are decided exactly and must be equal. Attention: with s = scale q.k, p = softmax(s), out = sum p v the kernels'
error is at most
  * of the scores, in fp32: |ds| <= (D + 4) 2^-23 |scale| sum_d |q_d k_d|, which changes p by the factor e^(2 ds) at most;
  * of p, rounded to fp16 (2^-11) after an exponential good to 2^-22 and a few fp32 products: 2^-11 + 2^-19 of p |v|;
  * of p below the smallest normal fp16 number: p carries 2^7 and may lie 2^8 below its running maximum's place, which leaves an absolute
    error of 2^-25 2^-7 of the largest term a token, times max |v|, over the sum (at least the largest term 1, or 2^-8 of it): 2^-24 L max|v|;
  * the result's rounding, eps / 2."""
import math

import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def b():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a CUDA device")
    from paper_2608_09291_b200 import binding
    torch.cuda.set_device(0)
    return binding


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def make(b, lens, Hkv=2, D=128, T=64, seed=0, spare=3, width=None, spread=0.5):
    """A cache with sequences of these lengths on blocks in any order; blocks of no sequence hold NaN steps, unused table entries rubbish."""
    g = gen(seed)
    per = [-(-n // T) for n in lens]
    blocks = sum(per) + spare
    order = torch.randperm(blocks, device="cuda", generator=g).int()
    width = max([1, width or 0] + per)
    table = torch.full((len(lens), width), -7, dtype=torch.int32, device="cuda")
    at = 0
    steps = [torch.full((blocks, Hkv), float("nan"), device="cuda") for _ in range(2)]
    for s, n in enumerate(per):
        ids = order[at:at + n]
        table[s, :n] = ids
        for t in steps:
            t[ids.long()] = torch.exp2((torch.rand(n, Hkv, device="cuda", generator=g) - 0.5) * 2 * spread) / 32
        at += n
    codes = [(torch.randn(blocks, Hkv, T, D, device="cuda", generator=g) * 32).round().clamp(-127, 127).to(torch.int8) for _ in range(2)]
    cache = b.KVCache(codes[0], codes[1], steps[0], steps[1])
    return cache, table, torch.tensor(lens, dtype=torch.int32, device="cuda")


def values(cache, table, n, s):
    """K and V of sequence s in 64 bits, (n, Hkv, D)."""
    T = cache.block_tokens
    ids = table[s, :-(-n // T)].long()
    return [(c[ids].double() * st[ids].double()[..., None, None]).transpose(1, 2).flatten(0, 1)[:n]
            for c, st in ((cache.k_codes, cache.k_steps), (cache.v_codes, cache.v_steps))]


def reference(cache, table, lens, new, q, scale, causal=True, window=0):
    """(out, bound on the error before the last rounding, lse) in 64 bits."""
    outs, bounds, lses, at = [], [], [], 0
    Hq, D = q.shape[1:]
    for s, (L, n) in enumerate(zip(lens, new)):
        x = q[at:at + n].double()
        at += n
        if n == 0:
            continue
        if L == 0:
            outs.append(torch.zeros_like(x)); bounds.append(torch.zeros_like(x)); lses.append(torch.full((n, Hq), -math.inf, device="cuda", dtype=torch.float64))
            continue
        k, v = values(cache, table, L, s)
        rep = Hq // k.shape[1]
        k, v = k.repeat_interleave(rep, 1), v.repeat_interleave(rep, 1)
        a = torch.einsum("nhd,lhd->hnl", x, k) * scale
        mag = torch.einsum("nhd,lhd->hnl", x.abs(), k.abs()) * abs(scale)
        t, pos = torch.arange(L, device="cuda"), torch.arange(L - n, L, device="cuda")[:, None]
        hidden = torch.zeros(n, L, dtype=torch.bool, device="cuda")
        if causal:
            hidden |= t > pos
        if window:
            hidden |= t <= pos - window
        a = a.masked_fill(hidden, -math.inf)
        lse = torch.logsumexp(a, -1)
        p = torch.nan_to_num(torch.exp(a - lse[..., None]))
        ds = (D + 4) * 2.0 ** -23 * mag.masked_fill(hidden, 0).amax(-1)
        o, m = torch.einsum("hnl,lhd->nhd", p, v), torch.einsum("hnl,lhd->nhd", p, v.abs())
        rel = (torch.expm1(2 * ds) + 2.0 ** -11 + 2.0 ** -19).t()[..., None]
        outs.append(o)
        bounds.append(rel * m + 2.0 ** -24 * L * v.abs().amax())
        lses.append(lse.t())
    return torch.cat(outs), torch.cat(bounds), torch.cat(lses)


def check(got, ref, bound):
    assert not torch.isnan(got).any()
    lim = bound + torch.finfo(got.dtype).eps / 2 * (ref.abs() + bound) + torch.finfo(got.dtype).tiny
    d = (got.double() - ref).abs()
    assert (d <= lim).all(), f"off by {float((d / lim.clamp(min=1e-300)).max()):.2f} bounds"


def cu_of(new):
    return torch.tensor([0] + torch.tensor(new).cumsum(0).tolist(), dtype=torch.int32, device="cuda")


def run(b, lens, new, Hq, Hkv, D, T, dtype, seed=0, causal=True, window=0, scale=None, width=None, spread=0.5):
    cache, table, lengths = make(b, lens, Hkv, D, T, seed, width=width, spread=spread)
    q = torch.randn(sum(new), Hq, D, device="cuda", generator=gen(seed + 1)).to(dtype)
    single = all(n == 1 for n in new)
    lse = torch.full((sum(new), Hq), 5.0, device="cuda")
    out = cache.attention(q, table, lengths, None if single else cu_of(new), scale=scale, causal=causal, window=window, lse=lse)
    cache.check()
    ref, bound, rl = reference(cache, table, lens, new, q, D ** -0.5 if scale is None else scale, causal, window)
    check(out, ref, bound)
    seen = torch.isfinite(rl)
    assert torch.equal(torch.isfinite(lse), seen)
    # the logarithm of a sum whose terms are off by the scores' error, in fp32
    assert (lse.double() - rl)[seen].abs().le(1e-5 * (1 + rl[seen].abs()) + 1e-4).all()
    return cache, table, lengths, q, out


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("D,T", [(128, 16), (128, 64), (64, 32), (64, 256)])
@pytest.mark.parametrize("G", [1, 3, 8, 9, 16, 40])
def test_single_tokens(b, dtype, D, T, G):
    run(b, [1, 2, 15, 16, 17, 63, 64, 65, 127, 128, 129, 500, 1000], [1] * 13, 2 * G, 2, D, T, dtype, seed=G)


@pytest.mark.parametrize("D,T", [(128, 32), (64, 128)])
@pytest.mark.parametrize("new", [[2, 1, 3], [5, 17, 1], [100, 1, 260], [33, 300, 128], [0, 7, 0]])
@pytest.mark.parametrize("G", [1, 4, 8])
def test_prompts(b, D, T, new, G):
    run(b, [300, 400, 260], new, 2 * G, 2, D, T, torch.bfloat16 if G == 4 else torch.float16, seed=sum(new))


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("window", [1, 2, 50, 64, 129, 1000])
@pytest.mark.parametrize("new", [[1, 1, 1], [40, 3, 200]])
def test_masks(b, causal, window, new):
    run(b, [333, 70, 512], new, 8, 2, 128, 16, torch.float16, causal=causal, window=window, seed=window)


@pytest.mark.parametrize("new", [[1], [9], [300]])
@pytest.mark.parametrize("scale", [0.0, -0.1, 1.0, 1e-4])
def test_scale(b, scale, new):
    """Also scores of a hundred and more, and negative and no weight."""
    run(b, [700], new, 4, 2, 128, 64, torch.float16, scale=scale)


@pytest.mark.parametrize("new", [[1, 1], [20, 150]])
@pytest.mark.parametrize("D", [64, 128])
def test_steps_that_differ_a_lot(b, new, D):
    """Steps over eight orders of two either way, growing along a sequence; blocks of zeros."""
    cache, table, lengths = make(b, [900, 640], 2, D, 16, 5, spread=4.0)
    ids = table[0, :56].long()
    cache.v_steps[ids] = cache.v_steps[ids].sort(0).values
    cache.v_steps[table[1, 3].long()] = 0
    cache.k_steps[table[1, 4].long()] = 0
    cache.v_codes[table[0, 5].long()] = 0
    q = torch.randn(sum(new), 8, D, device="cuda", generator=gen(1)).half()
    out = cache.attention(q, table, lengths, None if max(new) == 1 else cu_of(new))
    cache.check()
    ref, bound, _ = reference(cache, table, [900, 640], new, q, D ** -0.5)
    check(out, ref, bound)


@pytest.mark.parametrize("L,G,new", [(40000, 8, 1), (131072, 1, 1), (20000, 8, 16), (70000, 4, 70)])
def test_long(b, L, G, new):
    run(b, [L], [new], G, 1, 128, 64, torch.bfloat16, seed=1)


def closely(cache, table, L, n, q, scale=None, causal=True, window=0, exact_p=False):
    """(out, bound on the error before the last rounding) of one sequence in 64 bits, with a bound that stays below the outputs of long contexts.

    Of each row, with p normalised: the scores' error as above; p's rounding, 2^-11 (fp16; exact_p: it is kept, 2^-22) and 2^-19, of sum p |v|;
    p below the smallest normal fp16 number: p times V's step carries 2^7 relative to a place that is at most the largest of them, rounded up to
    a power of two: 2^-25 2^-7 2 max(p step) a token seen, times a code of 127; fp32 sums of numerator and denominator, each addition off by up
    to 2^-23 of the magnitudes: for up to 32 rows a head four in 128 tokens of a block's share, four warps and the parts of all shares, else one in 16 tokens."""
    D, Hkv, T = q.shape[2], cache.n_kv_heads, cache.block_tokens
    scale = D ** -0.5 if scale is None else scale
    x, rep = q.double(), q.shape[1] // Hkv
    k, v = [t.repeat_interleave(rep, 1) for t in values(cache, table, L, 0)]
    step = cache.v_steps[table[0, torch.arange(L, device="cuda") // T].long()].double().repeat_interleave(rep, 1).t()[:, None]    # (H, 1, L)
    a = torch.einsum("nhd,lhd->hnl", x, k) * scale
    mag = torch.einsum("nhd,lhd->hnl", x.abs(), k.abs()) * abs(scale)
    t, pos = torch.arange(L, device="cuda"), torch.arange(L - n, L, device="cuda")[:, None]
    seen = (t <= pos) if causal else torch.ones(n, L, dtype=torch.bool, device="cuda")
    if window:
        seen = seen & (t > pos - window)
    p = torch.softmax(a.masked_fill(~seen, -math.inf), -1)
    ds = (D + 4) * 2.0 ** -23 * mag.masked_fill(~seen, 0).amax(-1)
    if n * rep <= 32:
        blocks = 2 * torch.cuda.get_device_properties(0).multi_processor_count
        adds = 4 * -(-(-(-n * rep // 8) * Hkv * (L / 128 + 6)) // blocks) + 4 + min(blocks, L / 128 + 1)
    else:
        adds = L / 16 + 64
    rel = torch.expm1(2 * ds) + (2.0 ** -22 if exact_p else 2.0 ** -11) + 2.0 ** -19 + 2 * adds * 2.0 ** -23
    # (an exactly 0 p has no weight, whatever its step)
    absolute = 2.0 ** -31 * 127 * seen.sum(-1) * torch.where(p > 0, p * step, torch.zeros((), dtype=torch.float64, device="cuda")).amax(-1)
    vs = torch.where((p > 0).any(1).t()[..., None], v, torch.zeros((), dtype=torch.float64, device="cuda"))
    o, m = torch.einsum("hnl,lhd->nhd", p, vs), torch.einsum("hnl,lhd->nhd", p, vs.abs())
    return o, rel.t()[..., None] * m + absolute.t()[..., None]


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("G,new", [(1, 1), (3, 1), (8, 1), (9, 1), (16, 1), (32, 1), (5, 3), (2, 16)])
def test_float16_of_few_rows_is_off_by_its_own_rounding(b, G, new, D):
    """Up to 32 rows a cache head: p's rounding does not show. Scores are small, so that their own error does not either."""
    L = 40
    cache, table, lengths = make(b, [L], 4, D, 16, G)
    q = (torch.randn(new, 4 * G, D, device="cuda", generator=gen(3)) * 0.02).half()
    out = cache.attention(q, table, lengths, None if new == 1 else cu_of([new]))
    cache.check()
    ref, bound = closely(cache, table, L, new, q, exact_p=True)
    check(out, ref, bound)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("L,G,Hkv,new,D", [(131072, 1, 1, 1, 128), (131072, 8, 1, 1, 64), (40000, 16, 2, 1, 128), (30000, 5, 2, 3, 128), (20000, 8, 1, 16, 128), (70000, 4, 1, 70, 128)])
def test_long_contexts_closely(b, dtype, L, G, Hkv, new, D):
    """Outputs of long contexts are small: with a bound that is smaller still."""
    cache, table, lengths = make(b, [L], Hkv, D, 64, 2)
    q = torch.randn(new, G * Hkv, D, device="cuda", generator=gen(3)).to(dtype)
    out = cache.attention(q, table, lengths, None if new == 1 else cu_of([new]))
    cache.check()
    ref, bound = closely(cache, table, L, new, q, exact_p=dtype == torch.float16 and new * G <= 32)
    assert bound.square().mean() < ref.square().mean() / 9
    check(out, ref, bound)


# new tokens, query heads a cache head, blocks of the table: up to 32 rows a cache head take the kernel of single tokens, more the one of
# prompts; a table that is wide enough cuts its walk
KINDS = [(3, 2, 60), (8, 2, 60), (16, 2, 60), (32, 1, 2000), (60, 2, 60), (60, 2, 2000), (300, 1, 60)]


@pytest.mark.parametrize("new,G,width", KINDS)
@pytest.mark.parametrize("D,T", [(128, 16), (64, 64)])
@pytest.mark.parametrize("power", [12, 24, 60])
@pytest.mark.parametrize("window", [0, 100])
def test_steps_of_tokens_that_a_row_does_not_see(b, new, G, width, D, T, power, window):
    """Values of later tokens (and of ones in front of the window) that are larger by any factor: each row is as exact as its own tokens allow."""
    L = 900
    cache, table, lengths = make(b, [L], 2, D, T, 5, width=width)
    cache.v_steps[table[0, (L - 1) // T].long()] *= 2.0 ** power          # the last block: only the last rows see it
    if window:
        cache.v_steps[table[0, (L - new - 90) // T].long()] *= 2.0 ** power     # in front of the last rows' window, where there are enough rows
    q = torch.randn(new, 2 * G, D, device="cuda", generator=gen(1)).bfloat16()
    out = cache.attention(q, table, lengths, cu_of([new]), window=window)
    cache.check()
    ref, bound = closely(cache, table, L, new, q, window=window)
    check(out, ref, bound)
    # (a NaN among what a row does not see is none of its business)
    cache.v_steps[table[0, (L - 1) // T].long()] = float("nan")
    got = cache.attention(q, table, lengths, cu_of([new]), window=window)
    blind = L - new + torch.arange(new, device="cuda") < (L - 1) // T * T
    assert blind.any() == (new > 4)
    check(got[blind], ref[blind], bound[blind])
    assert torch.isnan(got[~blind]).all()


@pytest.mark.parametrize("new,G,width", [(1, 1, 60), (1, 8, 2000), (1, 16, 60)] + KINDS)
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("away,power", [(30, 24), (90, 40), (90, 100), (1000, 60), (12, 20)])
def test_steps_of_tokens_without_weight(b, new, G, width, D, away, power):
    """A block whose values are 2^power larger and whose scores are `away` below the others': what it adds counts for what it is."""
    L, T = 700, 16
    cache, table, lengths = make(b, [L], 1, D, T, 6, width=width)
    q = torch.randn(new, G, D, device="cuda", generator=gen(1))
    q[..., 0] = 4.0
    for i in (3, 30):
        blk = table[0, i].long()
        cache.k_codes[blk] = 0
        cache.k_codes[blk, :, :, 0] = -127
        cache.k_steps[blk] = away / (127 * 4.0 * D ** -0.5)
        cache.v_steps[blk] *= 2.0 ** power
    q = q.half()
    out = cache.attention(q, table, lengths, None if new == 1 else cu_of([new]))
    cache.check()
    ref, bound = closely(cache, table, L, new, q)
    ok = ref.abs() + bound < 60000                   # (fp16 holds them)
    assert not torch.isnan(out).any()
    check(out[ok], ref[ok], bound[ok])


def test_many_sequences(b):
    lens = [(37 * i) % 300 for i in range(1, 101)] + [0, 5000, 0, 1]
    run(b, lens, [1] * 104, 16, 2, 128, 64, torch.float16)
    new = [min(n, i % 5) for i, n in enumerate(lens)]
    run(b, lens, new, 16, 2, 128, 64, torch.float16)


@pytest.mark.parametrize("new", [1, 60])
def test_large_queries(b, new):
    """bfloat16 beyond fp16's range, and tiny ones: the scores are as exact."""
    cache, table, lengths = make(b, [200], 1, 128, 64, 3)
    q = torch.randn(new, 4, 128, device="cuda", generator=gen(4))
    q = (q * torch.tensor([1e6, 1.0, 1e-9, 1e-30], device="cuda")[:, None]).bfloat16()
    cu = cu_of([new])
    out = cache.attention(q, table, lengths, cu, scale=1e-7)
    ref, bound, _ = reference(cache, table, [200], [new], q, 1e-7)
    check(out, ref, bound)


@pytest.mark.parametrize("new", [1, 200])
def test_nan_stays_in_its_rows(b, new):
    cache, table, lengths = make(b, [300, 300], 2, 128, 64, 3)
    q = torch.randn(2 * new, 8, 128, device="cuda", generator=gen(4)).half()
    want = cache.attention(q, table, lengths, cu_of([new, new]))
    bad = q.clone()
    bad[0, 3, 7] = float("nan")
    bad[new, 5, 100] = float("inf")
    got = cache.attention(bad, table, lengths, cu_of([new, new]))
    hit = torch.zeros(2 * new, 8, dtype=torch.bool, device="cuda")
    hit[0, 3] = hit[new, 5] = True
    assert torch.isnan(got[hit]).all() and torch.equal(got[~hit], want[~hit])
    cache.v_steps[table[1, 2].long(), 0] = float("nan")       # a step that is NaN, where a sequence sees it
    got = cache.attention(q, table, lengths, cu_of([new, new]))
    assert torch.equal(got[:new], want[:new]) and torch.equal(got[new:, 4:], want[new:, 4:])
    assert torch.isnan(got[2 * new - 1, :4]).all()


@pytest.mark.parametrize("new,width", [(1, 4096), (60, 300), (60, 4096), (500, 4096)])
@pytest.mark.parametrize("D", [64, 128])
def test_nan_stays_in_its_rows_of_cut_items(b, new, width, D):
    """A table that is wide enough for the walk over a context to be cut: rows that are NaN are so in both results, the others are as without them."""
    cache, table, lengths = make(b, [3000], 2, D, 64, 3, width=width // 64 + 45)
    q = torch.randn(new, 8, D, device="cuda", generator=gen(4)).half()
    cu, hit = cu_of([new]), torch.zeros(new, 8, dtype=torch.bool, device="cuda")
    lse = [torch.full((new, 8), 5.0, device="cuda") for _ in range(3)]
    want = cache.attention(q, table, lengths, cu, lse=lse[0])
    bad = q.clone()
    bad[0, 3, 7], bad[new - 1, 5, 40] = float("nan"), float("inf")
    hit[0, 3] = hit[new - 1, 5] = True
    got = cache.attention(bad, table, lengths, cu, lse=lse[1])
    assert torch.isnan(got[hit]).all() and torch.equal(got[~hit], want[~hit])
    assert torch.isnan(lse[1][hit]).all() and torch.equal(lse[1][~hit], lse[0][~hit])
    cache.k_steps[table[0, 20].long(), 1] = float("nan")       # all rows of a head see it
    got = cache.attention(q, table, lengths, cu, lse=lse[2])
    assert torch.isnan(got[:, 4:]).all() and torch.equal(got[:, :4], want[:, :4])
    assert torch.isnan(lse[2][:, 4:]).all() and torch.equal(lse[2][:, :4], lse[0][:, :4])
    cache.check()


@pytest.mark.parametrize("new", [[1, 1, 1], [2, 40, 9], [100, 30, 250]])
def test_strides_and_rows_behind(b, new):
    """q and out as views of wider rows, heads outermost; rows behind the last sequence stay as they are."""
    lens, N = [300, 50, 400], sum(new)
    cache, table, lengths = make(b, lens, 2, 64, 32, 9)
    cu = cu_of(new)
    wide = torch.randn(N + 3, 12 * 64 + 5, device="cuda", generator=gen(2)).half()
    q = wide[:, 3:3 + 8 * 64].unflatten(1, (8, 64))
    out = torch.full((8, N + 3, 70), 2.0, device="cuda", dtype=torch.float16)
    view = out[:, :, 1:65].transpose(0, 1)
    got = cache.attention(q, table, lengths, cu, out=view)
    cache.check()
    assert got is view
    ref, bound, _ = reference(cache, table, lens, new, q[:N], 64 ** -0.5)
    check(view[:N], ref, bound)
    assert (view[N:] == 2).all() and (out[:, :, 0] == 2).all() and (out[:, :, 65:] == 2).all()
    assert torch.equal(view[:N], cache.attention(q[:N].contiguous(), table, lengths, cu))


@pytest.mark.parametrize("new", [[1, 1, 1], [1, 1, 50]])
def test_padded_batch(b, new):
    """Empty sequences with rows: 0, and no complaint."""
    cache, table, lengths = make(b, [100, 0, 200], 2, 128, 64, 2)
    q = torch.randn(sum(new), 4, 128, device="cuda", generator=gen(3)).half()
    k = torch.randn(sum(new), 2, 128, device="cuda", generator=gen(4)).half()
    cu = None if max(new) == 1 else cu_of(new)
    before = cache.k_codes.clone()
    cache.append(k, k, table, lengths, cu)
    out = cache.attention(q, table, lengths, cu)
    cache.check()
    assert (out[1] == 0).all()
    ref, bound, _ = reference(cache, table, [100, 0, 200], new, q, 128 ** -0.5)
    check(out, ref, bound)
    touched = (cache.k_codes != before).flatten(1).any(1).nonzero().flatten().tolist()
    assert set(touched) <= set(table[0, 1:2].tolist() + table[2, (200 - new[2]) // 64:].tolist())


def test_blocks_shared_and_gone(b):
    """Two sequences on the same blocks; blocks in front of every window may be any number."""
    cache, table, lengths = make(b, [256, 256], 2, 128, 16, 2)
    table[1, :8] = table[0, :8]
    q = torch.randn(2, 4, 128, device="cuda", generator=gen(3)).half()
    out = cache.attention(q, table, lengths)
    ref, bound, _ = reference(cache, table, [256, 256], [1, 1], q, 128 ** -0.5)
    check(out, ref, bound)
    for new in (1, 30):
        qn = torch.randn(2 * new, 4, 128, device="cuda", generator=gen(5)).half()
        want = cache.attention(qn, table, lengths, cu_of([new, new]), window=40)
        gone = table.clone()
        gone[:, :(256 - new - 40 + 1) // 16] = -1
        got = cache.attention(qn, gone, lengths, cu_of([new, new]), window=40)
        cache.check()
        assert torch.equal(got, want)


def test_indices_out_of_range_are_reported(b):
    """A bad block number, length or token count: an error, nothing written outside, the other sequences' results as ever."""
    cache, table, lengths = make(b, [200, 130, 90], 2, 128, 64, 2)
    q = torch.randn(3, 4, 128, device="cuda", generator=gen(3)).half()
    kn = torch.randn(3, 2, 128, device="cuda", generator=gen(4)).half()
    want = cache.attention(q, table, lengths)
    cache.check()

    held = (cache.k_codes, cache.k_steps, cache.v_codes, cache.v_steps)
    before = [t.clone() for t in held]

    def restore():   # (an append has written the good sequences' tokens)
        for t, o in zip(held, before):
            t.copy_(o)

    def bad(f):
        f()
        with pytest.raises(b.UsError) as e:
            cache.check()
        assert e.value.status == 9
        cache.check()      # reported once

    for entry in (cache.n_blocks, -1, 2 ** 31 - 1):
        t = table.clone()
        t[1, 0] = entry
        out = []
        bad(lambda: out.append(cache.attention(q, t, lengths)))
        assert torch.equal(out[0][0], want[0]) and torch.equal(out[0][2], want[2]) and not torch.isnan(out[0][1]).any()
        qn = torch.randn(180, 4, 128, device="cuda", generator=gen(5)).half()
        cu = cu_of([60, 60, 60])
        full = cache.attention(qn, table, lengths, cu)
        bad(lambda: out.append(cache.attention(qn, t, lengths, cu)))
        assert torch.equal(out[1][:60], full[:60]) and torch.equal(out[1][120:], full[120:])
        bad(lambda: cache.read(t, lengths, 100))
        t[1, 0] = table[1, 0]
        t[1, 2] = entry                           # the block that gets the new token
        one = lambda: cache.append(kn, kn, t, lengths)  # noqa: E731
        bad(one)
        ids = [int(table[0, 3]), int(table[2, 1])]
        keep = [i for i in range(cache.n_blocks) if i not in ids]
        for t_now, o in zip(held, before):
            assert same(t_now[keep], o[keep])
        restore()
    for value in (-1, 10 ** 6):
        n = lengths.clone()
        n[1] = value
        bad(lambda: cache.attention(q, table, n))
        bad(lambda: cache.append(kn, kn, table, n))
        bad(lambda: cache.read(table, n, 100))
        restore()
    for cu in ([0, 1, 0, 3], [0, 1, 2, 4], [-1, 1, 2, 3], [0, 0, 200, 200]):
        c = torch.tensor(cu, dtype=torch.int32, device="cuda")
        bad(lambda: cache.attention(q, table, lengths, c))
        bad(lambda: cache.append(kn, kn, table, lengths, c))
        restore()


# ---- append ----

def ref_append(cache, table, lens, new, k, v):
    """The cache's codes and steps after the call, by the definition in 64 bits (steps rounded to fp32)."""
    T = cache.block_tokens
    out = []
    for codes, steps, x in ((cache.k_codes, cache.k_steps, k), (cache.v_codes, cache.v_steps, v)):
        codes, steps, x, at = codes.clone(), steps.clone(), x.double(), 0
        for s, (L, n) in enumerate(zip(lens, new)):
            for j in range((L - n) // T, -(-L // T)) if n else ():
                lo, hi, blk = max(j * T, L - n), min(L, j * T + T), int(table[s, j])
                part = x[at + lo - (L - n):at + hi - (L - n)].transpose(0, 1)
                fin = torch.where(torch.isfinite(part), part.abs(), torch.zeros((), dtype=torch.float64, device="cuda"))
                step = (fin.amax((1, 2)).float() / torch.tensor(127.0, device="cuda"))
                a = lo - j * T
                if a:
                    old = steps[blk]
                    step = torch.maximum(old, step)
                    r = torch.where((step > old)[:, None, None], (codes[blk, :, :a].double() * old.double()[:, None, None] / step.double()[:, None, None].clamp(min=1e-300)).round(),
                                    codes[blk, :, :a].double())
                    codes[blk, :, :a] = r.to(torch.int8)
                steps[blk] = step
                d = step.double()[:, None, None]
                c = torch.where(d > 0, part / d, torch.zeros((), dtype=torch.float64, device="cuda")).round().clamp(-127, 127)
                codes[blk, :, a:a + hi - lo] = torch.nan_to_num(c, nan=0.0).to(torch.int8)
            at += n
        out += [codes, steps]
    return out


def same(a, c):
    return torch.equal(a.nan_to_num(1e30), c.nan_to_num(1e30)) if a.is_floating_point() else torch.equal(a, c)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,D,Hkv", [(16, 128, 5), (32, 64, 1), (64, 128, 2), (128, 128, 3), (256, 64, 4)])
@pytest.mark.parametrize("new", [[1, 1, 1, 1], [3, 1, 200, 0], [64, 300, 17, 5]])
def test_append_is_exact(b, dtype, T, D, Hkv, new):
    lens = [64, 300, 257, 5]
    cache, table, lengths = make(b, lens, Hkv, D, T, T)
    N = sum(new)
    x = torch.randn(N, 3 * Hkv, D, device="cuda", generator=gen(N)) * torch.exp2(torch.randint(-3, 3, (N, 1, 1), device="cuda", generator=gen(1)).float())
    x = x.to(dtype)
    k, v = x[:, Hkv:2 * Hkv], x[:, 2 * Hkv:]
    want = ref_append(cache, table, lens, new, k, v)
    cache.append(k, v, table, lengths, None if max(new) == 1 and min(new) == 1 else cu_of(new))
    cache.check()
    for got, ref in zip((cache.k_codes, cache.k_steps, cache.v_codes, cache.v_steps), want):
        assert same(got, ref)
    K, V = cache.read(table, lengths, 300)
    for s, L in enumerate(lens):
        rk, rv = values(cache, table, L, s)
        assert torch.equal(K[s, :L], rk.float()) and torch.equal(V[s, :L], rv.float()) and (K[s, L:] == 0).all() and (V[s, L:] == 0).all()
    for t in (torch.float16, torch.bfloat16):
        a, c = cache.read(table, lengths, 70, dtype=t)
        assert torch.equal(a, K[:, :70].to(t)) and torch.equal(c, V[:, :70].to(t))


def test_append_borders_and_special_values(b):
    """Quotients on the border between codes and next to it; zeros, subnormal and huge values, infinities, NaN; unaligned rows."""
    cache, table, lengths = make(b, [16] * 6, 2, 64, 16, 1)
    cache.k_steps.zero_(), cache.v_steps.zero_()
    i = torch.arange(16 * 2 * 64, device="cuda").view(16, 2, 64)
    x = torch.zeros(6 * 16, 2, 65, device="cuda")[:, :, 1:]
    half = ((i % 254) - 127).float() + 0.5
    x[:16] = half / 127 * 1.0                       # step 1 / 127
    x[:16, :, 0] = 1.0
    x[16:32] = torch.nextafter(half * 0.03, torch.tensor(9e9, device="cuda"))
    x[16:32, :, 0] = 127 * 0.03
    x[32:48] = 0
    x[48:64] = 2.0 ** -140 * ((i % 250) - 120)
    x[64:80] = 3e38 * (((i % 250) - 125) / 125.0)
    x[80:96] = half
    x[85, 0, 3], x[86, 1, 4], x[87, 0, 5] = float("inf"), float("-inf"), float("nan")
    new = [16] * 6
    want = ref_append(cache, table, [16] * 6, new, x, -x)
    cache.append(x, -x, table, lengths, cu_of(new))
    cache.check()
    for got, ref in zip((cache.k_codes, cache.k_steps, cache.v_codes, cache.v_steps), want):
        assert same(got, ref)


def test_append_token_by_token(b):
    """A sequence that grows by single tokens and by a few, larger ones later: the older codes follow the step as the definition says."""
    cache, table, _ = make(b, [100], 2, 128, 32, 1)
    cache.k_steps.zero_(), cache.v_steps.zero_()
    at, i = 0, 0
    while at < 100:
        n = min(100 - at, [1, 1, 3, 1, 40][i % 5])
        x = torch.randn(n, 2, 128, device="cuda", generator=gen(i)) * (1 + 0.3 * i)
        at, i = at + n, i + 1
        lengths = torch.tensor([at], dtype=torch.int32, device="cuda")
        want = ref_append(cache, table, [at], [n], x, 2 * x)
        cache.append(x, 2 * x, table, lengths, None if n == 1 else cu_of([n]))
        for got, ref in zip((cache.k_codes, cache.k_steps, cache.v_codes, cache.v_steps), want):
            assert same(got, ref)
    cache.check()


@pytest.mark.parametrize("Hkv", [1, 2, 3, 5])
@pytest.mark.parametrize("T,D,n", [(256, 64, 1), (256, 128, 1), (32, 128, 2), (64, 64, 3), (16, 128, 2)])
def test_older_codes_are_rescaled_once(b, T, D, n, Hkv):
    """Hundreds of sequences whose only block fills up while every call makes its step grow: head counts that leave teams of a block of
    the grid without a head, for each size of a team. Codes and steps must be equal to the definition's after every call."""
    S = 400
    g = gen(Hkv)
    codes = [torch.randint(-127, 128, (S, Hkv, T, D), device="cuda", generator=g).to(torch.int8) for _ in range(2)]
    steps = [0.01 + 0.01 * torch.rand(S, Hkv, device="cuda", generator=g) for _ in range(2)]
    want = [[c.clone(), s.clone()] for c, s in zip(codes, steps)]
    cache = b.KVCache(codes[0], codes[1], steps[0], steps[1])
    order = torch.randperm(S, device="cuda", generator=g)
    table, cu = order.int()[:, None], None if n == 1 else cu_of([n] * S)
    for L in range(max(n, T - 40 * n), T + 1, n):
        x = torch.randn(S * n, 2 * Hkv, D, device="cuda", generator=g)
        for i in range(2):       # the largest magnitude of each new token is above all that the block holds
            x[:, i * Hkv:(i + 1) * Hkv, L % D] = (want[i][1][order] * 127 * 1.03).repeat_interleave(n, 0)
        cache.append(x[:, :Hkv], x[:, Hkv:], table, torch.full((S,), L, dtype=torch.int32, device="cuda"), cu)
        for i, (c, s) in enumerate(want):
            part = x[:, i * Hkv:(i + 1) * Hkv].view(S, n, Hkv, D).transpose(1, 2)
            now = torch.maximum(s[order], part.abs().amax((2, 3)) / torch.tensor(127.0, device="cuda"))
            assert L == n or (now > s[order]).all()
            d = now.double()[..., None, None]
            c[order, :, :L - n] = (c[order, :, :L - n].double() * s[order].double()[..., None, None] / d).round().to(torch.int8)
            c[order, :, L - n:L] = (part.double() / d).round().clamp(-127, 127).to(torch.int8)
            s[order] = now
        for got, ref in zip((cache.k_codes, cache.k_steps, cache.v_codes, cache.v_steps), (want[0][0], want[0][1], want[1][0], want[1][1])):
            assert torch.equal(got, ref)
    cache.check()


def test_offsets_past_32_bits(b):
    """A pool of more than 2^32 bytes of codes, its last blocks in use."""
    blocks, Hkv, T, D = 33000, 8, 128, 128
    codes = [torch.empty(blocks, Hkv, T, D, dtype=torch.int8, device="cuda") for _ in range(2)]
    steps = [torch.empty(blocks, Hkv, device="cuda") for _ in range(2)]
    cache = b.KVCache(*codes, *steps)
    table = torch.tensor([[blocks - 1, 5, blocks - 2], [blocks - 3, blocks - 4, 7]], dtype=torch.int32, device="cuda")
    lens, new = [300, 290], [300, 290]
    lengths = torch.tensor(lens, dtype=torch.int32, device="cuda")
    x = torch.randn(590, 2 * Hkv, D, device="cuda", generator=gen(1)).half()
    cache.append(x[:, :Hkv], x[:, Hkv:], table, lengths, cu_of(new))
    K, V = cache.read(table, lengths, 300)
    at = 0
    for s, L in enumerate(lens):
        rk, rv = values(cache, table, L, s)
        assert torch.equal(K[s, :L], rk.float()) and torch.equal(V[s, :L], rv.float())
        # (half a step of the block's largest magnitude, which no normal draw here passes 6 with)
        assert (K[s, :L] - x[at:at + L, :Hkv].float()).abs().max() <= 0.5 * 6 / 127 + 1e-6
        at += L
    for n in (1, 100):
        q = torch.randn(2 * n, 16, D, device="cuda", generator=gen(2)).half()
        out = cache.attention(q, table, lengths, cu_of([n, n]))
        cache.check()
        ref, bound, _ = reference(cache, table, lens, [n, n], q, D ** -0.5)
        check(out, ref, bound)


# ---- streams, graphs, the layer ----

@pytest.mark.parametrize("new", [1, 40])
def test_another_stream_and_graph(b, new):
    """On other streams; captured and replayed while the sequences grow; an eager call between replays, a second graph at the same time."""
    cache, table, lengths = make(b, [400, 300], 2, 128, 64, 1)
    lengths.copy_(torch.tensor([200, 100], dtype=torch.int32))
    N = 2 * new
    cu = None if new == 1 else cu_of([new, new])
    q, x = torch.randn(N, 8, 128, device="cuda", generator=gen(1)).half(), torch.randn(N, 4, 128, device="cuda", generator=gen(2)).half()

    def step():
        cache.append(x[:, :2], x[:, 2:], table, lengths, cu)
        return cache.attention(q, table, lengths, cu)

    want = step()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        a = step()
    c = cache.attention(q, table, lengths, cu, stream=s.cuda_stream)
    s.synchronize()
    assert torch.equal(a, want) and torch.equal(c, want)
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            y = step()
        graphs.append((g, y))
    other = torch.cuda.Stream()
    for _ in range(3):
        lengths += new
        x.normal_(generator=gen(int(lengths[0])))
        torch.cuda.synchronize()
        graphs[0][0].replay()
        torch.cuda.synchronize()
        with torch.cuda.stream(other):
            graphs[1][0].replay()
        torch.cuda.synchronize()
        eager = cache.attention(q, table, lengths, cu)
        assert torch.equal(graphs[0][1], eager) and torch.equal(graphs[1][1], eager)
        lens = lengths.tolist()
        ref, bound, _ = reference(cache, table, lens, [new, new], q, 128 ** -0.5)
        check(eager, ref, bound)
    cache.check()
    del graphs


def test_two_streams_at_once(b):
    """Calls on one cache at the same time: each has scratch of its own."""
    cache, table, lengths = make(b, [5000, 3000], 2, 128, 64, 1)
    qs = [torch.randn(2 * n, 16, 128, device="cuda", generator=gen(n)).half() for n in (1, 2, 60)]
    cus = [None, cu_of([2, 2]), cu_of([60, 60])]
    want = [cache.attention(q, table, lengths, cu) for q, cu in zip(qs, cus)]
    streams = [torch.cuda.Stream() for _ in qs]
    torch.cuda.synchronize()
    got = [[] for _ in qs]
    for _ in range(10):
        for i, st in enumerate(streams):
            with torch.cuda.stream(st):
                got[i].append(cache.attention(qs[i], table, lengths, cus[i]))
    torch.cuda.synchronize()
    cache.check()
    for w, g in zip(want, got):
        assert all(torch.equal(y, w) for y in g)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("S,G,n", [(3, 8, 1), (3000, 8, 1), (2000, 2, 3), (1500, 16, 1)])
def test_what_follows_attention_waits_for_it(b, dtype, S, G, n):
    """Contexts of at most 128 tokens in a table of 4096: nothing is cut, so the kernel that joins parts has none. What the library launches
    behind it (a product that reads the output, an append that writes the blocks, the next attention into the same output) gives what it
    gives with a synchronisation in between."""
    Hkv, D, T = 2, 128, 64
    lens = [n + (29 * i) % (128 - n) for i in range(S)]
    cache, table, lengths = make(b, lens, Hkv, D, T, 3, width=4096 // T)
    cu = None if n == 1 else cu_of([n] * S)
    q = [torch.randn(S * n, G * Hkv, D, device="cuda", generator=gen(i)).to(dtype) for i in (4, 5)]
    w = b.mx4_quantize(torch.randn(128, G * Hkv * D, device="cuda", generator=gen(6)) / 32).freeze()
    x = torch.randn(S * n, 2 * Hkv, D, device="cuda", generator=gen(7)).to(dtype)
    held = (cache.k_codes, cache.k_steps, cache.v_codes, cache.v_steps)
    before = [t.clone() for t in held]
    out = torch.empty_like(q[0])

    def calls(pause):
        ys = []
        for part in q:
            cache.attention(part, table, lengths, cu, out=out)
            pause()
            ys.append(b.mx4_linear(out.flatten(1), w))
            pause()
        cache.attention(q[0], table, lengths, cu, out=out)
        pause()
        cache.append(x[:, :Hkv], x[:, Hkv:], table, lengths, cu)
        pause()
        return ys

    def restore():
        for t, o in zip(held, before):
            t.copy_(o)
        out.fill_(1000)
        torch.cuda.synchronize()

    restore()
    want = calls(torch.cuda.synchronize) + [out.clone()]
    ref, bound, _ = reference(cache_of(b, before), table, lens[:40], [n] * min(S, 40), q[0][:40 * n], D ** -0.5)
    check(want[2][:40 * n], ref, bound)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = calls(lambda: None)
    for _ in range(5):
        restore()
        got = calls(lambda: None)
        torch.cuda.synchronize()
        assert all(torch.equal(a, c) for a, c in zip(want, got + [out]))
        restore()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, c) for a, c in zip(want, captured + [out]))
    cache.check()
    b.mx4_check()
    del graph


def cache_of(b, held):
    return b.KVCache(held[0], held[2], held[1], held[3])


def test_refusals(b):
    cache, table, lengths = make(b, [100, 50], 2, 128, 64, 1)
    q, k = torch.zeros(2, 4, 128, device="cuda").half(), torch.zeros(2, 2, 128, device="cuda").half()
    for bad in (q.float(), q[:, :3], q[..., :64], q[:1], q.transpose(1, 2), q.cpu()):
        with pytest.raises((ValueError, b.UsError)):
            cache.attention(bad, table, lengths)
    for bad in (k[:, :1], k.int(), k[:1], k[..., ::2]):
        with pytest.raises((ValueError, b.UsError)):
            cache.append(bad, k, table, lengths)
    for t, n in ((table.long(), lengths), (table, lengths.long()), (table, lengths[:1]), (table[0], lengths), (table.cpu(), lengths)):
        with pytest.raises(ValueError):
            cache.attention(q, t, n)
    with pytest.raises(ValueError):
        cache.attention(q, table, lengths, torch.zeros(2, dtype=torch.int32, device="cuda"))
    with pytest.raises(ValueError):
        cache.attention(q, table, lengths, out=torch.zeros(2, 4, 64, device="cuda").half())
    with pytest.raises(ValueError):
        cache.attention(q, table, lengths, lse=torch.zeros(2, 5, device="cuda"))
    with pytest.raises((ValueError, b.UsError)):
        cache.attention(q, table, lengths, window=-1)
    with pytest.raises(b.UsError):
        cache.attention(q, table, lengths, scale=float("nan"))
    with pytest.raises(b.UsError):
        cache.read(table, lengths, 10 ** 6)
    with pytest.raises(b.UsError):
        b.KVCache.new(4, 2, 96)
    cache.close()
    with pytest.raises(b.UsError):
        cache.attention(q, table, lengths)


def test_decoder_layer(b):
    """The attention block of a decoder layer as a program runs it: the stacked Q/K/V projection (dense MX4, or sparse INT4), append,
    attention, the O projection, for a prompt and then token by token; each stage against the definition on the device's own input."""
    from paper_2608_09291_b200 import workloads
    H, Hkv, D, hidden = 8, 2, 128, 1024
    g = gen(1)
    wqkv = b.mx4_quantize(torch.randn((H + 2 * Hkv) * D, hidden, device="cuda", generator=g) / 32).freeze()
    s_w = workloads.make_chain_weight_scales(hidden, H * D, 3)
    wo = b.SparseWeight(workloads.make_weight(hidden, H * D, 0.5, seed=3), s_w, max_N=16)
    wo4 = b.mx4_quantize(torch.randn(hidden, H * D, device="cuda", generator=g) / 32).freeze()
    cache = b.KVCache.new(16, Hkv, D, 64)
    table = torch.randperm(16, device="cuda", generator=g).int().view(2, 8)
    lens = [0, 0]
    for new in ([200, 70], [1, 1], [1, 1], [3, 2]):
        lens = [a + n for a, n in zip(lens, new)]
        lengths, cu = torch.tensor(lens, dtype=torch.int32, device="cuda"), (None if max(new) == 1 else cu_of(new))
        x = torch.randn(sum(new), hidden, device="cuda", generator=g).half()
        qkv = b.mx4_linear(x, wqkv)
        heads = qkv.unflatten(1, (H + 2 * Hkv, D))
        q, k, v = heads[:, :H], heads[:, H:H + Hkv], heads[:, H + Hkv:]
        want = ref_append(cache, table, lens, new, k, v)
        cache.append(k, v, table, lengths, cu)
        for got, ref in zip((cache.k_codes, cache.k_steps, cache.v_codes, cache.v_steps), want):
            assert same(got, ref)
        o = cache.attention(q, table, lengths, cu)
        ref, bound, _ = reference(cache, table, lens, new, q, D ** -0.5)
        check(o, ref, bound)
        rows = o.flatten(1)
        y = b.mx4_linear(rows, wo4, dtype=torch.float32)
        xq = b.mx4_quantize(rows).dequantize().double()
        wq = wo4.dequantize().double()
        assert ((y.double() - xq @ wq.t()).abs() <= H * D * 2.0 ** -23 * (xq.abs() @ wq.abs().t()) + 2.0 ** -24 * (xq @ wq.t()).abs()).all()
        if sum(new) <= 16:
            z = wo.spmm_requant(rows, sum(new), b.absmax_f16(rows))
            assert z.shape == (sum(new), hidden) and torch.isfinite(z).all()
    cache.check()
    b.mx4_check()
    wo.check()
    wo.close()
