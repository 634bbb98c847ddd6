"""A pool that runs full in the middle of a step: what `extend` had no room for is left alone by `append`, and the step can be finished later."""
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

from test_gpu_pages import b, ints  # noqa: F401

H, D, T = 2, 64, 16


def tokens(n, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return [torch.randn(n, H, D, device="cuda", generator=g).half() * (1 + seed % 3) for _ in range(2)]   # (steps that grow)


def prompt(b, blocks, n, children, width=5):  # noqa: F811
    """Children of one prompt of n tokens, which is given up."""
    cache = b.KVCache.new(blocks, H, D, T)
    pages = b.KVPages(cache)
    table, lengths, granted = torch.zeros(1, width, dtype=torch.int32, device="cuda"), ints([0]), ints([-1])
    pages.extend(table, lengths, n, granted=granted)
    assert granted.tolist() == [n]
    cache.append(*tokens(n, 1), table, lengths, ints([0, n]), granted=granted)
    table, lengths = pages.fork(table, lengths, ints([0] * children))
    return cache, pages, table, lengths


def codes(cache):
    return [x.clone() for x in (cache.k_codes, cache.v_codes, cache.k_steps, cache.v_steps)]


# a prompt of whole blocks: the last token's block is shared by all; one that ends inside a block: copies; one new token or several
@pytest.mark.parametrize("n,new,children,blocks", [(16, 1, 3, 3), (16, 1, 3, 1), (21, 1, 3, 3), (21, 1, 3, 2), (32, 20, 4, 6), (40, 30, 5, 9), (16, 1, 40, 20)])
def test_a_step_that_does_not_fit_and_is_finished_later(b, n, new, children, blocks):  # noqa: F811
    cache, pages, table, lengths = prompt(b, blocks, n, children)
    held = [x.clone() for x in cache.read(table, lengths, n)]
    granted = torch.full((children,), -1, dtype=torch.int32, device="cuda")
    x, cu = tokens(children * new, 2), ints([new * i for i in range(children + 1)])
    pages.extend(table, lengths, new, granted=granted)
    with pytest.raises(b.UsError, match="free blocks"):
        pages.check()
    fit = [g == new for g in granted.tolist()]
    assert not all(fit) and set(granted.tolist()) <= {0, new} and lengths.tolist() == [n + g for g in granted.tolist()]
    before, tables = codes(cache), table.tolist()
    cache.append(*x, table, lengths, None if new == 1 else cu, granted=granted)
    pages.check()
    mine = {t for s in range(children) if fit[s] for t in tables[s][n // T:-(-(n + new) // T)]}   # blocks that may be written
    rest = [i for i in range(blocks) if i not in mine]
    for old, now in zip(before, codes(cache)):
        assert torch.equal(old[rest], now[rest])
    now = cache.read(table, lengths, n)
    for s in range(children):
        if not fit[s]:
            assert torch.equal(now[0][s], held[0][s]) and torch.equal(now[1][s], held[1][s])
    # a pool with room holds the same prompt, and the same tokens for those that fitted; then the others get theirs
    big, bpages, btable, blengths = prompt(b, 8 * children + 8, n, children)
    more = b.KVCache.new(8 * children + 8, H, D, T)
    for a, c in ((more.k_codes, cache.k_codes), (more.v_codes, cache.v_codes), (more.k_steps, cache.k_steps), (more.v_steps, cache.v_steps)):
        a[:blocks] = c
    mpages = b.KVPages(more)
    mpages.refs[:blocks] = pages.refs
    g2 = torch.full_like(granted, -1)
    mpages.extend(table, lengths, new - granted, granted=g2)
    assert g2.tolist() == [new - g for g in granted.tolist()]
    more.append(*x, table, lengths, cu, granted=g2)   # (those that have theirs are granted 0, and left out)
    bpages.extend(btable, blengths, new)
    big.append(*x, btable, blengths, cu)
    mpages.check()
    assert torch.equal(lengths, blengths)
    for y, z in zip(more.read(table, lengths, n + new), big.read(btable, blengths, n + new)):
        assert torch.equal(y, z)


def test_what_does_not_fit_otherwise(b):  # noqa: F811
    """Entries and lengths out of range grant nothing; nor does a sequence without new tokens."""
    cache = b.KVCache.new(20, H, D, T)
    pages = b.KVPages(cache)
    pages.refs[:4] = 1
    table, lengths = ints([[0, 1, 0], [2, 99, 0], [3, 0, 0], [0, 0, 0], [0, 0, 0]]), ints([20, 20, 5, 49, 0])
    granted = ints([-1] * 5)
    pages.extend(table, lengths, ints([3, 3, 0, 1, 7]), granted=granted)
    with pytest.raises(b.UsError):
        pages.check()
    assert granted.tolist() == [3, 0, 0, 0, 7] and lengths.tolist() == [23, 20, 5, 49, 7]


@pytest.mark.parametrize("S", [1000, 2100])
def test_many_sequences(b, S):  # noqa: F811
    cache = b.KVCache.new(S, H, D, T)
    pages = b.KVPages(cache)
    table, lengths = torch.zeros(S, 2, dtype=torch.int32, device="cuda"), torch.zeros(S, dtype=torch.int32, device="cuda")
    want, granted = torch.arange(S, device="cuda").int() % 33, torch.full((S,), -1, dtype=torch.int32, device="cuda")
    pages.extend(table, lengths, want, granted=granted)
    assert torch.equal(granted, lengths) and torch.equal(granted[granted > 0], want[granted > 0])
    assert bool((granted != want).any())
    with pytest.raises(b.UsError, match="free blocks"):
        pages.check()


def test_captured(b):  # noqa: F811
    """A captured step, replayed until the pool is full and beyond: contents of those that stay behind do not change."""
    cache, pages, table, lengths = prompt(b, 6, 30, 3)
    granted = torch.zeros(3, dtype=torch.int32, device="cuda")
    x = tokens(3, 5)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        pages.extend(table, lengths, 1, granted=granted)
        cache.append(*x, table, lengths, granted=granted)
    old, full = lengths.tolist(), 0
    for step in range(24):
        was = [t.clone() for t in cache.read(table, lengths, 64)]
        x[0].normal_(), x[1].normal_()
        graph.replay()
        torch.cuda.synchronize()
        got = granted.tolist()
        assert lengths.tolist() == [a + g for a, g in zip(old, got)]
        now = cache.read(table, lengths, 64)
        for s in range(3):
            if got[s] == 0:
                full += 1
                assert torch.equal(now[0][s], was[0][s]) and torch.equal(now[1][s], was[1][s])
        old = lengths.tolist()
    assert 0 < full
    with pytest.raises(b.UsError, match="free blocks"):
        pages.check()


def test_refusals(b):  # noqa: F811
    cache, pages, table, lengths = prompt(b, 10, 16, 3)
    x = tokens(3, 0)
    for g in (torch.zeros(2, dtype=torch.int32, device="cuda"), torch.zeros(3, dtype=torch.int64, device="cuda"), torch.zeros(3, dtype=torch.int32),
              torch.zeros(6, dtype=torch.int32, device="cuda")[::2], torch.zeros(1, 3, dtype=torch.int32, device="cuda")):
        with pytest.raises(ValueError):
            pages.extend(table, lengths, 1, granted=g)
        with pytest.raises(ValueError):
            cache.append(*x, table, lengths, granted=g)
    assert lengths.tolist() == [16] * 3
    none = table[:0]
    pages.extend(none, lengths[:0], 1, granted=lengths[:0])
    pages.check()
