"""Blocks of the 8-bit cache on the GPU against the same steps in Python: tables, counts, codes and steps are moved, never computed, and must be equal."""
import random

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


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


class Model:
    """The pool in plain Python; a block's content is a list of T tokens (any value) and a step."""

    def __init__(self, blocks, T):
        self.T, self.refs = T, [0] * blocks
        self.content = None

    def count(self, n):
        return -(-n // self.T)

    def extend(self, table, lengths, tokens):
        """True unless the blocks ran out."""
        todo = []
        last = {}
        for s, (L, n) in enumerate(zip(lengths, tokens)):
            have = self.count(L)
            part = n > 0 and L % self.T > 0 and self.refs[table[s][have - 1]] > 1
            if part:
                last.setdefault(table[s][have - 1], []).append(s)
            todo.append((self.count(L + n) - have if n else 0, part))
        plan = []
        for s, (need, part) in enumerate(todo):
            if part:
                x = table[s][self.count(lengths[s]) - 1]
                part = not (len(last[x]) >= self.refs[x] and last[x][0] == s)
            plan.append((need, part))
        free = [i for i, r in enumerate(self.refs) if r == 0]
        at, ok = 0, True
        ends, stuck = [], set()   # blocks that a sequence goes on holding for want of a copy: nobody else writes into them
        for need, part in plan:
            at += need + part
            ends.append(at)
        for s, (need, part) in enumerate(plan):
            if part and ends[s] > len(free):
                stuck.add(table[s][self.count(lengths[s]) - 1])
        keeps = {x: who[0] for x, who in last.items()}
        at = 0
        for s, (need, part) in enumerate(plan):
            all_ = need + part
            here = free[at:at + all_]
            at += all_
            block = table[s][self.count(lengths[s]) - 1] if lengths[s] else None
            if len(here) < all_ or (not part and block in stuck and keeps.get(block) == s):
                ok = False
                continue
            have = self.count(lengths[s])
            if part:
                x, y = table[s][have - 1], here.pop(0)
                self.copy(x, y, lengths[s] % self.T)
                self.refs[x] -= 1
                self.refs[y] = 1
                table[s][have - 1] = y
            for j, y in enumerate(here):
                table[s][have + j] = y
                self.refs[y] = 1
            lengths[s] += tokens[s]
        return ok

    def copy(self, x, y, held):
        for c in self.content:
            if c.dim() == 2:
                c[y] = c[x]
            else:
                c[y, :, :held] = c[x, :, :held]

    def fork(self, table, lengths, parents, keep):
        width = len(table[0])
        rows, lens = [], []
        for p in parents:
            n = 0 if p < 0 else self.count(lengths[p])
            rows.append([table[p][j] if j < n else 0 for j in range(width)])
            lens.append(0 if p < 0 else lengths[p])
            for x in rows[-1][:n]:
                self.refs[x] += 1
        if not keep:
            self.release(table, lengths)
        return rows, lens

    def release(self, table, lengths):
        for row, L in zip(table, lengths):
            for x in row[:self.count(L)]:
                self.refs[x] -= 1


def make(b, blocks, T=16, Hkv=2, D=64, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    codes = [torch.randint(-127, 128, (blocks, Hkv, T, D), device="cuda", dtype=torch.int8, generator=g) for _ in range(2)]
    steps = [torch.rand(blocks, Hkv, device="cuda", generator=g) for _ in range(2)]
    cache = b.KVCache(*codes, *steps)
    m = Model(blocks, T)
    m.content = [x.cpu().clone() for x in (*codes, *steps)]
    return cache, b.KVPages(cache), m


def same(cache, pages, m, table=None, lengths=None, rows=None, lens=None):
    assert pages.refs.tolist() == m.refs
    for x, y in zip((cache.k_codes, cache.v_codes, cache.k_steps, cache.v_steps), m.content):
        assert torch.equal(x.cpu(), y)
    if table is not None:
        assert lengths.tolist() == lens and table.tolist() == rows


@pytest.mark.parametrize("T,D,Hkv", [(16, 64, 2), (32, 128, 1), (64, 128, 3), (128, 64, 8), (256, 128, 2)])
@pytest.mark.parametrize("seed", [0, 1])
def test_a_life_of_a_pool(b, T, D, Hkv, seed):
    """Sequences grow, fork, are kept, dropped and given up, in any order, until the pool is full and beyond."""
    r = random.Random(seed)
    blocks, width = 53, 9
    cache, pages, m = make(b, blocks, T, Hkv, D, seed)
    rows, lens = [[0] * width for _ in range(4)], [0] * 4
    table, lengths = ints(rows), ints(lens)
    held = []
    for _ in range(40):
        what = r.choice(["extend", "extend", "one", "fork", "keep", "release"])
        if what in ("extend", "one"):
            tokens = [1] * len(lens) if what == "one" else [r.choice([0, 0, 1, 3, T, 2 * T + 1]) for _ in lens]
            tokens = [min(n, width * T - L) for n, L in zip(tokens, lens)]
            # (a full row takes no token)
            pages.extend(table, lengths, 1 if what == "one" and all(n == 1 for n in tokens) else ints(tokens))
            ok = m.extend(rows, lens, tokens)
            if not ok:
                with pytest.raises(b.UsError, match="free blocks"):
                    pages.check()
        elif what in ("fork", "keep"):
            parents = [r.randrange(-1, len(lens)) for _ in range(r.choice([1, 3, 4, 6]))]
            old = (table, lengths, rows, lens)
            table, lengths = pages.fork(table, lengths, ints(parents), keep=what == "keep")
            rows, lens = m.fork(rows, lens, parents, what == "keep")
            if what == "keep":
                held.append(old)
        elif held:
            t, n, tr, nl = held.pop(r.randrange(len(held)))
            pages.release(t, n)
            m.release(tr, nl)
        same(cache, pages, m, table, lengths, rows, lens)
        pages.check()
    for t, n, tr, nl in held:
        pages.release(t, n)
    pages.release(table, lengths)
    pages.check()
    assert not pages.refs.any()


def test_who_keeps_the_last_block(b):
    """Three children of a parent that is given up: the first writes on in its block, two get copies of the tokens held and no more; of a parent that stays: all three."""
    for keep in (False, True):
        cache, pages, m = make(b, 20, 16)
        rows, lens = [[0] * 4], [0]
        table, lengths = ints(rows), ints(lens)
        pages.extend(table, lengths, 21)
        m.extend(rows, lens, [21])
        child, n = pages.fork(table, lengths, ints([0, 0, 0]), keep=keep)
        crow, cn = m.fork(rows, lens, [0, 0, 0], keep)
        pages.extend(child, n)
        m.extend(crow, cn, [1, 1, 1])
        same(cache, pages, m, child, n, crow, cn)
        assert [row[1] for row in crow] == ([2, 3, 4] if keep else [1, 2, 3])
        # whole blocks need no copy: the next token goes to a block of its own
        pages.extend(child, n, 10)
        m.extend(crow, cn, [10] * 3)
        again, k = pages.fork(child, n, ints([0, 0]))
        arow, an = m.fork(crow, cn, [0, 0], False)
        pages.extend(again, k)
        m.extend(arow, an, [1, 1])
        same(cache, pages, m, again, k, arow, an)
        pages.check()


@pytest.mark.parametrize("spare", [0, 1, 2])
def test_a_block_is_not_written_while_another_holds_it(b, spare):
    """Three children, fewer free blocks than copies: the one that would write on in the parents' block waits, too, unless all others have theirs."""
    cache, pages, m = make(b, 2 + spare, 16)
    rows, lens = [[0] * 3], [0]
    table, lengths = ints(rows), ints(lens)
    pages.extend(table, lengths, 21)
    m.extend(rows, lens, [21])
    child, n = pages.fork(table, lengths, ints([0, 0, 0]))
    crow, cn = m.fork(rows, lens, [0, 0, 0], False)
    pages.extend(child, n)
    assert m.extend(crow, cn, [1, 1, 1]) == (spare == 2)
    assert cn == {0: [21, 21, 21], 1: [21, 22, 21], 2: [22, 22, 22]}[spare]
    if spare < 2:
        with pytest.raises(b.UsError, match="free blocks"):
            pages.check()
    same(cache, pages, m, child, n, crow, cn)
    pages.check()


@pytest.mark.parametrize("blocks", [1, 15, 16, 17, 16383, 16385, 40000])
def test_pools_of_many_blocks(b, blocks):
    """The lowest free blocks, wherever they are; all of them, and one more than there are."""
    r = random.Random(blocks)
    cache, pages, m = make(b, blocks, 16, 1, 64)
    taken = [r.random() < 0.9 for _ in range(blocks)]
    taken[-1] = False
    m.refs = [3 * t for t in taken]
    pages.refs.copy_(ints(m.refs))
    free = taken.count(False)
    table, lengths = torch.zeros(2, free + 1, dtype=torch.int32, device="cuda"), ints([0, 0])
    pages.extend(table, lengths, ints([16 * (free // 2), 16 * (free - free // 2)]))
    pages.check()
    where = [i for i, t in enumerate(taken) if not t]
    assert table[0, :free // 2].tolist() == where[:free // 2] and table[1, :free - free // 2].tolist() == where[free // 2:]
    assert lengths.tolist() == [16 * (free // 2), 16 * (free - free // 2)] and bool((pages.refs > 0).all())
    pages.release(table, lengths)
    table, lengths = torch.full((2, free + 1), 5, dtype=torch.int32, device="cuda"), ints([0, 0])
    pages.extend(table, lengths, ints([16 * free + 1, 1]))   # the first does not fit, and so the second does not
    with pytest.raises(b.UsError, match="free blocks"):
        pages.check()
    assert lengths.tolist() == [0, 0] and bool((table == 5).all()) and pages.refs.tolist() == m.refs


@pytest.mark.parametrize("S", [1, 31, 33, 1023, 1025, 2100])
def test_many_sequences(b, S):
    r = random.Random(S)
    cache, pages, m = make(b, 2 * S + 10, 16, 1, 64)
    rows, lens = [[0, 0] for _ in range(S)], [0] * S
    table, lengths = ints(rows), ints(lens)
    for _ in range(2):
        tokens = [r.choice([0, 1, 7, 16]) for _ in range(S)]
        pages.extend(table, lengths, ints(tokens))
        assert m.extend(rows, lens, tokens)
        same(cache, pages, m, table, lengths, rows, lens)
    parents = [r.randrange(-1, S) for _ in range(S)]
    table, lengths = pages.fork(table, lengths, ints(parents))
    rows, lens = m.fork(rows, lens, parents, False)
    same(cache, pages, m, table, lengths, rows, lens)
    tokens = [1 if n < 32 else 0 for n in lens]
    pages.extend(table, lengths, ints(tokens))
    m.extend(rows, lens, tokens)
    same(cache, pages, m, table, lengths, rows, lens)


def test_a_copy_takes_part_in_attention(b):
    """Two continuations of one prompt, each with tokens of its own, as if each had been there from the start."""
    H, D, T = 2, 128, 64
    g = torch.Generator(device="cuda").manual_seed(3)
    k, v = (torch.randn(100, H, D, device="cuda", generator=g).half() for _ in range(2))
    more = [[torch.randn(2, H, D, device="cuda", generator=g).half() for _ in range(2)] for _ in range(5)]
    q = torch.randn(2, H, D, device="cuda", generator=g).half()
    cache = b.KVCache.new(16, H, D, T)
    pages = b.KVPages(cache)
    table, lengths = torch.zeros(1, 4, dtype=torch.int32, device="cuda"), ints([0])
    pages.extend(table, lengths, 100)
    cache.append(k, v, table, lengths, ints([0, 100]))
    table, lengths = pages.fork(table, lengths, ints([0, 0]))
    for x, y in more:
        pages.extend(table, lengths)
        cache.append(x, y, table, lengths)
    out = cache.attention(q, table, lengths)
    pages.check()
    for s in range(2):
        alone = b.KVCache.new(4, H, D, T)
        t = ints([[0, 1, 2, 3]])
        alone.append(k, v, t, ints([100]), ints([0, 100]))
        for i, (x, y) in enumerate(more):
            alone.append(x[s:s + 1], y[s:s + 1], t, ints([101 + i]))
        assert torch.equal(alone.attention(q[s:s + 1], t, ints([105])), out[s:s + 1])
        for a, c in zip(alone.read(t, ints([105]), 105), cache.read(table[s:s + 1].contiguous(), lengths[s:s + 1].contiguous(), 105)):
            assert torch.equal(a, c)


@pytest.mark.parametrize("blocks", [1, 2, 17, 500, 16384, 16385, 33000])
@pytest.mark.parametrize("fill", [0.0, 0.3, 0.9, 1.0])
def test_compact(b, blocks, fill):
    r = random.Random(blocks)
    cache, pages, m = make(b, blocks, 16, 1, 64)
    ids = r.sample(range(blocks), int(fill * blocks))
    S = 3
    per = [ids[s::S] for s in range(S)]
    width = max(1, max(len(p) for p in per))
    rows = [p + [blocks + 5] * (width - len(p)) for p in per]   # (entries behind a sequence's blocks are nobody's)
    table, lengths = ints(rows), ints([max(0, 16 * len(p) - 3) for p in per])
    twin, twin_n = table[:1].clone(), lengths[:1].clone()
    for x in ids:
        m.refs[x] = 1
    for x in per[0]:
        m.refs[x] += 1
    pages.refs.copy_(ints(m.refs))
    before = [x.clone() for x in cache.read(table, lengths, 16 * width)]
    more = [(table[s:s + 1].clone(), lengths[s:s + 1].clone()) for s in (0, 1, 2, 1, 0)]
    used = pages.compact([(table, lengths), (twin, twin_n), (table[:0], lengths[:0])] + more)
    pages.check()
    n = len(ids)
    src, dst = [i for i in range(n, blocks) if m.refs[i]], [i for i in range(n) if not m.refs[i]]
    to = dict(zip(src, dst))
    for x, y in to.items():
        m.copy(x, y, 16)
        m.refs[x], m.refs[y] = 0, m.refs[x]
    assert used.dim() == 0 and int(used) == n and all(m.refs[:n]) and not any(m.refs[n:])
    same(cache, pages, m, table, lengths, [[to.get(x, x) if j < len(p) else x for j, x in enumerate(row)] for p, row in zip(per, rows)], lengths.tolist())
    assert torch.equal(twin[0, :len(per[0])], table[0, :len(per[0])])
    for (t, _), s in zip(more, (0, 1, 2, 1, 0)):   # (more tables than one launch takes)
        assert torch.equal(t[0, :len(per[s])], table[s, :len(per[s])])
    for x, y in zip(before, cache.read(table, lengths, 16 * width)):
        assert torch.equal(x, y)


def test_copy_blocks(b):
    cache, pages, m = make(b, 30, 32, 3, 128)
    src, dst = [3, 7, 9, 3, 2], [20, -1, 11, 0, 29]
    cache.copy_blocks(ints(src), ints(dst))
    for x, y in zip(src, dst):
        if y >= 0:
            m.copy(x, y, 32)
    same(cache, pages, m)
    cache.check()
    cache.copy_blocks(ints([]), ints([]))
    for s, d in ((30, 4), (-1, 4), (4, 30), (4, -2)):   # left out, and reported
        cache.copy_blocks(ints([s]), ints([d]))
        with pytest.raises(b.UsError):
            cache.check()
    same(cache, pages, m)


def test_entries_out_of_range(b):
    """What does not fit is left out and reported; counts of blocks that are there stay right."""
    def state():
        cache, pages, m = make(b, 10, 16)
        pages.refs[:4] = 1
        return cache, pages, ints([[0, 1, 0], [2, 99, 0], [3, 0, 0]]), ints([20, 20, 5])

    cache, pages, table, lengths = state()
    child, n = pages.fork(table, lengths, ints([0, 1, 7, -2, 2]), keep=True)
    with pytest.raises(b.UsError):
        pages.check()
    assert n.tolist() == [20, 20, 0, 0, 5] and pages.refs.tolist() == [2, 2, 2, 2] + [0] * 6
    cache, pages, table, lengths = state()
    pages.extend(table, lengths, 3)   # the second sequence's last block is none of the pool's
    with pytest.raises(b.UsError):
        pages.check()
    assert lengths.tolist() == [23, 20, 8] and table.tolist() == [[0, 1, 0], [2, 99, 0], [3, 0, 0]]
    for bad, tokens in (([-1, 0, 0], [1, 1, 1]), ([49, 0, 0], [1, 1, 1]), ([40, 0, 0], [9, 1, 1]), ([0, 0, 0], [-1, 1, 1])):
        cache, pages, table, _ = state()
        lengths = ints(bad)
        pages.extend(table, lengths, ints(tokens))
        with pytest.raises(b.UsError):
            pages.check()
        assert lengths.tolist() == [bad[0], 1, 1] and table[1, 0] == 4 and table[2, 0] == 5
    cache, pages, table, lengths = state()
    pages.release(table, lengths)
    with pytest.raises(b.UsError):
        pages.check()
    assert not pages.refs.any()
    pages.release(table, ints([20, 0, 0]))   # nobody holds them: they stay free
    with pytest.raises(b.UsError):
        pages.check()
    assert not pages.refs.any()
    cache, pages, table, lengths = state()
    pages.compact([(table, lengths)])
    with pytest.raises(b.UsError):
        pages.check()
    pages.check()


def test_graph_and_stream(b):
    """A step of a beam search captured once and replayed: the graph's results are those of the same calls made one by one."""
    def start():
        cache, pages, m = make(b, 40, 16, 2, 64, seed=9)
        table, lengths = torch.zeros(4, 6, dtype=torch.int32, device="cuda"), ints([0] * 4)
        pages.extend(table, lengths, 13)
        return cache, pages, table, lengths

    def step(pages, table, lengths, parents):
        t, n = pages.fork(table, lengths, parents)
        pages.extend(t, n)
        table.copy_(t)
        lengths.copy_(n)

    picks = [[0, 0, 1, 2], [3, 3, 3, 3], [0, 1, 2, 3], [1, 0, 1, 0], [2, 2, 0, 0], [0, 0, 0, 1]]
    cache, pages, table, lengths = start()
    for p in picks:
        step(pages, table, lengths, ints(p))
    pages.check()
    c2, p2, t2, n2 = start()
    parents = ints(picks[0])
    refs, held = p2.refs.clone(), (t2.clone(), n2.clone())
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        step(p2, t2, n2, parents)
    assert torch.equal(p2.refs, refs) and torch.equal(t2, held[0])   # (captured, not run)
    for p in picks:
        parents.copy_(ints(p))
        graph.replay()
    torch.cuda.synchronize()
    p2.check()
    assert torch.equal(t2, table) and torch.equal(n2, lengths) and torch.equal(p2.refs, pages.refs)
    for x, y in zip((cache.k_codes, cache.v_codes, cache.k_steps, cache.v_steps), (c2.k_codes, c2.v_codes, c2.k_steps, c2.v_steps)):
        assert torch.equal(x, y)
    st.wait_stream(torch.cuda.current_stream())
    p2.extend(t2, n2, 2, stream=st.cuda_stream)
    p2.release(t2, n2, stream=st.cuda_stream)
    st.synchronize()
    p2.check()
    assert not p2.refs.any()


def test_refusals(b):
    cache, pages, m = make(b, 10, 16)
    table, lengths = torch.zeros(2, 3, dtype=torch.int32, device="cuda"), ints([0, 0])
    for call in (lambda: b.KVPages(cache, torch.zeros(9, dtype=torch.int32, device="cuda")), lambda: b.KVPages(cache, torch.zeros(10, dtype=torch.int64, device="cuda")),
                 lambda: b.KVPages(cache, torch.zeros(10, dtype=torch.int32)), lambda: b.KVPages(cache, torch.zeros(11, dtype=torch.int32, device="cuda")[1:]),
                 lambda: pages.extend(table.long(), lengths), lambda: pages.extend(table, lengths[:1]), lambda: pages.extend(table, lengths, -1),
                 lambda: pages.extend(table, lengths, ints([1])), lambda: pages.extend(table, lengths, 1 << 31), lambda: pages.fork(table, lengths, ints([0]).long()),
                 lambda: pages.fork(table, lengths, torch.zeros(1, dtype=torch.int32)), lambda: pages.release(table.t(), lengths),
                 lambda: pages.compact([(table, lengths), (table.cpu(), lengths)]), lambda: cache.copy_blocks(ints([1]), ints([1, 2]))):
        with pytest.raises(ValueError):
            call()
    assert not pages.refs.any()
    none = torch.zeros(0, 3, dtype=torch.int32, device="cuda")
    pages.extend(none, ints([]))
    pages.release(none, ints([]))
    t, n = pages.fork(none, ints([]), ints([-1, -1]))
    assert t.shape == (2, 3) and n.tolist() == [0, 0] and int(pages.compact([])) == 0
    t, n = pages.fork(table, lengths, ints([]))
    assert t.shape == (0, 3) and n.numel() == 0
    pages.check()
