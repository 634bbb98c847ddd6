"""Blocks that nobody holds, met by fork, release and extend: reported every time; and forks of many children and wide tables, which never are."""
import random

import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

from test_gpu_pages import Model, b, ints, make, same  # noqa: F401


@pytest.mark.parametrize("keep", [True, False])
@pytest.mark.parametrize("parents", [[0], [1], [0, 0, 0], [1, 0], [-1, 1, 1, 0], [2, 1], [1] * 40])
def test_fork(b, keep, parents):  # noqa: F811
    """Sequence 1 has a block that is free; whoever continues it is told so, in whatever order the rows are done. The children have what the parents had."""
    for _ in range(20):
        cache, pages, m = make(b, 10, 16)
        m.refs = [1, 1, 1, 0, 1, 0, 0, 0, 0, 0]
        pages.refs.copy_(ints(m.refs))
        rows, lens = [[0, 1], [2, 3], [4, 0]], [20, 30, 3]
        table, lengths = pages.fork(ints(rows), ints(lens), ints(parents), keep=keep)
        if keep and 1 not in parents:
            pages.check()
        else:
            with pytest.raises(b.UsError, match="out of range"):
                pages.check()
        assert lengths.tolist() == [0 if p < 0 else lens[p] for p in parents]
        assert table.tolist() == [[0, 0] if p < 0 else [x if j < -(-lens[p] // 16) else 0 for j, x in enumerate(rows[p])] for p in parents]
        want = [n + sum(parents.count(p) for p in range(3) if x in rows[p][:-(-lens[p] // 16)]) for x, n in enumerate(m.refs)]
        if not keep:
            want = [max(0, n - (x in (0, 1, 2, 3, 4))) for x, n in enumerate(want)]
        assert pages.refs.tolist() == want
        pages.check()


def test_extend(b):  # noqa: F811
    """A sequence whose last, partly filled block is free stays as it is; where no token goes into that block, it is not looked at."""
    cache, pages, m = make(b, 10, 16)
    pages.refs[:3] = 1
    table, lengths = ints([[0, 0, 0], [7, 0, 0], [1, 8, 0], [2, 9, 0]]), ints([5, 5, 32, 20])
    pages.extend(table, lengths, ints([1, 1, 1, 0]))
    with pytest.raises(b.UsError, match="out of range"):
        pages.check()
    assert lengths.tolist() == [6, 5, 33, 20] and table.tolist() == [[0, 0, 0], [7, 0, 0], [1, 8, 3], [2, 9, 0]]
    assert pages.refs.tolist() == [1, 1, 1, 1] + [0] * 6


@pytest.mark.parametrize("S,C,width", [(3, 5, 300), (40, 200, 3), (300, 1024, 2), (1024, 1024, 1), (300, 1025, 2), (4096, 4096, 1), (2, 9000, 2), (5000, 5000, 1)])
@pytest.mark.parametrize("keep", [True, False])
def test_many_children(b, S, C, width, keep):  # noqa: F811
    """Counts are those of the same steps in Python, and nothing is reported: sequences in any order, without children, and of blocks that several parents share."""
    r = random.Random(S + C)
    blocks = S * width
    cache, pages, m = make(b, blocks, 16, 1, 64)
    lens = [r.randrange(16 * width + 1) for _ in range(S)]
    rows = [[s * width + j for j in range(width)] for s in range(S)]
    for s in range(1, S, 3):
        rows[s], lens[s] = list(rows[s - 1]), lens[s - 1]
    for row, n in zip(rows, lens):
        for x in row[:m.count(n)]:
            m.refs[x] += 1
    pages.refs.copy_(ints(m.refs))
    for parents in ([r.randrange(-1, S) for _ in range(C)], [S - 1] * C, [i % S for i in range(C)], [S - 1 - i % S for i in range(C)]):
        refs = list(m.refs)
        table, lengths = pages.fork(ints(rows), ints(lens), ints(parents), keep=keep)
        crow, clen = m.fork(rows, lens, parents, keep)
        same(cache, pages, m, table, lengths, crow, clen)
        pages.check()
        m.refs = refs
        pages.refs.copy_(ints(refs))
