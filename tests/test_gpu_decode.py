"""A decoder layer of several continuations of two prompts, as a program runs it: projection with bias, norms and rotation of the heads, blocks of the cache shared by
fork and extend, append, attention behind the shared blocks, projections with residual and gate. Each stage against its definition on the device's own input (the
bounds of the stages' own tests); and captured once and replayed."""
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

import test_gpu_epilogue as epilogue
import test_gpu_heads as heads
import test_gpu_shared as shared

H, HKV, D, T, HIDDEN, FFN = 8, 2, 128, 64, 512, 768
EPS = 1e-5


@pytest.fixture(scope="module")
def b():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a CUDA device")
    from paper_2608_09291_b200 import binding
    torch.cuda.set_device(0)
    return binding


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


class Layer:
    def __init__(self, b, seed):
        g = torch.Generator(device="cuda").manual_seed(seed)
        rnd = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
        self.b = b
        self.qkv, self.o = (b.mx4_quantize(rnd(n, k) / k ** 0.5).freeze() for n, k in (((H + 2 * HKV) * D, HIDDEN), (HIDDEN, H * D)))
        self.gate_up, self.down = (b.mx4_quantize(rnd(n, k) / k ** 0.5).freeze() for n, k in ((2 * FFN, HIDDEN), (HIDDEN, FFN)))
        self.bias, self.qw, self.kw = rnd((H + 2 * HKV) * D).half(), (1 + 0.1 * rnd(D)).half(), (1 + 0.1 * rnd(D)).half()
        self.rotary = b.Rotary(D, base=500000.0)
        self.cache = b.KVCache.new(40, HKV, D, T)
        self.pages = b.KVPages(self.cache)

    def attend_in(self, x, positions, table, lengths, cu):
        """Projection, heads, append; returns what attention reads, and the stages' values."""
        qkv = self.b.mx4_linear(x, self.qkv, bias=self.bias)
        h = qkv.unflatten(1, (H + 2 * HKV, D))
        q, k = self.b.qk_norm_rope(h[:, :H], h[:, H:H + HKV], positions, self.rotary, self.qw, self.kw, eps=EPS)
        self.cache.append(k, h[:, H + HKV:], table, lengths, cu)
        return qkv, q, k

    def finish(self, x, o):
        y = self.b.mx4_linear(o.flatten(1), self.o, residual=x)
        f = self.b.mx4_linear(y, self.gate_up, act="silu", gated=True)
        return y, f, self.b.mx4_linear(f, self.down, residual=y)


def values(w):
    return w.dequantize()


def test_continuations(b):
    m = Layer(b, 1)
    g = torch.Generator(device="cuda").manual_seed(2)
    new = [200, 130]
    table, lengths = torch.zeros(2, 6, dtype=torch.int32, device="cuda"), ints([0, 0])
    m.pages.extend(table, lengths, ints(new))
    x = torch.randn(sum(new), HIDDEN, device="cuda", generator=g).half()
    m.attend_in(x, torch.cat([torch.arange(n, device="cuda") for n in new]).int(), table, lengths, ints([0, 200, 330]))
    m.pages.check()
    prompt, plens = table[:, :2].clone(), ints([2 * T, 2 * T])           # whole blocks that all continuations share
    table, lengths = m.pages.fork(table, lengths, ints([0, 0, 0, 1, 1]))
    cu_seqs, group = ints([0, 3, 5]), [0, 0, 0, 1, 1]
    for parents in ([0, 1, 2, 3, 4], [1, 1, 0, 4, 4], [2, 0, 0, 3, 4], [0, 0, 0, 3, 3]):
        table, lengths = m.pages.fork(table, lengths, ints(parents))
        m.pages.extend(table, lengths)
        x = torch.randn(5, HIDDEN, device="cuda", generator=g).half()
        positions = lengths - 1
        qkv, q, k = m.attend_in(x, positions, table, lengths, None)
        epilogue.check(qkv, values(b.mx4_quantize(x)), values(m.qkv), m.bias, None, False, None)
        hd = qkv.unflatten(1, (H + 2 * HKV, D))
        freq = [500000.0 ** (-2 * i / D) for i in range(D // 2)]
        for got, raw, w in ((q, hd[:, :H], m.qw), (k, hd[:, H:H + HKV], m.kw)):
            heads.check(got, *heads.reference(raw, w, positions[None], freq, [0] * (D // 2), D, False, EPS))
        o = m.cache.shared_attention(q, prompt, plens, cu_seqs, table[:, 2:], lengths - 2 * T)
        m.pages.check()
        own = [n - 2 * T for n in lengths.tolist()]
        ref, bound, _ = shared.reference(m.cache, prompt, [2 * T] * 2, group, table[:, 2:], own, [1] * 5, q, D ** -0.5)
        shared.check(o, ref, bound)
        shared.check(m.cache.attention(q, table, lengths), ref, bound)   # each for itself
        y, f, z = m.finish(x, o)
        epilogue.check(y, values(b.mx4_quantize(o.flatten(1))), values(m.o), None, None, False, x)
        epilogue.check(f, values(b.mx4_quantize(y)), values(m.gate_up), None, "silu", True, None)
        epilogue.check(z, values(b.mx4_quantize(f)), values(m.down), None, None, False, y)
    assert lengths.tolist() == [204, 204, 204, 134, 134]
    before = [t.clone() for t in m.cache.read(table, lengths, 6 * T)]
    used = m.pages.compact([(table, lengths), (prompt, plens)])
    m.pages.check()
    assert int(used) == int((m.pages.refs > 0).sum()) and bool((m.pages.refs[:int(used)] > 0).all())
    for x, y in zip(before, m.cache.read(table, lengths, 6 * T)):
        assert torch.equal(x, y)
    b.mx4_check()


def test_a_step_captured_and_replayed(b):
    """The graph of one step of a beam search, replayed with other beams and tokens: what the same calls give one by one."""
    def start():
        m = Layer(b, 3)
        g = torch.Generator(device="cuda").manual_seed(4)
        table, lengths = torch.zeros(1, 5, dtype=torch.int32, device="cuda"), ints([0])
        m.pages.extend(table, lengths, 150)
        m.attend_in(torch.randn(150, HIDDEN, device="cuda", generator=g).half(), torch.arange(150, device="cuda").int(), table, lengths, ints([0, 150]))
        prompt = table[:, :2].clone()
        table, lengths = m.pages.fork(table, lengths, ints([0] * 4))
        return m, prompt, ints([2 * T]), ints([0, 4]), table, lengths

    def step(m, prompt, plen, cu_seqs, table, lengths, parents, x):
        t, n = m.pages.fork(table, lengths, parents)
        m.pages.extend(t, n)
        _, q, _ = m.attend_in(x, n - 1, t, n, None)
        _, _, z = m.finish(x, m.cache.shared_attention(q, prompt, plen, cu_seqs, t[:, 2:], n - 2 * T))
        table.copy_(t)
        lengths.copy_(n)
        return z

    g = torch.Generator(device="cuda").manual_seed(5)
    beams = [([0, 1, 2, 3], torch.randn(4, HIDDEN, device="cuda", generator=g).half()) for _ in range(1)] + [
        (p, torch.randn(4, HIDDEN, device="cuda", generator=g).half()) for p in ([0, 0, 0, 0], [3, 1, 1, 2], [2, 2, 3, 3], [1, 0, 0, 0])]
    one = start()
    want = [step(*one, ints(p), x).clone() for p, x in beams]
    two = start()
    parents, x = ints(beams[0][0]), beams[0][1].clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        z = step(*two, parents, x)
    for (p, y), w in zip(beams, want):
        parents.copy_(ints(p))
        x.copy_(y)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(z, w)
    assert torch.equal(one[4], two[4]) and torch.equal(one[5], two[5]) and torch.equal(one[0].pages.refs, two[0].pages.refs)
    two[0].pages.check()
    b.mx4_check()
