"""Cases of the operators that complete a decoder layer on low-bit weights and let many continuations share one cache.

``linear``    ``mx4_linear`` with what follows a projection in its epilogue: bias, activation (gated or not), residual.
``heads``     ``qk_norm_rope``: the norm of every query and key head and the rotation of its position, in one pass; positions with one
              axis (text) or several (time, height, width).
``fork``      ``KVPages``: continuations of a batch of sequences share their blocks (``fork``), get room for new tokens, with a copy of the
              block that they would write into (``extend``), and are given up again (``release``).
``compact``   ``KVPages.compact``: the blocks in use move to the front of the pool.
``shared``    ``KVCache.shared_attention``: attention of sequences over a prefix that groups of them share and the tokens of their own.

The listed shapes are the LLaMA-2-7B / 70B shaped layers of this repository's configurations and odd ones that divide into nothing.
"""
from __future__ import annotations

import math
import random

import torch

own = False

BLOCK = 32                                   # columns that share an MX scale
TYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
BYTES = {"f16": 2, "bf16": 2, "f32": 4}
EPS = 1e-6


def listed():
    def linear(name, N, M, K, x, act, gated=False, bias=False, residual=False):
        return {"name": name, "op": "linear", "N": N, "M": M, "K": K, "x": x, "act": act, "gated": gated, "bias": bias, "residual": residual}

    def heads(name, N, Hq, Hkv, D, rotary, axes, x, interleaved=False, norm=True):
        return {"name": name, "op": "heads", "N": N, "Hq": Hq, "Hkv": Hkv, "D": D, "rotary": rotary, "axes": axes, "x": x, "interleaved": interleaved,
                "norm": norm}

    def fork(name, S, C, L, n, T, Hkv, D):
        return {"name": name, "op": "fork", "S": S, "C": C, "L": L, "n": n, "T": T, "Hkv": Hkv, "D": D}

    def shared(name, groups, S, P, L, n, Hq, Hkv, D, T, x):
        return {"name": name, "op": "shared", "groups": groups, "S": S, "P": P, "L": L, "n": n, "Hq": Hq, "Hkv": Hkv, "D": D, "T": T, "x": x}

    return [
        # a decode step of one user: gate and up projections of a 7B-shaped FFN
        linear("linear_1x22016x4096_gated", 1, 22016, 4096, "f16", "silu", gated=True),
        # a prompt through the same projections; everything that an epilogue can do
        linear("linear_4096x22016x4096_gated", 4096, 22016, 4096, "bf16", "silu", gated=True, bias=True, residual=True),
        # sizes that divide into nothing, added to the hidden state
        linear("linear_33x1001x2003_gelu", 33, 1001, 2003, "f16", "gelu", bias=True, residual=True),
        # one token (decode), 64 query heads and 8 key heads
        heads("heads_1x64x8x128", 1, 64, 8, 128, 128, 1, "f16"),
        # a prompt with an image: three axes
        heads("heads_8192x64x8x128_3axes", 8192, 64, 8, 128, 128, 3, "bf16"),
        # part of a head is rotated, neighbours are pairs, 32 bits
        heads("heads_1001x32x32x80_part", 1001, 32, 32, 80, 32, 1, "f32", interleaved=True, norm=False),
        # 8 beams of one prompt, one token each; 16 samples of each of 16 prompts
        fork("fork_8_of_1x1000", 1, 8, 1000, 1, 64, 8, 128),
        fork("fork_256_of_16x4000", 16, 256, 4000, 1, 64, 8, 128),
        # a small pool with a few holes; a large one half full, in disorder
        {"name": "compact_300x16", "op": "compact", "blocks": 300, "S": 5, "fill": 0.9, "T": 16, "Hkv": 32, "D": 128},
        {"name": "compact_4096x64", "op": "compact", "blocks": 4096, "S": 32, "fill": 0.5, "T": 64, "Hkv": 8, "D": 128},
        # 4 beams behind a prompt of 1000 tokens (7B-shaped)
        shared("shared_1x4_1000", 1, 4, 1000, 30, 1, 32, 32, 128, 64, "f16"),
        # 64 samples of one long prompt (70B-shaped)
        shared("shared_1x64_8192", 1, 64, 8192, 512, 1, 64, 8, 128, 64, "bf16"),
    ]


def draw(rng):
    """One more case of the same ranges: sizes spread over their logarithm, any remainder."""
    def size(lo, hi):
        return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))

    most = [work(c) for c in listed()]
    flops, data = max(w["flops"] for w in most), max(w["bytes"] for w in most)
    while True:
        op = rng.choice(["linear", "linear", "heads", "heads", "fork", "compact", "shared", "shared"])
        x = rng.choice(["f16", "bf16", "f32"])
        if op == "linear":
            c = {"op": op, "N": size(1, 4096), "M": size(64, 28672), "K": size(32, 16384), "x": x, "act": rng.choice(["none", "relu", "silu", "gelu", "gelu_tanh"]),
                 "gated": rng.random() < 0.5, "bias": rng.random() < 0.5, "residual": rng.random() < 0.5}
            if rng.random() < 0.5:   # widths of models divide well
                c["M"], c["K"] = -(-c["M"] // 128) * 128, -(-c["K"] // 128) * 128
            c["M"] += c["M"] % 2 if c["gated"] else 0
        elif op == "heads":
            Hkv, D = rng.choice([1, 2, 4, 8, 32]), rng.choice([64, 80, 96, 128, 192, 256])
            c = {"op": op, "N": size(1, 8192), "Hq": Hkv * rng.choice([1, 2, 4, 7, 8]), "Hkv": Hkv, "D": D,
                 "rotary": rng.choice([D, D, D // 2, D // 4 * 2, 32]), "axes": rng.choice([1, 1, 2, 3]), "x": x, "interleaved": rng.random() < 0.3,
                 "norm": rng.random() < 0.7}
        elif op == "fork":
            c = {"op": op, "S": size(1, 64), "C": 0, "L": size(1, 8192), "n": 1 if rng.random() < 0.6 else size(2, 200), "T": rng.choice([16, 32, 64, 128]),
                 "Hkv": rng.choice([1, 2, 4, 8, 32]), "D": rng.choice([64, 128])}
            c["C"] = size(1, 256)
            if pool_of(c) * c["T"] * c["Hkv"] * c["D"] > 1 << 29:
                continue
        elif op == "compact":
            c = {"op": op, "blocks": size(2, 20000), "S": size(1, 64), "fill": round(rng.uniform(0.05, 0.95), 2), "T": rng.choice([16, 32, 64, 128]),
                 "Hkv": rng.choice([1, 2, 4, 8, 32]), "D": rng.choice([64, 128])}
            if c["blocks"] * c["T"] * c["Hkv"] * c["D"] > 1 << 29:
                continue
        else:
            Hkv = rng.choice([1, 2, 4, 8, 32])
            groups = 1 if rng.random() < 0.5 else size(1, 8)
            c = {"op": op, "groups": groups, "S": groups - 1 + size(1, 64), "P": size(1, 16384), "L": 0, "n": 1 if rng.random() < 0.6 else size(2, 64),
                 "Hq": Hkv * rng.choice([1, 2, 4, 7, 8][:5 if Hkv <= 8 else 1]), "Hkv": Hkv, "D": rng.choice([64, 128]), "T": rng.choice([16, 32, 64, 128]),
                 "x": rng.choice(["f16", "bf16"])}
            c["L"] = size(1, 2048) + c["n"] - 1
            if c["S"] * c["Hq"] * c["n"] * (c["P"] + c["L"]) > 5e8 or (groups * c["P"] + c["S"] * c["L"]) * Hkv * c["D"] > 1 << 28:
                continue
        w = work(c)
        if w["flops"] <= flops and w["bytes"] <= data:
            return c


# ---- the state ----------------------------------------------------------------------------------------------------------

def sequences(c):
    """Lengths that the case alone decides: plain lists. fork: tokens of each parent, parent of each child; compact: blocks of each sequence;
    shared: sequences and prefix tokens of each group, own tokens and new tokens of each sequence."""
    r = random.Random(repr(sorted((k, v) for k, v in c.items() if k != "name")))
    if c["op"] == "fork":
        lens = [c["L"]] + [r.randint(1, c["L"]) for _ in range(c["S"] - 1)]
        parents = sorted(r.randrange(c["S"]) for _ in range(c["C"]))
        return lens, parents
    if c["op"] == "compact":
        total = max(1, int(c["fill"] * c["blocks"]))
        cuts = sorted(r.randint(0, total) for _ in range(c["S"] - 1))
        return [b - a for a, b in zip([0] + cuts, cuts + [total])]
    g, S = c["groups"], c["S"]
    cuts = sorted(r.sample(range(1, S), g - 1))
    count = [b - a for a, b in zip([0] + cuts, cuts + [S])]
    prefix = [c["P"]] + [r.randint(1, c["P"]) for _ in range(g - 1)]
    new = [c["n"] if s == 0 or c["n"] == 1 else r.randint(1, c["n"]) for s in range(S)]
    lens = [c["L"]] + [r.randint(new[s], c["L"]) for s in range(1, S)]
    return count, prefix, lens, new


def pool_of(c):
    """Blocks of a fork's pool: the parents', what the children can need, and some that stay free."""
    T = c["T"]
    return c["S"] * -(-c["L"] // T) + c["C"] * (2 + -(-c["n"] // T)) + 16


def scattered(counts, order):
    """A block table with these numbers of blocks a row, block numbers from `order` in turn: int32 on the host."""
    table = torch.zeros(len(counts), max(1, max(counts)), dtype=torch.int32)
    at = 0
    for s, b in enumerate(counts):
        table[s, :b] = order[at:at + b]
        at += b
    return table


def pool(st, blocks, Hkv, T, D, g):
    for name in ("k", "v"):
        codes = torch.empty(blocks, Hkv, T, D, dtype=torch.int8, device="cuda")
        for b in range(0, blocks, 4096):
            part = codes[b:b + 4096]
            part.copy_(torch.randn(part.shape, device="cuda", dtype=torch.float16, generator=g).mul_(32).round_().clamp_(-127, 127))
        st[name + "_codes"] = codes
        st[name + "_steps"] = (0.7 + 0.7 * torch.rand(blocks, Hkv, device="cuda", generator=g)) / 32
    if own:
        from paper_2608_09291_b200 import binding
        st["cache"] = binding.KVCache(st["k_codes"], st["v_codes"], st["k_steps"], st["v_steps"])


def pairs_of(c):
    """Pairs that each axis of the positions turns."""
    n = c["rotary"] // 2
    if c["axes"] == 1:
        return [n]
    first = n // 4 if c["axes"] == 3 else n // 2
    rest = n - first
    return [first, rest] if c["axes"] == 2 else [first, rest // 2, rest - rest // 2]


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    op = case["op"]
    st = {"case": case}
    if op == "linear":
        N, M, K, t = case["N"], case["M"], case["K"], TYPES[case["x"]]
        # hidden states: a spread of their own for each token, a few channels much larger
        x = torch.randn(N, K, device="cuda", generator=g)
        x *= 0.2 + 2.8 * torch.rand(N, 1, device="cuda", generator=g)
        x *= 1 + 7 * (torch.rand(K, device="cuda", generator=g) < 1 / 256)
        st["x"] = x.to(t)
        st["w_codes"], st["w_scales"] = mx4_codes(torch.randn(M, K, device="cuda", generator=g) * 0.02)
        out = M // 2 if case["gated"] else M
        st["bias"] = (torch.randn(M, device="cuda", generator=g) * 0.1).to(t) if case["bias"] else None
        st["residual"] = torch.randn(N, out, device="cuda", generator=g).to(t) if case["residual"] else None
        if own:   # a program holds its weights in the form that the product reads
            from paper_2608_09291_b200 import binding
            st["w"] = binding.mx4_from_codes(st["w_codes"], st["w_scales"], K)
        return st
    if op == "heads":
        N, Hq, Hkv, D, t = case["N"], case["Hq"], case["Hkv"], case["D"], TYPES[case["x"]]
        qkv = torch.randn(N, Hq + 2 * Hkv, D, device="cuda", generator=g)
        qkv *= 0.3 + 2 * torch.rand(N, Hq + 2 * Hkv, 1, device="cuda", generator=g)
        qkv = qkv.to(t)   # one stacked projection's output; q and k are columns of it
        st["q"], st["k"] = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv]
        st["q_weight"] = (1 + 0.2 * torch.randn(D, device="cuda", generator=g)).to(t) if case["norm"] else None
        st["k_weight"] = (1 + 0.2 * torch.randn(D, device="cuda", generator=g)).to(t) if case["norm"] else None
        # places behind an earlier part of the text, up to 131072; an image's patches have a row and a column
        first = int(torch.randint(0, 131072 - N, (1,), device="cuda", generator=g))
        pos = torch.arange(first, first + N, device="cuda", dtype=torch.int32)
        if case["axes"] > 1:
            side = max(1, int(math.sqrt(N)))
            i = torch.arange(N, device="cuda", dtype=torch.int32)
            pos = torch.stack([pos - i % 7, first + i // side, first + i % side][:case["axes"]])
        st["positions"] = pos
        if own:
            from paper_2608_09291_b200 import binding
            st["rotary"] = binding.Rotary(D, base=500000.0, rotary_dim=case["rotary"], interleaved=case["interleaved"], sections=pairs_of(case))
        return st
    if op == "fork":
        S, T = case["S"], case["T"]
        lens, parents = sequences(case)
        blocks = pool_of(case)
        order = torch.randperm(blocks, device="cuda", generator=g).to(torch.int32)   # blocks in use lie anywhere in the pool
        counts = [-(-n // T) for n in lens]
        table = torch.zeros(S, -(-(case["L"] + case["n"]) // T), dtype=torch.int32)
        rows = scattered(counts, order.cpu())
        table[:, :rows.shape[1]] = rows
        st["table"], st["lengths"] = table.cuda(), torch.tensor(lens, dtype=torch.int32).cuda()
        st["parents"] = torch.tensor(parents, dtype=torch.int32).cuda()
        st["refs"] = torch.zeros(blocks, dtype=torch.int32, device="cuda")
        st["refs"][order[:sum(counts)].long()] = 1
        pool(st, blocks, case["Hkv"], T, case["D"], g)
        if own:
            from paper_2608_09291_b200 import binding
            st["pages"] = binding.KVPages(st["cache"], st["refs"])
        return st
    if op == "compact":
        counts, T = sequences(case), case["T"]
        order = torch.randperm(case["blocks"], device="cuda", generator=g).to(torch.int32)
        st["saved_table"] = scattered(counts, order.cpu()).cuda()
        st["lengths"] = torch.tensor([b * T for b in counts], dtype=torch.int32).cuda()
        st["saved_refs"] = torch.zeros(case["blocks"], dtype=torch.int32, device="cuda")
        st["saved_refs"][order[:sum(counts)].long()] = 1
        st["table"], st["refs"] = st["saved_table"].clone(), st["saved_refs"].clone()
        pool(st, case["blocks"], case["Hkv"], T, case["D"], g)
        if own:
            from paper_2608_09291_b200 import binding
            st["pages"] = binding.KVPages(st["cache"], st["refs"])
        return st
    Hq, Hkv, D, T = (case[k] for k in ("Hq", "Hkv", "D", "T"))
    count, prefix, lens, new = sequences(case)
    counts = [-(-n // T) for n in prefix + lens]
    order = torch.randperm(sum(counts), device="cuda", generator=g).to(torch.int32).cpu()
    G = case["groups"]
    st["prefix_table"] = scattered(counts[:G], order).cuda()
    st["table"] = scattered(counts[G:], order[sum(counts[:G]):]).cuda()
    ints = lambda v: torch.tensor(v, dtype=torch.int32).cuda()  # noqa: E731
    sums = lambda v: ints([0] + torch.tensor(v).cumsum(0).tolist())  # noqa: E731
    st["prefix_lengths"], st["lengths"], st["cu_seqs"] = ints(prefix), ints(lens), sums(count)
    st["sequences"] = count, prefix, new
    st["cu"] = None if max(new) == 1 else sums(new)
    pool(st, sum(counts), Hkv, T, D, g)
    st["q"] = torch.randn(sum(new), (Hq + 2 * Hkv) * D, device="cuda", generator=g).to(TYPES[case["x"]])[:, :Hq * D].unflatten(1, (Hq, D))
    return st


# ---- plain forms ----------------------------------------------------------------------------------------------------------

def mx4_codes(x):
    """(rows, K) -> E2M1 codes packed two a byte (even column in the low bits), E8M0 scale bytes (rows, ceil(K / 32))."""
    rows, K = x.shape
    kb = -(-K // BLOCK)
    b = torch.zeros(rows, kb * BLOCK, device=x.device)
    b[:, :K] = x
    b = b.view(rows, kb, BLOCK)
    a = b.abs().amax(-1)
    e = torch.where(a > 0, torch.frexp(a).exponent - 3, torch.full_like(a, -127, dtype=torch.int32)).clamp(-127, 127)
    y = b * ((127 - e) << 23).view(torch.float32).unsqueeze(-1)   # times 2^-e
    m = y.abs()
    # a value on a border goes to the even code
    code = ((m > 0.25).to(torch.uint8) + (m >= 0.75) + (m > 1.25) + (m >= 1.75) + (m > 2.5) + (m >= 3.5) + (m > 5))
    code = (code | ((y < 0) * 8)).to(torch.uint8).view(rows, kb * BLOCK)[:, :K + K % 2]
    if code.shape[1] % 2:
        code = torch.cat([code, code.new_zeros(rows, 1)], 1)
    return code[:, 0::2] | (code[:, 1::2] << 4), (e + 127).to(torch.uint8)


def mx4_values(codes, scales, K):
    grid = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6, 0, -.5, -1, -1.5, -2, -3, -4, -6], device=codes.device)
    v = grid[torch.stack([codes & 15, codes >> 4], -1).int()].flatten(1)[:, :K]
    s = scales.int()
    s = torch.where(s > 0, s << 23, torch.full_like(s, 1 << 22)).view(torch.float32)   # 2^(byte - 127)
    return v * s.repeat_interleave(BLOCK, 1)[:, :K]


def activated(y, act):
    if act == "relu":
        return y.clamp(min=0)
    if act == "silu":
        return y / (1 + torch.exp(-y))
    if act == "gelu":
        return 0.5 * y * (1 + torch.erf(y * math.sqrt(0.5)))
    if act == "gelu_tanh":
        return y / (1 + torch.exp(-2 * math.sqrt(2 / math.pi) * (y + 0.044715 * y * y * y)))
    return y


def linear_plain(st):
    c = st["case"]
    K = c["K"]
    y = torch.matmul(mx4_values(*mx4_codes(st["x"].float()), K), mx4_values(st["w_codes"], st["w_scales"], K).t())
    if st["bias"] is not None:
        y += st["bias"].float()
    y = activated(y[:, 0::2], c["act"]) * y[:, 1::2] if c["gated"] else activated(y, c["act"])
    if st["residual"] is not None:
        y = y + st["residual"].float()
    return y.to(TYPES[c["x"]])


def turned(st, x, weight, cos, sin):
    """Normed heads, the first columns turned: pairs (i, i + half), or neighbours."""
    c, r = st["case"], st["case"]["rotary"]
    y = x.float()
    if weight is not None:
        y = y * torch.rsqrt((y * y).mean(-1, keepdim=True) + EPS) * weight.float()
    a, b = (y[..., 0:r:2], y[..., 1:r:2]) if c["interleaved"] else (y[..., :r // 2], y[..., r // 2:r])
    u, v = a * cos - b * sin, b * cos + a * sin
    u = torch.stack([u, v], -1).flatten(-2) if c["interleaved"] else torch.cat([u, v], -1)
    return torch.cat([u, y[..., r:]], -1).to(x.dtype)


def heads_plain(st):
    c, r = st["case"], st["case"]["rotary"]
    # (angles of far positions in 64 bits)
    f = 500000.0 ** (-2 * torch.arange(r // 2, device="cuda", dtype=torch.float64) / r)
    axis = torch.repeat_interleave(torch.arange(c["axes"], device="cuda"), torch.tensor(pairs_of(c), device="cuda"), output_size=r // 2)
    pos = st["positions"].view(c["axes"], -1)[axis].t().double()
    cos, sin = torch.cos(pos * f).float()[:, None], torch.sin(pos * f).float()[:, None]
    return [turned(st, st["q"], st["q_weight"], cos, sin), turned(st, st["k"], st["k_weight"], cos, sin)]


def blocks_of(lengths, T):
    return (lengths + (T - 1)) // T


def free_blocks(refs):
    """Block numbers, the free ones first, each kind in order."""
    return torch.argsort((refs > 0).to(torch.int32), stable=True).to(torch.int32)


def copy_plain(st, src, dst, tokens):
    """The first `tokens` of block src to dst, for each pair with tokens > 0."""
    T = st["case"]["T"]
    real = tokens > 0
    src, dst = src.long(), torch.where(real, dst, src).long()
    keep = (torch.arange(T, device="cuda") < tokens[:, None])[:, None, :, None]
    for name in ("k", "v"):
        codes, steps = st[name + "_codes"], st[name + "_steps"]
        moved = torch.where(keep, codes[src], codes[dst])
        held = steps[src]
        pick = real.nonzero()[:, 0]
        codes[dst[pick]] = moved[pick]
        steps[dst[pick]] = held[pick]


def fork_plain(st):
    T, n, refs = st["case"]["T"], st["case"]["n"], st["refs"]
    p = st["parents"].long()
    lengths = st["lengths"][p]
    have = blocks_of(lengths, T)
    col = torch.arange(st["table"].shape[1], device="cuda", dtype=torch.int32)
    table = torch.where(col < have[:, None], st["table"][p], torch.zeros((), dtype=torch.int32, device="cuda"))

    def count(sign):
        refs.index_add_(0, table.long().flatten(), torch.where(col < blocks_of(lengths, T)[:, None], sign, 0).to(torch.int32).flatten())

    count(1)
    # a block that would be written into and belongs to others, too: all of the batch copy it, but the first if nobody else has it
    last = table.gather(1, (have - 1).clamp(min=0).long()[:, None])[:, 0]
    partial = (lengths % T > 0)
    same = (last[:, None] == last[None, :]) & partial[:, None] & partial[None, :]
    first = same.to(torch.int32).cumsum(1).diagonal() == 1
    copies = partial & ~(first & (refs[last.long()] == same.sum(1)))
    need = blocks_of(lengths + n, T) - have
    at = (need + copies).cumsum(0) - (need + copies)
    free = free_blocks(refs)
    fresh = free[(at[:, None] + copies[:, None] + col - have[:, None]).clamp(0, len(free) - 1).long()]
    table = torch.where((col >= have[:, None]) & (col < (have + need)[:, None]), fresh, table)
    own_copy = free[at.clamp(max=len(free) - 1).long()]
    copy_plain(st, last, own_copy, torch.where(copies, lengths % T, 0))
    refs.index_add_(0, last.long(), -copies.to(torch.int32))
    table.scatter_(1, (have - 1).clamp(min=0).long()[:, None], torch.where(copies, own_copy, table.gather(1, (have - 1).clamp(min=0).long()[:, None])[:, 0])[:, None])
    refs.index_add_(0, own_copy.long(), copies.to(torch.int32))
    refs.index_add_(0, table.long().flatten(), ((col >= have[:, None]) & (col < (have + need)[:, None])).to(torch.int32).flatten())
    lengths = lengths + n
    count(-1)
    return [table, lengths, refs, st["k_codes"], st["v_codes"], st["k_steps"], st["v_steps"]]


def compact_plain(st):
    refs, table = st["refs"], st["table"]
    refs.copy_(st["saved_refs"])
    table.copy_(st["saved_table"])
    used = refs > 0
    total = used.sum()
    number = torch.arange(len(refs), device="cuda")
    src, dst = (used & (number >= total)).nonzero()[:, 0], (~used & (number < total)).nonzero()[:, 0]
    for name in ("k_codes", "v_codes", "k_steps", "v_steps"):
        st[name][dst] = st[name][src]
    to = number.to(torch.int32)
    to[src] = dst.to(torch.int32)
    col = torch.arange(table.shape[1], device="cuda")
    table.copy_(torch.where(col < blocks_of(st["lengths"], st["case"]["T"])[:, None], to[table.long()], table))
    refs[dst] = refs[src]
    refs[src] = 0
    return [table, refs, total.to(torch.int32), st["k_codes"], st["v_codes"], st["k_steps"], st["v_steps"]]


def gathered(st, name, table):
    """K or V of every row of a table, (rows, tokens, Hkv, D) in 32 bits."""
    t = table.long()
    v = st[name + "_codes"][t].float() * st[name + "_steps"][t][..., None, None]
    return v.permute(0, 1, 3, 2, 4).flatten(1, 2)


def softmax_part(q, k, v, seen):
    """Scores' maximum, sum and weighted values over tokens: q (..., rows, D), k and v (..., tokens, D), seen broadcast to the scores."""
    s = torch.matmul(q, k.transpose(-1, -2)) * q.shape[-1] ** -0.5
    s = s.masked_fill_(~seen, -math.inf)
    m = s.amax(-1)
    p = (s - m.clamp(min=torch.finfo(torch.float32).min)[..., None]).exp_()
    return m, p.sum(-1), torch.matmul(p, v)


def shared_plain(st):
    c = st["case"]
    Hq, Hkv, D, S = c["Hq"], c["Hkv"], c["D"], c["S"]
    R = Hq // Hkv
    count, prefix, new = st["sequences"]
    # the sequences' own tokens: rows (sequence, cache head, query head, new token)
    tok = torch.arange(sum(new), device="cuda")
    cu = st["cu"].long() if st["cu"] is not None else torch.arange(S + 1, device="cuda")
    seq = torch.searchsorted(cu[1:].contiguous(), tok, right=True)
    i, n = tok - cu[seq], max(new)
    q = torch.zeros(S, n, Hq, D, device="cuda")
    q[seq, i] = st["q"].float()
    q = q.view(S, n, Hkv, R, D).permute(0, 2, 3, 1, 4).reshape(S, Hkv, R * n, D)
    k, v = (gathered(st, name, st["table"]).permute(0, 2, 1, 3) for name in ("k", "v"))
    at = st["lengths"].long() - (cu[1:] - cu[:-1])
    t = torch.arange(k.shape[2], device="cuda")
    seen = (t <= (at[:, None] + torch.arange(n, device="cuda"))[..., None]) & (t < st["lengths"][:, None, None])   # (S, n, tokens)
    m, l, o = softmax_part(q, k, v, seen[:, None, None].expand(-1, -1, R, -1, -1).flatten(2, 3))
    # the groups' prefixes: all of a group's rows at once
    s0 = 0
    for g in range(c["groups"]):
        s1 = s0 + count[g]
        k, v = (gathered(st, name, st["prefix_table"][g:g + 1])[0].transpose(0, 1) for name in ("k", "v"))
        rows = q[s0:s1].transpose(0, 1).flatten(1, 2)
        mp, lp, op = softmax_part(rows, k, v, torch.arange(k.shape[1], device="cuda") < prefix[g])
        mp, lp, op = (x.unflatten(1, (s1 - s0, R * n)).transpose(0, 1) for x in (mp, lp, op))
        top = torch.maximum(m[s0:s1], mp)
        a, b = torch.exp(m[s0:s1] - top), torch.exp(mp - top)
        m[s0:s1], l[s0:s1], o[s0:s1] = top, a * l[s0:s1] + b * lp, a[..., None] * o[s0:s1] + b[..., None] * op
        s0 = s1
    o = (o / l[..., None]).view(S, Hkv, R, n, D)
    return o.permute(0, 3, 1, 2, 4).reshape(S, n, Hq, D)[seq, i].to(TYPES[c["x"]])


def run(state):
    c = state["case"]
    op = c["op"]
    if not own:
        return {"linear": linear_plain, "heads": heads_plain, "fork": fork_plain, "compact": compact_plain, "shared": shared_plain}[op](state)
    from paper_2608_09291_b200 import binding
    if op == "linear":
        return binding.mx4_linear(state["x"], state["w"], bias=state["bias"], act=None if c["act"] == "none" else c["act"], gated=c["gated"],
                                  residual=state["residual"])
    if op == "heads":
        return list(binding.qk_norm_rope(state["q"], state["k"], state["positions"], state["rotary"], state["q_weight"], state["k_weight"], eps=EPS))
    if op == "shared":
        return state["cache"].shared_attention(state["q"], state["prefix_table"], state["prefix_lengths"], state["cu_seqs"], state["table"],
                                               state["lengths"], state["cu"])
    pages, held = state["pages"], [state[name] for name in ("k_codes", "v_codes", "k_steps", "v_steps")]
    if op == "fork":
        table, lengths = pages.fork(state["table"], state["lengths"], state["parents"], keep=True)
        pages.extend(table, lengths, c["n"])
        pages.release(table, lengths)
        return [table, lengths, state["refs"], *held]
    state["refs"].copy_(state["saved_refs"])
    state["table"].copy_(state["saved_table"])
    used = pages.compact([(state["table"], state["lengths"])])
    return [state["table"], state["refs"], used, *held]


def work(case):
    op = case["op"]
    if op == "linear":
        N, M, K = case["N"], case["M"], case["K"]
        b = BYTES[case["x"]]
        out = N * (M // 2 if case["gated"] else M)
        packed = M * (-(-K // 2) + -(-K // BLOCK))
        return {"bytes": N * K * b + packed + out * b * (2 if case["residual"] else 1) + (M * b if case["bias"] else 0), "flops": 2 * N * K * M}
    if op == "heads":
        n = case["N"] * (case["Hq"] + case["Hkv"]) * case["D"]
        return {"bytes": 2 * n * BYTES[case["x"]] + 4 * case["N"] * case["axes"], "flops": 8 * n}
    if op == "fork":
        lens, parents = sequences(case)
        T, block = case["T"], case["Hkv"] * case["D"]
        rows = sum(-(-lens[p] // T) for p in parents)
        copied = sum(lens[p] % T for p in parents)
        return {"bytes": 4 * copied * block + 16 * rows + 16 * len(parents), "flops": copied * block}
    if op == "compact":
        counts = sequences(case)
        total, block = sum(counts), case["Hkv"] * case["T"] * case["D"]
        moves = int(total * (1 - total / case["blocks"]))   # of blocks anywhere in the pool
        return {"bytes": 4 * moves * block + 8 * case["blocks"] + 8 * total, "flops": moves * block}
    count, prefix, lens, new = sequences(case)
    Hq, Hkv, D, T = (case[k] for k in ("Hq", "Hkv", "D", "T"))
    tokens = sum(prefix) + sum(lens)
    pairs = sum(m * (n - m) + m * (m + 1) // 2 for n, m in zip(lens, new))
    s0 = 0
    for g, p in enumerate(prefix):
        pairs += p * sum(new[s0:s0 + count[g]])
        s0 += count[g]
    tables = 4 * sum(-(-n // T) for n in prefix + lens) + 4 * (len(prefix) + len(lens))
    return {"bytes": 2 * tokens * Hkv * (D + 4 / T) + 2 * sum(new) * Hq * D * BYTES[case["x"]] + tables, "flops": 4 * pairs * Hq * D}


# ---- the definitions in 64 bits ---------------------------------------------------------------------------------------------

def exact(case, seed):
    op = case["op"]
    if op in ("fork", "compact"):   # whole numbers that are moved
        return None
    st = prepare(case, seed)
    if op == "linear":
        x, K, outs = exact_mx4(st["x"].double()), case["K"], []
        for m in range(0, case["M"], 4096):   # some rows of the weight at a time
            codes, scales = st["w_codes"][m:m + 4096].long(), st["w_scales"][m:m + 4096].long()
            half = []
            for nib in (codes % 16, codes // 16):
                sign, ex, man = 1 - 2 * (nib // 8).double(), (nib // 2) % 4, (nib % 2).double()
                half.append(sign * torch.where(ex == 0, man / 2, (1 + man / 2) * power(ex - 1)))
            v = torch.stack(half, -1).flatten(1)[:, :K]
            y = x @ (v * power(scales - 127)[:, torch.arange(K, device="cuda") // BLOCK]).t()
            if case["bias"]:
                y = y + st["bias"][m:m + 4096].double()
            f = y[:, 0::2] if case["gated"] else y
            if case["act"] == "relu":
                f = torch.maximum(f, torch.zeros_like(f))
            elif case["act"] == "silu":
                f = f * torch.sigmoid(f)
            elif case["act"] == "gelu":
                f = f * (0.5 * torch.erfc(-f / math.sqrt(2)))
            elif case["act"] == "gelu_tanh":
                f = 0.5 * f * (1 + torch.tanh(math.sqrt(2 / math.pi) * (f + 0.044715 * f ** 3)))
            outs.append(f * y[:, 1::2] if case["gated"] else f)
        y = torch.cat(outs, 1)
        return y + st["residual"].double() if case["residual"] else y
    if op == "heads":
        r, outs = case["rotary"], []
        axis = [a for a, n in enumerate(pairs_of(case)) for _ in range(n)]
        pos = st["positions"].reshape(case["axes"], -1).double()
        for x, w in ((st["q"], st["q_weight"]), (st["k"], st["k_weight"])):
            y = x.double()
            if w is not None:
                y = y / torch.sqrt(y.square().sum(-1, keepdim=True) / case["D"] + EPS) * w.double()
            out = y.clone()
            for i in range(r // 2):
                a, b = (2 * i, 2 * i + 1) if case["interleaved"] else (i, i + r // 2)
                t = (pos[axis[i]] / 500000.0 ** (2 * i / r))[:, None]
                out[..., a] = y[..., a] * torch.cos(t) - y[..., b] * torch.sin(t)
                out[..., b] = y[..., a] * torch.sin(t) + y[..., b] * torch.cos(t)
            outs.append(out)
        return outs
    count, prefix, lens, new = sequences(case)
    Hq, Hkv, D, T = (case[k] for k in ("Hq", "Hkv", "D", "T"))
    group = [g for g, n in enumerate(count) for _ in range(n)]

    def values(name, row, n):
        blk = row[:-(-n // T)].long()
        x = st[name + "_codes"][blk].double() * st[name + "_steps"][blk].double()[..., None, None]
        return x.transpose(1, 2).flatten(0, 1)[:n].transpose(0, 1)   # (Hkv, n, D)

    outs, n0, held = [], 0, (None, None, None)
    for s in range(case["S"]):
        g = group[s]
        if held[0] != g:
            held = (g, *(values(name, st["prefix_table"][g], prefix[g]) for name in ("k", "v")))
        k, v = (torch.cat([held[1 + i], values(name, st["table"][s], lens[s])], 1) for i, name in enumerate(("k", "v")))
        n, L = new[s], k.shape[1]
        q = st["q"][n0:n0 + n].double().view(n, Hkv, Hq // Hkv, D).permute(1, 2, 0, 3).flatten(1, 2)   # (Hkv, heads x n, D)
        a = torch.einsum("hrd,htd->hrt", q, k) / math.sqrt(D)
        place = torch.arange(L - n, L, device="cuda").repeat(Hq // Hkv)
        a = a.masked_fill(torch.arange(L, device="cuda") > place[:, None], -math.inf)
        o = torch.softmax(a, -1) @ v
        outs.append(o.unflatten(1, (Hq // Hkv, n)).permute(2, 0, 1, 3).flatten(1, 2))
        n0 += n
    return torch.cat(outs)


def power(e):
    """2^e in 64 bits, exactly."""
    return ((e + 1023) << 52).view(torch.float64)


def exact_mx4(x):
    """The MX4 values of x, both in 64 bits: the nearest of the grid, on a border the one with the even code."""
    rows, K = x.shape
    grid = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64, device=x.device)
    out = torch.zeros_like(x)
    whole = K // BLOCK * BLOCK
    for lo, hi in ((0, whole), (whole, K)):
        if lo == hi:
            continue
        b = x[:, lo:hi].reshape(rows, -1, min(BLOCK, hi - lo))
        a = b.abs().amax(-1, keepdim=True)
        scale = torch.where(a > 0, power(torch.frexp(a).exponent.long() - 3), torch.ones_like(a)).clamp(min=2.0 ** -127)
        m = (b.abs() / scale).clamp(max=6)
        up = torch.searchsorted(grid, m).clamp(min=1)          # grid[up - 1] < m <= grid[up]
        low, high = grid[up - 1], grid[up]
        mid = (low + high) / 2
        pick = torch.where((m > mid) | ((m == mid) & (up % 2 == 0)), high, low)
        out[:, lo:hi] = (torch.sign(b) * pick * scale).reshape(rows, hi - lo)
    return out
