"""Cases of the operators that a decoder needs beside the sparse product: MX4 (microscaled 4-bit floating point)
quantisation and product, and the 8-bit cache of keys and values with the attention over it.

``linear``    ``mx4_linear``: activations in 16 or 32 bits, quantised within the call, times a dense MX4 weight that the program
              holds. One token is a decode step, thousands are a prompt.
``quantize``  ``mx4_quantize`` and the values back: what a program that loads weights or looks at rounding errors does.
``append``    ``KVCache.append`` and ``KVCache.read``: new tokens of a batch of sequences, of one token or a prompt each, go to the
              paged cache; the sequences are read back.
``attend``    ``KVCache.attention``: a batch of sequences, of one query token each (decode) or several (prompt), over its cache.

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


def listed():
    def linear(name, N, M, K, x, out):
        return {"name": name, "op": "linear", "N": N, "M": M, "K": K, "x": x, "out": out}

    def quantize(name, N, K, x):
        return {"name": name, "op": "quantize", "N": N, "K": K, "x": x}

    def kv(name, op, S, Hq, Hkv, D, T, L, n, x, spread, causal=True, window=0):
        return {"name": name, "op": op, "S": S, "Hq": Hq, "Hkv": Hkv, "D": D, "T": T, "L": L, "n": n, "x": x, "spread": spread,
                "causal": causal, "window": window}

    return [
        # a decode step of one user: a 7B-shaped projection, where latency counts
        linear("linear_1x4096x4096", 1, 4096, 4096, "f16", "f16"),
        # a small batch, the largest matrix (70B-shaped FFN)
        linear("linear_8x28672x8192", 8, 28672, 8192, "f16", "f16"),
        # sizes that divide into nothing
        linear("linear_33x1001x2003", 33, 1001, 2003, "bf16", "bf16"),
        # a prompt through the 70B-shaped FFN
        linear("linear_4096x28672x8192", 4096, 28672, 8192, "bf16", "bf16"),
        # a few rows with a ragged last block; a weight matrix
        quantize("quantize_5x4100", 5, 4100, "f32"),
        quantize("quantize_8192x8192", 8192, 8192, "bf16"),
        # a decode step's new tokens of a batch, and prompts of unequal length behind earlier tokens
        kv("append_64x1", "append", 64, 64, 8, 128, 64, 300, 1, "bf16", True),
        kv("append_3_prompts", "append", 3, 32, 32, 128, 16, 2500, 2000, "f16", True),
        # one user's short context, all heads their own (7B-shaped)
        kv("attend_1x1000", "attend", 1, 32, 32, 128, 64, 1000, 1, "f16", False),
        # a batch of users with contexts of unequal length (70B-shaped, 8 query heads a cache head)
        kv("attend_64x8192", "attend", 64, 64, 8, 128, 64, 8192, 1, "bf16", True),
        # one long context
        kv("attend_1x131072", "attend", 1, 64, 8, 128, 64, 131072, 1, "f16", False),
        # prompts of unequal length, in part behind an earlier part of theirs
        kv("attend_3_prompts", "attend", 3, 64, 8, 128, 64, 4500, 2000, "bf16", True),
    ]


def draw(rng):
    """One more case of the same ranges: sizes spread over their logarithm, any remainder."""
    def size(lo, hi):
        return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))

    most = [work(c) for c in listed()]
    flops, data = max(w["flops"] for w in most), max(w["bytes"] for w in most)
    while True:
        op = rng.choice(["linear", "linear", "quantize", "append", "attend", "attend"])
        x = rng.choice(["f16", "bf16", "f32"])
        if op == "linear":
            c = {"op": op, "N": size(1, 4096), "M": size(64, 28672), "K": size(32, 16384), "x": x, "out": rng.choice(["f16", "bf16"])}
            if rng.random() < 0.5:   # widths of models divide well
                c["M"], c["K"] = -(-c["M"] // 128) * 128, -(-c["K"] // 128) * 128
        elif op == "quantize":
            c = {"op": op, "N": size(1, 8192), "K": size(1, 16384), "x": x}
        else:
            x = "bf16" if x == "f32" and op == "attend" else x
            Hkv = rng.choice([1, 2, 4, 8, 32])
            n = 1 if rng.random() < 0.6 else size(2, 2000)
            S = size(1, 64)
            c = {"op": op, "S": S, "Hq": Hkv * rng.choice([1, 2, 4, 7, 8, 16][:6 if Hkv <= 4 else 3 if Hkv == 8 else 1]), "Hkv": Hkv,
                 "D": rng.choice([64, 128]), "T": rng.choice([16, 32, 64, 128]), "L": size(1, 32768 if op == "attend" else 4096) + n - 1, "n": n, "x": x,
                 "spread": rng.random() < 0.7, "causal": rng.random() < 0.9, "window": rng.choice([0, 0, 0, 1, 100, 1024])}
            whole = c["S"] * c["L"] * Hkv * c["D"]   # elements of K in 32 bits, in the plain form
            if whole > 64 * 8192 * 8 * 128 / (4 if op == "append" else 1) or c["S"] * c["Hq"] * n * c["L"] > 1.5e9:
                continue
        w = work(c)
        if w["flops"] <= flops and w["bytes"] <= data:
            return c


# ---- the state ----------------------------------------------------------------------------------------------------------

def lengths_of(c):
    """Lengths of the sequences with their new tokens, and how many tokens of each are new: plain lists from the case alone."""
    r = random.Random(c["S"] * 1000003 + c["L"])
    lens, new = [], []
    for s in range(c["S"]):
        full = s == 0 or not c["spread"]
        n = c["n"] if full or c["n"] == 1 else r.randint(1, c["n"])
        lens.append(c["L"] if full else r.randint(n, c["L"]))
        new.append(n)
    return lens, new


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    if case["op"] in ("linear", "quantize"):
        N, K = case["N"], case["K"]
        # hidden states: a spread of their own for each token, a few channels much larger
        x = torch.randn(N, K, device="cuda", generator=g)
        x *= 0.2 + 2.8 * torch.rand(N, 1, device="cuda", generator=g)
        x *= 1 + 7 * (torch.rand(K, device="cuda", generator=g) < 1 / 256)
        st = {"case": case, "x": x.to(TYPES[case["x"]])}
        if case["op"] == "linear":
            M = case["M"]
            w = torch.randn(M, K, device="cuda", generator=g) * 0.02
            st["w_codes"], st["w_scales"] = mx4_codes(w)
            if own:   # a program holds its weights in the form that the product reads
                from paper_2608_09291_b200 import binding
                st["w"] = binding.mx4_from_codes(st["w_codes"], st["w_scales"], K)
        return st
    S, Hq, Hkv, D, T = (case[k] for k in ("S", "Hq", "Hkv", "D", "T"))
    lens, new = lengths_of(case)
    width = -(-max(lens) // T)
    blocks = sum(-(-n // T) for n in lens)
    order = torch.randperm(blocks, device="cuda", generator=g).to(torch.int32)   # pages lie anywhere in the pool
    table = torch.zeros(S, width, dtype=torch.int32)
    at, flat = 0, order.cpu()
    for s, n in enumerate(lens):
        b = -(-n // T)
        table[s, :b] = flat[at:at + b]
        at += b
    st = {"case": case, "table": table.cuda(), "lengths": torch.tensor(lens, dtype=torch.int32).cuda(), "width": max(lens)}
    for name in ("k", "v"):
        codes = torch.empty(blocks, Hkv, T, D, dtype=torch.int8, device="cuda")
        for b in range(0, blocks, 4096):
            part = codes[b:b + 4096]
            part.copy_(torch.randn(part.shape, device="cuda", dtype=torch.float16, generator=g).mul_(32).round_().clamp_(-127, 127))
        st[name + "_codes"] = codes
        st[name + "_steps"] = (0.7 + 0.7 * torch.rand(blocks, Hkv, device="cuda", generator=g)) / 32
    N = sum(new)
    st["N"], st["most"] = N, max(new)
    st["cu"] = None if max(new) == 1 else torch.tensor([0] + torch.tensor(new).cumsum(0).tolist(), dtype=torch.int32).cuda()
    # q, k and v are columns of one stacked projection's output
    qkv = torch.randn(N, (Hq + 2 * Hkv) * D, device="cuda", generator=g).to(TYPES[case["x"]])
    st["q"] = qkv[:, :Hq * D].unflatten(1, (Hq, D))
    st["k"] = qkv[:, Hq * D:(Hq + Hkv) * D].unflatten(1, (Hkv, D))
    st["v"] = qkv[:, (Hq + Hkv) * D:].unflatten(1, (Hkv, D))
    if own:
        from paper_2608_09291_b200 import binding
        st["cache"] = binding.KVCache(st["k_codes"], st["v_codes"], st["k_steps"], st["v_steps"])
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


def places(st):
    """For each new token: its sequence, its place in it, its block in the pool and its place there; for each sequence its length before."""
    case, lengths, T = st["case"], st["lengths"].long(), st["case"]["T"]
    tok = torch.arange(st["N"], device="cuda")
    if st["cu"] is None:
        seq, first, new = tok, tok, torch.ones_like(lengths)
    else:
        cu = st["cu"].long()
        seq = torch.searchsorted(cu[1:].contiguous(), tok, right=True)
        first, new = cu[seq], cu[1:] - cu[:-1]
    before = lengths - new
    pos = before[seq] + tok - first
    return seq, pos, st["table"][seq, pos // T].long(), pos % T, before, tok - first


def gathered(st, name):
    """K or V of every sequence, (S, longest, Hkv, D) in 32 bits; behind a sequence's end what the table's first entries hold."""
    T = st["case"]["T"]
    t = st["table"].long()
    v = st[name + "_codes"][t].float() * st[name + "_steps"][t][..., None, None]
    return v.permute(0, 1, 3, 2, 4).flatten(1, 2)[:, :st["width"]]


def append_plain(st):
    T, Hkv = st["case"]["T"], st["case"]["Hkv"]
    seq, pos, blk, off, before, _ = places(st)
    first = st["table"].gather(1, (before // T).clamp(max=st["table"].shape[1] - 1)[:, None].long())[:, 0].long()   # each sequence's first block that gets tokens
    held = before % T
    for name in ("k", "v"):
        codes, steps, x = st[name + "_codes"], st[name + "_steps"], st[name].float()
        fresh = torch.zeros_like(steps).index_reduce_(0, blk, x.abs().amax(-1) / torch.tensor(127., device="cuda"), "amax")
        old = torch.where(held[:, None] > 0, steps[first], torch.zeros_like(steps[first]))
        now = torch.maximum(old, fresh[first])
        # (quotients in 64 bits: many lie next to a border between two codes, or on one)
        n64 = torch.where(now > 0, now, torch.ones_like(now)).double()[..., None, None]
        kept = (codes[first].double() * old.double()[..., None, None] / n64).round()
        keep = torch.arange(T, device="cuda")[None, :] < held[:, None]
        codes[first] = torch.where(keep[:, None, :, None], kept.to(torch.int8), codes[first])
        steps[blk] = fresh[blk]
        steps[first] = now
        s = steps[blk].double()[..., None]
        codes[blk, :, off] = torch.where(s > 0, x / s, torch.zeros_like(s)).round().clamp(-127, 127).to(torch.int8)
    seen = (torch.arange(st["width"], device="cuda")[None, :] < st["lengths"][:, None])[..., None, None]
    return [torch.where(seen, gathered(st, name), torch.zeros((), device="cuda")) for name in ("k", "v")]


def seen_by(st, pos):
    """(S, n, longest): which tokens a query at place `pos` (S, n) of its sequence sees."""
    t = torch.arange(st["width"], device="cuda")
    seen = (t < st["lengths"][:, None])[:, None, :].expand(-1, pos.shape[1], -1)
    if st["case"]["causal"]:
        seen = seen & (t <= pos[..., None])
    if st["case"]["window"]:
        seen = seen & (t > pos[..., None] - st["case"]["window"])
    return seen


def attend_plain(st):
    c = st["case"]
    S, Hq, Hkv, D, n = c["S"], c["Hq"], c["Hkv"], c["D"], st["most"]
    seq, pos, _, _, before, i = places(st)
    q = torch.zeros(S, n, Hq, D, device="cuda")
    q[seq, i] = st["q"].float()
    q = q.view(S, n, Hkv, Hq // Hkv, D).permute(0, 2, 3, 1, 4).reshape(S, Hkv, -1, D)
    k = gathered(st, "k").permute(0, 2, 3, 1)
    s = torch.matmul(q, k).view(S, Hkv, Hq // Hkv, n, -1) * D ** -0.5
    del k
    seen = seen_by(st, before[:, None] + torch.arange(n, device="cuda"))[:, None, None]
    s = s.masked_fill_(~seen, -math.inf)
    p = (s - s.amax(-1, keepdim=True).clamp(min=torch.finfo(torch.float32).min)).exp_()
    l = p.sum(-1)
    o = torch.matmul(p.flatten(2, 3), gathered(st, "v").permute(0, 2, 1, 3)).view(S, Hkv, Hq // Hkv, n, D)
    o = torch.where(l[..., None] > 0, o / l[..., None], torch.zeros((), device="cuda"))
    return o.permute(0, 3, 1, 2, 4).reshape(S, n, Hq, D)[seq, i].to(TYPES[c["x"]])


def run(state):
    op = state["case"]["op"]
    if own:
        from paper_2608_09291_b200 import binding
        if op == "linear":
            return binding.mx4_linear(state["x"], state["w"], dtype=TYPES[state["case"]["out"]])
        if op == "quantize":
            return binding.mx4_quantize(state["x"]).dequantize(torch.bfloat16)
        cache = state["cache"]
        if op == "append":
            cache.append(state["k"], state["v"], state["table"], state["lengths"], state["cu"])
            return list(cache.read(state["table"], state["lengths"], state["width"], dtype=torch.float32))
        return cache.attention(state["q"], state["table"], state["lengths"], state["cu"], causal=state["case"]["causal"],
                               window=state["case"]["window"])
    if op in ("linear", "quantize"):
        x = state["x"].float()
        K = x.shape[1]
        values = mx4_values(*mx4_codes(x), K)
        if op == "quantize":
            return values.to(torch.bfloat16)
        w = mx4_values(state["w_codes"], state["w_scales"], K)
        return torch.matmul(values, w.t()).to(TYPES[state["case"]["out"]])
    return append_plain(state) if op == "append" else attend_plain(state)


def work(case):
    if case["op"] in ("linear", "quantize"):
        N, K = case["N"], case["K"]
        x = N * K * BYTES[case["x"]]
        packed = lambda rows: rows * (-(-K // 2) + -(-K // BLOCK))  # noqa: E731
        if case["op"] == "quantize":   # codes and scales are written, and read back
            return {"bytes": x + 2 * packed(N) + 2 * N * K, "flops": 10 * N * K}
        return {"bytes": x + packed(case["M"]) + N * case["M"] * BYTES[case["out"]], "flops": 2 * N * K * case["M"]}
    lens, new = lengths_of(case)
    Hq, Hkv, D, T, w = case["Hq"], case["Hkv"], case["D"], case["T"], case["window"]
    tables = sum(4 * (-(-n // T)) for n in lens) + 4 * case["S"]
    if case["op"] == "append":
        N = sum(new)
        kept = sum(lens)
        return {"bytes": 2 * N * Hkv * D * (BYTES[case["x"]] + 1) + 2 * kept * Hkv * D + 2 * case["S"] * max(lens) * Hkv * D * 4 + tables,
                "flops": 2 * Hkv * D * (4 * N + kept)}
    pairs = tokens = 0
    for n, m in zip(lens, new):
        if case["causal"]:
            seen = [min(p + 1, w) if w else p + 1 for p in range(n - m, n)]
            tokens += min(n, w + m - 1) if w else n
        else:
            seen = [min(n, n - (p - w + 1)) if w and p >= w else n for p in range(n - m, n)]
            tokens += min(n, n - (n - m - w + 1)) if w and n - m >= w else n
        pairs += sum(seen)
    return {"bytes": 2 * tokens * Hkv * (D + 4 / T) + 2 * sum(new) * Hq * D * BYTES[case["x"]] + tables, "flops": 4 * pairs * Hq * D}


# ---- the definitions in 64 bits ---------------------------------------------------------------------------------------------

def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] in ("linear", "quantize"):
        x = exact_mx4(st["x"].double())
        if case["op"] == "quantize":
            return x
        rows = []
        for m in range(0, case["M"], 4096):   # the weight's values, some rows at a time
            codes, scales = st["w_codes"][m:m + 4096].long(), st["w_scales"][m:m + 4096].long()
            half = []
            for nib in (codes % 16, codes // 16):
                sign, ex, man = 1 - 2 * (nib // 8).double(), (nib // 2) % 4, (nib % 2).double()
                half.append(sign * torch.where(ex == 0, man / 2, (1 + man / 2) * power(ex - 1)))
            v = torch.stack(half, -1).flatten(1)[:, :case["K"]]
            k = torch.arange(case["K"], device="cuda") // BLOCK
            rows.append(x @ (v * power(scales - 127)[:, k]).t())
        return torch.cat(rows, 1)
    lens, new = lengths_of(case)
    S, Hq, Hkv, D, T = (case[k] for k in ("S", "Hq", "Hkv", "D", "T"))
    n0, outs = 0, [[], []]
    for s in range(S):
        L, n = lens[s], new[s]
        blk = st["table"][s, :-(-L // T)].long()
        kv = []
        for name in ("k", "v"):
            codes, steps = st[name + "_codes"][blk].double(), st[name + "_steps"][blk].double()
            if case["op"] == "append":
                x = st[name][n0:n0 + n].double()
                for j in range((L - n) // T, len(blk)):
                    lo, hi = max(j * T, L - n), min(j * T + T, L)
                    part = x[lo - (L - n):hi - (L - n)].transpose(0, 1)                     # (Hkv, tokens, D)
                    step = (part.abs().amax((1, 2)) / 127).float().double()                 # (a step is held in 32 bits)
                    a = lo - j * T
                    if a:
                        step = torch.maximum(step, steps[j])
                        codes[j, :, :a] = (codes[j, :, :a] * steps[j][:, None, None] / step[:, None, None]).round()
                    steps[j] = step
                    codes[j, :, a:a + hi - lo] = (part / step.clamp(min=1e-300)[:, None, None]).round().clamp(-127, 127)
            kv.append((codes * steps[..., None, None]).transpose(1, 2).flatten(0, 1)[:L])   # (L, Hkv, D)
        if case["op"] == "append":
            for o, v in zip(outs, kv):
                o.append(torch.nn.functional.pad(v, (0, 0, 0, 0, 0, st["width"] - L)))
        else:
            q = st["q"][n0:n0 + n].double()
            t, pos = torch.arange(L, device="cuda"), torch.arange(L - n, L, device="cuda")[:, None]
            hidden = torch.zeros(n, L, dtype=torch.bool, device="cuda")
            if case["causal"]:
                hidden |= t > pos
            if case["window"]:
                hidden |= t <= pos - case["window"]
            heads = []
            for h in range(Hq):
                k, v = kv[0][:, h // (Hq // Hkv)], kv[1][:, h // (Hq // Hkv)]
                a = (q[:, h] @ k.t()) / math.sqrt(D)
                a[hidden] = -math.inf
                p = torch.exp(a - a.amax(1, keepdim=True))
                heads.append((p / p.sum(1, keepdim=True)) @ v)
            outs[0].append(torch.stack(heads, 1))
        n0 += n
    if case["op"] == "append":
        return [torch.stack(o) for o in outs]
    return torch.cat(outs[0])


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
