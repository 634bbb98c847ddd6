// Attention over the 8-bit cache for many query rows a cache head (prompts): the 5th-generation tensor cores.
//
// A CTA takes up to 256 query rows (tokens x the query heads that share a cache head) of one (sequence, head) in two tiles of 128, and walks
// its 128-token units of the cache:
//   convert   four warps load the codes of a unit, a unit ahead, and write them as fp16 (exact) where the MMA reads: K with D contiguous
//             (K-major), V as it lies (MN-major), both swizzled over 128 bytes.
//   MMA       one warp: S = Q K^T into tensor memory, O += P V with P from tensor memory, for the two tiles in turn: while one tile's
//             scores are being turned into P the other tile's products run.
//   softmax   four warps a tile, a thread a row: no exchange between lanes. Steps: one number for 16 tokens, K's a factor of the
//             scores, V's in the exponent of p (relative to a second running maximum of each row, see us_kv.cuh), so that a unit's P V
//             needs no scaling. P takes the place of S.
// P has 11 bits, for fp16 outputs, too: a second product of what its rounding leaves (it fits beside P, in the other half of S's place) takes
// the error against 64 bits from 2.9e-4 to 2.1e-4, and the softmax threads' time from 714 to 937 us (three prompts of up to 2000 tokens, fp16);
// V's codes are rounded to half a 127th of their largest. Behind shared prefixes (kGroups, kOwn) fp16 has that product: a single token's row
// meets this kernel only because others share its prefix, and is to be as exact as alone (64 sequences of 8 rows a cache head behind 8192 tokens, 512 of their own: 59.9 us
// without, 60.5 with; 16 behind 4096: 25.8, 28.2; 8 of 20 new tokens and 4 rows behind 3000: 75.9, 87.7; 2.8e-4 and 2.1e-4 against 64 bits). bf16 goes without: its own rounding is eight
// times as large (1.67e-3 and 1.66e-3; 64 sequences behind 8192 tokens, up to 512 of their own: 48.2 us, 57.4 with it).
// m follows the true maximum only where it is 2^8 behind; p carries 2^7, see us_kv.cuh. The scores' conversions, the
// 16384 exponentials (16 a cycle) and the two products (1024 cycles) of a tile and unit are each about 1000 cycles, and overlap.
// Three prompts of up to 2000 tokens, to contexts of up to 4500 (64/8 heads of 128, bf16): 723 us, 696 inside a graph; one of 8192 tokens: 1250 to
// 1281 us, 858 to 880 TFLOP/s. What
// bounds it is the softmax threads' own chain from scores to P. Slower: 16 softmax warps (914 us), units of 64 tokens (816), exponentials
// partly as polynomials (748 to 795). The softmax threads spill about 100 bytes.
#pragma once
#include "us_kv.cuh"

namespace us {

constexpr int kPrRows = 256, kPrTile = 128;

struct KvPrompt {
    KvPool pool;
    KvSeqs seqs;
    const void* q;
    int64_t q_token, q_head;
    void* out;
    int64_t o_token, o_head;
    float* lse;
    float* part;             // [row tile][head][split]: sums [D / 4][256 rows][4], then m[256], l[256]
    float scale2;            // |scale| log2(e); the sign goes to the queries
    int32_t negative;
    int32_t Hq, G;
    int32_t causal, window;
    int32_t q_vec, o_vec;
    int32_t log2_T;
    int32_t splits;
    int32_t beside;          // (kGroups) the kernel of the own tokens runs beside it: leaves parts, whatever their number
    KvRows rows;
};

template <int D>
struct PrShape {
    static constexpr int kQ = 128 * D * 2, kKV = kPrTile * D * 2;   // bytes
    static constexpr int kSmem = 1024 + 2 * kQ + 4 * kKV;
    static constexpr int64_t kPart = kPrRows * (D + 2);
    static constexpr int kThreads = 16 * 32;   // softmax 2 x 4 warps, conversion 4, MMA issue 1 (and three that only fill its group)
};

__device__ __forceinline__ void tc_mma_f16(uint32_t elected, uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate)
{
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 q, %5, 0;\n\tsetp.ne.u32 p, %4, 0;\n\t"
                 "@q tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                 ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate), "r"(elected) : "memory");
}
__device__ __forceinline__ void tc_mma_f16_ts(uint32_t elected, uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t accumulate)
{
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 q, %5, 0;\n\tsetp.ne.u32 p, %4, 0;\n\t"
                 "@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
                 ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"(accumulate), "r"(elected) : "memory");
}
__device__ __forceinline__ float max3(float a, float b, float c)
{
    float r;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
// two fp32 in one instruction
__device__ __forceinline__ uint64_t f32x2(float a, float b)
{
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ void f32x2_split(uint64_t v, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c)
{
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b)
{
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}

// The sequence and row tile of row tile `index` of the batch; row tiles of a sequence with the latest tokens (that see most) first.
// rows: query rows of a head in the tile.
struct PrItem {
    KvSeq seq;
    int s, row0, rows;
};
template <int MODE>
__device__ __forceinline__ bool pr_item(const KvPrompt& a, uint32_t index, int lane, PrItem& it, bool report)
{
    uint32_t before = 0;
    bool any = false, found = false;
    for (int base = 0; base < a.seqs.S; base += 32) {
        uint32_t cnt = 0;
        KvSeq mine = {0, 0, 0};
        if (base + lane < a.seqs.S) {
            bool wrong;
            mine = kv_seq<MODE>(a.seqs, a.pool, base + lane, wrong);
            any |= wrong;
            cnt = ((uint32_t)mine.n * (uint32_t)a.G + kPrRows - 1) / kPrRows;
        }
        uint32_t sum = cnt;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const uint32_t v = __shfl_up_sync(0xffffffffu, sum, o);
            if (lane >= o) sum += v;
        }
        const uint32_t who = __ballot_sync(0xffffffffu, index >= before + sum - cnt && index < before + sum);
        if (who) {
            const int l = __ffs(who) - 1;
            it.s = base + l;
            const uint32_t tiles = __shfl_sync(0xffffffffu, cnt, l), j = index - before - __shfl_sync(0xffffffffu, sum - cnt, l);
            it.seq.first = __shfl_sync(0xffffffffu, mine.first, l);
            it.seq.len = __shfl_sync(0xffffffffu, mine.len, l);
            it.seq.n = __shfl_sync(0xffffffffu, mine.n, l);
            it.row0 = (int)((tiles - 1 - j) * kPrRows);
            it.rows = min(kPrRows, it.seq.n * a.G - it.row0);
            found = true;
            break;
        }
        before += __shfl_sync(0xffffffffu, sum, 31);
    }
    if (any && report) atomicExch(a.pool.err, kErrIndex);
    return found;
}
// First and last + 1 unit of 128 tokens that the tile's rows see.
__device__ __forceinline__ void pr_units(const KvPrompt& a, const PrItem& it, int& u0, int& u1)
{
    const int pos0 = it.seq.len - it.seq.n, first = pos0 + it.row0 / a.G, last = pos0 + (it.row0 + it.rows - 1) / a.G;
    const int hi = a.causal ? last + 1 : it.seq.len, lo = a.window > 0 ? max(0, first - a.window + 1) : 0;
    u0 = lo / kPrTile;
    u1 = hi > lo ? (hi + kPrTile - 1) / kPrTile : u0;
}

// Whether what p's rounding leaves is multiplied, too.
template <bool BF16, int MODE>
constexpr bool kPrRest = MODE != kAlone && !BF16;
__device__ __forceinline__ uint32_t half2_rest(float a, float b, uint32_t rounded)
{
    const float2 r = __half22float2(*reinterpret_cast<const __half2*>(&rounded));
    return half2_bits(a - r.x, b - r.y);
}

template <int D, bool BF16, int MODE = kAlone>
__global__ void __launch_bounds__(PrShape<D>::kThreads, 1) us_kv_prompt_kernel(const __grid_constant__ KvPrompt a)
{
    using S = PrShape<D>;
    constexpr int HALVES = D / 64;   // 128-byte columns of fp16
    constexpr bool REST = kPrRest<BF16, MODE>;
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    __shared__ __align__(8) uint64_t bars[24];
    __shared__ float4 steps[4][8];   // of a unit's 16-token groups: K's step (-1: not there), V's, its log2 (-126 to 128), its inverse
    __shared__ uint32_t misc[2];
    uint8_t* sq = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
    uint8_t* sk = sq + 2 * S::kQ;
    uint8_t* sv = sk + 2 * S::kKV;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t bar = smem_u32(bars);
    const uint32_t b_q = bar, b_kf = bar + 16, b_ke = bar + 32, b_vf = bar + 48, b_ve = bar + 64, b_s = bar + 80, b_p = bar + 96, b_o = bar + 128, b_st = bar + 144, b_end = bar + 176;
    volatile uint32_t* dead = misc + 1;
    if (warp == 12) {
        if (lane == 0) {
            for (int i = 0; i < 2; ++i) {
                mbar_init(b_q + 8u * i, 4);
                mbar_init(b_kf + 8u * i, 4); mbar_init(b_ke + 8u * i, 1);
                mbar_init(b_vf + 8u * i, 4); mbar_init(b_ve + 8u * i, 1);
                mbar_init(b_s + 8u * i, 1); mbar_init(b_p + 16u * i, 4); mbar_init(b_p + 16u * i + 8, 4); mbar_init(b_o + 8u * i, 1);
            }
            for (int i = 0; i < 4; ++i) mbar_init(b_st + 8u * i, 4);
            mbar_init(b_end, 1);
            misc[1] = 0;
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        __syncwarp();
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(misc)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    // After the allocation (see us_mx4.cuh), and after the wait: the kernel that joins the parts reads lengths and token counts before its own.
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const uint32_t tm = *(volatile uint32_t*)misc;
    const KvPool& p = a.pool;
    const int split = (int)(blockIdx.x % a.splits), h = (int)(blockIdx.x / a.splits) % p.Hkv;
    const uint32_t index = blockIdx.x / ((unsigned)a.splits * p.Hkv);
    PrItem it;
    const bool have = pr_item<MODE>(a, index, lane, it, threadIdx.x < 32);
    bool ok = true;
    int u0 = 0, u1 = 0;
    if (have) {
        pr_units(a, it, u0, u1);
        const int n = u1 - u0;
        const int each = n / a.splits, more = n - each * a.splits;   // the first `more` parts have one unit more
        u0 += each * split + min(split, more);
        u1 = u0 + each + (split < more ? 1 : 0);
    }
    const int n = u1 - u0, nq = have && it.rows > 128 ? 2 : 1;
    // Registers of a thread: 128 at launch, 16 warps; 2 x 176 + 96 + 64 = 4 x 128.
    if (warp < 8) {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 176;");
        if (have) {
        // ================= softmax: a thread a row =================
        const int qi = warp >> 2, r = it.row0 + 128 * qi + 32 * (warp & 3) + lane, local = r - it.row0;
        const uint32_t lanes = (uint32_t)(warp & 3) << 21;
        const uint32_t t_s = tm + lanes + 128u * qi, t_o = tm + lanes + 256u + 128u * qi;
        const bool real = local < it.rows;
        const int tok = real ? r / a.G : 0, qh = h * a.G + (real ? r - tok * a.G : 0);
        const int pos = it.seq.len - it.seq.n + tok;
        // (rows past the last are zero queries that see everything; never stored)
        const int hi = real ? (a.causal ? pos + 1 : it.seq.len) : 0x7FFFFFFF, lo = real && a.window > 0 ? pos - a.window + 1 : -0x7FFFFFFF;
        float m = -INFINITY, l = 0.f, lead = 0.f, most = 0.f, f = a.scale2;   // lead: m less the reference of p times V's step; most: V's largest step so far
        if (qi < nq && n > 0) {
            // the row as fp16, bf16 times a power of two that brings it into range, to its place in the operand
            const uint16_t* src = static_cast<const uint16_t*>(a.q) + (it.seq.first + tok) * a.q_token + (int64_t)qh * a.q_head;
            float mul = a.negative ? -1.f : 1.f;
            auto load = [&](int c) -> uint4 {
                if (!real) return make_uint4(0, 0, 0, 0);
                if (a.q_vec) return __ldcg(reinterpret_cast<const uint4*>(src) + c);
                uint32_t w[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) w[i] = (uint32_t)src[8 * c + 2 * i] | ((uint32_t)src[8 * c + 2 * i + 1] << 16);
                return make_uint4(w[0], w[1], w[2], w[3]);
            };
            uint4 row[D / 8];
#pragma unroll
            for (int c = 0; c < D / 8; ++c) row[c] = load(c);
            if (BF16) {
                uint32_t big = 0;
#pragma unroll
                for (int c = 0; c < D / 8; ++c) {
                    const uint32_t w[4] = {row[c].x, row[c].y, row[c].z, row[c].w};
#pragma unroll
                    for (int i = 0; i < 4; ++i) big = max(big, max(w[i] & 0x7FFFu, (w[i] >> 16) & 0x7FFFu));
                }
                const int e = max(-112, min(114, (int)(big >> 7) - 127 - 14));
                mul *= __uint_as_float((uint32_t)(127 - e) << 23);
                f *= __uint_as_float((uint32_t)(127 + e) << 23);
            }
            const int rr = 32 * (warp & 3) + lane;
            uint8_t* dst = sq + qi * S::kQ + rr * 128;
#pragma unroll
            for (int c = 0; c < D / 8; ++c) {
                const uint32_t w[4] = {row[c].x, row[c].y, row[c].z, row[c].w};
                uint32_t y[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if (BF16) y[i] = half2_bits(__uint_as_float(w[i] << 16) * mul, __uint_as_float(w[i] & 0xFFFF0000u) * mul);
                    else y[i] = a.negative ? w[i] ^ 0x80008000u : w[i];
                }
                *reinterpret_cast<uint4*>(dst + (c >> 3) * (128 * 128) + 16 * ((c & 7) ^ (rr & 7))) = make_uint4(y[0], y[1], y[2], y[3]);
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0) mbar_arrive(b_q + 8u * qi);
#pragma unroll 1
            for (int j = 0; j < n; ++j) {
                ok = ops_wait_warp(b_st + 8u * (j & 3), (uint32_t)(j >> 2) & 1u, kMxWait, dead);
                if (!ok) break;
                const float4* st = steps[j & 3];
                const int tok0 = (u0 + j) * kPrTile;
                // V's steps: the fast path has the sum of p from p times the step, and needs all of the unit's within 2^60 of the largest so far
                const float2 mine = *reinterpret_cast<const float2*>(&st[lane & 7]);
                most = fmaxf(most, mine.y);
                most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 1));
                most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 2));
                most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 4));
                const bool fast = __all_sync(0xffffffffu, mine.x >= 0.f && mine.y >= most * 0x1p-60f && mine.y > 1e-30f && most < 1e30f && lo <= tok0 && hi >= tok0 + kPrTile);
                float fk[8];
#pragma unroll
                for (int g = 0; g < 8; ++g) fk[g] = f * st[g].x;
                // (all of this before the scores are waited for)
                ok = ops_wait_warp(b_s + 8u * qi, (uint32_t)j & 1u, kMxWait, dead);
                if (!ok) break;
                tc_fence_after();
                uint32_t x[4][32];
#pragma unroll
                for (int c = 0; c < 4; ++c) tc_ld32(t_s + 32u * c, x[c]);
                tc_wait_ld();
#pragma unroll
                for (int c = 0; c < 4; ++c) pin32(x[c]);
                // which of the unit's tokens the row sees
                uint32_t sees[4];
                float mx = -INFINITY, my = -INFINITY;   // largest scores, and with V's steps
                if (!fast) {
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        const int t = tok0 + 32 * c;
                        const uint32_t from = lo <= t ? ~0u : lo - t >= 32 ? 0u : ~0u << (lo - t), to = hi - t >= 32 ? ~0u : hi <= t ? 0u : ~(~0u << (hi - t));
                        sees[c] = from & to & (st[2 * c].x < 0.f ? 0xFFFF0000u : ~0u) & (st[2 * c + 1].x < 0.f ? 0x0000FFFFu : ~0u);
#pragma unroll
                        for (int i = 0; i < 32; ++i)
                            if (!(sees[c] & (1u << i))) x[c][i] = 0xFF800000u;
                    }
                }
#pragma unroll
                for (int c = 0; c < 4; ++c)
#pragma unroll
                    for (int g = 0; g < 2; ++g) {
                        float v = __uint_as_float(x[c][16 * g + 15]);
#pragma unroll
                        for (int i = 0; i < 14; i += 2) v = max3(v, __uint_as_float(x[c][16 * g + i]), __uint_as_float(x[c][16 * g + i + 1]));
                        v = fmaxf(v, __uint_as_float(x[c][16 * g + 14]));
                        v *= fmaxf(fk[2 * c + g], 0.f);   // (a group that is not there: -inf x 0, no maximum)
                        mx = fmaxf(mx, v);
                        my = fmaxf(my, v + st[2 * c + g].z);
                    }
                // new maxima, only where an old one is 2^8 behind
                float alpha = 1.f;
                if (mx > m + 8.f || my > m - lead + 8.f) {
                    const float to = fmaxf(mx, m), now = fmaxf(to - fmaxf(my, m - lead), -126.f);   // (at most 126: no step's logarithm is below -126)
                    const float by = m - to;
                    alpha = exp2_fast(by + (now - lead));
                    l *= exp2_fast(by);
                    m = to;
                    lead = now;
                }
                if (__any_sync(0xffffffffu, alpha != 1.f) && j > 0) {   // (the sums so far are complete: their product was issued before S's)
#pragma unroll 1
                    for (int c = 0; c < D / 16; ++c) {
                        uint32_t o[16];
                        tc_ld16(t_o + 16u * c, o);
#pragma unroll
                        for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * alpha);
                        tc_st16_lanes(t_o + 16u * c, o);
                    }
                    tc_wait_st();
                }
                auto publish = [&](int half) {   // P of 64 tokens is in place: their product can begin
                    tc_wait_st();
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(b_p + 16u * qi + 8u * half);
                };
                const float base = 7.f - (m == -INFINITY ? 0.f : m);
                if (fast) {
                    const float back = exp2_fast(-lead);
                    float sum = 0.f;
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        uint32_t y[16];
                        // (step by step over the 32: all arguments, all exponentials, then what uses them)
#pragma unroll
                        for (int g = 0; g < 2; ++g) {
                            const float k = fk[2 * c + g], b = base + (st[2 * c + g].z + lead);
                            const uint64_t k2 = f32x2(k, k), b2 = f32x2(b, b);
#pragma unroll
                            for (int i = 16 * g; i < 16 * g + 16; i += 2) {
                                float e0, e1;
                                f32x2_split(fma2(f32x2(__uint_as_float(x[c][i]), __uint_as_float(x[c][i + 1])), k2, b2), e0, e1);
                                x[c][i] = __float_as_uint(e0);
                                x[c][i + 1] = __float_as_uint(e1);
                            }
                        }
#pragma unroll
                        for (int i = 0; i < 32; ++i) x[c][i] = __float_as_uint(exp2_fast(__uint_as_float(x[c][i])));
#pragma unroll
                        for (int g = 0; g < 2; ++g) {
                            uint64_t part = 0;
#pragma unroll
                            for (int i = 0; i < 8; ++i) {
                                const float e0 = __uint_as_float(x[c][16 * g + 2 * i]), e1 = __uint_as_float(x[c][16 * g + 2 * i + 1]);
                                part = add2(part, f32x2(e0, e1));
                                y[8 * g + i] = half2_bits(e0, e1);
                            }
                            float p0, p1;
                            f32x2_split(part, p0, p1);
                            sum = fmaf(p0 + p1, back * st[2 * c + g].w, sum);   // (p without V's step)
                        }
                        tc_st16_lanes(t_s + 16u * c, y);
                        if constexpr (REST) {
#pragma unroll
                            for (int i = 0; i < 16; ++i) y[i] = half2_rest(__uint_as_float(x[c][2 * i]), __uint_as_float(x[c][2 * i + 1]), y[i]);
                            tc_st16_lanes(t_s + 64u + 16u * c, y);
                        }
                        if (c == 1) publish(0);
                    }
                    l += sum;
                } else {
                    const float away = exp2_fast(lead);
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        uint32_t y[16], z[REST ? 16 : 1];
#pragma unroll
                        for (int g = 0; g < 2; ++g) {
                            const float2 kv = *reinterpret_cast<const float2*>(&st[2 * c + g]);
                            const float k = fk[2 * c + g], rel = kv.y * away;
#pragma unroll
                            for (int i = 0; i < 8; ++i) {
                                float e[2];
#pragma unroll
                                for (int b = 0; b < 2; ++b) {
                                    const int at = 16 * g + 2 * i + b;
                                    e[b] = exp2_fast(__uint_as_float(x[c][at]) * k + base);
                                    if (!(sees[c] & (1u << at))) e[b] = 0.f;
                                    l += e[b];
                                }
                                // (a group that is not there has no step)
                                const bool there = ((sees[c] >> (16 * g)) & 0xFFFFu) != 0;
                                const float p0 = e[0] == 0.f ? 0.f : e[0] * rel, p1 = e[1] == 0.f ? 0.f : e[1] * rel;
                                y[8 * g + i] = there ? half2_bits(p0, p1) : 0u;
                                if (REST) z[REST ? 8 * g + i : 0] = there ? half2_rest(p0, p1, y[8 * g + i]) : 0u;
                            }
                        }
                        tc_st16_lanes(t_s + 16u * c, y);
                        if constexpr (REST) tc_st16_lanes(t_s + 64u + 16u * c, z);
                        if (c == 1) publish(0);
                    }
                }
                publish(1);
            }
            if (ok) ok = ops_wait_warp(b_o + 8u * qi, 0, kMxWait, dead);
            tc_fence_after();
        }
        if (qi < nq && ok) {
            const float back = exp2_fast(-lead);
            // (kGroups, kOwn: the row's sums over a prefix)
            float* row = MODE == kAlone ? nullptr : a.rows.at + ((it.seq.first + tok) * a.Hq + qh) * a.rows.pitch;
            float keep = back, more = 0.f;   // factors of the sums here and there
            if (MODE == kOwn && a.splits == 1 && real && kv_has_prefix<MODE>(a.rows, it.s, it.seq.len)) {
                const float2 stat = __ldcg(reinterpret_cast<const float2*>(row + D));
                const float top = fmaxf(m, stat.x), base = top == -INFINITY ? 0.f : top, e = kv_weight(m, l, base);
                more = kv_weight(stat.x, stat.y, base);
                l = e * l + more * stat.y;
                keep *= e;
                m = top;
            }
            const float inv = l == 0.f ? 0.f : keep / l;
            if (MODE == kOwn) more = l == 0.f ? 0.f : more / l;
            float* part = a.part + (((int64_t)index * p.Hkv + h) * a.splits + split) * S::kPart;
            const bool parts = a.splits > 1 || (MODE == kGroups && a.beside);
            if (real && parts) {
                part[kPrRows * D + local] = m;
                part[kPrRows * D + kPrRows + local] = l;
            } else if (MODE == kGroups) {
                if (real) *reinterpret_cast<float2*>(row + D) = make_float2(m, l);
            } else if (real && a.lse) {
                a.lse[(it.seq.first + tok) * a.Hq + qh] = kv_lse(m, l);
            }
            uint16_t* dst = static_cast<uint16_t*>(a.out) + (it.seq.first + tok) * a.o_token + (int64_t)qh * a.o_head;
#pragma unroll 1
            for (int c = 0; c < (n == 0 && parts ? 0 : D / 32); ++c) {   // (a part without units has no sums)
                uint32_t x[32];
                if (n > 0) {
                    tc_ld32(t_o + 32u * c, x);
                    tc_wait_ld();
                    pin32(x);
                } else {
#pragma unroll
                    for (int i = 0; i < 32; ++i) x[i] = 0;
                }
                if (!real) continue;
                if (parts) {
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        *reinterpret_cast<float4*>(part + ((8 * c + i) * kPrRows + local) * 4) =
                            make_float4(__uint_as_float(x[4 * i]) * back, __uint_as_float(x[4 * i + 1]) * back, __uint_as_float(x[4 * i + 2]) * back, __uint_as_float(x[4 * i + 3]) * back);
                    continue;
                }
                if (MODE == kGroups) {
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        *reinterpret_cast<float4*>(row + 32 * c + 4 * i) =
                            make_float4(__uint_as_float(x[4 * i]) * back, __uint_as_float(x[4 * i + 1]) * back, __uint_as_float(x[4 * i + 2]) * back, __uint_as_float(x[4 * i + 3]) * back);
                    continue;
                }
                if (MODE == kOwn) {   // (a factor of 0 leaves sums out, whatever they are; l is NaN where a part is)
#pragma unroll
                    for (int i = 0; i < 32; i += 4) {
                        const float4 o = more == 0.f ? make_float4(0.f, 0.f, 0.f, 0.f) : __ldcg(reinterpret_cast<const float4*>(row + 32 * c + i));
                        const float z[4] = {o.x, o.y, o.z, o.w};
#pragma unroll
                        for (int k = 0; k < 4; ++k) x[i + k] = __float_as_uint((inv == 0.f ? 0.f : __uint_as_float(x[i + k]) * inv) + (more == 0.f ? 0.f : z[k] * more));
                    }
                }
                uint32_t y[16];
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const float v0 = l == 0.f ? 0.f : MODE == kOwn ? __uint_as_float(x[2 * i]) : __uint_as_float(x[2 * i]) * inv;
                    const float v1 = l == 0.f ? 0.f : MODE == kOwn ? __uint_as_float(x[2 * i + 1]) : __uint_as_float(x[2 * i + 1]) * inv;
                    if (BF16) {
                        const __nv_bfloat162 b = __floats2bfloat162_rn(v0, v1);
                        y[i] = *reinterpret_cast<const uint32_t*>(&b);
                    } else {
                        y[i] = half2_bits(v0, v1);
                    }
                }
                if (a.o_vec) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) *reinterpret_cast<uint4*>(dst + 32 * c + 8 * i) = make_uint4(y[4 * i], y[4 * i + 1], y[4 * i + 2], y[4 * i + 3]);
                } else {
#pragma unroll
                    for (int i = 0; i < 16; ++i) { dst[32 * c + 2 * i] = (uint16_t)y[i]; dst[32 * c + 2 * i + 1] = (uint16_t)(y[i] >> 16); }
                }
            }
            tc_fence_before();
        }
        }
    } else if (warp < 12) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 96;");
        if (have && n > 0) {
        // ================= codes -> fp16 operands =================
        // Warp w has tokens 32 w .. 32 w + 31 of a unit: two groups of 16, each in one block of the cache.
        const int w = warp - 8;
        const int32_t* row = a.seqs.table + (int64_t)it.s * a.seqs.table_stride;
        const int first_seen = a.window > 0 ? max(0, it.seq.len - it.seq.n + it.row0 / a.G - a.window + 1) : 0;
        // The block numbers of a unit are loaded two units ahead, its steps one: nothing here waits for a load that was just issued.
        int32_t blk[2] = {-1, -1};
        int64_t at[2] = {0, 0};   // the lane's first byte of the two groups (of the pool's first where a group is not there: its p is 0)
        const int64_t lane_at = (lane >> 2) * D + 16 * (lane & 3);
        float2 st[2];
        bool missing = false;
        auto token = [&](int j, int g) { return (u0 + j) * kPrTile + 32 * w + 16 * g; };
        auto needed = [&](int j, int t) { return j < n && t < it.seq.len && t + 16 > first_seen; };   // (blocks in front of every window may be gone)
        auto look = [&](int j) {
#pragma unroll
            for (int g = 0; g < 2; ++g) {
                const int t = token(j, g);
                blk[g] = needed(j, t) ? __ldcg(row + (t >> a.log2_T)) : 0;
            }
        };
        auto locate = [&](int j) {
#pragma unroll
            for (int g = 0; g < 2; ++g) {
                const int t = token(j, g);
                const bool in = (uint32_t)blk[g] < (uint32_t)p.blocks;
                at[g] = lane_at;
                st[g] = make_float2(-1.f, 0.f);
                if (needed(j, t)) {
                    missing |= !in;
                    if (in) {
                        const int64_t place = (int64_t)blk[g] * p.Hkv + h;
                        at[g] = ((place << a.log2_T) + (t & (p.T - 1))) * D + lane_at;
                        st[g] = make_float2(__ldcg(p.k_step + place), __ldcg(p.v_step + place));
                    }
                }
            }
        };
        // 16-byte pieces: rows of 4 lanes (64 bytes of D), 8 tokens an instruction, so that the stores below meet every bank once
        constexpr int IN = 4 * HALVES;
        auto fetch = [&](const int8_t* base, uint4 (&x)[IN]) {
#pragma unroll
            for (int i = 0; i < IN; ++i) {
                const int half = i % HALVES, t8 = i / HALVES;   // tokens 8 t8 .. of the warp's 32
                x[i] = __ldcg(reinterpret_cast<const uint4*>(base + at[t8 >> 1] + 8 * (t8 & 1) * D + 64 * half));
            }
        };
        auto store = [&](uint8_t* base, const uint4 (&x)[IN]) {
#pragma unroll
            for (int i = 0; i < IN; ++i) {
                const int half = i % HALVES, t8 = i / HALVES, t = 32 * w + 8 * t8 + (lane >> 2);
                uint8_t* d = base + half * (kPrTile * 128) + t * 128;
                const int c = 2 * (lane & 3);
                // (the loads are a unit old: nothing touches them before)
                const uint32_t x0 = x[i].x ^ 0x80808080u, x1 = x[i].y ^ 0x80808080u, x2 = x[i].z ^ 0x80808080u, x3 = x[i].w ^ 0x80808080u;
                *reinterpret_cast<uint4*>(d + 16 * (c ^ (t & 7))) = make_uint4(f16_low(x0), f16_high(x0), f16_low(x1), f16_high(x1));
                *reinterpret_cast<uint4*>(d + 16 * ((c + 1) ^ (t & 7))) = make_uint4(f16_low(x2), f16_high(x2), f16_low(x3), f16_high(x3));
            }
        };
        uint4 kx[IN], vx[IN];
        look(0);
        locate(0);
        look(1);
        fetch(p.k, kx);
        fetch(p.v, vx);
#pragma unroll 1
        for (int j = 0; j < n; ++j) {
            const int slot = j & 1;
            const uint32_t par = ((uint32_t)(j >> 1) & 1u) ^ 1u;
            const float2 here[2] = {st[0], st[1]};
            locate(j + 1);
            look(j + 2);
            ok = ops_wait_warp(b_ke + 8u * slot, par, kMxWait, dead);
            if (!ok) break;
            if (lane < 2) {
                const float2 s2 = lane ? here[1] : here[0];
                steps[j & 3][2 * w + lane] = make_float4(s2.x, s2.y, fminf(fmaxf(log2f(s2.y), -126.f), 128.f), 1.f / s2.y);
            }
            store(sk + slot * S::kKV, kx);
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0) { mbar_arrive(b_st + 8u * (j & 3)); mbar_arrive(b_kf + 8u * slot); }
            fetch(p.k, kx);
            ok = ops_wait_warp(b_ve + 8u * slot, par, kMxWait, dead);
            if (!ok) break;
            store(sv + slot * S::kKV, vx);
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0) mbar_arrive(b_vf + 8u * slot);
            fetch(p.v, vx);
        }
        if (missing) atomicExch(p.err, kErrIndex);
        }
    } else {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 64;");
        if (have && warp == 12 && n > 0) {
        // ================= MMA issue =================
        const uint32_t leader = tc_elect();
        const uint32_t id_s = (1u << 4) | (16u << 17) | (8u << 24);                              // fp32 += fp16 x fp16, both K-major, N = 128
        const uint32_t id_o = (1u << 4) | (1u << 16) | ((uint32_t)(D / 8) << 17) | (8u << 24);   // B (V) MN-major, N = D
        const uint64_t dq = mx4_desc(smem_u32(sq), 1024, 2), dk = mx4_desc(smem_u32(sk), 1024, 2);
        // V: 64 columns of D a swizzled row of 128 bytes; the next 64 after all tokens (leading offset), 8 tokens in 1024 bytes
        const uint64_t dv = mx4_desc(smem_u32(sv), 1024, 2) + (((uint64_t)((kPrTile * 128) >> 4) << 16) - (1ull << 16));
        auto scores = [&](int i, int slot) {
            const uint64_t a0 = dq + (uint32_t)(i * (S::kQ >> 4)), b0 = dk + (uint32_t)(slot * (S::kKV >> 4));
            const uint32_t d = tm + 128u * i;
#pragma unroll
            for (int k = 0; k < D / 16; ++k) tc_mma_f16(leader, d, a0 + ((k >> 2) * 1024 + (k & 3) * 2), b0 + ((k >> 2) * 1024 + (k & 3) * 2), id_s, k > 0);
        };
        auto output = [&](int i, int slot, int half, bool more) {
            const uint64_t b0 = dv + (uint32_t)(slot * (S::kKV >> 4) + 512 * half);
            const uint32_t d = tm + 256u + 128u * i, a0 = tm + 128u * i + 32u * half;
#pragma unroll
            for (int k = 0; k < 4; ++k) tc_mma_f16_ts(leader, d, a0 + 8u * k, b0 + 128u * k, id_o, more || half > 0 || k > 0);
            if (REST)
#pragma unroll
                for (int k = 0; k < 4; ++k) tc_mma_f16_ts(leader, d, a0 + 64u + 8u * k, b0 + 128u * k, id_o, 1);
        };
        for (int i = 0; i < nq && ok; ++i) ok = ops_wait_warp(b_q + 8u * i, 0, kMxWait, dead);
        if (ok) ok = ops_wait_warp(b_kf, 0, kMxWait, dead);
        tc_fence_after();
        if (ok) {
            for (int i = 0; i < nq; ++i) {
                scores(i, 0);
                tc_commit(leader, b_s + 8u * i);
            }
            tc_commit(leader, b_ke);
        }
        for (int j = 0; j < n && ok; ++j) {
            const int slot = j & 1, next = slot ^ 1;
            // (first what has long been there, so that nothing but P is waited for between the softmax and its products)
            ok = ops_wait_warp(b_vf + 8u * slot, (uint32_t)(j >> 1) & 1u, kMxWait, dead);
            if (ok && j + 1 < n) ok = ops_wait_warp(b_kf + 8u * next, (uint32_t)((j + 1) >> 1) & 1u, kMxWait, dead);
            for (int i = 0; i < nq && ok; ++i) {
                for (int half = 0; half < 2 && ok; ++half) {
                    ok = ops_wait_warp(b_p + 16u * i + 8u * half, (uint32_t)j & 1u, kMxWait, dead);
                    if (!ok) break;
                    tc_fence_after();
                    output(i, slot, half, j > 0);
                }
                if (!ok) break;
                if (i == nq - 1) tc_commit(leader, b_ve + 8u * slot);
                if (j + 1 < n) {
                    scores(i, next);
                    tc_commit(leader, b_s + 8u * i);
                    if (i == nq - 1) tc_commit(leader, b_ke + 8u * next);
                } else {
                    tc_commit(leader, b_o + 8u * i);
                }
            }
        }
        if (!ok) *dead = 1;
        // nothing is in flight when the tensor memory is given back
        tc_commit(leader, b_end);
        ops_wait(b_end, 0, kMxWait);
        __syncwarp();
        }
    }
    if (!ok && lane == 0) {
        *dead = 1;
        atomicExch(p.err, kErrTimeout);
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == 12) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tm));
}

// Joins the parts of a row tile that was split over the cache's length: a thread a row, 16 of D a block.
template <int D, bool BF16, int MODE = kAlone>
__global__ void __launch_bounds__(kPrRows) us_kv_prompt_join_kernel(const __grid_constant__ KvPrompt a)
{
    using S = PrShape<D>;
    const int lane = threadIdx.x & 31, local = threadIdx.x, c0 = 4 * (int)(blockIdx.x % (D / 16));
    const uint32_t u = blockIdx.x / (D / 16), index = u / (uint32_t)a.pool.Hkv;
    const int h = (int)(u - index * a.pool.Hkv);
    PrItem it;
    const bool have = pr_item<MODE>(a, index, lane, it, false);   // (lengths and token counts: complete before the kernel that left the parts went past its wait)
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    if (!have || local >= it.rows) return;
    const float* part = a.part + (int64_t)u * a.splits * S::kPart;
    float big = -INFINITY;
#pragma unroll 4
    for (int s = 0; s < a.splits; ++s) big = fmaxf(big, __ldcg(part + s * S::kPart + kPrRows * D + local));
    const float base = big == -INFINITY ? 0.f : big;
    float4 acc[4];
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) acc[i] = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 2
    for (int s = 0; s < a.splits; ++s) {
        const float* x = part + s * S::kPart;
        const float l = __ldcg(x + kPrRows * D + kPrRows + local), w = kv_weight(__ldcg(x + kPrRows * D + local), l, base);
        sum += w * l;             // (a part that is NaN has no maximum, and so no weight: its NaN comes from here)
        if (w == 0.f) continue;   // (a part without units has no sums)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float4 v = __ldcg(reinterpret_cast<const float4*>(x + ((c0 + i) * kPrRows + local) * 4));
            acc[i].x += w * v.x; acc[i].y += w * v.y; acc[i].z += w * v.z; acc[i].w += w * v.w;
        }
    }
    const int r = it.row0 + local, tok = r / a.G, qh = h * a.G + r - tok * a.G;
    if (MODE == kOwn) {
        const float* row = a.rows.at + ((it.seq.first + tok) * a.Hq + qh) * a.rows.pitch;
        if (kv_has_prefix<MODE>(a.rows, it.s, it.seq.len)) {
            const float2 stat = __ldcg(reinterpret_cast<const float2*>(row + D));
            const float own = big, own_sum = sum;
            float z[16] = {acc[0].x, acc[0].y, acc[0].z, acc[0].w, acc[1].x, acc[1].y, acc[1].z, acc[1].w, acc[2].x, acc[2].y, acc[2].z, acc[2].w, acc[3].x, acc[3].y, acc[3].z, acc[3].w};
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                big = own;
                sum = own_sum;
                kv_add_part(big, sum, z[i], stat, __ldcg(row + 4 * c0 + i));
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[i] = make_float4(z[4 * i], z[4 * i + 1], z[4 * i + 2], z[4 * i + 3]);
        }
    }
    const int64_t at = (it.seq.first + tok) * a.o_token + (int64_t)qh * a.o_head + 4 * c0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        o_put<BF16>(a.out, at + 4 * i, sum == 0.f ? 0.f : acc[i].x / sum);
        o_put<BF16>(a.out, at + 4 * i + 1, sum == 0.f ? 0.f : acc[i].y / sum);
        o_put<BF16>(a.out, at + 4 * i + 2, sum == 0.f ? 0.f : acc[i].z / sum);
        o_put<BF16>(a.out, at + 4 * i + 3, sum == 0.f ? 0.f : acc[i].w / sum);
    }
    if (a.lse && c0 == 0) a.lse[(it.seq.first + tok) * a.Hq + qh] = kv_lse(big, sum);
}

// (kGroups) The same into the rows: a thread a row, four of D a block, all parts' loads at once (64 sequences' rows of 64 heads, nine parts each, from memory: 9 us;
// 16 of D a block, two parts at a time: 14).
template <int D>
__global__ void __launch_bounds__(kPrRows) us_kv_rows_join_kernel(const __grid_constant__ KvPrompt a)
{
    using S = PrShape<D>;
    constexpr int MOST = 16;   // parts
    const int lane = threadIdx.x & 31, local = threadIdx.x, c = (int)(blockIdx.x % (D / 4));
    const uint32_t u = blockIdx.x / (D / 4), index = u / (uint32_t)a.pool.Hkv;
    const int h = (int)(u - index * a.pool.Hkv);
    PrItem it;
    const bool have = pr_item<kGroups>(a, index, lane, it, false);   // (complete, as above)
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    if (!have || local >= it.rows) return;
    const float* part = a.part + (int64_t)u * a.splits * S::kPart;
    float m[MOST], l[MOST];
    float4 x[MOST];
#pragma unroll
    for (int s = 0; s < MOST; ++s) {
        m[s] = -INFINITY;
        l[s] = 0.f;
        x[s] = make_float4(0.f, 0.f, 0.f, 0.f);
        if (s < a.splits) {
            m[s] = __ldcg(part + s * S::kPart + kPrRows * D + local);
            l[s] = __ldcg(part + s * S::kPart + kPrRows * D + kPrRows + local);
            x[s] = __ldcg(reinterpret_cast<const float4*>(part + s * S::kPart + (c * kPrRows + local) * 4));
        }
    }
    float big = -INFINITY, sum = 0.f;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int s = 0; s < MOST; ++s) big = fmaxf(big, m[s]);
#pragma unroll
    for (int s = 0; s < MOST; ++s) {
        const float w = kv_weight(m[s], l[s], big == -INFINITY ? 0.f : big);
        sum += w * l[s];          // (a part that is NaN has no maximum, and so no weight: its NaN comes from here)
        if (w == 0.f) continue;   // (a part without units has no sums)
        acc.x += w * x[s].x; acc.y += w * x[s].y; acc.z += w * x[s].z; acc.w += w * x[s].w;
    }
    const int r = it.row0 + local, tok = r / a.G, qh = h * a.G + r - tok * a.G;
    float* row = a.rows.at + ((it.seq.first + tok) * a.Hq + qh) * a.rows.pitch;
    *reinterpret_cast<float4*>(row + 4 * c) = acc;
    if (c == 0) *reinterpret_cast<float2*>(row + D) = make_float2(big, sum);
}

// The last step beside: the groups' parts and the rows of the own tokens. A thread has four of D of a row: 64 rows and 16 of D a block, all loads at once.
template <int D, bool BF16>
__global__ void __launch_bounds__(256) us_kv_shared_join_kernel(const __grid_constant__ KvPrompt a)
{
    using S = PrShape<D>;
    constexpr int MOST = 16, PER = 4 * (D / 16);   // parts; blocks of a row tile and head
    const int lane = threadIdx.x & 31, b = (int)(blockIdx.x % PER), local = 64 * (b & 3) + ((int)threadIdx.x & 63), c = 4 * (b >> 2) + ((int)threadIdx.x >> 6);
    const uint32_t u = blockIdx.x / PER, index = u / (uint32_t)a.pool.Hkv;
    const int h = (int)(u - index * a.pool.Hkv);
    PrItem it;
    const bool have = pr_item<kGroups>(a, index, lane, it, false);   // (complete, as above)
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    if (!have || local >= it.rows) return;
    const int r = it.row0 + local, tok = r / a.G, qh = h * a.G + r - tok * a.G;
    const float* row = a.rows.own + ((it.seq.first + tok) * a.Hq + qh) * a.rows.pitch;
    const float* part = a.part + (int64_t)u * a.splits * S::kPart;
    float m[MOST + 1], l[MOST + 1];
    float4 x[MOST + 1];
    const float2 stat = __ldcg(reinterpret_cast<const float2*>(row + D));
    m[MOST] = stat.x;
    l[MOST] = stat.y;
    x[MOST] = __ldcg(reinterpret_cast<const float4*>(row + 4 * c));
#pragma unroll
    for (int s = 0; s < MOST; ++s) {
        m[s] = -INFINITY;
        l[s] = 0.f;
        x[s] = make_float4(0.f, 0.f, 0.f, 0.f);
        if (s < a.splits) {
            m[s] = __ldcg(part + s * S::kPart + kPrRows * D + local);
            l[s] = __ldcg(part + s * S::kPart + kPrRows * D + kPrRows + local);
            x[s] = __ldcg(reinterpret_cast<const float4*>(part + s * S::kPart + (c * kPrRows + local) * 4));
        }
    }
    if (kv_row_done(stat)) return;   // (a padded row: it has its output)
    float big = -INFINITY, sum = 0.f;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int s = 0; s <= MOST; ++s) big = fmaxf(big, m[s]);
#pragma unroll
    for (int s = 0; s <= MOST; ++s) {
        const float w = kv_weight(m[s], l[s], big == -INFINITY ? 0.f : big);
        sum += w * l[s];          // (a part that is NaN has no maximum, and so no weight: its NaN comes from here)
        if (w == 0.f) continue;   // (a part without units has no sums)
        acc.x += w * x[s].x; acc.y += w * x[s].y; acc.z += w * x[s].z; acc.w += w * x[s].w;
    }
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
    const float y[4] = {acc.x * inv, acc.y * inv, acc.z * inv, acc.w * inv};
    uint16_t* out = static_cast<uint16_t*>(a.out) + (it.seq.first + tok) * a.o_token + (int64_t)qh * a.o_head + 4 * c;
    uint16_t v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = BF16 ? __bfloat16_as_ushort(__float2bfloat16_rn(sum == 0.f ? 0.f : y[i])) : __half_as_ushort(__float2half_rn(sum == 0.f ? 0.f : y[i]));
    if (a.o_vec) *reinterpret_cast<uint2*>(out) = make_uint2(v[0] | ((uint32_t)v[1] << 16), v[2] | ((uint32_t)v[3] << 16));
    else
#pragma unroll
        for (int i = 0; i < 4; ++i) out[i] = v[i];
    if (a.lse && c == 0) a.lse[(it.seq.first + tok) * a.Hq + qh] = kv_lse(big, sum);
}

}  // namespace us
