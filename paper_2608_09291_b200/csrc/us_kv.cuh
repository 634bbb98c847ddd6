// The cache of keys and values in 8 bits: append, read back, and attention over it.
//
// Pool of blocks of T tokens; codes int8 [block][kv head][T][D], one fp32 step for each (block, kv head), K and V apart:
// value = code * step. A sequence's token t lies in block table[s][t / T] at place t % T.
#pragma once
#include "us_mx4.cuh"

#include <cuda.h>

namespace us {

constexpr uint32_t kErrIndex = 2;   // a block number outside the pool, a length beyond the table, token counts that do not add up

struct KvSeqs {
    const int32_t* table;     // S rows of `width` block numbers
    int64_t table_stride;
    const int32_t* lengths;   // S, the new tokens included
    const int32_t* cu;        // S + 1 sums of the new tokens of the sequences before, or nullptr: one each
    int32_t S, width;
    int64_t N;                // new tokens
};

struct KvPool {
    int8_t *k, *v;
    float *k_step, *v_step;
    int32_t blocks, Hkv, T, D;
    uint32_t* err;
};

struct KvSeq {
    int64_t first;      // row of its first new token
    int32_t len, n;     // tokens in all, new ones (which may be more only where the sequence is empty, or wrong)
};
// Sequence s with everything that memory depends on brought into range; `wrong`: something was not. (An empty sequence may have rows: those
// of a padded batch.)
__device__ __forceinline__ KvSeq kv_seq(const KvSeqs& q, const KvPool& p, int s, bool& wrong)
{
    KvSeq r;
    const int64_t most = (int64_t)q.width * p.T;
    const int32_t len = __ldcg(q.lengths + s);
    int64_t a = s, b = (int64_t)s + 1;
    if (q.cu) { a = __ldcg(q.cu + s); b = __ldcg(q.cu + s + 1); }
    wrong = len < 0 || len > most || a < 0 || b < a || b > q.N || (len > 0 && b - a > len);
    r.len = (int32_t)max((int64_t)0, min((int64_t)len, most));
    r.first = max((int64_t)0, min(a, q.N));
    r.n = (int32_t)max((int64_t)0, min(b, q.N) - r.first);
    return r;
}

// ---- append --------------------------------------------------------------------------------------------------------------
// A team of 32 to 128 threads has a block and head: the largest new magnitude first, then codes, and the older codes once more where the step
// grew. Blocks have no order among them. Bound by memory where prompts are written (3 of up to 2000 tokens, 32 heads of 128, and contexts of up to
// 2500 read back: 86 us for both, 57 at memory's rate; the writing alone 35, 11 at that rate: blocks of 16 tokens, a team each), by the chain length -> table
// -> step -> codes where single tokens are (64: 4.8 us; with 300 tokens each read back 37, 27 of them the reading's bytes).
// code = RNE(x / s) for the exact quotient, x finite or not. The rounded product x * (1 / s) is within 2^-16 of the quotient: its nearest
// integer is the code unless it lies that close to a border (1 of 25000 values; kv_code_near), where the sign of a fused multiply-add says on which side x
// is (exact: a rounded sum is never on the other side of 0), or underflow would lose the border, where 64 bits decide.
__device__ __noinline__ int kv_code_near(float x, float s, float inv)
{
    if (s < 1e-30f) {
        const double q = s > 0.f ? rint((double)x / (double)s) : 0.0;
        return q != q ? 0 : (int)fmin(fmax(q, -127.0), 127.0);
    }
    float r = rintf(x * inv);
    const float up = fmaf(-(r + 0.5f), s, x), down = fmaf(-(r - 0.5f), s, x);
    const bool odd = (r - 2.f * truncf(0.5f * r)) != 0.f;
    if (up > 0.f || (up == 0.f && odd)) r += 1.f;
    else if (down < 0.f || (down == 0.f && odd)) r -= 1.f;
    return r != r ? 0 : (int)fminf(fmaxf(r, -127.f), 127.f);
}
// Eight of them; inv = 0 sends all to kv_code_near.
template <class T_>
__device__ __forceinline__ uint2 kv_codes8(const Eight<T_>& e, float s, float inv)
{
    uint32_t w[2] = {0, 0};
    float far = 0.f;   // the largest distance from an integer
    bool fine = inv > 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float x = to_f32(e.v[i]);
        const float t = fmaf(x, inv, 12582912.f);   // 1.5 2^23: the nearest integer in the low bits
        far = fmaxf(far, fabsf(fmaf(x, inv, 12582912.f - t)));
        fine = fine && fabsf(x) < 3.3e38f;   // (the maximum above passes over NaN)
        w[i >> 2] |= (__float_as_uint(t) & 0xFFu) << (8 * (i & 3));
    }
    if (!(fine && far < 0.49998f)) {
        w[0] = w[1] = 0;
#pragma unroll 1
        for (int i = 0; i < 8; ++i) {
            float x = 0.f;
#pragma unroll
            for (int k = 0; k < 8; ++k) if (k == i) x = to_f32(e.v[k]);
            const uint32_t c = ((uint32_t)kv_code_near(x, s, inv) & 0xFFu) << (8 * (i & 3));
            if (i < 4) w[0] |= c;
            else w[1] |= c;
        }
    }
    return make_uint2(w[0], w[1]);
}

struct KvAppend {
    KvPool pool;
    KvSeqs seqs;
    const void* x[2];              // K, V: new tokens
    int64_t token_stride[2], head_stride[2];
    int32_t vec;                   // rows take 16-byte loads
    int32_t log2_T;
};

// A team of TEAM threads takes one block that gets tokens, one head, K or V: largest magnitude, step, the older codes if the step grew,
// the new codes. A block of the grid has the teams of 128 / TEAM heads. The new tokens are on their way before the block's number is
// known. Bound by the bytes of the new tokens where there are many, by latency (lengths; tokens and block number; the block's step) for
// single ones.
template <class T_, int TEAM>
__global__ void __launch_bounds__(128) us_kv_append_kernel(const __grid_constant__ KvAppend a)
{
    __shared__ uint32_t red[4];
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const KvPool& p = a.pool;
    const int lane = threadIdx.x & 31, me = threadIdx.x % TEAM, which = blockIdx.z;
    // (A team past the last head has nothing to do but the barrier: codes are rescaled in place, which nobody may do a second time.)
    const int h = (int)(blockIdx.y * (128 / TEAM) + threadIdx.x / TEAM);
    const bool real = h < p.Hkv;
    // which sequence's which block
    int s = -1, j = 0;
    uint32_t before = 0;
    bool any_wrong = false;
    KvSeq q = {0, 0, 0};
    for (int base = 0; base < a.seqs.S; base += 32) {
        uint32_t cnt = 0;
        KvSeq mine = {0, 0, 0};
        if (base + lane < a.seqs.S) {
            bool wrong;
            mine = kv_seq(a.seqs, p, base + lane, wrong);
            any_wrong |= wrong;
            if (mine.n > 0 && mine.n <= mine.len && !wrong) cnt = ((mine.len - 1) >> a.log2_T) - ((mine.len - mine.n) >> a.log2_T) + 1;
        }
        uint32_t sum = cnt;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const uint32_t v = __shfl_up_sync(0xffffffffu, sum, o);
            if (lane >= o) sum += v;
        }
        const uint32_t who = __ballot_sync(0xffffffffu, blockIdx.x >= before + sum - cnt && blockIdx.x < before + sum);
        if (who) {
            const int l = __ffs(who) - 1;
            s = base + l;
            j = (int)(blockIdx.x - before - __shfl_sync(0xffffffffu, sum - cnt, l));
            q.first = __shfl_sync(0xffffffffu, mine.first, l);
            q.len = __shfl_sync(0xffffffffu, mine.len, l);
            q.n = __shfl_sync(0xffffffffu, mine.n, l);
            break;
        }
        before += __shfl_sync(0xffffffffu, sum, 31);
    }
    if (any_wrong) atomicExch(p.err, kErrIndex);
    if (s < 0) return;
    const int start = q.len - q.n, bi = (start >> a.log2_T) + j;
    const int lo = max(start, bi << a.log2_T), hi = min(q.len, (bi + 1) << a.log2_T), held = lo - (bi << a.log2_T), n = hi - lo;
    const int32_t blk = __ldcg(a.seqs.table + (int64_t)s * a.seqs.table_stride + bi);
    const int D = p.D, log2_per = D == 128 ? 4 : 3;   // D / 8 lanes a row
    const T_* x = static_cast<const T_*>(a.x[which]) + (q.first + lo - start) * a.token_stride[which] + (int64_t)h * a.head_stride[which];
    const int units = real ? n << log2_per : 0;
    constexpr int KEEP = sizeof(T_) == 4 ? 4 : 8;
    Eight<T_> kept[KEEP];
    uint32_t big = 0;
    auto load = [&](int u) {
        const int r = u >> log2_per, c = u & ((1 << log2_per) - 1);
        return load8(x + r * a.token_stride[which] + 8 * c, 8, a.vec != 0);
    };
    auto take = [&](const Eight<T_>& e) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t b = __float_as_uint(to_f32(e.v[i])) & 0x7FFFFFFFu;
            if (b < 0x7F800000u) big = max(big, b);   // (infinities and NaN do not count)
        }
    };
#pragma unroll
    for (int i = 0; i < KEEP; ++i)
        if (me + TEAM * i < units) kept[i] = load(me + TEAM * i);
    if (blk < 0 || blk >= p.blocks) {   // (all teams of the grid's block)
        if (threadIdx.x == 0) atomicExch(p.err, kErrIndex);
        return;
    }
    const int64_t place = (int64_t)blk * p.Hkv + h;
    float* step_at = (which ? p.v_step : p.k_step) + place;
    int8_t* codes = (which ? p.v : p.k) + ((place << a.log2_T) * D);
    const float old = held && real ? *step_at : 0.f;
#pragma unroll
    for (int i = 0; i < KEEP; ++i)
        if (me + TEAM * i < units) take(kept[i]);
    for (int u = me + TEAM * KEEP; u < units; u += TEAM) take(load(u));
    big = __reduce_max_sync(0xffffffffu, big);
    if (TEAM > 32) {
        if (lane == 0) red[threadIdx.x >> 5] = big;
        __syncthreads();
        const int w0 = threadIdx.x / TEAM * (TEAM / 32);
#pragma unroll
        for (int i = 0; i < TEAM / 32; ++i) big = max(big, red[w0 + i]);
    } else {
        __syncwarp();   // (all lanes have read the old step)
    }
    if (!real) return;
    const float step = fmaxf(old, __fdiv_rn(__uint_as_float(big), 127.f));
    if (me == 0) *step_at = step;
    const float inv = step >= 1e-30f ? __fdiv_rn(1.f, step) : 0.f;
    auto put = [&](int u, const Eight<T_>& e) { *reinterpret_cast<uint2*>(codes + (int64_t)held * D + 8 * (int64_t)u) = kv_codes8(e, step, inv); };
#pragma unroll
    for (int i = 0; i < KEEP; ++i)
        if (me + TEAM * i < units) put(me + TEAM * i, kept[i]);
    for (int u = me + TEAM * KEEP; u < units; u += TEAM) put(u, load(u));
    if (step > old && held) {   // the tokens that were there, in the larger step: RNE(code * old / step), close to a border decided in 64 bits
        const float ratio = __fdiv_rn(old, step);   // (the product with a code is within 2^-16 of the quotient)
        for (int u = me; u < held * D / 8; u += TEAM) {
            uint2* at = reinterpret_cast<uint2*>(codes) + u;
            const uint2 w = *at;
            uint32_t o[2] = {0, 0};
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int c = (int8_t)((i < 4 ? w.x : w.y) >> (8 * (i & 3)));
                const float t = fmaf((float)c, ratio, 12582912.f);
                uint32_t n = __float_as_uint(t);
                if (!(fabsf(fmaf((float)c, ratio, 12582912.f - t)) < 0.49998f) || step < 1e-30f) n = (uint32_t)(int)rint((double)c * (double)old / (double)step);
                o[i >> 2] |= (n & 0xFFu) << (8 * (i & 3));
            }
            *at = make_uint2(o[0], o[1]);
        }
    }
}

// ---- read ------------------------------------------------------------------------------------------------------------------
// value = RN(code * step), 16 tokens of kReadHeads heads a block; bound by the values it writes.
// K and V of the first `tokens` places of every sequence as values, [s][t][head][D]; 0 from a sequence's end on. Block (x, y, z): 16 tokens
// (in one block of the cache, as every block has a multiple of 16) of sequence z, kReadHeads heads. A thread has 16 bytes of the
// output at a time, so that a warp's stores are whole lines, four of them in flight. Bound by the bytes written.
constexpr int kReadHeads = 4;
template <class T_>
__global__ void __launch_bounds__(256) us_kv_read_kernel(KvPool p, KvSeqs q, int64_t tokens, int log2_T, T_* k_out, T_* v_out)
{
    constexpr int PER = 16 / (int)sizeof(T_), U = 4;   // columns of a piece
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int log2_row = (p.D == 128 ? 7 : 6) - (PER == 8 ? 3 : 2);   // pieces of a (token, head)
    const int64_t t0 = 16 * (int64_t)blockIdx.x, most = (int64_t)q.width << log2_T;
    const int h0 = kReadHeads * blockIdx.y;
    for (int s = blockIdx.z; s < q.S; s += gridDim.z) {
        const int32_t len = __ldcg(q.lengths + s);
        const bool wrong = len < 0 || len > most;
        const int seen = (int)max((int64_t)0, min((int64_t)16, min((int64_t)len, most) - t0));   // tokens here that the sequence has
        int32_t blk = 0;
        bool there = false;
        if (seen > 0) {
            blk = __ldcg(q.table + (int64_t)s * q.table_stride + (t0 >> log2_T));
            there = blk >= 0 && blk < p.blocks;
        }
        if (threadIdx.x == 0 && (wrong || (seen > 0 && !there))) atomicExch(p.err, kErrIndex);
        const int here = (int)min((int64_t)16, tokens - t0), units = here * kReadHeads << log2_row;
        const int64_t place0 = (int64_t)blk * p.Hkv, tok0 = t0 & ((1 << log2_T) - 1), out0 = (s * tokens + t0) * p.Hkv;
#pragma unroll 1
        for (int u0 = threadIdx.x; u0 < units; u0 += U * 256) {
            uint2 w[U][2];
            float f[U][2];
#pragma unroll
            for (int i = 0; i < U; ++i) {
                const int u = u0 + 256 * i, row = u >> log2_row, c = u & ((1 << log2_row) - 1), t = row / kReadHeads, h = h0 + row % kReadHeads;
                w[i][0] = w[i][1] = make_uint2(0, 0);
                f[i][0] = f[i][1] = 0.f;
                if (u < units && h < p.Hkv && there && t < seen) {
                    const int64_t at = (((place0 + h) << log2_T) + tok0 + t) * p.D + PER * c;
                    if (PER == 8) {
                        w[i][0] = __ldcg(reinterpret_cast<const uint2*>(p.k + at));
                        w[i][1] = __ldcg(reinterpret_cast<const uint2*>(p.v + at));
                    } else {
                        w[i][0].x = __ldcg(reinterpret_cast<const uint32_t*>(p.k + at));
                        w[i][1].x = __ldcg(reinterpret_cast<const uint32_t*>(p.v + at));
                    }
                    f[i][0] = __ldcg(p.k_step + place0 + h);
                    f[i][1] = __ldcg(p.v_step + place0 + h);
                }
            }
#pragma unroll
            for (int i = 0; i < U; ++i) {
                const int u = u0 + 256 * i, row = u >> log2_row, c = u & ((1 << log2_row) - 1), t = row / kReadHeads, h = h0 + row % kReadHeads;
                if (u >= units || h >= p.Hkv) continue;
#pragma unroll
                for (int b = 0; b < 2; ++b) {
                    union { uint4 v; T_ e[PER]; } y;
#pragma unroll
                    for (int k = 0; k < PER; ++k) y.e[k] = from_f32<T_>((float)(int8_t)((k < 4 ? w[i][b].x : w[i][b].y) >> (8 * (k & 3))) * f[i][b]);
                    __stcs(reinterpret_cast<uint4*>((b ? v_out : k_out) + (out0 + (int64_t)t * p.Hkv + h) * p.D + PER * c), y.v);
                }
            }
        }
    }
}

// ---- attention: few query rows a cache head (decode) ---------------------------------------------------------------------------
// out = sum_t p_t v_t / sum_t p_t, p_t = 2^(s_t - m), s = scale log2(e) q.k, in one pass with the running maximum m of each row.
//   * The rows of a tile are the query heads that share a cache head (times the sequence's new tokens): 8 NT of them are the N side
//     of mma.sync m16n8k16, 16 tokens (then 16 of D) the M side: the cache's bytes are read once for all of them.
//   * Codes become fp16 in registers, exactly (0x6400 | byte is 1024 + byte); a step is one number for 16 tokens, so K's is
//     a factor of the scores and V's a factor of p. What is rounded to fp16 is p v_step 2^7 relative to a second running maximum of
//     each row, that of s_t + log2 v_step: terms down to 2^-21 of a row's largest keep their 11 bits, whatever the steps of tokens
//     are that it does not see or that have no weight in it. sum p v is held relative to that one, sum p relative to m; both are fp32.
//   * Both follow the true maximum only where one is 2^8 behind, so most units need no reduction over lanes and no rescaling.
//   * All (sequence, row tile, head) items in a row, 128 tokens a unit and kKvStart units for beginning one: every CTA takes the same
//     number of units, whatever the lengths. (64 sequences of 1 to 8192 tokens, 64/8 heads, inside a graph: 148 us without the units for beginning,
//     where the CTAs with the short sequences were last, 120 with 2, 110 with 3, 104 with 4.) An item that is cut leaves its parts in scratch, and a second kernel joins
//     them in the order of the CTAs.
// A warp copies (TMA, swizzled so that the fragment loads meet no bank twice); four read, 32 tokens of a unit each (two groups side by
// side: their chains of products overlap), with sums of their own that are joined at an item's end.
// Bound by memory: 64 sequences of up to 8192 tokens, 64/8 heads, bf16: 98 us inside a graph, 5.7 TB/s (109 called); one of 131072 tokens, fp16:
// 55 us, 4.9 TB/s (59 called).
constexpr int kKvTile = 128;
constexpr int kKvStart = 4;   // what an item's queries, sums and output cost, in units
struct KvAttend {
    CUtensorMap k_map, v_map;
    KvPool pool;
    KvSeqs seqs;
    const void* q;
    int64_t q_token, q_head;
    void* out;
    int64_t o_token, o_head;
    float* lse;
    float* part;             // two parts a CTA: rows x D sums, then rows x {m, l}
    float scale2;            // scale log2(e)
    int32_t Hq, G;           // query heads, a cache head's
    int32_t causal, window;
    int32_t q_vec;
    int32_t stages;
    int32_t ctas;
    int32_t log2_T;
};

struct KvItem {
    KvSeq seq;
    int32_t rows;        // query rows of a head
    int32_t row_tiles;
    int32_t lo;          // first token that any of its queries sees
    int32_t t_lo, tiles; // first unit of the cache, units (1 if it sees nothing)
    __device__ __forceinline__ int cost() const { return kKvStart + tiles; }
};
template <int R>
__device__ __forceinline__ KvItem kv_item(const KvAttend& a, const KvSeq& seq)
{
    KvItem r;
    r.seq = seq;
    r.rows = r.seq.n * a.G;
    r.row_tiles = (r.rows + R - 1) / R;
    r.lo = a.window > 0 ? max(0, r.seq.len - r.seq.n - a.window + 1) : 0;
    r.t_lo = r.lo / kKvTile;
    r.tiles = max(1, (r.seq.len + kKvTile - 1) / kKvTile - r.t_lo);
    return r;
}
template <int R>
__device__ __forceinline__ KvItem kv_item(const KvAttend& a, int s)
{
    bool wrong;
    return kv_item<R>(a, kv_seq(a.seqs, a.pool, s, wrong));
}

// The units of all items in a row, cut in equal shares: CTA c has [begin(c), begin(c + 1)).
struct KvShares {
    long long total, each;
    int more;             // the first `more` CTAs have one unit more
    __device__ __forceinline__ long long begin(int c) const { return each * c + min(c, more); }
    __device__ __forceinline__ int owner(long long unit) const
    {
        const long long cut = (each + 1) * more;
        return (int)(unit < cut ? unit / (each + 1) : more + (unit - cut) / each);
    }
};
// Its own share, and where that begins. (All lanes of a warp; one trip to the lengths for up to 32 sequences.)
struct KvRange {
    KvShares shares;
    long long u0, u1;
    int s;                // sequence of unit u0
    long long in_seq;     // u0 from its first unit
    KvItem item;          // of that sequence
};
template <int R>
__device__ __forceinline__ KvRange kv_range(const KvAttend& a, int cta, int lane, bool report)
{
    KvRange r;
    r.shares.total = 0;
    bool any = false;
    KvSeq mine = {0, 0, 0};   // of the last sequences looked at
    long long c = 0, sum = 0;
    auto look = [&](int base) {
        c = 0;
        if (base + lane < a.seqs.S) {
            bool wrong;
            mine = kv_seq(a.seqs, a.pool, base + lane, wrong);
            any |= wrong;
            const KvItem it = kv_item<R>(a, mine);
            c = (long long)it.row_tiles * a.pool.Hkv * it.cost();
        }
        sum = c;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const long long v = __shfl_up_sync(0xffffffffu, sum, o);
            if (lane >= o) sum += v;
        }
    };
    for (int base = 0; base < a.seqs.S; base += 32) {
        look(base);
        r.shares.total += __shfl_sync(0xffffffffu, sum, 31);
    }
    if (any && report) atomicExch(a.pool.err, kErrIndex);
    if (r.shares.total >> 32) {
        r.shares.each = r.shares.total / a.ctas;
    } else {
        r.shares.each = (uint32_t)r.shares.total / (uint32_t)a.ctas;
    }
    r.shares.more = (int)(r.shares.total - r.shares.each * a.ctas);
    r.u0 = r.shares.begin(cta);
    r.u1 = r.shares.begin(cta + 1);
    r.s = a.seqs.S;
    r.in_seq = 0;
    if (r.u0 >= r.u1) return r;
    long long before = 0;
    for (int base = 0; base < a.seqs.S; base += 32) {
        if (a.seqs.S > 32) look(base);
        const uint32_t who = __ballot_sync(0xffffffffu, r.u0 < before + sum);
        if (who) {
            const int l = __ffs(who) - 1;
            r.s = base + l;
            r.in_seq = r.u0 - before - __shfl_sync(0xffffffffu, sum - c, l);
            KvSeq q;
            q.first = __shfl_sync(0xffffffffu, mine.first, l);
            q.len = __shfl_sync(0xffffffffu, mine.len, l);
            q.n = __shfl_sync(0xffffffffu, mine.n, l);
            r.item = kv_item<R>(a, q);
            break;
        }
        before += __shfl_sync(0xffffffffu, sum, 31);
    }
    return r;
}
__device__ __forceinline__ int kv_div(long long a, int b) { return a >> 31 ? (int)(a / b) : (int)((uint32_t)a / (uint32_t)b); }

__device__ __forceinline__ uint32_t f16_low(uint32_t w)    // bytes 0, 1 of (code ^ 0x80) -> two fp16
{
    const __half2 r = __hsub2(*reinterpret_cast<const __half2*>(&(w = prmt(w, 0x64646464u, 0x4140u))), __floats2half2_rn(1152.f, 1152.f));
    return *reinterpret_cast<const uint32_t*>(&r);
}
__device__ __forceinline__ uint32_t f16_high(uint32_t w)   // bytes 2, 3
{
    const __half2 r = __hsub2(*reinterpret_cast<const __half2*>(&(w = prmt(w, 0x64646464u, 0x4342u))), __floats2half2_rn(1152.f, 1152.f));
    return *reinterpret_cast<const uint32_t*>(&r);
}
__device__ __forceinline__ void mma_f16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose8(uint32_t v)
{
    uint32_t r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
    return r;
}
__device__ __forceinline__ float exp2_fast(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ uint32_t half2_bits(float a, float b)
{
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ void tma_rows(uint32_t dst, const CUtensorMap* map, int32_t row, uint32_t bar)
{
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
                 ::"r"(dst), "l"(map), "r"(0), "r"(row), "r"(bar) : "memory");
}
// Barrier of the four reading warps: whether any of them says `fail`.
__device__ __forceinline__ bool bar_consumers(bool fail = false)
{
    uint32_t any;
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\tbarrier.cta.red.or.pred q, 1, 128, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
                 : "=r"(any) : "r"((uint32_t)fail) : "memory");
    return any != 0;
}
// A number that log2 of a step is at most; -126 at least, so that what it is added to is not lost
__device__ __forceinline__ float kv_log2_above(float step) { return (float)((int)((__float_as_uint(step) >> 23) & 0xFFu) - 126); }
template <bool BF16>
__device__ __forceinline__ float q_at(const void* q, int64_t i) { return BF16 ? __bfloat162float(static_cast<const __nv_bfloat16*>(q)[i]) : __half2float(static_cast<const __half*>(q)[i]); }
template <bool BF16>
__device__ __forceinline__ void o_put(void* out, int64_t i, float y)
{
    if (BF16) static_cast<__nv_bfloat16*>(out)[i] = __float2bfloat16_rn(y);
    else static_cast<__half*>(out)[i] = __float2half_rn(y);
}
// log of the softmax's sum from a maximum (or -inf) and a sum that carries 2^7
__device__ __forceinline__ float kv_lse(float m, float l) { return l == 0.f ? -INFINITY : ((m == -INFINITY ? 0.f : m) + log2f(l) - 7.f) * 0.69314718f; }
// 2^(m - base) for a part with this maximum and sum; 0 for one that saw nothing
__device__ __forceinline__ float kv_weight(float m, float l, float base) { return m == -INFINITY && l == 0.f ? 0.f : exp2_fast(m - base); }

template <int D, int NT>
struct KvShape {
    static constexpr int R = 8 * NT;
    static constexpr int kHalf = kKvTile * D;                 // bytes of a stage's K (or V)
    static constexpr int kStage = 2 * kHalf;
    static constexpr int kPitch = D + 4;                      // floats of a row of the warps' sums
    static constexpr int kMerge = R * kPitch * 4 + 5 * R * 2 * 4;
    static constexpr int kMaxStages = 8;
    static constexpr int kPart = R * (D + 2);                 // floats of a part
};

template <int D, int NT, bool BF16>
__global__ void __launch_bounds__(160, 2) us_kv_attend_kernel(const __grid_constant__ KvAttend a)
{
    using S = KvShape<D, NT>;
    constexpr int R = S::R, KS = D / 16, MT = D / 16;
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    __shared__ __align__(8) uint64_t bars[2 * S::kMaxStages];
    __shared__ float2 steps[S::kMaxStages][8];   // of a unit's 16-token groups: K's (-1: not there), V's
    __shared__ uint32_t dead_word;
    uint8_t* ring = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
    float* sums = reinterpret_cast<float*>(ring + (size_t)a.stages * S::kStage);   // [row][pitch]
    float2* stats = reinterpret_cast<float2*>(sums + R * S::kPitch);               // [warp][row] m, l; then the four together
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t b_full = smem_u32(bars), b_empty = b_full + 8u * S::kMaxStages;
    volatile uint32_t* dead = &dead_word;
    if (threadIdx.x < (unsigned)a.stages) { mbar_init(b_full + 8u * threadIdx.x, 1); mbar_init(b_empty + 8u * threadIdx.x, 4); }
    if (threadIdx.x == 0) dead_word = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    __syncthreads();
    // The kernel that joins the parts may start once this one's CTAs are past the wait: it reads lengths and token counts before its own.
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const KvPool& p = a.pool;
    const KvRange range = kv_range<R>(a, blockIdx.x, lane, warp == 0);
    long long left = range.u1 - range.u0;
    bool ok = true;
    int stage = 0;
    uint32_t par = 0;
    int s = range.s;
    KvItem it = range.item;
    int item = 0, at_unit = 0;   // item of the sequence (row tile * Hkv + head), unit of the item (kKvStart of them before its first tokens)
    if (left > 0) {
        item = kv_div(range.in_seq, it.cost());
        at_unit = (int)(range.in_seq - (long long)item * it.cost());
    }
    auto next_seq = [&]() {   // (the units of this CTA end before the sequences do)
        if (item < it.row_tiles * p.Hkv) return;
        item = 0;
        do {
            if (++s >= a.seqs.S) { left = 0; return; }
            it = kv_item<R>(a, s);
        } while (it.rows == 0);
    };
    if (warp == 4) {
        // ---- copies ----
        const int box = min(p.T, kKvTile), nb = kKvTile / box;   // tokens of a copy, copies of a unit
        long long issued = 0;
        while (left > 0 && ok) {
            const int share = (int)min((long long)(it.cost() - at_unit), left);
            const int tile = max(0, at_unit - kKvStart), n = max(0, at_unit + share - kKvStart) - tile;   // tokens' units
            const int h = item % p.Hkv;
            const int32_t* row = a.seqs.table + (int64_t)s * a.seqs.table_stride;
            // 32 copies' block numbers and steps at a time, a lane each
            for (int i0 = 0; i0 < n && ok; i0 += 32 / nb) {
                const int t = (it.t_lo + tile + i0) * kKvTile + lane * box;   // the lane's first token
                int32_t blk = -1;
                float sk = -1.f, sv = 0.f;
                if (lane < nb * (n - i0) && t < it.seq.len && t + box > it.lo) {   // (blocks in front of every window may be gone)
                    blk = __ldcg(row + (t >> a.log2_T));
                    if (blk < 0 || blk >= p.blocks) {
                        atomicExch(p.err, kErrIndex);
                        blk = -1;
                    } else {
                        sk = __ldcg(p.k_step + (int64_t)blk * p.Hkv + h);
                        sv = __ldcg(p.v_step + (int64_t)blk * p.Hkv + h);
                    }
                }
                const int m = min(32 / nb, n - i0);
                for (int i = 0; i < m; ++i) {
                    ok = ops_wait_warp(b_empty + 8u * stage, par ^ 1u, kMxWait, dead);
                    if (!ok) break;
                    const bool mine = blk >= 0 && lane / nb == i;
                    const uint32_t valid = __popc(__ballot_sync(0xffffffffu, mine));
                    const uint32_t bar = b_full + 8u * stage;
                    if (lane == 0) mbar_expect_tx_only(bar, valid * 2u * (uint32_t)(box * D));
                    __syncwarp();
                    if (mine) {
                        const int32_t y = (blk * p.Hkv + h) * p.T + (t & (p.T - 1));
                        const uint32_t dst = smem_u32(ring + (size_t)stage * S::kStage) + (uint32_t)((lane - i * nb) * box * D);
                        tma_rows(dst, &a.k_map, y, bar);
                        tma_rows(dst + S::kHalf, &a.v_map, y, bar);
                    }
                    // the steps of the unit's eight 16-token groups (their loads take as long as the copies do: not waited for before them)
                    const int from = i * nb + (lane & 7) * 16 / box;
                    const float gk = __shfl_sync(0xffffffffu, sk, from), gv = __shfl_sync(0xffffffffu, sv, from);
                    if (lane < 8) steps[stage][lane] = make_float2(gk, gv);
                    __syncwarp();
                    if (lane == 0) mbar_arrive(bar);
                    ++issued;
                    if (++stage == a.stages) { stage = 0; par ^= 1u; }
                }
            }
            left -= share;
            at_unit = 0;
            ++item;
            if (left > 0) next_seq();
        }
        // (nothing may be in flight when the CTA ends)
        if (!ok)
            for (long long i = max(0ll, issued - a.stages); i < issued; ++i) ops_wait(b_full + 8u * (uint32_t)(i % a.stages), (uint32_t)(i / a.stages) & 1u, kMxWait);
        __syncwarp();
    } else {
        const int g = lane >> 2, t = lane & 3;
        while (left > 0 && ok) {
            const int share = (int)min((long long)(it.cost() - at_unit), left);
            const int tile = max(0, at_unit - kKvStart), n = max(0, at_unit + share - kKvStart) - tile;   // tokens' units
            if (n == 0) break;   // (the share ends with an item that the next CTA begins)
            const int h = item % p.Hkv, row0 = item / p.Hkv * R;
            // Q fragments: rows g of every 8, the lane's D/4 columns; fp16 times a power of two that brings bf16 into range
            uint32_t qf[NT][KS][2];
            float f[NT][2];
            int lo[NT][2], hi[NT][2];
            const int pos0 = it.seq.len - it.seq.n;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                const int r = row0 + 8 * nt + g;
                float v[D / 4];
                const bool in = r < it.rows;
                const int tok = in ? r / a.G : 0, qh = h * a.G + (in ? r - tok * a.G : 0);
                const int64_t at = (it.seq.first + tok) * a.q_token + (int64_t)qh * a.q_head + t * (D / 4);
                if (in && a.q_vec) {
                    const uint4* src = reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(a.q) + at);
#pragma unroll
                    for (int i = 0; i < D / 32; ++i) {
                        const uint4 w = __ldcg(src + i);
                        const uint32_t ww[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            if (BF16) {
                                v[8 * i + 2 * j] = __uint_as_float(ww[j] << 16);
                                v[8 * i + 2 * j + 1] = __uint_as_float(ww[j] & 0xFFFF0000u);
                            } else {
                                const float2 u = __half22float2(*reinterpret_cast<const __half2*>(&ww[j]));
                                v[8 * i + 2 * j] = u.x;
                                v[8 * i + 2 * j + 1] = u.y;
                            }
                        }
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < D / 4; ++i) v[i] = in ? q_at<BF16>(a.q, at + i) : 0.f;
                }
                float mul = 1.f, back = 1.f;
                if (BF16) {
                    uint32_t big = 0;
#pragma unroll
                    for (int i = 0; i < D / 4; ++i) big = max(big, __float_as_uint(v[i]) & 0x7FFFFFFFu);
                    big = max(big, __shfl_xor_sync(0xffffffffu, big, 1));
                    big = max(big, __shfl_xor_sync(0xffffffffu, big, 2));
                    // largest magnitude in [2^14, 2^15); exponents so that both factors are normal numbers
                    const int e = max(-112, min(114, (int)(big >> 23) - 127 - 14));
                    mul = __uint_as_float((uint32_t)(127 - e) << 23);
                    back = __uint_as_float((uint32_t)(127 + e) << 23);
                }
#pragma unroll
                for (int j = 0; j < KS; ++j) {
                    qf[nt][j][0] = half2_bits(v[4 * j] * mul, v[4 * j + 1] * mul);
                    qf[nt][j][1] = half2_bits(v[4 * j + 2] * mul, v[4 * j + 3] * mul);
                }
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    f[nt][c] = __shfl_sync(0xffffffffu, back, 4 * (2 * t + c)) * a.scale2;
                    const int rr = row0 + 8 * nt + 2 * t + c;
                    const int pos = pos0 + rr / a.G;
                    const bool real = rr < it.rows;   // (rows past the last are zero queries that see everything; never stored)
                    hi[nt][c] = real ? (a.causal ? pos + 1 : it.seq.len) : 0x7FFFFFFF;
                    lo[nt][c] = real && a.window > 0 ? pos - a.window + 1 : -0x7FFFFFFF;
                }
            }
            // tokens that no row sees are in front of it.lo or from the last row's bound on; all rows see [all_lo, all_hi)
            int all_lo = -0x7FFFFFFF, all_hi = 0x7FFFFFFF;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int c = 0; c < 2; ++c) { all_lo = max(all_lo, lo[nt][c]); all_hi = min(all_hi, hi[nt][c]); }
            all_lo = __reduce_max_sync(0xffffffffu, all_lo);
            all_hi = __reduce_min_sync(0xffffffffu, all_hi);
            const int last_hi = a.causal ? pos0 + (min(row0 + R, it.rows) - 1) / a.G + 1 : it.seq.len;
            float m[NT][2], r[NT][2], l[NT][2], o[MT][NT][4];   // r: m less the reference of p times V's step
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int c = 0; c < 2; ++c) { m[nt][c] = -INFINITY; r[nt][c] = l[nt][c] = 0.f; }
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int c = 0; c < 4; ++c) o[i][nt][c] = 0.f;
            int tok0 = (it.t_lo + tile) * kKvTile + 32 * warp;
#pragma unroll 1
            for (int i = 0; i < n; ++i, tok0 += kKvTile) {
                ok = ops_wait_warp(b_full + 8u * stage, par, kMxWait, dead);
                if (!ok) break;
                const float2 st0 = steps[stage][2 * warp], st1 = steps[stage][2 * warp + 1];
                const float stk[2] = {st0.x, st1.x}, stv[2] = {st0.y, st1.y};
                if (tok0 + 32 > it.lo && tok0 < last_hi && !(st0.x < 0.f && st1.x < 0.f)) {
                    const bool edge = tok0 < all_lo || tok0 + 32 > all_hi || st0.x < 0.f || st1.x < 0.f;
                    const uint32_t kb = smem_u32(ring + (size_t)stage * S::kStage), vb = kb + S::kHalf;
                    float sc[2][NT][4];
#pragma unroll
                    for (int b = 0; b < 2; ++b)
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                            for (int c = 0; c < 4; ++c) sc[b][nt][c] = 0.f;
                    // scores: two times 16 tokens x 8 NT rows
#pragma unroll
                    for (int c = 0; c < D / 64; ++c) {
                        uint32_t xs[2][4], ys[2][4];
#pragma unroll
                        for (int b = 0; b < 2; ++b) {
                            const int kr = 32 * warp + 16 * b + g, chunk = D == 128 ? ((2 * t + c) ^ (kr & 7)) : (t ^ ((kr >> 1) & 3));
                            const uint4 x = lds128(kb + (uint32_t)(kr * D + 16 * chunk)), y = lds128(kb + (uint32_t)((kr + 8) * D + 16 * chunk));
                            xs[b][0] = x.x; xs[b][1] = x.y; xs[b][2] = x.z; xs[b][3] = x.w;
                            ys[b][0] = y.x; ys[b][1] = y.y; ys[b][2] = y.z; ys[b][3] = y.w;
                        }
#pragma unroll
                        for (int j = 0; j < 4; ++j)
#pragma unroll
                            for (int b = 0; b < 2; ++b) {
                                const uint32_t xw = xs[b][j] ^ 0x80808080u, yw = ys[b][j] ^ 0x80808080u;
                                const uint32_t a0 = f16_low(xw), a1 = f16_low(yw), a2 = f16_high(xw), a3 = f16_high(yw);
#pragma unroll
                                for (int nt = 0; nt < NT; ++nt) mma_f16(sc[b][nt], a0, a1, a2, a3, qf[nt][4 * c + j][0], qf[nt][4 * c + j][1]);
                            }
                    }
                    // e = s - m + 7: more than 15 where m is more than 2^8 behind (or nothing was seen yet), or with V's step and r added
                    const float lv[2] = {kv_log2_above(stv[0]), kv_log2_above(stv[1])};
                    float e[2][NT][4];
                    bool behind = false;
                    auto exponents = [&]() {
#pragma unroll
                        for (int b = 0; b < 2; ++b)
#pragma unroll
                            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                                for (int c = 0; c < 4; ++c) e[b][nt][c] = fmaf(sc[b][nt][c], f[nt][c & 1] * stk[b], 7.f - m[nt][c & 1]);
                        if (edge)
#pragma unroll
                            for (int b = 0; b < 2; ++b)
#pragma unroll
                                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                                    for (int c = 0; c < 4; ++c) {
                                        const int tk = tok0 + 16 * b + g + 8 * (c >> 1);
                                        if (tk < lo[nt][c & 1] || tk >= hi[nt][c & 1] || stk[b] < 0.f) e[b][nt][c] = -INFINITY;
                                    }
                    };
                    exponents();
#pragma unroll
                    for (int b = 0; b < 2; ++b)
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                            for (int c = 0; c < 4; ++c) behind |= e[b][nt][c] > fminf(15.f, 15.f - (lv[b] + r[nt][c & 1]));
                    if (__any_sync(0xffffffffu, behind)) {
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                            for (int c = 0; c < 2; ++c) {
                                float x = -INFINITY, y = -INFINITY;   // largest scores, and with V's steps
#pragma unroll
                                for (int b = 0; b < 2; ++b)
#pragma unroll
                                    for (int q = 0; q < 2; ++q)
                                        if (e[b][nt][c + 2 * q] > -INFINITY) {
                                            const float sco = sc[b][nt][c + 2 * q] * (f[nt][c] * stk[b]);
                                            x = fmaxf(x, sco);
                                            y = fmaxf(y, sco + lv[b]);
                                        }
#pragma unroll
                                for (int i = 4; i <= 16; i *= 2) {
                                    x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, i));
                                    y = fmaxf(y, __shfl_xor_sync(0xffffffffu, y, i));
                                }
                                x = fmaxf(x, m[nt][c]);
                                y = fmaxf(y, m[nt][c] - r[nt][c]);
                                const float rn = x == -INFINITY ? 0.f : fmaxf(x - y, -126.f);   // (at most 126: kv_log2_above)
                                const float by = x == -INFINITY ? 0.f : m[nt][c] - x, alpha = exp2_fast(by + (rn - r[nt][c]));
                                l[nt][c] *= exp2_fast(by);
                                m[nt][c] = x;
                                r[nt][c] = rn;
#pragma unroll
                                for (int k = 0; k < MT; ++k) { o[k][nt][c] *= alpha; o[k][nt][c + 2] *= alpha; }
                            }
                        exponents();
                    }
                    // (fp16 output: what the rounding of p leaves is multiplied, too; else its 2^-12 would be as much as the output's own: an error
                    // of 2.9e-4 against 64 bits, 2.1e-4 with it. 64 sequences of up to 8192 tokens, 16 rows a cache head: 171 us without, 182 with.
                    // bf16's own rounding is eight times as large: 1.7e-3 either way)
                    constexpr bool REST = !BF16;
                    uint32_t pf[2][NT][2], pr[2][NT][2];
#pragma unroll
                    for (int b = 0; b < 2; ++b) {
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) {
                            float rel[2];   // V's step for each row; where a row sees none of the group 0, whatever the step is
#pragma unroll
                            for (int c = 0; c < 2; ++c) {
                                rel[c] = stv[b] * exp2_fast(r[nt][c]);
                                if (edge && (tok0 + 16 * b >= hi[nt][c] || tok0 + 16 * b + 16 <= lo[nt][c] || stk[b] < 0.f)) rel[c] = 0.f;
                            }
#pragma unroll
                            for (int c = 0; c < 4; ++c) {
                                e[b][nt][c] = exp2_fast(e[b][nt][c]);
                                l[nt][c & 1] += e[b][nt][c];
                            }
#pragma unroll
                            for (int c = 0; c < 2; ++c) {
                                const float p0 = e[b][nt][2 * c] * rel[0], p1 = e[b][nt][2 * c + 1] * rel[1];
                                const uint32_t h = half2_bits(p0, p1);
                                pf[b][nt][c] = transpose8(h);
                                if (REST) {
                                    const float2 r = __half22float2(*reinterpret_cast<const __half2*>(&h));
                                    pr[b][nt][c] = transpose8(half2_bits(p0 - r.x, p1 - r.y));
                                }
                            }
                        }
                    }
                    // sums: 16 of D x 8 NT rows at a time; a lane holds the same D columns of its four tokens
#pragma unroll
                    for (int b = 0; b < 2; ++b) {
                        const int v0 = 32 * warp + 16 * b + 2 * t;
                        uint32_t w[4][D / 32];
#pragma unroll
                        for (int q = 0; q < 4; ++q) {
                            const int r = v0 + (q & 1) + 8 * (q >> 1);
                            if (D == 128) {
                                const uint4 x = lds128(vb + (uint32_t)(r * D + 16 * (g ^ (r & 7))));
                                w[q][0] = x.x; w[q][1] = x.y; w[q][D / 32 - 2] = x.z; w[q][D / 32 - 1] = x.w;
                            } else {
                                const uint2 x = lds64(vb + (uint32_t)(r * D + 16 * ((g >> 1) ^ ((r >> 1) & 3)) + 8 * (g & 1)));
                                w[q][0] = x.x; w[q][1] = x.y;
                            }
                        }
#pragma unroll
                        for (int k = 0; k < D / 32; ++k) {
                            const uint32_t x0 = prmt(w[0][k], w[1][k], 0x5140u) ^ 0x80808080u, x1 = prmt(w[0][k], w[1][k], 0x7362u) ^ 0x80808080u;
                            const uint32_t y0 = prmt(w[2][k], w[3][k], 0x5140u) ^ 0x80808080u, y1 = prmt(w[2][k], w[3][k], 0x7362u) ^ 0x80808080u;
                            const uint32_t a0 = f16_low(x0), a1 = f16_high(x0), a2 = f16_low(y0), a3 = f16_high(y0);
                            const uint32_t b0 = f16_low(x1), b1 = f16_high(x1), b2 = f16_low(y1), b3 = f16_high(y1);
#pragma unroll
                            for (int nt = 0; nt < NT; ++nt) {
                                mma_f16(o[2 * k][nt], a0, a1, a2, a3, pf[b][nt][0], pf[b][nt][1]);
                                mma_f16(o[2 * k + 1][nt], b0, b1, b2, b3, pf[b][nt][0], pf[b][nt][1]);
                                if (REST) {
                                    mma_f16(o[2 * k][nt], a0, a1, a2, a3, pr[b][nt][0], pr[b][nt][1]);
                                    mma_f16(o[2 * k + 1][nt], b0, b1, b2, b3, pr[b][nt][0], pr[b][nt][1]);
                                }
                            }
                        }
                    }
                }
                __syncwarp();
                if (lane == 0) mbar_arrive(b_empty + 8u * stage);
                if (++stage == a.stages) { stage = 0; par ^= 1u; }
            }
            // the four warps' sums together
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    float x = l[nt][c];
                    x += __shfl_xor_sync(0xffffffffu, x, 4);
                    x += __shfl_xor_sync(0xffffffffu, x, 8);
                    x += __shfl_xor_sync(0xffffffffu, x, 16);
                    if (g == 0) stats[warp * R + 8 * nt + 2 * t + c] = make_float2(m[nt][c], x);
                }
            if (bar_consumers(!ok)) {   // (a warp gave up: all four do, at the same place)
                ok = false;
                break;
            }
            // each in turn adds what it has, relative to the largest maximum; place (2 j + e) * 8 + g of a row holds
            // d = (D / 8) g + 2 j + e, so that a warp's 32 accesses meet 32 banks
            float w[NT][2];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    const int r = 8 * nt + 2 * t + c;
                    float big = -INFINITY;
#pragma unroll
                    for (int k = 0; k < 4; ++k) big = fmaxf(big, stats[k * R + r].x);
                    const float2 own = stats[warp * R + r];
                    w[nt][c] = kv_weight(own.x, own.y, big == -INFINITY ? 0.f : big);
                }
            if (threadIdx.x < R) {
                float big = -INFINITY, sum = 0.f;
#pragma unroll
                for (int k = 0; k < 4; ++k) big = fmaxf(big, stats[k * R + threadIdx.x].x);
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const float2 x = stats[k * R + threadIdx.x];
                    sum += kv_weight(x.x, x.y, big == -INFINITY ? 0.f : big) * x.y;
                }
                stats[4 * R + threadIdx.x] = make_float2(big, sum);
            }
#pragma unroll 1
            for (int turn = 0; turn < 4; ++turn) {
                if (warp == turn)
#pragma unroll
                    for (int k = 0; k < MT; ++k)
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                            for (int c = 0; c < 4; ++c) {
                                float* at = sums + (8 * nt + 2 * t + (c & 1)) * S::kPitch + (2 * k + (c >> 1)) * 8 + g;
                                const float x = w[nt][c & 1] == 0.f ? 0.f : o[k][nt][c] * exp2_fast(-r[nt][c & 1]) * w[nt][c & 1];
                                *at = turn ? *at + x : x;
                            }
                bar_consumers();
            }
            const bool whole = n == it.tiles;
            float* part = a.part + ((int64_t)blockIdx.x * 2 + (tile == 0 ? 1 : 0)) * S::kPart;   // 1: the item begins here
            const int rows = min(R, it.rows - row0);
            for (int i = threadIdx.x; i < rows * D; i += 128) {
                const int r = i / D, d = i - r * D;
                const float big = stats[4 * R + r].x, sum = stats[4 * R + r].y;
                const float acc = sums[r * S::kPitch + (d % (D / 8)) * 8 + d / (D / 8)];
                if (whole) {
                    const int tok = (row0 + r) / a.G, qh = h * a.G + (row0 + r) - tok * a.G;
                    o_put<BF16>(a.out, (it.seq.first + tok) * a.o_token + (int64_t)qh * a.o_head + d, sum == 0.f ? 0.f : acc / sum);
                    if (a.lse && d == 0) a.lse[(it.seq.first + tok) * a.Hq + qh] = kv_lse(big, sum);
                } else {
                    part[r * D + d] = acc;
                    if (d == 0) {
                        part[R * D + 2 * r] = big;
                        part[R * D + 2 * r + 1] = sum;
                    }
                }
            }
            bar_consumers();
            left -= share;
            at_unit = 0;
            ++item;
            if (left > 0) next_seq();
        }
    }
    if (!ok && lane == 0) {
        *dead = 1;
        atomicExch(p.err, kErrTimeout);
    }
    __syncthreads();
}

// Joins the parts of the items that the kernel before has cut. Which those are depends on the lengths alone: a block finds it out before it
// waits for that kernel, beside its last CTAs (beside two of them, with the 168 registers a thread of D = 128, there is no room). An item of
// up to kJoinFew parts is joined by the block of the CTA that begins it, a warp a row. The rows of one of more parts are shared by the
// blocks of all CTAs that have one, and a row's parts by the warps: one trip to memory for up to eight a warp. (One sequence of 131072
// tokens, 8 cache heads, 37 parts each, inside a graph: 62 us with the first form alone, 53 with the second; 64 of 4096, 2 or 3 parts
// each: 95 and 102.) Parts are added in the same order every time.
// Every block waits for the kernel before, those without a part, too: what follows in the stream waits for this grid alone, so this
// grid may not end before the sums and outputs of the other one are there.
constexpr int kJoinWarps = 4, kJoinFew = 4;
template <int D, int NT, bool BF16>
__global__ void __launch_bounds__(32 * kJoinWarps, 5) us_kv_join_kernel(const __grid_constant__ KvAttend a)
{
    using S = KvShape<D, NT>;
    constexpr int R = S::R, C = D / 32;
    __shared__ float2 stat[kJoinWarps];
    __shared__ float accs[kJoinWarps][D];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, me = blockIdx.x;
    const KvRange range = kv_range<R>(a, me, lane, false);
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    bool waited = false;
    auto wait = [&]() {
        if (!waited) asm volatile("griddepcontrol.wait;" ::: "memory");
        waited = true;
    };
    auto join = [&](const KvItem& it, int item, int c0, int c1) {
        if (c1 - c0 < kJoinFew && me != c0) return;
        wait();
        const int h = item % a.pool.Hkv, row0 = item / a.pool.Hkv * R, rows = min(R, it.rows - row0);
        const int np = c1 - c0 + 1;
        if (np <= kJoinFew) {
#pragma unroll 1
            for (int r0 = warp; r0 < rows; r0 += 2 * kJoinWarps) {   // two rows a warp at a time: all loads first
                float m[2][kJoinFew], l[2][kJoinFew], x[2][kJoinFew][C];
#pragma unroll
                for (int b = 0; b < 2; ++b)
#pragma unroll
                    for (int k = 0; k < kJoinFew; ++k) {
                        const int r = r0 + kJoinWarps * b;
                        m[b][k] = -INFINITY;
                        l[b][k] = 0.f;
                        if (k < np && r < rows) {
                            const float* part = a.part + ((int64_t)(c0 + k) * 2 + (k == 0 ? 1 : 0)) * S::kPart;
                            const float2 u = __ldcg(reinterpret_cast<const float2*>(part + R * D + 2 * r));
                            m[b][k] = u.x;
                            l[b][k] = u.y;
#pragma unroll
                            for (int i = 0; i < C; ++i) x[b][k][i] = __ldcg(part + r * D + lane + 32 * i);
                        }
                    }
#pragma unroll
                for (int b = 0; b < 2; ++b) {
                    const int r = r0 + kJoinWarps * b;
                    if (r >= rows) break;
                    float all = -INFINITY, total = 0.f, y[C];
#pragma unroll
                    for (int i = 0; i < C; ++i) y[i] = 0.f;
#pragma unroll
                    for (int k = 0; k < kJoinFew; ++k) all = fmaxf(all, m[b][k]);
#pragma unroll
                    for (int k = 0; k < kJoinFew; ++k) {
                        const float e = kv_weight(m[b][k], l[b][k], all == -INFINITY ? 0.f : all);
                        total += e * l[b][k];
#pragma unroll
                        for (int i = 0; i < C; ++i) y[i] += e == 0.f ? 0.f : e * x[b][k][i];
                    }
                    const int tok = (row0 + r) / a.G, qh = h * a.G + (row0 + r) - tok * a.G;
                    const float inv = total == 0.f ? 0.f : 1.f / total;
#pragma unroll
                    for (int i = 0; i < C; ++i) o_put<BF16>(a.out, (it.seq.first + tok) * a.o_token + (int64_t)qh * a.o_head + lane + 32 * i, total == 0.f ? 0.f : y[i] * inv);
                    if (a.lse && lane == 0) a.lse[(it.seq.first + tok) * a.Hq + qh] = kv_lse(all, total);
                }
            }
            return;
        }
        const int mine = (rows - (me - c0) + np - 1) / np;   // rows me - c0, me - c0 + np, ...
        const int per = mine >= 3 ? 1 : mine == 2 ? 2 : kJoinWarps, groups = kJoinWarps / per;   // warps a row, rows at a time
        for (int k0 = 0; k0 < mine; k0 += groups) {
            const int k_mine = k0 + warp / per, r = me - c0 + k_mine * np;
            float big = -INFINITY, sum = 0.f, acc[C];
#pragma unroll
            for (int i = 0; i < C; ++i) acc[i] = 0.f;
            for (int cb = k_mine < mine ? c0 + warp % per : c1 + 1; cb <= c1; cb += 8 * per) {
                float m[8], l[8], x[8][C];
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const int c = cb + per * k;
                    m[k] = -INFINITY;
                    l[k] = 0.f;
                    if (c <= c1) {
                        const float* part = a.part + ((int64_t)c * 2 + (c == c0 ? 1 : 0)) * S::kPart;
                        const float2 u = __ldcg(reinterpret_cast<const float2*>(part + R * D + 2 * r));
                        m[k] = u.x;
                        l[k] = u.y;
#pragma unroll
                        for (int i = 0; i < C; ++i) x[k][i] = __ldcg(part + r * D + lane + 32 * i);
                    }
                }
                float top = big;
#pragma unroll
                for (int k = 0; k < 8; ++k) top = fmaxf(top, m[k]);
                const float base = top == -INFINITY ? 0.f : top, keep = kv_weight(big, sum, base);
                sum *= keep;
#pragma unroll
                for (int i = 0; i < C; ++i) acc[i] *= keep;
                big = top;
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const float e = kv_weight(m[k], l[k], base);
                    sum += e * l[k];
#pragma unroll
                    for (int i = 0; i < C; ++i) acc[i] += e == 0.f ? 0.f : e * x[k][i];
                }
            }
            if (lane == 0) stat[warp] = make_float2(big, sum);
#pragma unroll
            for (int i = 0; i < C; ++i) accs[warp][lane + 32 * i] = acc[i];
            __syncthreads();
            for (int i = threadIdx.x; i < groups * D; i += 32 * kJoinWarps) {
                const int gr = i / D, d = i - gr * D, row = me - c0 + (k0 + gr) * np;
                if (k0 + gr >= mine) break;
                float all = -INFINITY, total = 0.f, y = 0.f;
                for (int k = gr * per; k < (gr + 1) * per; ++k) all = fmaxf(all, stat[k].x);
                for (int k = gr * per; k < (gr + 1) * per; ++k) {
                    const float e = kv_weight(stat[k].x, stat[k].y, all == -INFINITY ? 0.f : all);
                    total += e * stat[k].y;
                    y += e == 0.f ? 0.f : e * accs[k][d];
                }
                const int tok = (row0 + row) / a.G, qh = h * a.G + (row0 + row) - tok * a.G;
                o_put<BF16>(a.out, (it.seq.first + tok) * a.o_token + (int64_t)qh * a.o_head + d, total == 0.f ? 0.f : y / total);
                if (a.lse && d == 0) a.lse[(it.seq.first + tok) * a.Hq + qh] = kv_lse(all, total);
            }
            __syncthreads();
        }
    };
    auto walk = [&]() {
        // the item that the CTA's first unit belongs to, if it began in an earlier CTA
        int s = range.s;
        KvItem it = range.item;
        long long start = range.u0 - range.in_seq;   // first unit of the sequence
        {
            const int item = kv_div(range.in_seq, it.cost());
            const long long first = start + (long long)item * it.cost() + kKvStart;
            if (first < range.u0) {
                join(it, item, range.shares.owner(first), range.shares.owner(first + it.tiles - 1));
                if (first + it.tiles >= range.u1) return;
            }
        }
        // the item that its last unit belongs to, if it begins here and ends in a later one
        long long units = (long long)it.row_tiles * a.pool.Hkv * it.cost();
        while (start + units <= range.u1 - 1) {
            start += units;
            if (++s >= a.seqs.S) return;
            it = kv_item<R>(a, s);
            units = (long long)it.row_tiles * a.pool.Hkv * it.cost();
        }
        const int item = kv_div(range.u1 - 1 - start, it.cost());
        const long long first = start + (long long)item * it.cost() + kKvStart, end = first + it.tiles;
        if (first >= range.u0 && first < range.u1 && end > range.u1) join(it, item, me, range.shares.owner(end - 1));
    };
    if (range.u0 < range.u1) walk();
    wait();
}

}  // namespace us
