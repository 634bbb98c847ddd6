// Norms of query and key heads and the rotation of their positions, in one pass: what stands between the Q/K/V projection and the cache.
#include "us_mx4.cuh"
#include "us_ops.h"

namespace us {
namespace {

// A head x of D values: y = x / sqrt(mean x^2 + eps) * w (where there are weights), and of y's first `rotary` values the pairs (i, i + rotary/2), or
// (2i, 2i + 1), turned by position * frequency_i.
//   * Turns are counted in 2^-64: position * turns wraps at a whole turn by itself, so that the angle of a far position has the frequency's own error and no
//     other (53 bits: below 2^-51 of position * frequency; in 32-bit arithmetic 131072 radians are known to 2^-7). What is left after quarter turns goes through two short polynomials.
//   * A lane has eight pairs in registers, as two pieces of eight values: both ends of a pair are its own. 1 to 16 lanes have a head (a power of two, D / 16
//     of them have values), a warp 32 / lanes heads at a time: a round. The sines and cosines of a lane's pairs are found once for all rounds that the warp
//     walks over; the values of the next round are on their way meanwhile. Sines, cosines and weights wait in shared memory.
//   * Pairs behind the rotated ones are values that only the norm touches.
// Bound by memory where there are many tokens (8192 of 64 + 8 heads of 128, bf16: 57 us, 5.3 TB/s), by launch and two trips to memory for a single one (2.6 us inside a
// graph). What is short of the copy rate (46 us) is the beginning of each of the three waves of blocks. Slower: more blocks an SM with the factors read from
// shared memory in every round (69 to 95 us for 5 to 8), three rounds under way (59 to 66), two to four warps a token (62 to 74).
struct Heads {
    const void* x;
    int64_t token, head;       // strides
    void* out;
    int64_t o_token, o_head;
    const void* weight;        // D values, or nullptr: no norm
    int32_t heads, w_type;
};
constexpr int kHeadsThreads = 128;
struct HeadsCall {
    Heads part[2];             // queries, keys
    const uint64_t* turns;     // rotary / 2
    const uint8_t* axis;       // of each pair, or nullptr: all 0
    const int32_t* positions;
    int64_t axis_stride;
    int64_t N;
    int32_t D, rotary, log2_lanes, per_token;   // per_token: warps that share a token's heads
    float eps, one_over_D;
};

__device__ __forceinline__ float weight_at(const void* w, int32_t type, int i)
{
    return type == US_F32 ? static_cast<const float*>(w)[i] : type == US_F16 ? __half2float(static_cast<const __half*>(w)[i]) :
                            __bfloat162float(static_cast<const __nv_bfloat16*>(w)[i]);
}
// cos and sin of `part` / 2^64 turns. With x = the rest of a quarter turn in half turns, |x| <= 1/4: sin(pi x) = x S(x^2), cos(pi x) = C(x^2). S and C: of the polynomials of degree 3 and 4
// in u = x^2 those whose largest distance from sin(pi x) / x and cos(pi x) over u = 0 .. 1/16 is least (Remez's exchange), coefficients rounded to fp32. In fp32 arithmetic sine and
// cosine are off by 1.7 2^-24 and 1.25 2^-24 at most (32 million arguments against 64 bits).
__device__ __forceinline__ void turn(uint64_t part, float& c, float& s)
{
    const uint64_t r = part + (1ull << 61);                                    // quarters: the nearest one, and -1/8 .. 1/8 turn from it
    const int32_t rest = (int32_t)(uint32_t)((r << 2) >> 32) ^ (int32_t)0x80000000;   // (2 bits of quarter gone; 2^-34 turns each)
    const float x = (float)rest * 0x1p-33f, u = x * x;
    float a = fmaf(-0.589078656f, u, 2.5497673f), b = fmaf(0.231329752f, u, -1.33504457f);
    a = fmaf(a, u, -5.16770783f);
    b = fmaf(b, u, 4.05870726f);
    a = fmaf(a, u, 3.14159264f) * x;
    b = fmaf(b, u, -4.93480216f);
    b = fmaf(b, u, 1.f);
    const uint32_t q = (uint32_t)(r >> 62);
    const float cc = q & 1 ? a : b, ss = q & 1 ? b : a;
    c = q == 1 || q == 2 ? -cc : cc;
    s = q >= 2 ? -ss : ss;
}
// V values in one access of V sizeof(T) bytes (two of 16 where that is 32)
template <class T, int V>
__device__ __forceinline__ void get(const T* p, T* v)
{
    constexpr int B = V * (int)sizeof(T);
    if constexpr (B >= 16)
#pragma unroll
        for (int i = 0; i < B / 16; ++i) reinterpret_cast<uint4*>(v)[i] = __ldcg(reinterpret_cast<const uint4*>(p) + i);
    else if constexpr (B == 8) *reinterpret_cast<uint2*>(v) = __ldcg(reinterpret_cast<const uint2*>(p));
    else if constexpr (B == 4) *reinterpret_cast<uint32_t*>(v) = __ldcg(reinterpret_cast<const uint32_t*>(p));
    else *reinterpret_cast<uint16_t*>(v) = __ldcg(reinterpret_cast<const uint16_t*>(p));
}
template <class T, int V>
__device__ __forceinline__ void put(T* p, const T* v)
{
    constexpr int B = V * (int)sizeof(T);
    if constexpr (B >= 16)
#pragma unroll
        for (int i = 0; i < B / 16; ++i) reinterpret_cast<uint4*>(p)[i] = reinterpret_cast<const uint4*>(v)[i];
    else if constexpr (B == 8) *reinterpret_cast<uint2*>(p) = *reinterpret_cast<const uint2*>(v);
    else if constexpr (B == 4) *reinterpret_cast<uint32_t*>(p) = *reinterpret_cast<const uint32_t*>(v);
    else *reinterpret_cast<uint16_t*>(p) = *reinterpret_cast<const uint16_t*>(v);
}

// two fp32 in one instruction
__device__ __forceinline__ uint64_t two(float a, float b)
{
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ void split(uint64_t v, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c)
{
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b)
{
    uint64_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
template <class T>
__device__ __forceinline__ uint64_t widen(const T* v) { return two(to_f32(v[0]), to_f32(v[1])); }
template <>
__device__ __forceinline__ uint64_t widen<__nv_bfloat16>(const __nv_bfloat16* v)
{
    const uint32_t w = *reinterpret_cast<const uint32_t*>(v);
    return two(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u));
}
template <class T>
__device__ __forceinline__ void narrow(uint64_t x, T* v)
{
    float a, b;
    split(x, a, b);
    v[0] = from_f32<T>(a);
    v[1] = from_f32<T>(b);
}
template <>
__device__ __forceinline__ void narrow<__nv_bfloat16>(uint64_t x, __nv_bfloat16* v)
{
    float a, b;
    split(x, a, b);
    *reinterpret_cast<__nv_bfloat162*>(v) = __floats2bfloat162_rn(a, b);
}
template <>
__device__ __forceinline__ void narrow<__half>(uint64_t x, __half* v)
{
    float a, b;
    split(x, a, b);
    *reinterpret_cast<__half2*>(v) = __floats2half2_rn(a, b);
}

// V: pairs that lie side by side in memory (8, 4 or 1), which divide rotary / 2 and D / 2. A lane's values: v[0 .. 7] the first ends of its pairs, v[8 .. 15] the
// others; interleaved, V of the 2 V values of a group each. Weight, sine and cosine are one factor each: with own = w cos and cross = +- (the other end's w) sin
// y = x own + (the other end's x) cross, two values an instruction.
// LOG: of the lanes a head has, where that is known (0: it is not).
template <class T, int V, bool INTERLEAVED, int LOG>
__global__ void __launch_bounds__(kHeadsThreads, sizeof(T) == 2 && V == 8 ? 5 : 4) us_heads_kernel(const __grid_constant__ HeadsCall a)
{
    constexpr int G = 8 / V, DEEP = 2;   // rounds under way
    __shared__ float weights[2][256];   // of lane l: its 16 at l + 16 i
    __shared__ __align__(16) float2 turned[kHeadsThreads / 32][128];   // of a warp's token: cosine and sine of each pair (1, 0 behind the turned ones)
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int lane = threadIdx.x & 31, log2_lanes = LOG ? LOG : a.log2_lanes, lanes = 1 << log2_lanes, slot = lane >> log2_lanes, slots = 32 >> log2_lanes;
    const int l = lane & (lanes - 1), p0 = 8 * l, half = a.rotary / 2;   // the lane's first pair
    const uint32_t warp = blockIdx.x * (kHeadsThreads / 32) + (threadIdx.x >> 5);   // (fewer than 2^31: more than one a token only where there are few)
    const uint32_t n = warp / (uint32_t)a.per_token;
    const int share = (int)(warp - n * a.per_token);
    const bool real = n < a.N;
    // places of the first values of pair group g, and of their other ends
    int at[G], other[G];
    bool in[G], turns[G];
#pragma unroll
    for (int g = 0; g < G; ++g) {
        const int p = p0 + V * g;
        in[g] = real && p < a.D / 2;
        turns[g] = p < half;
        at[g] = INTERLEAVED || !turns[g] ? 2 * p : p;
        other[g] = INTERLEAVED || !turns[g] ? 2 * p + V : p + half;
    }
    uint64_t step[4];   // of pairs lane, lane + 32, ...
    uint32_t axis[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int p = lane + 32 * i;
        step[i] = p < half ? __ldg(a.turns + p) : 0;   // (constant since the handle was made)
        axis[i] = p < half && a.axis ? __ldg(a.axis + p) : 0;
    }
    asm volatile("griddepcontrol.wait;" ::: "memory");
    struct Values { __align__(16) T v[16]; };
    auto fetch = [&](const T* src, bool there, Values& x) {   // (values that are not there stay 0; a head that is not there is not stored)
        if (!there) return;
#pragma unroll
        for (int g = 0; g < G; ++g)
            if (in[g]) {
                get<T, V>(src + at[g], x.v + V * g);
                get<T, V>(src + other[g], x.v + 8 + V * g);
            }
    };
    // rounds: queries' first, then keys'
    const int first = (a.part[0].heads + slots - 1) >> (5 - log2_lanes), rounds = first + ((a.part[1].heads + slots - 1) >> (5 - log2_lanes));
    Values x[DEEP];   // of the round that is next, and of those behind
#pragma unroll
    for (int k = 0; k < DEEP; ++k)
#pragma unroll
        for (int i = 0; i < 16; ++i) x[k].v[i] = from_f32<T>(0.f);
    auto begin = [&](int round) {   // the first rounds of a part
        const bool keys = round >= first;
        const Heads& p = keys ? a.part[1] : a.part[0];
        int h = (round - (keys ? first : 0)) * slots + slot;
        const T* src = static_cast<const T*>(p.x) + n * p.token + h * p.head;
#pragma unroll
        for (int k = 0; k < DEEP; ++k) {
            fetch(src, h < p.heads, x[k]);
            h += a.per_token * slots;
            src += (int64_t)a.per_token * slots * p.head;
        }
    };
    begin(share);
    // weights: place i of lane l is value at(i / V) + i % V, place 8 + i its pair's other end
    for (int i = threadIdx.x; i < 2 * 8 * lanes; i += kHeadsThreads) {
        const int which = i >= 8 * lanes, q = i - (which ? 8 * lanes : 0), g = q / V * V;
        const Heads& p = which ? a.part[1] : a.part[0];
        const bool apart = INTERLEAVED || g >= half;
        const bool has = p.weight && q < a.D / 2;
        weights[which][(q >> 3) + 16 * (q & 7)] = has ? weight_at(p.weight, p.w_type, (apart ? 2 * g : g) + q % V) : 1.f;
        weights[which][(q >> 3) + 16 * (8 + (q & 7))] = has ? weight_at(p.weight, p.w_type, (apart ? 2 * g + V : g + half) + q % V) : 1.f;
    }
    if (real) {
        int32_t pos[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) pos[i] = lane + 32 * i < half ? __ldcg(a.positions + (int64_t)axis[i] * a.axis_stride + n) : 0;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (lane + 32 * i < 8 * lanes) {
                float2 x = make_float2(1.f, 0.f);
                if (lane + 32 * i < half) turn((uint64_t)(int64_t)pos[i] * step[i], x.x, x.y);
                turned[threadIdx.x >> 5][lane + 32 * i] = x;
            }
    }
    __syncthreads();
    if (!real) return;
    int round = share;
#pragma unroll 1
    for (int which = 0; which < 2; ++which) {
        const int base = which ? first : 0, end = which ? rounds : first;
        if (round >= end) continue;
        const Heads& p = which ? a.part[1] : a.part[0];
        // factors of values 2 j and 2 j + 1 of the lane's 16 (V = 1: of each apart)
        uint64_t own[8], cross[8];
        {
            float o[16], r[16];
#pragma unroll
            for (int g = 0; g < G; ++g)
#pragma unroll
                for (int i = 0; i < V; ++i) {   // pair V g + i: its two values
                    const int u = INTERLEAVED && V > 1 ? (2 * i < V ? V * g + 2 * i : 8 + V * g + 2 * i - V) : V * g + i, v = INTERLEAVED && V > 1 ? u + 1 : u + 8;
                    const float2 cs = turned[threadIdx.x >> 5][p0 + V * g + i];
                    const float c = cs.x, sn = cs.y, wu = weights[which][l + 16 * u], wv = weights[which][l + 16 * v];
                    o[u] = wu * c;
                    r[u] = -wv * sn;
                    o[v] = wv * c;
                    r[v] = wu * sn;
                }
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                own[j] = two(o[2 * j], o[2 * j + 1]);
                cross[j] = two(r[2 * j], r[2 * j + 1]);
            }
        }
        const bool norm = p.weight != nullptr;
        const int64_t step_x = (int64_t)a.per_token * slots * p.head, step_o = (int64_t)a.per_token * slots * p.o_head;
        int h = (round - base) * slots + slot;
        const int more = a.per_token * slots;
        const T* src = static_cast<const T*>(p.x) + n * p.token + (h + (DEEP - 1) * more) * p.head;
        T* dst = static_cast<T*>(p.out) + n * p.o_token + h * p.o_head;
        if (round != share) begin(round);
        auto finish = [&](const Values& x) {
            uint64_t f[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) f[j] = widen<T>(x.v + 2 * j);
            if (norm) {
                uint64_t sum2 = mul2(f[0], f[0]);
#pragma unroll
                for (int j = 1; j < 8; ++j) sum2 = fma2(f[j], f[j], sum2);
                float sum, rest;
                split(sum2, sum, rest);
                sum += rest;
                if (LOG) {
#pragma unroll
                    for (int o = 1; o < 1 << LOG; o <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
                } else {
                    for (int o = 1; o < lanes; o <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
                }
                const float inv = rsqrtf(fmaf(sum, a.one_over_D, a.eps));
                const uint64_t inv2 = two(inv, inv);
#pragma unroll
                for (int j = 0; j < 8; ++j) f[j] = mul2(f[j], inv2);
            }
            Values y;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                uint64_t r = mul2(f[j], own[j]);
                if (V == 1) {   // (pairs of one instruction may differ in whether they are turned)
                    const uint64_t with = fma2(f[j ^ 4], cross[j], r);
                    float r0, r1, w0, w1;
                    split(r, r0, r1);
                    split(with, w0, w1);
                    r = two(turns[(2 * j) & (G - 1)] ? w0 : r0, turns[(2 * j + 1) & (G - 1)] ? w1 : r1);
                } else if (turns[2 * j % 8 / V]) {   // (else nothing of the other end counts, not even a NaN)
                    if (INTERLEAVED) {
                        float u, v;
                        split(f[j], u, v);
                        r = fma2(two(v, u), cross[j], r);
                    } else {
                        r = fma2(f[j ^ 4], cross[j], r);
                    }
                }
                narrow<T>(r, y.v + 2 * j);
            }
            if (h < p.heads)
#pragma unroll
                for (int g = 0; g < G; ++g)
                    if (in[g]) {
                        put<T, V>(dst + at[g], y.v + V * g);
                        put<T, V>(dst + other[g], y.v + 8 + V * g);
                    }
            h += more;
            dst += step_o;
            round += a.per_token;
        };
#pragma unroll 1
        while (round < end) {
#pragma unroll
            for (int k = 0; k < DEEP; ++k) {
                if (k && round >= end) break;
                finish(x[k]);
                src += step_x;
                fetch(src, h + (DEEP - 1) * more < p.heads, x[k]);
            }
        }
    }
}

template <class T, bool INTERLEAVED>
const void* heads_kernel(int v, int log2_lanes)
{
    if (v == 8)
        return log2_lanes == 3 ? (const void*)us_heads_kernel<T, 8, INTERLEAVED, 3> : log2_lanes == 2 ? (const void*)us_heads_kernel<T, 8, INTERLEAVED, 2> :
               (const void*)us_heads_kernel<T, 8, INTERLEAVED, 0>;
    return v == 4 ? (const void*)us_heads_kernel<T, 4, INTERLEAVED, 0> : (const void*)us_heads_kernel<T, 1, INTERLEAVED, 0>;
}
template <class T>
const void* heads_kernel(int v, int log2_lanes, bool interleaved) { return interleaved ? heads_kernel<T, true>(v, log2_lanes) : heads_kernel<T, false>(v, log2_lanes); }

bool aligned(const void* p, int64_t b) { return reinterpret_cast<uintptr_t>(p) % (uintptr_t)b == 0; }

}  // namespace
}  // namespace us

using namespace us;

us_status us_qk_norm_rope(const us_rotary* r, const int32_t* positions, int64_t axis_stride, int64_t N, int32_t D, int32_t type, const us_heads* q,
                          const us_heads* k, float eps, void* stream)
{
    if (!r || !r->turns || !aligned(r->turns, 8) || r->rotary_dim < 2 || r->rotary_dim % 2 || r->rotary_dim > D || r->axes < 1 || r->axes > 255 || (r->axes > 1 && !r->axis) ||
        D < 2 || D % 2 || D > 256 || type < 0 || type > 2 || !q || N < 0 || N >= (1ll << 31) || !(eps >= 0.f)) return US_ERR_INVALID_ARG;
    const int64_t size = type == US_F32 ? 4 : 2;
    HeadsCall a = {};
    int vec = 8;
    auto fits = [&](int v, const void* p, int64_t token, int64_t head) {   // accesses of v values
        const int64_t b = std::min<int64_t>(16, v * size);
        return aligned(p, b) && token * size % b == 0 && head * size % b == 0;
    };
    for (int v : {8, 4, 1}) {
        vec = v;
        if (r->rotary_dim / 2 % v == 0 && D / 2 % v == 0) break;
    }
    for (int i = 0; i < 2; ++i) {
        const us_heads* h = i ? k : q;
        if (!h || h->heads == 0) continue;
        if (h->heads < 0 || h->heads > 65535) return US_ERR_INVALID_ARG;
        if (N == 0) continue;
        if (!h->x || !h->out || !aligned(h->x, size) || !aligned(h->out, size) || (h->weight && (h->weight_type < 0 || h->weight_type > 2 ||
            !aligned(h->weight, h->weight_type == US_F32 ? 4 : 2)))) return US_ERR_INVALID_ARG;
        if ((N > 1 && (h->token_stride < D || h->out_token_stride < D)) || (h->heads > 1 && (h->head_stride < D || h->out_head_stride < D)) || h->token_stride < 0 ||
            h->head_stride < 0 || h->out_token_stride < 0 || h->out_head_stride < 0) return US_ERR_INVALID_ARG;
        Heads& p = a.part[i];
        p.x = h->x; p.token = N > 1 ? h->token_stride : 0; p.head = h->heads > 1 ? h->head_stride : 0;
        p.out = h->out; p.o_token = N > 1 ? h->out_token_stride : 0; p.o_head = h->heads > 1 ? h->out_head_stride : 0;
        p.weight = h->weight; p.w_type = h->weight_type; p.heads = h->heads;
        while (vec > 1 && !(fits(vec, p.x, p.token, p.head) && fits(vec, p.out, p.o_token, p.o_head))) vec = vec == 8 ? 4 : 1;
    }
    const int64_t heads = (int64_t)a.part[0].heads + a.part[1].heads;
    if (N == 0 || heads == 0) return US_OK;
    if (!positions || !aligned(positions, 4) || (r->axes > 1 && axis_stride < 0)) return US_ERR_INVALID_ARG;
    a.turns = r->turns;
    a.axis = r->axes > 1 ? r->axis : nullptr;
    a.positions = positions;
    a.axis_stride = axis_stride;
    a.N = N;
    a.D = D; a.rotary = r->rotary_dim;
    a.eps = eps;
    a.one_over_D = 1.f / (float)D;
    while ((16 << a.log2_lanes) < D) ++a.log2_lanes;
    // A token's rounds go to as many warps as the GPU holds at once; each finds the factors anew. (1001 tokens of 32 + 32 heads, 16 rounds each, in fp32: 20.9 us with one
    // warp a token, 12.9 with two, 14.6 with three, 15.4 with six.)
    const int64_t slots = 32 >> a.log2_lanes, rounds = (a.part[0].heads + slots - 1) / slots + (a.part[1].heads + slots - 1) / slots;
    a.per_token = (int32_t)std::max<int64_t>(1, std::min<int64_t>(rounds, 16 * ops_sms() / N));
    const int64_t blocks = (N * a.per_token + kHeadsThreads / 32 - 1) / (kHeadsThreads / 32);
    const bool inter = r->interleaved != 0;
    const void* kernel = type == US_F16 ? heads_kernel<__half>(vec, a.log2_lanes, inter) : type == US_BF16 ? heads_kernel<__nv_bfloat16>(vec, a.log2_lanes, inter) :
                                          heads_kernel<float>(vec, a.log2_lanes, inter);
    void* args[] = {&a};
    const cudaError_t e = ops_launch(kernel, dim3((unsigned)blocks), kHeadsThreads, 0, static_cast<cudaStream_t>(stream), args);
    if (e == cudaSuccess) return US_OK;
    cudaGetLastError();
    return US_ERR_CUDA;
}
