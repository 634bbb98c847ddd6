// Norms of query and key heads and the rotation of their positions, in one pass: what stands between the Q/K/V projection and the cache.
#include "us_mx4.cuh"
#include "us_ops.h"

namespace us {
namespace {

// A head x of D values: y = x / sqrt(mean x^2 + eps) * w (where there are weights), and of y's first `rotary` values the pairs (i, i + rotary/2), or
// (2i, 2i + 1), turned by position * frequency_i.
//   * Turns are counted in 2^-64: position * turns wraps at a whole turn by itself, so that the angle of a far position is as good as a near
//     one's (in 32-bit arithmetic 131072 radians are known to 2^-7). What is left after quarter turns goes through two short polynomials.
//   * A lane has eight pairs in registers, as two pieces of eight values: both ends of a pair are its own. 1 to 16 lanes have a head (a power of two, D / 16
//     of them have values), a warp 32 / lanes heads at a time: a round. The sines and cosines of a lane's pairs are found once for all rounds that the warp
//     walks over; the values of the next round are on their way meanwhile. Weights wait in shared memory.
//   * Pairs behind the rotated ones are values that only the norm touches.
// Bound by memory where there are many tokens, by launch and two trips to memory for a single one (MEASURED).
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
    float eps;
};

__device__ __forceinline__ float weight_at(const void* w, int32_t type, int i)
{
    return type == US_F32 ? static_cast<const float*>(w)[i] : type == US_F16 ? __half2float(static_cast<const __half*>(w)[i]) :
                            __bfloat162float(static_cast<const __nv_bfloat16*>(w)[i]);
}
// cos and sin of `part` / 2^64 turns. With x = the rest of a quarter turn in half turns, |x| <= 1/4: sin(pi x) = x S(x^2), cos(pi x) = C(x^2), polynomials fitted here;
// off by 1.5 2^-24 and 2^-24 at most, in fp32 arithmetic.
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

// V: pairs that lie side by side in memory (8, 4 or 1), which divide rotary / 2 and D / 2.
template <class T, int V, bool INTERLEAVED>
__global__ void __launch_bounds__(kHeadsThreads) us_heads_kernel(const __grid_constant__ HeadsCall a)
{
    __shared__ __align__(16) float weights[2][256];   // of lane l: its 16 at 16 l
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int lane = threadIdx.x & 31, lanes = 1 << a.log2_lanes, slot = lane >> a.log2_lanes, slots = 32 >> a.log2_lanes;
    const int l = lane & (lanes - 1), p0 = 8 * l, half = a.rotary / 2;   // the lane's first pair
    const int64_t warp = ((int64_t)blockIdx.x * blockDim.x + threadIdx.x) >> 5;
    const int64_t n = warp / a.per_token;
    const int share = (int)(warp - n * a.per_token);
    // places of the first values of pair group g of V pairs, and of their other ends
    auto in = [&](int g) { return p0 + V * g < a.D / 2; };
    auto turns = [&](int g) { return p0 + V * g < half; };
    auto at = [&](int g) { return INTERLEAVED || !turns(g) ? 2 * (p0 + V * g) : p0 + V * g; };
    auto other = [&](int g) { return INTERLEAVED || !turns(g) ? 2 * (p0 + V * g) + V : p0 + V * g + half; };
    uint64_t step[8];
    uint32_t axis[2] = {0, 0};   // of the pairs, a byte each
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        step[i] = p0 + i < half ? __ldg(a.turns + p0 + i) : 0;   // (constant since the handle was made)
        if (a.axis && p0 + i < half) axis[i >> 2] |= (uint32_t)__ldg(a.axis + p0 + i) << (8 * (i & 3));
    }
    asm volatile("griddepcontrol.wait;" ::: "memory");
    // rounds: queries' first, then keys'
    const int first = (a.part[0].heads + slots - 1) >> (5 - a.log2_lanes), rounds = first + ((a.part[1].heads + slots - 1) >> (5 - a.log2_lanes));
    struct Values { __align__(16) T v[16]; };
    auto fetch = [&](int round, Values& x) {
        const int which = round >= first, h = (round - (which ? first : 0)) * slots + slot;
        const Heads& p = a.part[which];
#pragma unroll
        for (int i = 0; i < 16; ++i) x.v[i] = from_f32<T>(0.f);
        if (n >= a.N || round >= rounds || h >= p.heads) return;
        const T* src = static_cast<const T*>(p.x) + n * p.token + h * p.head;
#pragma unroll
        for (int g = 0; g < 8 / V; ++g)
            if (in(g)) {
                get<T, V>(src + at(g), x.v + V * g);
                get<T, V>(src + other(g), x.v + 8 + V * g);
            }
    };
    Values x, ahead;
    fetch(share, x);
    // weights: place 16 l + i is value at(i / V) + i % V, 16 l + 8 + i its pair's other end
    for (int i = threadIdx.x; i < 2 * 8 * lanes; i += blockDim.x) {
        const int which = i >= 8 * lanes, q = i - (which ? 8 * lanes : 0), g = q / V * V;
        const Heads& p = a.part[which];
        if (!p.weight || q >= a.D / 2) continue;
        const bool turned = g < half;
        const int from = (INTERLEAVED || !turned ? 2 * g : g) + q % V, to = INTERLEAVED || !turned ? 2 * g + V + q % V : g + half + q % V;
        weights[which][(q >> 3) * 16 + (q & 7)] = weight_at(p.weight, p.w_type, from);
        weights[which][(q >> 3) * 16 + 8 + (q & 7)] = weight_at(p.weight, p.w_type, to);
    }
    float c[8], s[8];
    if (n < a.N) {
        int64_t pos[8];
        if (a.axis) {
#pragma unroll
            for (int i = 0; i < 8; ++i) pos[i] = __ldcg(a.positions + (int64_t)((axis[i >> 2] >> (8 * (i & 3))) & 0xFFu) * a.axis_stride + n);
        } else {
            pos[0] = __ldcg(a.positions + n);
#pragma unroll
            for (int i = 1; i < 8; ++i) pos[i] = pos[0];
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) turn((uint64_t)pos[i] * step[i], c[i], s[i]);
    }
    __syncthreads();
    if (n >= a.N) return;
#pragma unroll 1
    for (int round = share; round < rounds; round += a.per_token) {
        fetch(round + a.per_token, ahead);
        const int which = round >= first, h = (round - (which ? first : 0)) * slots + slot;
        const Heads& p = a.part[which];
        float f[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) f[i] = to_f32(x.v[i]);
        if (p.weight) {
            float sum = 0.f;
#pragma unroll
            for (int i = 0; i < 16; ++i) sum = fmaf(f[i], f[i], sum);
            for (int o = 1; o < lanes; o <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
            const float inv = __frsqrt_rn(sum / (float)a.D + a.eps);
#pragma unroll
            for (int i = 0; i < 16; i += 4) {
                const float4 w = *reinterpret_cast<const float4*>(&weights[which][16 * l + i]);
                f[i] = f[i] * inv * w.x;
                f[i + 1] = f[i + 1] * inv * w.y;
                f[i + 2] = f[i + 2] * inv * w.z;
                f[i + 3] = f[i + 3] * inv * w.w;
            }
        }
#pragma unroll
        for (int g = 0; g < 8 / V; ++g)
            if (turns(g)) {
                const int b = V * g;
                if (INTERLEAVED) {   // values 2 i and 2 i + 1 of the 2 V that lie in a row
                    auto value = [&](int i) -> float& { return f[i < V ? b + i : 8 + b + i - V]; };
#pragma unroll
                    for (int i = 0; i < V; ++i) {
                        const float u = value(2 * i), v = value(2 * i + 1);
                        value(2 * i) = u * c[b + i] - v * s[b + i];
                        value(2 * i + 1) = v * c[b + i] + u * s[b + i];
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < V; ++i) {
                        const float u = f[b + i], v = f[8 + b + i];
                        f[b + i] = u * c[b + i] - v * s[b + i];
                        f[8 + b + i] = v * c[b + i] + u * s[b + i];
                    }
                }
            }
        if (h < p.heads) {
            T* dst = static_cast<T*>(p.out) + n * p.o_token + h * p.o_head;
            Values y;
#pragma unroll
            for (int i = 0; i < 16; ++i) y.v[i] = from_f32<T>(f[i]);
#pragma unroll
            for (int g = 0; g < 8 / V; ++g)
                if (in(g)) {
                    put<T, V>(dst + at(g), y.v + V * g);
                    put<T, V>(dst + other(g), y.v + 8 + V * g);
                }
        }
        x = ahead;
    }
}

template <class T>
const void* heads_kernel(int v, bool interleaved)
{
    if (interleaved) return v == 8 ? (const void*)us_heads_kernel<T, 8, true> : v == 4 ? (const void*)us_heads_kernel<T, 4, true> : (const void*)us_heads_kernel<T, 1, true>;
    return v == 8 ? (const void*)us_heads_kernel<T, 8, false> : v == 4 ? (const void*)us_heads_kernel<T, 4, false> : (const void*)us_heads_kernel<T, 1, false>;
}

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
    while ((16 << a.log2_lanes) < D) ++a.log2_lanes;
    // A token's rounds go to as many warps as fill the GPU; each finds the sines and cosines anew.
    const int64_t slots = 32 >> a.log2_lanes, rounds = (a.part[0].heads + slots - 1) / slots + (a.part[1].heads + slots - 1) / slots;
    a.per_token = (int32_t)std::max<int64_t>(1, std::min<int64_t>(rounds, (32ll * ops_sms() + N - 1) / N));
    const int64_t blocks = (N * a.per_token + kHeadsThreads / 32 - 1) / (kHeadsThreads / 32);
    const void* kernel = type == US_F16 ? heads_kernel<__half>(vec, r->interleaved != 0) : type == US_BF16 ? heads_kernel<__nv_bfloat16>(vec, r->interleaved != 0) :
                                          heads_kernel<float>(vec, r->interleaved != 0);
    void* args[] = {&a};
    const cudaError_t e = ops_launch(kernel, dim3((unsigned)blocks), kHeadsThreads, 0, static_cast<cudaStream_t>(stream), args);
    if (e == cudaSuccess) return US_OK;
    cudaGetLastError();
    return US_ERR_CUDA;
}
