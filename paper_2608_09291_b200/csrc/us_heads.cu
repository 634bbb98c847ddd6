// Norms of query and key heads and the rotation of their positions, in one pass: what stands between the Q/K/V projection and the cache.
#include "us_mx4.cuh"
#include "us_ops.h"

namespace us {
namespace {

// A head x of D values: y = x / sqrt(mean x^2 + eps) * w (where there are weights), and of y's first `rotary` values the pairs (i, i + rotary/2), or
// (2i, 2i + 1), turned by position * frequency_i.
//   * Turns are counted in 2^-64: position * turns wraps at a whole turn by itself, so that the angle of a far position is as good as a near
//     one's (in 32-bit arithmetic 131072 radians are known to 2^-7). What is left after quarter turns goes to sincospi.
//   * A lane has eight pairs in registers, as two pieces of eight values: both ends of a pair are its own. 2 to 16 lanes have a head (a power of two, D / 16
//     of them have values), a warp 32 / lanes heads at a time. The sines and cosines of a lane's pairs are found once for all heads that the warp walks
//     over.
//   * Pairs behind the rotated ones are values that only the norm touches.
// Bound by memory where there are many tokens, by launch and one trip to memory for a single one.
struct Heads {
    const void* x;
    int64_t token, head;       // strides
    void* out;
    int64_t o_token, o_head;
    const void* weight;        // D values, or nullptr: no norm
    int32_t heads, w_type;
};
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

template <class T>
__device__ __forceinline__ float weight_at(const void* w, int32_t type, int i)
{
    return type == US_F32 ? static_cast<const float*>(w)[i] : type == US_F16 ? __half2float(static_cast<const __half*>(w)[i]) :
                            __bfloat162float(static_cast<const __nv_bfloat16*>(w)[i]);
}
// cos and sin of `part` / 2^64 turns
__device__ __forceinline__ void turn(uint64_t part, float& c, float& s)
{
    const uint64_t r = part + (1ull << 61);                                    // quarters: the nearest one, and -1/8 .. 1/8 turn from it
    const int32_t rest = (int32_t)(uint32_t)((r << 2) >> 32) ^ (int32_t)0x80000000;   // (2 bits of quarter gone; 2^-34 turns each)
    float a, b;
    sincospif((float)rest * 0x1p-33f, &a, &b);
    const uint32_t q = (uint32_t)(r >> 62);
    const float cc = q & 1 ? a : b, ss = q & 1 ? b : a;
    c = q == 1 || q == 2 ? -cc : cc;
    s = q >= 2 ? -ss : ss;
}
// V values in one access of V sizeof(T) bytes, 16 at most
template <class T, int V>
__device__ __forceinline__ void get(const T* p, float* v)
{
    constexpr int B = V * (int)sizeof(T);
    union { uint4 q[B > 16 ? B / 16 : 1]; uint2 d; uint32_t w; uint16_t h; T e[V]; } u;
    if (B >= 16)
#pragma unroll
        for (int i = 0; i < B / 16; ++i) u.q[i] = __ldcg(reinterpret_cast<const uint4*>(p) + i);
    else if (B == 8) u.d = __ldcg(reinterpret_cast<const uint2*>(p));
    else if (B == 4) u.w = __ldcg(reinterpret_cast<const uint32_t*>(p));
    else u.h = __ldcg(reinterpret_cast<const uint16_t*>(p));
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = to_f32(u.e[i]);
}
template <class T, int V>
__device__ __forceinline__ void put(T* p, const float* v)
{
    constexpr int B = V * (int)sizeof(T);
    union { uint4 q[B > 16 ? B / 16 : 1]; uint2 d; uint32_t w; uint16_t h; T e[V]; } u;
#pragma unroll
    for (int i = 0; i < V; ++i) u.e[i] = from_f32<T>(v[i]);
    if (B >= 16)
#pragma unroll
        for (int i = 0; i < B / 16; ++i) reinterpret_cast<uint4*>(p)[i] = u.q[i];
    else if (B == 8) *reinterpret_cast<uint2*>(p) = u.d;
    else if (B == 4) *reinterpret_cast<uint32_t*>(p) = u.w;
    else *reinterpret_cast<uint16_t*>(p) = u.h;
}

// V: pairs that lie side by side in memory (8, 4 or 1), which divide rotary / 2 and D / 2.
template <class T, int V, bool INTERLEAVED>
__global__ void __launch_bounds__(256) us_heads_kernel(const __grid_constant__ HeadsCall a)
{
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int lane = threadIdx.x & 31, lanes = 1 << a.log2_lanes, slot = lane >> a.log2_lanes, slots = 32 >> a.log2_lanes;
    const int p0 = 8 * (lane & (lanes - 1)), half = a.rotary / 2;   // the lane's first pair
    const int64_t warp = ((int64_t)blockIdx.x * blockDim.x + threadIdx.x) >> 5;
    const int64_t n = warp / a.per_token;
    const int share = (int)(warp - n * a.per_token);
    // places of the first values of its groups of V pairs, and of their other ends
    int at[8 / V], other[8 / V];
    bool in[8 / V], turns[8 / V];
#pragma unroll
    for (int g = 0; g < 8 / V; ++g) {
        const int p = p0 + V * g;
        in[g] = p < a.D / 2;
        turns[g] = p < half;
        at[g] = INTERLEAVED || !turns[g] ? 2 * p : p;
        other[g] = INTERLEAVED || !turns[g] ? 2 * p + V : p + half;
    }
    uint64_t step[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) step[i] = turns[i / V] && p0 + i < half ? __ldg(a.turns + p0 + i) : 0;   // (constant since the handle was made)
    asm volatile("griddepcontrol.wait;" ::: "memory");
    if (n >= a.N) return;
    float c[8], s[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        c[i] = 1.f;
        s[i] = 0.f;
        if (turns[i / V]) {
            const int64_t pos = __ldcg(a.positions + (a.axis ? (int64_t)__ldg(a.axis + p0 + i) * a.axis_stride : 0) + n);
            turn((uint64_t)pos * step[i], c[i], s[i]);
        }
    }
    const int total = a.part[0].heads + a.part[1].heads;
    float w[16];
    int held = -1;   // whose weights are in w
    for (int h0 = share * slots; h0 < total; h0 += a.per_token * slots) {
        const int hh = h0 + slot, which = hh >= a.part[0].heads ? 1 : 0, h = hh - (which ? a.part[0].heads : 0);
        const bool real = hh < total;
        const Heads& p = a.part[which];
        float x[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) x[i] = 0.f;
        if (real) {
            const T* src = static_cast<const T*>(p.x) + n * p.token + h * p.head;
#pragma unroll
            for (int g = 0; g < 8 / V; ++g)
                if (in[g]) {
                    get<T, V>(src + at[g], x + V * g);
                    get<T, V>(src + other[g], x + 8 + V * g);
                }
        }
        if (p.weight && held != which) {
#pragma unroll
            for (int g = 0; g < 8 / V; ++g)
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    w[V * g + i] = in[g] ? weight_at<T>(p.weight, p.w_type, at[g] + i) : 0.f;
                    w[8 + V * g + i] = in[g] ? weight_at<T>(p.weight, p.w_type, other[g] + i) : 0.f;
                }
            held = which;
        }
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) sum = fmaf(x[i], x[i], sum);
        for (int o = 1; o < lanes; o <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        if (!real) continue;
        if (p.weight) {
            const float inv = __frsqrt_rn(sum / (float)a.D + a.eps);
#pragma unroll
            for (int i = 0; i < 16; ++i) x[i] = x[i] * inv * w[i];
        }
        float y[16];
#pragma unroll
        for (int g = 0; g < 8 / V; ++g) {
            const int b = V * g;
            if (INTERLEAVED && turns[g]) {   // values 2 i and 2 i + 1 of the 2 V that lie in a row
                float r[2 * V];
#pragma unroll
                for (int i = 0; i < V; ++i) { r[i] = x[b + i]; r[V + i] = x[8 + b + i]; }
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const float u = r[2 * i], v = r[2 * i + 1];
                    r[2 * i] = u * c[b + i] - v * s[b + i];
                    r[2 * i + 1] = v * c[b + i] + u * s[b + i];
                }
#pragma unroll
                for (int i = 0; i < V; ++i) { y[b + i] = r[i]; y[8 + b + i] = r[V + i]; }
            } else {
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const float u = x[b + i], v = x[8 + b + i];
                    y[b + i] = turns[g] ? u * c[b + i] - v * s[b + i] : u;
                    y[8 + b + i] = turns[g] ? v * c[b + i] + u * s[b + i] : v;
                }
            }
        }
        T* dst = static_cast<T*>(p.out) + n * p.o_token + h * p.o_head;
#pragma unroll
        for (int g = 0; g < 8 / V; ++g)
            if (in[g]) {
                put<T, V>(dst + at[g], y + V * g);
                put<T, V>(dst + other[g], y + 8 + V * g);
            }
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
    // A token's heads go to as many warps as fill the GPU; each finds the sines and cosines anew.
    const int64_t slots = 32 >> a.log2_lanes, rounds = (heads + slots - 1) / slots;
    a.per_token = (int32_t)std::max<int64_t>(1, std::min<int64_t>(rounds, (48ll * ops_sms() + N - 1) / N));
    const int64_t blocks = (N * a.per_token + 7) / 8;
    const void* kernel = type == US_F16 ? heads_kernel<__half>(vec, r->interleaved != 0) : type == US_BF16 ? heads_kernel<__nv_bfloat16>(vec, r->interleaved != 0) :
                                          heads_kernel<float>(vec, r->interleaved != 0);
    void* args[] = {&a};
    const cudaError_t e = ops_launch(kernel, dim3((unsigned)blocks), 256, 0, static_cast<cudaStream_t>(stream), args);
    if (e == cudaSuccess) return US_OK;
    cudaGetLastError();
    return US_ERR_CUDA;
}
