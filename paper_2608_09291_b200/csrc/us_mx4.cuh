// MX4: dense matrices in microscaled 4-bit floating point (E2M1 values, one E8M0 scale for 32 of a row), their
// quantisation and their product on the block-scaled tensor-core path of sm_100a.
//
// Held form ("tiles"): a matrix of rows x K is cut in tiles of 128 rows x 256 columns, row tiles outermost. A tile is 17 KB in one
// piece, in the order that the tensor core reads it from shared memory, so that one untiled bulk copy brings an operand stage:
//   [0, 1024)      scale bytes: half h (128 columns), row r, 32-column block b of the half: 512 h + 16 (r % 32) + 4 (r / 32) + b
//   [1024, 17408)  codes: row r, block c (0..7) of 16 bytes at 128 r + 16 (c ^ (r % 8)); even column in the low bits of a byte
// Columns past K in the last tile are zero codes with scale byte 0. Rows past the last one are never written: a row of an operand
// meets only its own row (column) of the product, and those are not stored.
#pragma once
#include "us_spmm_tc.cuh"

#include <cuda_bf16.h>

namespace us {

constexpr int kMxScales = 1024, kMxCodes = 16384, kMxTile = kMxScales + kMxCodes;   // bytes

__host__ __device__ __forceinline__ int64_t mx4_tiles(int64_t n, int64_t per) { return (n + per - 1) / per; }
__device__ __forceinline__ uint32_t mx4_code_off(uint32_t r, uint32_t c) { return (uint32_t)kMxScales + 128u * r + 16u * (c ^ (r & 7u)); }
__device__ __forceinline__ uint32_t mx4_scale_off(uint32_t r, uint32_t half) { return 512u * half + 16u * (r & 31u) + 4u * (r >> 5); }

// Bounded wait of a whole warp: a few hundred tries, each of which sleeps on the barrier, before the clock is first read (reading it
// costs more than most of these waits take; behind it as tc_wait_warp, which see).
__device__ __forceinline__ bool ops_wait_warp(uint32_t bar, uint32_t parity, uint32_t limit_hi, volatile uint32_t* dead, bool after = false)
{
#pragma unroll 1
    for (int i = 0; i < 256; ++i) {
        if (__all_sync(0xffffffffu, mbar_try_wait(bar, parity))) return true;
        if (__any_sync(0xffffffffu, *dead)) return false;
    }
    return tc_wait_warp(bar, parity, limit_hi, dead, after);
}
// The same for one thread.
__device__ __forceinline__ bool ops_wait(uint32_t bar, uint32_t parity, uint32_t limit_hi)
{
#pragma unroll 1
    for (int i = 0; i < 256; ++i)
        if (mbar_try_wait(bar, parity)) return true;
    return mbar_wait_bounded(bar, parity, limit_hi);
}

// ---- quantisation ----------------------------------------------------------------------------------------------------
// Scale byte of a block whose largest magnitude has these fp32 bits: e = floor(log2 a) - 2 clamped to [-127, 127], + 127. With the
// biased exponent x of a that is x - 2 (subnormal and 0: 0); Inf and NaN: 255, the scale's NaN.
__device__ __forceinline__ uint32_t mx4_scale_byte(uint32_t amax_bits)
{
    const uint32_t x = amax_bits >> 23;
    return x >= 255u ? 255u : (x > 2u ? x - 2u : 0u);
}
// 2^(127 - byte), exact; 0 for the NaN scale (whose codes are all 0)
__device__ __forceinline__ float mx4_inverse(uint32_t byte) { return byte == 255u ? 0.f : __uint_as_float((254u - byte) << 23); }
// eight values -> eight codes, element e in nibble e (the conversion rounds to nearest even and saturates at 6)
__device__ __forceinline__ uint32_t mx4_codes8(const float (&v)[8], float inv)
{
    uint32_t w;
    asm("{\n\t.reg .b8 a, b, c, d;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n\t"
        "mov.b32 %0, {a, b, c, d};\n\t}"
        : "=r"(w)
        : "f"(v[0] * inv), "f"(v[1] * inv), "f"(v[2] * inv), "f"(v[3] * inv), "f"(v[4] * inv), "f"(v[5] * inv), "f"(v[6] * inv), "f"(v[7] * inv));
    return w;
}

template <class T> __device__ __forceinline__ float to_f32(T v);
template <> __device__ __forceinline__ float to_f32<__half>(__half v) { return __half2float(v); }
template <> __device__ __forceinline__ float to_f32<__nv_bfloat16>(__nv_bfloat16 v) { return __bfloat162float(v); }
template <> __device__ __forceinline__ float to_f32<float>(float v) { return v; }
template <class T> __device__ __forceinline__ T from_f32(float v);
template <> __device__ __forceinline__ __half from_f32<__half>(float v) { return __float2half_rn(v); }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ float from_f32<float>(float v) { return v; }

// Eight elements of a row as they are; `whole`: 16-byte aligned and inside the row.
template <class T>
struct Eight {
    T v[8];
};
template <class T>
__device__ __forceinline__ Eight<T> load8(const T* p, int64_t left, bool whole)
{
    Eight<T> r;
    if (whole) {
#pragma unroll
        for (int i = 0; i < (int)sizeof(Eight<T>) / 16; ++i) reinterpret_cast<uint4*>(&r)[i] = __ldcg(reinterpret_cast<const uint4*>(p) + i);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) r.v[i] = i < left ? p[i] : from_f32<T>(0.f);
    }
    return r;
}

// A warp quantises the 256 columns of one row of one tile: four lanes a block, eight columns a lane. Returns the lane's word of
// codes; `sc` has, in lanes 0 and 16, the four scale bytes of the half that begins there.
template <class T>
__device__ __forceinline__ uint32_t mx4_quantize_row(const Eight<T>& x, uint32_t& sc)
{
    float f[8];
    uint32_t big = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        f[i] = to_f32(x.v[i]);
        big = max(big, __float_as_uint(f[i]) & 0x7FFFFFFFu);
    }
    big = max(big, __shfl_xor_sync(0xffffffffu, big, 1));
    big = max(big, __shfl_xor_sync(0xffffffffu, big, 2));
    const uint32_t byte = mx4_scale_byte(big);
    if (byte == 255u)
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = 0.f;
    const uint32_t codes = mx4_codes8(f, mx4_inverse(byte));
    uint32_t s = byte | (__shfl_down_sync(0xffffffffu, byte, 4) << 8);
    sc = s | (__shfl_down_sync(0xffffffffu, s, 8) << 16);
    return codes;
}

// Unit u of rows of `per` units: its row and its place there. (A 64-bit division takes longer than a unit's arithmetic.)
__device__ __forceinline__ void mx4_unit(int64_t u, int64_t per, int64_t& row, int64_t& place)
{
    if ((u | per) >> 32) {
        row = u / per;
        place = u - row * per;
    } else {
        const uint32_t r = (uint32_t)u / (uint32_t)per;
        row = r;
        place = (uint32_t)u - r * (uint32_t)per;
    }
}

// 32 bytes in one access
__device__ __forceinline__ void load32b(const void* p, uint32_t* w)
{
    asm volatile("ld.global.v8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                 : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7]) : "l"(p) : "memory");
}
__device__ __forceinline__ void store32b(void* p, const uint32_t* w)
{
    asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};"
                 ::"l"(p), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7]) : "memory");
}
// Sixteen elements of a row as they are, in 32-bit words. vec: bytes of an access (32, 16, 8, 4, or 1: one element at a time).
template <class T>
struct Sixteen {
    uint32_t w[4 * sizeof(T)];
};
template <class T>
__device__ __forceinline__ void load16(Sixteen<T>& r, const T* p, int64_t left, int vec)
{
    constexpr int W = 4 * (int)sizeof(T);
    if (left >= 16 && vec == 32) {
#pragma unroll
        for (int i = 0; i < W; i += 8) load32b(reinterpret_cast<const uint32_t*>(p) + i, r.w + i);
    } else if (left >= 16 && vec == 16) {
#pragma unroll
        for (int i = 0; i < W; i += 4) {
            const uint4 v = __ldcg(reinterpret_cast<const uint4*>(reinterpret_cast<const uint32_t*>(p) + i));
            r.w[i] = v.x; r.w[i + 1] = v.y; r.w[i + 2] = v.z; r.w[i + 3] = v.w;
        }
    } else if (left >= 16 && vec == 8) {
#pragma unroll
        for (int i = 0; i < W; i += 2) {
            const uint2 v = __ldcg(reinterpret_cast<const uint2*>(reinterpret_cast<const uint32_t*>(p) + i));
            r.w[i] = v.x; r.w[i + 1] = v.y;
        }
    } else if (left >= 16 && vec == 4) {
#pragma unroll
        for (int i = 0; i < W; ++i) r.w[i] = __ldcg(reinterpret_cast<const uint32_t*>(p) + i);
    } else {
        union { uint32_t w[W]; T v[16]; } u;
#pragma unroll
        for (int i = 0; i < 16; ++i) u.v[i] = i < left ? p[i] : from_f32<T>(0.f);
#pragma unroll
        for (int i = 0; i < W; ++i) r.w[i] = u.w[i];
    }
}
// The bits of the largest magnitude of sixteen, as an fp32's
template <class T>
__device__ __forceinline__ uint32_t amax16(const Sixteen<T>& x)
{
    uint32_t m[4 * sizeof(T)];
#pragma unroll
    for (int i = 0; i < 4 * (int)sizeof(T); ++i) m[i] = x.w[i] & (sizeof(T) == 2 ? 0x7FFF7FFFu : 0x7FFFFFFFu);
    if (sizeof(T) == 4) {
#pragma unroll
        for (int n = 8; n; n >>= 1)
#pragma unroll
            for (int i = 0; i < n; ++i) m[i] = max(m[i], m[(i + n) % (4 * sizeof(T))]);
        return m[0];
    }
#pragma unroll
    for (int n = 4; n; n >>= 1)   // (magnitudes order like their bits: both halves at once)
#pragma unroll
        for (int i = 0; i < n; ++i) m[i] = __vmaxu2(m[i], m[i + n]);
    const uint32_t b = max(m[0] & 0xFFFFu, m[0] >> 16);
    return std::is_same<T, __half>::value ? __float_as_uint(__half2float(__ushort_as_half((unsigned short)b))) : b << 16;
}
template <class T>
__device__ __forceinline__ void pair16(const Sixteen<T>& x, int i, float& a, float& b)   // elements 2 i, 2 i + 1
{
    if (sizeof(T) == 4) {
        a = __uint_as_float(x.w[2 * i % (4 * sizeof(T))]);
        b = __uint_as_float(x.w[(2 * i + 1) % (4 * sizeof(T))]);
    } else if (std::is_same<T, __half>::value) {
        const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&x.w[i]));
        a = f.x;
        b = f.y;
    } else {
        a = __uint_as_float(x.w[i] << 16);
        b = __uint_as_float(x.w[i] & 0xFFFF0000u);
    }
}

// X (rows x K, row stride ldx) -> tiles. A warp takes 512 columns of a row (two tiles), sixteen a lane, two lanes a block; kMxUnroll of
// them at a time, all loads first. With eight columns a lane the arithmetic around the elements kept the GPU at half its memory's rate
// (8192 x 8192 bf16, 170 MB: 38 us; with sixteen 29, 26 at memory's rate).
constexpr int kMxUnroll = 2;
template <class T>
__global__ void __launch_bounds__(256) us_mx4_quantize_kernel(const T* X, int64_t ldx, int64_t rows, int64_t K, uint8_t* mx, int vec)
{
    const int lane = threadIdx.x & 31;
    const int64_t kt = mx4_tiles(K, 256), groups = mx4_tiles(kt, 2 * kMxUnroll);
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    for (int64_t u = ((int64_t)blockIdx.x * blockDim.x + threadIdx.x) >> 5; u < rows * groups; u += ((int64_t)gridDim.x * blockDim.x) >> 5) {
        int64_t r, j0;
        mx4_unit(u, groups, r, j0);
        j0 = 2 * kMxUnroll * j0 + (lane >> 4);   // the lane's tile
        const int l = lane & 15;
        const T* src = X + r * ldx + 256 * j0 + 16 * l;
        Sixteen<T> x[kMxUnroll];
#pragma unroll
        for (int i = 0; i < kMxUnroll; ++i) load16(x[i], src + 512 * i, K - 256 * (j0 + 2 * i) - 16 * l, vec);
        const uint32_t rr = (uint32_t)(r & 127);
        uint8_t* tile = mx + ((r >> 7) * kt + j0) * kMxTile;
        const uint32_t at_code = mx4_code_off(rr, l >> 1) + 8 * (l & 1), at_scale = mx4_scale_off(rr, l >> 3);
#pragma unroll
        for (int i = 0; i < kMxUnroll; ++i) {
            uint32_t big = amax16(x[i]);
            big = max(big, __shfl_xor_sync(0xffffffffu, big, 1));
            const uint32_t byte = mx4_scale_byte(big);
            const float inv = mx4_inverse(byte);
            uint32_t c[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                float f[8];
#pragma unroll
                for (int e = 0; e < 4; ++e) pair16(x[i], 4 * h + e, f[2 * e], f[2 * e + 1]);
                c[h] = mx4_codes8(f, inv);
            }
            // the four scale bytes of the lane's half, in its first lane of eight
            uint32_t s = byte | (__shfl_down_sync(0xffffffffu, byte, 2) << 8);
            s |= __shfl_down_sync(0xffffffffu, s, 4) << 16;
            if (j0 + 2 * i < kt) {
                *reinterpret_cast<uint2*>(tile + at_code) = byte == 255u ? make_uint2(0, 0) : make_uint2(c[0], c[1]);
                if ((l & 7) == 0) *reinterpret_cast<uint32_t*>(tile + at_scale) = s;
            }
            tile += 2 * kMxTile;
        }
    }
}

// eight codes -> their values
__device__ __forceinline__ void mx4_values8(uint32_t w, float (&v)[8])
{
    uint32_t h[4];
    asm("{\n\t.reg .b8 a, b, c, d;\n\tmov.b32 {a, b, c, d}, %4;\n\t"
        "cvt.rn.f16x2.e2m1x2 %0, a;\n\tcvt.rn.f16x2.e2m1x2 %1, b;\n\tcvt.rn.f16x2.e2m1x2 %2, c;\n\tcvt.rn.f16x2.e2m1x2 %3, d;\n\t}"
        : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3]) : "r"(w));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h[i]));
        v[2 * i] = f.x;
        v[2 * i + 1] = f.y;
    }
}
// 2^(byte - 127)
__device__ __forceinline__ float mx4_scale(uint32_t byte)
{
    return byte == 255u ? __uint_as_float(0x7FC00000u) : __uint_as_float(byte ? byte << 23 : 0x00400000u);
}

// Tiles -> values: 512 columns of a row a warp, sixteen a lane, as above.
template <class T>
__global__ void __launch_bounds__(256) us_mx4_dequantize_kernel(const uint8_t* mx, int64_t rows, int64_t K, T* out, int64_t ldo, int vec)
{
    constexpr int W = 4 * (int)sizeof(T);
    const int lane = threadIdx.x & 31;
    const int64_t kt = mx4_tiles(K, 256), groups = mx4_tiles(kt, 2 * kMxUnroll);
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    for (int64_t u = ((int64_t)blockIdx.x * blockDim.x + threadIdx.x) >> 5; u < rows * groups; u += ((int64_t)gridDim.x * blockDim.x) >> 5) {
        int64_t r, j0;
        mx4_unit(u, groups, r, j0);
        j0 = 2 * kMxUnroll * j0 + (lane >> 4);
        const int l = lane & 15;
        const uint32_t rr = (uint32_t)(r & 127);
        const uint8_t* tile = mx + ((r >> 7) * kt + j0) * kMxTile;
        const uint32_t at_code = mx4_code_off(rr, l >> 1) + 8 * (l & 1), at_scale = mx4_scale_off(rr, l >> 3) + ((l >> 1) & 3);
        uint2 w[kMxUnroll];
        uint32_t b[kMxUnroll];
#pragma unroll
        for (int i = 0; i < kMxUnroll; ++i) {
            const bool in = j0 + 2 * i < kt;
            w[i] = in ? __ldcg(reinterpret_cast<const uint2*>(tile + 2 * i * kMxTile + at_code)) : make_uint2(0, 0);
            b[i] = in ? __ldcg(tile + 2 * i * kMxTile + at_scale) : 0u;
        }
        T* dst = out + r * ldo + 256 * j0 + 16 * l;
#pragma unroll
        for (int i = 0; i < kMxUnroll; ++i) {
            const int64_t left = K - 256 * (j0 + 2 * i) - 16 * l;
            if (left <= 0) break;
            const float s = mx4_scale(b[i]);
            union { uint32_t w[W]; T v[16]; } y;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                float v[8];
                mx4_values8(h ? w[i].y : w[i].x, v);
#pragma unroll
                for (int e = 0; e < 8; ++e) y.v[8 * h + e] = from_f32<T>(v[e] * s);
            }
            if (left >= 16 && vec == 32) {
#pragma unroll
                for (int k = 0; k < W; k += 8) store32b(reinterpret_cast<uint32_t*>(dst) + k, y.w + k);
            } else if (left >= 16 && vec == 16) {
#pragma unroll
                for (int k = 0; k < W; k += 4) *reinterpret_cast<uint4*>(reinterpret_cast<uint32_t*>(dst) + k) = make_uint4(y.w[k], y.w[k + 1], y.w[k + 2], y.w[k + 3]);
            } else if (left >= 16 && vec == 8) {
#pragma unroll
                for (int k = 0; k < W; k += 2) *reinterpret_cast<uint2*>(reinterpret_cast<uint32_t*>(dst) + k) = make_uint2(y.w[k], y.w[k + 1]);
            } else if (left >= 16 && vec == 4) {
#pragma unroll
                for (int k = 0; k < W; ++k) reinterpret_cast<uint32_t*>(dst)[k] = y.w[k];
            } else {
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    if (e < left) dst[e] = y.v[e];
            }
            dst += 512;
        }
    }
}

// Row-major codes (two a byte) and scale bytes <-> tiles: a warp a row of a tile, byte by byte. What a checkpoint's loading does once: 28672 x 8192,
// 250 MB there and back: 220 us, unpacked 196, where memory's rate would give 38.
template <bool PACK>
__global__ void __launch_bounds__(256) us_mx4_repack_kernel(uint8_t* codes, int64_t ldc, uint8_t* scales, int64_t lds, int64_t rows, int64_t K, uint8_t* mx)
{
    const int lane = threadIdx.x & 31;
    const int64_t kt = mx4_tiles(K, 256);
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    for (int64_t u = ((int64_t)blockIdx.x * blockDim.x + threadIdx.x) >> 5; u < rows * kt; u += ((int64_t)gridDim.x * blockDim.x) >> 5) {
        int64_t r, j;
        mx4_unit(u, kt, r, j);
        uint8_t* tile = mx + ((r >> 7) * kt + j) * kMxTile;
        const uint32_t rr = (uint32_t)(r & 127);
        uint32_t* word = reinterpret_cast<uint32_t*>(tile + mx4_code_off(rr, lane >> 2) + 4 * (lane & 3));
        const int64_t k0 = 256 * j + 8 * lane, b = 8 * j + lane;
        uint32_t w = PACK ? 0u : *word;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int64_t k = k0 + 2 * i;
            if (k >= K) break;
            uint8_t* c = codes + r * ldc + (k >> 1);
            const uint32_t keep = k + 1 < K ? 0xFFu : 0x0Fu;
            if (PACK) w |= ((uint32_t)*c & keep) << (8 * i);
            else *c = (uint8_t)((w >> (8 * i)) & keep);
        }
        if (PACK) *word = w;
        if (lane < 8) {
            uint8_t* s = tile + mx4_scale_off(rr, lane >> 2) + (lane & 3);
            if (PACK) *s = 32 * b < K ? scales[r * lds + b] : (uint8_t)0;
            else if (32 * b < K) scales[r * lds + b] = *s;
        }
    }
}

// ---- the product ---------------------------------------------------------------------------------------------------------
// D (128 weight rows x NB tokens, fp32, tensor memory) += W tile * X tile^T, 64 columns an instruction, the scale bytes copied from
// shared to tensor memory in front of the four instructions of a 256-column stage. One warp copies (untiled bulk copies into a ring
// of stages), one issues, four read the sums back and store.
//   * Weights are the M side: every lane of tensor memory has a weight row, whatever the number of tokens; N = 16 .. 128 (more: pairs, below).
//   * Few row tiles: the columns are split over a cluster of up to 16 CTAs, whose sums are added through distributed shared memory
//     in the order of the ranks: no workspace, no atomics, the same result every time.
//   * Bound by the weights' way from memory: 28672 x 8192, 8 tokens: 22 us, 5.6 TB/s; 4096 x 4096, one token: 4.6 us, most of it latency.
//   * Few tokens (FUSE): the CTA quantises its own columns of X while its weights are on the way: one launch instead of two.
struct Mx4Params {
    const uint8_t* w;
    const uint8_t* x;      // tiles, or
    const void* X;         // (FUSE) rows of x_type
    void* Y;
    int64_t ldx, ldy;
    int32_t M, N, K, kt;
    int32_t split, col_tiles, tiles;   // tiles: of the whole product
    int32_t stages;        // ring stages
    int32_t x_type, y_type;
    int32_t x_vec, y_vec;  // rows of X, of Y take 16-byte accesses
    int32_t w_stable;      // the weights are complete whatever the stream's earlier work does
    uint32_t* err;
};
enum { kF16 = 0, kBF16 = 1, kF32 = 2 };
constexpr uint32_t kMxWait = 2000000u;   // bounded waits, ns >> 10

template <int NB, bool FUSE>
struct Mx4Shape {
    static_assert(NB <= 128, "one tile of activations holds the tokens");
    static constexpr int kXTile = kMxScales + NB * 128;                    // bytes of a stage's activations
    static constexpr int kStage = kMxTile + (FUSE ? 0 : kXTile);
    static constexpr int kSfCols = 16;                                     // tensor-memory columns of a stage's scales
    static constexpr int kCols = NB + 2 * kSfCols <= 64 ? 64 : NB + 2 * kSfCols <= 128 ? 128 : NB + 2 * kSfCols <= 256 ? 256 : 512;
    static constexpr int kMaxStages = 12;
};

__device__ __forceinline__ uint64_t mx4_desc(uint32_t addr, uint32_t sbo, uint32_t swizzle)
{
    return ((uint64_t)1 << 16) | ((uint64_t)(sbo >> 4) << 32) | (1ull << 46) | ((uint64_t)swizzle << 61) | (uint64_t)((addr & 0x3FFFFu) >> 4);
}
__device__ __forceinline__ void mx4_mma(uint32_t elected, uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t sfa, uint32_t sfb, uint32_t accumulate)
{
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 q, %7, 0;\n\tsetp.ne.u32 p, %6, 0;\n\t"
                 "@q tcgen05.mma.cta_group::1.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
                 ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(sfa), "r"(sfb), "r"(accumulate), "r"(elected) : "memory");
}
// 512 bytes of scales (128 rows, 4 blocks) -> 4 columns, the same in all four lane quarters
__device__ __forceinline__ void mx4_copy_scales(uint32_t elected, uint32_t d, uint64_t s)
{
    asm volatile("{\n\t.reg .pred q;\n\tsetp.ne.u32 q, %2, 0;\n\t@q tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;\n\t}"
                 ::"r"(d), "l"(s), "r"(elected) : "memory");
}
#define US_R8(r, i) "=r"(r[i]), "=r"(r[i + 1]), "=r"(r[i + 2]), "=r"(r[i + 3]), "=r"(r[i + 4]), "=r"(r[i + 5]), "=r"(r[i + 6]), "=r"(r[i + 7])
#define US_I8(r, i) "r"(r[i]), "r"(r[i + 1]), "r"(r[i + 2]), "r"(r[i + 3]), "r"(r[i + 4]), "r"(r[i + 5]), "r"(r[i + 6]), "r"(r[i + 7])
// 32 columns of the thread's lane, fetched without waiting
__device__ __forceinline__ void tc_ld32(uint32_t addr, uint32_t (&r)[32])
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,"
                 "%27,%28,%29,%30,%31}, [%32];" : US_R8(r, 0), US_R8(r, 8), US_R8(r, 16), US_R8(r, 24) : "r"(addr));
}
__device__ __forceinline__ void tc_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tc_st32(uint32_t addr, const uint32_t (&r)[32])
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,"
                 "%27,%28,%29,%30,%31};" ::US_I8(r, 0), US_I8(r, 8), US_I8(r, 16), US_I8(r, 24), "r"(addr) : "memory");
}
__device__ __forceinline__ void tc_st16_lanes(uint32_t addr, const uint32_t (&r)[16])
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15};"
                 ::US_I8(r, 0), US_I8(r, 8), "r"(addr) : "memory");
}
// (values that an asynchronous load writes must not be moved in front of its wait)
__device__ __forceinline__ void pin32(uint32_t (&r)[32])
{
#pragma unroll
    for (int i = 0; i < 32; ++i) asm volatile("" : "+r"(r[i])::"memory");
}
__device__ __forceinline__ void tc_ld16(uint32_t addr, uint32_t (&r)[16])
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
                   "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
                 : "r"(addr));
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ float4 ld_cluster_f32x4(uint32_t local, uint32_t rank)
{
    uint32_t a;
    float4 v;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(local), "r"(rank));
    asm volatile("ld.shared::cluster.v4.f32 {%0,%1,%2,%3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(a) : "memory");
    return v;
}
// Y[n][m .. m + 3] (the matrix ends at M)
__device__ __forceinline__ void mx4_store4(const Mx4Params& p, int64_t n, int64_t m, const float (&v)[4])
{
    const int64_t at = n * p.ldy + m;
    const bool whole = p.y_vec && m + 4 <= p.M;
    if (p.y_type == kF32) {
        float* y = static_cast<float*>(p.Y) + at;
        if (whole) *reinterpret_cast<float4*>(y) = make_float4(v[0], v[1], v[2], v[3]);
        else for (int i = 0; i < 4; ++i) if (m + i < p.M) y[i] = v[i];
    } else {
        uint16_t h[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) h[i] = p.y_type == kF16 ? __half_as_ushort(__float2half_rn(v[i])) : __bfloat16_as_ushort(__float2bfloat16_rn(v[i]));
        uint16_t* y = static_cast<uint16_t*>(p.Y) + at;
        if (whole) *reinterpret_cast<uint2*>(y) = make_uint2(h[0] | ((uint32_t)h[1] << 16), h[2] | ((uint32_t)h[3] << 16));
        else for (int i = 0; i < 4; ++i) if (m + i < p.M) y[i] = h[i];
    }
}
__device__ __forceinline__ void bar_epilogue() { asm volatile("bar.sync 1, 128;" ::: "memory"); }
// The same barrier, and whether any of its threads says so.
__device__ __forceinline__ bool bar_any(bool say)
{
    uint32_t any;
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\tbarrier.cta.red.or.pred q, 1, 128, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
                 : "=r"(any) : "r"((uint32_t)say) : "memory");
    return any != 0;
}

// The tile's sums (four warps, lane quarter `quarter`): 32 tokens at a time to shared memory as they are stored, [token][weight row], and
// from there in whole lines: every thread 16 bytes of a token's 256 (512). Straight from the registers a warp's store of one token is 64
// bytes; 4096 x 28672 x 8192 took 705 us that way, whatever the products took.
template <class T>
__device__ __forceinline__ void mx4_write_tile(const Mx4Params& p, uint32_t tm, int quarter, int lane, int64_t m0, int64_t n0, int nn, uint8_t* stage)
{
    constexpr int PITCH = 128 * (int)sizeof(T) + 16, PER = 16 / (int)sizeof(T), ROW = 128 / PER;   // bytes of a token, values of a piece, pieces of a token
    const int row = 32 * quarter + lane, tid = row;
    const int m_here = (int)min((int64_t)128, p.M - m0);
    int buf = 0;
#pragma unroll 1
    for (int c = 0; c < nn; c += 32) {
        uint32_t r[32];
        tc_ld32(tm + ((uint32_t)quarter << 21) + (uint32_t)c, r);
        tc_wait_ld();
        pin32(r);
        uint8_t* b = stage + buf * (32 * PITCH);
#pragma unroll
        for (int i = 0; i < 32; ++i) *reinterpret_cast<T*>(b + i * PITCH + row * sizeof(T)) = from_f32<T>(__uint_as_float(r[i]));
        bar_epilogue();   // (two buffers: whoever is a chunk behind still reads the other one)
        const int rows = min(32, nn - c);
        if (p.y_vec && m_here == 128) {
#pragma unroll
            for (int k = 0; k < 32 * ROW / 128; ++k) {
                const int i = tid + 128 * k, n = i / ROW, piece = i % ROW;
                if (n < rows) *reinterpret_cast<uint4*>(static_cast<T*>(p.Y) + (n0 + c + n) * p.ldy + m0 + piece * PER) = *reinterpret_cast<const uint4*>(b + n * PITCH + 16 * piece);
            }
        } else {
            for (int n = 0; n < rows; ++n)
                if (tid < m_here) static_cast<T*>(p.Y)[(n0 + c + n) * p.ldy + m0 + tid] = *reinterpret_cast<const T*>(b + n * PITCH + tid * sizeof(T));
        }
        buf ^= 1;
    }
}

// (FUSE) warps w of nw: the CTA's columns [256 t0, 256 t1) of the N tokens, quantised into operand tiles in shared memory
template <class T, int NB>
__device__ __forceinline__ void mx4_quantize_slice(const Mx4Params& p, uint8_t* xs, int t0, int t1, int w, int nw, int lane)
{
    constexpr int U = 4;
    const int units = (t1 - t0) * p.N;
    const uint32_t inv = ((1u << 24) + p.N - 1) / p.N;   // u / N = u inv / 2^24: N <= 16, and u inv < 2^32 for up to 255 tiles
#pragma unroll 1
    for (int u0 = w; u0 < units; u0 += U * nw) {
        Eight<T> x[U];
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const uint32_t u = u0 + i * nw, t = u * inv >> 24, n = u - t * p.N;
            const int64_t k = 256 * (int64_t)(t0 + t) + 8 * lane;
            if (u < units) x[i] = load8(static_cast<const T*>(p.X) + n * p.ldx + k, p.K - k, p.x_vec && k + 8 <= p.K);
        }
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const uint32_t u = u0 + i * nw, t = u * inv >> 24, n = u - t * p.N;
            if (u >= units) break;
            uint32_t sc;
            const uint32_t codes = mx4_quantize_row(x[i], sc);
            uint8_t* tile = xs + t * Mx4Shape<NB, true>::kXTile;
            *reinterpret_cast<uint32_t*>(tile + mx4_code_off(n, lane >> 2) + 4 * (lane & 3)) = codes;
            if ((lane & 15) == 0) *reinterpret_cast<uint32_t*>(tile + mx4_scale_off(n, lane >> 4)) = sc;
        }
    }
}

template <int NB, bool FUSE>
__global__ void __launch_bounds__(192, NB <= 64 ? 4 : 1) us_mx4_product_kernel(const __grid_constant__ Mx4Params p)
{
    using S = Mx4Shape<NB, FUSE>;
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    __shared__ __align__(8) uint64_t bars[2 * S::kMaxStages + 2];
    __shared__ uint32_t misc[2];   // tensor-memory address, dead
    uint8_t* ring = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
    uint8_t* xs = ring + (size_t)p.stages * S::kStage;   // (FUSE)
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t b_full = smem_u32(bars), b_empty = b_full + 8u * S::kMaxStages, b_x = b_empty + 8u * S::kMaxStages, b_done = b_x + 8u;
    volatile uint32_t* dead = misc + 1;
    const int rank = (int)blockIdx.x % p.split, tile = (int)blockIdx.x / p.split;
    const int mt = tile / p.col_tiles, nt = tile - mt * p.col_tiles;
    const int t0 = (int)((int64_t)rank * p.kt / p.split), t1 = (int)((int64_t)(rank + 1) * p.kt / p.split);
    const int n0 = nt * NB, nn = min(NB, p.N - n0);
    if (warp == 1) {
        if (lane < S::kMaxStages) { mbar_init(b_full + 8u * lane, 1); mbar_init(b_empty + 8u * lane, 1); }
        if (lane == 0) { mbar_init(b_x, 4); mbar_init(b_done, 1); misc[1] = 0; }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        __syncwarp();
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(misc)), "n"(S::kCols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    // Only now: a dependent's CTA that fits beside this one takes tensor memory of its own, and then waits for this kernel.
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const uint32_t tm = *(volatile uint32_t*)misc;
    bool ok = true;
    if (warp == 0) {
        // ---- copies ----
        if (lane == 0) {
            const uint8_t* w = p.w + ((int64_t)mt * p.kt + t0) * kMxTile;
            const int n = t1 - t0;
            const bool early = p.w_stable != 0;
            int issued = 0;
            // activations: the rows that hold tokens, rounded up to whole 8-row groups (the others' sums are not stored)
            const uint32_t x_bytes = FUSE ? 0u : (uint32_t)(kMxScales + 128 * ((nn + 7) & ~7));
            const uint8_t* x = p.x + ((int64_t)(n0 >> 7) * p.kt + t0) * kMxTile;
            auto copy_w = [&](int i, int s) {
                mbar_expect_tx(b_full + 8u * s, (uint32_t)kMxTile + x_bytes);
                bulk_g2s(smem_u32(ring + (size_t)s * S::kStage), w + (int64_t)i * kMxTile, kMxTile, b_full + 8u * s);
            };
            auto copy_x = [&](int i, int s) {
                bulk_g2s(smem_u32(ring + (size_t)s * S::kStage + kMxTile), x + (int64_t)i * kMxTile, x_bytes, b_full + 8u * s);
            };
            const int first = min(n, p.stages);
            if (early) for (int i = 0; i < first; ++i) copy_w(i, i);
            asm volatile("griddepcontrol.wait;" ::: "memory");
            for (int i = 0; i < first; ++i) {
                if (!early) copy_w(i, i);
                if (!FUSE) copy_x(i, i);
            }
            issued = first;
            int s = 0;
            uint32_t par = 0;
            for (int i = first; i < n; ++i) {
                if (!ops_wait(b_empty + 8u * s, par, kMxWait)) { ok = false; break; }
                copy_w(i, s);
                if (!FUSE) copy_x(i, s);
                ++issued;
                if (++s == p.stages) { s = 0; par ^= 1u; }
            }
            // (nothing may be in flight when the CTA ends: the last copies are waited for here if the other warps gave up)
            if (!ok)
                for (int i = max(0, issued - p.stages); i < issued; ++i) ops_wait(b_full + 8u * (i % p.stages), (uint32_t)(i / p.stages) & 1u, kMxWait);
        }
        __syncwarp();
    } else if (warp == 1) {
        // ---- MMA issue: the whole warp walks the loop, one elected lane issues ----
        const uint32_t leader = tc_elect();
        // D = fp32; A, B = E2M1, K-major; scales E8M0 (bit 23); scale bytes 0, 1 of a column's four, or (| kUpper) 2, 3
        const uint32_t idesc = (1u << 7) | (1u << 10) | ((uint32_t)(NB / 8) << 17) | (1u << 23) | (8u << 24);
        const uint32_t kUpper = (2u << 4) | (2u << 29);
        if (FUSE) {
            ok = ops_wait_warp(b_x, 0, kMxWait, dead, true);
            tc_fence_after();
        }
        int s = 0;
        uint32_t par = 0;
        for (int t = t0; t < t1 && ok; ++t) {
            ok = ops_wait_warp(b_full + 8u * s, par, kMxWait, dead, true);
            if (!ok) break;
            tc_fence_after();
            const uint32_t a = smem_u32(ring + (size_t)s * S::kStage);
            const uint32_t x = FUSE ? smem_u32(xs + (size_t)(t - t0) * S::kXTile) : a + kMxTile;
            const uint32_t sf = tm + NB + (uint32_t)((t - t0) & 1) * S::kSfCols;   // (the other half may still be read)
            const uint64_t sa = mx4_desc(a, 128, 0), sx = mx4_desc(x, 128, 0);
#pragma unroll
            for (uint32_t h = 0; h < 2; ++h) {
                mx4_copy_scales(leader, sf + 4u * h, sa + 32u * h);
                mx4_copy_scales(leader, sf + 8u + 4u * h, sx + 32u * h);
            }
            const uint64_t da = mx4_desc(a + kMxScales, 1024, 2), db = mx4_desc(x + kMxScales, 1024, 2);
#pragma unroll
            for (uint32_t j = 0; j < 4; ++j)
                mx4_mma(leader, tm, da + 2u * j, db + 2u * j, idesc | ((j & 1u) ? kUpper : 0u), sf + 4u * (j >> 1),
                        sf + 8u + 4u * (j >> 1), t > t0 || j > 0);
            tc_commit(leader, b_empty + 8u * s);
            if (++s == p.stages) { s = 0; par ^= 1u; }
        }
        if (!ok) *dead = 1;
        tc_commit(leader, b_done);
        __syncwarp();
    } else {
        const int w = warp - 2;
        asm volatile("griddepcontrol.wait;" ::: "memory");
        if (FUSE) {
            if (p.x_type == kF16) mx4_quantize_slice<__half, NB>(p, xs, t0, t1, w, 4, lane);
            else if (p.x_type == kBF16) mx4_quantize_slice<__nv_bfloat16, NB>(p, xs, t0, t1, w, 4, lane);
            else mx4_quantize_slice<float, NB>(p, xs, t0, t1, w, 4, lane);
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0) mbar_arrive(b_x);
        }
        ok = ops_wait_warp(b_done, 0, 4 * kMxWait, dead);
        tc_fence_after();
        const uint32_t quarter = (uint32_t)(warp & 3);
        const int row = 32 * (int)quarter + lane;
        // (the ring is free: all copies have landed and have been read)
        if (p.split > 1) {
            float* part = reinterpret_cast<float*>(ring);
            if (ok)
#pragma unroll 1
                for (int c = 0; c < nn; c += 16) {
                    uint32_t r[16];
                    tc_ld16(tm + (quarter << 21) + (uint32_t)c, r);
#pragma unroll
                    for (int i = 0; i < 16; ++i) part[(c + i) * 128 + row] = __uint_as_float(r[i]);
                }
        } else if (!*dead) {   // (*dead is set before the sums are announced, or never)
            if (p.y_type == kF32) mx4_write_tile<float>(p, tm, (int)quarter, lane, 128 * (int64_t)mt, n0, nn, ring);
            else if (p.y_type == kF16) mx4_write_tile<__half>(p, tm, (int)quarter, lane, 128 * (int64_t)mt, n0, nn, ring);
            else mx4_write_tile<__nv_bfloat16>(p, tm, (int)quarter, lane, 128 * (int64_t)mt, n0, nn, ring);
        }
        tc_fence_before();
    }
    if (!ok && lane == 0) {
        *dead = 1;
        atomicExch(p.err, kErrTimeout);
    }
    __syncthreads();
    tc_fence_after();
    if (warp == 1) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tm), "n"(S::kCols));
    if (p.split > 1) {
        asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
        // each rank adds the sums of a share of the tile's (token, four rows), four ranks' at a time on their way
        const int total = nn * 32, per = (total + p.split - 1) / p.split, lo = min(total, rank * per), hi = min(total, lo + per);
        const uint32_t part = smem_u32(ring);
        for (int i = lo + (int)threadIdx.x; i < hi; i += 192) {
            float v[4] = {0.f, 0.f, 0.f, 0.f};
            for (int r0 = 0; r0 < p.split; r0 += 4) {
                float4 x[4];
#pragma unroll
                for (int r = 0; r < 4; ++r) x[r] = r0 + r < p.split ? ld_cluster_f32x4(part + 16u * i, (uint32_t)(r0 + r)) : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
                for (int r = 0; r < 4; ++r) { v[0] += x[r].x; v[1] += x[r].y; v[2] += x[r].z; v[3] += x[r].w; }
            }
            mx4_store4(p, n0 + (i >> 5), 128 * (int64_t)mt + 4 * (i & 31), v);
        }
        asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
    }
}

// ---- the product of many tokens -------------------------------------------------------------------------------------------
// Pairs of blocks (a cluster of two SMs, cta_group::2) walk over tiles of 256 weight rows x 256 tokens, all tokens of the rows in turn: X
// stays in L2, W is read about once. Each block has 128 of the rows, and loads half of the tokens for both: 35 KB a block and 256
// columns, 52 KB for a block that works alone (4096 x 28672 x 8192, the tokens' quantisation included, on a GPU that was idle before: 384 to 410 us =
// 5.0 to 4.7 PFLOP/s, 445 alone; call after call 453 under the power cap, below;
// K = 28672, M = 8192: 445 and 478).
// Copies run ahead over the tiles' ends, and the sums of a tile leave tensor memory for shared memory, rounded, before the next
// tile's products begin (half of the tokens at a time); they are stored while those run. What bounds it is the way from L2 to the SMs
// (a block alone takes 307 us without its copies and 390 with a quarter of its products) and, call after call, the power cap: 991 W at 1620 of
// 1965 MHz. W in two copies a stage: 3 % slower. 4, 5, 6 stages: 415, 406, 413 us.
// The first block of a pair issues for both: it learns from the second's idle MMA warp that its stage is full, and tells both when a
// stage has been read and when a tile is done.
struct Mx4Pair {
    static constexpr int kStage = kMxTile + 2 * kMxScales + kMxCodes;            // W: scales, codes; X: scales of 256 tokens, codes of 128
    static constexpr int kStages = 5, kOut = 128 * (128 * 2 + 16);               // bytes of half a block's sums, 16 bits each (or a quarter's in 32)
    static constexpr int kSmem = 1024 + kStages * kStage + kOut;
    static constexpr int kSfCols = 24;                                           // tensor-memory columns of a stage's scales
    static_assert(kSmem <= 226 * 1024 && 64 * (128 * 4 + 16) <= kOut && 256 + 2 * kSfCols <= 512, "shared and tensor memory");
};

__device__ __forceinline__ uint32_t cluster_addr(uint32_t local, uint32_t rank)
{
    uint32_t a;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(local), "r"(rank));
    return a;
}
// (Relaxed: no thread's writes are handed over, only copies whose end was seen and tensor memory whose reads have ended. A release of
// cluster scope waits for all that the SM has under way, and took 630 us in place of 400 for 4096 x 28672 x 8192.)
__device__ __forceinline__ void mbar_arrive_cluster(uint32_t bar)
{
    asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
// Bounded wait of a warp for arrivals from the other block.
__device__ __forceinline__ bool ops_wait_cluster(uint32_t bar, uint32_t parity, volatile uint32_t* dead)
{
    const uint64_t t0 = global_timer_ns();
#pragma unroll 1
    for (uint32_t it = 0; it < (1u << 24); ++it) {
        uint32_t ok;
        asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
                     : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
        if (__all_sync(0xffffffffu, ok)) return true;
        if ((it & 255u) == 255u && __any_sync(0xffffffffu, *dead || ((global_timer_ns() - t0) >> 10) > kMxWait)) break;
    }
    return false;
}
__device__ __forceinline__ void pair_commit(uint32_t elected, uint32_t bar, uint16_t blocks)
{
    asm volatile("{\n\t.reg .pred q;\n\tsetp.ne.u32 q, %2, 0;\n\t"
                 "@q tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;\n\t}" ::"r"(bar), "h"(blocks), "r"(elected) : "memory");
}
__device__ __forceinline__ void pair_mma(uint32_t elected, uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t sfa, uint32_t sfb, uint32_t accumulate)
{
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 q, %7, 0;\n\tsetp.ne.u32 p, %6, 0;\n\t"
                 "@q tcgen05.mma.cta_group::2.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
                 ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(sfa), "r"(sfb), "r"(accumulate), "r"(elected) : "memory");
}
__device__ __forceinline__ void pair_copy_scales(uint32_t elected, uint32_t d, uint64_t s)   // (in both blocks, each from its own shared memory)
{
    asm volatile("{\n\t.reg .pred q;\n\tsetp.ne.u32 q, %2, 0;\n\t@q tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;\n\t}"
                 ::"r"(d), "l"(s), "r"(elected) : "memory");
}

// A block's sums (four warps) to shared memory and out; free_bar: the pair's first block's barrier, told when they are out of tensor memory.
template <class T>
__device__ __forceinline__ void mx4_pair_store(const Mx4Params& p, uint32_t tm, int quarter, int lane, int64_t m0, int64_t n0, int nn, uint8_t* stage, uint32_t free_bar)
{
    constexpr int PITCH = 128 * (int)sizeof(T) + 16, PER = 16 / (int)sizeof(T), ROW = 128 / PER, PASS = 256 / (int)sizeof(T);
    const int row = 32 * quarter + lane, m_here = (int)max((int64_t)0, min((int64_t)128, p.M - m0));   // (0: the pair's rows end with its first block)
#pragma unroll 1
    for (int c0 = 0; c0 < nn; c0 += PASS) {
        const int cols = min(PASS, nn - c0);
        bar_epilogue();   // (what was here has been stored)
#pragma unroll 1
        for (int c = 0; c < cols; c += 32) {
            uint32_t r[32];
            tc_ld32(tm + ((uint32_t)quarter << 21) + (uint32_t)(c0 + c), r);
            tc_wait_ld();
            pin32(r);
#pragma unroll
            for (int i = 0; i < 32; ++i) *reinterpret_cast<T*>(stage + (c + i) * PITCH + row * sizeof(T)) = from_f32<T>(__uint_as_float(r[i]));
        }
        if (c0 + PASS >= nn) {
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_cluster(free_bar);
        }
        bar_epilogue();
        if (p.y_vec && m_here == 128) {
#pragma unroll 4
            for (int i = row; i < cols * ROW; i += 128) {
                const int n = i / ROW, piece = i % ROW;
                *reinterpret_cast<uint4*>(static_cast<T*>(p.Y) + (n0 + c0 + n) * p.ldy + m0 + piece * PER) = *reinterpret_cast<const uint4*>(stage + n * PITCH + 16 * piece);
            }
        } else {
            for (int n = 0; n < cols; ++n)
                if (row < m_here) static_cast<T*>(p.Y)[(n0 + c0 + n) * p.ldy + m0 + row] = *reinterpret_cast<const T*>(stage + n * PITCH + row * sizeof(T));
        }
    }
}

template <int ST>   // ring stages
__global__ void __launch_bounds__(192, 1) us_mx4_pair_kernel(const __grid_constant__ Mx4Params p)
{
    using S = Mx4Pair;
    constexpr int NB = 256;
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    __shared__ __align__(8) uint64_t bars[3 * ST + 3];
    __shared__ uint32_t misc[2];
    uint8_t* ring = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
    uint8_t* out = ring + ST * S::kStage;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t b_full = smem_u32(bars), b_other = b_full + 8u * ST, b_empty = b_other + 8u * ST, b_done = b_empty + 8u * ST, b_free = b_done + 8u, b_end = b_free + 8u;
    volatile uint32_t* dead = misc + 1;
    const int rank = (int)(blockIdx.x & 1u), row_tiles = (int)mx4_tiles(p.M, 128);
    if (warp == 1) {
        if (lane < ST) { mbar_init(b_full + 8u * lane, 1); mbar_init(b_other + 8u * lane, 1); mbar_init(b_empty + 8u * lane, 1); }
        if (lane == 0) { mbar_init(b_done, 1); mbar_init(b_free, 8); mbar_init(b_end, 1); misc[1] = 0; }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        __syncwarp();
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(misc)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
    tc_fence_after();
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");   // (after the allocation, as above)
    const uint32_t tm = *(volatile uint32_t*)misc;
    bool ok = true;
    if (warp == 0) {
        // ---- copies ----
        if (lane == 0) {
            asm volatile("griddepcontrol.wait;" ::: "memory");
            uint32_t count = 0;   // stages filled
            for (int tile = blockIdx.x >> 1; tile < p.tiles && ok; tile += gridDim.x >> 1) {
                const int pair = tile / p.col_tiles, n0 = (tile - pair * p.col_tiles) * NB, nn = min(NB, p.N - n0);
                const int mt = min(2 * pair + rank, row_tiles - 1);   // (past the last row tile: its products are not stored)
                const int rows = max(0, min(128, (nn - 128 * rank + 7) & ~7));   // this block's tokens, in whole 8-row groups
                const bool two = nn > 128;
                const uint32_t bytes = (uint32_t)(kMxTile + kMxScales + (two ? kMxScales : 0) + 128 * rows);
                const uint8_t* w = p.w + (int64_t)mt * p.kt * kMxTile;
                const uint8_t* x0 = p.x + (int64_t)(n0 >> 7) * p.kt * kMxTile;
                const uint8_t* x1 = x0 + (int64_t)p.kt * kMxTile;
                const uint8_t* xc = (rank ? x1 : x0) + kMxScales;
                for (int t = 0; t < p.kt; ++t, ++count) {
                    const uint32_t s = count % ST;
                    if (count >= ST && !ops_wait(b_empty + 8u * s, (count / ST - 1u) & 1u, kMxWait)) { ok = false; break; }
                    const uint32_t b = b_full + 8u * s, d = smem_u32(ring + s * S::kStage);
                    mbar_expect_tx(b, bytes);
                    bulk_g2s(d, w + (int64_t)t * kMxTile, kMxTile, b);
                    bulk_g2s(d + kMxTile, x0 + (int64_t)t * kMxTile, kMxScales, b);
                    if (two) bulk_g2s(d + kMxTile + kMxScales, x1 + (int64_t)t * kMxTile, kMxScales, b);
                    if (rows) bulk_g2s(d + kMxTile + 2 * kMxScales, xc + (int64_t)t * kMxTile, 128u * rows, b);
                }
            }
            // (nothing may be in flight when the block ends: no copies into it, and no word from the first block that a stage has been read)
            for (uint32_t c = count > ST ? count - ST : 0; c < count; ++c) ops_wait((ok ? b_empty : b_full) + 8u * (c % ST), (c / ST) & 1u, kMxWait);
        }
        __syncwarp();
    } else if (warp == 1 && rank == 0) {
        // ---- MMA issue, for both blocks ----
        const uint32_t leader = tc_elect();
        const uint32_t idesc = (1u << 7) | (1u << 10) | ((uint32_t)(NB / 8) << 17) | (1u << 23) | (16u << 24);   // M = 256
        const uint32_t kUpper = (2u << 4) | (2u << 29);
        uint32_t count = 0, n = 0, s = 0, par = 0;
        for (int tile = blockIdx.x >> 1; tile < p.tiles && ok; tile += gridDim.x >> 1, ++n) {
            if (n > 0) ok = ops_wait_cluster(b_free, (n - 1u) & 1u, dead);
            for (int t = 0; t < p.kt && ok; ++t, ++count) {
                ok = ops_wait_warp(b_full + 8u * s, par, kMxWait, dead, true);
                if (ok) ok = ops_wait_cluster(b_other + 8u * s, par, dead);
                if (!ok) break;
                tc_fence_after();
                const uint32_t a = smem_u32(ring + s * S::kStage), x = a + kMxTile, sf = tm + NB + (count & 1u) * S::kSfCols;
                const uint64_t sa = mx4_desc(a, 128, 0), sx = mx4_desc(x, 128, 0);
#pragma unroll
                for (uint32_t h = 0; h < 2; ++h) {
                    pair_copy_scales(leader, sf + 4u * h, sa + 32u * h);
#pragma unroll
                    for (uint32_t g = 0; g < 2; ++g) pair_copy_scales(leader, sf + 8u + 4u * (2u * h + g), sx + 32u * h + (kMxScales / 16) * g);
                }
                const uint64_t da = mx4_desc(a + kMxScales, 1024, 2), db = mx4_desc(x + 2 * kMxScales, 1024, 2);
#pragma unroll
                for (uint32_t j = 0; j < 4; ++j)
                    pair_mma(leader, tm, da + 2u * j, db + 2u * j, idesc | ((j & 1u) ? kUpper : 0u), sf + 4u * (j >> 1), sf + 8u + 8u * (j >> 1), t > 0 || j > 0);
                pair_commit(leader, b_empty + 8u * s, 3);
                if (++s == ST) { s = 0; par ^= 1u; }
            }
            if (ok) pair_commit(leader, b_done, 3);
        }
        if (!ok) *dead = 1;
        pair_commit(leader, b_end, 1);   // nothing is in flight when the tensor memory is given back
        ops_wait(b_end, 0, kMxWait);
        __syncwarp();
    } else if (warp == 1) {
        // ---- the second block's stages are announced to the first ----
        uint32_t s = 0, par = 0;
        const uint32_t first = cluster_addr(b_other, 0);
        for (int tile = blockIdx.x >> 1; tile < p.tiles && ok; tile += gridDim.x >> 1)
            for (int t = 0; t < p.kt && ok; ++t) {
                ok = ops_wait_warp(b_full + 8u * s, par, kMxWait, dead, true);
                if (!ok) break;
                if (lane == 0) mbar_arrive_cluster(first + 8u * s);
                if (++s == ST) { s = 0; par ^= 1u; }
            }
    } else {
        // ---- sums out ----
        const int quarter = warp & 3;
        const uint32_t free_bar = cluster_addr(b_free, 0);
        asm volatile("griddepcontrol.wait;" ::: "memory");
        uint32_t n = 0;
        for (int tile = blockIdx.x >> 1; tile < p.tiles; tile += gridDim.x >> 1, ++n) {
            ok = ops_wait_warp(b_done, n & 1u, 4 * kMxWait, dead);
            if (bar_any(!ok)) {   // (all four warps leave at the same place)
                ok = false;
                break;
            }
            tc_fence_after();
            const int pair = tile / p.col_tiles, n0 = (tile - pair * p.col_tiles) * NB, nn = min(NB, p.N - n0);
            const int64_t m0 = 128 * (int64_t)(2 * pair + rank);
            if (p.y_type == kF32) mx4_pair_store<float>(p, tm, quarter, lane, m0, n0, nn, out, free_bar);
            else if (p.y_type == kF16) mx4_pair_store<__half>(p, tm, quarter, lane, m0, n0, nn, out, free_bar);
            else mx4_pair_store<__nv_bfloat16>(p, tm, quarter, lane, m0, n0, nn, out, free_bar);
        }
    }
    if (!ok && lane == 0) {
        *dead = 1;
        atomicExch(p.err, kErrTimeout);
    }
    tc_fence_before();
    __syncthreads();
    // (neither block ends while the other may still reach its barriers or operands)
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
    tc_fence_after();
    if (warp == 1) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, 512;" ::"r"(tm));
}

}  // namespace us
