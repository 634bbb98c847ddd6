// MX4 entry points: checks, launch plans.
#include "us_mx4.cuh"
#include "us_ops.h"

namespace us {
namespace {

__device__ uint32_t g_mx4_err;   // whether a bounded wait has run out since us_mx4_last_error was asked

struct Plan {
    const void* kernel;
    int nb, split, col_tiles, stages, cluster;
    int64_t smem, tiles, blocks;
    bool fuse;
};

template <int NB, bool FUSE>
void shape(Plan* p, int64_t slice_tiles, int64_t budget)
{
    using S = Mx4Shape<NB, FUSE>;
    p->kernel = (const void*)us_mx4_product_kernel<NB, FUSE>;
    const int64_t xs = FUSE ? slice_tiles * S::kXTile : 0;
    // (the split's partial sums, 128 x NB fp32, take the ring's place; else two buffers of 32 tokens on their way out)
    const int64_t least = ((p->split > 1 ? 128 * 4 * NB : 2 * 32 * (512 + 16)) + S::kStage - 1) / S::kStage;
    p->stages = (int)std::max(least, std::min({(int64_t)S::kMaxStages, slice_tiles, (budget - 1024 - xs) / S::kStage}));
    p->smem = 1024 + xs + (int64_t)p->stages * S::kStage;
}

constexpr int64_t kHalfSm = 112 * 1024, kWholeSm = 226 * 1024;   // shared memory of a CTA with and without room for a second one

// How a product of N tokens is cut. can_fuse: the activations are rows in 16 or 32 bits.
Plan plan(int64_t N, int64_t M, int64_t K, bool can_fuse, int sms)
{
    Plan p = {};
    const int64_t kt = mx4_tiles(K, 256), rt = mx4_tiles(M, 128);
    p.nb = N <= 16 ? 16 : N <= 32 ? 32 : N <= 64 ? 64 : N <= 128 ? 128 : 256;
    // (half as many columns a CTA where the tiles would not fill the GPU, or where tokens that are not there would be more than an eighth of
    // the work. 28672 x 8192 in tiles of 256, of 128: 256 tokens 38.2, 41.0 us, 300: 63.1, 55.1, 512: 67.0, 74.7)
    if (p.nb == 256 && (rt * mx4_tiles(N, 256) < sms || 8 * mx4_tiles(N, 256) * 2 > 9 * mx4_tiles(N, 128))) p.nb = 128;
    p.col_tiles = (int)mx4_tiles(N, p.nb);
    p.tiles = rt * p.col_tiles;
    // The columns are split while that fills SMs and leaves every CTA four tiles of them (16 where the sums to exchange are 64 KB). 4096 x
    // 4096 and one token: 7.3 us whole, 5.7, 4.6, 5.0, 9.6 us in 2, 4, 8, 16; 128 tokens: 8.7, 11.0, 9.4 us whole, in 2, 4.
    const int64_t most = p.nb <= 64 ? 2 * sms : sms, least = p.nb <= 64 ? 4 : 16;
    p.split = 1;
    if (p.nb <= 128)
        while (p.split < 16 && p.tiles * p.split * 2 <= most && least * p.split * 2 <= kt) p.split *= 2;
    const int64_t slice = mx4_tiles(kt, p.split);
    // A CTA quantises its activations itself where that is one trip to memory for its four warps (four tiles of a token each); beyond, every
    // CTA's own copy of the work takes longer than a launch for all (11008 x 4096, 8 tokens: 11.2 us against 6.9).
    p.fuse = can_fuse && p.nb == 16 && slice * N <= 16;
    if (p.fuse) shape<16, true>(&p, slice, kHalfSm);
    else if (p.nb == 16) shape<16, false>(&p, slice, kHalfSm);
    else if (p.nb == 32) shape<32, false>(&p, slice, kHalfSm);
    else if (p.nb == 64) shape<64, false>(&p, slice, kHalfSm);
    else if (p.nb == 128) shape<128, false>(&p, slice, p.tiles * p.split > sms ? kHalfSm : kWholeSm);
    p.blocks = p.tiles * p.split;
    p.cluster = p.split;
    if (p.nb == 256) {   // pairs of blocks that walk over pairs of tiles
        p.kernel = (const void*)us_mx4_pair_kernel<Mx4Pair::kStages>;
        p.smem = Mx4Pair::kSmem;
        p.tiles = mx4_tiles(rt, 2) * p.col_tiles;
        p.blocks = 2 * std::min<int64_t>(p.tiles, sms / 2);
        p.cluster = 2;
    }
    return p;
}

bool type_ok(int32_t t) { return t >= 0 && t <= 2; }
int64_t size_of(int32_t t) { return t == US_F32 ? 4 : 2; }
bool aligned(const void* p, int64_t b) { return reinterpret_cast<uintptr_t>(p) % (uintptr_t)b == 0; }
bool rows_vec(const void* p, int64_t ld, int64_t size) { return aligned(p, 16) && ld * size % 16 == 0; }
// Bytes of an access to rows: 32, 16, 8, 4, or 1 (an element at a time).
int access(const void* p, int64_t ld, int64_t size)
{
    for (int b = 32; b >= 4; b /= 2)
        if (aligned(p, b) && ld * size % b == 0) return b;
    return 1;
}
us_status cuda(cudaError_t e)
{
    if (e == cudaSuccess) return US_OK;
    cudaGetLastError();
    return US_ERR_CUDA;
}
// Grid of the kernels that give a warp to each of `warps` pieces of work, 8 warps a block.
dim3 warps_grid(int64_t warps) { return dim3((unsigned)std::max<int64_t>(1, std::min<int64_t>((warps + 7) / 8, 148 * 16))); }

// Rows and columns that every index of the kernels holds: a matrix of at most 2^31 rows and 2^30 columns.
bool shape_ok(int64_t rows, int64_t K) { return rows >= 0 && rows < (1ll << 31) && K >= 1 && K <= (1ll << 30); }

us_status product(const void* X, int32_t x_type, int64_t ldx, const void* x_mx, int64_t N, const void* w_mx, int64_t M, int64_t K, void* Y,
                  int32_t y_type, int64_t ldy, const Plan& pl, uint32_t flags, cudaStream_t st)
{
    static void* kept[kMaxDevices];
    void* err = nullptr;
    if (ops_symbol(kept, &g_mx4_err, &err) != cudaSuccess) { cudaGetLastError(); return US_ERR_CUDA; }
    Mx4Params p = {};
    p.w = static_cast<const uint8_t*>(w_mx);
    p.x = static_cast<const uint8_t*>(x_mx);
    p.X = X;
    p.Y = Y;
    p.ldx = ldx; p.ldy = ldy;
    p.M = (int32_t)M; p.N = (int32_t)N; p.K = (int32_t)K; p.kt = (int32_t)mx4_tiles(K, 256);
    p.split = pl.split; p.col_tiles = pl.col_tiles; p.tiles = (int32_t)pl.tiles; p.stages = pl.stages;
    p.x_type = x_type; p.y_type = y_type;
    p.x_vec = X && rows_vec(X, ldx, size_of(x_type));
    p.y_vec = rows_vec(Y, N > 1 ? ldy : 0, size_of(y_type));
    p.w_stable = (flags & US_MX4_W_STABLE) != 0;
    p.err = static_cast<uint32_t*>(err);
    const cudaError_t e = ops_kernel_allow(pl.kernel, (int)kWholeSm);
    if (e != cudaSuccess) return cuda(e);
    void* args[] = {&p};
    return cuda(ops_launch(pl.kernel, dim3((unsigned)pl.blocks), 192, pl.smem, st, args, (unsigned)pl.cluster));
}

}  // namespace
}  // namespace us

using namespace us;

int64_t us_mx4_bytes(int64_t rows, int64_t K)
{
    if (!shape_ok(rows, K)) return -1;
    return mx4_tiles(rows, 128) * mx4_tiles(K, 256) * kMxTile;
}

us_status us_mx4_quantize(const void* X, int32_t x_type, int64_t ldx, int64_t rows, int64_t K, void* mx, void* stream)
{
    if (!type_ok(x_type) || !shape_ok(rows, K)) return US_ERR_INVALID_ARG;
    if (rows == 0) return US_OK;
    if (!X || !mx || (rows > 1 && ldx < K) || !aligned(X, size_of(x_type)) || !aligned(mx, 16)) return US_ERR_INVALID_ARG;
    if (rows == 1) ldx = 0;   // (a single row's stride means nothing)
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    uint8_t* out = static_cast<uint8_t*>(mx);
    int vec = access(X, ldx, size_of(x_type));
    const dim3 g = warps_grid(rows * mx4_tiles(mx4_tiles(K, 256), 2 * kMxUnroll));
    const void* k = x_type == US_F16 ? (const void*)us_mx4_quantize_kernel<__half> :
                    x_type == US_BF16 ? (const void*)us_mx4_quantize_kernel<__nv_bfloat16> : (const void*)us_mx4_quantize_kernel<float>;
    void* args[] = {&X, &ldx, &rows, &K, &out, &vec};
    return cuda(ops_launch(k, g, 256, 0, st, args));
}

us_status us_mx4_dequantize(const void* mx, int64_t rows, int64_t K, void* out, int32_t type, int64_t ldo, void* stream)
{
    if (!type_ok(type) || !shape_ok(rows, K)) return US_ERR_INVALID_ARG;
    if (rows == 0) return US_OK;
    if (!mx || !out || (rows > 1 && ldo < K) || !aligned(out, size_of(type)) || !aligned(mx, 16)) return US_ERR_INVALID_ARG;
    if (rows == 1) ldo = 0;
    int vec = access(out, ldo, size_of(type));
    const dim3 g = warps_grid(rows * mx4_tiles(mx4_tiles(K, 256), 2 * kMxUnroll));
    const void* k = type == US_F16 ? (const void*)us_mx4_dequantize_kernel<__half> :
                    type == US_BF16 ? (const void*)us_mx4_dequantize_kernel<__nv_bfloat16> : (const void*)us_mx4_dequantize_kernel<float>;
    void* args[] = {&mx, &rows, &K, &out, &ldo, &vec};
    return cuda(ops_launch(k, g, 256, 0, static_cast<cudaStream_t>(stream), args));
}

static us_status repack(bool pack, void* codes, int64_t ldc, void* scales, int64_t lds, int64_t rows, int64_t K, void* mx, void* stream)
{
    if (!shape_ok(rows, K)) return US_ERR_INVALID_ARG;
    if (rows == 0) return US_OK;
    if (!codes || !scales || !mx || !aligned(mx, 16) || (rows > 1 && (ldc < (K + 1) / 2 || lds < (K + 31) / 32))) return US_ERR_INVALID_ARG;
    const void* k = pack ? (const void*)us_mx4_repack_kernel<true> : (const void*)us_mx4_repack_kernel<false>;
    void* args[] = {&codes, &ldc, &scales, &lds, &rows, &K, &mx};
    return cuda(ops_launch(k, warps_grid(rows * mx4_tiles(K, 256)), 256, 0, static_cast<cudaStream_t>(stream), args));
}
us_status us_mx4_pack(const void* codes, int64_t ldc, const void* scales, int64_t lds, int64_t rows, int64_t K, void* mx, void* stream)
{
    return repack(true, const_cast<void*>(codes), ldc, const_cast<void*>(scales), lds, rows, K, mx, stream);
}
us_status us_mx4_unpack(const void* mx, int64_t rows, int64_t K, void* codes, int64_t ldc, void* scales, int64_t lds, void* stream)
{
    return repack(false, codes, ldc, scales, lds, rows, K, const_cast<void*>(mx), stream);
}

static bool product_ok(int64_t N, const void* w_mx, int64_t M, int64_t K, const void* Y, int32_t y_type, int64_t ldy)
{
    return shape_ok(N, K) && shape_ok(M, K) && M >= 1 && type_ok(y_type) &&
           (N == 0 || (w_mx && aligned(w_mx, 16) && Y && aligned(Y, size_of(y_type)) && (N == 1 || ldy >= M))) &&
           us::mx4_tiles(M, 128) * us::mx4_tiles(N, 16) * 16 < (1ll << 31);
}

us_status us_mx4_matmul(const void* x_mx, int64_t N, const void* w_mx, int64_t M, int64_t K, void* Y, int32_t y_type, int64_t ldy, uint32_t flags, void* stream)
{
    if (!product_ok(N, w_mx, M, K, Y, y_type, ldy) || (N && (!x_mx || !aligned(x_mx, 16)))) return US_ERR_INVALID_ARG;
    if (N == 0) return US_OK;
    return product(nullptr, 0, 0, x_mx, N, w_mx, M, K, Y, y_type, ldy, plan(N, M, K, false, ops_sms()), flags, static_cast<cudaStream_t>(stream));
}

int64_t us_mx4_linear_scratch(int64_t N, int64_t M, int64_t K)
{
    if (!shape_ok(N, K) || !shape_ok(M, K) || M < 1) return -1;
    return N == 0 || plan(N, M, K, true, ops_sms()).fuse ? 0 : us_mx4_bytes(N, K);
}

us_status us_mx4_linear(const void* X, int32_t x_type, int64_t ldx, int64_t N, const void* w_mx, int64_t M, int64_t K, void* Y, int32_t y_type,
                        int64_t ldy, void* scratch, int64_t scratch_bytes, uint32_t flags, void* stream)
{
    if (!type_ok(x_type) || !product_ok(N, w_mx, M, K, Y, y_type, ldy)) return US_ERR_INVALID_ARG;
    if (N == 0) return US_OK;
    if (!X || !aligned(X, size_of(x_type)) || (N > 1 && ldx < K)) return US_ERR_INVALID_ARG;
    if (N == 1) ldx = 0;
    const Plan pl = plan(N, M, K, true, ops_sms());
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (pl.fuse) return product(X, x_type, ldx, nullptr, N, w_mx, M, K, Y, y_type, ldy, pl, flags, st);
    if (!scratch || !aligned(scratch, 16) || scratch_bytes < us_mx4_bytes(N, K)) return US_ERR_SCRATCH_TOO_SMALL;
    const us_status s = us_mx4_quantize(X, x_type, ldx, N, K, scratch, stream);
    if (s != US_OK) return s;
    return product(nullptr, 0, 0, scratch, N, w_mx, M, K, Y, y_type, ldy, pl, flags, st);
}

us_status us_mx4_last_error(void)
{
    uint32_t flag = 0;
    const uint32_t zero = 0;
    cudaError_t e = cudaDeviceSynchronize();
    if (e == cudaSuccess) e = cudaMemcpyFromSymbol(&flag, g_mx4_err, 4);
    if (e == cudaSuccess && flag) e = cudaMemcpyToSymbol(g_mx4_err, &zero, 4);
    if (e != cudaSuccess) return cuda(e);
    return flag ? US_ERR_DEVICE_TIMEOUT : US_OK;
}
