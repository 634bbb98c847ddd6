// The 8-bit cache's entry points: checks, launch plans.
#include "us_kv_prompt.cuh"
#include "us_ops.h"

#include <cmath>
#include <mutex>
#include <new>

namespace us {
namespace {

__device__ uint32_t g_kv_err;   // the last failure that a kernel met since us_kv_last_error was asked

us_status cuda(cudaError_t e)
{
    if (e == cudaSuccess) return US_OK;
    cudaGetLastError();
    return US_ERR_CUDA;
}
bool aligned(const void* p, int64_t b) { return reinterpret_cast<uintptr_t>(p) % (uintptr_t)b == 0; }
int64_t size_of(int32_t t) { return t == US_F32 ? 4 : 2; }

using EncodeTiled = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                 const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
EncodeTiled encode_tiled()
{
    static const EncodeTiled f = [] {
        void* p = nullptr;
        cudaDriverEntryPointQueryResult r;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &r) != cudaSuccess) cudaGetLastError();
        return reinterpret_cast<EncodeTiled>(p);
    }();
    return f;
}

}  // namespace
}  // namespace us

struct us_kv {
    us::KvPool pool{};
    int device = -1;      // that the pool lies on; -1: not known (no driver, or memory that is not one device's)
    std::mutex lock;      // of the maps: made by the first attention call
    bool mapped = false;
    CUtensorMap k_map, v_map;
};

namespace us {
namespace {

us_status error_word(uint32_t** err)
{
    static void* kept[kMaxDevices];
    return cuda(ops_symbol(kept, &g_kv_err, reinterpret_cast<void**>(err)));
}

// The codes as rows of D bytes; a copy brings a block's tokens, 64 at most, swizzled over a row's 128 (64) bytes.
bool encode_map(CUtensorMap* map, void* base, const KvPool& p)
{
    if (!encode_tiled()) return false;
    const cuuint64_t dims[2] = {(cuuint64_t)p.D, (cuuint64_t)p.blocks * p.Hkv * p.T}, strides[1] = {(cuuint64_t)p.D};
    const cuuint32_t box[2] = {(cuuint32_t)p.D, (cuuint32_t)std::min(p.T, kKvTile)}, step[2] = {1, 1};
    return encode_tiled()(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, base, dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
                          p.D == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                          CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

bool maps(us_kv* h)
{
    std::lock_guard<std::mutex> hold(h->lock);
    if (!h->mapped) h->mapped = encode_map(&h->k_map, h->pool.k, h->pool) && encode_map(&h->v_map, h->pool.v, h->pool);
    return h->mapped;
}

// The device that an address lies on, or -1.
int device_of(const void* p)
{
    cudaPointerAttributes a = {};
    if (cudaPointerGetAttributes(&a, p) != cudaSuccess) cudaGetLastError();
    else if (a.type == cudaMemoryTypeDevice) return a.device;
    return -1;
}
// Whether the current device is the pool's: every call that launches asks.
us_status on_device(const us_kv* h)
{
    if (h->device < 0) return US_OK;
    int dev = -1;
    const us_status s = cuda(cudaGetDevice(&dev));
    return s != US_OK ? s : dev == h->device ? US_OK : US_ERR_INVALID_ARG;
}

bool seqs_ok(const us_kv* h, const us_kv_seqs* q, int64_t N)
{
    if (!h || !q || N < 0 || N >= (1ll << 31) || q->n_seqs < 0 || (!q->cu_tokens && N != q->n_seqs)) return false;
    if (q->n_seqs == 0 || N == 0) return true;
    return q->block_table && q->lengths && q->table_width >= 1 && (int64_t)q->table_width * h->pool.T < (1ll << 31) - (1 << 16) &&
           (q->n_seqs == 1 || q->table_stride >= q->table_width) && aligned(q->block_table, 4) && aligned(q->lengths, 4) && aligned(q->cu_tokens, 4);
}
KvSeqs seqs(const us_kv_seqs* q, int64_t N)
{
    KvSeqs r = {};
    r.table = q->block_table;
    r.table_stride = q->table_stride;
    r.lengths = q->lengths;
    r.cu = q->cu_tokens;
    r.S = q->n_seqs;
    r.width = q->table_width;
    r.N = N;
    return r;
}
// Rows (token, head, D): every stride holds a row, and the 16-byte path's condition.
bool strides_ok(const void* x, int32_t type, int64_t token, int64_t head, int64_t N, int64_t heads, int32_t D)
{
    return x && aligned(x, size_of(type)) && (N == 1 || token >= D) && (heads == 1 || head >= D) && token >= 0 && head >= 0;
}
bool rows_vec(const void* x, int32_t type, int64_t token, int64_t head)
{
    return aligned(x, 16) && token * size_of(type) % 16 == 0 && head * size_of(type) % 16 == 0;
}

template <class T>
const void* append_kernel(int team)
{
    return team == 32 ? (const void*)us_kv_append_kernel<T, 32> : team == 64 ? (const void*)us_kv_append_kernel<T, 64> : (const void*)us_kv_append_kernel<T, 128>;
}

// ---- attention: which kernels ----
struct AttendPlan {
    const void *kernel, *join;
    int rows, stages, smem, ctas;
    int splits;        // (prompts) of the cache's length
    int64_t tiles;     // (prompts) row tiles, at most; 0: the kernel for few rows
    int64_t scratch;
};
template <int D, bool BF16>
AttendPlan prompt_shape(int64_t N, int64_t S, int64_t G, int64_t Hkv, int64_t longest, int sms)
{
    AttendPlan p = {};
    p.kernel = (const void*)us_kv_prompt_kernel<D, BF16>;
    p.join = (const void*)us_kv_prompt_join_kernel<D, BF16>;
    p.smem = PrShape<D>::kSmem;
    p.tiles = N * G / kPrRows + S;
    // a tile's walk over the cache is split where the tiles would leave SMs idle, in parts of at least four units
    const int64_t likely = std::max(S, (N * G + kPrRows - 1) / kPrRows) * Hkv;
    p.splits = (int)std::max<int64_t>(1, std::min<int64_t>({16, sms / likely, longest / (4 * kPrTile)}));
    p.scratch = p.splits > 1 ? p.tiles * Hkv * p.splits * PrShape<D>::kPart * 4 : 0;
    return p;
}
template <int D, int NT, bool BF16>
AttendPlan attend_shape(int sms)
{
    using S = KvShape<D, NT>;
    AttendPlan p = {};
    p.kernel = (const void*)us_kv_attend_kernel<D, NT, BF16>;
    p.join = (const void*)us_kv_join_kernel<D, NT, BF16>;
    p.rows = S::R;
    p.stages = std::min(S::kMaxStages, (111 * 1024 - 1024 - S::kMerge) / S::kStage);   // two CTAs an SM
    p.smem = 1024 + p.stages * S::kStage + S::kMerge;
    p.ctas = 2 * sms;
    p.scratch = (int64_t)p.ctas * 2 * S::kPart * 4;
    return p;
}
template <int D, int NT>
AttendPlan attend_shape(bool bf16, int sms) { return bf16 ? attend_shape<D, NT, true>(sms) : attend_shape<D, NT, false>(sms); }
AttendPlan attend_plan(int D, bool bf16, int64_t N, int64_t S, int64_t G, int64_t Hkv, int64_t longest, int sms)
{
    // Rows a cache head has on average decide. 64 sequences of 4096 tokens, 8 cache heads of 128, bf16, this kernel and the other one: 16 rows 154, 341 us, 32
    // rows 288, 342, 40 rows 414, 343, 128 rows 1082, 349; four sequences of 32768: 32 rows 140, 170, 40 rows 191, 172. (64 of 300: 24 rows 76, 66.)
    if (N * G > 32 * S) {
        if (D == 128) return bf16 ? prompt_shape<128, true>(N, S, G, Hkv, longest, sms) : prompt_shape<128, false>(N, S, G, Hkv, longest, sms);
        return bf16 ? prompt_shape<64, true>(N, S, G, Hkv, longest, sms) : prompt_shape<64, false>(N, S, G, Hkv, longest, sms);
    }
    // rows a cache head has on average: 8 a tile are enough for them, or 16
    const bool few = N * G <= 8 * S;
    if (D == 128) return few ? attend_shape<128, 1>(bf16, sms) : attend_shape<128, 2>(bf16, sms);
    return few ? attend_shape<64, 1>(bf16, sms) : attend_shape<64, 2>(bf16, sms);
}

}  // namespace
}  // namespace us

using namespace us;

us_status us_kv_create(void* k_codes, void* v_codes, void* k_steps, void* v_steps, int64_t n_blocks, int32_t n_kv_heads, int32_t block_tokens,
                       int32_t head_dim, us_kv** out)
{
    if (!out) return US_ERR_INVALID_ARG;
    *out = nullptr;
    if (!k_codes || !v_codes || !k_steps || !v_steps || n_blocks < 1 || n_kv_heads < 1 || n_kv_heads > 65535 || block_tokens < 1 || head_dim < 1)
        return US_ERR_INVALID_ARG;
    if (!aligned(k_codes, 16) || !aligned(v_codes, 16) || !aligned(k_steps, 4) || !aligned(v_steps, 4)) return US_ERR_INVALID_ARG;
    if ((head_dim != 64 && head_dim != 128) || (block_tokens != 16 && block_tokens != 32 && block_tokens != 64 && block_tokens != 128 && block_tokens != 256))
        return US_ERR_UNSUPPORTED;
    if (n_blocks >= (1ll << 31) || n_blocks > ((1ll << 31) - 1) / n_kv_heads / block_tokens) return US_ERR_UNSUPPORTED;
    int device = -1;
    for (const void* p : {(const void*)k_codes, (const void*)v_codes, (const void*)k_steps, (const void*)v_steps}) {
        const int d = device_of(p);
        if (d >= 0 && device >= 0 && d != device) return US_ERR_INVALID_ARG;
        if (d >= 0) device = d;
    }
    us_kv* h = new (std::nothrow) us_kv();
    if (!h) return US_ERR_ALLOC;
    h->device = device;
    h->pool.k = static_cast<int8_t*>(k_codes);
    h->pool.v = static_cast<int8_t*>(v_codes);
    h->pool.k_step = static_cast<float*>(k_steps);
    h->pool.v_step = static_cast<float*>(v_steps);
    h->pool.blocks = (int32_t)n_blocks;
    h->pool.Hkv = n_kv_heads;
    h->pool.T = block_tokens;
    h->pool.D = head_dim;
    *out = h;
    return US_OK;
}

us_status us_kv_destroy(us_kv* h)
{
    delete h;
    return US_OK;
}

us_status us_kv_append(us_kv* h, const us_kv_seqs* q, int64_t N, const void* K, const void* V, int32_t type, int64_t k_token_stride, int64_t k_head_stride,
                       int64_t v_token_stride, int64_t v_head_stride, void* stream)
{
    if (!seqs_ok(h, q, N) || type < 0 || type > 2) return US_ERR_INVALID_ARG;
    if (N == 0 || q->n_seqs == 0) return US_OK;
    if (!strides_ok(K, type, k_token_stride, k_head_stride, N, h->pool.Hkv, h->pool.D) ||
        !strides_ok(V, type, v_token_stride, v_head_stride, N, h->pool.Hkv, h->pool.D)) return US_ERR_INVALID_ARG;
    us_status s = on_device(h);
    if (s != US_OK) return s;
    KvAppend a = {};
    a.pool = h->pool;
    a.seqs = seqs(q, N);
    a.x[0] = K; a.x[1] = V;
    a.token_stride[0] = k_token_stride; a.token_stride[1] = v_token_stride;
    a.head_stride[0] = k_head_stride; a.head_stride[1] = v_head_stride;
    a.vec = rows_vec(K, type, k_token_stride, k_head_stride) && rows_vec(V, type, v_token_stride, v_head_stride);
    s = error_word(&a.pool.err);
    if (s != US_OK) return s;
    // blocks that get tokens: at most n / T + 2 of a sequence with n new tokens, and n
    const int64_t most = std::min(N, N / h->pool.T + 2 * (int64_t)q->n_seqs);
    // a team's threads keep up to 64 elements each of a whole block; single tokens need half a warp
    const int team = !q->cu_tokens || h->pool.T * h->pool.D <= 2048 ? 32 : h->pool.T * h->pool.D <= 4096 ? 64 : 128;
    while ((1 << a.log2_T) < h->pool.T) ++a.log2_T;
    const dim3 grid((unsigned)most, (unsigned)((h->pool.Hkv + 128 / team - 1) / (128 / team)), 2);
    const void* k = type == US_F16 ? append_kernel<__half>(team) : type == US_BF16 ? append_kernel<__nv_bfloat16>(team) : append_kernel<float>(team);
    void* args[] = {&a};
    return cuda(ops_launch(k, grid, 128, 0, static_cast<cudaStream_t>(stream), args));
}

us_status us_kv_read(us_kv* h, const us_kv_seqs* q, int64_t tokens, void* K, void* V, int32_t type, void* stream)
{
    if (!h || !q || q->n_seqs < 0 || tokens < 0 || type < 0 || type > 2) return US_ERR_INVALID_ARG;
    if (q->n_seqs == 0 || tokens == 0) return US_OK;
    us_kv_seqs one = *q;
    one.cu_tokens = nullptr;
    if (!seqs_ok(h, &one, one.n_seqs) || !K || !V || !aligned(K, 16) || !aligned(V, 16) || tokens > (int64_t)q->table_width * h->pool.T) return US_ERR_INVALID_ARG;
    KvPool p = h->pool;
    KvSeqs s = seqs(&one, 0);
    us_status st = on_device(h);
    if (st == US_OK) st = error_word(&p.err);
    if (st != US_OK) return st;
    const dim3 grid((unsigned)((tokens + 15) / 16), (unsigned)((p.Hkv + kReadHeads - 1) / kReadHeads), (unsigned)std::min(s.S, 65535));
    int log2_T = 0;
    while ((1 << log2_T) < p.T) ++log2_T;
    const void* k = type == US_F16 ? (const void*)us_kv_read_kernel<__half> :
                    type == US_BF16 ? (const void*)us_kv_read_kernel<__nv_bfloat16> : (const void*)us_kv_read_kernel<float>;
    void* args[] = {&p, &s, &tokens, &log2_T, &K, &V};
    return cuda(ops_launch(k, grid, 256, 0, static_cast<cudaStream_t>(stream), args));
}

int64_t us_kv_attention_scratch(const us_kv* h, const us_kv_seqs* q, int64_t N, int32_t n_heads)
{
    if (!seqs_ok(h, q, N) || n_heads < 1 || n_heads % h->pool.Hkv) return -1;
    if (N == 0 || q->n_seqs == 0) return 0;
    return attend_plan(h->pool.D, false, N, q->n_seqs, n_heads / h->pool.Hkv, h->pool.Hkv, (int64_t)q->table_width * h->pool.T, ops_sms()).scratch;
}

us_status us_kv_attention(us_kv* h, const us_kv_seqs* q, int64_t N, const void* Q, int32_t type, int32_t n_heads, int64_t q_token_stride,
                          int64_t q_head_stride, float scale, int32_t causal, int32_t window, void* out, int64_t o_token_stride, int64_t o_head_stride,
                          float* lse, void* scratch, int64_t scratch_bytes, void* stream)
{
    if (!seqs_ok(h, q, N) || n_heads < 1 || n_heads % h->pool.Hkv || window < 0 || !(scale == scale) || scale > 3e38f || scale < -3e38f) return US_ERR_INVALID_ARG;
    if (type != US_F16 && type != US_BF16) return type == US_F32 ? US_ERR_UNSUPPORTED : US_ERR_INVALID_ARG;
    if (N == 0 || q->n_seqs == 0) return US_OK;
    if (!strides_ok(Q, type, q_token_stride, q_head_stride, N, n_heads, h->pool.D) || !strides_ok(out, type, o_token_stride, o_head_stride, N, n_heads, h->pool.D) ||
        !aligned(lse, 4)) return US_ERR_INVALID_ARG;
    us_status s = on_device(h);
    if (s != US_OK) return s;
    const int64_t G = n_heads / h->pool.Hkv;
    if (N * G >= (1ll << 31) - (1 << 16)) return US_ERR_UNSUPPORTED;
    const AttendPlan pl = attend_plan(h->pool.D, type == US_BF16, N, q->n_seqs, G, h->pool.Hkv, (int64_t)q->table_width * h->pool.T, ops_sms());
    if (pl.scratch > 0 && (!scratch || !aligned(scratch, 16) || scratch_bytes < pl.scratch)) return US_ERR_SCRATCH_TOO_SMALL;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (pl.tiles > 0) {
        const int64_t blocks = pl.tiles * h->pool.Hkv * std::max(pl.splits, h->pool.D / 16);
        if (blocks >= (1ll << 31)) return US_ERR_UNSUPPORTED;
        KvPrompt a = {};
        a.pool = h->pool;
        a.seqs = seqs(q, N);
        a.q = Q; a.q_token = q_token_stride; a.q_head = q_head_stride;
        a.out = out; a.o_token = o_token_stride; a.o_head = o_head_stride;
        a.lse = lse;
        a.part = static_cast<float*>(scratch);
        a.scale2 = (float)(std::fabs((double)scale) * 1.4426950408889634);
        a.negative = scale < 0.f;
        a.Hq = n_heads; a.G = (int32_t)G;
        a.causal = causal != 0; a.window = window;
        a.q_vec = rows_vec(Q, type, q_token_stride, q_head_stride);
        a.o_vec = rows_vec(out, type, o_token_stride, o_head_stride);
        a.splits = pl.splits;
        while ((1 << a.log2_T) < h->pool.T) ++a.log2_T;
        s = error_word(&a.pool.err);
        if (s != US_OK) return s;
        void* args[] = {&a};
        cudaError_t e = ops_kernel_allow(pl.kernel, pl.smem);
        const int threads = PrShape<128>::kThreads;
        if (e == cudaSuccess) e = ops_launch(pl.kernel, dim3((unsigned)(pl.tiles * h->pool.Hkv * pl.splits)), threads, pl.smem, st, args);
        if (e == cudaSuccess && pl.splits > 1) e = ops_launch(pl.join, dim3((unsigned)(pl.tiles * h->pool.Hkv * (h->pool.D / 16))), kPrRows, 0, st, args);
        return cuda(e);
    }
    if (!maps(h)) return US_ERR_CUDA;
    KvAttend a = {};
    a.k_map = h->k_map; a.v_map = h->v_map;
    a.pool = h->pool;
    a.seqs = seqs(q, N);
    a.q = Q; a.q_token = q_token_stride; a.q_head = q_head_stride;
    a.out = out; a.o_token = o_token_stride; a.o_head = o_head_stride;
    a.lse = lse;
    a.part = static_cast<float*>(scratch);
    a.scale2 = (float)((double)scale * 1.4426950408889634);
    a.Hq = n_heads; a.G = (int32_t)G;
    a.causal = causal != 0; a.window = window;
    a.q_vec = rows_vec(Q, type, q_token_stride, q_head_stride);
    a.stages = pl.stages;
    a.ctas = pl.ctas;
    while ((1 << a.log2_T) < h->pool.T) ++a.log2_T;
    s = error_word(&a.pool.err);
    if (s != US_OK) return s;
    cudaError_t e = ops_kernel_allow(pl.kernel, pl.smem);
    void* args[] = {&a};
    if (e == cudaSuccess) e = ops_launch(pl.kernel, dim3((unsigned)pl.ctas), 160, pl.smem, st, args);
    // (an item of one unit is never cut)
    if (e == cudaSuccess && (int64_t)q->table_width * h->pool.T > kKvTile) e = ops_launch(pl.join, dim3((unsigned)pl.ctas), 32 * kJoinWarps, 0, st, args);
    return cuda(e);
}

us_status us_kv_last_error(void)
{
    uint32_t flag = 0;
    const uint32_t zero = 0;
    cudaError_t e = cudaDeviceSynchronize();
    if (e == cudaSuccess) e = cudaMemcpyFromSymbol(&flag, g_kv_err, 4);
    if (e == cudaSuccess && flag) e = cudaMemcpyToSymbol(g_kv_err, &zero, 4);
    if (e != cudaSuccess) return cuda(e);
    return flag == 0 ? US_OK : flag == kErrIndex ? US_ERR_DEVICE_INDEX : US_ERR_DEVICE_TIMEOUT;
}
