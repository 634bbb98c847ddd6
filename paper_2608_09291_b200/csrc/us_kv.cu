// The 8-bit cache's entry points: checks, launch plans.
#include "us_kv_host.h"
#include "us_kv_plan.cuh"

#include <new>

namespace us {
namespace {

__device__ uint32_t g_kv_err;   // the last failure that a kernel met since us_kv_last_error was asked

us_status cuda(cudaError_t e) { return kv_cuda(e); }
bool aligned(const void* p, int64_t b) { return kv_aligned(p, b); }
us_status on_device(const us_kv* h) { return kv_on_device(h); }
bool seqs_ok(const us_kv* h, const us_kv_seqs* q, int64_t N) { return kv_seqs_ok(h, q, N); }
KvSeqs seqs(const us_kv_seqs* q, int64_t N) { return kv_seqs(q, N); }
us_status error_word(uint32_t** err) { return kv_error_word(err); }

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

us_status kv_error_word(uint32_t** err)
{
    static void* kept[kMaxDevices];
    return kv_cuda(ops_symbol(kept, &g_kv_err, reinterpret_cast<void**>(err)));
}

namespace {

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

}  // namespace

bool kv_maps(us_kv* h)
{
    std::lock_guard<std::mutex> hold(h->lock);
    if (!h->mapped) h->mapped = encode_map(&h->k_map, h->pool.k, h->pool) && encode_map(&h->v_map, h->pool.v, h->pool);
    return h->mapped;
}

namespace {

// The device that an address lies on, or -1.
int device_of(const void* p)
{
    cudaPointerAttributes a = {};
    if (cudaPointerGetAttributes(&a, p) != cudaSuccess) cudaGetLastError();
    else if (a.type == cudaMemoryTypeDevice) return a.device;
    return -1;
}
template <class T>
const void* append_kernel(int team)
{
    return team == 32 ? (const void*)us_kv_append_kernel<T, 32> : team == 64 ? (const void*)us_kv_append_kernel<T, 64> : (const void*)us_kv_append_kernel<T, 128>;
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
    return us_kv_append_granted(h, q, N, K, V, type, k_token_stride, k_head_stride, v_token_stride, v_head_stride, nullptr, stream);
}

us_status us_kv_append_granted(us_kv* h, const us_kv_seqs* q, int64_t N, const void* K, const void* V, int32_t type, int64_t k_token_stride, int64_t k_head_stride,
                               int64_t v_token_stride, int64_t v_head_stride, const int32_t* granted, void* stream)
{
    if (!seqs_ok(h, q, N) || type < 0 || type > 2 || !aligned(granted, 4)) return US_ERR_INVALID_ARG;
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
    a.granted = granted;
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
    return attend_plan<kAlone>(h->pool.D, false, N, q->n_seqs, n_heads / h->pool.Hkv, h->pool.Hkv, (int64_t)q->table_width * h->pool.T, ops_sms()).scratch;
}

us_status us_kv_attention(us_kv* h, const us_kv_seqs* q, int64_t N, const void* Q, int32_t type, int32_t n_heads, int64_t q_token_stride,
                          int64_t q_head_stride, float scale, int32_t causal, int32_t window, void* out, int64_t o_token_stride, int64_t o_head_stride,
                          float* lse, void* scratch, int64_t scratch_bytes, void* stream)
{
    AttendArgs x = {Q, q_token_stride, q_head_stride, out, o_token_stride, o_head_stride, lse, type, n_heads, scale, causal, window};
    us_status s = attend_check(h, q, N, x);
    if (s != US_OK || N == 0 || q->n_seqs == 0) return s;
    const int64_t G = n_heads / h->pool.Hkv;
    const AttendPlan pl = attend_plan<kAlone>(h->pool.D, type == US_BF16, N, q->n_seqs, G, h->pool.Hkv, (int64_t)q->table_width * h->pool.T, ops_sms());
    if (pl.scratch > 0 && (!scratch || !aligned(scratch, 16) || scratch_bytes < pl.scratch)) return US_ERR_SCRATCH_TOO_SMALL;
    return attend_run(h, seqs(q, N), x, pl, KvRows{}, scratch, static_cast<cudaStream_t>(stream));
}

us_status us_kv_last_error(void)
{
    uint32_t flag = 0;
    const uint32_t zero = 0;
    cudaError_t e = cudaDeviceSynchronize();
    if (e == cudaSuccess) e = cudaMemcpyFromSymbol(&flag, g_kv_err, 4);
    if (e == cudaSuccess && flag) e = cudaMemcpyToSymbol(g_kv_err, &zero, 4);
    if (e != cudaSuccess) return cuda(e);
    return flag == 0 ? US_OK : flag == kErrIndex ? US_ERR_DEVICE_INDEX : flag == kErrFull ? US_ERR_OUT_OF_BLOCKS : US_ERR_DEVICE_TIMEOUT;
}
