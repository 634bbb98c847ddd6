// Attention over the 8-bit cache: which kernels a call takes, and their launches.
#pragma once
#include "us_kv_host.h"
#include "us_kv_prompt.cuh"

#include <cmath>

namespace us {

// (us_kv.cu) The tensor maps of a pool's codes.
bool kv_maps(us_kv* h);

inline int64_t size_of(int32_t t) { return t == US_F32 ? 4 : 2; }
// Rows (token, head, D): every stride holds a row, and the 16-byte path's condition.
inline bool strides_ok(const void* x, int32_t type, int64_t token, int64_t head, int64_t N, int64_t heads, int32_t D)
{
    return x && kv_aligned(x, size_of(type)) && (N == 1 || token >= D) && (heads == 1 || head >= D) && token >= 0 && head >= 0;
}
inline bool rows_vec(const void* x, int32_t type, int64_t token, int64_t head)
{
    return kv_aligned(x, 16) && token * size_of(type) % 16 == 0 && head * size_of(type) % 16 == 0;
}

struct AttendPlan {
    const void *kernel, *join;
    int rows, stages, smem, ctas;
    int join_blocks;   // (prompts) of a row tile and head
    int splits;        // (prompts) of the cache's length
    int beside;        // (prompts of groups) the kernel of the own tokens runs beside it
    int64_t tiles;     // (prompts) row tiles, at most; 0: the kernel for few rows
    int64_t scratch;
};
template <int D, bool BF16, int MODE>
AttendPlan prompt_shape(int64_t N, int64_t S, int64_t G, int64_t Hkv, int64_t longest, int sms)
{
    AttendPlan p = {};
    p.kernel = (const void*)us_kv_prompt_kernel<D, BF16, MODE>;
    if constexpr (MODE == kGroups) p.join = (const void*)us_kv_rows_join_kernel<D>;
    else p.join = (const void*)us_kv_prompt_join_kernel<D, BF16, MODE>;
    p.join_blocks = MODE == kGroups ? D / 4 : D / 16;
    p.smem = PrShape<D>::kSmem;
    p.tiles = N * G / kPrRows + S;
    // a tile's walk over the cache is split where the tiles would leave SMs idle, in parts of at least four units
    const int64_t likely = std::max(S, (N * G + kPrRows - 1) / kPrRows) * Hkv;
    p.splits = (int)std::max<int64_t>(1, std::min<int64_t>({16, sms / likely, longest / (4 * kPrTile)}));
    p.scratch = p.splits > 1 ? p.tiles * Hkv * p.splits * PrShape<D>::kPart * 4 : 0;
    return p;
}
template <int D, int NT, bool BF16, int MODE>
AttendPlan attend_shape(int sms)
{
    using S = KvShape<D, NT>;
    AttendPlan p = {};
    p.kernel = (const void*)us_kv_attend_kernel<D, NT, BF16, MODE>;
    p.join = (const void*)us_kv_join_kernel<D, NT, BF16, MODE>;
    p.rows = S::R;
    p.stages = std::min(S::kMaxStages, (111 * 1024 - 1024 - S::kMerge) / S::kStage);   // two CTAs an SM
    p.smem = 1024 + p.stages * S::kStage + S::kMerge;
    p.ctas = 2 * sms;
    p.scratch = (int64_t)p.ctas * 2 * S::kPart * 4;
    return p;
}
template <int D, int NT, int MODE>
AttendPlan attend_shape(bool bf16, int sms) { return bf16 ? attend_shape<D, NT, true, MODE>(sms) : attend_shape<D, NT, false, MODE>(sms); }
// The kernel for few rows.
template <int MODE>
AttendPlan few_plan(int D, bool bf16, int64_t N, int64_t S, int64_t G, int sms)
{
    // rows a cache head has on average: 8 a tile are enough for them, or 16
    const bool few = N * G <= 8 * S;
    if (D == 128) return few ? attend_shape<128, 1, MODE>(bf16, sms) : attend_shape<128, 2, MODE>(bf16, sms);
    return few ? attend_shape<64, 1, MODE>(bf16, sms) : attend_shape<64, 2, MODE>(bf16, sms);
}
// The join of groups with few rows and their sequences' own tokens.
template <int D, int NT>
const void* last_join(bool bf16) { return bf16 ? (const void*)us_kv_join_kernel<D, NT, true, kLast> : (const void*)us_kv_join_kernel<D, NT, false, kLast>; }
template <int MODE>
AttendPlan attend_plan(int D, bool bf16, int64_t N, int64_t S, int64_t G, int64_t Hkv, int64_t longest, int sms)
{
    // Rows a cache head has on average decide. 64 sequences of 4096 tokens, 8 cache heads of 128, bf16, this kernel and the other one: 16 rows 154, 341 us, 32
    // rows 288, 342, 40 rows 414, 343, 128 rows 1082, 349; four sequences of 32768: 32 rows 140, 170, 40 rows 191, 172. (64 of 300: 24 rows 76, 66.)
    if (N * G > 32 * S) {
        if (D == 128) return bf16 ? prompt_shape<128, true, MODE>(N, S, G, Hkv, longest, sms) : prompt_shape<128, false, MODE>(N, S, G, Hkv, longest, sms);
        return bf16 ? prompt_shape<64, true, MODE>(N, S, G, Hkv, longest, sms) : prompt_shape<64, false, MODE>(N, S, G, Hkv, longest, sms);
    }
    return few_plan<MODE>(D, bf16, N, S, G, sms);
}

struct AttendArgs {
    const void* q;
    int64_t q_token, q_head;
    void* out;
    int64_t o_token, o_head;
    float* lse;
    int32_t type, heads;
    float scale;
    int32_t causal, window;
};
inline us_status attend_check(us_kv* h, const us_kv_seqs* q, int64_t N, const AttendArgs& x)
{
    if (!kv_seqs_ok(h, q, N) || x.heads < 1 || x.heads % h->pool.Hkv || x.window < 0 || !(x.scale == x.scale) || x.scale > 3e38f || x.scale < -3e38f) return US_ERR_INVALID_ARG;
    if (x.type != US_F16 && x.type != US_BF16) return x.type == US_F32 ? US_ERR_UNSUPPORTED : US_ERR_INVALID_ARG;
    if (N == 0 || q->n_seqs == 0) return US_OK;
    if (!strides_ok(x.q, x.type, x.q_token, x.q_head, N, x.heads, h->pool.D) || !strides_ok(x.out, x.type, x.o_token, x.o_head, N, x.heads, h->pool.D) ||
        !kv_aligned(x.lse, 4)) return US_ERR_INVALID_ARG;
    const us_status s = kv_on_device(h);
    if (s != US_OK) return s;
    return N * (x.heads / h->pool.Hkv) >= (1ll << 31) - (1 << 16) ? US_ERR_UNSUPPORTED : US_OK;
}
// What a call of attention passes to either kernel for few rows.
inline us_status attend_args(const us_kv* h, const KvSeqs& q, const AttendArgs& x, const KvRows& rows, KvAttend* a)
{
    *a = KvAttend{};
    a->pool = h->pool;
    a->seqs = q;
    a->q = x.q; a->q_token = x.q_token; a->q_head = x.q_head;
    a->out = x.out; a->o_token = x.o_token; a->o_head = x.o_head;
    a->lse = x.lse;
    a->scale2 = (float)((double)x.scale * 1.4426950408889634);
    a->Hq = x.heads; a->G = x.heads / h->pool.Hkv;
    a->causal = x.causal != 0 && !q.groups; a->window = x.window;   // (a group's rows see all of their prefix)
    a->q_vec = rows_vec(x.q, x.type, x.q_token, x.q_head);
    a->rows = rows;
    while ((1 << a->log2_T) < h->pool.T) ++a->log2_T;
    return kv_error_word(&a->pool.err);
}
// The kernel of short contexts, beside the groups' kernel; join: of both.
struct Beside {
    const void *kernel, *join;
    KvSeqs own;
    int64_t blocks;
};
inline us_status short_run(us_kv* h, const AttendArgs& x, const Beside& b, const KvRows& rows, cudaStream_t st)
{
    KvAttend a;
    const us_status s = attend_args(h, b.own, x, rows, &a);
    if (s != US_OK) return s;
    void* args[] = {&a};
    const cudaError_t e = ops_kernel_beside(b.kernel);
    return kv_cuda(e != cudaSuccess ? e : ops_launch(b.kernel, dim3((unsigned)b.blocks), 32, 0, st, args));
}
// rows: see KvRows (unused by kAlone's kernels). beside: (groups) what runs beside them, and joins all.
inline us_status attend_run(us_kv* h, const KvSeqs& q, const AttendArgs& x, const AttendPlan& pl, const KvRows& rows, void* scratch, cudaStream_t st,
                            const Beside* beside = nullptr)
{
    const int64_t G = x.heads / h->pool.Hkv;
    if (pl.tiles > 0) {
        const int64_t blocks = pl.tiles * h->pool.Hkv * std::max(pl.splits, pl.join_blocks);
        if (blocks >= (1ll << 31)) return US_ERR_UNSUPPORTED;
        KvPrompt a = {};
        a.pool = h->pool;
        a.seqs = q;
        a.q = x.q; a.q_token = x.q_token; a.q_head = x.q_head;
        a.out = x.out; a.o_token = x.o_token; a.o_head = x.o_head;
        a.lse = x.lse;
        a.part = static_cast<float*>(scratch);
        a.scale2 = (float)(std::fabs((double)x.scale) * 1.4426950408889634);
        a.negative = x.scale < 0.f;
        a.Hq = x.heads; a.G = (int32_t)G;
        a.causal = x.causal != 0 && !q.groups; a.window = x.window;   // (a group's rows see all of their prefix)
        a.q_vec = rows_vec(x.q, x.type, x.q_token, x.q_head);
        a.o_vec = rows_vec(x.out, x.type, x.o_token, x.o_head);
        a.splits = pl.splits;
        a.beside = pl.beside;
        a.rows = rows;
        while ((1 << a.log2_T) < h->pool.T) ++a.log2_T;
        const us_status s = kv_error_word(&a.pool.err);
        if (s != US_OK) return s;
        void* args[] = {&a};
        cudaError_t e = ops_kernel_allow(pl.kernel, pl.smem);
        const int threads = PrShape<128>::kThreads;
        if (e == cudaSuccess) e = ops_launch(pl.kernel, dim3((unsigned)(pl.tiles * h->pool.Hkv * pl.splits)), threads, pl.smem, st, args);
        if (e == cudaSuccess && beside) {
            const us_status s = short_run(h, x, *beside, rows, st);
            if (s != US_OK) return s;
            e = ops_launch(beside->join, dim3((unsigned)(pl.tiles * h->pool.Hkv * (h->pool.D / 4))), 256, 0, st, args);
        } else if (e == cudaSuccess && pl.splits > 1) e = ops_launch(pl.join, dim3((unsigned)(pl.tiles * h->pool.Hkv * pl.join_blocks)), kPrRows, 0, st, args);
        return kv_cuda(e);
    }
    if (!kv_maps(h)) return US_ERR_CUDA;
    KvAttend a;
    const us_status s = attend_args(h, q, x, rows, &a);
    if (s != US_OK) return s;
    a.k_map = h->k_map; a.v_map = h->v_map;
    a.part = static_cast<float*>(scratch);
    a.stages = pl.stages;
    a.ctas = pl.ctas;
    cudaError_t e = ops_kernel_allow(pl.kernel, pl.smem);
    void* args[] = {&a};
    if (e == cudaSuccess) e = ops_launch(pl.kernel, dim3((unsigned)pl.ctas), 160, pl.smem, st, args);
    if (beside) {
        if (e == cudaSuccess) {
            const us_status b = short_run(h, x, *beside, rows, st);
            if (b != US_OK) return b;
        }
        if (e == cudaSuccess) e = ops_launch(beside->join, dim3((unsigned)pl.ctas), 32 * kJoinWarps, 0, st, args);
        return kv_cuda(e);
    }
    // (an item of one unit is never cut)
    if (e == cudaSuccess && (int64_t)q.width * h->pool.T > kKvTile) e = ops_launch(pl.join, dim3((unsigned)pl.ctas), 32 * kJoinWarps, 0, st, args);
    return kv_cuda(e);
}

}  // namespace us
