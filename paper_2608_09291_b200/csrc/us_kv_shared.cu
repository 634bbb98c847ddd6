// Attention of sequences that share prefixes: entry points.
//
// A softmax over a prefix and own tokens is the join of two: for each query and head, sums relative to a maximum over either. The sequences of a group read their
// prefix as one long row of queries, so its keys and values come from memory once for all of them (and their products fill the tensor cores'
// tiles); the own tokens are read as ever, and what writes an output joins the two.
#include "us_kv_plan.cuh"

namespace us {
namespace {

struct SharedPlan {
    AttendPlan groups, own;
    int64_t rows, first, bytes;   // bytes of the rows; where the own part's scratch begins; in all
    const void *short_kernel, *join;   // short contexts: their kernel runs beside the groups', another joins what they leave; nullptr: the own tokens' kernel does
    int64_t short_blocks;
};
// Tokens (of a table's width) up to which a sequence's own are read by a warp for itself, beside the groups' kernel, and not by the kernel that cuts them into units, behind it.
// A warp takes 32 in 2.4 us; the other kernel has 2 to 50 us more to begin with, the more the more sequences. us beside and behind, contexts as long as their table,
// S x query heads / cache heads x head size behind P tokens. Up to 32 sequences 512 tokens: 4 x 32/8 x 128 behind 1000 34.1, 30.2 (256 tokens 23.9, 25.9); 16 x 64/8 x 128 behind 8192
// 41.8, 38.6 (256: 27.4, 36.2); 32 x 64/8 x 128 behind 8192 54.5, 52.1 (768: 74.4, 56.9). More sequences 1024: 40 x 32/8 x 128 behind 1000 63.6, 65.7; 64 x 64/8 x 128 behind 8192
// 103.7, 94.2 (768: 82.1, 88.2); 200 x 64/8 x 128 behind 1000 145, 160. Heads without groups cross earlier (16 x 32/32 x 128 behind 8192: 256 tokens 69.7, 62.6), heads of 64
// later (64 x 32/4 x 64 behind 1000: 1024 tokens 36.4, 40.6).
int64_t short_tokens(int64_t sequences) { return sequences > 32 ? 1024 : 512; }
int64_t pitch(const us_kv* h) { return h->pool.D + 4; }
int64_t up16(int64_t n) { return (n + 15) / 16 * 16; }
SharedPlan shared_plan(const us_kv* h, const us_kv_seqs* p, const us_kv_seqs* q, int64_t N, int32_t heads, bool bf16)
{
    SharedPlan r = {};
    const int64_t G = heads / h->pool.Hkv, T = h->pool.T;
    const int sms = ops_sms();
    r.own = attend_plan<kOwn>(h->pool.D, bf16, N, q->n_seqs, G, h->pool.Hkv, q->table_width * T, sms);
    if (p->n_seqs > 0) {
        r.groups = attend_plan<kGroups>(h->pool.D, bf16, N, p->n_seqs, G, h->pool.Hkv, p->table_width * T, sms);
        r.rows = N * heads * pitch(h) * 4;   // (twice, where the own tokens have rows, too)
    }
    const int64_t longest = q->table_width * T;
    if (p->n_seqs > 0 && r.own.tiles == 0 && longest <= short_tokens(q->n_seqs)) {
        r.short_blocks = (q->cu_tokens ? N * G / 8 + q->n_seqs : N * ((G + 7) / 8)) * h->pool.Hkv;   // a warp an item: as many as there may be
        r.short_kernel = h->pool.D == 128 ? (bf16 ? (const void*)us_kv_short_kernel<128, true> : (const void*)us_kv_short_kernel<128, false>) :
                                            (bf16 ? (const void*)us_kv_short_kernel<64, true> : (const void*)us_kv_short_kernel<64, false>);
        r.own.scratch = 0;
        if (r.groups.tiles == 0) {
            const bool eight = r.groups.rows == 8;
            if (h->pool.D == 128) r.join = eight ? last_join<128, 1>(bf16) : last_join<128, 2>(bf16);
            else r.join = eight ? last_join<64, 1>(bf16) : last_join<64, 2>(bf16);
        }
    }
    if (r.short_kernel && r.groups.tiles > 0) {
        // Many rows a group, short contexts of their own: the first kernel is bound by its softmax, the second by latency, so they share the GPU. The number of parts that
        // a prefix is cut in says how many SMs the groups take, and the one is chosen with which both are expected to end first. Times in us: a row tile's unit 2.9, beginning and
        // end 12; a warp's item 4 and 2.4 for 32 tokens, half of the longest, while the other kernel runs, of which an SM has eight at a time. (64 sequences of 64/8
        // heads behind 8192 tokens, bf16, with up to 512 of their own: 52, 48, 53, 73 us for 5, 6, 7, 8 parts, 77 one behind the other. Of 13 batches, 16 to 100 sequences behind 1000
        // to 16000 tokens, heads of 64 and 128 in groups of 1, 4 and 8, both types, its number is within 5 % of the best in 11; 64 x 64/8 x 128 behind 8192, 128 of their own: 8 parts
        // 50.5, 7 43.0; 64 x 32/4 x 64 behind 8192, 256 of their own: 16 parts 32.1, 14 25.4. A unit takes fp16 2.9, bf16 2.3.)
        const int64_t row_tiles = std::max<int64_t>(p->n_seqs, (N * G + kPrRows - 1) / kPrRows) * h->pool.Hkv, units = (p->table_width * T + kPrTile - 1) / kPrTile;
        const double own = (double)std::max<int64_t>(q->n_seqs, (N * G + 7) / 8) * h->pool.Hkv * (4 + 2.4 * (double)longest / 64) / 8;
        double best = 0;
        for (int s = 1; s <= 16 && (s == 1 || s * 4 <= units); ++s) {
            const int64_t blocks = row_tiles * s, left = std::max<int64_t>(1, sms - blocks);
            const double t = std::max(std::ceil((double)blocks / (double)sms) * (12 + 2.9 * std::ceil((double)units / s)), 4 + own / (double)left);
            if (s == 1 || t < best) {
                best = t;
                r.groups.splits = s;
            }
        }
        r.groups.beside = 1;
        r.groups.scratch = r.groups.tiles * h->pool.Hkv * r.groups.splits * (h->pool.D == 128 ? PrShape<128>::kPart : PrShape<64>::kPart) * 4;
        r.join = h->pool.D == 128 ? (bf16 ? (const void*)us_kv_shared_join_kernel<128, true> : (const void*)us_kv_shared_join_kernel<128, false>) :
                                    (bf16 ? (const void*)us_kv_shared_join_kernel<64, true> : (const void*)us_kv_shared_join_kernel<64, false>);
    }
    if (r.short_kernel) r.rows *= 2;
    r.first = up16(r.rows) + up16(r.groups.scratch);
    r.bytes = r.first + r.own.scratch;
    return r;
}
// The prefixes: cu_tokens has the groups' sequences.
bool groups_ok(const us_kv* h, const us_kv_seqs* p)
{
    if (!p || p->n_seqs < 0) return false;
    if (p->n_seqs == 0) return true;
    return p->cu_tokens && kv_seqs_ok(h, p, 1);
}
bool shared_ok(const us_kv* h, const us_kv_seqs* p, const us_kv_seqs* q, int64_t N, int32_t heads)
{
    return kv_seqs_ok(h, q, N) && groups_ok(h, p) && heads >= 1 && heads % h->pool.Hkv == 0;
}

}  // namespace
}  // namespace us

using namespace us;

int64_t us_kv_shared_attention_scratch(const us_kv* h, const us_kv_seqs* prefixes, const us_kv_seqs* q, int64_t N, int32_t n_heads)
{
    if (!shared_ok(h, prefixes, q, N, n_heads)) return -1;
    if (N == 0 || q->n_seqs == 0) return 0;
    return shared_plan(h, prefixes, q, N, n_heads, false).bytes;
}

us_status us_kv_shared_attention(us_kv* h, const us_kv_seqs* prefixes, const us_kv_seqs* q, int64_t N, const void* Q, int32_t type, int32_t n_heads,
                                 int64_t q_token_stride, int64_t q_head_stride, float scale, int32_t causal, void* out, int64_t o_token_stride, int64_t o_head_stride,
                                 float* lse, void* scratch, int64_t scratch_bytes, void* stream)
{
    if (!shared_ok(h, prefixes, q, N, n_heads)) return US_ERR_INVALID_ARG;
    if (prefixes->n_seqs == 0)   // (nobody shares anything)
        return us_kv_attention(h, q, N, Q, type, n_heads, q_token_stride, q_head_stride, scale, causal, 0, out, o_token_stride, o_head_stride, lse, scratch, scratch_bytes, stream);
    AttendArgs x = {Q, q_token_stride, q_head_stride, out, o_token_stride, o_head_stride, lse, type, n_heads, scale, causal, 0};
    us_status s = attend_check(h, q, N, x);
    if (s != US_OK || N == 0 || q->n_seqs == 0) return s;
    const SharedPlan pl = shared_plan(h, prefixes, q, N, n_heads, type == US_BF16);
    if (pl.bytes > 0 && (!scratch || !kv_aligned(scratch, 16) || scratch_bytes < pl.bytes)) return US_ERR_SCRATCH_TOO_SMALL;
    uint8_t* mem = static_cast<uint8_t*>(scratch);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    KvRows rows = {};
    rows.pitch = (int32_t)pitch(h);
    rows.at = static_cast<float*>(scratch);
    rows.groups = prefixes->cu_tokens;
    rows.n_groups = prefixes->n_seqs;
    KvSeqs g = kv_seqs(prefixes, N);
    g.cu = q->cu_tokens;
    g.groups = prefixes->cu_tokens;
    g.members = q->n_seqs;
    if (pl.short_kernel) {
        if (pl.short_blocks >= (1ll << 31)) return US_ERR_UNSUPPORTED;
        const Beside beside = {pl.short_kernel, pl.join, kv_seqs(q, N), pl.short_blocks};
        rows.own = rows.at + N * n_heads * pitch(h);
        return attend_run(h, g, x, pl.groups, rows, mem + up16(pl.rows), st, &beside);
    }
    s = attend_run(h, g, x, pl.groups, rows, mem + up16(pl.rows), st);   // (writes rows alone)
    if (s != US_OK) return s;
    return attend_run(h, kv_seqs(q, N), x, pl.own, rows, mem + pl.first, st);
}
