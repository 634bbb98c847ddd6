// Blocks of the 8-bit cache: which are in use, by how many table entries, and their copies.
//
// refs[b] counts the table entries that hold block b; 0: free. All of it lies on the device and is decided there, in an order that the call's data
// alone give: nothing waits for the host, and every call can be captured into a graph.
#include "us_kv_host.h"

namespace us {
namespace {

struct Pages {
    KvPool pool;
    int32_t* refs;
    int32_t log2_T;
};
__device__ __forceinline__ int blocks_of(int64_t tokens, int log2_T) { return (int)((tokens + (1 << log2_T) - 1) >> log2_T); }
__device__ __forceinline__ bool in_pool(const Pages& a, int32_t b) { return (uint32_t)b < (uint32_t)a.pool.blocks; }
__device__ __forceinline__ void wrong(const Pages& a) { atomicExch(a.pool.err, kErrIndex); }
// One entry less for a block; one that no entry holds stays free.
__device__ __forceinline__ void give_up(const Pages& a, int32_t b)
{
    if (atomicSub(a.refs + b, 1) <= 0) {
        atomicAdd(a.refs + b, 1);
        wrong(a);
    }
}

// Children's rows (blockIdx.y; a thread an entry, kEntries a block): the parent's blocks, each held once more; then, unless they are kept, the parents' rows, whose
// blocks are held once less. Where they are given up, a parent's first child takes its entries over, and only a parent without one gives them up: so an entry's own count is there
// whenever it is looked at, in whatever order the rows are done, and a count of 0 says that nobody holds the block. Bound by four trips to memory, one
// behind the other (the last is the counts' answers): 8 children of one parent 2.2 us inside a graph, 256 of 16 3.6.
constexpr int kEntries = 128;
// Whether s is among the first n parents (all threads of a block).
__device__ __forceinline__ bool among(const int32_t* parents, int64_t n, int64_t s)
{
    bool is = false;
    for (int64_t i = threadIdx.x; i < n && !is; i += kEntries) is = __ldcg(parents + i) == s;
    return __syncthreads_or(is) != 0;
}
__global__ void __launch_bounds__(kEntries) us_kv_fork_kernel(Pages a, KvSeqs q, const int32_t* parents, int children, int32_t* table, int64_t stride, int32_t* lengths,
                                                              int give)
{
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int64_t rows = (int64_t)children + (give ? q.S : 0);
    const int j = (int)(blockIdx.x * kEntries + threadIdx.x);
    for (int64_t w = blockIdx.y; w < rows; w += gridDim.y) {
        const bool child = w < children;
        const int64_t s = child ? __ldcg(parents + w) : w - children;
        bool bad = s < -1 || s >= q.S;
        int32_t len = bad || s < 0 ? 0 : __ldcg(q.lengths + s);
        if (len < 0 || len > (int64_t)q.width << a.log2_T) {
            bad = true;
            len = 0;
        }
        const int n = blocks_of(len, a.log2_T);
        const int32_t entry = j < n ? __ldcg(q.table + s * q.table_stride + j) : 0;   // (on its way meanwhile)
        const bool other = give && among(parents, child ? w : children, s);           // another child takes the parent's entries over
        if (j < (child ? q.width : n)) {
            const int32_t b = entry;
            if (j < n) {
                if (!in_pool(a, b)) bad = true;
                else if (!child) {
                    if (!other) give_up(a, b);
                } else if (give && !other) bad |= __ldcg(a.refs + b) <= 0;
                else bad |= atomicAdd(a.refs + b, 1) <= 0;
            }
            if (child) table[w * stride + j] = b;
        }
        if (child && j == 0) lengths[w] = len;
        if (bad) wrong(a);
    }
}

// Exclusive sum over the 1024 threads of a block, and the total.
template <class N>
__device__ __forceinline__ N block_sum(N v, N* shared, N& total)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    N x = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const N y = __shfl_up_sync(0xffffffffu, x, o);
        if (lane >= o) x += y;
    }
    __syncthreads();   // (whoever still reads the last sums)
    if (lane == 31) shared[warp] = x;
    __syncthreads();
    N w = shared[lane];
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const N y = __shfl_up_sync(0xffffffffu, w, o);
        if (lane >= o) w += y;
    }
    total = __shfl_sync(0xffffffffu, w, 31);
    const N front = __shfl_sync(0xffffffffu, w, (warp + 31) & 31);
    return x - v + (warp ? front : 0);
}
// The counts of 16 blocks from b on (behind the pool's end: 1).
__device__ __forceinline__ void sixteen(const Pages& a, int64_t b, int32_t (&r)[16])
{
#pragma unroll
    for (int i = 0; i < 16; i += 4) {
        if (b + i + 4 <= a.pool.blocks) {
            const int4 v = __ldcg(reinterpret_cast<const int4*>(a.refs + b + i));
            r[i] = v.x; r[i + 1] = v.y; r[i + 2] = v.z; r[i + 3] = v.w;
        } else {
#pragma unroll
            for (int k = 0; k < 4; ++k) r[i + k] = b + i + k < a.pool.blocks ? __ldcg(a.refs + b + i + k) : 1;
        }
    }
}

// Room for new tokens, one block of 1024 threads.
//   1. Each sequence's last block, if new tokens go into it and other entries hold it, too: how many of the batch do, and which first.
//   2. What each needs: a copy of that block (all but the first, if nobody else holds it), and blocks behind it; a sum over the sequences says which
//      of the free blocks, lowest first, are whose.
//   3. The free blocks, 16384 counts at a time (the first are on their way from the beginning), until there are enough.
//   4. Tables, counts and lengths; what is to be copied is left for the next kernel.
// A thread has a sequence, or several 1024 apart; what it knows of them waits in shared memory, in scratch where there are more than 1024.
// Bound by its trips to memory, one behind the other: 8 us alone and from memory, for 8 sequences as for 256.
struct Extend {
    int32_t* table;
    int64_t stride;
    int32_t width, S;
    int32_t* lengths;
    const int32_t* tokens;
    int32_t each;
    int32_t *count, *first, *list;          // of blocks
    int32_t *need, *at, *src, *dst, *held;  // of sequences; need: blocks behind the last, + 2^30 for a copy; -1: left as it is
    int32_t* granted;                       // (or nullptr) by how many tokens each has grown
};
constexpr int32_t kCopy = 1 << 30;
__global__ void __launch_bounds__(1024) us_kv_extend_kernel(Pages a, Extend e)
{
    __shared__ uint32_t sums[32];
    __shared__ unsigned long long sums64[32];
    __shared__ int32_t near[3][1024];
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int64_t most = (int64_t)e.width << a.log2_T;
    const int lane = threadIdx.x & 31;
    const bool few = e.S <= 1024;
    int32_t *need_of = few ? near[0] : e.need, *at_of = few ? near[1] : e.at, *last_of = few ? near[2] : e.src;
    int32_t r[16];
    sixteen(a, 16 * threadIdx.x, r);
    // 1.
    for (int s = threadIdx.x; s < e.S; s += 1024) {
        const int64_t len = __ldcg(e.lengths + s), n = e.tokens ? __ldcg(e.tokens + s) : e.each;
        int32_t need = 0, last = -1;
        if (len < 0 || n < 0 || len + n > most) {
            wrong(a);
            need = -1;
        } else if (n > 0) {
            const int have = blocks_of(len, a.log2_T);
            need = blocks_of(len + n, a.log2_T) - have;
            if (len & ((1 << a.log2_T) - 1)) {
                const int32_t b = __ldcg(e.table + s * e.stride + have - 1);
                const int32_t held = in_pool(a, b) ? __ldcg(a.refs + b) : 0;
                if (held <= 0) {
                    wrong(a);
                    need = -1;
                } else if (held > 1) {
                    last = b;
                    e.count[b] = 0;
                    e.first[b] = 0x7FFFFFFF;
                }
            }
        }
        need_of[s] = need;
        last_of[s] = last;
    }
    __syncthreads();
    for (int s = threadIdx.x; s < e.S; s += 1024)
        if (last_of[s] >= 0) {
            atomicAdd(e.count + last_of[s], 1);
            atomicMin(e.first + last_of[s], s);
        }
    __syncthreads();
    // 2.
    unsigned long long total = 0;
    for (int base = 0; base < e.S; base += 1024) {
        const int s = base + threadIdx.x;
        unsigned long long mine = 0, sum;
        if (s < e.S && need_of[s] >= 0) {
            mine = need_of[s];
            const int32_t b = last_of[s];
            if (b >= 0 && !(__ldcg(e.count + b) >= __ldcg(a.refs + b) && __ldcg(e.first + b) == s)) {
                need_of[s] |= kCopy;
                ++mine;
            }
        }
        const unsigned long long before = block_sum(mine, sums64, sum);
        if (s < e.S) at_of[s] = (int32_t)min(total + before, 1ull << 30);   // (a pool has fewer blocks than that)
        total += sum;
    }
    // 3.
    const uint32_t wanted = (uint32_t)min(total, (unsigned long long)a.pool.blocks);
    uint32_t found = 0;
    for (int64_t b0 = 0; b0 < a.pool.blocks && found < wanted; b0 += 16384) {
        const int64_t b = b0 + 16 * threadIdx.x;
        if (b0) sixteen(a, b, r);
        uint32_t n = 0, sum;
#pragma unroll
        for (int i = 0; i < 16; ++i) n += r[i] <= 0;
        uint32_t k = found + block_sum(n, sums, sum);
#pragma unroll
        for (int i = 0; i < 16; ++i)
            if (r[i] <= 0) {
                if (k < wanted) e.list[k] = (int32_t)b + i;
                ++k;
            }
        found += sum;
    }
    __syncthreads();
    // (Where blocks are short: a block that a sequence would keep for itself, and that another one goes on holding for want of a copy, is not written into.)
    const bool want = total > found;
    if (want) {
        for (int s = threadIdx.x; s < e.S; s += 1024)
            if (need_of[s] >= kCopy && (uint32_t)at_of[s] + (need_of[s] & (kCopy - 1)) + 1u > found) atomicExch(e.count + last_of[s], -1);
        __syncthreads();
    }
    // 4. (a sequence's blocks: its thread, or all of the warp where one of its sequences gets many)
    for (int base = threadIdx.x & ~31; base < e.S; base += 1024) {
        const int s = base + lane;
        const int32_t what = s < e.S ? need_of[s] : -1;
        int32_t dst = -1, held = 0, have = 0, n = 0, more = 0;
        uint32_t from = 0;
        bool fits = what >= 0;
        if (fits) {
            const uint32_t need = what & (kCopy - 1), copy = what & kCopy ? 1 : 0, at = (uint32_t)at_of[s];
            const bool stuck = want && !copy && last_of[s] >= 0 && __ldcg(e.count + last_of[s]) < 0;
            if (stuck || (need + copy > 0 && at + need + copy > found)) {
                atomicExch(a.pool.err, kErrFull);
                fits = false;
            } else {
                const int32_t len = e.lengths[s];
                more = e.tokens ? __ldcg(e.tokens + s) : e.each;
                have = blocks_of(len, a.log2_T);
                if (copy) {
                    dst = e.list[at];
                    held = len & ((1 << a.log2_T) - 1);
                    e.table[s * e.stride + have - 1] = dst;
                    a.refs[dst] = 1;
                    atomicSub(a.refs + last_of[s], 1);
                }
                n = (int32_t)need;
                from = at + copy;
                e.lengths[s] = len + more;
            }
        }
        if (s < e.S) {
            e.src[s] = last_of[s];
            e.dst[s] = dst;
            e.held[s] = held;
            if (e.granted) e.granted[s] = more;
        }
        const uint32_t many = __ballot_sync(0xffffffffu, n > 4);
        if (n <= 4)
            for (int j = 0; j < n; ++j) {
                const int32_t b = e.list[from + j];
                e.table[s * e.stride + have + j] = b;
                a.refs[b] = 1;
            }
        for (uint32_t m = many; m; m &= m - 1) {
            const int l = __ffs(m) - 1;
            const int count = __shfl_sync(0xffffffffu, n, l), first = __shfl_sync(0xffffffffu, have, l);
            const uint32_t where = __shfl_sync(0xffffffffu, from, l);
            for (int j = lane; j < count; j += 32) {
                const int32_t b = e.list[where + j];
                e.table[(int64_t)(base + l) * e.stride + first + j] = b;
                a.refs[b] = 1;
            }
        }
    }
}

// A table's entry j of sequence s after the blocks have moved.
__device__ __forceinline__ void remap(const Pages& a, const int32_t* map, const KvSeqs& q, int64_t s, int j)
{
    const int32_t len = __ldcg(q.lengths + s);
    const bool bad = len < 0 || len > (int64_t)q.width << a.log2_T;
    if (bad && j == 0) wrong(a);
    if (bad || j >= blocks_of(len, a.log2_T)) return;
    int32_t* at = const_cast<int32_t*>(q.table) + s * q.table_stride + j;
    const int32_t b = *at;
    if (in_pool(a, b)) *at = __ldcg(map + b);
    else wrong(a);
}
// Tables whose entries follow the blocks in the launch that moves them.
constexpr int kTables = 4;
struct Tables {
    KvSeqs q[kTables];
    const int32_t* map;
    int32_t n;
};

// Copies of blocks: the first `held` tokens (or all) of block src[i] and the steps to block dst[i], where dst[i] >= 0. A warp has 4 KB of a head at a time.
// Bound by memory.
__global__ void __launch_bounds__(256) us_kv_copy_kernel(Pages a, const int32_t* src, const int32_t* dst, const int32_t* held, int64_t n, const int32_t* n_device,
                                                         const __grid_constant__ Tables tables)
{
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    if (n_device) n = __ldcg(n_device);
    for (int t = 0; t < tables.n; ++t) {
        const KvSeqs& q = tables.q[t];
        for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < (int64_t)q.S * q.width; i += (int64_t)gridDim.x * blockDim.x)
            remap(a, tables.map, q, i / q.width, (int)(i % q.width));
    }
    const KvPool& p = a.pool;
    const int lane = threadIdx.x & 31, size = p.D << a.log2_T, chunks = (size + 4095) / 4096;
    const int64_t units = n * 2 * p.Hkv * chunks, step = ((int64_t)gridDim.x * blockDim.x) >> 5;
    for (int64_t u = ((int64_t)blockIdx.x * blockDim.x + threadIdx.x) >> 5; u < units; u += step) {
        const int64_t i = u / (2 * p.Hkv * chunks);
        const int rest = (int)(u - i * (2 * p.Hkv * chunks)), which = rest / (p.Hkv * chunks), h = (rest - which * p.Hkv * chunks) / chunks, c = rest % chunks;
        const int32_t from = __ldcg(src + i), to = __ldcg(dst + i);
        if (to < 0) {
            if (to != -1) wrong(a);
            continue;
        }
        if (!in_pool(a, from) || !in_pool(a, to)) {
            if (lane == 0) wrong(a);
            continue;
        }
        const int64_t x = (int64_t)from * p.Hkv + h, y = (int64_t)to * p.Hkv + h;
        const int bytes = held ? __ldcg(held + i) * p.D : size, left = min(4096, bytes - 4096 * c);
        const int8_t* codes = which ? p.v : p.k;
        const uint4* s = reinterpret_cast<const uint4*>(codes + x * size + 4096 * c);
        uint4* d = reinterpret_cast<uint4*>(const_cast<int8_t*>(codes) + y * size + 4096 * c);
        uint4 v[8];
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (16 * (32 * k + lane) < left) v[k] = __ldcg(s + 32 * k + lane);
        float* steps = which ? p.v_step : p.k_step;
        if (c == 0 && lane == 0) steps[y] = steps[x];
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (16 * (32 * k + lane) < left) d[32 * k + lane] = v[k];
    }
}

// Which blocks move where so that the ones in use are the pool's first: those behind, in order, to the free ones in front, in order. One block of threads.
__global__ void __launch_bounds__(1024) us_kv_compact_kernel(Pages a, int32_t* map, int32_t* used, int32_t* src, int32_t* dst, int32_t* moves)
{
    __shared__ uint32_t sums[32];
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    int64_t total = 0;
    int32_t r[16];
    for (int64_t b0 = 0; b0 < a.pool.blocks; b0 += 16384) {
        const int64_t b = b0 + 16 * threadIdx.x;
        sixteen(a, b, r);
        uint32_t n = 0, sum;
#pragma unroll
        for (int i = 0; i < 16; ++i) n += b + i < a.pool.blocks && r[i] > 0;
        block_sum(n, sums, sum);
        total += sum;
    }
    uint32_t from = 0, to = 0;
    for (int64_t b0 = 0; b0 < a.pool.blocks; b0 += 16384) {
        const int64_t b = b0 + 16 * threadIdx.x;
        if (a.pool.blocks > 16384) sixteen(a, b, r);
        uint32_t n = 0, sum;   // movers, and holes 2^16 each
#pragma unroll
        for (int i = 0; i < 16; ++i)
            if (b + i < a.pool.blocks) n += r[i] > 0 ? (b + i >= total ? 1u : 0u) : (b + i < total ? 0x10000u : 0u);
        const uint32_t before = block_sum(n, sums, sum);
        uint32_t x = from + (before & 0xFFFFu), y = to + (before >> 16);
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            if (b + i >= a.pool.blocks) break;
            map[b + i] = (int32_t)(b + i);
            if (r[i] > 0 && b + i >= total) src[x++] = (int32_t)(b + i);
            if (r[i] <= 0 && b + i < total) dst[y++] = (int32_t)(b + i);
        }
        from += sum & 0xFFFFu;
        to += sum >> 16;
    }
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < from; i += 1024) {
        const int32_t x = src[i], y = dst[i];
        map[x] = y;
        a.refs[y] = a.refs[x];
        a.refs[x] = 0;
    }
    if (threadIdx.x == 0) {
        *used = (int32_t)total;
        *moves = (int32_t)from;
    }
}

// A row blockIdx.y, a thread an entry.
__global__ void __launch_bounds__(kEntries) us_kv_remap_kernel(Pages a, const int32_t* map, KvSeqs q)
{
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int j = (int)(blockIdx.x * kEntries + threadIdx.x);
    for (int64_t s = blockIdx.y; s < q.S; s += gridDim.y) remap(a, map, q, s, j);
}

// Children that every row looks through; more: a launch for them, and one that gives the parents up. (As many parents as children, tables of 16 blocks: 1024 5.2 us and 6.5 in two
// launches, 2048 10.3 and 9.1, 4096 25.1 and 14.6.)
constexpr int kLooked = 1024;
dim3 entries(int64_t rows, int64_t width) { return dim3((unsigned)std::max<int64_t>(1, (width + kEntries - 1) / kEntries), (unsigned)std::min<int64_t>(rows, 65535)); }

bool refs_ok(const int32_t* refs) { return refs && kv_aligned(refs, 16); }
// What all calls' kernels get, on the pool's device.
us_status begin(us_kv* h, int32_t* refs, Pages* a)
{
    us_status s = kv_on_device(h);
    if (s != US_OK) return s;
    *a = Pages{};
    a->pool = h->pool;
    a->refs = refs;
    while ((1 << a->log2_T) < h->pool.T) ++a->log2_T;
    return kv_error_word(&a->pool.err);
}
us_status copy(const Pages& a, const int32_t* src, const int32_t* dst, const int32_t* held, int64_t n, const int32_t* n_device, cudaStream_t st, const Tables* tables = nullptr)
{
    Tables none = {};
    const int64_t chunks = ((int64_t)a.pool.D * a.pool.T + 4095) / 4096, units = n * 2 * a.pool.Hkv * chunks;
    const dim3 grid((unsigned)std::max<int64_t>(1, std::min<int64_t>((units + 7) / 8, 8 * ops_sms())));
    void* args[] = {const_cast<Pages*>(&a), &src, &dst, &held, &n, &n_device, tables ? const_cast<Tables*>(tables) : &none};
    return kv_cuda(ops_launch((const void*)us_kv_copy_kernel, grid, 256, 0, st, args));
}

}  // namespace
}  // namespace us

using namespace us;

us_status us_kv_copy_blocks(us_kv* h, const int32_t* src, const int32_t* dst, int64_t n, void* stream)
{
    if (!h || n < 0 || n >= (1ll << 31)) return US_ERR_INVALID_ARG;
    if (n == 0) return US_OK;
    if (!src || !dst || !kv_aligned(src, 4) || !kv_aligned(dst, 4)) return US_ERR_INVALID_ARG;
    Pages a;
    const us_status s = begin(h, nullptr, &a);
    if (s != US_OK) return s;
    return copy(a, src, dst, nullptr, n, nullptr, static_cast<cudaStream_t>(stream));
}

us_status us_kv_fork(us_kv* h, int32_t* refs, const us_kv_seqs* q, const int32_t* parents, int32_t n_children, int32_t* table, int64_t table_stride,
                     int32_t* lengths, int32_t keep, void* stream)
{
    us_kv_seqs one = q ? *q : us_kv_seqs{};
    one.cu_tokens = nullptr;
    if (!q || !kv_seqs_ok(h, &one, one.n_seqs) || n_children < 0) return US_ERR_INVALID_ARG;
    if (n_children > 0 && (!parents || !table || !lengths || !kv_aligned(parents, 4) || !kv_aligned(table, 4) || !kv_aligned(lengths, 4) || q->table_width < 0 ||
                           (n_children > 1 && table_stride < q->table_width))) return US_ERR_INVALID_ARG;
    if (!refs_ok(refs)) return US_ERR_INVALID_ARG;
    Pages a;
    const us_status s = begin(h, refs, &a);
    if (s != US_OK) return s;
    int32_t give = keep == 0;
    const int64_t rows = (int64_t)n_children + (give ? q->n_seqs : 0);
    if (rows == 0) return US_OK;
    if (give && n_children > kLooked) {
        const us_status k = us_kv_fork(h, refs, q, parents, n_children, table, table_stride, lengths, 1, stream);
        return k != US_OK ? k : us_kv_release(h, refs, q, stream);
    }
    KvSeqs k = kv_seqs(&one, 0);
    void* args[] = {&a, &k, &parents, &n_children, &table, &table_stride, &lengths, &give};
    return kv_cuda(ops_launch((const void*)us_kv_fork_kernel, entries(rows, q->table_width), kEntries, 0, static_cast<cudaStream_t>(stream), args));
}

us_status us_kv_release(us_kv* h, int32_t* refs, const us_kv_seqs* q, void* stream)
{
    return us_kv_fork(h, refs, q, nullptr, 0, nullptr, 0, nullptr, 0, stream);
}

int64_t us_kv_extend_scratch(const us_kv* h, int32_t n_seqs)
{
    return !h || n_seqs < 0 ? -1 : 4 * (3 * (int64_t)h->pool.blocks + 5 * (int64_t)n_seqs);
}

us_status us_kv_extend(us_kv* h, int32_t* refs, int32_t* table, int64_t table_stride, int32_t table_width, int32_t* lengths, int32_t n_seqs,
                       const int32_t* tokens, int32_t tokens_each, void* scratch, int64_t scratch_bytes, void* stream)
{
    return us_kv_extend_granted(h, refs, table, table_stride, table_width, lengths, n_seqs, tokens, tokens_each, nullptr, scratch, scratch_bytes, stream);
}

us_status us_kv_extend_granted(us_kv* h, int32_t* refs, int32_t* table, int64_t table_stride, int32_t table_width, int32_t* lengths, int32_t n_seqs,
                               const int32_t* tokens, int32_t tokens_each, int32_t* granted, void* scratch, int64_t scratch_bytes, void* stream)
{
    us_kv_seqs q = {};
    q.block_table = table;
    q.table_stride = table_stride;
    q.lengths = lengths;
    q.n_seqs = n_seqs;
    q.table_width = table_width;
    if (!kv_seqs_ok(h, &q, n_seqs) || (tokens ? !kv_aligned(tokens, 4) : tokens_each < 0) || !kv_aligned(granted, 4) || !refs_ok(refs)) return US_ERR_INVALID_ARG;
    if (n_seqs == 0) return US_OK;
    if (!scratch || !kv_aligned(scratch, 16) || scratch_bytes < us_kv_extend_scratch(h, n_seqs)) return US_ERR_SCRATCH_TOO_SMALL;
    Pages a;
    const us_status s = begin(h, refs, &a);
    if (s != US_OK) return s;
    Extend e = {};
    e.table = table;
    e.stride = table_stride;
    e.width = table_width;
    e.S = n_seqs;
    e.lengths = lengths;
    e.tokens = tokens;
    e.each = tokens_each;
    e.count = static_cast<int32_t*>(scratch);
    e.first = e.count + a.pool.blocks;
    e.list = e.first + a.pool.blocks;
    e.need = e.list + a.pool.blocks;
    e.at = e.need + n_seqs;
    e.src = e.at + n_seqs;
    e.dst = e.src + n_seqs;
    e.held = e.dst + n_seqs;
    e.granted = granted;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    void* args[] = {&a, &e};
    const us_status k = kv_cuda(ops_launch((const void*)us_kv_extend_kernel, dim3(1), 1024, 0, st, args));
    return k != US_OK ? k : copy(a, e.src, e.dst, e.held, n_seqs, nullptr, st);
}

int64_t us_kv_compact_scratch(const us_kv* h) { return h ? 4 * (2 * (int64_t)h->pool.blocks + 1) : -1; }

// A table as the kernels see it, its entries to be written.
static bool table_ok(const us_kv* h, const us_kv_seqs* t)
{
    us_kv_seqs q = *t;
    q.cu_tokens = nullptr;
    return kv_seqs_ok(h, &q, q.n_seqs);
}

us_status us_kv_compact(us_kv* h, int32_t* refs, const us_kv_seqs* tables, int32_t n_tables, int32_t* map, int32_t* used, void* scratch, int64_t scratch_bytes, void* stream)
{
    if (!h || !refs_ok(refs) || n_tables < 0 || (n_tables > 0 && !tables) || !map || !used || !kv_aligned(map, 4) || !kv_aligned(used, 4)) return US_ERR_INVALID_ARG;
    for (int i = 0; i < n_tables; ++i)   // (all of them before a block moves)
        if (!table_ok(h, tables + i)) return US_ERR_INVALID_ARG;
    if (!scratch || !kv_aligned(scratch, 16) || scratch_bytes < us_kv_compact_scratch(h)) return US_ERR_SCRATCH_TOO_SMALL;
    Pages a;
    us_status s = begin(h, refs, &a);
    if (s != US_OK) return s;
    int32_t *src = static_cast<int32_t*>(scratch), *dst = src + a.pool.blocks, *moves = dst + a.pool.blocks;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    void* args[] = {&a, &map, &used, &src, &dst, &moves};
    s = kv_cuda(ops_launch((const void*)us_kv_compact_kernel, dim3(1), 1024, 0, st, args));
    Tables here = {};
    here.map = map;
    int i = 0;
    for (; i < n_tables && here.n < kTables; ++i)
        if (tables[i].n_seqs > 0) here.q[here.n++] = kv_seqs(tables + i, 0);
    if (s == US_OK) s = copy(a, src, dst, nullptr, a.pool.blocks, moves, st, &here);
    for (; s == US_OK && i < n_tables; ++i) s = us_kv_remap(h, map, tables + i, stream);
    return s;
}

us_status us_kv_remap(us_kv* h, const int32_t* map, const us_kv_seqs* table, void* stream)
{
    if (!h || !table || !table_ok(h, table) || !map || !kv_aligned(map, 4)) return US_ERR_INVALID_ARG;
    if (table->n_seqs == 0) return US_OK;
    Pages a;
    const us_status s = begin(h, nullptr, &a);
    if (s != US_OK) return s;
    KvSeqs q = kv_seqs(table, 0);
    void* args[] = {&a, &map, &q};
    return kv_cuda(ops_launch((const void*)us_kv_remap_kernel, entries(q.S, q.width), kEntries, 0, static_cast<cudaStream_t>(stream), args));
}
