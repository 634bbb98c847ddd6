// What the entry points of the 8-bit cache share (internal to the library).
#pragma once
#include "us_kv.cuh"
#include "us_ops.h"

#include <mutex>

struct us_kv {
    us::KvPool pool{};
    int device = -1;      // that the pool lies on; -1: not known (no driver, or memory that is not one device's)
    std::mutex lock;      // of the maps: made by the first attention call
    bool mapped = false;
    CUtensorMap k_map, v_map;
};

namespace us {

constexpr uint32_t kErrFull = 3;   // fewer free blocks than needed (kErrIndex, kErrTimeout: see us_kv.cuh)

// (us_kv.cu) Where kernels leave the last failure on the current device.
us_status kv_error_word(uint32_t** err);

inline us_status kv_cuda(cudaError_t e)
{
    if (e == cudaSuccess) return US_OK;
    cudaGetLastError();
    return US_ERR_CUDA;
}
inline bool kv_aligned(const void* p, int64_t b) { return reinterpret_cast<uintptr_t>(p) % (uintptr_t)b == 0; }
// Whether the current device is the pool's: every call that launches asks.
inline us_status kv_on_device(const us_kv* h)
{
    if (h->device < 0) return US_OK;
    int dev = -1;
    const us_status s = kv_cuda(cudaGetDevice(&dev));
    return s != US_OK ? s : dev == h->device ? US_OK : US_ERR_INVALID_ARG;
}
inline bool kv_seqs_ok(const us_kv* h, const us_kv_seqs* q, int64_t N)
{
    if (!h || !q || N < 0 || N >= (1ll << 31) || q->n_seqs < 0 || (!q->cu_tokens && N != q->n_seqs)) return false;
    if (q->n_seqs == 0 || N == 0) return true;
    return q->block_table && q->lengths && q->table_width >= 1 && (int64_t)q->table_width * h->pool.T < (1ll << 31) - (1 << 16) &&
           (q->n_seqs == 1 || q->table_stride >= q->table_width) && kv_aligned(q->block_table, 4) && kv_aligned(q->lengths, 4) && kv_aligned(q->cu_tokens, 4);
}
inline KvSeqs kv_seqs(const us_kv_seqs* q, int64_t N)
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

}  // namespace us
