// What the calls on batches of sequences in pages share: the batch as the kernels see it, and its checks.
#pragma once

#include "kvcomm_device.h"

namespace kvc {

struct PoolStrides {
    int64_t layer, head, page, token;
};
static inline PoolStrides strides_of(const kvcomm_pages &t) { return PoolStrides{t.stride_layer, t.stride_head, t.stride_page, t.stride_token}; }

struct Batch {
    const int32_t *table, *lens, *starts;   // starts null: one row per sequence
    int64_t table_stride;
    int32_t n_seqs, n_rows;
    int32_t n_pages, log_page;
    int32_t cap;   // tokens that a sequence's entries of the table reach; 0: there are no pages
};

// Rows of a sequence, and its tokens.  Whatever starts and lens hold, rows stay in [0, n_rows).
template <class B>   // Batch, in any address space
__device__ __forceinline__ void sequence_rows(const B &p, int b, int &first, int &n)
{
    if (!p.starts) {
        first = b;
        n = 1;
        return;
    }
    first = max(0, min(p.starts[b], p.n_rows));
    n = max(0, min(p.starts[b + 1], p.n_rows) - first);
}
template <class B>
__device__ __forceinline__ int sequence_len(const B &p, int b) { return max(0, p.lens[b]); }

// Sequence of a row, -1: none.  Each lane of the wavefront may ask for another row.
__device__ __forceinline__ int sequence_of(const Batch &p, int row, int lane)
{
    if (!p.starts) return row < p.n_seqs ? row : -1;
    int b = 0;
    if (p.n_seqs <= 64) {   // all ends in one load, the search between registers
        const int end = lane < p.n_seqs ? p.starts[lane + 1] : INT32_MAX, first = p.starts[0];
#pragma unroll
        for (int step = 32; step >= 1; step >>= 1)
            if (__shfl(end, b + step - 1) <= row) b += step;
        b += __shfl(end, b) <= row ? 1 : 0;
        return row >= first && b < p.n_seqs ? b : -1;
    }
    int n = p.n_seqs;   // ends before `b` are known not to lie behind the row, those from b + n on to do
    while (n > 0) {
        const int half = n >> 1;
        if (p.starts[b + half + 1] <= row) {
            b += half + 1;
            n -= half + 1;
        } else {
            n = half;
        }
    }
    return row >= p.starts[0] && b < p.n_seqs ? b : -1;
}

// Page of token t >= 0 of the sequence, -1: none.
template <class B>
__device__ __forceinline__ int page_of(const B &p, int b, int t)
{
    if (t >= p.cap) return -1;
    const int e = p.table[(int64_t)b * p.table_stride + (t >> p.log_page)];
    return (uint32_t)e < (uint32_t)p.n_pages ? e : -1;
}

// ------------------------------------------------------------------------- host-side checks
static inline int check_pages(const kvcomm_pages &t, int dtype)
{
    const int st = check_tensor(kvcomm_tensor{t.ptr, t.stride_layer, t.stride_head, t.stride_token}, dtype, true);
    return st ? st : check_tensor(kvcomm_tensor{nullptr, t.stride_page, 0, 0}, dtype, false);
}

static inline bool aligned4(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

constexpr int64_t kMaxPagedTokens = (int64_t)1 << 30;

static inline int check_batch(const kvcomm_batch *b, Batch &out)
{
    if (!b || !b->lens || !aligned4(b->lens) || !aligned4(b->starts) || !aligned4(b->table)) return KVCOMM_EINVAL;
    if (b->n_seqs <= 0 || b->n_rows <= 0 || b->table_width < 0 || b->n_pages < 0 || b->table_stride < 0 || b->max_rows < 0 || b->page_size <= 0) return KVCOMM_EINVAL;
    if (!b->starts && b->n_rows != b->n_seqs) return KVCOMM_EINVAL;
    if (b->page_size < 16 || b->page_size > 65536 || (b->page_size & (b->page_size - 1))) return KVCOMM_EUNSUPPORTED;
    if (b->n_seqs > KVCOMM_MAX_SEQS || (int64_t)b->table_width * b->page_size > kMaxPagedTokens) return KVCOMM_EUNSUPPORTED;
    const bool pages = b->table_width > 0 && b->n_pages > 0;
    if (pages && !b->table) return KVCOMM_EINVAL;
    out = Batch{b->table, b->lens, b->starts, b->table_stride, b->n_seqs, b->n_rows, b->n_pages, __builtin_ctz((unsigned)b->page_size),
                pages ? b->table_width * b->page_size : 0};
    return KVCOMM_OK;
}

}  // namespace kvc
