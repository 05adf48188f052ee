// Attention of a batch of sequences over the pages of a pool, behind a cache that all of them continue: what its kernels share.
//   out_i = softmax_j(scale <q_i, k_j>) v_j   over the prefix's tokens and the tokens of row i's sequence up to its own.
// The keys of a sequence are counted in halves of tiles, 32 keys each: first the prefix's (the last of which may be short), then those of its pages.  An
// item of work is a tile of packed (row, query head) rows r = i * G + g of one kv head (of one sequence, or of all sequences over
// the prefix) and a run of halves; where a row's halves go to several items, each leaves an unnormalised output, a reference and a sum,
// which attn_paged_combine_kernel joins.
#pragma once

#include "attn_common.h"
#include "paged.h"

namespace kvc {

struct PagedAttnParams {
    const void *q, *k, *v, *prefix_k, *prefix_v;
    void *out;
    float *lse;
    Strides s_q, s_o, s_pk, s_pv;
    PoolStrides s_k, s_v;
    Batch batch;
    int32_t L, Hkv, G, n_prefix;
    float scale, scale_log2;
    divisor_t by_G, by_Hkv;
};

// A sequence's tokens from row i of n on: the last one that it sees, -1 or less: none.
__device__ __forceinline__ int last_seen(int len, int n, int i, int cap) { return min(len - n + i, min(len, cap) - 1); }

// One row (sequence b, row `row` of the queries, query head hq) over the halves [h0, h1) by the formula, key by key, in fp32; what the row does not
// see (`last`: the last token of its pages that it sees) is not looked at.  Whole rows: halves 0 ... of the prefix, then of the pages.
// Returns reference and sum; lanes 0 ... D / 8 - 1 hold channels 8 * lane ... of the unnormalised output.
template <typename T, int D>
__device__ __forceinline__ void paged_exact_row(const PagedAttnParams &p, int l, int hkv, int hq, int row, int b, int last, int prefix_halves, int h0, int h1, int lane,
                                                float &m, float &sum, float (&o)[8])
{
    constexpr int CL = D / 8, EPV = Elem<T>::EPV;
    const T *q = static_cast<const T *>(p.q) + l * p.s_q.layer + (int64_t)hq * p.s_q.head + (int64_t)row * p.s_q.token;
    auto at = [&](int x, bool values) -> const T * {   // row of key x, counted from half 0; null: not there
        if (x < 32 * prefix_halves) {
            if (x >= p.n_prefix) return nullptr;
            const Strides &s = values ? p.s_pv : p.s_pk;
            return static_cast<const T *>(values ? p.prefix_v : p.prefix_k) + l * s.layer + hkv * s.head + (int64_t)x * s.token;
        }
        const int t = x - 32 * prefix_halves;
        if (t > last) return nullptr;
        const int page = page_of(p.batch, b, t);
        if (page < 0) return nullptr;
        const PoolStrides &s = values ? p.s_v : p.s_k;
        return static_cast<const T *>(values ? p.v : p.k) + l * s.layer + hkv * s.head + (int64_t)page * s.page + (int64_t)(t & ((1 << p.batch.log_page) - 1)) * s.token;
    };
    auto load8 = [](const T *src, float (&x)[8]) {
#pragma unroll
        for (int i = 0; i < 8 / EPV; ++i) {
            float y[EPV];
            unpack<T>(load16(src + i * EPV), y);
#pragma unroll
            for (int j = 0; j < EPV; ++j) x[i * EPV + j] = y[j];
        }
    };
    m = -INFINITY;
    sum = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) o[j] = 0.f;
    const int end = (int)min((int64_t)32 * h1, (int64_t)32 * prefix_halves + last + 1);
#pragma unroll 1
    for (int x0 = 32 * h0; x0 < end && sum == sum; x0 += 64) {   // a key per lane; a sum that is not a number stays so, and the row with it
        const T *kr = x0 + lane < end ? at(x0 + lane, false) : nullptr;
        const bool seen = kr != nullptr;
        float s = -INFINITY;
        if (seen) {
            s = 0.f;
#pragma unroll 1
            for (int c = 0; c < D; c += 8) {
                float kk[8], qq[8];
                load8(kr + c, kk);
                load8(q + c, qq);
#pragma unroll
                for (int j = 0; j < 8; ++j) s = fmaf(qq[j], kk[j], s);
            }
        }
        float mx = s;
#pragma unroll
        for (int off = 32; off >= 1; off >>= 1) mx = fmaxf(mx, __shfl_xor(mx, off));
        const float m_new = fmaxf(m, mx);
        const float corr = m == -INFINITY ? 0.f : exp2f((m - m_new) * p.scale_log2);
        m = m_new;
        const float e = seen ? exp2f((s - (m == -INFINITY ? 0.f : m)) * p.scale_log2) : 0.f;
        float es = e;
#pragma unroll
        for (int off = 32; off >= 1; off >>= 1) es += __shfl_xor(es, off);
        sum = sum * corr + es;
#pragma unroll
        for (int j = 0; j < 8; ++j) o[j] *= corr;
        for (uint64_t todo = __builtin_amdgcn_ballot_w64(seen); todo; todo &= todo - 1) {
            const int j = __builtin_ctzll(todo);
            const float pj = __shfl(e, j);
            if (lane < CL) {
                float vv[8];
                load8(at(x0 + j, true) + 8 * lane, vv);
#pragma unroll
                for (int c = 0; c < 8; ++c) o[c] = fmaf(pj, vv[c], o[c]);
            }
        }
    }
}

// The row's result.  A row that saw nothing: 0 and -infinity.
template <typename T, int D>
__device__ __forceinline__ void paged_store_row(const PagedAttnParams &p, int l, int hq, int row, int lane, float m, float sum, const float (&o)[8])
{
    constexpr int EPV = Elem<T>::EPV;
    const bool none = m == -INFINITY && sum == 0.f;
    if (lane < D / 8) {
        T *out = static_cast<T *>(p.out) + l * p.s_o.layer + (int64_t)hq * p.s_o.head + (int64_t)row * p.s_o.token + 8 * lane;
#pragma unroll
        for (int h = 0; h < 8 / EPV; ++h) {
            float x[EPV];
#pragma unroll
            for (int j = 0; j < EPV; ++j) x[j] = none ? 0.f : o[h * EPV + j] / sum;
            *reinterpret_cast<u32x4 *>(out + h * EPV) = pack<T>(x);
        }
    }
    if (p.lse && lane == 0) p.lse[((int64_t)l * p.Hkv * p.G + hq) * p.batch.n_rows + row] = none ? -INFINITY : m * p.scale + logf(sum);
}

}  // namespace kvc
