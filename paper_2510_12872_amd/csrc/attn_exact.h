// Attention of single rows by the formula, key by key, in fp32: a key that a query does not see is not looked at.  The tiled kernels multiply
// whole tiles, where a hidden key has probability 0: with an infinity or NaN among its values the product is NaN.  They check what they
// computed at the end, and a block that holds anything that is not finite computes its rows again here (a launch whose
// every tile meets a NaN is a rare one, and should be right rather than fast).  The time goes by (row, key) pairs, about 8 G a second on a full chip: 8 kv heads, G = 4,
// D = 128, one layer, us without / with a NaN that every query sees: a window of 1024, Tq 512 28.9 / 9540; 4 bits, 4000 keys, one token 9.6 / 69, Tq 512 48 / 8780,
// 32000 keys 19.7 / 579, 220 / 66300 (32 layers, one token 192 / 7250); f32, 4000 keys, Tq 128 109 / 2470.
#pragma once

#include "attn_common.h"
#include "fp4.h"

namespace kvc {

struct fp4_t {};   // element type of a compact cache

// Eight channels from channel c (a multiple of 8) of row `key` of a cache, as floats.
template <typename T>
struct CacheRows {
    const T *base;
    int64_t token;
    template <class P>
    __device__ __forceinline__ CacheRows(const P &p, bool values, int l, int hkv)
    {
        const int64_t layer = values ? p.s_v.layer : p.s_k.layer, head = values ? p.s_v.head : p.s_k.head;
        base = static_cast<const T *>(values ? p.v : p.k) + l * layer + hkv * head;
        token = values ? p.s_v.token : p.s_k.token;
    }
    __device__ __forceinline__ void load8(int key, int c, float (&out)[8]) const
    {
        constexpr int EPV = Elem<T>::EPV;
#pragma unroll
        for (int i = 0; i < 8 / EPV; ++i) {
            float x[EPV];
            unpack<T>(load16(base + (int64_t)key * token + c + i * EPV), x);
#pragma unroll
            for (int j = 0; j < EPV; ++j) out[i * EPV + j] = x[j];
        }
    }
};
template <>
struct CacheRows<fp4_t> {
    const uint8_t *base, *scales;
    int64_t token, s_token;
    template <class P>
    __device__ __forceinline__ CacheRows(const P &p, bool values, int l, int hkv)
    {
        const int64_t layer = values ? p.s_v.layer : p.s_k.layer, head = values ? p.s_v.head : p.s_k.head;
        base = static_cast<const uint8_t *>(values ? p.v : p.k) + l * layer + hkv * head;
        scales = (values ? p.v_scales : p.k_scales) + l * (values ? p.s_vs.layer : p.s_ks.layer) + hkv * (values ? p.s_vs.head : p.s_ks.head);
        token = values ? p.s_v.token : p.s_k.token;
        s_token = values ? p.s_vs.token : p.s_ks.token;
    }
    __device__ __forceinline__ void load8(int key, int c, float (&out)[8]) const
    {
        const uint32_t codes = *reinterpret_cast<const uint32_t *>(base + (int64_t)key * token + c / 2);
        u32x4 raw[2];
        fp4_decode8(codes, fp4_scale(scales[(int64_t)key * s_token + c / 32]), raw);
#pragma unroll
        for (int i = 0; i < 8; ++i) out[i] = __uint_as_float(raw[i >> 2][i & 3]);
    }
};

// Keys of an item: [first, first_end) (sinks) and [begin, end), which do not overlap; what a row does not see of them is left out.
struct KeyRanges {
    int first, first_end, begin, end;
};

// Rows [row0, row0 + n_rows) of the packed (query, head) axis of (layer, kv head) lh: wavefront `wave` of n_waves takes every n_waves-th.
// Results go to `out`, or, where the keys are cut, to the partial results of run `split` (groups of group_rows rows).
template <typename T, typename Q, int D, class P>   // P: AttnParams, in any address space
__device__ __forceinline__ void attn_exact_rows(const P &p, int lh, int row0, int n_rows, KeyRanges keys, int split, int group_rows, int wave,
                                                int n_waves, int lane)
{
    constexpr int CL = D / 8;           // lanes that hold the 8 channels c = 8 * lane of an output row
    const int l = div_by(lh, p.by_Hkv), hkv = lh - l * p.Hkv;
    const CacheRows<T> k(p, false, l, hkv), v(p, true, l, hkv);
#pragma unroll 1
    for (int r = wave; r < n_rows; r += n_waves) {
        const int i = div_by(row0 + r, p.by_G);
        if (i >= p.tq) return;
        const int hq = hkv * p.G + row0 + r - i * p.G, pos = p.n_ctx + i;
        const Q *q = static_cast<const Q *>(p.q) + l * p.s_q.layer + (int64_t)hq * p.s_q.head + (int64_t)i * p.s_q.token;
        float m = -INFINITY, sum = 0.f, o[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) o[j] = 0.f;
#pragma unroll 1
        for (int part = 0; part < 2; ++part) {
            const int begin = part ? keys.begin : keys.first, end = min(part ? keys.end : keys.first_end, pos + 1);
#pragma unroll 1
            for (int key0 = begin; key0 < end && sum == sum; key0 += 64) {   // a key per lane; a sum that is not a number stays so, and the row with it
                const int key = key0 + lane;
                const bool seen = key < end && (p.window == 0 || key > pos - p.window || key < p.n_sinks);
                float s = -INFINITY;
                if (seen) {
                    s = 0.f;
#pragma unroll 1
                    for (int c = 0; c < D; c += 8) {
                        float kk[8], qq[8];
                        k.load8(key, c, kk);
#pragma unroll
                        for (int h = 0; h < 8 / Elem<Q>::EPV; ++h) {
                            float x[Elem<Q>::EPV];
                            unpack<Q>(load16(q + c + h * Elem<Q>::EPV), x);
#pragma unroll
                            for (int j = 0; j < Elem<Q>::EPV; ++j) qq[h * Elem<Q>::EPV + j] = x[j];
                        }
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
                        v.load8(key0 + j, 8 * lane, vv);
#pragma unroll
                        for (int c = 0; c < 8; ++c) o[c] = fmaf(pj, vv[c], o[c]);
                    }
                }
            }
        }
        if (p.n_splits > 1) {
            const int64_t part = ((int64_t)lh * p.n_row_tiles * p.groups_per_tile + (row0 + r) / group_rows) * p.n_splits + split;
            const int n = (row0 + r) % group_rows;
            if (lane < CL) {
                f32x4 *po = reinterpret_cast<f32x4 *>(p.part_o + part * (group_rows * D));
                po[2 * lane * group_rows + n] = f32x4{o[0], o[1], o[2], o[3]};
                po[(2 * lane + 1) * group_rows + n] = f32x4{o[4], o[5], o[6], o[7]};
            }
            if (lane < 2) p.part_ml[part * 2 * group_rows + lane * group_rows + n] = lane ? sum : m;
        } else {
            if (lane < CL) {
                Q *out = static_cast<Q *>(p.out) + l * p.s_o.layer + (int64_t)hq * p.s_o.head + (int64_t)i * p.s_o.token + 8 * lane;
                constexpr int EPV = Elem<Q>::EPV;
#pragma unroll
                for (int h = 0; h < 8 / EPV; ++h) {
                    float x[EPV];
#pragma unroll
                    for (int j = 0; j < EPV; ++j) x[j] = o[h * EPV + j] / sum;
                    *reinterpret_cast<u32x4 *>(out + h * EPV) = pack<Q>(x);
                }
            }
            if (p.lse && lane == 0) p.lse[((int64_t)l * p.Hkv * p.G + hq) * p.tq + i] = m * p.scale + logf(sum);
        }
    }
}

}  // namespace kvc
