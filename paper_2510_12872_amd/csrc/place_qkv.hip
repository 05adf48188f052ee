// kvcomm_place_qkv: a suffix's projected queries, keys and values become what the attention reads.  Every head's query and key is optionally
// divided by its root mean square (and multiplied by a weight per channel), then rotated to its token's position; queries go to their tensor, keys and
// values to their rows of the agent's cache.
//   x' = x / sqrt(mean_c x_c^2 + eps) * w_c;   out_c = x'_c cos - x'_{c + D/2} sin,   out_{c + D/2} = x'_{c + D/2} cos + x'_c sin,
// the angle of pair c being position * theta^(-2c/D).  fp32 throughout, one rounding at the store.
// HBM bound (each value is read and written once: 402 MB of 32 layers x 512 tokens in 75 us, 5.4 TB/s, a copy's rate; 63 us on the same tensors again and again, part of
// which the last-level cache then holds); with a token or two the launch is one chain of load, trigonometry, reduction and store (2.6 us; 3.6 us from launch to launch).
// A thread owns the 16 bytes of channels c ... and the 16 bytes of c + D/2 ..., both members of its pairs, and keeps its (token, channels)
// from head to head: the cosines and sines, in double up to their rounding, are formed once per thread and stay in registers.
// kvcomm_place_qkv_paged: the same kernel for the rows of a batch; a row's sequence, position and slot are found while its values travel.  What bounds it is the same:
// 32 layers, six prompts of 100 to 1200 tokens with norms (2.55 GB) 494 us = 5.2 TB/s, half read and half written (a copy of 2 GiB: 4.9); a token of 8 sequences, one layer, 3.6 us.
#include <float.h>

#include <type_traits>

#include "paged.h"

namespace {

using namespace kvc;

constexpr int kBlock = 256;

// Sum over the LPR neighbouring lanes of a row (4, 8, 16, 32), in all of them.
template <int LPR>
__device__ __forceinline__ float row_sum(float x)
{
    auto add = [](float v, auto ctrl) { return v + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), decltype(ctrl)::value, 0xf, 0xf, true)); };
    x = add(x, std::integral_constant<int, 0xB1>{});                       // lanes 1, 0, 3, 2
    x = add(x, std::integral_constant<int, 0x4E>{});                       // lanes 2, 3, 0, 1
    if constexpr (LPR >= 8) x = add(x, std::integral_constant<int, 0x141>{});    // mirrored in eight
    if constexpr (LPR >= 16) x = add(x, std::integral_constant<int, 0x140>{});   // mirrored in sixteen
    if constexpr (LPR >= 32) x += __shfl_xor(x, 16);
    return x;
}

struct PlaceParams {
    const void *in[3];      // q, k, v; null: there is none
    void *out[3];
    Strides s_in[3], s_out[3];
    const void *weight[2];  // of queries and keys, [layers, D]; null: ones
    int64_t s_weight[2];    // elements from layer to layer
    int32_t n, first_pos;
    int32_t heads[3];
    int32_t group_end[3];   // groups of heads up to this tensor's last: a block moves one group of one tensor
    int32_t heads_per_group;
    int32_t n_tiles;        // blocks of tokens
    int32_t log_tokens;     // tokens of a block: 1 << log_tokens
    float eps;              // 0: no norm
    divisor_t by_tiles, by_groups;
    double inv_freq[128];
};

// Of a batch: outs of keys and values are pools, their strides those of a slot.
struct PagedPlaceParams : PlaceParams {
    Batch batch;
    int64_t page[2];   // from page to page
};

// NORM: eps > 0.  U: heads whose loads a thread has in flight together (two as fast as four: 62.7 and 63.3 us for 32 layers x 512 tokens, the same ones every time).
template <typename T, int D, bool NORM, int U, class P>
__global__ __launch_bounds__(kBlock) void place_kernel(const P p)
{
    constexpr bool PAGED = std::is_same_v<P, PagedPlaceParams>;
    constexpr int EPV = Elem<T>::EPV, LPR = D / 2 / EPV;   // channels of a 16-byte piece, lanes of a row
    const int c = threadIdx.x % LPR, slot = threadIdx.x / LPR;
    double freq[EPV];   // the arguments lie in memory that no cache holds yet: all that is needed of them is requested first (one token 3.8 -> 3.6 us)
#pragma unroll
    for (int i = 0; i < EPV; ++i) freq[i] = p.inv_freq[c * EPV + i];
    await_args(arg_word(&p), arg_word(&p.s_in[1]), arg_word(&p.s_out), arg_word(&p.s_out[2]));
    await_args(arg_word(&p.heads), arg_word(&p.by_groups));
    const int rest = div_by(blockIdx.x, p.by_tiles), tile = blockIdx.x - rest * p.n_tiles;
    const int l = div_by(rest, p.by_groups), group = rest - l * p.group_end[2];
    const int which = group < p.group_end[0] ? 0 : group < p.group_end[1] ? 1 : 2;
    const int head0 = (group - (which ? p.group_end[which - 1] : 0)) * p.heads_per_group;
    const int end = min(head0 + p.heads_per_group, p.heads[which]);
    const int t = (tile << p.log_tokens) + (slot & ((1 << p.log_tokens) - 1));
    const int step = (kBlock / LPR) >> p.log_tokens;       // heads that the block moves at once
    bool live = t < p.n;
    const int tt = min(t, p.n - 1);
    int head = head0 + (slot >> p.log_tokens);
    const int64_t in_head = p.s_in[which].head, out_head = p.s_out[which].head;
    const T *src = static_cast<const T *>(p.in[which]) + l * p.s_in[which].layer + (int64_t)tt * p.s_in[which].token + c * EPV;
    T *dst = static_cast<T *>(p.out[which]) + l * p.s_out[which].layer + (int64_t)tt * p.s_out[which].token + c * EPV;
    u32x4 a[U], b[U];
    auto load = [&](int h0) {
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const T *row = src + (int64_t)min(h0 + i * step, end - 1) * in_head;
            a[i] = load16_stream(row);
            b[i] = load16_stream(row + D / 2);
        }
    };
    auto store = [&](int i, int h) {
        if (live && h < end) {
            *reinterpret_cast<u32x4 *>(dst + (int64_t)h * out_head) = a[i];
            *reinterpret_cast<u32x4 *>(dst + (int64_t)h * out_head + D / 2) = b[i];
        }
    };
    load(head);
    int pos = p.first_pos + tt;
    if constexpr (PAGED) {
        const int b = sequence_of(p.batch, tt, threadIdx.x & 63), bb = max(b, 0);
        int first, n;
        sequence_rows(p.batch, bb, first, n);
        const int i = tt - first, token = sequence_len(p.batch, bb) - n + i;
        live &= b >= 0 && i >= 0 && i < n;
        pos = (int)max((int64_t)INT32_MIN, min((int64_t)INT32_MAX, (int64_t)p.first_pos + token));   // (beyond: in no page)
        if (which) {
            const int page = live && token >= 0 ? page_of(p.batch, bb, token) : -1;
            live &= page >= 0;
            const int slot = token & ((1 << p.batch.log_page) - 1);
            dst += (live ? (int64_t)page * p.page[which - 1] + (int64_t)slot * p.s_out[which].token : 0) - (int64_t)tt * p.s_out[which].token;
        }
    }
    if (which == 2) {
        while (true) {
#pragma unroll
            for (int i = 0; i < U; ++i) store(i, head + i * step);
            head += U * step;
            if (head >= end) return;
            load(head);
        }
    }
    u32x4 w_raw[2];
    if constexpr (NORM) {
        if (p.weight[which]) {
            const T *w = static_cast<const T *>(p.weight[which]) + l * p.s_weight[which] + c * EPV;
            w_raw[0] = load16(w);
            w_raw[1] = load16(w + D / 2);
        }
    }
    float co[EPV], si[EPV];
#pragma unroll
    for (int i = 0; i < EPV; ++i) {
        const float2 cs = rope_cos_sin(pos, freq[i]);
        co[i] = cs.x;
        si[i] = cs.y;
    }
    float wx[EPV], wy[EPV];
    if constexpr (NORM) {
        if (p.weight[which]) {
            unpack<T>(w_raw[0], wx);
            unpack<T>(w_raw[1], wy);
        } else {
#pragma unroll
            for (int i = 0; i < EPV; ++i) wx[i] = wy[i] = 1.f;
        }
    }
    while (true) {
#pragma unroll
        for (int k = 0; k < U; ++k) {
            float x[EPV], y[EPV];
            unpack<T>(a[k], x);
            unpack<T>(b[k], y);
            if constexpr (NORM) {
                float sum = 0.f;
#pragma unroll
                for (int i = 0; i < EPV; ++i) sum = fmaf(x[i], x[i], fmaf(y[i], y[i], sum));
                sum = row_sum<LPR>(sum);
                const float r = 1.f / sqrtf(sum * (1.f / D) + p.eps);
#pragma unroll
                for (int i = 0; i < EPV; ++i) {
                    x[i] *= r * wx[i];
                    y[i] *= r * wy[i];
                }
            }
#pragma unroll
            for (int i = 0; i < EPV; ++i) {
                const float u = x[i], v = y[i];
                x[i] = u * co[i] - v * si[i];
                y[i] = v * co[i] + u * si[i];
            }
            a[k] = pack<T>(x);
            b[k] = pack<T>(y);
            store(k, head + k * step);
        }
        head += U * step;
        if (head >= end) return;   // (the lanes of a row go together)
        load(head);
    }
}

template <typename T, int D, class P>
int launch_place(P &p, int L, hipStream_t s)
{
    constexpr int rows = kBlock / (D / 2 / Elem<T>::EPV);   // of a block at once
    p.log_tokens = 0;
    while ((1 << p.log_tokens) < std::min(p.n, rows)) ++p.log_tokens;
    p.n_tiles = (int)(((int64_t)p.n + (1 << p.log_tokens) - 1) >> p.log_tokens);
    const int at_once = rows >> p.log_tokens;
    // A thread moves four heads, fewer where the launch would have less than half a block per unit.  32 query and 8 kv heads, D = 128, norm, us on the same tensors every time with 1 / 2 / 4 / 8 / 16
    // heads: 32 layers x 512 tokens 84.7 / 65.1 / 62.7 / 64.2 / 68.9, one layer 32 tokens 4.0 / 4.3 / 5.1 / 6.8 / 9.4, 512 tokens 6.1 / 5.9 / 5.9 / 7.6 / 10.1.
    int64_t groups = 0, blocks = 0;
    for (int heads = 4; heads >= 1 && blocks < 128; heads /= 2) {
        p.heads_per_group = heads * at_once;
        groups = 0;
        for (int i = 0; i < 3; ++i) p.group_end[i] = (int)(groups += (p.heads[i] + p.heads_per_group - 1) / p.heads_per_group);
        blocks = L * groups * p.n_tiles;
    }
    if (blocks >= 1 << 24) return KVCOMM_EUNSUPPORTED;   // a launch holds fewer than 2^32 threads along an axis
    p.by_tiles = make_divisor((uint32_t)p.n_tiles);
    p.by_groups = make_divisor((uint32_t)groups);
    const auto one = p.eps > 0.f ? place_kernel<T, D, true, 1, P> : place_kernel<T, D, false, 1, P>;
    const auto two = p.eps > 0.f ? place_kernel<T, D, true, 2, P> : place_kernel<T, D, false, 2, P>;
    return launch(p.heads_per_group == at_once ? one : two, dim3((unsigned)blocks), dim3(kBlock), 0, s, p);
}

template <class P>
int launch_place(const kvcomm_model &m, P &p, hipStream_t s)
{
    const bool f32 = m.dtype == KVCOMM_F32;
    switch (m.head_dim) {
        case 64: return f32 ? launch_place<float, 64>(p, m.n_layers, s) : launch_place<bf16_t, 64>(p, m.n_layers, s);
        case 128: return f32 ? launch_place<float, 128>(p, m.n_layers, s) : launch_place<bf16_t, 128>(p, m.n_layers, s);
        default: return f32 ? launch_place<float, 256>(p, m.n_layers, s) : launch_place<bf16_t, 256>(p, m.n_layers, s);
    }
}

}  // namespace

extern "C" int kvcomm_place_qkv(const kvcomm_model *model, kvcomm_tensor q, kvcomm_tensor k, kvcomm_tensor v, int32_t n_tokens, int32_t first_pos,
                                const void *q_weight, const void *k_weight, int64_t q_weight_stride, int64_t k_weight_stride, float norm_eps,
                                kvcomm_tensor q_out, kvcomm_tensor k_out, kvcomm_tensor v_out, void *stream)
{
    int st = check_model(model);
    if (st) return st;
    if (n_tokens <= 0 || (int64_t)first_pos + n_tokens - 1 > INT32_MAX) return KVCOMM_EINVAL;
    if (!(norm_eps >= 0.f) || norm_eps > FLT_MAX) return KVCOMM_EINVAL;
    const int dt = model->dtype, es = elem_size(dt), D = model->head_dim, L = model->n_layers;
    const kvcomm_tensor in[3] = {q, k, v}, out[3] = {q_out, k_out, v_out};
    const int heads[3] = {model->n_q_heads, model->n_kv_heads, model->n_kv_heads};
    const void *weight[2] = {q_weight, k_weight};
    const int64_t w_stride[2] = {q_weight_stride, k_weight_stride};
    PlaceParams p{};
    Extent from[5], to[3];
    int n_from = 0, n_to = 0, is[3];
    for (int i = 0; i < 3; ++i) {
        if (!in[i].ptr && !out[i].ptr) continue;
        if ((st = check_tensor(in[i], dt, true)) || (st = check_tensor(out[i], dt, true))) return st;
        p.in[i] = in[i].ptr;
        p.out[i] = out[i].ptr;
        p.s_in[i] = strides_of(in[i]);
        p.s_out[i] = strides_of(out[i]);
        p.heads[i] = heads[i];
        from[n_from++] = extent_of(in[i], L, heads[i], n_tokens, D, es);
        is[n_to] = i;
        to[n_to++] = extent_of(out[i], L, heads[i], n_tokens, D, es);
    }
    if (n_to == 0) return KVCOMM_EINVAL;
    const int n_pairs = n_to;
    for (int i = 0; i < 2; ++i) {
        if (!weight[i]) continue;
        if (norm_eps == 0.f || !p.in[i]) return KVCOMM_EINVAL;   // a weight that nothing would be multiplied by
        const kvcomm_tensor w = {const_cast<void *>(weight[i]), w_stride[i], 0, 0};
        if ((st = check_tensor(w, dt, true))) return st;
        p.weight[i] = weight[i];
        p.s_weight[i] = w_stride[i];
        from[n_from++] = extent_of(w, L, 1, 1, D, es);
    }
    auto apart = [&](int i, int j, const kvcomm_tensor &y) { return beside_each_other(out[is[i]], heads[is[i]], D * es, es, y, heads[is[j]], D * es, es, L); };
    for (int i = 0; i < n_to; ++i) {
        for (int j = 0; j < n_from; ++j) {
            const bool pair = j < n_pairs;
            if (!(i == j && pair && same_extent(to[i], from[j])) && extents_overlap(to[i], from[j]) && !(pair && apart(i, j, in[is[j]]))) return KVCOMM_EINVAL;
        }
        for (int j = 0; j < i; ++j)
            if (extents_overlap(to[i], to[j]) && !apart(i, j, out[is[j]])) return KVCOMM_EINVAL;
    }
    p.n = n_tokens;
    p.first_pos = first_pos;
    p.eps = norm_eps;
    fill_inv_freq(p.inv_freq, model->rope_theta, D);
    return launch_place(*model, p, static_cast<hipStream_t>(stream));
}

namespace {

// A pool as the caller described it: four axes of rows of `row` bytes, strides in bytes.
struct PoolExtent {
    uintptr_t base;
    int64_t stride[4], row;
    int32_t n[4];
    uintptr_t hi() const
    {
        uintptr_t end = base + (uintptr_t)row;
        for (int i = 0; i < 4; ++i) end += (uintptr_t)((n[i] - 1) * stride[i]);
        return end;
    }
};

PoolExtent extent_of(const kvcomm_pages &t, const kvcomm_model &m, const kvcomm_batch &b)
{
    const int es = elem_size(m.dtype);
    PoolExtent e = {reinterpret_cast<uintptr_t>(t.ptr), {t.stride_layer * es, t.stride_head * es, t.stride_page * es, t.stride_token * es},
                    (int64_t)m.head_dim * es, {m.n_layers, m.n_kv_heads, b.n_pages, b.page_size}};
    for (int i = 1; i < 4; ++i)   // longest stride first
        for (int j = i; j > 0 && e.stride[j - 1] < e.stride[j]; --j) {
            std::swap(e.stride[j - 1], e.stride[j]);
            std::swap(e.n[j - 1], e.n[j]);
        }
    return e;
}

// Do rows of two pools of the same strides and sizes meet, the second one's base `d` bytes behind the first's?  Some sum of d and multiples |k_i| < n_i of
// the strides from axis `i` on then lies within a row.  What the shorter strides reach leaves few k_i of each; many (strides that do not nest) count as met.
bool rows_meet(const PoolExtent &e, int i, int64_t d)
{
    if (i == 4) return d > -e.row && d < e.row;
    int64_t reach = e.row;
    for (int j = i + 1; j < 4; ++j) reach += (e.n[j] - 1) * e.stride[j];
    if (e.stride[i] == 0) return rows_meet(e, i + 1, d);
    const int64_t lo = std::max<int64_t>(floor_div(-reach - d, e.stride[i]) + 1, -(int64_t)(e.n[i] - 1));
    const int64_t hi = std::min<int64_t>(-floor_div(d - reach, e.stride[i]) - 1, e.n[i] - 1);
    if (hi - lo > 4) return true;
    for (int64_t k = lo; k <= hi; ++k)
        if (rows_meet(e, i + 1, d + k * e.stride[i])) return true;
    return false;
}

bool pools_meet(const PoolExtent &a, const PoolExtent &b)
{
    if (a.hi() <= b.base || b.hi() <= a.base) return false;
    for (int i = 0; i < 4; ++i)
        if (a.stride[i] != b.stride[i] || a.n[i] != b.n[i]) return true;
    return rows_meet(a, 0, (int64_t)(b.base - a.base));
}

}  // namespace

extern "C" int kvcomm_place_qkv_paged(const kvcomm_model *model, kvcomm_tensor q, kvcomm_tensor k, kvcomm_tensor v, const kvcomm_batch *batch,
                                      int32_t first_pos, const void *q_weight, const void *k_weight, int64_t q_weight_stride,
                                      int64_t k_weight_stride, float norm_eps, kvcomm_tensor q_out, kvcomm_pages pages_k, kvcomm_pages pages_v, void *stream)
{
    int st = check_model(model);
    if (st) return st;
    PagedPlaceParams p{};
    if ((st = check_batch(batch, p.batch))) return st;
    const int dt = model->dtype, es = elem_size(dt), D = model->head_dim, L = model->n_layers, n = batch->n_rows;
    if ((int64_t)first_pos + p.batch.cap > INT32_MAX) return KVCOMM_EINVAL;
    if (!(norm_eps >= 0.f) || norm_eps > FLT_MAX) return KVCOMM_EINVAL;
    if ((double)L * ((double)model->n_q_heads + 2.0 * model->n_kv_heads) * n * D >= 34359738368.0) return KVCOMM_EUNSUPPORTED;   // 2^35 values: see launch_place()
    const bool pages = p.batch.cap > 0;   // else there is nothing to store into: keys and values are not looked at
    const kvcomm_tensor in[3] = {q, k, v};
    const kvcomm_pages *pool[2] = {&pages_k, &pages_v};
    const int heads[3] = {model->n_q_heads, model->n_kv_heads, model->n_kv_heads};
    const void *weight[2] = {q_weight, k_weight};
    const int64_t w_stride[2] = {q_weight_stride, k_weight_stride};
    Extent from[5];
    int n_from = 0, of[5] = {3, 3, 3, 3, 3};   // which of the inputs, 3: a weight
    for (int i = 0; i < 3; ++i) {
        const void *out = i ? (pages ? pool[i - 1]->ptr : in[i].ptr) : q_out.ptr;
        if (!in[i].ptr && !out) continue;
        if ((st = check_tensor(in[i], dt, true)) || (st = i ? (pages ? check_pages(*pool[i - 1], dt) : KVCOMM_OK) : check_tensor(q_out, dt, true))) return st;
        of[n_from] = i;
        from[n_from++] = extent_of(in[i], L, heads[i], n, D, es);
        if (i && !pages) continue;
        p.in[i] = in[i].ptr;
        p.out[i] = const_cast<void *>(out);
        p.s_in[i] = strides_of(in[i]);
        p.s_out[i] = i ? Strides{pool[i - 1]->stride_layer, pool[i - 1]->stride_head, pool[i - 1]->stride_token} : strides_of(q_out);
        if (i) p.page[i - 1] = pool[i - 1]->stride_page;
        p.heads[i] = heads[i];
    }
    if (n_from == 0) return KVCOMM_EINVAL;
    for (int i = 0; i < 2; ++i) {
        if (!weight[i]) continue;
        if (norm_eps == 0.f || !in[i].ptr) return KVCOMM_EINVAL;
        const kvcomm_tensor w = {const_cast<void *>(weight[i]), w_stride[i], 0, 0};
        if ((st = check_tensor(w, dt, true))) return st;
        p.weight[i] = weight[i];
        p.s_weight[i] = w_stride[i];
        from[n_from++] = extent_of(w, L, 1, 1, D, es);
    }
    // What the device reads of the batch is an input, too.
    const int64_t entries = p.batch.cap ? ((int64_t)batch->n_seqs - 1) * batch->table_stride + batch->table_width : 0;
    const Extent ints[3] = {extent_flat(batch->lens, 4 * (size_t)batch->n_seqs), extent_flat(batch->starts, batch->starts ? 4 * ((size_t)batch->n_seqs + 1) : 0),
                            extent_flat(batch->table, 4 * (size_t)entries)};
    auto within = [](const Extent &x, uintptr_t lo, uintptr_t hi) { return x.lo() < hi && lo < x.hi() && x.run > 0; };
    PoolExtent to[2] = {};
    for (int i = 0; i < 2; ++i) {
        if (!p.out[i + 1]) continue;
        to[i] = extent_of(*pool[i], *model, *batch);
        for (int j = 0; j < n_from; ++j)
            if (within(from[j], to[i].base, to[i].hi())) return KVCOMM_EINVAL;
        for (const Extent &x : ints)
            if (within(x, to[i].base, to[i].hi())) return KVCOMM_EINVAL;
    }
    if (p.out[1] && p.out[2] && pools_meet(to[0], to[1])) return KVCOMM_EINVAL;
    if (p.out[0]) {
        const Extent out = extent_of(q_out, L, heads[0], n, D, es);
        for (int j = 0; j < n_from; ++j) {
            const int i = of[j];
            if (i == 0 && same_extent(out, from[j])) continue;
            if (extents_overlap(out, from[j]) && !(i < 3 && beside_each_other(q_out, heads[0], D * es, es, in[i], heads[i], D * es, es, L))) return KVCOMM_EINVAL;
        }
        for (const Extent &x : ints)
            if (within(x, out.lo(), out.hi())) return KVCOMM_EINVAL;
        for (int i = 0; i < 2; ++i)
            if (p.out[i + 1] && within(out, to[i].base, to[i].hi())) return KVCOMM_EINVAL;
    }
    if (!p.out[0] && !p.out[1] && !p.out[2]) return KVCOMM_OK;   // keys and values alone, and no page to store them in
    p.n = n;
    p.first_pos = first_pos;
    p.eps = norm_eps;
    fill_inv_freq(p.inv_freq, model->rope_theta, D);
    return launch_place(*model, p, static_cast<hipStream_t>(stream));
}
