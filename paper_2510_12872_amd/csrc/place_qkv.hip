// kvcomm_place_qkv: a suffix's projected queries, keys and values become what the attention reads.  Every head's query and key is optionally
// divided by its root mean square (and multiplied by a weight per channel), then rotated to its token's position; queries go to their tensor, keys and
// values to their rows of the agent's cache.
//   x' = x / sqrt(mean_c x_c^2 + eps) * w_c;   out_c = x'_c cos - x'_{c + D/2} sin,   out_{c + D/2} = x'_{c + D/2} cos + x'_c sin,
// the angle of pair c being position * theta^(-2c/D).  fp32 throughout, one rounding at the store.
// HBM bound (each value is read and written once: 402 MB of 32 layers x 512 tokens in 75 us, 5.4 TB/s, a copy's rate; 63 us on the same tensors again and again, part of
// which the last-level cache then holds); with a token or two the launch is one chain of load, trigonometry, reduction and store (2.6 us; 3.6 us from launch to launch).
// A thread owns the 16 bytes of channels c ... and the 16 bytes of c + D/2 ..., both members of its pairs, and keeps its (token, channels)
// from head to head: the cosines and sines, in double up to their rounding, are formed once per thread and stay in registers.
#include <float.h>

#include <type_traits>

#include "kvcomm_device.h"

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

// NORM: eps > 0.  U: heads whose loads a thread has in flight together (two as fast as four: 62.7 and 63.3 us for 32 layers x 512 tokens, the same ones every time).
template <typename T, int D, bool NORM, int U>
__global__ __launch_bounds__(kBlock) void place_kernel(const PlaceParams p)
{
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
    const bool live = t < p.n;
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
        const float2 cs = rope_cos_sin(p.first_pos + tt, freq[i]);
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

template <typename T, int D>
int launch_place(PlaceParams &p, int L, hipStream_t s)
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
    const auto one = p.eps > 0.f ? place_kernel<T, D, true, 1> : place_kernel<T, D, false, 1>;
    const auto two = p.eps > 0.f ? place_kernel<T, D, true, 2> : place_kernel<T, D, false, 2>;
    return launch(p.heads_per_group == at_once ? one : two, dim3((unsigned)blocks), dim3(kBlock), 0, s, p);
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
    hipStream_t s = static_cast<hipStream_t>(stream);
    const bool f32 = dt == KVCOMM_F32;
    switch (D) {
        case 64: return f32 ? launch_place<float, 64>(p, L, s) : launch_place<bf16_t, 64>(p, L, s);
        case 128: return f32 ? launch_place<float, 128>(p, L, s) : launch_place<bf16_t, 128>(p, L, s);
        default: return f32 ? launch_place<float, 256>(p, L, s) : launch_place<bf16_t, 256>(p, L, s);
    }
}
