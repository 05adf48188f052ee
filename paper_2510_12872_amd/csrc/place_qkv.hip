// kvcomm_place_qkv: a suffix's projected queries, keys and values become what the attention reads.  Every head's query and key is optionally
// divided by its root mean square (and multiplied by a weight per channel), then rotated to its token's position; queries go to their tensor, keys and
// values to their rows of the agent's cache.
//   x' = x / sqrt(mean_c x_c^2 + eps) * w_c;   out_c = x'_c cos - x'_{c + D/2} sin,   out_{c + D/2} = x'_{c + D/2} cos + x'_c sin,
// the angle of pair c being position * theta^(-2c/D).  fp32 throughout, one rounding at the store.
// HBM bound (each value is read and written once); with a token or two the launch is one chain of load, trigonometry, reduction and store.
// A thread owns the 16 bytes of channels c ... and the 16 bytes of c + D/2 ..., both members of its pairs, and keeps its (token, channels)
// from head to head: the cosines and sines, in double up to their rounding, are formed once per thread and stay in registers.
#include <float.h>

#include "kvcomm_device.h"

namespace {

using namespace kvc;

constexpr int kBlock = 256;

struct PlaceParams {
    const void *in[3];      // q, k, v; null: there is none
    void *out[3];
    Strides s_in[3], s_out[3];
    const void *weight[2];  // of queries and keys, [layers, D]; null: ones
    int64_t s_weight[2];    // elements from layer to layer
    int32_t n, first_pos;
    int32_t heads[3];       // 0 where there is no tensor
    int32_t n_heads;        // their sum
    int32_t head_groups, heads_per_group;   // a block's share of the heads
    int32_t n_tiles;        // blocks of tokens
    int32_t log_tokens;     // tokens of a block: 1 << log_tokens
    float eps;              // 0: no norm
    divisor_t by_tiles, by_groups;
    double inv_freq[128];
};

template <typename T, int D>
__global__ __launch_bounds__(kBlock) void place_kernel(const PlaceParams p)
{
    constexpr int EPV = Elem<T>::EPV, LPR = D / 2 / EPV;   // channels of a 16-byte piece, lanes of a row
    const int c = threadIdx.x % LPR, slot = threadIdx.x / LPR;
    const int rest = div_by(blockIdx.x, p.by_tiles), tile = blockIdx.x - rest * p.n_tiles;
    const int l = div_by(rest, p.by_groups), group = rest - l * p.head_groups;
    const int t = (tile << p.log_tokens) + (slot & ((1 << p.log_tokens) - 1));
    const int step = (kBlock / LPR) >> p.log_tokens;       // heads that the block moves at once
    const int end = min((group + 1) * p.heads_per_group, p.n_heads);
    float co[EPV], si[EPV];
#pragma unroll
    for (int i = 0; i < EPV; ++i) {
        const float2 cs = rope_cos_sin(p.first_pos + min(t, p.n - 1), p.inv_freq[c * EPV + i]);
        co[i] = cs.x;
        si[i] = cs.y;
    }
    for (int head = group * p.heads_per_group + (slot >> p.log_tokens); head < end; head += step) {
        const int which = head < p.heads[0] ? 0 : head < p.heads[0] + p.heads[1] ? 1 : 2;
        const int h = head - (which > 0 ? p.heads[0] : 0) - (which > 1 ? p.heads[1] : 0);
        const bool live = t < p.n;
        const int tt = min(t, p.n - 1);
        const T *src = static_cast<const T *>(p.in[which]) + l * p.s_in[which].layer + h * p.s_in[which].head + (int64_t)tt * p.s_in[which].token + c * EPV;
        u32x4 a = load16(src), b = load16(src + D / 2);
        if (which < 2) {
            float x[EPV], y[EPV];
            unpack<T>(a, x);
            unpack<T>(b, y);
            if (p.eps > 0.f) {
                float sum = 0.f;
#pragma unroll
                for (int i = 0; i < EPV; ++i) sum = fmaf(x[i], x[i], fmaf(y[i], y[i], sum));
#pragma unroll
                for (int off = LPR / 2; off >= 1; off >>= 1) sum += __shfl_xor(sum, off);
                const float r = 1.f / sqrtf(sum * (1.f / D) + p.eps);
                float wx[EPV], wy[EPV];
                if (p.weight[which]) {
                    const T *w = static_cast<const T *>(p.weight[which]) + l * p.s_weight[which] + c * EPV;
                    unpack<T>(load16(w), wx);
                    unpack<T>(load16(w + D / 2), wy);
                } else {
#pragma unroll
                    for (int i = 0; i < EPV; ++i) wx[i] = wy[i] = 1.f;
                }
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
            a = pack<T>(x);
            b = pack<T>(y);
        }
        if (live) {
            T *dst = static_cast<T *>(p.out[which]) + l * p.s_out[which].layer + h * p.s_out[which].head + (int64_t)t * p.s_out[which].token + c * EPV;
            *reinterpret_cast<u32x4 *>(dst) = a;
            *reinterpret_cast<u32x4 *>(dst + D / 2) = b;
        }
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
    p.heads_per_group = std::min(p.n_heads, 8 * at_once);
    p.head_groups = (p.n_heads + p.heads_per_group - 1) / p.heads_per_group;
    const int64_t blocks = (int64_t)L * p.head_groups * p.n_tiles;
    if (blocks >= 1 << 24) return KVCOMM_EUNSUPPORTED;   // a launch holds fewer than 2^32 threads along an axis
    p.by_tiles = make_divisor((uint32_t)p.n_tiles);
    p.by_groups = make_divisor((uint32_t)p.head_groups);
    return launch(place_kernel<T, D>, dim3((unsigned)blocks), dim3(kBlock), 0, s, p);
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
    int n_from = 0, n_to = 0;
    for (int i = 0; i < 3; ++i) {
        if (!in[i].ptr && !out[i].ptr) continue;
        if ((st = check_tensor(in[i], dt, true)) || (st = check_tensor(out[i], dt, true))) return st;
        p.in[i] = in[i].ptr;
        p.out[i] = out[i].ptr;
        p.s_in[i] = strides_of(in[i]);
        p.s_out[i] = strides_of(out[i]);
        p.heads[i] = heads[i];
        from[n_from++] = extent_of(in[i], L, heads[i], n_tokens, D, es);
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
    for (int i = 0; i < n_to; ++i) {
        for (int j = 0; j < n_from; ++j)
            if (!(i == j && j < n_pairs && same_extent(to[i], from[j])) && extents_overlap(to[i], from[j])) return KVCOMM_EINVAL;
        for (int j = 0; j < i; ++j)
            if (extents_overlap(to[i], to[j])) return KVCOMM_EINVAL;
    }
    p.n = n_tokens;
    p.first_pos = first_pos;
    const int64_t n_heads = (int64_t)p.heads[0] + p.heads[1] + p.heads[2];
    if (n_heads > INT32_MAX / 2) return KVCOMM_EUNSUPPORTED;
    p.n_heads = (int)n_heads;
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
