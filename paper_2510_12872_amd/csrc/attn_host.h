// What the attention calls check and fill in alike.
#pragma once

#include "attn_plan.h"
#include "fp4.h"

namespace kvc {

// Checks of every attention call but those of its cache, and the parameters that depend on no plan.
static inline int attn_params(const kvcomm_model *model, const kvcomm_tensor &q, int32_t n_ctx, int32_t tq, float softmax_scale, const kvcomm_tensor &out,
                              float *lse_out, AttnParams &p)
{
    int st = check_model(model);
    if (st) return st;
    if (tq <= 0 || n_ctx < 0) return KVCOMM_EINVAL;
    if ((st = check_tensor(q, model->dtype, true)) || (st = check_tensor(out, model->dtype, true))) return st;
    p.q = q.ptr;
    p.out = out.ptr;
    p.lse = lse_out;
    p.s_q = strides_of(q);
    p.s_o = strides_of(out);
    p.L = model->n_layers;
    p.Hkv = model->n_kv_heads;
    p.G = model->n_q_heads / model->n_kv_heads;
    p.n_ctx = n_ctx;
    p.tq = tq;
    p.N = (int32_t)((int64_t)n_ctx + tq);   // (refused if it does not fit)
    p.scale = softmax_scale > 0.f ? softmax_scale : (float)(1.0 / sqrt((double)model->head_dim));
    p.scale_log2 = (float)((double)p.scale * 1.4426950408889634);
    p.n_splits = 1;
    p.groups_per_tile = 1;
    return KVCOMM_OK;
}

// The cache of a call, [L, Hkv, n_ctx + tq, D] of the model's type.
static inline int attn_cache(const kvcomm_model &model, const kvcomm_tensor &k, const kvcomm_tensor &v, AttnParams &p)
{
    int st;
    if ((st = check_tensor(k, model.dtype, true)) || (st = check_tensor(v, model.dtype, true))) return st;
    p.k = k.ptr;
    p.v = v.ptr;
    p.s_k = strides_of(k);
    p.s_v = strides_of(v);
    return KVCOMM_OK;
}

// The kernels' direct loads address a row group as a 64-bit scalar base plus an unsigned 32-bit per-lane byte
// offset that spans up to 64 * 8 / D rows: the token stride has to leave that offset below 2^32.
static inline bool direct_loads_reach(const Strides &cache, int D)
{
    const int64_t rows_per_load = 64 * 8 / D;
    return cache.token < ((int64_t)1 << 31) / (2 * rows_per_load);
}

// fp32: row tiles of `groups` * 16 packed rows.
static inline int launch_f32(AttnParams &p, int D, int groups, int max_blocks, hipStream_t s)
{
    p.groups_per_tile = groups;
    const int rows = 16 * groups;
    p.n_row_tiles = (int32_t)(((int64_t)p.G * p.tq + rows - 1) / rows);
    const int64_t n_items = (int64_t)p.L * p.Hkv * p.n_row_tiles;
    if (n_items > 0x7fffffff) return KVCOMM_EUNSUPPORTED;
    p.n_items = (int32_t)n_items;
    set_divisors(p);
    return launch_attn_f32(p, D, (unsigned)(max_blocks > 0 ? std::min(max_blocks, p.n_items) : p.n_items), s);
}

// The same in 4 bits.
static inline int attn_cache4(const kvcomm_model &model, const kvcomm_tensor4 &k, const kvcomm_tensor4 &v, AttnParams &p)
{
    int st;
    if ((st = check_tensor4(k, model.head_dim)) || (st = check_tensor4(v, model.head_dim))) return st;
    p.k = k.codes.ptr;
    p.v = v.codes.ptr;
    p.s_k = strides_of(k.codes);
    p.s_v = strides_of(v.codes);
    p.k_scales = static_cast<const uint8_t *>(k.scales.ptr);
    p.v_scales = static_cast<const uint8_t *>(v.scales.ptr);
    p.s_ks = strides_of(k.scales);
    p.s_vs = strides_of(v.scales);
    return KVCOMM_OK;
}

// Tokens of a cache whose tiles, and packed rows, that the kernels count with 32-bit integers; and fewer (layer, kv head, row) triples than a launch
// holds threads: no kernel has fewer than two for a row.  The plan is made within these bounds; launch_attn() and launch_attn_f32() look at its blocks.
constexpr int64_t kMaxTokens = (int64_t)1 << 30, kMaxRows = ((int64_t)1 << 31) - 512;
static inline bool plannable(const kvcomm_model &m, int n_ctx, int tq, int64_t max_tokens = kMaxTokens, double max_all_rows = 2147483648.0)
{
    const int64_t rows = (int64_t)(m.n_q_heads / m.n_kv_heads) * tq;
    return (int64_t)n_ctx + tq <= max_tokens && rows <= kMaxRows && (double)m.n_layers * m.n_kv_heads * (double)rows < max_all_rows;
}
// Whole caches: as far as 32-bit tokens and 64-bit plans reach (a confined launch of few blocks may walk any number of items).
static inline bool plannable_whole(const kvcomm_model &m, int n_ctx, int tq) { return plannable(m, n_ctx, tq, kMaxRows, 1099511627776.0); }

}  // namespace kvc
