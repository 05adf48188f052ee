// kvcomm_suffix_attn_window and kvcomm_suffix_attn_kv4.
#include "attn_exact.h"
#include "attn_host.h"

namespace {

using namespace kvc;

// 16 packed (query, head) rows of a (layer, kv head) per block, row by row.
template <typename T, typename Q, int D>
__global__ __launch_bounds__(256) void attn_exact_kernel(const AttnParams p)
{
    const int lh = div_by(blockIdx.x, p.by_row_tiles), row0 = (blockIdx.x - lh * p.n_row_tiles) * 16;
    const int pos = p.n_ctx + min(div_by(row0, p.by_G), p.tq - 1);
    const int begin = p.window == 0 ? 0 : max(0, pos + 1 - p.window);
    const KeyRanges keys = {0, min(p.n_sinks, begin), begin, p.N};
    attn_exact_rows<T, Q, D>(p, lh, row0, 16, keys, 0, 16, threadIdx.x >> 6, 4, threadIdx.x & 63);
}

template <typename T, typename Q>
int launch_exact(AttnParams &p, int D, void *stream)
{
    p.n_row_tiles = (int32_t)(((int64_t)p.G * p.tq + 15) / 16);
    const int64_t n_items = (int64_t)p.L * p.Hkv * p.n_row_tiles;
    if (n_items >= 1 << 24) return KVCOMM_EUNSUPPORTED;
    p.n_items = (int32_t)n_items;
    set_divisors(p);
    const dim3 grid((unsigned)n_items), block(256);
    hipStream_t s = static_cast<hipStream_t>(stream);
    switch (D) {
        case 64: return launch(attn_exact_kernel<T, Q, 64>, grid, block, 0, s, p);
        case 128: return launch(attn_exact_kernel<T, Q, 128>, grid, block, 0, s, p);
        default: return launch(attn_exact_kernel<T, Q, 256>, grid, block, 0, s, p);
    }
}

// What a window beyond the cache or sinks beyond it change: nothing.
void clamp_window(int32_t n_ctx, int32_t tq, int32_t &window, int32_t &n_sinks)
{
    const int64_t N = (int64_t)n_ctx + tq;
    window = (int32_t)std::min<int64_t>(window, N);
    n_sinks = (int32_t)std::min<int64_t>(n_sinks, N);
}

}  // namespace

extern "C" size_t kvcomm_suffix_attn_window_workspace(const kvcomm_model *model, int32_t n_ctx, int32_t tq, int32_t window, int32_t n_sinks)
{
    if (check_model(model) || tq <= 0 || n_ctx < 0 || window <= 0 || n_sinks < 0 || model->dtype != KVCOMM_BF16) return 0;
    if ((int64_t)n_ctx + tq > kMaxTokens) return 0;
    clamp_window(n_ctx, tq, window, n_sinks);
    return attn_workspace(*model, attn_plan_window(*model, n_ctx, tq, window, n_sinks, true));
}

extern "C" int kvcomm_suffix_attn_window(const kvcomm_model *model, kvcomm_tensor q, kvcomm_tensor cache_k, kvcomm_tensor cache_v, int32_t n_ctx,
                                         int32_t tq, int32_t window, int32_t n_sinks, float softmax_scale, kvcomm_tensor out, float *lse_out,
                                         void *workspace, size_t workspace_bytes, void *stream)
{
    AttnParams p{};
    int st = attn_params(model, q, n_ctx, tq, softmax_scale, out, lse_out, p);
    if (st || (st = attn_cache(*model, cache_k, cache_v, p))) return st;
    if (window <= 0 || n_sinks < 0) return KVCOMM_EINVAL;
    if (!fits_a_launch(p)) return KVCOMM_EUNSUPPORTED;
    clamp_window(n_ctx, tq, window, n_sinks);
    p.window = window;
    p.n_sinks = n_sinks;
    const int D = model->head_dim;
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (model->dtype == KVCOMM_F32) return launch_f32(p, D, attn_f32_groups(*model, tq, 0), 0, s);
    if (!direct_loads_reach(p.s_k, D) || !direct_loads_reach(p.s_v, D)) return KVCOMM_EUNSUPPORTED;
    return launch_attn(*model, p, attn_plan_window(*model, n_ctx, tq, window, n_sinks, true), attn_plan_window(*model, n_ctx, tq, window, n_sinks, false), 0,
                       workspace, workspace_bytes, s);
}

extern "C" size_t kvcomm_suffix_attn_kv4_workspace(const kvcomm_model *, int32_t, int32_t) { return 0; }

extern "C" int kvcomm_suffix_attn_kv4(const kvcomm_model *model, kvcomm_tensor q, kvcomm_tensor4 cache_k, kvcomm_tensor4 cache_v, int32_t n_ctx,
                                      int32_t tq, float softmax_scale, kvcomm_tensor out, float *lse_out, void *, size_t, void *stream)
{
    AttnParams p{};
    int st = attn_params(model, q, n_ctx, tq, softmax_scale, out, lse_out, p);
    if (st || (st = attn_cache4(*model, cache_k, cache_v, p))) return st;
    if (model->dtype != KVCOMM_BF16 || !fits_a_launch(p)) return KVCOMM_EUNSUPPORTED;
    return launch_exact<fp4_t, bf16_t>(p, model->head_dim, stream);
}
