// kvcomm_suffix_attn_window: the kernels of kvcomm_suffix_attn over the tiles that a window and the sinks leave (Keys::kWindow).
#include "attn_host.h"

namespace {

using namespace kvc;

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
    if (!plannable(*model, n_ctx, tq)) return 0;
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
    if (!plannable(*model, n_ctx, tq)) return KVCOMM_EUNSUPPORTED;
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
