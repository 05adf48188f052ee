// kvcomm_paged_attn, kvcomm_paged_attn_prefix: causal attention of a batch of sequences over the pages of a pool, each behind the same cache or none.
#include "attn_host.h"
#include "attn_paged.h"

namespace {

using namespace kvc;

// One wavefront per (layer, query head, row).
template <typename T, int D>
__global__ __launch_bounds__(256) void attn_paged_row_kernel(const PagedAttnParams p)
{
    const int lane = threadIdx.x & 63, Hq = p.Hkv * p.G;
    const int64_t item = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (item >= (int64_t)p.L * Hq * p.batch.n_rows) return;
    const int row = (int)(item % p.batch.n_rows), head = (int)(item / p.batch.n_rows), l = head / Hq, hq = head - l * Hq;
    const int b = sequence_of(p.batch, row, lane);
    if (b < 0) return;
    int first, n;
    sequence_rows(p.batch, b, first, n);
    if (row < first || row >= first + n) return;
    const int len = sequence_len(p.batch, b), last = last_seen(len, n, row - first, p.batch.cap);
    const int prefix_halves = (p.n_prefix + 31) / 32;
    float m, sum, o[8];
    paged_exact_row<T, D>(p, l, hq / p.G, hq, row, b, last, prefix_halves, 0, prefix_halves + (last + 32) / 32, lane, m, sum, o);
    paged_store_row<T, D>(p, l, hq, row, lane, m, sum, o);
}

int paged_attn(const kvcomm_model *model, const kvcomm_tensor &q, const kvcomm_tensor &prefix_k, const kvcomm_tensor &prefix_v, int32_t n_prefix,
               const kvcomm_pages &pages_k, const kvcomm_pages &pages_v, const kvcomm_batch *batch, float softmax_scale, const kvcomm_tensor &out,
               float *lse_out, void *workspace, size_t workspace_bytes, void *stream)
{
    PagedAttnParams p{};
    int st = check_model(model);
    if (st || (st = check_batch(batch, p.batch))) return st;
    const int dt = model->dtype, D = model->head_dim;
    if ((st = check_tensor(q, dt, true)) || (st = check_tensor(out, dt, true))) return st;
    if (n_prefix && ((st = check_tensor(prefix_k, dt, true)) || (st = check_tensor(prefix_v, dt, true)))) return st;
    if (p.batch.cap && ((st = check_pages(pages_k, dt)) || (st = check_pages(pages_v, dt)))) return st;
    if (!aligned4(lse_out)) return KVCOMM_EINVAL;
    if (n_prefix > kMaxPagedTokens) return KVCOMM_EUNSUPPORTED;
    p.q = q.ptr;
    p.out = out.ptr;
    p.lse = lse_out;
    p.k = pages_k.ptr;
    p.v = pages_v.ptr;
    p.prefix_k = prefix_k.ptr;
    p.prefix_v = prefix_v.ptr;
    p.s_q = strides_of(q);
    p.s_o = strides_of(out);
    p.s_pk = strides_of(prefix_k);
    p.s_pv = strides_of(prefix_v);
    p.s_k = strides_of(pages_k);
    p.s_v = strides_of(pages_v);
    p.L = model->n_layers;
    p.Hkv = model->n_kv_heads;
    p.G = model->n_q_heads / model->n_kv_heads;
    p.n_prefix = n_prefix;
    p.scale = softmax_scale > 0.f ? softmax_scale : (float)(1.0 / sqrt((double)D));
    p.scale_log2 = (float)((double)p.scale * 1.4426950408889634);
    p.by_G = make_divisor((uint32_t)p.G);
    p.by_Hkv = make_divisor((uint32_t)p.Hkv);
    const double rows = (double)p.L * p.Hkv * p.G * p.batch.n_rows;
    if (rows >= 67108864.0) return KVCOMM_EUNSUPPORTED;
    const dim3 grid((unsigned)((rows + 3) / 4)), block(256);
    hipStream_t s = static_cast<hipStream_t>(stream);
    const bool f32 = dt == KVCOMM_F32;
    switch (D) {
        case 64: return launch(f32 ? attn_paged_row_kernel<float, 64> : attn_paged_row_kernel<bf16_t, 64>, grid, block, 0, s, p);
        case 128: return launch(f32 ? attn_paged_row_kernel<float, 128> : attn_paged_row_kernel<bf16_t, 128>, grid, block, 0, s, p);
        default: return launch(f32 ? attn_paged_row_kernel<float, 256> : attn_paged_row_kernel<bf16_t, 256>, grid, block, 0, s, p);
    }
}

}  // namespace

extern "C" size_t kvcomm_paged_attn_workspace(const kvcomm_model *model, const kvcomm_batch *batch) { return 0; }

extern "C" int kvcomm_paged_attn(const kvcomm_model *model, kvcomm_tensor q, kvcomm_pages pages_k, kvcomm_pages pages_v, const kvcomm_batch *batch,
                                 float softmax_scale, kvcomm_tensor out, float *lse_out, void *workspace, size_t workspace_bytes, void *stream)
{
    const kvcomm_tensor none = {nullptr, 0, 0, 0};
    return paged_attn(model, q, none, none, 0, pages_k, pages_v, batch, softmax_scale, out, lse_out, workspace, workspace_bytes, stream);
}

extern "C" size_t kvcomm_paged_attn_prefix_workspace(const kvcomm_model *model, int32_t n_prefix, const kvcomm_batch *batch) { return 0; }

extern "C" int kvcomm_paged_attn_prefix(const kvcomm_model *model, kvcomm_tensor q, kvcomm_tensor prefix_k, kvcomm_tensor prefix_v, int32_t n_prefix,
                                        kvcomm_pages pages_k, kvcomm_pages pages_v, const kvcomm_batch *batch, float softmax_scale, kvcomm_tensor out,
                                        float *lse_out, void *workspace, size_t workspace_bytes, void *stream)
{
    if (n_prefix <= 0) return KVCOMM_EINVAL;
    return paged_attn(model, q, prefix_k, prefix_v, n_prefix, pages_k, pages_v, batch, softmax_scale, out, lse_out, workspace, workspace_bytes, stream);
}
