// kvcomm_paged_attn, kvcomm_paged_attn_prefix: causal attention of a batch of sequences over the pages of a pool, each behind the same cache or none.
#include "attn_host.h"
#include "attn_paged.h"

namespace {

using namespace kvc;

// The results of rows whose keys went to several wavefronts or runs: out = sum_s f_s O_s / sum_s f_s l_s, f_s = exp2((m_s - max m) scale log2 e), parts in
// a fixed order.  A wavefront takes `heads` query heads of a (layer, row); D / 4 lanes hold an output's channels, and the 64 / (D / 4) such groups take the
// parts in turn.  W = 4: the four wavefronts of a block share one head's parts, where there are few rows (8 sequences, 32 heads, up to 49 parts of a row: see launch_combine()).
struct CombineParams : PagedAttnParams {
    int32_t heads, chunks;   // query heads of a wavefront, such pieces of a row
    divisor_t by_chunks, by_rows;
};
template <typename T, int D, int W>
__global__ __launch_bounds__(256) void attn_paged_combine_kernel(const CombineParams p)
{
    constexpr int CL = D / 4, NG = 64 / CL, U = 8;
    const int lane = threadIdx.x & 63, Hq = p.Hkv * p.G, n_rows = p.batch.n_rows;
    const int sub = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), unit = W == 4 ? blockIdx.x : blockIdx.x * 4 + sub;
    const int lr = div_by(unit, p.by_chunks), chunk = unit - lr * p.chunks, l = div_by(lr, p.by_rows), row = lr - l * n_rows;
    if (l >= p.L) return;
    // (One row of up to tile_rows heads per sequence: its item is known.  Else, for rows of no sequence, item_of holds whatever.)
    const bool known = !p.batch.starts && p.G <= p.tile_rows;
    const int item = known ? p.prefix_tiles + row : p.item_of[2 * row], number = known ? 0 : p.item_of[2 * row + 1];
    int first, n;
    all_rows(p, first, n);
    if (row < first || row >= first + n || (item < 0 && (item != kWhole || p.prefix_part < p.tile_runs))) return;   // kDirect
    const bool apart = p.n_prefix > 0 && p.walked_prefix == 0;
    // What the walks left of an item: `count` slots from wavefront `wave` on, the last of them an item's end; or parts by rows.  (Clamped, and only
    // parts that there is room for: where starts decreases, items and item_of are not written for every row.)
    struct Parts {
        int wave, count, row;
        bool whole;
    };
    const int64_t all = (int64_t)p.L * Hq * n_rows;
    const int group = lane / CL, c = 4 * (lane % CL);
    __shared__ float joined_ml[W][2];
    __shared__ __align__(16) float joined_o[W][D];
    auto parts_of = [&](int hkv, int index, int packed) -> Parts {
        const int32_t *e = p.items + ((int64_t)(l * p.Hkv + hkv) * p.max_items + max(0, min(index, p.max_items - 1))) * 2;
        const int w0 = e[0], w1 = e[1];
        if (w0 < 0) return Parts{w0 == kWhole && p.prefix_part > 0 ? kWhole : kDirect, 1, 0, true};
        const int last = max(0, min(w1, p.n_waves - 1)), from = min(w0, last);
        return Parts{from, last - from + 1, packed & (p.tile_rows - 1), false};
    };
    auto own_of = [&](int hq) -> Parts {
        if (item < 0) return Parts{item, p.tile_runs, 0, true};
        const int hkv = div_by(hq, p.by_G), packed = number * p.G + hq - hkv * p.G;
        return parts_of(hkv, item + (int)((uint32_t)packed / (uint32_t)p.tile_rows), packed);
    };
    // A head per lane: which of them are not done (of most large batches nearly all are).
    const int head0 = chunk * p.heads, head = head0 + lane;
    // (W = 4: one, looked at where what lies before its parts has been asked for, too: a way to memory less, 14.2 -> 13.3 us for the
    // fp32 batch of the tiny configuration while it took this form)
    for (uint64_t todo = W == 4 ? 1 : __builtin_amdgcn_ballot_w64(lane < p.heads && head < Hq && own_of(min(head, Hq - 1)).wave != kDirect); todo; todo &= todo - 1) {
        const int hq = head0 + __builtin_ctzll(todo), hkv = div_by(hq, p.by_G), g = hq - hkv * p.G;
        const int64_t flat = ((int64_t)l * Hq + hq) * n_rows + row;
        const Parts own = own_of(hq);
        Parts before = {0, p.prefix_runs, 0, true};
        if (p.prefix_tiles) {
            const int at = (row - first) * p.G + g;
            before = parts_of(hkv, (int)((uint32_t)at / (uint32_t)p.tile_rows), at);
        }
        if (W == 4 && own.wave == kDirect) return;
        const int count = own.count + (apart ? before.count : 0);
        auto place = [&](int k, const float *&o, const float *&ml) {
            const bool b = k >= own.count;
            const Parts &x = b ? before : own;
            if (b) k -= own.count;
            if (x.whole) {
                const int64_t at = flat + (b ? p.prefix_part + k : k) * all;
                o = p.row_o + at * D;
                ml = p.row_ml + at * 2;
            } else {
                const int64_t at = (2 * (int64_t)(x.wave + k) + (k + 1 < x.count ? 1 : 0)) * p.tile_rows + x.row;
                o = p.slot_o + at * D;
                ml = p.slot_ml + at * 2;
            }
        };
        // Parts k0 ... of this group, whose loads are all in flight at once, against the largest reference so far.  (Those behind the last one are not read: 2048 rows of 3 parts
        // each 25.1 -> 23.6 us with the kernel before.)
        float M = -INFINITY, sum = 0.f;
        f32x4 acc = {0.f, 0.f, 0.f, 0.f};
        for (int k0 = W == 4 ? sub * NG + group : group; k0 < count; k0 += W * NG * U) {
            f32x4 os[U];
            float ms[U], ls[U], top = M;
#pragma unroll
            for (int u = 0; u < U; ++u) ms[u] = -INFINITY, ls[u] = 0.f, os[u] = f32x4{0.f, 0.f, 0.f, 0.f};
            auto get = [&](int u) __attribute__((always_inline)) {
                const float *o, *ml;
                place(k0 + u * W * NG, o, ml);
                ms[u] = ml[0];
                ls[u] = ml[1];
                os[u] = *reinterpret_cast<const f32x4 *>(o + c);
            };
            if (k0 + (U - 1) * W * NG < count) {
#pragma unroll
                for (int u = 0; u < U; ++u) get(u);
            } else {
#pragma unroll
                for (int u = 0; u < U - 1; ++u)
                    if (k0 + u * W * NG < count) get(u);
            }
#pragma unroll
            for (int u = 0; u < U; ++u) top = fmaxf(top, ms[u]);
            const float f0 = M == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((M - top) * p.scale_log2);
            sum = M == -INFINITY ? sum : sum * f0;   // (nothing seen: 0)
            acc *= f0;
            M = top;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (ms[u] != -INFINITY) {
                    const float f = __builtin_amdgcn_exp2f((ms[u] - M) * p.scale_log2);
                    sum = fmaf(f, ls[u], sum);
                    acc += f * os[u];
                } else {
                    sum += ls[u];   // (outputs of a part that has seen nothing may never have been written)
                }
            }
        }
#pragma unroll
        for (int off = CL; off < 64; off <<= 1) {   // the groups
            float f, f2;
            const float m2 = __shfl_xor(M, off), l2 = __shfl_xor(sum, off);
            join_part(M, sum, m2, l2, p.scale_log2, f, f2);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float a2 = __shfl_xor(acc[i], off);
                acc[i] = acc[i] * f + a2 * f2;
            }
        }
        if constexpr (W > 1) {   // the wavefronts (heads is 1 then, and the block goes through here together)
            if (lane == 0) joined_ml[sub][0] = M, joined_ml[sub][1] = sum;
            if (group == 0) *reinterpret_cast<f32x4 *>(&joined_o[sub][c]) = acc;
            __syncthreads();
            if (sub) return;
#pragma unroll
            for (int w = 1; w < W; ++w) {
                float f, f2;
                join_part(M, sum, joined_ml[w][0], joined_ml[w][1], p.scale_log2, f, f2);
                acc = acc * f + *reinterpret_cast<const f32x4 *>(&joined_o[w][c]) * f2;
            }
        }
        const bool none = M == -INFINITY && sum == 0.f;
        if (group == 0) {
            const float inv = none ? 0.f : 1.f / sum;
            T *out = static_cast<T *>(p.out) + l * p.s_o.layer + (int64_t)hq * p.s_o.head + (int64_t)row * p.s_o.token + c;
            if constexpr (sizeof(T) == 2)
                *reinterpret_cast<u32x2 *>(out) = u32x2{pack_bf16x2(acc[0] * inv, acc[1] * inv), pack_bf16x2(acc[2] * inv, acc[3] * inv)};
            else
                *reinterpret_cast<f32x4 *>(out) = acc * inv;
        }
        if (p.lse && lane == 0) p.lse[flat] = none ? -INFINITY : M * p.scale + logf(sum);
    }
}

template <typename T>
int launch_combine(const PagedAttnParams &a, hipStream_t s)
{
    CombineParams p{};
    static_cast<PagedAttnParams &>(p) = a;
    const int Hq = a.Hkv * a.G;
    const int64_t rows = (int64_t)a.L * a.batch.n_rows;
    // Few rows: a block per head.  us, the kernel alone, 8 sequences of 600 to 3100 tokens, one layer: 8.7 as a wavefront per head, 4.9 so.  Many: as many heads of a wavefront as
    // leave 16384 of them (64 sequences behind a prefix, 32 layers: 22; with 4096 of them 45).
    // The line, us for the whole call with a block / a wavefront per head, D = 128, 32 heads but for the f32 ones (D = 64, 8): (layer, head, row) triples 256 11.5 / 13.0, 512 f32 13.1 / 13.5,
    // 1024 17.5 / 17.5, 121.4 / 120.9 and f32 20.8 / 20.6, 2048 27.6 / 26.1, 107.8 / 106.2 and f32 32.3 / 31.7, 4096 45.5 / 43.6, 119.1 / 115.9 and f32 40.5 / 37.7, 8192 84.3 / 79.4.
    const bool few = rows * Hq <= 1024;
    p.heads = few ? 1 : (int)std::min<int64_t>(std::min(Hq, 64), std::max<int64_t>(1, rows * Hq / 16384));
    p.chunks = (Hq + p.heads - 1) / p.heads;
    p.by_chunks = make_divisor((uint32_t)p.chunks);
    p.by_rows = make_divisor((uint32_t)a.batch.n_rows);
    const dim3 grid((unsigned)(few ? rows * p.chunks : (rows * p.chunks + 3) / 4)), block(256);
    switch (a.D) {
        case 64: return launch(few ? attn_paged_combine_kernel<T, 64, 4> : attn_paged_combine_kernel<T, 64, 1>, grid, block, 0, s, p);
        case 128: return launch(few ? attn_paged_combine_kernel<T, 128, 4> : attn_paged_combine_kernel<T, 128, 1>, grid, block, 0, s, p);
        default: return launch(few ? attn_paged_combine_kernel<T, 256, 4> : attn_paged_combine_kernel<T, 256, 1>, grid, block, 0, s, p);
    }
}

// How a call is carried out: what depends on the model, the batch's host side and the prefix's length alone.
//   Sequences of up to kFewRows packed rows go to the wavefront kernel, longer ones, if there may be any, to the tiles kernel; the prefix, for the rows of all of them, to one
//   or the other.  us with 32 / 64 / 128 as the line, D = 128, 8 kv heads, G = 4: one layer, 8 sequences of 16 to 40 rows behind 300 to 3000 tokens 38 / 45 / 60, four
//   layers 81 / 85 / 155; 32 of 10 to 30 behind 100 to 500, one layer 25 / 47 / 40, 32 layers 336 / 473 / 685.
constexpr int kFewRows = 32;
// A prefix for more rows than that, one of each of many sequences, goes to the wavefront kernel where that has up to so many halves of it for each wavefront.  us for the whole call
// by that kernel / by the tiles kernel, D = 128, 8 kv heads, G = 4; halves of a wavefront: one layer, 16 sequences, prefix 8192 (2) 32 / 51, 32 sequences (4) 44 / 52,
// 64 (8) 70 / 69, 128 (16) 113 / 81; 4 layers, 10 sequences, prefix 1000 (1) 27 / 35, 64 (4) 66 / 65; 16 layers, 16, prefix 8192 (32) 241 / 150.
constexpr int kPrefixHalves = 4;
// Runs of the keys of a sequence's row tile, at most.
constexpr int kSeqMaxRuns = 16;

struct Plan {
    int tile_rows, n_waves, prefix_tiles;   // of the wavefront kernel
    bool tiles;                             // is the tiles kernel launched for sequences
    int seq_rows, seq_runs, prefix_rows, prefix_runs;   // its row tiles and runs; prefix_runs 0: it is not launched for the prefix
    int64_t seq_units, prefix_units;        // its blocks per (layer, kv head)
    int64_t max_items, seq_parts, row_parts;   // parts by rows: [row_parts][layer, query head, row], sequences' first
    size_t bytes;
};

Plan plan_of(const kvcomm_model &m, const kvcomm_batch &b, int n_prefix)
{
    Plan pl{};
    const int G = m.n_q_heads / m.n_kv_heads, D = m.head_dim;
    const int64_t LH = (int64_t)m.n_layers * m.n_kv_heads, rows = (int64_t)b.n_rows * G;
    const int64_t most = b.starts ? (b.max_rows ? std::min<int64_t>(b.max_rows, b.n_rows) : b.n_rows) * G : G;
    const bool f32 = m.dtype == KVCOMM_F32;   // the wavefront kernel takes it all
    pl.tiles = !f32 && most > kFewRows;
    bool few_prefix = n_prefix && (f32 || rows <= kFewRows);
    if (n_prefix && !few_prefix && !pl.tiles) {
        const int tr = D < 256 ? 32 : 16;
        few_prefix = (double)LH * ((rows + tr - 1) / tr) * ((n_prefix + 31) / 32) <= (double)kPrefixHalves * kChipCUs * paged_rows_waves(D, tr);
    }
    pl.tile_rows = f32 ? 16 : D < 256 && (most > 16 || (few_prefix && rows > 16)) ? 32 : 16;
    pl.n_waves = kChipCUs * (f32 ? paged_f32_waves(D) : paged_rows_waves(D, pl.tile_rows));
    pl.max_items = b.starts ? (pl.tiles ? (int64_t)b.n_seqs * (kFewRows / pl.tile_rows) : rows / pl.tile_rows + b.n_seqs) : (int64_t)b.n_seqs * ((G + pl.tile_rows - 1) / pl.tile_rows);
    pl.seq_runs = 1;
    if (pl.tiles) {
        pl.seq_rows = D == 256 || rows < 512 * (int64_t)b.n_seqs ? 128 : 256;
        const int64_t tiles = rows / pl.seq_rows + std::min<int64_t>(b.n_seqs, rows / (kFewRows + 1) + 1), reach = (int64_t)b.table_width * b.page_size;
        // Keys are cut where the row tiles are few, up to two blocks per compute unit (of the tiles that there may be, many are not there).  The lengths lie on the
        // device: by what the table reaches, and into runs of 512 at least.  Up to two blocks / one, one layer, 8 kv heads, G = 4, us: 4 sequences, 64 rows behind
        // 1000 to 4000 tokens 38 / 51 (D = 256 63 / 88), 512 rows behind 3100 55 / 71, 128 behind 9000 44 / 53; up to four 40 (D = 256 76), 54, 44.
        while (pl.seq_runs < kSeqMaxRuns && tiles * LH * pl.seq_runs * 2 <= 2 * kChipCUs && reach >= 1024 * pl.seq_runs) pl.seq_runs *= 2;
        pl.seq_units = tiles * pl.seq_runs;
    }
    if (few_prefix) {
        pl.prefix_tiles = (int)((rows + pl.tile_rows - 1) / pl.tile_rows);
        pl.max_items += pl.prefix_tiles;
    } else if (n_prefix) {
        pl.prefix_rows = D == 256 || rows <= 128 ? 128 : 256;
        const int64_t tiles = (rows + pl.prefix_rows - 1) / pl.prefix_rows, keys = (n_prefix + 63) / 64;
        double best = INFINITY;
        for (int ns = 1; ns == 1 || (ns <= kTileMaxSplits && tiles * LH <= 2 * kChipCUs && ns * kMinRunTiles <= keys); ++ns) {
            const double t = pl.prefix_rows == 128 && D < 256 ? attn_tiles128_us(m, tiles * LH, keys, ns) : attn_tiles_us(m, tiles * LH, pl.prefix_rows, keys, ns);
            if (t < 0.95 * best) best = t, pl.prefix_runs = ns;
        }
        pl.prefix_units = tiles * pl.prefix_runs;
    }
    pl.seq_parts = pl.prefix_tiles ? 1 : pl.seq_runs > 1 ? pl.seq_runs : 0;
    pl.row_parts = pl.seq_parts + (pl.prefix_tiles ? 1 : pl.prefix_runs);
    pl.bytes = sizeof(float) * (size_t)(D + 2) * ((size_t)pl.n_waves * 2 * pl.tile_rows + (size_t)(pl.row_parts * LH * rows)) +
               sizeof(int32_t) * ((size_t)(2 * LH * pl.max_items) + 2 * (size_t)b.n_rows);
    return pl;
}

// What attention calls refuse before anything else is looked at: sizes that their 32-bit counts do not hold.
bool countable(const kvcomm_model &m, const kvcomm_batch &b)
{
    const double G = m.n_q_heads / m.n_kv_heads;
    return (double)b.n_rows * G <= (double)kMaxRows && (double)b.n_rows * m.n_q_heads * m.n_layers < 67000000.0 && (double)m.n_layers * m.n_kv_heads <= INT32_MAX;
}

// The direct loads' 32-bit offsets: see direct_loads_reach().
bool reaches(int64_t token_stride, int D) { return direct_loads_reach(Strides{0, 0, token_stride}, D); }

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
    {   // queries are read again after outputs of the same rows have been written
        const int L = model->n_layers, Hq = model->n_q_heads, es = elem_size(dt);
        if (extents_overlap(extent_of(out, L, Hq, batch->n_rows, D, es), extent_of(q, L, Hq, batch->n_rows, D, es)) &&
            !beside_each_other(out, Hq, D * es, es, q, Hq, D * es, es, L))
            return KVCOMM_EINVAL;
    }
    if ((int64_t)n_prefix + p.batch.cap > kMaxPagedTokens || !countable(*model, *batch)) return KVCOMM_EUNSUPPORTED;
    if (dt == KVCOMM_BF16 && ((p.batch.cap && (!reaches(pages_k.stride_token, D) || !reaches(pages_v.stride_token, D))) ||
                              (n_prefix && (!reaches(prefix_k.stride_token, D) || !reaches(prefix_v.stride_token, D)))))
        return KVCOMM_EUNSUPPORTED;
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
    p.D = D;
    const int64_t rows = (int64_t)p.L * p.Hkv * p.G * p.batch.n_rows;
    hipStream_t s = static_cast<hipStream_t>(stream);
    const Plan pl = plan_of(*model, *batch, n_prefix);
    const bool scratch = workspace && aligned16(workspace) && workspace_bytes >= pl.bytes;
    const int64_t LH = (int64_t)p.L * p.Hkv;
    const double most_blocks = 4294967296.0 / 512;   // a launch holds fewer than 2^32 threads
    if ((double)pl.seq_units * LH >= most_blocks || (double)pl.prefix_units * LH >= most_blocks || pl.max_items > INT32_MAX / 2) return KVCOMM_EUNSUPPORTED;
    // The axis: halves of a (layer, kv head) in 31 bits, and of a run up to kPagedMostRun (less what the wavefronts add to their share against rounding).
    const int64_t most_tiles = batch->starts ? rows / ((int64_t)p.L * p.Hkv * pl.tile_rows) + batch->n_seqs : (int64_t)batch->n_seqs * ((p.G + pl.tile_rows - 1) / pl.tile_rows);
    const double axis = (double)most_tiles * ((double)(p.batch.cap + 31) / 32 + (scratch ? 0.0 : (double)(n_prefix + 31) / 32) + 1) + (double)pl.prefix_tiles * ((n_prefix + 31) / 32);
    if (axis >= 2147483647.0 || axis * LH / pl.n_waves >= 0.99 * kPagedMostRun) return KVCOMM_EUNSUPPORTED;
    p.tile_rows = pl.tile_rows;
    p.n_waves = pl.n_waves;
    p.per_wave = 1.000001f / (float)pl.n_waves;
    p.most_rows = scratch && pl.tiles ? kFewRows : INT32_MAX;
    p.max_items = (int32_t)pl.max_items;
    if (!scratch) {
        p.walked_prefix = (n_prefix + 31) / 32;
        return dt == KVCOMM_F32 ? launch_paged_f32(p, s) : launch_paged_rows(p, pl.tile_rows, s);
    }
    float *x = static_cast<float *>(workspace);
    auto take = [&](int64_t n) { float *y = x; x += n; return y; };
    p.slot_o = take((int64_t)pl.n_waves * 2 * pl.tile_rows * D);
    p.row_o = take(pl.row_parts * rows * D);
    p.slot_ml = take((int64_t)pl.n_waves * 2 * pl.tile_rows * 2);
    p.row_ml = take(pl.row_parts * rows * 2);
    p.items = reinterpret_cast<int32_t *>(take(2 * LH * pl.max_items));
    p.item_of = reinterpret_cast<int32_t *>(x);
    p.prefix_tiles = pl.prefix_tiles;
    p.prefix_runs = pl.prefix_runs;
    p.prefix_part = (int32_t)pl.seq_parts;
    p.tile_runs = pl.seq_runs;
    auto tiles_of = [&](bool over_prefix) {
        PagedTileParams t{};
        static_cast<PagedAttnParams &>(t) = p;
        t.over_prefix = over_prefix;
        t.n_items = 1;
        t.n_splits = over_prefix ? pl.prefix_runs : pl.seq_runs;
        t.more_rows = kFewRows;
        t.part = over_prefix ? p.prefix_part : 0;
        t.slot_mask = over_prefix ? INT32_MAX : (1 << p.batch.log_page) - 1;
        t.by_LH = make_divisor((uint32_t)LH);
        t.by_splits = make_divisor((uint32_t)t.n_splits);
        if (over_prefix) {
            t.k = p.prefix_k;
            t.v = p.prefix_v;
            t.s_k = PoolStrides{p.s_pk.layer, p.s_pk.head, 0, p.s_pk.token};
            t.s_v = PoolStrides{p.s_pv.layer, p.s_pv.head, 0, p.s_pv.token};
        }
        if (!over_prefix && pl.seq_runs == 1) {   // (then a prefix has parts by rows: its rows are more than kFewRows)
            t.row_o = nullptr;
            t.join_runs = pl.prefix_runs;
            t.join_part = p.prefix_part;
            t.join_o = p.row_o;
            t.join_ml = p.row_ml;
        }
        return launch_paged_tiles(t, over_prefix ? pl.prefix_rows : pl.seq_rows, (unsigned)((over_prefix ? pl.prefix_units : pl.seq_units) * LH), s);
    };
    if (pl.prefix_runs && (st = tiles_of(true))) return st;
    if (pl.tiles && (st = tiles_of(false))) return st;
    if (dt == KVCOMM_F32) {
        st = launch_paged_f32(p, s);
        return st ? st : launch_combine<float>(p, s);
    }
    if ((st = launch_paged_rows(p, pl.tile_rows, s))) return st;
    return launch_combine<bf16_t>(p, s);
}

size_t workspace_of(const kvcomm_model *model, const kvcomm_batch *batch, int32_t n_prefix)
{
    Batch b;
    if (check_model(model) || check_batch(batch, b) || n_prefix < 0 || (int64_t)n_prefix + b.cap > kMaxPagedTokens || !countable(*model, *batch)) return 0;
    return plan_of(*model, *batch, n_prefix).bytes;
}

}  // namespace

extern "C" size_t kvcomm_paged_attn_workspace(const kvcomm_model *model, const kvcomm_batch *batch)
{
    return workspace_of(model, batch, 0);
}

extern "C" int kvcomm_paged_attn(const kvcomm_model *model, kvcomm_tensor q, kvcomm_pages pages_k, kvcomm_pages pages_v, const kvcomm_batch *batch,
                                 float softmax_scale, kvcomm_tensor out, float *lse_out, void *workspace, size_t workspace_bytes, void *stream)
{
    const kvcomm_tensor none = {nullptr, 0, 0, 0};
    return paged_attn(model, q, none, none, 0, pages_k, pages_v, batch, softmax_scale, out, lse_out, workspace, workspace_bytes, stream);
}

extern "C" size_t kvcomm_paged_attn_prefix_workspace(const kvcomm_model *model, int32_t n_prefix, const kvcomm_batch *batch)
{
    return n_prefix <= 0 ? 0 : workspace_of(model, batch, n_prefix);
}

extern "C" int kvcomm_paged_attn_prefix(const kvcomm_model *model, kvcomm_tensor q, kvcomm_tensor prefix_k, kvcomm_tensor prefix_v, int32_t n_prefix,
                                        kvcomm_pages pages_k, kvcomm_pages pages_v, const kvcomm_batch *batch, float softmax_scale, kvcomm_tensor out,
                                        float *lse_out, void *workspace, size_t workspace_bytes, void *stream)
{
    if (n_prefix <= 0) return KVCOMM_EINVAL;
    return paged_attn(model, q, prefix_k, prefix_v, n_prefix, pages_k, pages_v, batch, softmax_scale, out, lse_out, workspace, workspace_bytes, stream);
}
