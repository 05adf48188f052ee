// fp32 attention over pages and a prefix: single wavefronts on the walk of attn_paged.h.
#include "attn_paged.h"

namespace {

using namespace kvc;

// attn_paged_f32_kernel: 16 packed rows on 16x16x4 fp32 MFMAs, products and operand layout as in attn_f32_kernel: a lane owns one query column, and every
// operand comes from global memory in the layout the instruction wants (of K and Q 16-byte pieces, piece j of lane (n, g) holding channels 16 * j + 4 * g ... + 3,
// of V four consecutive channels of one key).  A wavefront is alone and walks 16 keys after the other, which lie in one page; the next ones are requested
// when this one's operands have been multiplied.  What bounds it: matrix cores where there is much of it (fp32 MFMA, 1/16 of the bf16 rate), else the chain of
// one wavefront.  2 layers of 4 heads, D = 64, 5 sequences of up to 300 tokens and 33 rows: 8.1 us, the whole call 12.9 (165 with a block
// per tile of rows); one layer, 8 heads, 8 sequences of 600 to 3100 tokens at D = 128, one row each, G = 4: the whole call 29 us, 16 by its bytes.
template <int D>
__global__ __launch_bounds__(64 * kPagedBlockWaves, D == 256 ? 1 : 2) void attn_paged_f32_kernel(const PagedAttnParams)
{
    PagedArgs &p = paged_args();
    await_paged_args(p);
    constexpr int TR = 16, NJ = D / 16, NT = D / 64;   // 16-byte pieces of a K row in a lane, loads of a V row
    const int wave = __builtin_amdgcn_readfirstlane((int)blockIdx.x * kPagedBlockWaves + (int)(threadIdx.x >> 6));
    const int lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
    PagedWalk<TR> walk(lane);
    int64_t pos = -1, end;
    int h;

    // ---- the keys: a sub-step is 16 of them, two to a half
    const float *kp, *vp, *kf, *vf;
    const_int *table = nullptr;
    int tokens = 0;
    auto enter = [&]() __attribute__((always_inline)) {   // walk.item
        PagedArgs &p = paged_args();
        const PagedItem &it = walk.item;
        const int l = div_by(it.lh, p.by_Hkv), hkv = it.lh - l * p.Hkv;
        kp = static_cast<const float *>(p.k) + l * p.s_k.layer + hkv * p.s_k.head;
        vp = static_cast<const float *>(p.v) + l * p.s_v.layer + hkv * p.s_v.head;
        kf = static_cast<const float *>(p.prefix_k) + l * p.s_pk.layer + hkv * p.s_pk.head;
        vf = static_cast<const float *>(p.prefix_v) + l * p.s_pv.layer + hkv * p.s_pv.head;
        tokens = it.b < 0 ? 0 : min(it.len, p.batch.cap);
        table = scalar(p.batch.table) + (int64_t)max(it.b, 0) * p.batch.table_stride;
    };
    struct Sub {
        int at, limit;   // first key, and how many there are (0: nothing is read)
        int prefix, page;   // truth values (as bool they left bytes between, which were copied through memory)
        int64_t k, v;    // elements from the (layer, head)'s begin to the first key's row
    };
    auto sub_at = [&](int h_, int part) __attribute__((always_inline)) -> Sub {
        Sub x = {32 * h_ + 16 * part, p.n_prefix, h_ < walk.item.walk, 1, 0, 0};
        if (x.prefix) {
            const int64_t t = min(x.at, p.n_prefix - 1);   // (the second half of the last one may lie behind it)
            x.k = t * p.s_pk.token;
            x.v = t * p.s_pv.token;
            return x;
        }
        x.at -= 32 * walk.item.walk;
        x.limit = tokens;
        if (tokens > 0) {
            const int t = min(x.at, tokens - 1), e = table[t >> p.batch.log_page], slot = t & ((1 << p.batch.log_page) - 1);
            x.page = (uint32_t)e < (uint32_t)p.batch.n_pages;
            x.k = (int64_t)(x.page ? e : 0) * p.s_k.page + (int64_t)slot * p.s_k.token;
            x.v = (int64_t)(x.page ? e : 0) * p.s_v.page + (int64_t)slot * p.s_v.token;
        }
        return x;
    };
    // Row r of a sub-step; rows behind the last one are read as that one.
    auto row_in = [&](const Sub &x, int r) __attribute__((always_inline)) -> int64_t { return max(0, min(r, x.limit - 1 - x.at)); };
    f32x4 k[NJ], v[4][NT];
    auto load_k = [&](const Sub &x) __attribute__((always_inline)) {
        if (x.limit == 0) return;
        const float *row = (x.prefix ? kf : kp) + x.k + row_in(x, n) * (x.prefix ? p.s_pk.token : p.s_k.token) + 4 * g;
#pragma unroll
        for (int j = 0; j < NJ; ++j) k[j] = *reinterpret_cast<const f32x4 *>(row + 16 * j);
    };
    auto load_v = [&](const Sub &x) __attribute__((always_inline)) {   // score r of this lane is key 4 * g + r
        if (x.limit == 0) return;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const float *row = (x.prefix ? vf : vp) + x.v + row_in(x, 4 * g + r) * (x.prefix ? p.s_pv.token : p.s_v.token) + 4 * n;
#pragma unroll
            for (int t = 0; t < NT; ++t) v[r][t] = *reinterpret_cast<const f32x4 *>(row + 64 * t);
        }
    };

    // ---- the rows of an item
    PagedItem cur;
    f32x4 qf[NJ], o[NT][4];
    float m, lsum;   // lsum: this lane's quarter of the row sum
    int last = 0, last_min = 0, seg0 = 0;
    bool no_page = false;
    auto rows = [&](int first_half) __attribute__((always_inline)) {
        PagedArgs &p = paged_args();
        cur = walk.item;
        seg0 = first_half;
        no_page = false;
        const int l = div_by(cur.lh, p.by_Hkv), hkv = cur.lh - l * p.Hkv;
        const int r = cur.tile * TR + n, i = div_by(r, p.by_G), ii = max(0, min(i, cur.n - 1)), row = min(cur.first + ii, p.batch.n_rows - 1);
        last = last_seen(cur.len, cur.n, ii, p.batch.cap);
        last_min = last_seen(cur.len, cur.n, min(div_by(cur.tile * TR, p.by_G), cur.n - 1), p.batch.cap);
        const float *q = static_cast<const float *>(p.q) + l * p.s_q.layer + (int64_t)(hkv * p.G + r - i * p.G) * p.s_q.head + (int64_t)row * p.s_q.token + 4 * g;
#pragma unroll
        for (int j = 0; j < NJ; ++j) qf[j] = *reinterpret_cast<const f32x4 *>(q + 16 * j);
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int c = 0; c < 4; ++c) o[t][c] = f32x4{0.f, 0.f, 0.f, 0.f};
        m = first_reference(cur, seg0, last);
        lsum = 0.f;
    };

    while (walk.begin(wave, pos, end, h)) {   // (again where a segment has been computed by the formula: nothing is kept for the walk across that)
    enter();
#pragma unroll
    for (int j = 0; j < NJ; ++j) k[j] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int t = 0; t < NT; ++t) v[r][t] = f32x4{0.f, 0.f, 0.f, 0.f};
    Sub x = sub_at(h, 0);
    int part = 0;
    load_k(x);
    load_v(x);
    rows(h);

    while (true) {
        const bool ends = part == 1 && h + 1 == cur.count;   // the item
        pos += part;
        bool more = part == 0 || (pos < end && !(ends && walk.pad > 1)) || (!p.slot_o && !ends);
        int nh = h + part;
        const int npart = part ^ 1;
        no_page |= !x.page;
        if (more && ends) {
            more = walk.next();
            nh = 0;
            if (more) enter();
        }
        Sub nx = x;
        if (more) nx = sub_at(nh, npart);

        f32x4 s = {0.f, 0.f, 0.f, 0.f};   // score r of this lane: key 4 * g + r
#pragma unroll
        for (int j = 0; j < NJ; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) s = __builtin_amdgcn_mfma_f32_16x16x4f32(k[j][e], qf[j][e], s, 0, 0, 0);
        if (more) load_k(nx);
        if ((x.prefix ? p.n_prefix - 1 : last_min) - x.at < 15) {   // some key is hidden from some row
            const int limit = (x.prefix ? p.n_prefix - 1 : last) - x.at - 4 * g;
#pragma unroll
            for (int r = 0; r < 4; ++r)
                if (r > limit) s[r] = -INFINITY;
        }
        const float mx = query_max(fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3])));
        if (__builtin_amdgcn_ballot_w64(mx > m) != 0) {
            const float m_new = fmaxf(m, mx);
            const float corr = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((m - m_new) * p.scale_log2);
            lsum *= corr;
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int c = 0; c < 4; ++c) o[t][c] *= corr;
            m = m_new;
        }
        const float ref = m == -INFINITY ? 0.f : m;   // a row that sees no key: exponentials 0
#pragma unroll
        for (int r = 0; r < 4; ++r) s[r] = __builtin_amdgcn_exp2f((s[r] - ref) * p.scale_log2);
        lsum += (s[0] + s[1]) + (s[2] + s[3]);
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int c = 0; c < 4; ++c) o[t][c] = __builtin_amdgcn_mfma_f32_16x16x4f32(v[r][t][c], s[r], o[t][c], 0, 0, 0);
        if (more) load_v(nx);

        if (ends || !more) {
            // ---- the segment [seg0, h] of the item is done.  Lane (n, g) holds channels 64 * t + 16 * g + 4 * r + c of row n.
            PagedArgs &p = paged_args();
            const PagedPlace to = paged_place<TR>(p, cur, seg0, h, pos, walk.run, wave, lane);
            if (x.limit == 0) {   // an item without tokens: nothing was loaded, and what an earlier item has left in the registers does not count
#pragma unroll
                for (int i = 0; i < 4 * NT; ++i) o[i / 4][i % 4] = f32x4{0.f, 0.f, 0.f, 0.f};
            }
            lsum = query_sum(lsum);
            float zero = lsum * 0.f;
#pragma unroll
            for (int i = 0; i < 16 * NT; ++i) zero = fmaf(o[i / 16][i / 4 % 4][i % 4], 0.f, zero);
            if (__builtin_expect(__builtin_amdgcn_ballot_w64(no_page || paged_state_is_odd(zero, m, lsum)) != 0, 0)) {
                paged_exact_segment<float, D, TR>(p, cur, to, seg0, h, lane);
                if (!more) return;
                break;
            }
            const PagedRow row = paged_row(p, cur, to, TR, n);
            f32x4 pieces[D / 16];
#pragma unroll
            for (int i = 0; i < D / 16; ++i) pieces[i] = f32x4{o[i / 4][0][i % 4], o[i / 4][1][i % 4], o[i / 4][2][i % 4], o[i / 4][3][i % 4]};
            if (row.valid) paged_finish_row<float, D>(p, to, row, g, m, lsum, pieces, [&](int i) { return 64 * (i / 4) + 16 * g + 4 * (i % 4); });
            if (!more) return;
            rows(nh);
        }
        x = nx;
        h = nh;
        part = npart;
    }
    }
}

}  // namespace

namespace kvc {

int launch_paged_f32(const PagedAttnParams &p, hipStream_t s)
{
    const dim3 grid((unsigned)(p.n_waves / kPagedBlockWaves)), block(64 * kPagedBlockWaves);
    switch (p.D) {
        case 64: return launch(attn_paged_f32_kernel<64>, grid, block, 0, s, p);
        case 128: return launch(attn_paged_f32_kernel<128>, grid, block, 0, s, p);
        default: return launch(attn_paged_f32_kernel<256>, grid, block, 0, s, p);
    }
}

}  // namespace kvc
