// bf16 attention of few rows over pages and a prefix (decoded tokens): single wavefronts on the walk of attn_paged.h.
#include "attn_paged.h"

namespace {

using namespace kvc;

template <int N>
__device__ __forceinline__ void wait_loads()   // at most N of this wavefront's vector-memory operations stay outstanding
{
    asm volatile("s_waitcnt vmcnt(%0)" : : "n"(N) : "memory");
}
__device__ __forceinline__ void wait_lds() { asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory"); }

// attn_paged_rows_kernel: 16 * RH packed rows on 16x16x32 MFMAs, products, operand layout and LDS swizzles as in attn_rows_kernel16, but a wavefront is alone: it
// walks 32 keys after the other of its run, K and V of a half go global -> LDS into its own 64 * D bytes, and those of the next half, of whatever item, are
// requested as soon as the operands of this one are in registers.  Nothing is joined inside the launch, so that no wavefront waits for another one.
// A half lies in one page or in two, whose entries are read, through the scalar cache, a half ahead.
// What bounds it: HBM in large launches.  32 layers, 16 sequences of 500 to 16 000 tokens (13.5 GB) 2.01 ms = 6.7 TB/s, every byte read once; a
// prefix of 32 768 for four sequences (4.3 GB) 0.69 ms.  In small ones the chain of a wavefront: one layer, 8 sequences (55 MB) 13 us, of which the first
// rows arrive after 4.5 and the halves after that take 1.1 each.
// Wavefronts of a compute unit, the large launch, ms with cached / non-temporal loads: 10 (what fits LDS) 2.38 / 2.18, 8 2.20 / 2.01, 6 - / 2.07, 4 - / 1.99
// (4 leave the small launches' chains longer).  Wavefronts of a block, large launch / fp32 kernel of the tiny one: 1 2.08 ms / 9.2 us, 2 2.08 / 9.2, 4 2.00 / 8.2, 8 2.01 / 10.0.
template <int D, int RH>
__global__ __launch_bounds__(64 * kPagedBlockWaves, RH == 2 || D >= 128 ? 2 : 4) void attn_paged_rows_kernel(const PagedAttnParams)
{
    PagedArgs &p = paged_args();
    await_paged_args(p);
    constexpr int TR = 16 * RH;
    constexpr int NF = D / 16, KCH = D / 8, ROWB = D * 2, HALFB = 32 * ROWB;
    constexpr int RPL = 64 / KCH, LPT = 32 / RPL;              // key rows filled by one wavefront-wide direct load, loads of a half
    constexpr int KD = 16 / RPL, VD = RPL < 8 ? 8 / RPL : 1;   // loads after which the swizzle pattern of the rows repeats
    constexpr bool NT = true;   // non-temporal: nobody reads a half again in this launch
    auto k_swz = [](int key) __attribute__((always_inline)) -> int { return D == 64 ? (key >> 1) & 7 : key & 15; };
    auto v_swz = [](int key) __attribute__((always_inline)) -> int {
        return D == 64 ? (2 * (key & 2)) | ((key >> 1) & 2) : 4 * (key & 3) | ((key >> 1) & 2);
    };
    constexpr int NW = kPagedBlockWaves;   // of a block, which share nothing but their arguments' way to the caches
    __shared__ __align__(16) unsigned char smem[NW * 2 * HALFB];
    const int wave = __builtin_amdgcn_readfirstlane((int)blockIdx.x * NW + (int)(threadIdx.x >> 6));
    const int lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4, lq = lane / KCH;
    lds_byte *kbuf = (lds_byte *)smem + (wave % NW) * 2 * HALFB, *vbuf = kbuf + HALFB;

    PagedWalk<TR> walk(lane);
    int64_t pos = -1, end;
    int h;

    // ---- where the halves of an item lie
    const unsigned char *kp, *vp, *kf, *vf;   // (layer, head) of the pools and of the prefix
    const_int *table = nullptr;
    int tokens = 0;                           // of the sequence that exist
    auto enter = [&]() __attribute__((always_inline)) {   // walk.item
        PagedArgs &p = paged_args();
        const PagedItem &it = walk.item;
        const int l = div_by(it.lh, p.by_Hkv), hkv = it.lh - l * p.Hkv;
        kp = reinterpret_cast<const unsigned char *>(static_cast<const bf16_t *>(p.k) + l * p.s_k.layer + hkv * p.s_k.head);
        vp = reinterpret_cast<const unsigned char *>(static_cast<const bf16_t *>(p.v) + l * p.s_v.layer + hkv * p.s_v.head);
        kf = reinterpret_cast<const unsigned char *>(static_cast<const bf16_t *>(p.prefix_k) + l * p.s_pk.layer + hkv * p.s_pk.head);
        vf = reinterpret_cast<const unsigned char *>(static_cast<const bf16_t *>(p.prefix_v) + l * p.s_pv.layer + hkv * p.s_pv.head);
        tokens = it.b < 0 ? 0 : min(it.len, p.batch.cap);
        table = scalar(p.batch.table) + (int64_t)max(it.b, 0) * p.batch.table_stride;
    };
    struct Half {       // of an item, to be loaded
        int at, limit;  // first key of the prefix or token of the pages, and how many there are: 0: an item without tokens, nothing is read
        int prefix;     // truth value (as bool it left bytes between, which were copied through memory)
        int page[2];    // of the tokens at ... and at + 16 ...
    };
    auto half_at = [&](int h_) __attribute__((always_inline)) -> Half {
        Half x = {32 * h_, p.n_prefix, h_ < walk.item.walk, {0, 0}};
        if (!x.prefix) {
            x.at -= 32 * walk.item.walk;
            x.limit = tokens;
            if (tokens > 0) {
                x.page[0] = table[x.at >> p.batch.log_page];
                x.page[1] = table[min(x.at + 16, tokens - 1) >> p.batch.log_page];
            }
        }
        return x;
    };
    auto is_page = [&](int e) __attribute__((always_inline)) -> bool { return (uint32_t)e < (uint32_t)p.batch.n_pages; };
    uint32_t k_chunk[KD], v_chunk[VD];   // bytes inside a row that this lane fetches
#pragma unroll
    for (int i = 0; i < KD; ++i) k_chunk[i] = ((lane % KCH) ^ k_swz(i * RPL + lq)) * 16;
#pragma unroll
    for (int i = 0; i < VD; ++i) v_chunk[i] = ((lane % KCH) ^ v_swz(i * RPL + lq)) * 16;
    bool no_page = false;   // of the segment
    // The rows of a half from `base` on, pages (of one prefix: none) and rows so many bytes apart.  Rows behind the last one are read as that one.
    auto load = [&](const Half &x, const unsigned char *base, int64_t page_bytes, uint32_t row_bytes, auto &chunk, auto swz, lds_byte *dst) __attribute__((always_inline)) {
        constexpr int NC = sizeof(chunk) / sizeof(chunk[0]);
        const int mask = x.prefix ? INT32_MAX : (1 << p.batch.log_page) - 1;
        if (__builtin_expect(x.at + 32 <= x.limit, 1)) {
            const uint32_t in = (uint32_t)lq * row_bytes;
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const int page = is_page(x.page[half]) ? x.page[half] : 0;
                const unsigned char *row = base + (x.prefix ? 0 : page * page_bytes) + (uint64_t)(uint32_t)((x.at + 16 * half) & mask) * row_bytes;
#pragma unroll
                for (int i = half * LPT / 2; i < (half + 1) * LPT / 2; ++i, row += RPL * (uint64_t)row_bytes) dma16_sbase<NT>(row, in + chunk[i % NC], dst + i * RPL * ROWB);
            }
        } else if (x.limit > 0) {
#pragma unroll 1
            for (int i = 0; i < LPT; ++i) {
                const int r = min(x.at + i * RPL, x.limit - 1), e = x.page[r >= x.at + 16];   // (page[1] where that is behind the last one: the last one's)
                const unsigned char *row = base + (x.prefix ? 0 : (is_page(e) ? e : 0) * page_bytes) + (uint64_t)(uint32_t)(r & mask) * row_bytes;
                dma16_sbase<NT>(row, (uint32_t)min(lq, x.limit - 1 - r) * row_bytes + ((lane % KCH) ^ swz(i * RPL + lq)) * 16, dst + i * RPL * ROWB);
            }
        }
    };
    auto load_k = [&](const Half &x) __attribute__((always_inline)) {
        load(x, x.prefix ? kf : kp, p.s_k.page * 2, (uint32_t)(x.prefix ? p.s_pk.token : p.s_k.token) * 2, k_chunk, k_swz, kbuf);
    };
    auto load_v = [&](const Half &x) __attribute__((always_inline)) {
        load(x, x.prefix ? vf : vp, p.s_v.page * 2, (uint32_t)(x.prefix ? p.s_pv.token : p.s_v.token) * 2, v_chunk, v_swz, vbuf);
    };

    // ---- the rows of an item
    PagedItem cur;
    bf16x8 qf[RH][NF / 2];
    int last[RH], last_min = 0;    // last token that this lane's row sees, and that the tile's first row does
    f32x4 o[RH][NF];
    float m[RH], mc[RH], lsum[RH];   // lsum: this lane's quarter of the row sum
    int seg0 = 0;                    // first half of the segment
    auto rows = [&](int first_half) __attribute__((always_inline)) {
        PagedArgs &p = paged_args();
        cur = walk.item;
        seg0 = first_half;
        no_page = false;
        const int l = div_by(cur.lh, p.by_Hkv), hkv = cur.lh - l * p.Hkv;
        last_min = last_seen(cur.len, cur.n, min(div_by(cur.tile * TR, p.by_G), cur.n - 1), p.batch.cap);
#pragma unroll
        for (int x = 0; x < RH; ++x) {
            const int r = cur.tile * TR + 16 * x + n, i = div_by(r, p.by_G), ii = max(0, min(i, cur.n - 1));
            const int row = min(cur.first + ii, p.batch.n_rows - 1);
            last[x] = last_seen(cur.len, cur.n, ii, p.batch.cap);
            const bf16_t *q = static_cast<const bf16_t *>(p.q) + l * p.s_q.layer + (int64_t)(hkv * p.G + r - i * p.G) * p.s_q.head + (int64_t)row * p.s_q.token;
#pragma unroll
            for (int ks = 0; ks < NF / 2; ++ks) qf[x][ks] = as_bf16x8(load16(q + ks * 32 + g * 8));
#pragma unroll
            for (int db = 0; db < NF; ++db) o[x][db] = f32x4{0.f, 0.f, 0.f, 0.f};
            m[x] = first_reference(cur, seg0, last[x]), mc[x] = 0.f, lsum[x] = 0.f;
        }
        __builtin_amdgcn_s_waitcnt(0x0f70);   // vmcnt(0), seen by the compiler: it puts no wait for the queries into the loop
    };

    // Operand addresses: K chunk 4 * ks + g of key n (and 16 + n); V^T is transposed on the way out of LDS.
    int k_off[NF / 2], v_off[NF];
#pragma unroll
    for (int ks = 0; ks < NF / 2; ++ks) k_off[ks] = n * ROWB + (((4 * ks + g) ^ k_swz(n)) * 16);
    {
        const int row = 4 * g + (n >> 2);
#pragma unroll
        for (int db = 0; db < NF; ++db) {
            const int col = 16 * db + 4 * (n & 3);
            v_off[db] = row * ROWB + ((col >> 3) ^ v_swz(row)) * 16 + (col & 7) * 2;
        }
    }

    while (walk.begin(wave, pos, end, h)) {   // (again where a segment has been computed by the formula: nothing is kept for the walk across that)
    enter();
    Half x = half_at(h);
    load_k(x);
    load_v(x);
    rows(h);
    while (true) {
        const bool ends = h + 1 == cur.count;   // the item
        ++pos;
        bool more = (pos < end && !(ends && walk.pad > 1)) || (!p.slot_o && !ends);
        int nh = h + 1;
        if (!x.prefix) no_page |= x.limit > 0 && !(is_page(x.page[0]) && is_page(x.page[1]));
        if (more && ends) {
            more = walk.next();
            nh = 0;
            if (more) enter();
        }
        Half nx = x;
        if (more) nx = half_at(nh);

        // Every counted wait below stands behind loads that are certain to have been issued: a half has LPT loads of K and LPT of V, or, where its
        // item has no tokens (limit 0), none of either.
        wait_loads<LPT>();               // K has landed (V may be outstanding)
        bf16x8 ka[NF];                   // all operand reads in flight at once: ks = i / 2, keys 16 * (i & 1) ...
#pragma unroll
        for (int i = 0; i < NF; ++i) ka[i] = as_bf16x8(*(const __attribute__((address_space(3))) u32x4 *)(kbuf + (i & 1) * 16 * ROWB + k_off[i >> 1]));
        wait_lds();                      // K has been read: its buffer is free
        if (more) load_k(nx);
        f32x4 s[RH][2];                  // score j of this lane: key 16 * (j / 4) + 4 * g + j % 4
#pragma unroll
        for (int i = 0; i < NF; ++i)
#pragma unroll
            for (int r = 0; r < RH; ++r)
                s[r][i & 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ka[i], qf[r][i >> 1], i < 2 ? f32x4{0.f, 0.f, 0.f, 0.f} : s[r][i & 1], 0, 0, 0);
        if ((x.prefix ? p.n_prefix - 1 : last_min) - x.at < 31) {   // some key is hidden from some row
#pragma unroll
            for (int r = 0; r < RH; ++r) {
                const int limit = (x.prefix ? p.n_prefix - 1 : last[r]) - x.at - 4 * g;
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (16 * (j >> 2) + (j & 3) > limit) s[r][j >> 2][j & 3] = -INFINITY;
            }
        }
        float mx[RH];
        bool grows = false;
#pragma unroll
        for (int r = 0; r < RH; ++r) {
            mx[r] = s[r][0][0];
#pragma unroll
            for (int j = 1; j < 8; ++j) mx[r] = fmaxf(mx[r], s[r][j >> 2][j & 3]);
            mx[r] = query_max(mx[r]);
            grows |= mx[r] > m[r];
        }
        if (__builtin_amdgcn_ballot_w64(grows) != 0) {
#pragma unroll
            for (int r = 0; r < RH; ++r) {   // (a row whose reference stays is multiplied by 1)
                const float m_new = fmaxf(m[r], mx[r]);
                const float corr = m[r] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((m[r] - m_new) * p.scale_log2);
                lsum[r] *= corr;
#pragma unroll
                for (int db = 0; db < NF; ++db) o[r][db] *= corr;
                m[r] = m_new;
                mc[r] = m[r] == -INFINITY ? 0.f : m[r] * p.scale_log2;   // a row that sees no key: exponentials 0
            }
        }
        // Probabilities are rounded to bf16 for the second product, as in the other attention kernels; their sums take them unrounded.
        bf16x8 pf[RH];
#pragma unroll
        for (int r = 0; r < RH; ++r) {
            u32x4 pk;
            float rs0 = 0.f, rs1 = 0.f;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float e0 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[r][j >> 1][2 * (j & 1)], p.scale_log2, -mc[r]));
                const float e1 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[r][j >> 1][2 * (j & 1) + 1], p.scale_log2, -mc[r]));
                rs0 += e0;
                rs1 += e1;
                pk[j] = pack_bf16x2(e0, e1);
            }
            pf[r] = as_bf16x8(pk);
            lsum[r] += rs0 + rs1;
        }
        if (more && nx.limit > 0)
            wait_loads<LPT>();   // V has landed (K of the next half may be outstanding)
        else
            wait_loads<0>();     // (no K behind it)
        bf16x8 va[NF];
#pragma unroll
        for (int db = 0; db < NF; ++db) va[db] = lds_read_tr_pair(vbuf + v_off[db], vbuf + v_off[db] + 16 * ROWB);
        wait_lds();                      // V has been read
        if (more) load_v(nx);
#pragma unroll
        for (int db = 0; db < NF; ++db)
#pragma unroll
            for (int r = 0; r < RH; ++r) o[r][db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(va[db], pf[r], o[r][db], 0, 0, 0);

        if (ends || !more) {
            // ---- the segment [seg0, h] of the item is done
            PagedArgs &p = paged_args();
            const PagedPlace to = paged_place<TR>(p, cur, seg0, h, pos, walk.run, wave, lane);
            bool odd = no_page;
            if (x.limit == 0) {   // an item without tokens: nothing was loaded, and what earlier work has left in LDS, NaN perhaps, does not count
#pragma unroll
                for (int i = 0; i < RH * NF; ++i) o[i / NF][i % NF] = f32x4{0.f, 0.f, 0.f, 0.f};
            }
#pragma unroll
            for (int r = 0; r < RH; ++r) {
                lsum[r] = query_sum(lsum[r]);
                float zero = lsum[r] * 0.f;
#pragma unroll
                for (int i = 0; i < 4 * NF; ++i) zero = fmaf(o[r][i / 4][i % 4], 0.f, zero);
                odd |= paged_state_is_odd(zero, m[r], lsum[r]);
            }
            if (__builtin_expect(__builtin_amdgcn_ballot_w64(odd) != 0, 0)) {
                paged_exact_segment<bf16_t, D, TR>(p, cur, to, seg0, h, lane);
                if (!more) return;
                wait_loads<0>();   // (the next half's, which is requested again)
                break;
            }
#pragma unroll
            for (int r = 0; r < RH; ++r) {
                const PagedRow row = paged_row(p, cur, to, TR, 16 * r + n);
                if (row.valid) paged_finish_row<bf16_t, D>(p, to, row, g, m[r], lsum[r], o[r], [&](int i) { return 16 * i + 4 * g; });
            }
            if (!more) return;
            rows(nh);
        }
        x = nx;
        h = nh;
    }
    }
}

}  // namespace

namespace kvc {

int launch_paged_rows(const PagedAttnParams &p, int tile_rows, hipStream_t s)
{
    const dim3 grid((unsigned)(p.n_waves / kPagedBlockWaves)), block(64 * kPagedBlockWaves);
    const bool one = tile_rows == 16;
    switch (p.D) {
        case 64: return launch(one ? attn_paged_rows_kernel<64, 1> : attn_paged_rows_kernel<64, 2>, grid, block, 0, s, p);
        case 128: return launch(one ? attn_paged_rows_kernel<128, 1> : attn_paged_rows_kernel<128, 2>, grid, block, 0, s, p);
        default: return launch(attn_paged_rows_kernel<256, 1>, grid, block, 0, s, p);
    }
}

}  // namespace kvc
