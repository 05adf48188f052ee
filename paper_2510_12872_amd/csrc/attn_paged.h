// Attention of a batch of sequences over the pages of a pool, behind a cache that all of them continue: what its kernels share.
//   out_i = softmax_j(scale <q_i, k_j>) v_j   over the prefix's tokens and the tokens of row i's sequence up to its own.
// Keys are counted in halves of tiles, 32 each.  An item of work is a tile of packed (row, query head) rows r = i * G + g of one kv head, of one
// sequence over its pages (and over the prefix before them, where that is not done for all sequences together), or of all sequences over the prefix.
//
// The walk of the wavefront kernels (attn_paged_rows.hip, attn_paged_f32.hip): the halves of all items of all (layer, kv head) pairs lie behind each
// other on one axis, which is cut into as many equal runs as wavefronts fit the chip.  Every wavefront walks its run, whatever the lengths are, without a word to
// another one.  An item that lies in one run is finished there.  Of one that does not, each wavefront leaves its part: unnormalised output, reference and sum of each
// row, in the second of its two slots, or, if it holds the item's last half, in the first.  attn_paged_combine_kernel joins them.
#pragma once

#include <float.h>

#include "attn_common.h"
#include "paged.h"

namespace kvc {

struct PagedAttnParams {
    const void *q, *k, *v, *prefix_k, *prefix_v;
    void *out;
    float *lse;
    Strides s_q, s_o, s_pk, s_pv;
    PoolStrides s_k, s_v;
    Batch batch;
    int32_t L, Hkv, G, D, n_prefix;
    float scale, scale_log2;
    divisor_t by_G, by_Hkv;
    // The plan.
    int32_t walked_prefix;   // halves of the prefix before a sequence's own: all of them or, where the prefix has items of its own, 0
    int32_t prefix_tiles;    // row tiles of the prefix's items on the wavefronts' axis
    int32_t prefix_runs;     // or: runs that the tiles kernel cuts the prefix into
    int32_t prefix_part;     // first part by rows that is the prefix's
    int32_t tile_runs;       // runs of a sequence that the tiles kernel takes
    int32_t tile_rows;
    int32_t n_waves;         // runs of the axis
    float per_wave;          // 1 / n_waves and a little
    int32_t most_rows;       // packed rows of the sequences that the launch takes
    int32_t max_items;       // of a (layer, kv head) on the axis, at most
    // Scratch, or null: then an item is the work of the wavefront in whose run it begins.  A row's part: D outputs; reference and sum.
    float *slot_o, *slot_ml;   // [n_waves][2][tile rows]
    float *row_o, *row_ml;     // parts by rows, [part][layer, query head, row]: whole items or the tiles kernel's runs of sequences, then the prefix's
    int32_t *items;            // [layer, kv head][max_items][2]: first and last wavefront of an item; kDirect, kWhole
    int32_t *item_of;          // [n_rows][2]: item of its sequence's first tile, its number in the sequence; kDirect, kWhole: the tiles kernel's
};
// A wavefront kernel's parameters, where they are used: what is read once per item is loaded there and not kept in scalar registers all along.  (There are too few of them all the same: 91 to
// 121 are spilled, to lanes of vector registers and not to memory, and some read back in the loop over the halves.)
typedef const __attribute__((address_space(4))) PagedAttnParams PagedArgs;
__device__ __forceinline__ PagedArgs &paged_args()
{
    PagedArgs *p = (PagedArgs *)__builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(p));
    return *p;
}
__device__ __forceinline__ void await_paged_args(PagedArgs &p)   // see await_args(): a word of each 64-byte line
{
    auto word = [&](int line) { return *(const __attribute__((address_space(4))) uint32_t *)((const __attribute__((address_space(4))) char *)&p + 64 * line); };
    constexpr int last = (sizeof(PagedAttnParams) - 1) / 64;
    static_assert(last >= 5 && last <= 7, "six to eight lines");
    await_args(word(0), word(1), word(2), word(3), word(4), word(5), word(last - 1), word(last));
}
enum : int32_t { kDirect = -1, kWhole = -2 };   // its rows lie in `out`; in row_o

// The rows of all sequences.
template <class P>   // PagedAttnParams, in any address space
__device__ __forceinline__ void all_rows(const P &p, int &first, int &n)
{
    first = p.batch.starts ? max(0, min(p.batch.starts[0], p.batch.n_rows)) : 0;
    n = p.batch.starts ? max(0, min(p.batch.starts[p.batch.n_seqs], p.batch.n_rows) - first) : p.batch.n_rows;
}

// A sequence's tokens from row i of n on: the last one that it sees, -1 or less: none.
__device__ __forceinline__ int last_seen(int len, int n, int i, int cap) { return min(len - n + i, min(len, cap) - 1); }

// The same parameters, loaded again where they are used from here on: nothing that was read of them before is kept across this.
template <class P>
__device__ __forceinline__ P &again(P &p)
{
    P *q = &p;
    asm volatile("" : "+s"(q));
    return *q;
}

// The reference that a row, or a part of one, begins with if it sees a key: if none of its scores is above -infinity, it ends with that and sum 0, which beside
// another part's score weighs nothing and alone is the formula's 0 / 0.  A row that sees no key has -infinity all along, and becomes 0.
constexpr float kNoScore = -FLT_MAX;
__device__ __forceinline__ bool paged_state_is_odd(float zero, float m, float sum) { return state_is_odd(zero, m <= kNoScore ? -INFINITY : m, sum); }

// One row (sequence b, row `row` of the queries, query head hq) over the halves [h0, h1) by the formula, key by key, in fp32; what the row does not
// see (`last`: the last token of its pages that it sees) is not looked at.  Whole rows: halves 0 ... of the prefix, then of the pages.
// Returns reference and sum; lanes 0 ... D / 8 - 1 hold channels 8 * lane ... of the unnormalised output.
template <typename T, int D, class P>
__device__ __forceinline__ void paged_exact_row(const P &p0, int l, int hkv, int hq, int row, int b, int last, int prefix_halves, int h0, int h1, int lane,
                                                float &m, float &sum, float (&o)[8])
{
    constexpr int CL = D / 8, EPV = Elem<T>::EPV;
    auto at = [&](const P &p, int x, bool values) __attribute__((always_inline)) -> const T * {   // row of key x, counted from half 0; null: not there
        if (x < 32 * prefix_halves) {
            if (x >= p.n_prefix) return nullptr;
            const int64_t layer = values ? p.s_pv.layer : p.s_pk.layer, head = values ? p.s_pv.head : p.s_pk.head, token = values ? p.s_pv.token : p.s_pk.token;
            return static_cast<const T *>(values ? p.prefix_v : p.prefix_k) + l * layer + hkv * head + (int64_t)x * token;
        }
        const int t = x - 32 * prefix_halves;
        if (t > last) return nullptr;
        const int page = page_of(p.batch, b, t);
        if (page < 0) return nullptr;
        const int64_t layer = values ? p.s_v.layer : p.s_k.layer, head = values ? p.s_v.head : p.s_k.head, token = values ? p.s_v.token : p.s_k.token;
        return static_cast<const T *>(values ? p.v : p.k) + l * layer + hkv * head + (int64_t)page * (values ? p.s_v.page : p.s_k.page) +
               (int64_t)(t & ((1 << p.batch.log_page) - 1)) * token;
    };
    auto load8 = [](const T *src, float (&x)[8]) {
#pragma unroll
        for (int i = 0; i < 8 / EPV; ++i) {
            float y[EPV];
            unpack<T>(load16(src + i * EPV), y);
#pragma unroll
            for (int j = 0; j < EPV; ++j) x[i * EPV + j] = y[j];
        }
    };
    m = -INFINITY;
    sum = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) o[j] = 0.f;
    const int end = (int)min((int64_t)32 * h1, (int64_t)32 * prefix_halves + last + 1);
#pragma unroll 1
    for (int x0 = 32 * h0; x0 < end && sum == sum; x0 += 64) {   // a key per lane; a sum that is not a number stays so, and the row with it
        const P &p = again(p0);
        const T *q = static_cast<const T *>(p.q) + l * p.s_q.layer + (int64_t)hq * p.s_q.head + (int64_t)row * p.s_q.token;
        const T *kr = x0 + lane < end ? at(p, x0 + lane, false) : nullptr;
        const bool seen = kr != nullptr;
        float s = -INFINITY;
        if (seen) {
            s = 0.f;
#pragma unroll 1
            for (int c = 0; c < D; c += 8) {
                float kk[8], qq[8];
                load8(kr + c, kk);
                load8(q + c, qq);
#pragma unroll
                for (int j = 0; j < 8; ++j) s = fmaf(qq[j], kk[j], s);
            }
        }
        float mx = seen ? fmaxf(s, kNoScore) : -INFINITY;
#pragma unroll
        for (int off = 32; off >= 1; off >>= 1) mx = fmaxf(mx, __shfl_xor(mx, off));
        const float m_new = fmaxf(m, mx);
        const float corr = m == -INFINITY ? 0.f : exp2f((m - m_new) * p.scale_log2);
        m = m_new;
        const float e = seen ? exp2f((s - (m == -INFINITY ? 0.f : m)) * p.scale_log2) : 0.f;
        float es = e;
#pragma unroll
        for (int off = 32; off >= 1; off >>= 1) es += __shfl_xor(es, off);
        sum = sum * corr + es;
#pragma unroll
        for (int j = 0; j < 8; ++j) o[j] *= corr;
        for (uint64_t todo = __builtin_amdgcn_ballot_w64(seen); todo; todo &= todo - 1) {
            const int j = __builtin_ctzll(todo);
            const float pj = __shfl(e, j);
            if (lane < CL) {
                float vv[8];
                load8(at(again(p0), x0 + j, true) + 8 * lane, vv);
#pragma unroll
                for (int c = 0; c < 8; ++c) o[c] = fmaf(pj, vv[c], o[c]);
            }
        }
    }
}

// The row's result.  A row that saw nothing: 0 and -infinity.
template <typename T, int D, class P>
__device__ __forceinline__ void paged_store_row(const P &p, int l, int hq, int row, int lane, float m, float sum, const float (&o)[8])
{
    constexpr int EPV = Elem<T>::EPV;
    const bool none = m == -INFINITY && sum == 0.f;
    if (lane < D / 8) {
        T *out = static_cast<T *>(p.out) + l * p.s_o.layer + (int64_t)hq * p.s_o.head + (int64_t)row * p.s_o.token + 8 * lane;
#pragma unroll
        for (int h = 0; h < 8 / EPV; ++h) {
            float x[EPV];
#pragma unroll
            for (int j = 0; j < EPV; ++j) x[j] = none ? 0.f : o[h * EPV + j] / sum;
            *reinterpret_cast<u32x4 *>(out + h * EPV) = pack<T>(x);
        }
    }
    if (p.lse && lane == 0) p.lse[((int64_t)l * p.Hkv * p.G + hq) * p.batch.n_rows + row] = none ? -INFINITY : m * p.scale + logf(sum);
}

// ------------------------------------------------------------------------------------------ the walk
// Runs of up to so many halves are cut within items.  (What is cut so has up to twice as many: half of the wavefronts may be the items' last ones.)  us for the whole call, D = 128, 8 kv heads, G = 4,
// cut within items / across them, halves of a run: 8 sequences, one layer, 1.1 16.2 / 16.8, 2.8 22.6 / 23.5, 4.8 34.2 / 34.9, 7.3 45.4 / 46.6, 10.4 61.3 / 61.4, 19 106.8 / 106.9; 32 sequences 1.2 16.5 / 17.3,
// 4.5 32.4 / 33.5, 8.5 52.4 / 52.9, 18 101.6 / 103.3; fp32 1.9 29.4 / 29.1, 5.5 75.9 / 75.3, 10.3 133.3 / 130.8: longer ones gain 1 % or lose 2.
// The shortest run in any case is one half: one layer, prefix 2560 and 8 tokens, with runs of 1 / 2 / 4 / 8 halves at least: 12.4 / 15.5 / 21.9 / 37.3 us.
constexpr int kPagedShortRun = 8;
// Halves of a run, at most: longer ones are refused before the launch.
constexpr int kPagedMostRun = 1000000000;
typedef const __attribute__((address_space(4))) int32_t const_int;   // read through the scalar cache (whole-wavefront values)
__device__ __forceinline__ const_int *scalar(const int32_t *x) { return (const_int *)(uintptr_t)x; }

// An item; all of it the same in all lanes.
struct PagedItem {
    int lh, b;          // b < 0: the rows of all sequences over the prefix
    int tile, tiles;    // row tile, row tiles of the sequence
    int first, n;       // rows
    int len;            // tokens by `lens`
    int walk;           // halves of the prefix at the item's beginning
    int count;          // halves of the tile, 1 at least (an item without keys has its place on the axis)
    int index;          // among the items of lh
};

// Sum over the lanes up to each one's.
__device__ __forceinline__ int wave_scan(int x)
{
    auto add = [](int v, auto ctrl, auto rows) { return v + __builtin_amdgcn_update_dpp(0, v, decltype(ctrl)::value, decltype(rows)::value, 0xf, false); };
    x = add(x, std::integral_constant<int, 0x111>{}, std::integral_constant<int, 0xf>{});   // from one, two, four, eight lanes before in each row of sixteen
    x = add(x, std::integral_constant<int, 0x112>{}, std::integral_constant<int, 0xf>{});
    x = add(x, std::integral_constant<int, 0x114>{}, std::integral_constant<int, 0xf>{});
    x = add(x, std::integral_constant<int, 0x118>{}, std::integral_constant<int, 0xf>{});
    x = add(x, std::integral_constant<int, 0x142>{}, std::integral_constant<int, 0xa>{});   // a row's last lane to the second and the fourth row,
    x = add(x, std::integral_constant<int, 0x143>{}, std::integral_constant<int, 0xc>{});   // the second row's last to the third and the fourth
    return x;
}
// x / d, both positive, the quotient below 2^31
__device__ __forceinline__ int quotient(int64_t x, int64_t d)
{
    int64_t q = (int64_t)((double)x * __builtin_amdgcn_rcp((double)d));   // (next to it at least)
    while (q * d > x) --q;
    while ((q + 1) * d <= x) ++q;
    return (int)q;
}

// The sizes are such that what one (layer, kv head) has on the axis fits 31 bits, and a run, too (paged_attn()).
// What bounds its start is the way to memory: arguments, then rows and lengths of 64 sequences at a time, a lane each, all requested together; from then on
// they are read from the lanes.  (Loaded where they were used, scalars among them, a wavefront took 8 to 15 us to its first item.)
template <int TR>   // packed rows of a tile
struct PagedWalk {
    const int lane;
    int width = 0;   // halves of a (layer, kv head) on the axis
    int run = 0;     // of a wavefront
    int pad = 1;     // items begin at multiples of this on the axis: 1, or `run`
    PagedItem item = {};

    __device__ __forceinline__ explicit PagedWalk(int lane) : lane(lane) {}

    // The item at `pos` of the axis (negative: where the run of wavefront `wave` begins) and its half there; false: the run ends before.
    __device__ __forceinline__ bool begin(int wave, int64_t &pos, int64_t &end, int &h0)
    {
        const Args a;
        pad = 1;
        bool falls = load(a, 0);
        const int before0 = a.prefix_tiles * a.prefix_count();
        int upto = wave_scan(tiles(a) * count(a, len)), before = wave_scan(tiles(a));   // (kept: most batches have no more)
        int ahead = before0, items = a.prefix_tiles + __builtin_amdgcn_readlane(before, 63);
        width = ahead + __builtin_amdgcn_readlane(upto, 63);
        for (int c = 64; c < a.n_seqs; c += 64) {
            falls |= load(a, c);
            width += __builtin_amdgcn_readlane(wave_scan(tiles(a) * count(a, len)), 63);
            items += __builtin_amdgcn_readlane(wave_scan(tiles(a)), 63);
        }
        int64_t total = (int64_t)width * a.heads;
        // (a little more than its share each, so that rounding leaves nothing)
        // Where `starts` falls, sequences may share rows, and have more of them together than the batch: sums that 31 bits do not hold.  Nothing is walked then.
        // (Where it does not, the sequences' rows are those of the batch at most, whose halves the host has counted.)
        if (falls || width <= 0) return false;
        run = __builtin_amdgcn_readfirstlane((int)fminf((float)total * a.per_wave, (float)kPagedMostRun)) + 1;
        // Short runs are cut within items: a wavefront that ends one item and begins another takes as long as two.  The items' last runs may be short then, so there have
        // to be wavefronts enough for one more of each.
        if (run <= kPagedShortRun && a.slots && 2 * (int64_t)items * a.heads <= a.n_waves) {
            run = pad = __builtin_amdgcn_readfirstlane((int)((uint32_t)total / (uint32_t)(a.n_waves - items * a.heads)) + 1);
            ahead = a.prefix_tiles * padded(a.prefix_count());
            width = ahead;
            for (int c = 0; c < a.n_seqs; c += 64) {
                if (chunk != c) load(a, c);
                const int x = wave_scan(tiles(a) * padded(count(a, len)));
                if (c == 0) upto = x;
                width += __builtin_amdgcn_readlane(x, 63);
            }
            total = (int64_t)width * a.heads;
        }
        end = min((int64_t)run * wave + run, total);
        if (pos < 0) pos = (int64_t)run * wave;
        if (pos >= end) return false;
        item.lh = __builtin_amdgcn_readfirstlane(quotient(pos, width));
        int at = (int)(pos - (int64_t)item.lh * width);
        if (at < ahead) {
            const int each = padded(a.prefix_count());
            set_prefix(a, __builtin_amdgcn_readfirstlane(at / each));
            h0 = at - item.tile * each;
        } else {
            at -= ahead;
            int index = a.prefix_tiles;
            for (int c = 0;; c += 64) {
                if (c >= a.n_seqs) return false;
                if (chunk != c) load(a, c);
                if (c) upto = wave_scan(tiles(a) * padded(count(a, len))), before = wave_scan(tiles(a));
                const int sum = __builtin_amdgcn_readlane(upto, 63);
                if (at < sum) {
                    const int j = __builtin_ctzll(__builtin_amdgcn_ballot_w64(upto > at));
                    at -= j ? __builtin_amdgcn_readlane(upto, j - 1) : 0;
                    index += j ? __builtin_amdgcn_readlane(before, j - 1) : 0;
                    todo = __builtin_amdgcn_ballot_w64(tiles(a) > 0 && lane > j);
                    set_sequence(a, j);
                    const int each = padded(item.count);
                    item.tile = item.tiles == 1 ? 0 : __builtin_amdgcn_readfirstlane(at / each);
                    item.index = index + item.tile;
                    h0 = at - item.tile * each;
                    break;
                }
                at -= sum;
                index += __builtin_amdgcn_readlane(before, 63);
            }
        }
        if (!a.slots && h0 > 0) {   // the item is another one's: on to the next
            pos += item.count - h0;
            h0 = 0;
            if (pos >= end) return false;
            return next();
        }
        return true;
    }
    // The item behind it; false: there is none.
    __device__ __forceinline__ bool next()
    {
        ++item.index;
        if (item.tile + 1 < item.tiles) {
            ++item.tile;
            return true;
        }
        const Args a;
        if (item.b < 0) enter(a, 0);   // (from the prefix)
        while (todo == 0) {
            int c = chunk + 64;
            if (c >= a.n_seqs) {
                if (++item.lh >= a.heads) return false;
                item.index = 0;
                if (a.prefix_tiles) {
                    set_prefix(a, 0);
                    return true;
                }
                c = 0;
            }
            enter(a, c);
        }
        const int j = __builtin_ctzll(todo);
        todo &= todo - 1;
        set_sequence(a, j);
        return true;
    }

private:
    int chunk = -1;           // the sequences chunk ... chunk + 63 in the lanes: their rows and lengths
    int first = 0, n = 0, len = 0;
    uint64_t todo = 0;        // those behind the item's that have items here

    struct Args {   // of the launch, requested together
        const int32_t *starts, *lens;
        int n_seqs, n_rows, cap, G, most_rows, walked, prefix_tiles, n_prefix, heads, n_waves;
        float per_wave;
        bool slots;
        __device__ __forceinline__ Args()
        {
            PagedArgs &p = paged_args();
            starts = p.batch.starts, lens = p.batch.lens;
            n_seqs = p.batch.n_seqs, n_rows = p.batch.n_rows, cap = p.batch.cap, G = p.G, most_rows = p.most_rows, walked = p.walked_prefix;
            prefix_tiles = p.prefix_tiles, n_prefix = p.n_prefix, heads = p.L * p.Hkv, n_waves = p.n_waves, per_wave = p.per_wave;
            slots = p.slot_o != nullptr;
            asm volatile("" : : "s"(starts), "s"(lens), "s"(n_seqs), "s"(n_rows), "s"(cap), "s"(G), "s"(most_rows), "s"(walked), "s"(prefix_tiles), "s"(n_prefix), "s"(heads),
                         "s"(n_waves), "s"(per_wave));
        }
        __device__ __forceinline__ int prefix_count() const { return (n_prefix + 31) / 32; }
    };

    __device__ __forceinline__ bool load(const Args &a, int c)   // does `starts` fall there?
    {
        chunk = c;
        const int b = min(c + lane, a.n_seqs - 1);
        const int l = a.lens[b];
        first = b;
        n = 1;
        if (a.starts) {
            const int s0 = a.starts[b], s1 = a.starts[b + 1];
            first = max(0, min(s0, a.n_rows));
            n = max(0, min(s1, a.n_rows)) - first;
        }
        const bool falls = __builtin_amdgcn_ballot_w64(n < 0) != 0;
        n = c + lane < a.n_seqs ? max(0, n) : 0;
        len = max(0, l);
        return falls;
    }
    __device__ __forceinline__ void enter(const Args &a, int c)
    {
        if (chunk != c) load(a, c);
        todo = __builtin_amdgcn_ballot_w64(tiles(a) > 0);
    }
    __device__ __forceinline__ int tiles(const Args &a) const   // of the lane's sequence
    {
        const int rows = n * a.G;
        return rows <= a.most_rows ? (rows + TR - 1) / TR : 0;
    }
    __device__ __forceinline__ static int count(const Args &a, int len) { return max(1, a.walked + (min(len, a.cap) + 31) / 32); }
    __device__ __forceinline__ int padded(int count) const { return pad == 1 ? count : (int)((uint32_t)(count + pad - 1) / (uint32_t)pad) * pad; }
    __device__ __forceinline__ void set_prefix(const Args &a, int tile)
    {
        item.b = -1;
        item.tile = tile;
        item.tiles = a.prefix_tiles;
        item.index = tile;
        item.count = item.walk = a.prefix_count();
        item.len = 0;
        item.first = 0;
        item.n = a.n_rows;
        if (a.starts) {
            const_int *s = scalar(a.starts);
            item.first = max(0, min(s[0], a.n_rows));
            item.n = max(0, min(s[a.n_seqs], a.n_rows) - item.first);
        }
    }
    __device__ __forceinline__ void set_sequence(const Args &a, int j)   // of lane j
    {
        item.b = chunk + j;
        item.first = __builtin_amdgcn_readlane(first, j);
        item.n = __builtin_amdgcn_readlane(n, j);
        item.len = __builtin_amdgcn_readlane(len, j);
        item.tile = 0;
        item.tiles = (item.n * a.G + TR - 1) / TR;
        item.walk = a.walked;
        item.count = count(a, item.len);
    }
};

constexpr int kPagedBlockWaves = 4;   // of a wavefront kernel's block, which share nothing
// Wavefronts of attn_paged_rows_kernel on a compute unit: LDS has room for 10 of 16 KB at D = 128 (8 are faster, see there), 5 at D = 256 and 20 at D = 64, registers for 8 with
// tiles of 32 rows.
constexpr int paged_rows_waves(int D, int rows) { return D == 256 ? 4 : D == 128 || rows == 32 ? 8 : 16; }

constexpr int paged_f32_waves(int D) { return D == 256 ? 4 : 8; }

int launch_paged_rows(const PagedAttnParams &p, int tile_rows, hipStream_t s);
int launch_paged_f32(const PagedAttnParams &p, hipStream_t s);   // tiles of 16 rows

// Where the results of a segment, halves seg0 ... h of an item, go.  pos: the axis behind the segment, run: a wavefront's run of it.
struct PagedPlace {
    int kind;        // kDirect; kWhole: row_o; 0: a slot of the wavefront
    float *o, *ml;   // of the slot's rows, or of rows by (layer, query head, row)
};
template <int TR, class P>
__device__ __forceinline__ PagedPlace paged_place(const P &p, const PagedItem &it, int seg0, int h, int64_t pos, int run, int64_t wave, int lane)
{
    const bool ends = h + 1 == it.count, whole = ends && seg0 == 0;
    // (a prefix with items of its own on this axis: every row is joined; with parts by rows: they are there already)
    PagedPlace to = {whole ? p.prefix_tiles ? kWhole : kDirect : 0, nullptr, nullptr};
    if (!p.slot_o) return to;
    if (to.kind == kWhole) {
        const int64_t all = (int64_t)p.L * p.Hkv * p.G * p.batch.n_rows * (it.b < 0 ? p.prefix_part : 0);
        to.o = p.row_o + all * p.D;
        to.ml = p.row_ml + all * 2;
    } else if (to.kind == 0) {
        const int64_t slot = (2 * wave + (ends ? 0 : 1)) * TR;
        to.o = p.slot_o + slot * p.D;
        to.ml = p.slot_ml + slot * 2;
    }
    if (ends) {
        if (lane < 2 && (uint32_t)it.index < (uint32_t)p.max_items) {
            const int64_t begin = pos - it.count;   // of the item, on the axis
            const int first = to.kind ? to.kind : quotient(begin, run);
            p.items[((int64_t)it.lh * p.max_items + it.index) * 2 + lane] = lane ? (int)wave : first;
        }
        if (it.lh == 0 && it.b >= 0) {   // the rows whose first head lies in this tile
            const int i0 = div_by(it.tile * TR + p.G - 1, p.by_G);
            if (lane < TR && i0 + lane < it.n && (i0 + lane) * p.G < (it.tile + 1) * TR) {
                p.item_of[2 * (it.first + i0 + lane)] = it.index - it.tile;
                p.item_of[2 * (it.first + i0 + lane) + 1] = i0 + lane;
            }
        }
    }
    return to;
}

// Another part of a row, (m2, l2), joined to (m, l): its outputs are to be multiplied by f2 (and left out where that is 0: they may never have been written), the
// row's own by f.  A reference of -infinity has seen no key and has sum 0.
__device__ __forceinline__ void join_part(float &m, float &l, float m2, float l2, float scale_log2, float &f, float &f2)
{
    const float M = fmaxf(m, m2);
    f = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((m - M) * scale_log2);
    f2 = m2 == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((m2 - M) * scale_log2);
    l = (m == -INFINITY ? l : l * f) + (m2 == -INFINITY ? l2 : l2 * f2);
    m = M;
}

// What the reference of a row whose last token is `last` begins with, over a segment from half seg0 of the item on.
__device__ __forceinline__ float first_reference(const PagedItem &it, int seg0, int last)
{
    return seg0 < it.walk || last >= 32 * (seg0 - it.walk) ? kNoScore : -INFINITY;
}

// Row r of an item's tile, in that place.
struct PagedRow {
    bool valid;
    int l, hq, i, row;
    int64_t flat;   // (layer, query head, row)
    int64_t o;      // in the place
};
template <class P>
__device__ __forceinline__ PagedRow paged_row(const P &p, const PagedItem &it, const PagedPlace &to, int tile_rows, int r)
{
    PagedRow x;
    const int packed = it.tile * tile_rows + r;
    x.l = div_by(it.lh, p.by_Hkv);
    const int hkv = it.lh - x.l * p.Hkv;
    x.i = div_by(packed, p.by_G);
    x.hq = hkv * p.G + packed - x.i * p.G;
    x.valid = x.i < it.n;
    x.row = it.first + x.i;
    x.flat = ((int64_t)x.l * p.Hkv * p.G + x.hq) * p.batch.n_rows + x.row;
    x.o = to.kind == 0 ? r : x.flat;
    return x;
}

// A row's results: the lanes g = 0 ... 3 of a row hold reference, sum and, in pieces of four channels from channel(i) on, its outputs.
template <typename T, int D, class P, class C>
__device__ __forceinline__ void paged_finish_row(const P &p, const PagedPlace &to, const PagedRow &row, int g, float m, float l, f32x4 (&o)[D / 16], C channel)
{
    if (to.kind != kDirect) {
#pragma unroll
        for (int i = 0; i < D / 16; ++i) *reinterpret_cast<f32x4 *>(to.o + row.o * D + channel(i)) = o[i];
        if (g < 2) to.ml[row.o * 2 + g] = g ? l : m;
        return;
    }
    for (int run = 0; run < p.prefix_runs; ++run) {
        const int64_t at = row.flat + (int64_t)(p.prefix_part + run) * p.L * p.Hkv * p.G * p.batch.n_rows;
        float f, f2;
        join_part(m, l, p.row_ml[2 * at], p.row_ml[2 * at + 1], p.scale_log2, f, f2);
#pragma unroll
        for (int i = 0; i < D / 16; ++i) {
            o[i] *= f;
            if (f2 != 0.f) o[i] += f2 * *reinterpret_cast<const f32x4 *>(p.row_o + at * D + channel(i));
        }
    }
    const bool none = m == -INFINITY && l == 0.f;
    const float inv = none ? 0.f : 1.f / l;
    T *out = static_cast<T *>(p.out) + row.l * p.s_o.layer + (int64_t)row.hq * p.s_o.head + (int64_t)row.row * p.s_o.token;
#pragma unroll
    for (int i = 0; i < D / 16; ++i) {
        if constexpr (sizeof(T) == 2)
            *reinterpret_cast<u32x2 *>(out + channel(i)) = u32x2{pack_bf16x2(o[i][0] * inv, o[i][1] * inv), pack_bf16x2(o[i][2] * inv, o[i][3] * inv)};
        else
            *reinterpret_cast<f32x4 *>(out + channel(i)) = o[i] * inv;
    }
    if (p.lse && g == 0) p.lse[row.flat] = none ? -INFINITY : m * p.scale + logf(l);
}

// The segment by the formula.
template <typename T, int D, int TR, class P>
__device__ __forceinline__ void paged_exact_segment(const P &p0, const PagedItem &it, const PagedPlace &to, int seg0, int h, int lane)
{
#pragma unroll 1
    for (int r = 0; r < TR; ++r) {
        const P &p = again(p0);
        const PagedRow row = paged_row(p, it, to, TR, r);
        if (!row.valid) return;
        float m, sum, o[8];
        paged_exact_row<T, D>(p, row.l, it.lh - row.l * p.Hkv, row.hq, row.row, it.b, it.b < 0 ? -1 : last_seen(it.len, it.n, row.i, p.batch.cap), it.walk, seg0, h + 1, lane, m, sum, o);
        if (to.kind == kDirect) {
            for (int run = 0; run < p.prefix_runs; ++run) {
                const int64_t at = row.flat + (int64_t)(p.prefix_part + run) * p.L * p.Hkv * p.G * p.batch.n_rows;
                float f, f2;
                join_part(m, sum, p.row_ml[2 * at], p.row_ml[2 * at + 1], p.scale_log2, f, f2);
#pragma unroll
                for (int j = 0; j < 8; ++j) o[j] = o[j] * f + (f2 != 0.f && lane < D / 8 ? f2 * p.row_o[at * D + 8 * lane + j] : 0.f);
            }
            paged_store_row<T, D>(p, row.l, row.hq, row.row, lane, m, sum, o);
        } else {
            if (lane < D / 8) {
                f32x4 *po = reinterpret_cast<f32x4 *>(to.o + row.o * D + 8 * lane);
                po[0] = f32x4{o[0], o[1], o[2], o[3]};
                po[1] = f32x4{o[4], o[5], o[6], o[7]};
            }
            if (lane < 2) to.ml[row.o * 2 + lane] = lane ? sum : m;
        }
    }
}

// ------------------------------------------------------------------------------------------ tiles of many rows
// attn_mfma_kernel (suffix_attn.hip) with Keys::kPaged: a block is a tile of rows and a run of 64-key tiles of one sequence's pages, or of the prefix.
// What bounds it: the matrix cores with their vector work, as over a whole cache.  4 layers, 6 sequences of 100 to 2000 rows behind up to 6000 tokens (1258 GFLOP)
// 1.19 ms = 1.05 PFLOP/s, matrix pipes busy in 51 % of the cycles; 32 layers, a prefix of 8192 for 64 rows of each (layer, head) 0.25 ms (54 %).
// Blocks of 128 rows at D = 128 and those at D = 256 have more values than vector registers: 28 and 48 bytes of scratch memory a lane, of which D = 256 reads some again inside
// the loop over the tiles.
// Where a call has both, a sequence's block joins the prefix's parts to its rows at its end: 8 layers, 16 suffixes behind a prefix of 4096, 0.45 ms; with all of
// them joined by the combine kernel 0.51 (110 us of it there).
struct PagedTileParams : PagedAttnParams {   // row_o null: rows go to `out`.  Over the prefix: k, v and their strides are the prefix's, one page
    int32_t over_prefix;
    int32_t n_items;
    int32_t n_splits;      // runs
    int32_t more_rows;     // packed rows that the sequences of the launch have more than
    int32_t part;          // by rows: of run 0
    int32_t join_runs, join_part;   // rows that go to `out` are joined with these parts
    float *join_o, *join_ml;
    int32_t slot_mask;     // slot of a token in its page
    divisor_t by_LH, by_splits;
    // what the kernel's other forms have
    static constexpr int32_t window = 0, n_sinks = 0;
    static constexpr Strides s_ks = {0, 0, 0}, s_vs = {0, 0, 0};
};

struct PagedTile {
    int tile, b, first, n, len, tokens;   // tokens: that exist
    int cap;
    bool prefix;
    __device__ __forceinline__ int last(int i) const { return prefix ? tokens - 1 : last_seen(len, n, i, cap); }
    // Entry of token t < tokens, as a vector load.
    template <class P>
    __device__ __forceinline__ int entry(const P &p, int t) const
    {
        if (prefix) return 0;
        int i = t >> p.batch.log_page;
        asm volatile("" : "+v"(i));
        return p.batch.table[(int64_t)b * p.batch.table_stride + i];
    }
    // Does one of the tokens t0 ... t1 - 1 that this thread looks at have an entry that is no page?
    template <class P>
    __device__ __forceinline__ bool odd_entries(const P &p, int t0, int t1, int tid, int threads) const
    {
        bool odd = false;
        if (!prefix && t0 < t1)
            for (int i = (t0 >> p.batch.log_page) + tid; i <= (t1 - 1) >> p.batch.log_page; i += threads)
                odd |= (uint32_t)p.batch.table[(int64_t)b * p.batch.table_stride + i] >= (uint32_t)p.batch.n_pages;
        return odd;
    }
};

// The u-th tile of BM packed rows of a launch, the last rows of a sequence first; false: there is none.
template <int BM, class P>
__device__ __forceinline__ bool find_paged_tile(const P &p, int u, int lane, PagedTile &x)
{
    x.prefix = p.over_prefix != 0;
    x.cap = p.batch.cap;
    if (x.prefix) {
        all_rows(p, x.first, x.n);
        x.first = __builtin_amdgcn_readfirstlane(x.first);
        x.n = __builtin_amdgcn_readfirstlane(x.n);
        x.tile = u;
        x.b = -1;
        x.len = 0;
        x.tokens = p.n_prefix;
        return u * BM < x.n * p.G;
    }
    for (int c = 0; c < p.batch.n_seqs; c += 64) {
        int first = 0, n = 0, len = 0;
        if (c + lane < p.batch.n_seqs) {
            sequence_rows(p.batch, c + lane, first, n);
            len = sequence_len(p.batch, c + lane);
        }
        const int tiles = n * p.G > p.more_rows ? (n * p.G + BM - 1) / BM : 0;
        int upto = tiles;
#pragma unroll
        for (int off = 1; off < 64; off <<= 1) {
            const int y = __shfl_up(upto, off);
            if (lane >= off) upto += y;
        }
        const int sum = __builtin_amdgcn_readlane(upto, 63);
        if (u < sum) {
            const int j = __builtin_ctzll(__builtin_amdgcn_ballot_w64(upto > u));
            x.tile = __builtin_amdgcn_readlane(upto, j) - 1 - u;
            x.b = c + j;
            x.first = __builtin_amdgcn_readlane(first, j);
            x.n = __builtin_amdgcn_readlane(n, j);
            x.len = __builtin_amdgcn_readlane(len, j);
            x.tokens = min(x.len, x.cap);
            return true;
        }
        u -= sum;
    }
    return false;
}

// Of a row's part: (part, layer, query head, row).
template <class P>
__device__ __forceinline__ int64_t paged_part_row(const P &p, int l, int hkv, int g, int row, int part)
{
    const int64_t Hq = (int64_t)p.Hkv * p.G;
    return ((int64_t)part * p.L * Hq + l * Hq + hkv * p.G + g) * p.batch.n_rows + row;
}

// For the combine kernel: the rows whose first head lies in the tile are this kernel's.
template <int BM, class P>
__device__ __forceinline__ void paged_note_rows(const P &p, const PagedTile &x, int tid)
{
    if (!p.item_of || x.prefix || tid >= BM) return;
    const int i = div_by(x.tile * BM + p.G - 1, p.by_G) + tid;
    if (i < x.n && i * p.G < (x.tile + 1) * BM) p.item_of[2 * (x.first + i)] = p.row_o ? kWhole : kDirect;
}

// A tile whose rows see nothing in this run.
template <int D, class P>
__device__ __forceinline__ void paged_empty_tile(const P &p, const PagedTile &x, int l, int hkv, int split, int bm, int tid, int threads)
{
    for (int r = tid; r < bm; r += threads) {
        const int packed = x.tile * bm + r, i = div_by(packed, p.by_G), g = packed - i * p.G;
        if (i >= x.n) return;
        if (p.row_o) {
            const int64_t at = paged_part_row(p, l, hkv, g, x.first + i, p.part + split);
            p.row_ml[2 * at] = -INFINITY;
            p.row_ml[2 * at + 1] = 0.f;
        } else {
            const int hq = hkv * p.G + g;
            bf16_t *out = static_cast<bf16_t *>(p.out) + l * p.s_o.layer + (int64_t)hq * p.s_o.head + (int64_t)(x.first + i) * p.s_o.token;
            float m = -INFINITY, sum = 0.f, f, f2;
            for (int run = 0; run < p.join_runs; ++run) {
                const int64_t at = paged_part_row(p, l, hkv, g, x.first + i, p.join_part + run);
                join_part(m, sum, p.join_ml[2 * at], p.join_ml[2 * at + 1], p.scale_log2, f, f2);
            }
            for (int c = 0; c < D; c += 8) {
                float o[8] = {};
                for (int run = 0; run < p.join_runs; ++run) {
                    const int64_t at = paged_part_row(p, l, hkv, g, x.first + i, p.join_part + run);
                    const float mr = p.join_ml[2 * at];
                    if (mr != -INFINITY)
                        for (int j = 0; j < 8; ++j) o[j] += __builtin_amdgcn_exp2f((mr - m) * p.scale_log2) * p.join_o[at * D + c + j];
                }
                for (int j = 0; j < 8; ++j) o[j] = m == -INFINITY && sum == 0.f ? 0.f : o[j] / sum;
                *reinterpret_cast<u32x4 *>(out + c) = pack<bf16_t>(o);
            }
            if (p.lse) p.lse[((int64_t)l * p.Hkv * p.G + hq) * p.batch.n_rows + x.first + i] = m == -INFINITY && sum == 0.f ? -INFINITY : m * p.scale + logf(sum);
        }
    }
}

// The whole block's work by the formula, over the halves h0 ... h1 - 1; all that it needs formed again (see exact_tile()).
template <int D, int BM>
__device__ __forceinline__ void paged_exact_tile(int h0, int h1, int split, int tid, int n_waves)
{
    typedef const __attribute__((address_space(4))) PagedTileParams ParamT;
    ParamT *ptr = (ParamT *)__builtin_amdgcn_kernarg_segment_ptr();
    int block = blockIdx.x;
    asm volatile("" : "+s"(ptr));
    asm volatile("" : "+s"(block));
    ParamT &p = *ptr;
    const int lane = tid & 63, unit = div_by(block, p.by_LH), lh = block - unit * (p.L * p.Hkv), l = div_by(lh, p.by_Hkv), hkv = lh - l * p.Hkv;
    PagedTile x;
    if (!find_paged_tile<BM>(p, div_by(unit, p.by_splits), lane, x)) return;
#pragma unroll 1
    for (int r = __builtin_amdgcn_readfirstlane(tid >> 6); r < BM; r += n_waves) {
        const int packed = x.tile * BM + r, i = div_by(packed, p.by_G), g = packed - i * p.G;
        if (i >= x.n) return;
        float m, sum, o[8];
        paged_exact_row<bf16_t, D>(p, l, hkv, hkv * p.G + g, x.first + i, x.b, x.prefix ? -1 : x.last(i), x.prefix ? (p.n_prefix + 31) / 32 : 0, h0, h1, lane, m, sum, o);
        if (!p.row_o) {
            for (int run = 0; run < p.join_runs; ++run) {
                const int64_t at = paged_part_row(p, l, hkv, g, x.first + i, p.join_part + run);
                float f, f2;
                join_part(m, sum, p.join_ml[2 * at], p.join_ml[2 * at + 1], p.scale_log2, f, f2);
#pragma unroll
                for (int j = 0; j < 8; ++j) o[j] = o[j] * f + (f2 != 0.f && lane < D / 8 ? f2 * p.join_o[at * D + 8 * lane + j] : 0.f);
            }
            paged_store_row<bf16_t, D>(p, l, hkv * p.G + g, x.first + i, lane, m, sum, o);
            continue;
        }
        const int64_t at = paged_part_row(p, l, hkv, g, x.first + i, p.part + split);
        if (lane < D / 8) {
            f32x4 *po = reinterpret_cast<f32x4 *>(p.row_o + at * D + 8 * lane);
            po[0] = f32x4{o[0], o[1], o[2], o[3]};
            po[1] = f32x4{o[4], o[5], o[6], o[7]};
        }
        if (lane < 2) p.row_ml[at * 2 + lane] = lane ? sum : m;
    }
}

int launch_paged_tiles(const PagedTileParams &p, int tile_rows, unsigned n_blocks, hipStream_t s);

}  // namespace kvc
