// kvcomm_suffix_attn_kv4: suffix attention over a cache held in 4 bits per value (fp4.h).  Many query rows: attn_mfma_kernel, which decodes
// every tile into LDS once per block of 256 (128) rows.  Few query rows: attn_kv4_rows_kernel.  f32 models: attn_f32_kernel.
#include "attn_exact.h"
#include "attn_host.h"

namespace {

using namespace kvc;

// 16 packed (query, head) rows per block, shared by the wavefronts: each takes every NW-th 32-key sub-step of the block's key run with its own softmax
// state, joined through LDS at the end (the split, the products and the join of attn_rows_kernel16).
//   * Codes go from global memory to registers, two sub-steps ahead.  A contraction may take the channels in any order as long as both operands agree: lane
//     (n, g) of K Q^T owns D / 4 neighbouring channels of key n, one 16-byte load at D = 128 and one scale, and feeds them to the MFMAs straight out
//     of the conversion (v_cvt_scalef32_pk_bf16_fp4: two values and their scale in one full-rate instruction).
//   * V is contracted over the keys, so it has to be transposed: decoded rows go through the wavefront's own LDS buffer and leave it with
//     ds_read_b64_tr_b16.  No block barrier in the loop.
// What bounds it: HBM where every layer is in one launch, the latency of a wavefront's chain in small launches.
template <int D>
struct Kv4Rows {
    static constexpr int NW = 8;                         // wavefronts
    static constexpr int NF = D / 16, ROWB = D * 2;
    static constexpr int KW = D / 32;                    // words of codes of a lane and key; MFMA steps of a key
    static constexpr int KS = D == 256 ? 2 : 1;          // their scales
    static constexpr int VPR = D / 32, VR = 64 / VPR;    // V: lanes of a row (16 bytes, one scale each), rows of a load
    static constexpr int VL = 32 / VR;                   // loads of a sub-step
};

template <bool NT, typename T>
__device__ __forceinline__ T fetch(const uint8_t *p)   // NT: non-temporal (data that nobody reads again)
{
    return NT ? __builtin_nontemporal_load(reinterpret_cast<const T *>(p)) : *reinterpret_cast<const T *>(p);
}

template <int D, bool NT>
__global__ __launch_bounds__(512, D == 256 ? 2 : 4) void attn_kv4_rows_kernel(const AttnParams p)
{
    using C = Kv4Rows<D>;
    constexpr int NW = C::NW, NF = C::NF, ROWB = C::ROWB, KW = C::KW, KS = C::KS, VPR = C::VPR, VR = C::VR, VL = C::VL, ROWS = 16;
    constexpr int BUF = 32 * ROWB;           // bytes of a wavefront's decoded V
    constexpr int JW = D * ROWS / 4;         // 16-byte slots of its outputs
    static_assert(JW * 16 <= BUF, "a wavefront's outputs fit its own buffer");
    auto v_swz = [](int key) __attribute__((always_inline)) -> int {   // as in attn_mfma_kernel
        return D == 64 ? (2 * (key & 2)) | ((key >> 1) & 2) : 4 * (key & 3) | ((key >> 1) & 2);
    };
    __shared__ __align__(16) unsigned char smem[NW * BUF];
    __shared__ float ml[2][NW][ROWS];

    await_attn_args(p);
    await_args(arg_word(&p.k_scales), arg_word(&p.s_vs));
    const int tid = threadIdx.x;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int lane = tid & 63, n = lane & 15, g = lane >> 4;
    lds_byte *vbuf = (lds_byte *)smem + wave * BUF;

    const int x_id = blockIdx.x & 7;   // XCD x takes one contiguous range of the items
    const int logical = x_id * (p.n_items >> 3) + min(x_id, p.n_items & 7) + (blockIdx.x >> 3);
    const int run = div_by(logical, p.by_row_tiles);
    const int rt = logical - run * p.n_row_tiles;   // the row tiles of a key run are neighbours: they share its L2 lines
    const int lh = div_by(run, p.by_splits), split = run - lh * p.n_splits;
    const int l = div_by(lh, p.by_Hkv), hkv = lh - l * p.Hkv;
    const int r_row = rt * ROWS + n, i_row = div_by(r_row, p.by_G);
    const bool valid = i_row < p.tq;
    const int qi = min(i_row, p.tq - 1), hq = hkv * p.G + r_row - i_row * p.G;
    const int imax = min(p.tq - 1, div_by(rt * ROWS + ROWS - 1, p.by_G)), imin = min(p.tq - 1, div_by(rt * ROWS, p.by_G));
    const int units = (p.n_ctx + imax + 32) / 32;   // sub-steps that some query of the tile sees
    const int u0 = div_by(split * units, p.by_splits), u1 = div_by((split + 1) * units, p.by_splits);

    const uint8_t *kc = static_cast<const uint8_t *>(p.k) + l * p.s_k.layer + hkv * p.s_k.head, *vc = static_cast<const uint8_t *>(p.v) + l * p.s_v.layer + hkv * p.s_v.head;
    const uint8_t *ksc = p.k_scales + l * p.s_ks.layer + hkv * p.s_ks.head, *vsc = p.v_scales + l * p.s_vs.layer + hkv * p.s_vs.head;
    // V: lane -> row of a load.  Every second group of VPR lanes takes a row four further on: rows whose chunks the swizzle moves apart, so that the
    // stores of decoded values meet in no bank.
    const int vi = lane / VPR;
    const int v_row0 = VR >= 16 ? ((vi & 1) << 2) | ((vi >> 1) & 3) | (vi & ~7) : vi, v_part = lane % VPR;

    struct Raw {   // codes and scales of a sub-step
        uint32_t k[2][KW], v[VL][4], ks[2][KS], vs[VL];
    };
    const uint32_t k_tok = (uint32_t)p.s_k.token, v_tok = (uint32_t)p.s_v.token, ks_tok = (uint32_t)p.s_ks.token, vs_tok = (uint32_t)p.s_vs.token;
    auto load = [&](Raw &r, int u) __attribute__((always_inline)) {
        const int key0 = 32 * u, last = p.N - 1 - key0;   // rows past the cache end re-read the last one; they are always masked
        const uint8_t *kb = kc + (int64_t)key0 * k_tok, *vb = vc + (int64_t)key0 * v_tok, *ksb = ksc + (int64_t)key0 * ks_tok, *vsb = vsc + (int64_t)key0 * vs_tok;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const uint32_t row = (uint32_t)min(16 * h + n, last);
            const uint8_t *src = kb + (row * k_tok + (uint32_t)(g * (D / 8))), *sc = ksb + (row * ks_tok + (uint32_t)(g * (D / 4) / 32));
            if constexpr (KW == 2) {
                const u32x2 w = fetch<NT, u32x2>(src);
                r.k[h][0] = w[0], r.k[h][1] = w[1];
            } else {
#pragma unroll
                for (int i = 0; i < KW; i += 4) {
                    const u32x4 w = fetch<NT, u32x4>(src + 4 * i);
#pragma unroll
                    for (int j = 0; j < 4; ++j) r.k[h][i + j] = w[j];
                }
            }
#pragma unroll
            for (int i = 0; i < KS; ++i) r.ks[h][i] = sc[i];
        }
#pragma unroll
        for (int i = 0; i < VL; ++i) {
            const uint32_t row = (uint32_t)min(VR * i + v_row0, last);
            const u32x4 w = fetch<NT, u32x4>(vb + (row * v_tok + (uint32_t)(16 * v_part)));
#pragma unroll
            for (int j = 0; j < 4; ++j) r.v[i][j] = w[j];
            r.vs[i] = vsb[row * vs_tok + (uint32_t)v_part];
        }
    };

    bf16x8 qf[KW];
    const bf16_t *qrow = static_cast<const bf16_t *>(p.q) + l * p.s_q.layer + (int64_t)hq * p.s_q.head + (int64_t)qi * p.s_q.token;
#pragma unroll
    for (int ks = 0; ks < KW; ++ks) qf[ks] = as_bf16x8(load16(qrow + g * (D / 4) + ks * 8));
    Raw ra = {}, rb = {};
    int u = u0 + wave;
    if (u < u1) load(ra, u);
    if (u + NW < u1) load(rb, u + NW);

    int v_off[NF];   // V^T operands: transposing reads, as in attn_mfma_kernel
    {
        const int row = 4 * g + (n >> 2);
#pragma unroll
        for (int db = 0; db < NF; ++db) {
            const int col = 16 * db + 4 * (n & 3);
            v_off[db] = row * ROWB + ((col >> 3) ^ v_swz(row)) * 16 + (col & 7) * 2;
        }
    }
    f32x4 o[NF];
#pragma unroll
    for (int db = 0; db < NF; ++db) o[db] = f32x4{0.f, 0.f, 0.f, 0.f};
    float m = -INFINITY, mc = 0.f, lsum = 0.f;   // lsum: this lane's quarter of the row sum

    auto sub_step = [&](Raw &r, int u, int next) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < VL; ++i) {
            const int row = VR * i + v_row0;
            const float scale = fp4_scale(r.vs[i]);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                u32x4 x[1];
                fp4_decode8(r.v[i][j], scale, x);
                *(__attribute__((address_space(3))) u32x4 *)(vbuf + row * ROWB + ((4 * v_part + j) ^ v_swz(row)) * 16) = x[0];
            }
        }
        f32x4 s[2];
#pragma unroll
        for (int ks = 0; ks < KW; ++ks)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                u32x4 x[1];
                fp4_decode8(r.k[h][ks], fp4_scale(r.ks[h][ks / 4]), x);
                s[h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(x[0]), qf[ks], ks == 0 ? f32x4{0.f, 0.f, 0.f, 0.f} : s[h], 0, 0, 0);
            }
        if (next < u1) load(r, next);
        if (32 * u + 31 > p.n_ctx + imin) {   // some key is hidden from some query
            const int limit = p.n_ctx + qi - 32 * u - 4 * g;
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (16 * (j >> 2) + (j & 3) > limit) s[j >> 2][j & 3] = -INFINITY;
        }
        float mx = s[0][0];
#pragma unroll
        for (int j = 1; j < 8; ++j) mx = fmaxf(mx, s[j >> 2][j & 3]);
        mx = query_max(mx);
        if (__builtin_amdgcn_ballot_w64(mx > m) != 0) {
            const float m_new = fmaxf(m, mx);
            const float corr = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((m - m_new) * p.scale_log2);
            lsum *= corr;
#pragma unroll
            for (int db = 0; db < NF; ++db) o[db] *= corr;
            m = m_new;
            mc = m == -INFINITY ? 0.f : m * p.scale_log2;   // a row that sees no key of this run yet: exponentials 0
        }
        // Probabilities as bf16, which the second product takes: each is off by up to 2^-8 of itself, half a step, and a sum of many by far less, which the
        // result's own rounding to bf16 exceeds.  Sums stay fp32 and are of the unrounded ones.
        u32x4 pk;
        float rs0 = 0.f, rs1 = 0.f;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float e0 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[j >> 1][2 * (j & 1)], p.scale_log2, -mc));
            const float e1 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[j >> 1][2 * (j & 1) + 1], p.scale_log2, -mc));
            rs0 += e0;
            rs1 += e1;
            pk[j] = pack_bf16x2(e0, e1);
        }
        lsum += rs0 + rs1;
        // the reads below touch what other lanes of this wavefront wrote: LDS operations of a wavefront complete in order
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
#pragma unroll
        for (int db = 0; db < NF; ++db)
            o[db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(lds_read_tr_pair(vbuf + v_off[db], vbuf + v_off[db] + 16 * ROWB), as_bf16x8(pk), o[db], 0, 0, 0);
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");   // ... and the next sub-step's stores overwrite what has been read
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    };
    while (u < u1) {
        sub_step(ra, u, u + 2 * NW);
        u += NW;
        if (u >= u1) break;
        sub_step(rb, u, u + 2 * NW);
        u += NW;
    }

    // ---- join the wavefronts' states: outputs as they are go over the wavefront's own buffer, lane (n, g) holds channels 16 * db + 4 * g ... + 3 of row n:
    // slot (4 * db + g, n).
    lsum = query_sum(lsum);
    float zero = lsum * 0.f;
#pragma unroll
    for (int i = 0; i < 4 * NF; ++i) zero = fmaf(o[i / 4][i % 4], 0.f, zero);
    if (g == 0) {
        ml[0][wave][n] = m;
        ml[1][wave][n] = lsum;
    }
    f32x4 *join = reinterpret_cast<f32x4 *>(smem);
#pragma unroll
    for (int db = 0; db < NF; ++db) join[wave * JW + 64 * db + lane] = o[db];
    if (__syncthreads_or(state_is_odd(zero, m, lsum))) {   // a hidden key's NaN may have been multiplied by its probability 0
        const KeyRanges keys = {0, 0, 32 * u0, min(32 * u1, p.N)};
        attn_exact_rows<fp4_t, bf16_t, D>(p, lh, rt * ROWS, ROWS, keys, split, ROWS, wave, NW, lane);
        return;
    }
    float M = ml[0][0][n];
#pragma unroll
    for (int w = 1; w < NW; ++w) M = fmaxf(M, ml[0][w][n]);
    float f[NW], ltot = 0.f;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
        f[w] = ml[0][w][n] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((ml[0][w][n] - M) * p.scale_log2);
        ltot = fmaf(ml[1][w][n], f[w], ltot);
    }
    if (!valid) return;
    const int64_t part = (int64_t)(lh * p.n_row_tiles + rt) * p.n_splits + split;
    const float inv = 1.f / ltot;
#pragma unroll
    for (int i = 0; i < JW; i += 64 * NW) {
        const int slot = i + 64 * wave + lane;
        if (JW % (64 * NW) && slot >= JW) break;
        f32x4 a = join[slot] * f[0];
#pragma unroll
        for (int w = 1; w < NW; ++w) a += join[w * JW + slot] * f[w];
        if (p.n_splits > 1) {
            reinterpret_cast<f32x4 *>(p.part_o + part * (ROWS * D))[slot] = a;
        } else {
            bf16_t *orow = static_cast<bf16_t *>(p.out) + l * p.s_o.layer + (int64_t)hq * p.s_o.head + (int64_t)qi * p.s_o.token;
            *reinterpret_cast<u32x2 *>(orow + slot / ROWS * 4) = u32x2{pack_bf16x2(a[0] * inv, a[1] * inv), pack_bf16x2(a[2] * inv, a[3] * inv)};
        }
    }
    if (wave == 0 && g == 0) {
        if (p.n_splits > 1) {
            p.part_ml[part * 2 * ROWS + n] = M;
            p.part_ml[part * 2 * ROWS + ROWS + n] = ltot;
        } else if (p.lse) {
            p.lse[((int64_t)l * p.Hkv * p.G + hq) * p.tq + qi] = M * p.scale + logf(ltot);
        }
    }
}

// Microseconds of a launch of the rows kernel with the keys of `items` (16-row tile, layer, kv head) triples cut into ns runs, `its` iterations (32 keys of every
// wavefront) of a whole cache: 4 us, and per iteration 1.2 us when few units are busy, 1.5 with a block on each, 2.5 with two and 2.5 us more for their start, 1.5 us for the start of every two that follow (D = 256: one block
// per unit, in rounds); 3.5 us for the combine launch and the partial results at about 8 TB/s.
double kv4_rows_us(const kvcomm_model &m, int64_t items, int64_t its, int64_t ns)
{
    const double x = (double)(items * ns) / kChipCUs, run = (double)((its + ns - 1) / ns);
    const double one = 1.2 + 0.3 * std::min(1.0, x), two = x <= 1 ? one : x <= 2 ? 0.5 + x : 1.25 * x;
    const double us = m.head_dim == 256 ? attn_rounds(x) * (4.0 + 1.9 * one * run)
                                        : 4.0 + 2.5 * std::min(1.0, std::max(0.0, x - 1)) + 0.75 * std::max(0.0, x - 2) + (m.head_dim == 64 ? 0.65 : 1.0) * two * run;
    return us + (ns > 1 ? 3.5 + (double)(items * ns) * 16 * m.head_dim * 8 / 8e6 : 0.0);
}

// The same of attn_mfma_kernel, which here decodes its tiles: 9 us and 1.4 ... 1.65 us per 64-key tile (attn_tiles_us() for a bf16 cache).
double kv4_tiles_us(const kvcomm_model &m, int64_t items, int tile_rows, int64_t tiles, int64_t ns)
{
    const double x = (double)(items * ns) / kChipCUs, scale = m.head_dim == 64 ? 0.68 : m.head_dim == 128 ? 1.0 : 1.7;
    return attn_rounds(x) * (9.0 + scale * (1.4 + 0.25 * std::min(1.0, x)) * (double)((tiles + ns - 1) / ns)) +
           (ns > 1 ? 3.5 + (double)(items * ns) * tile_rows * m.head_dim * 8 / 8e6 : 0.0);
}

// The same in blocks of 128 rows: 10 us and 1.13 us per tile with a block per unit at most (its wavefronts have a SIMD each); with two on a unit every tile is decoded twice
// there, and at D = 128 the registers do not suffice.  us in 256 rows / 128, best cuts: one layer, 4000 keys, D 128, Tq 128 26.0 / 22.2, Tq 512 44.8 / 50.6, 32 layers, G = 1, Tq 128
// 115 / 80; D 64: 19.3 / 15.2, 31.4 / 31.5, 77 / 51; 8 layers, 8704 keys, Tq 512, D 128 451 / 502, D 64 294 / 301.
double kv4_tiles128_us(const kvcomm_model &m, int64_t items, int64_t tiles, int64_t ns)
{
    const double x = (double)(items * ns) / kChipCUs, t = (double)((tiles + ns - 1) / ns);
    const double us = x <= 1 ? 10.0 + (m.head_dim == 64 ? 0.65 : 1.13) * t : attn_rounds(0.5 * x) * (10.0 + (m.head_dim == 64 ? 1.03 : 1.8) * t);
    return us + (ns > 1 ? 3.5 + (double)(items * ns) * 128 * m.head_dim * 8 / 8e6 : 0.0);
}

// Which kernel, in how many runs of keys: the least by these times.  Measured, 8 kv heads, G = 4, D = 128, us: rows kernel in 1 / 2 / 4 / 8 / 16 runs and
// attn_mfma_kernel in 1 / 2 / 4 / 8
//   one layer, 4000 keys, Tq 8    24.3 / 17.4 / 12.7 / 10.6 / 9.9     97 / 55 / 32.5 / 21.4
//                         Tq 32   25.1 / 18.5 / 14.2 / 16.0 / 20.0    96 / 55 / 32.5 / 21.5
//                         Tq 64   25.9 / 19.7 / 20.9 / 24.3 / 31.8    98 / 57 / 33.9 / 23.3
//                         Tq 128  27.9 / 30.1 / 33.2 / 39.9           99 / 58 / 36.4 / 26.7
//                         Tq 256  44.3 / 51.1                         102 / 61 / 38.5 / 31.4
//   8 layers, 8192 keys,  Tq 16   46.6 / 44.4 / 48.2 / 55.1           190 / 110 / 67 / 74
//                         Tq 64   128 / 142                           190 / 111 / 71.5 / 82
//   32 layers, 32768 keys, Tq 1   225 / 209 / 227 / 245
AttnPlan plan_kv4(const kvcomm_model &m, int n_ctx, int tq, bool may_split)
{
    const int64_t rows = (int64_t)(m.n_q_heads / m.n_kv_heads) * tq, LH = (int64_t)m.n_layers * m.n_kv_heads, N = (int64_t)n_ctx + tq;
    const int tile_rows = m.head_dim == 256 ? 128 : 32 * kAttnWaves;
    const int64_t items = LH * ((rows + 15) / 16), its = (N + 32 * 8 - 1) / (32 * 8);
    const int64_t tile_items = LH * ((rows + tile_rows - 1) / tile_rows), tiles = (N + 63) / 64;
    AttnPlan pl = {true, 16, (int)((rows + 15) / 16), 1, 16};
    double best = kv4_rows_us(m, items, its, 1);
    for (int ns = 2; may_split && ns <= kRowsMaxSplits && ns <= its && items * ns <= 2 * kChipCUs; ++ns) {
        const double t = kv4_rows_us(m, items, its, ns);
        if (t < best) best = t, pl.n_splits = ns;
    }
    auto may_cut = [&](int64_t blocks, int ns) { return ns == 1 || (may_split && ns <= kTileMaxSplits && ns * kMinRunTiles <= tiles && blocks * ns <= 2 * kChipCUs); };
    for (int ns = 1; may_cut(tile_items, ns); ++ns) {
        const double t = kv4_tiles_us(m, tile_items, tile_rows, tiles, ns);
        if (t < best) best = t, pl = {false, tile_rows, (int)((rows + tile_rows - 1) / tile_rows), ns, 32};
    }
    const int64_t items128 = LH * ((rows + 127) / 128);
    for (int ns = 1; m.head_dim != 256 && may_cut(items128, ns); ++ns) {
        const double t = kv4_tiles128_us(m, items128, tiles, ns);
        if (t < best) best = t, pl = {false, 128, (int)((rows + 127) / 128), ns, 32};
    }
    return pl;
}

}  // namespace

namespace kvc {

template <int D>
static int launch_rows(const AttnParams &p, unsigned n_blocks, hipStream_t stream)
{
    const bool nt = p.n_row_tiles == 1 && (int64_t)p.L * p.Hkv * p.N * D > kLastLevelCache;   // (as launch_attn_rows(); 32 layers, 32768 keys 187 us with it, 209 without)
    return launch(nt ? attn_kv4_rows_kernel<D, true> : attn_kv4_rows_kernel<D, false>, dim3(n_blocks), dim3(512), 0, stream, p);
}

int launch_attn_kv4_rows(const AttnParams &p, int D, unsigned n_blocks, hipStream_t stream)
{
    switch (D) {
        case 64: return launch_rows<64>(p, n_blocks, stream);
        case 128: return launch_rows<128>(p, n_blocks, stream);
        default: return launch_rows<256>(p, n_blocks, stream);
    }
}

}  // namespace kvc

extern "C" size_t kvcomm_suffix_attn_kv4_workspace(const kvcomm_model *model, int32_t n_ctx, int32_t tq)
{
    if (check_model(model) || tq <= 0 || n_ctx < 0 || model->dtype != KVCOMM_BF16 || !plannable(*model, n_ctx, tq)) return 0;
    return attn_workspace(*model, plan_kv4(*model, n_ctx, tq, true));
}

extern "C" int kvcomm_suffix_attn_kv4(const kvcomm_model *model, kvcomm_tensor q, kvcomm_tensor4 cache_k, kvcomm_tensor4 cache_v, int32_t n_ctx,
                                      int32_t tq, float softmax_scale, kvcomm_tensor out, float *lse_out, void *workspace, size_t workspace_bytes,
                                      void *stream)
{
    AttnParams p{};
    int st = attn_params(model, q, n_ctx, tq, softmax_scale, out, lse_out, p);
    if (st || (st = attn_cache4(*model, cache_k, cache_v, p))) return st;
    if (!plannable(*model, n_ctx, tq)) return KVCOMM_EUNSUPPORTED;
    if (model->dtype == KVCOMM_F32) return launch_f32(p, model->head_dim, attn_f32_groups(*model, tq, 0), 0, static_cast<hipStream_t>(stream));
    // Rows of a 64-key tile are addressed by a 32-bit offset from the first.
    for (const Strides &t : {p.s_k, p.s_v, p.s_ks, p.s_vs})
        if (t.token >= 1 << 26) return KVCOMM_EUNSUPPORTED;
    return launch_attn(*model, p, plan_kv4(*model, n_ctx, tq, true), plan_kv4(*model, n_ctx, tq, false), 0, workspace, workspace_bytes,
                       static_cast<hipStream_t>(stream));
}
