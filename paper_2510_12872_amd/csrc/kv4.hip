// A cache held in 4 bits per value: kvcomm_quantize_kv4 and kvcomm_dequantize_kv4.
// 32 neighbouring channels of a row share a scale 2^e (one byte, e + 127); a value is stored as the OCP 4-bit floating-point code (E2M1:
// 0, 0.5, 1, 1.5, 2, 3, 4, 6 and a sign) of x / 2^e, rounded to nearest, ties to the even code.  e is the least exponent with
// max|x| <= 7 * 2^e: the top step of the format is 2, so 7 is as far from 6 as 5 is from 4 and 6, and no value of the block is off by more than 2^e.
// (With 6 * 2^e as the limit the scale of every block whose maximum lies in (6, 7] * 2^e would be twice as coarse.)
// gfx950's v_cvt_scalef32_pk_fp4_{f32,bf16} and v_cvt_scalef32_pk_{f32,bf16}_fp4 do exactly this division, rounding and multiplication; a
// scale byte of 255 is NaN to them and to the format, and stands here for a block with a NaN or an infinity, which no scale fits.
#include "fp4.h"

namespace {

using namespace kvc;

constexpr int kBlock = 256;

// One thread holds 8 channels of a row, so four lanes share a scale.  HBM bound: 2 * D * es + D bytes (and D / 16 of scales) per token, kv head and layer.
struct Kv4Params {
    const void *x[2];        // values of keys and values (quantise: in, dequantise: out)
    uint8_t *codes[2], *scales[2];
    Strides s_x[2], s_codes[2], s_scales[2];
    int32_t n, n_tiles;      // tokens, blocks of tokens of a (layer, head)
    divisor_t by_tiles, by_H;
    int32_t H;
};

template <typename T>
__device__ __forceinline__ void load8(const T *p, u32x4 (&raw)[8 / Elem<T>::EPV])
{
#pragma unroll
    for (int i = 0; i < 8 / Elem<T>::EPV; ++i) raw[i] = load16_stream(p + i * Elem<T>::EPV);
}

// Bits of the largest magnitude of the 8 channels as an fp32 pattern: integers order like the magnitudes, infinity and NaN above all.
__device__ __forceinline__ uint32_t max_bits(const u32x4 (&raw)[2])
{
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, raw[i >> 2][i & 3] & 0x7fffffffu);
    return m;
}
__device__ __forceinline__ uint32_t max_bits(const u32x4 (&raw)[1])
{
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) m = max(m, max(raw[0][i] << 16 & 0x7fffffffu, raw[0][i] & 0x7fff0000u));
    return m;
}

template <typename T, int D>
__global__ __launch_bounds__(kBlock) void quantize_kv4_kernel(const Kv4Params p)
{
    constexpr int LPR = D / 8, RPB = kBlock / LPR;   // lanes of a row, rows of a block
    const int w = blockIdx.y;
    await_args(arg_word(&p), arg_word(&p.s_x), arg_word(&p.s_codes), arg_word(&p.s_scales));
    await_args(arg_word(&p.s_scales[1]), arg_word(&p.by_H));
    const int lh = div_by(blockIdx.x, p.by_tiles), tile = blockIdx.x - lh * p.n_tiles;
    const int l = div_by(lh, p.by_H), h = lh - l * p.H;
    const int t = tile * RPB + threadIdx.x / LPR, c = threadIdx.x % LPR;
    if (t >= p.n) return;   // (the four lanes of a scale go together)
    u32x4 raw[8 / Elem<T>::EPV];
    load8(static_cast<const T *>(p.x[w]) + l * p.s_x[w].layer + h * p.s_x[w].head + (int64_t)t * p.s_x[w].token + 8 * c, raw);
    uint32_t most = max_bits(raw);
    most = max(most, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)most, 0xB1, 0xf, 0xf, true));   // lanes 1, 0, 3, 2
    most = max(most, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)most, 0x4E, 0xf, 0xf, true));   // lanes 2, 3, 0, 1
    const uint32_t byte = fp4_scale_byte(most);
    uint8_t *codes = p.codes[w] + l * p.s_codes[w].layer + h * p.s_codes[w].head + (int64_t)t * p.s_codes[w].token;
    *reinterpret_cast<uint32_t *>(codes + 4 * c) = fp4_encode8(raw, fp4_scale(byte));
    if (c % 4 == 0) p.scales[w][l * p.s_scales[w].layer + h * p.s_scales[w].head + (int64_t)t * p.s_scales[w].token + c / 4] = (uint8_t)byte;
}

template <typename T, int D>
__global__ __launch_bounds__(kBlock) void dequantize_kv4_kernel(const Kv4Params p)
{
    constexpr int LPR = D / 8, RPB = kBlock / LPR;
    const int w = blockIdx.y;
    await_args(arg_word(&p), arg_word(&p.s_x), arg_word(&p.s_codes), arg_word(&p.s_scales));
    await_args(arg_word(&p.s_scales[1]), arg_word(&p.by_H));
    const int lh = div_by(blockIdx.x, p.by_tiles), tile = blockIdx.x - lh * p.n_tiles;
    const int l = div_by(lh, p.by_H), h = lh - l * p.H;
    const int t = tile * RPB + threadIdx.x / LPR, c = threadIdx.x % LPR;
    if (t >= p.n) return;
    const uint32_t code = *reinterpret_cast<const uint32_t *>(p.codes[w] + l * p.s_codes[w].layer + h * p.s_codes[w].head + (int64_t)t * p.s_codes[w].token + 4 * c);
    const uint32_t byte = p.scales[w][l * p.s_scales[w].layer + h * p.s_scales[w].head + (int64_t)t * p.s_scales[w].token + c / 4];
    T *out = static_cast<T *>(const_cast<void *>(p.x[w])) + l * p.s_x[w].layer + h * p.s_x[w].head + (int64_t)t * p.s_x[w].token + 8 * c;
    u32x4 raw[8 / Elem<T>::EPV];
    fp4_decode8(code, fp4_scale(byte), raw);
#pragma unroll
    for (int i = 0; i < 8 / Elem<T>::EPV; ++i) store16_stream(out + i * Elem<T>::EPV, raw[i]);
}

template <typename T, int D>
int launch_kv4(bool back, Kv4Params &p, int64_t LH, hipStream_t s)
{
    constexpr int RPB = kBlock / (D / 8);
    p.n_tiles = (p.n + RPB - 1) / RPB;
    if (LH * p.n_tiles >= 1 << 24) return KVCOMM_EUNSUPPORTED;   // a launch holds fewer than 2^32 threads along an axis
    p.by_tiles = make_divisor((uint32_t)p.n_tiles);
    return launch(back ? dequantize_kv4_kernel<T, D> : quantize_kv4_kernel<T, D>, dim3((unsigned)(LH * p.n_tiles), 2), dim3(kBlock), 0, s, p);
}

int kv4_call(bool back, const kvcomm_model *model, const kvcomm_tensor (&x)[2], const kvcomm_tensor4 (&x4)[2], int32_t n, void *stream)
{
    int st = check_model(model);
    if (st) return st;
    if (n <= 0) return KVCOMM_EINVAL;
    const int L = model->n_layers, H = model->n_kv_heads, D = model->head_dim;
    struct Part {   // a tensor of the call, bytes of its rows and of what its strides count
        kvcomm_tensor t;
        int64_t row;
        int es;
    } in[6], out[6];
    int n_in = 0, n_out = 0;
    Kv4Params p{};
    for (int w = 0; w < 2; ++w) {
        if ((st = check_tensor(x[w], model->dtype, true)) || (st = check_tensor4(x4[w], D))) return st;
        p.x[w] = x[w].ptr;
        p.codes[w] = static_cast<uint8_t *>(x4[w].codes.ptr);
        p.scales[w] = static_cast<uint8_t *>(x4[w].scales.ptr);
        p.s_x[w] = strides_of(x[w]);
        p.s_codes[w] = strides_of(x4[w].codes);
        p.s_scales[w] = strides_of(x4[w].scales);
        const int es = elem_size(model->dtype);
        (back ? out[n_out++] : in[n_in++]) = Part{x[w], (int64_t)D * es, es};
        (back ? in[n_in++] : out[n_out++]) = Part{x4[w].codes, D / 2, 1};
        (back ? in[n_in++] : out[n_out++]) = Part{x4[w].scales, D / 32, 1};
    }
    auto extent = [&](const Part &a) { return extent_of(a.t, L, H, n, (int)(a.row / a.es), a.es); };
    auto meet = [&](const Part &a, const Part &b) { return extents_overlap(extent(a), extent(b)) && !beside_each_other(a.t, H, a.row, a.es, b.t, H, b.row, b.es, L); };
    for (int i = 0; i < n_out; ++i) {
        for (int j = 0; j < n_in; ++j)
            if (meet(out[i], in[j])) return KVCOMM_EINVAL;
        for (int j = 0; j < i; ++j)
            if (meet(out[i], out[j])) return KVCOMM_EINVAL;
    }
    p.n = n;
    p.H = H;
    p.by_H = make_divisor((uint32_t)H);
    const int64_t LH = (int64_t)L * H;
    hipStream_t s = static_cast<hipStream_t>(stream);
    const bool f32 = model->dtype == KVCOMM_F32;
    switch (D) {
        case 64: return f32 ? launch_kv4<float, 64>(back, p, LH, s) : launch_kv4<bf16_t, 64>(back, p, LH, s);
        case 128: return f32 ? launch_kv4<float, 128>(back, p, LH, s) : launch_kv4<bf16_t, 128>(back, p, LH, s);
        default: return f32 ? launch_kv4<float, 256>(back, p, LH, s) : launch_kv4<bf16_t, 256>(back, p, LH, s);
    }
}

}  // namespace

extern "C" int kvcomm_quantize_kv4(const kvcomm_model *model, kvcomm_tensor k, kvcomm_tensor v, int32_t n_tokens, kvcomm_tensor4 out_k,
                                   kvcomm_tensor4 out_v, void *stream)
{
    return kv4_call(false, model, {k, v}, {out_k, out_v}, n_tokens, stream);
}

extern "C" int kvcomm_dequantize_kv4(const kvcomm_model *model, kvcomm_tensor4 k, kvcomm_tensor4 v, int32_t n_tokens, kvcomm_tensor out_k,
                                     kvcomm_tensor out_v, void *stream)
{
    return kv4_call(true, model, {out_k, out_v}, {k, v}, n_tokens, stream);
}
