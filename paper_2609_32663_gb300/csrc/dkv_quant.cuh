// Rotary positions and the paged cache in 8 bits (dkv_rope.cu, dkv_quant.cu, dkv_quant_attn.cu):
// declarations shared with the host side (dkv_pages_api.cu), and a row's scale and e4m3 values.
#pragma once

#include "dkv_pages.cuh"

namespace dkv {

struct RopeArgs {
    const uint16_t* q;     // [T] rows of q_stride elements, H x 128 used, or null
    uint16_t* q_out;
    const uint16_t* k;     // [T] rows of kv_stride elements, Hkv x 128 used, or null
    const uint16_t* v;
    int64_t q_stride, out_stride, kv_stride;
    const int32_t* positions;  // [T], or null where nothing is turned (rot = 0)
    const int32_t* cu;     // [B + 1], or null: all T rows are tokens
    const int32_t* table;  // the layer's slabs: [B * Hkv][max_pages]
    const int32_t* len;    // [B * Hkv]
    void* Kp;              // 16-bit or 8-bit pools
    void* Vp;
    uint8_t* Ks;           // null: 16-bit pools
    uint8_t* Vs;
    int32_t* status;
    int T, B, H, Hkv, P, num_pages, max_pages;
    int fp16, interleaved, rot;
    float magnitude;
    uint64_t turns[64];
};
cudaError_t rope_setup();  // the kernels' attributes in the current context
cudaError_t launch_rope(const RopeArgs& a, cudaStream_t st);

struct QuantCompactArgs {
    PageCompactArgs c;     // (Kp and Vp are pools of bytes)
    uint8_t* Ks;
    uint8_t* Vs;
    int fp16;
};
cudaError_t launch_quant_compact(const QuantCompactArgs& a, cudaStream_t st);

struct QuantAttnArgs {
    const uint16_t* q;      // [T] rows of q_stride elements, H x 128 used
    int64_t q_stride;
    const int32_t* cu;      // [B + 1]
    const int32_t* table;   // the layer's slabs: [B * Hkv][max_pages]
    const int32_t* len;     // [B * Hkv]
    const uint8_t* Kp;
    const uint8_t* Vp;
    const uint8_t* Ks;
    const uint8_t* Vs;
    uint16_t* out;          // [T][H][128]
    int32_t* status;
    void* work;
    int T, B, H, Hkv, G, P, num_pages, max_pages;
    int most, few;          // tokens of a sequence, at most; of one that quant_attn_kernel deals with
    int causal, fp16;
    float qscale;           // softmax scale * log2(e)
};
int64_t quant_workspace_bytes();
cudaError_t quant_setup();  // the kernels' attributes in the current context
// short_boxes (fault injection): page copies deliver half the bytes that a stage expects, inside the
// stage, so that every wait for them runs out.
cudaError_t launch_quant_attn(const QuantAttnArgs& a, bool short_boxes, cudaStream_t st);

#ifdef __CUDACC__
}  // namespace dkv

#include <cuda_fp16.h>

namespace dkv {
namespace {

// Scale byte u of a row whose largest element is `size`: the least e = u - 127 with size <= 448 2^e.
// 448 = 1.75 2^8, so for size = 1.m 2^x it is x - 8, or one more where 1.m > 1.75.
__device__ __forceinline__ uint32_t scale_byte(float size)
{
    const uint32_t bits = __float_as_uint(size);
    const int u = (int)(bits >> 23) - 8 + ((bits & 0x7fffffu) > 0x600000u ? 1 : 0);
    return (uint32_t)max(u, 1);
}

// 2^(u - 127) and its inverse (u in [1, 253]).
__device__ __forceinline__ float scale_of(uint32_t u) { return __uint_as_float(u << 23); }
__device__ __forceinline__ float inverse_scale(uint32_t u) { return __uint_as_float((254u - u) << 23); }

// Rows of 16-bit values, 8 lanes a row (in groups of 8 neighbours): the lane's 16 elements w as 16 e4m3 values, and the row's
// scale byte. All lanes of the warp.
template <bool F16>
__device__ __forceinline__ uint4 hold_lane(const uint32_t (&w)[8], uint32_t& u);
__device__ __forceinline__ uint4 hold_lane(const float (&x)[16], uint32_t& u);  // the same of 32-bit values

// Four e4m3 values, the first in the lowest byte.
__device__ __forceinline__ uint32_t pack_e4m3(float x0, float x1, float x2, float x3)
{
    uint32_t v;
    asm("{\n\t.reg .b16 lo, hi;\n\t"
        "cvt.rn.satfinite.e4m3x2.f32 lo, %2, %1;\n\t"
        "cvt.rn.satfinite.e4m3x2.f32 hi, %4, %3;\n\t"
        "mov.b32 %0, {lo, hi};\n\t}"
        : "=r"(v)
        : "f"(x0), "f"(x1), "f"(x2), "f"(x3));
    return v;
}

// Two e4m3 values of a pair of fp16 values.
__device__ __forceinline__ uint32_t pack_e4m3_f16(uint32_t x)
{
    uint32_t v;
    asm("{\n\t.reg .b16 y;\n\tcvt.rn.satfinite.e4m3x2.f16x2 y, %1;\n\tmov.b32 %0, {y, 0};\n\t}" : "=r"(v) : "r"(x));
    return v;
}

template <bool F16>
__device__ __forceinline__ uint4 hold_lane(const uint32_t (&w)[8], uint32_t& u)
{
    // The largest element as its 15 bits, which order as the sizes do; infinities and NaN come after all others.
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = __vmaxu2(m, w[i] & 0x7fff7fffu);
#pragma unroll
    for (int o = 1; o < 8; o <<= 1) m = __vmaxu2(m, __shfl_xor_sync(0xffffffffu, m, o));
    m = max(m & 0xffffu, m >> 16);
    const float size = F16 ? __half2float(__ushort_as_half((uint16_t)m)) : __uint_as_float(m << 16);
    u = scale_byte(size);
    // fp16: the factor 2^(127 - u) has to be one, and what it takes below 2^-14 is below a half of the least step, 2^-10.
    const bool plain = m < (F16 ? 0x7c00u : 0x7f80u) && (!F16 || (u >= 112u && u <= 141u));
    uint32_t y[8];
    if (__all_sync(0xffffffffu, plain)) {
        const uint32_t f = F16 ? (142u - u) << 10 : (254u - u) << 7, f2 = f | f << 16;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            uint32_t z;
            if (F16) {
                asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(z) : "r"(w[i]), "r"(f2));
                y[i] = pack_e4m3_f16(z);
            } else {
                asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(z) : "r"(w[i]), "r"(f2));
                y[i] = z;
            }
        }
        uint4 v;
        uint32_t* x = &v.x;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            x[i] = F16 ? __byte_perm(y[2 * i], y[2 * i + 1], 0x5410)
                       : pack_e4m3(__uint_as_float(y[2 * i] << 16), __uint_as_float(y[2 * i] & 0xffff0000u), __uint_as_float(y[2 * i + 1] << 16),
                                   __uint_as_float(y[2 * i + 1] & 0xffff0000u));
        return v;
    }
    float f[16];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        f[2 * i] = F16 ? __half2float(__ushort_as_half((uint16_t)w[i])) : __uint_as_float(w[i] << 16);
        f[2 * i + 1] = F16 ? __half2float(__ushort_as_half((uint16_t)(w[i] >> 16))) : __uint_as_float(w[i] & 0xffff0000u);
    }
    return hold_lane(f, u);
}

__device__ __forceinline__ uint4 hold_lane(const float (&x)[16], uint32_t& u)
{
    float f[16], most = 0.f, odd = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        f[i] = x[i];
        most = fmaxf(most, fabsf(x[i]));
        odd = fmaf(x[i], 0.f, odd);  // NaN if any is not finite
    }
    if (__any_sync(0xffffffffu, odd != odd)) {  // those are NaN, and the scale goes by the others
        most = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const bool finite = fabsf(x[i]) < INFINITY;
            most = fmaxf(most, finite ? fabsf(x[i]) : 0.f);
            if (!finite) f[i] = __uint_as_float(0x7fffffffu);
        }
    }
#pragma unroll
    for (int o = 1; o < 8; o <<= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, o));
    u = scale_byte(most);
    const float z = inverse_scale(u);
    return make_uint4(pack_e4m3(f[0] * z, f[1] * z, f[2] * z, f[3] * z), pack_e4m3(f[4] * z, f[5] * z, f[6] * z, f[7] * z),
                      pack_e4m3(f[8] * z, f[9] * z, f[10] * z, f[11] * z), pack_e4m3(f[12] * z, f[13] * z, f[14] * z, f[15] * z));
}

// The four e4m3 values of a word as fp16 pairs.
__device__ __forceinline__ void widen_e4m3(uint32_t w, uint32_t& lo, uint32_t& hi)
{
    asm("{\n\t.reg .b16 l, h;\n\t"
        "mov.b32 {l, h}, %2;\n\t"
        "cvt.rn.f16x2.e4m3x2 %0, l;\n\t"
        "cvt.rn.f16x2.e4m3x2 %1, h;\n\t}"
        : "=r"(lo), "=r"(hi)
        : "r"(w));
}

}  // namespace
#endif

}  // namespace dkv
