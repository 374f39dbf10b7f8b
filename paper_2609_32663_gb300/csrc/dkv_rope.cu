// Rotary positions, and a step's rows on their way to the pages.
//
// Pair (a, b) of a row at position p becomes m (a cos x - b sin x, b cos x + a sin x), x = p f. A
// frequency is held in 2^-64 of a turn, so p f modulo a turn is the low half of a 64-bit product, exact for any
// p; its nearest quarter turn is taken off in integers, which leaves at most an eighth of a turn
// with 29 bits, and cos and sin are taken of that in fp32.
//
//   rope_kernel  a CTA has some tokens; its threads first compute their pairs' cos and sin into shared
//                memory, one pair a thread, which serve all heads of a token. Then 8 lanes have a row: lane s
//                turns pairs 8s .. 8s + 7, which lie in two 16-byte chunks in either layout, or copies two chunks
//                behind rot_dim. k and v rows go to their pages, 16-bit or (after the row's largest
//                element is found over the 8 lanes) as e4m3 values with a scale byte.
//
// What bounds it: memory, each row in and out once.
#include "dkv_quant.cuh"

#include "dkv_tcgen05.cuh"

#include <cuda_bf16.h>
#include <cuda_fp16.h>

namespace dkv {
namespace {

constexpr int kRopeThreads = 256;
constexpr int kRopeTokens = 8;  // tokens of a CTA, at most
constexpr int kBatch = 4;       // rows of 8 lanes on the way at once

template <bool F16>
__device__ __forceinline__ float2 widen16(uint32_t u)
{
    if (F16) return __half22float2(*reinterpret_cast<const __half2*>(&u));
    return make_float2(__uint_as_float(u << 16), __uint_as_float(u & 0xffff0000u));
}

template <bool F16>
__device__ __forceinline__ uint32_t narrow16(float lo, float hi)
{
    if (F16) {
        const __half2 x = __floats2half2_rn(lo, hi);
        return *reinterpret_cast<const uint32_t*>(&x);
    }
    return pack_bf16(lo, hi);
}

// cos and sin of `turns` (units of 2^-64 of a turn, modulo 1), times m.
__device__ __forceinline__ float2 turn(uint64_t turns, float m)
{
    const uint32_t hi = (uint32_t)(turns >> 32), lo = (uint32_t)turns;
    const uint32_t quarter = (hi + 0x20000000u) >> 30;  // the nearest (modulo 4)
    const int32_t rest = (int32_t)(hi - (quarter << 30));
    // In half turns, [-1/4, 1/4]: 2^-31 of `rest`, whose lower bits are in `lo`.
    const float x = fmaf((float)(lo >> 8), 0x1p-55f, (float)rest * 0x1p-31f);
    float s, c;
    sincospif(x, &s, &c);
    const float c1 = quarter & 1 ? -s : c, s1 = quarter & 1 ? c : s;
    return quarter & 2 ? make_float2(-c1 * m, -s1 * m) : make_float2(c1 * m, s1 * m);
}

__device__ __forceinline__ void report(const RopeArgs& a, int bits)
{
    if (a.status) atomicOr(a.status, bits);
}

// POOL: bits of an element of the pools; 0: no k and v.
template <bool F16, bool INTER, int POOL>
__global__ void __launch_bounds__(kRopeThreads) rope_kernel(const __grid_constant__ RopeArgs a, int tokens)
{
    __shared__ float4 cs[kRopeTokens][32];  // a pair's (cos, sin), two pairs
    __shared__ int32_t cu[kMaxSlots + 1];
    const int tid = threadIdx.x, per = kRopeThreads / tokens, mine = tid / per, t = blockIdx.x * tokens + mine;
    const int sub = tid & 7, group = (tid - mine * per) >> 3, groups = per >> 3, pairs = a.rot >> 1;
    const int heads = a.q ? a.H : 0, all = POOL ? heads + 2 * a.Hkv : heads;
    const bool turned = sub < a.rot >> 4;
    // The lane's two chunks of 8 elements.
    const int chunk0 = turned ? (INTER ? 2 * sub : sub) : 2 * sub, chunk1 = turned && !INTER ? sub + (a.rot >> 4) : chunk0 + 1;
    uint4 x[kBatch][2];
    auto load = [&](int h0) {
#pragma unroll
        for (int y = 0; y < kBatch; ++y) {
            const int h = h0 + y * groups + group;
            if (h < all && t < a.T) {
                const uint16_t* src = h < heads ? a.q + t * a.q_stride + (int64_t)h * kHeadDim
                                                : (h < heads + a.Hkv ? a.k + (int64_t)(h - heads) * kHeadDim
                                                                     : a.v + (int64_t)(h - heads - a.Hkv) * kHeadDim) +
                                                      t * a.kv_stride;
                x[y][0] = __ldcs(reinterpret_cast<const uint4*>(src) + chunk0);
                x[y][1] = __ldcs(reinterpret_cast<const uint4*>(src) + chunk1);
            } else {
                x[y][0] = x[y][1] = make_uint4(0u, 0u, 0u, 0u);
            }
        }
    };
    pdl_wait();
    pdl_launch_dependents();
    load(0);  // on their way while cos and sin are found
    for (int i = tid; i < tokens * pairs; i += kRopeThreads) {
        const int x = i / pairs, pair = i - x * pairs, at = blockIdx.x * tokens + x;
        if (at < a.T) reinterpret_cast<float2*>(cs[x])[pair] = turn(a.turns[pair] * (uint64_t)(int64_t)a.positions[at], a.magnitude);
    }
    bool bad = false;
    if (a.cu) {
        for (int b = tid; b <= a.B; b += kRopeThreads) {
            const int c0 = a.cu[b];
            cu[b] = c0;
            if (b < a.B) {
                const int c1 = a.cu[b + 1];
                bad |= c1 < c0 || c1 > a.T || (b == 0 && c0 != 0);
            }
        }
    }
    if (__syncthreads_or(bad)) {
        if (blockIdx.x == 0 && tid == 0) report(a, DKV_DEV_PAGE_RANGE);
        return;
    }
    if (t >= (a.cu ? cu[a.B] : a.T)) return;  // (whole warps)
    float c[8], s[8];
    if (turned) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float4 x = cs[mine][4 * sub + i];
            c[2 * i] = x.x;
            s[2 * i] = x.y;
            c[2 * i + 1] = x.z;
            s[2 * i + 1] = x.w;
        }
    }
    const int log_P = 31 - __clz(max(a.P, 1));
    int b = 0, back = 0;  // the token's sequence, and how far from the end of its slabs the token's row lies
    if (POOL) {
        int hi = a.B - 1;  // the last sequence that starts at t or before
        while (b < hi) {
            const int mid = (b + hi + 1) >> 1;
            if (cu[mid] <= t)
                b = mid;
            else
                hi = mid - 1;
        }
        back = cu[b + 1] - t;
    }
#pragma unroll 1
    for (int h0 = 0; h0 < all; h0 += kBatch * groups) {
        if (h0) load(h0);
        int page[kBatch], row[kBatch];  // of k and v: the page, and the row in it
#pragma unroll
        for (int y = 0; y < kBatch; ++y) {
            const int h = h0 + y * groups + group;
            page[y] = -1;
            row[y] = 0;
            if (POOL && h >= heads && h < all) {
                const int64_t slab = (int64_t)b * a.Hkv + (h - heads < a.Hkv ? h - heads : h - heads - a.Hkv);
                const int n = a.len[slab], r = n - back;
                if (r >= 0 && n <= a.max_pages * a.P) {  // (the product is below 2^31)
                    page[y] = a.table[slab * a.max_pages + (r >> log_P)];
                    row[y] = r & (a.P - 1);
                }
            }
        }
#pragma unroll
        for (int y = 0; y < kBatch; ++y) {
            const int h = h0 + y * groups + group;
            const bool pooled = POOL && h >= heads && h < all, key = h < heads + a.Hkv;
            if (POOL != 8 && h >= all) continue;
            uint32_t w[8] = {x[y][0].x, x[y][0].y, x[y][0].z, x[y][0].w, x[y][1].x, x[y][1].y, x[y][1].z, x[y][1].w};
            float f[16];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float2 v = widen16<F16>(w[i]);
                f[2 * i] = v.x;
                f[2 * i + 1] = v.y;
            }
            if (turned && key) {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int p = INTER ? 2 * i : i, q = INTER ? 2 * i + 1 : i + 8;
                    const float u = f[p], v = f[q];
                    f[p] = fmaf(u, c[i], -v * s[i]);
                    f[q] = fmaf(v, c[i], u * s[i]);
                }
#pragma unroll
                for (int i = 0; i < 8; ++i) w[i] = narrow16<F16>(f[2 * i], f[2 * i + 1]);
            }
            if (!pooled && h < all) {
                uint4* dst = reinterpret_cast<uint4*>(a.q_out + t * a.out_stride + (int64_t)h * kHeadDim);
                dst[chunk0] = make_uint4(w[0], w[1], w[2], w[3]);
                dst[chunk1] = make_uint4(w[4], w[5], w[6], w[7]);
            }
            if (POOL == 0) continue;
            const bool placed = pooled && page[y] >= 0 && page[y] < a.num_pages;
            if (pooled && !placed && sub == 0) report(a, DKV_DEV_PAGE_RANGE);
            const int64_t at = (int64_t)page[y] * a.P + row[y];
            if (POOL == 16) {
                if (placed) {
                    uint4* dst = reinterpret_cast<uint4*>(static_cast<uint16_t*>(key ? a.Kp : a.Vp) + at * kHeadDim);
                    dst[chunk0] = make_uint4(w[0], w[1], w[2], w[3]);
                    dst[chunk1] = make_uint4(w[4], w[5], w[6], w[7]);
                }
            } else if (__any_sync(kFull, pooled)) {
                float most = 0.f;
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    float size;
                    f[i] = held(f[i], size);
                    most = fmaxf(most, size);
                }
#pragma unroll
                for (int o = 1; o < 8; o <<= 1) most = fmaxf(most, __shfl_xor_sync(kFull, most, o));
                const uint32_t u = scale_byte(most);
                const float z = inverse_scale(u);
                if (placed) {
                    uint2* dst = reinterpret_cast<uint2*>(static_cast<uint8_t*>(key ? a.Kp : a.Vp) + at * kHeadDim);
                    dst[chunk0] = make_uint2(pack_e4m3(f[0] * z, f[1] * z, f[2] * z, f[3] * z), pack_e4m3(f[4] * z, f[5] * z, f[6] * z, f[7] * z));
                    dst[chunk1] = make_uint2(pack_e4m3(f[8] * z, f[9] * z, f[10] * z, f[11] * z),
                                             pack_e4m3(f[12] * z, f[13] * z, f[14] * z, f[15] * z));
                    if (sub == 0) (key ? a.Ks : a.Vs)[at] = (uint8_t)u;
                }
            }
        }
    }
}

template <bool F16, bool INTER>
cudaError_t launch_pool(const RopeArgs& a, int grid, int tokens, cudaStream_t st)
{
    if (!a.k) return launch_pdl(rope_kernel<F16, INTER, 0>, grid, kRopeThreads, 0, st, a, tokens);
    return a.Ks ? launch_pdl(rope_kernel<F16, INTER, 8>, grid, kRopeThreads, 0, st, a, tokens)
                : launch_pdl(rope_kernel<F16, INTER, 16>, grid, kRopeThreads, 0, st, a, tokens);
}

}  // namespace

cudaError_t launch_rope(const RopeArgs& a, cudaStream_t st)
{
    int sms = 0;
    const cudaError_t e = page_setup(&sms);
    if (e != cudaSuccess) return e;
    // A CTA has so many tokens that a thread has its rows in one batch; fewer, where the SMs would not all have a CTA.
    const int heads = (a.q ? a.H : 0) + (a.k ? 2 * a.Hkv : 0);
    int tokens = kRopeTokens;
    while (tokens > 1 && (tokens * heads > kBatch * kRopeThreads / 8 || a.T < 2 * sms * tokens)) tokens >>= 1;
    const int grid = (a.T + tokens - 1) / tokens;
    if (a.fp16) return a.interleaved ? launch_pool<true, true>(a, grid, tokens, st) : launch_pool<true, false>(a, grid, tokens, st);
    return a.interleaved ? launch_pool<false, true>(a, grid, tokens, st) : launch_pool<false, false>(a, grid, tokens, st);
}

}  // namespace dkv
