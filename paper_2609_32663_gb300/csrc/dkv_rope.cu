// Rotary positions, and a step's rows on their way to the pages.
//
// Pair (a, b) of a row at position p becomes m (a cos x - b sin x, b cos x + a sin x), x = p f. A
// frequency is held in 2^-64 of a turn, so p f modulo a turn is the low half of a 64-bit product, exact for any
// p; its nearest quarter turn is taken off in integers, which leaves at most an eighth of a turn
// with 29 bits, and cos and sin are taken of that in fp32.
//
//   rope_kernel  one CTA an SM. An item is some heads of a token; a warp takes every n-th item, whose rows
//                land in a ring of its own by bulk copies (the heads of a token lie together), and finds the token's
//                cos and sin, two pairs a lane. Then 8 lanes have a row: lane s turns pairs 8s .. 8s + 7, which lie in two
//                16-byte chunks in either layout, or copies two chunks behind rot_dim. k and v rows go to their
//                pages, 16-bit or (after the row's largest element is found over the 8 lanes) as e4m3 values with a
//                scale byte.
//
// What bounds it: memory, each row in and out once: 30,001 tokens of 28 heads, 430 MB, take 75 us, where a plain copy of as much
// takes 70; 16K tokens of 8 heads in a wider projection 18.7 us (67 MB: 14.4), a turn of 4K tokens to 8-bit pages 22 (92 MB: 17):
// a launch, the first rows' latency and three to seven items a warp. As a grid of short CTAs that kept rows in registers these
// took 69, 22 and 30 us; two CTAs an SM of half the warps, 24 warps, or no unrolling change nothing or cost up to 5 us.
#include "dkv_quant.cuh"

#include "dkv_tcgen05.cuh"

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <algorithm>

namespace dkv {
namespace {

constexpr int kRopeWarps = 16;
constexpr int kRopeThreads = 32 * kRopeWarps;
constexpr int kMostHeads = 24;      // rows of an item, at most
constexpr int kMostStages = 8;      // of a warp's ring
constexpr int kRopeRing = 192 * 1024;
// Shared memory: the rings, then a warp's (cos, sin) of its item's pairs, its barriers, and the token offsets.
constexpr int kOffTurns = kRopeRing, kOffRopeBars = kOffTurns + kRopeWarps * 64 * 8, kOffCu = kOffRopeBars + kRopeWarps * kMostStages * 8,
              kRopeSmem = kOffCu + (kMaxSlots + 1) * 4;
static_assert(kRopeRing % (kRopeWarps * kRowBytes) == 0, "a warp's ring starts on a row's alignment");
static_assert(kRopeSmem <= 227 * 1024 && kRopeWarps * 2 * kMostHeads * kRowBytes <= kRopeRing, "fits one CTA, two stages a warp");

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

// How a call is cut: a token's `all` heads (of q, k and v) in `parts` items of up to `heads` rows, rings of `stages`.
struct RopeCut {
    int all, parts, heads, stages;
};

// Part `part` of token t. Items lie part after part, so that a warp has some of every part (those of k and v cost more).
struct Item {
    int t, part;
    __device__ __forceinline__ void advance(int by_t, int by_part, int tokens)
    {
        t += by_t;
        part += by_part;
        if (t >= tokens) {
            t -= tokens;
            ++part;
        }
    }
};

// POOL: bits of an element of the pools; 0: no k and v.
template <bool F16, bool INTER, int POOL>
__global__ void __launch_bounds__(kRopeThreads, 1) rope_kernel(const __grid_constant__ RopeArgs a, const RopeCut cut)
{
    extern __shared__ __align__(128) unsigned char sm[];
    const int tid = threadIdx.x, warp = uniform(tid >> 5), lane = tid & 31, sub = lane & 7, pairs = a.rot >> 1;
    unsigned char* ring = sm + warp * (kRopeRing / kRopeWarps);
    float2* cs = reinterpret_cast<float2*>(sm + kOffTurns) + warp * 64;
    uint64_t* full = reinterpret_cast<uint64_t*>(sm + kOffRopeBars) + warp * kMostStages;
    int32_t* cu = reinterpret_cast<int32_t*>(sm + kOffCu);
    if (lane < cut.stages) mbar_init(smem_u32(full + lane), 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    fence_proxy_async_smem();
    __syncwarp();
    const int qheads = a.q ? a.H : 0;
    const bool turned = sub < a.rot >> 4;
    // The lane's two chunks of 8 elements.
    const int chunk0 = turned ? (INTER ? 2 * sub : sub) : 2 * sub, chunk1 = turned && !INTER ? sub + (a.rot >> 4) : chunk0 + 1;
    const int log_P = 31 - __clz(max(a.P, 1));
    pdl_wait();
    pdl_launch_dependents();
    int tokens = a.T;
    if (a.cu) {
        bool bad = false;
        for (int b = tid; b <= a.B; b += kRopeThreads) {
            const int c0 = a.cu[b];
            cu[b] = c0;
            if (b < a.B) {
                const int c1 = a.cu[b + 1];
                bad |= c1 < c0 || c1 > a.T || (b == 0 && c0 != 0);
            }
        }
        if (__syncthreads_or(bad)) {
            if (blockIdx.x == 0 && tid == 0) report(a, DKV_DEV_PAGE_RANGE);
            return;
        }
        tokens = cu[a.B];
    }
    if (tokens <= 0) return;
    // Every n-th item from the first on; a few lie in as many SMs. (There are fewer than 2^31, see tokens_ok.)
    const int first = blockIdx.x + gridDim.x * warp, stride = gridDim.x * kRopeWarps, by_part = stride / tokens, by_t = stride - by_part * tokens;
    Item now{first % tokens, first / tokens};
    if (now.part >= cut.parts) return;
    const int stage_bytes = cut.heads * kRowBytes;
    const uint64_t pol = evict_first_policy();
    // Rows [h0, h1) of an item: heads of q, then of k, then of v.
    auto fetch = [&](const Item& x, int stage) {
        if (x.part >= cut.parts) return;
        const int t = x.t, h0 = x.part * cut.heads, h1 = min(h0 + cut.heads, cut.all);
        if (lane == 0) {
            const uint32_t bar = smem_u32(full + stage), dst = smem_u32(ring) + stage * stage_bytes;
            mbar_arrive_expect_tx(bar, (h1 - h0) * kRowBytes);
            const int q1 = min(h1, qheads);
            // (dkv_rope's heads may be more than 2^24: their elements pass 32 bits. Those of a geometry do not.)
            if (q1 > h0) bulk_g2s(dst, a.q + t * a.q_stride + (int64_t)h0 * kHeadDim, (q1 - h0) * kRowBytes, bar, pol);
            if (POOL) {
                const int k0 = max(h0, qheads), k1 = min(h1, qheads + a.Hkv), v0 = max(h0, qheads + a.Hkv);
                const int64_t row = t * a.kv_stride;
                if (k1 > k0) bulk_g2s(dst + (k0 - h0) * kRowBytes, a.k + row + (k0 - qheads) * kHeadDim, (k1 - k0) * kRowBytes, bar, pol);
                if (h1 > v0) bulk_g2s(dst + (v0 - h0) * kRowBytes, a.v + row + (v0 - qheads - a.Hkv) * kHeadDim, (h1 - v0) * kRowBytes, bar, pol);
            }
        }
        __syncwarp();
    };
    // Lane x: the place in its slab of row x of an item, if that is one of k or v (-1: none).
    auto place = [&](const Item& x, int64_t& entry) {
        entry = 0;
        if (!POOL || x.part >= cut.parts) return -1;
        const int t = x.t, h = x.part * cut.heads + lane;
        if (h < qheads || h >= min((x.part + 1) * cut.heads, cut.all)) return -1;
        int b = 0, hi = a.B - 1;  // the last sequence that starts at t or before
        while (b < hi) {
            const int mid = (b + hi + 1) >> 1;
            if (cu[mid] <= t)
                b = mid;
            else
                hi = mid - 1;
        }
        const int64_t slab = (int64_t)b * a.Hkv + (h - qheads < a.Hkv ? h - qheads : h - qheads - a.Hkv);
        // (Both ends of n are looked at before the place is formed: a length near -2^31 would wrap to one that passes.)
        const int n = a.len[slab], behind = cu[b + 1] - t;  // behind: 1 .. T
        if (n < behind || n > a.max_pages * a.P) {          // (the product is below 2^31)
            report(a, DKV_DEV_PAGE_RANGE);
            return -1;
        }
        entry = slab * a.max_pages;
        return n - behind;
    };
    static_assert(kMostHeads <= 32, "a lane each");
    Item ahead = now;
    for (int s = 0; s < cut.stages; ++s) {
        fetch(ahead, s);
        ahead.advance(by_t, by_part, tokens);
    }
    int64_t entry;
    int pos = pairs ? a.positions[now.t] : 0, row = place(now, entry), stage = 0;
    uint32_t phase = 0;
    bool ok = true;
#pragma unroll 1
    while (now.part < cut.parts) {
        const int t = now.t, h0 = now.part * cut.heads, h1 = min(h0 + cut.heads, cut.all);
        int page = -1;
        if (POOL && row >= 0) {
            page = in_bounds(row >> log_P < a.max_pages, a.status) ? a.table[entry + (row >> log_P)] : -1;
            row &= a.P - 1;
        }
        for (int i = lane; i < pairs; i += 32) cs[i] = turn(a.turns[i] * (uint64_t)(int64_t)pos, a.magnitude);
        const int place0 = row;
        now.advance(by_t, by_part, tokens);
        if (pairs && now.part < cut.parts) pos = a.positions[now.t];
        row = place(now, entry);
        int64_t at = -1;  // the pool row
        if (POOL && h0 + lane >= qheads && h0 + lane < h1) {
            if (page >= 0 && page < a.num_pages)
                at = (int64_t)page * a.P + place0;
            else
                report(a, DKV_DEV_PAGE_RANGE);
        }
        __syncwarp();
        float c[8], s[8];
        if (turned) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float4 x = *reinterpret_cast<const float4*>(cs + 8 * sub + 2 * i);
                c[2 * i] = x.x;
                s[2 * i] = x.y;
                c[2 * i + 1] = x.z;
                s[2 * i + 1] = x.w;
            }
        }
        if (!__all_sync(kFull, mbar_wait(smem_u32(full + stage), phase))) {
            ok = false;
            break;
        }
        const unsigned char* rows = ring + stage * stage_bytes;
        uint16_t* out = a.q_out + t * a.out_stride;
#pragma unroll 2
        for (int x0 = 0; x0 < h1 - h0; x0 += 4) {
            const int x = x0 + (lane >> 3), h = h0 + x;
            const bool some = h < h1, pooled = POOL && some && h >= qheads, key = h < qheads + a.Hkv;
            const uint4 lo = *reinterpret_cast<const uint4*>(rows + min(x, cut.heads - 1) * kRowBytes + chunk0 * 16),
                        hi = *reinterpret_cast<const uint4*>(rows + min(x, cut.heads - 1) * kRowBytes + chunk1 * 16);
            uint32_t w[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
            const int64_t to = POOL ? __shfl_sync(kFull, at, min(x, 31)) : -1;
            const bool turns = __any_sync(kFull, some && key && turned);
            float f[16];
            if (turns) {
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
                    if (POOL != 8 || !pooled) {
#pragma unroll
                        for (int i = 0; i < 8; ++i) w[i] = narrow16<F16>(f[2 * i], f[2 * i + 1]);
                    }
                }
            }
            if (some && !(POOL && pooled)) {
                uint4* dst = reinterpret_cast<uint4*>(out + (int64_t)h * kHeadDim);
                dst[chunk0] = make_uint4(w[0], w[1], w[2], w[3]);
                dst[chunk1] = make_uint4(w[4], w[5], w[6], w[7]);
            }
            if (POOL == 16 && pooled && to >= 0) {
                uint4* dst = reinterpret_cast<uint4*>(static_cast<uint16_t*>(key ? a.Kp : a.Vp) + to * kHeadDim);
                dst[chunk0] = make_uint4(w[0], w[1], w[2], w[3]);
                dst[chunk1] = make_uint4(w[4], w[5], w[6], w[7]);
            }
            if (POOL == 8 && __any_sync(kFull, pooled)) {
                uint4 v;
                uint32_t u;
                if (!__any_sync(kFull, pooled && !(key && turns))) {
                    v = hold_lane(f, u);
                } else {
                    v = hold_lane<F16>(w, u);
                    if (turns) {  // rows of both kinds
                        uint32_t u1;
                        const uint4 v1 = hold_lane(f, u1);
                        if (key) v = v1, u = u1;
                    }
                }
                if (pooled && to >= 0) {
                    uint2* dst = reinterpret_cast<uint2*>(static_cast<uint8_t*>(key ? a.Kp : a.Vp) + to * kHeadDim);
                    dst[chunk0] = make_uint2(v.x, v.y);
                    dst[chunk1] = make_uint2(v.z, v.w);
                    if (sub == 0) (key ? a.Ks : a.Vs)[to] = (uint8_t)u;
                }
            }
        }
        __syncwarp();  // the stage, and cos and sin, are read
        fetch(ahead, stage);
        ahead.advance(by_t, by_part, tokens);
        if (++stage == cut.stages) {
            stage = 0;
            phase ^= 1;
        }
    }
    if (!ok) {
        if (lane == 0) report(a, DKV_DEV_TMA_TIMEOUT);
        for (int s = 0; s < cut.stages; ++s)  // copies in flight land, or run out of time, before the CTA exits
            for (int parity = 0; parity < 2; ++parity) mbar_wait(smem_u32(full + s), parity);
    }
}

template <bool F16, bool INTER, int POOL>
cudaError_t launch_one(const RopeArgs& a, const RopeCut& cut, int grid, cudaStream_t st)
{
    return launch_pdl(rope_kernel<F16, INTER, POOL>, grid, kRopeThreads, kRopeSmem, st, a, cut);
}

template <bool F16, bool INTER>
cudaError_t launch_pool(const RopeArgs& a, const RopeCut& cut, int grid, cudaStream_t st)
{
    if (!a.k) return launch_one<F16, INTER, 0>(a, cut, grid, st);
    return a.Ks ? launch_one<F16, INTER, 8>(a, cut, grid, st) : launch_one<F16, INTER, 16>(a, cut, grid, st);
}

template <bool F16, bool INTER>
cudaError_t setup_pools()
{
    const auto attr = cudaFuncAttributeMaxDynamicSharedMemorySize;
    cudaError_t e = cudaFuncSetAttribute(rope_kernel<F16, INTER, 0>, attr, kRopeSmem);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(rope_kernel<F16, INTER, 8>, attr, kRopeSmem);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(rope_kernel<F16, INTER, 16>, attr, kRopeSmem);
    return e;
}

}  // namespace

cudaError_t rope_setup()
{
    cudaError_t e = setup_pools<false, false>();
    if (e == cudaSuccess) e = setup_pools<false, true>();
    if (e == cudaSuccess) e = setup_pools<true, false>();
    if (e == cudaSuccess) e = setup_pools<true, true>();
    return e;
}

cudaError_t launch_rope(const RopeArgs& a, cudaStream_t st)
{
    int sms = 0;
    const cudaError_t e = page_setup(&sms);
    if (e != cudaSuccess) return e;
    RopeCut cut;
    cut.all = (a.q ? a.H : 0) + (a.k ? 2 * a.Hkv : 0);
    // Items of as many rows as a ring takes, or of fewer (four are the lanes of a warp), where the warps would not all have one.
    const int64_t warps = (int64_t)sms * kRopeWarps, wanted = (warps + a.T - 1) / a.T;
    const int most = (int)std::min<int64_t>((cut.all + 3) / 4, std::max<int64_t>(wanted, (cut.all + kMostHeads - 1) / kMostHeads));
    cut.heads = ((cut.all + most - 1) / most + 3) / 4 * 4;
    cut.parts = (cut.all + cut.heads - 1) / cut.heads;
    cut.stages = std::min(kMostStages, kRopeRing / kRopeWarps / (cut.heads * kRowBytes));
    const int grid = (int)std::min<int64_t>(sms, (int64_t)a.T * cut.parts);
    if (a.fp16) return a.interleaved ? launch_pool<true, true>(a, cut, grid, st) : launch_pool<true, false>(a, cut, grid, st);
    return a.interleaved ? launch_pool<false, true>(a, cut, grid, st) : launch_pool<false, false>(a, cut, grid, st);
}

}  // namespace dkv
