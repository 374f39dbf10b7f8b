// Prune-and-pack into 8-bit pages: the kept rows of a plan's slabs, as e4m3 values with a scale byte a row.
//
//   quant_compact_kernel  a warp has consecutive kept rows, 32 at a time: lane x finds row x's places in the
//                         dense caches and in the pools; then 8 lanes have a row (32 bytes a lane of
//                         K and of V), 4 rows at once, and find its largest element among them.
//
// What bounds it: memory, 512 bytes in and 258 out a row: a 16K prompt of 32 layers, 1.27 GB, in 209 us, 6.05 TB/s (0.91 of a plain
// copy); three ragged ones, 578 MB in pages of 16 rows, in 101. With each element widened to fp32 and looked at for what is
// not finite these took 279 and 119: the row's largest element is found from the 16-bit patterns instead, which order as sizes do.
#include "dkv_quant.cuh"

#include "dkv_decode_common.cuh"

#include <algorithm>

namespace dkv {
namespace {

constexpr int kQcThreads = 256;
constexpr int kQcRows = 4;   // rows of 8 lanes on the way at once

// The last slab h with ioff[h] <= row (one warp: 32 probes a round).
__device__ __forceinline__ int slab_of(const int64_t* ioff, int NH, int64_t row)
{
    const int lane = threadIdx.x & 31;
    int lo = 0, n = NH;  // in [lo, lo + n)
    while (n > 1) {
        const int step = (n + 31) / 32, x = lo + lane * step;
        const unsigned m = __ballot_sync(kFull, lane * step < n && ioff[x] <= row);
        const int k = m ? 31 - __clz(m) : 0;
        n = min(step, n - k * step);
        lo += k * step;
    }
    return lo;
}

template <bool F16>
__device__ __forceinline__ void hold_row(const uint4 (&x)[2], uint8_t* pool, uint8_t* scales, int64_t at, int sub)
{
    const uint32_t w[8] = {x[0].x, x[0].y, x[0].z, x[0].w, x[1].x, x[1].y, x[1].z, x[1].w};
    uint32_t u;
    const uint4 v = hold_lane<F16>(w, u);
    if (at < 0) return;
    reinterpret_cast<uint4*>(pool + at * kHeadDim)[sub] = v;
    if (sub == 0) scales[at] = (uint8_t)u;
}

template <bool F16>
__global__ void __launch_bounds__(kQcThreads) quant_compact_kernel(const __grid_constant__ QuantCompactArgs q, int64_t rows_per_warp)
{
    const PageCompactArgs& a = q.c;
    const int lane = threadIdx.x & 31, sub = lane & 7;
    const int64_t first = ((int64_t)blockIdx.x * (kQcThreads / 32) + (threadIdx.x >> 5)) * rows_per_warp,
                  end = min(a.plan.kept, first + rows_per_warp);
    if (first >= end) return;
    const int NH = a.plan.L * a.plan.B * a.plan.Hkv;
    // The lane's slab: its kept rows end at n1; row r lies at position r + shift of its pool slab.
    int hr = slab_of(a.plan.ioff, NH, first) - 1;
    int64_t n1 = first, shift = 0, entries = 0;  // (no slab yet)
    bool slot_ok = true;
    uint8_t *Kp = reinterpret_cast<uint8_t*>(a.Kp), *Vp = reinterpret_cast<uint8_t*>(a.Vp);
#pragma unroll 1
    for (int64_t r0 = first; r0 < end; r0 += 32) {
        const int64_t r = r0 + lane;
        int64_t from = -1, to = -1;
        if (r < end) {
            const int32_t ix = a.plan.idx[r];
            if (r >= n1) {
                do ++hr;
                while (a.plan.ioff[hr + 1] <= r);
                n1 = a.plan.ioff[hr + 1];
                const int lb = hr / a.plan.Hkv, l = lb / a.plan.B, i = lb - l * a.plan.B, b = a.seq ? a.seq[i] : i;
                slot_ok = b >= 0 && b < a.B && in_bounds(hr < NH && l < a.plan.L, a.status);
                const int64_t h = ((int64_t)l * a.B + (slot_ok ? b : 0)) * a.plan.Hkv + (hr - lb * a.plan.Hkv);
                entries = h * a.max_pages;
                shift = a.len[h] - n1;
            }
            const int64_t pos = r + shift;
            int page = -1;
            if (slot_ok && pos >= 0 && pos < (int64_t)a.max_pages * a.P && ix >= 0 && ix < a.T_stride)
                page = a.table[entries + (int)pos / a.P];
            if (page >= 0 && page < a.num_pages) {
                from = (int64_t)hr * a.T_stride + ix;
                to = (int64_t)page * a.P + (int)pos % a.P;
            } else if (a.status) {
                atomicOr(a.status, DKV_DEV_PAGE_RANGE);
            }
        }
#pragma unroll 1
        for (int x0 = 0; x0 < 32 && r0 + x0 < end; x0 += 4 * kQcRows) {
            uint4 K[kQcRows][2], V[kQcRows][2];
            int64_t at[kQcRows];
#pragma unroll
            for (int y = 0; y < kQcRows; ++y) {
                const int x = x0 + 4 * y + (lane >> 3);
                const int64_t src = __shfl_sync(kFull, from, x);
                at[y] = __shfl_sync(kFull, to, x);
                K[y][0] = K[y][1] = V[y][0] = V[y][1] = make_uint4(0u, 0u, 0u, 0u);
                if (src >= 0) {
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        K[y][i] = __ldcs(reinterpret_cast<const uint4*>(a.K + src * kHeadDim) + 2 * sub + i);
                        V[y][i] = __ldcs(reinterpret_cast<const uint4*>(a.V + src * kHeadDim) + 2 * sub + i);
                    }
                }
            }
#pragma unroll
            for (int y = 0; y < kQcRows; ++y) {
                hold_row<F16>(K[y], Kp, q.Ks, at[y], sub);
                hold_row<F16>(V[y], Vp, q.Vs, at[y], sub);
            }
        }
    }
}

}  // namespace

cudaError_t launch_quant_compact(const QuantCompactArgs& a, cudaStream_t st)
{
    if (a.c.plan.kept == 0) return cudaSuccess;
    int sms = 0;
    const cudaError_t e = page_setup(&sms);
    if (e != cudaSuccess) return e;
    const int64_t groups = (a.c.plan.kept + 31) / 32, per = kQcThreads / 32, warps = std::min<int64_t>(groups, (int64_t)sms * 2 * per);
    const int64_t rows_per_warp = (groups + warps - 1) / warps * 32;
    const unsigned grid = (unsigned)((warps + per - 1) / per);
    if (a.fp16)
        quant_compact_kernel<true><<<grid, kQcThreads, 0, st>>>(a, rows_per_warp);
    else
        quant_compact_kernel<false><<<grid, kQcThreads, 0, st>>>(a, rows_per_warp);
    return cudaGetLastError();
}

}  // namespace dkv
