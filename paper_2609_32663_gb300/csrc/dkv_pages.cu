// The page tables of a paged cache: pages for new rows, the slot map of new tokens,
// pages given back, and the prune-and-pack (Sec. 3.4) into pages.
//
// Row r of slab h is row table[h][r / P] * P + r % P of the page pools (P rows a
// page, a power of two). A slab of len rows holds its first ceil(len / P) entries.
//
//   grow     slab h takes need_h = ceil((len_h + n_h) / P) - ceil(len_h / P) pages; in slab
//            order they come from the end of the free list: the k-th page that the call
//            takes is free[count - 1 - k].
//   release  an ended slab gives back its pages, in slab order behind the free list's end.
//
// Two launches: page_scan_kernel checks every argument that lives on the device, scans the
// slabs' page counts and writes lengths, counts and token offsets (nothing, if a check
// fails or the free list is too short); page_fill_kernel then writes the table entries (or
// the free list's) and the slot map from the scan.
#include "dkv_decode_common.cuh"
#include "dkv_pages.cuh"
#include "dkv_pool.cuh"

#include <mutex>

namespace dkv {
namespace {

constexpr int kScanThreads = 1024;
constexpr int kDevExhausted = DKV_DEV_PAGES_EXHAUSTED;
constexpr int kDevRange = DKV_DEV_PAGE_RANGE;

// Sum of x over the block's earlier threads; *total receives the whole sum.
__device__ __forceinline__ int64_t block_scan(int64_t x, int64_t* sh, int64_t* total)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int64_t v = x;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int64_t y = __shfl_up_sync(kFull, v, o);
        if (lane >= o) v += y;
    }
    __syncthreads();
    if (lane == 31) sh[warp] = v;
    __syncthreads();
    if (warp == 0) {
        int64_t w = lane < (int)(blockDim.x >> 5) ? sh[lane] : 0;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int64_t y = __shfl_up_sync(kFull, w, o);
            if (lane >= o) w += y;
        }
        sh[lane] = w;
    }
    __syncthreads();
    *total = sh[31];
    return v - x + (warp ? sh[warp - 1] : 0);
}

// Rows that slab h of the pool gains (grow; negative: out of range) or gives up (release).
// per_slot: per sequence slot, the new tokens, the ended flag or the plan's sequence (-1: none).
__device__ __forceinline__ int slab_rows(const PageArgs& a, const int32_t* per_slot, int h, int len)
{
    const int b = h / a.Hkv % a.B;
    const int x = per_slot[b];
    if (a.mode == kGrowTokens) return x;
    if (a.mode == kRelease) return x ? len : 0;
    const int l = h / (a.Hkv * a.B);
    return x < 0 ? 0 : a.plan_len[((int64_t)l * a.planB + x) * a.Hkv + h % a.Hkv];
}

__device__ __forceinline__ int pages_of(int64_t rows, int P) { return (int)((rows + P - 1) / P); }

__global__ void __launch_bounds__(kScanThreads) page_scan_kernel(const PageArgs a)
{
    __shared__ int64_t sh[32];
    __shared__ int32_t per_slot[kMaxSlots];
    __shared__ int bad;
    const int tid = threadIdx.x;
    pdl_wait();
    pdl_launch_dependents();
    if (tid == 0) bad = 0;
    for (int b = tid; b < a.B; b += kScanThreads) per_slot[b] = a.mode == kGrowPlan ? -1 : a.tokens[b];
    __syncthreads();
    int flags = 0;
    if (a.mode == kGrowPlan) {
        for (int i = tid; i < a.planB; i += kScanThreads) {
            const int b = a.seq ? a.seq[i] : i;
            if (b < 0 || b >= a.B || (a.seq && i > 0 && a.seq[i - 1] >= b))
                flags |= kDevRange;  // slots ascend, so that no slot is named twice
            else
                per_slot[b] = i;
        }
        __syncthreads();
    }
    // Token offsets.
    int64_t tokens = 0;
    if (a.mode == kGrowTokens) {
        const int n = tid < a.B ? per_slot[tid] : 0;
        if (n < 0) flags |= kDevRange;
        const int64_t before = block_scan(max(n, 0), sh, &tokens);
        if (a.cu && tid < a.B) a.cu[tid] = (int)min(before, (int64_t)INT32_MAX);
        if (a.cu && tid == 0) a.cu[a.B] = (int)min(tokens, (int64_t)INT32_MAX);
        if (tokens > (a.slots ? a.max_tokens : (int64_t)INT32_MAX)) flags |= kDevRange;
    }
    // Pages of this thread's slabs, a contiguous piece of them.
    const int64_t per = (a.NH + kScanThreads - 1) / kScanThreads;
    const int64_t h0 = min((int64_t)a.NH, tid * per), h1 = min((int64_t)a.NH, h0 + per);
    const int64_t cap = (int64_t)a.max_pages * a.P;
    int64_t mine = 0;
    for (int64_t h = h0; h < h1; ++h) {
        const int len = a.len[h], n = slab_rows(a, per_slot, (int)h, len);
        if (len < 0 || n < 0 || (int64_t)len + (a.mode == kRelease ? 0 : n) > cap) {
            flags |= kDevRange;
            continue;
        }
        mine += a.mode == kRelease ? (n ? pages_of(len, a.P) : 0) : pages_of((int64_t)len + n, a.P) - pages_of(len, a.P);
    }
    int64_t pages;
    int64_t at = block_scan(mine, sh, &pages);
    const int count = *a.free_count;
    if (count < 0 || count > a.num_pages)
        flags |= kDevRange;
    else if (a.mode == kRelease ? count + pages > a.num_pages : pages > count)
        flags |= a.mode == kRelease ? kDevRange : kDevExhausted;
    if (flags) atomicOr(&bad, flags);
    __syncthreads();
    const bool ok = bad == 0;
    if (!ok && a.cu)
        for (int b = tid; b <= a.B; b += kScanThreads) a.cu[b] = 0;
    for (int64_t h = h0; h < h1; ++h) {
        const int len = a.len[h], n = ok ? slab_rows(a, per_slot, (int)h, len) : 0;
        a.before[h] = len;
        a.first[h] = (int)at;
        if (ok) at += a.mode == kRelease ? (n ? pages_of(len, a.P) : 0) : pages_of((int64_t)len + n, a.P) - pages_of(len, a.P);
        a.new_len[h] = a.mode == kRelease ? len - n : len + n;
    }
    if (tid == 0) {
        *a.head = PageHead{ok, count, (int)min(tokens, (int64_t)INT32_MAX), (int)pages};
        *a.new_count = ok ? (int)(a.mode == kRelease ? count + pages : count - pages) : count;
        if (!ok && a.status) atomicOr(a.status, bad);
    }
}

constexpr int kFillThreads = 256;

__global__ void __launch_bounds__(kFillThreads) page_fill_kernel(const PageArgs a)
{
    __shared__ int32_t cu[kMaxSlots + 1];
    pdl_wait();
    const PageHead head = *a.head;
    if (!head.ok) return;
    const int lane = threadIdx.x & 31;
    // Pages: one warp a slab.
    for (int h = (blockIdx.x * kFillThreads + threadIdx.x) >> 5; h < a.NH; h += gridDim.x * (kFillThreads / 32)) {
        const int first = a.first[h], next = h + 1 < a.NH ? a.first[h + 1] : head.pages;
        int32_t* row = a.table + (int64_t)h * a.max_pages;
        if (a.mode == kRelease) {
            for (int j = lane; j < next - first; j += 32) a.free_pages[head.count + first + j] = row[j];
        } else {
            row += pages_of(a.before[h], a.P);
            for (int j = lane; j < next - first; j += 32) row[j] = a.free_pages[head.count - 1 - first - j];
        }
    }
    if (!a.slots) return;
    for (int b = threadIdx.x; b <= a.B; b += kFillThreads) cu[b] = a.cu[b];
    __syncthreads();
    // Slot map: [L][t][Hkv], one thread an entry.
    const int64_t per_layer = (int64_t)head.total * a.Hkv, n = per_layer * a.L;
    for (int64_t i = (int64_t)blockIdx.x * kFillThreads + threadIdx.x; i < n; i += (int64_t)gridDim.x * kFillThreads) {
        const int l = (int)(i / per_layer);
        const int64_t x = i - l * per_layer;
        const int t = (int)(x / a.Hkv), g = (int)(x - (int64_t)t * a.Hkv);
        int lo = 0, hi = a.B - 1;  // the last sequence that starts at t or before
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (cu[mid] <= t)
                lo = mid;
            else
                hi = mid - 1;
        }
        const int h = (l * a.B + lo) * a.Hkv + g;
        const int before = a.before[h], r = before + t - cu[lo], p = r / a.P, had = pages_of(before, a.P);
        const int page = p < had ? a.table[(int64_t)h * a.max_pages + p] : a.free_pages[head.count - 1 - a.first[h] - (p - had)];
        a.slots[((int64_t)l * a.max_tokens + t) * a.Hkv + g] = page * a.P + r % a.P;
    }
}

// ---------------------------------------------------------------- prune-and-pack into pages
// pool[row(h, len_h - n_h + r)] = K[h'][idx[ioff[h'] + r]] for the n_h kept rows of plan slab h'
// = (l, i, g) and pool slab h = (l, seq[i], g); the same for V. A copy of bytes, as
// compact_kernel: a half-warp moves a 256-byte row, 8 rows a warp, all loads before the stores.
constexpr int kPcThreads = 256;
constexpr int kPcPairs = 4;
constexpr int kPcRows = 2 * kPcPairs * (kPcThreads / 32);  // rows a CTA

__global__ void __launch_bounds__(kPcThreads) page_compact_kernel(const PageCompactArgs a)
{
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, half = lane >> 4, sub = lane & 15;
    const int64_t r0 = ((int64_t)blockIdx.x * (kPcThreads / 32) + warp) * (2 * kPcPairs);
    if (r0 >= a.plan.kept) return;
    const int NH = a.plan.L * a.plan.B * a.plan.Hkv;
    int lo = 0, hi = NH - 1;  // the last slab with ioff <= r0
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (a.plan.ioff[mid] <= r0)
            lo = mid;
        else
            hi = mid - 1;
    }
    uint4 kv[kPcPairs], vv[kPcPairs];
    int64_t dst[kPcPairs];
#pragma unroll
    for (int i = 0; i < kPcPairs; ++i) {
        const int64_t row = r0 + 2 * i + half;
        dst[i] = -1;
        if (row < a.plan.kept) {
            int hr = lo;
            while (a.plan.ioff[hr + 1] <= row) ++hr;
            const int64_t n0 = a.plan.ioff[hr], n = a.plan.ioff[hr + 1] - n0;
            const int s = hr / a.plan.Hkv % a.plan.B, l = hr / (a.plan.Hkv * a.plan.B);
            const int b = a.seq ? a.seq[s] : s;
            const int32_t ix = a.plan.idx[row];
            bool ok = b >= 0 && b < a.B && ix >= 0 && ix < a.T_stride;
            if (ok) {
                const int64_t h = ((int64_t)l * a.B + b) * a.plan.Hkv + hr % a.plan.Hkv;
                const int64_t pos = a.len[h] - n + (row - n0);
                ok = pos >= 0 && pos < (int64_t)a.max_pages * a.P;
                const int page = ok ? a.table[h * a.max_pages + pos / a.P] : -1;
                ok = page >= 0 && page < a.num_pages;
                if (ok) dst[i] = (int64_t)page * a.P + pos % a.P;
            }
            if (!ok) {
                if (sub == 0 && a.status) atomicOr(a.status, kDevRange);
                continue;
            }
            const int64_t src = ((int64_t)hr * a.T_stride + ix) * kHeadDim;
            kv[i] = __ldcs(reinterpret_cast<const uint4*>(a.K + src) + sub);
            vv[i] = __ldcs(reinterpret_cast<const uint4*>(a.V + src) + sub);
        }
    }
#pragma unroll
    for (int i = 0; i < kPcPairs; ++i)
        if (dst[i] >= 0) {
            __stcs(reinterpret_cast<uint4*>(a.Kp + dst[i] * kHeadDim) + sub, kv[i]);
            __stcs(reinterpret_cast<uint4*>(a.Vp + dst[i] * kHeadDim) + sub, vv[i]);
        }
}

}  // namespace

cudaError_t page_setup(int* sms)
{
    struct Known {
        unsigned long long context;
        int sms;
    };
    constexpr int kMost = 64;  // contexts; later ones are looked up on every call
    static std::mutex mu;
    static Known known[kMost];
    static int count = 0;
    unsigned long long id = 0;
    cudaError_t e = current_context_id(&id);
    if (e != cudaSuccess) return e;
    std::lock_guard<std::mutex> lock(mu);
    for (int i = 0; i < count; ++i)
        if (known[i].context == id) {
            *sms = known[i].sms;
            return cudaSuccess;
        }
    int dev = 0;
    if ((e = cudaGetDevice(&dev)) != cudaSuccess) return e;
    if ((e = cudaDeviceGetAttribute(sms, cudaDevAttrMultiProcessorCount, dev)) != cudaSuccess) return e;
    if ((e = chunk_setup()) != cudaSuccess) return e;
    if (count < kMost) known[count++] = Known{id, *sms};
    return cudaSuccess;
}

cudaError_t launch_page_tables(const PageArgs& a, cudaStream_t st)
{
    int sms = 0;
    cudaError_t e = page_setup(&sms);
    if (e != cudaSuccess) return e;
    if ((e = launch_pdl(page_scan_kernel, 1, kScanThreads, 0, st, a)) != cudaSuccess) return e;
    return launch_pdl(page_fill_kernel, 4 * sms, kFillThreads, 0, st, a);
}

cudaError_t launch_page_compact(const PageCompactArgs& a, cudaStream_t st)
{
    if (a.plan.kept == 0) return cudaSuccess;
    page_compact_kernel<<<(unsigned)((a.plan.kept + kPcRows - 1) / kPcRows), kPcThreads, 0, st>>>(a);
    return cudaGetLastError();
}

}  // namespace dkv
