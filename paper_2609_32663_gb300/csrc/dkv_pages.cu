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
// The whole call needs the scan of all slabs' page counts, and every CTA its part of it. Up to
// kFusedSlabs slabs each CTA scans them all itself (64 KB through L2 at 16,384 slabs, 2-3 us) into
// shared memory and then fills its share: one launch and 6.9 us for a step of 4,096 slabs, where a
// scan kernel and a fill kernel behind it took 12.4. Lengths and counts that are updated in place
// are committed by a second, tiny launch (1.2 us), as CTAs may still be reading them. More slabs: one
// CTA scans into the workspace, then all fill.
// Lengths, counts and slots are checked in the scan: nothing is written if a check fails or the free list is
// too short. The page numbers themselves are looked at where they move: one that is out of range is reported,
// and -1 (no page) moves in its place, so that no table, list or slot map ever leads out of the pools.
//
// What bounds it: the launch and the scan for a decode step (4.4 us of its 6.9); instructions more than bytes for
// the large calls: 12.8 M pages given back, 103 MB, in 29.3 us, of which launch and scan take 8.5 and chunks that hold
// several slabs 4; 256 K pages and 4.1 M slots, 17.7 MB, in 12.2 us.
#include "dkv_decode_common.cuh"
#include "dkv_pages.cuh"
#include "dkv_pool.cuh"

#include <algorithm>
#include <mutex>

namespace dkv {
namespace {

constexpr int kThreads = 1024;
constexpr int kFusedSlabs = 48 * 1024;  // prefix sums in shared memory: 192 KB
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
    int64_t w = sh[lane];
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int64_t y = __shfl_up_sync(kFull, w, o);
        if (lane >= o) w += y;
    }
    *total = __shfl_sync(kFull, w, 31);
    const int64_t before = __shfl_sync(kFull, w, (warp + 31) & 31);
    return v - x + (warp ? before : 0);
}

// rows: at most max_pages * P, which the host keeps to 2^31 - 256.
__device__ __forceinline__ int pages_of(const PageArgs& a, int rows) { return (rows + a.P - 1) >> a.log_P; }

// A slab's place, moved on without divisions.
struct Slab {
    int l, b, g;
    __device__ __forceinline__ void at(const PageArgs& a, int h)
    {
        const int lb = h / a.Hkv;
        g = h - lb * a.Hkv;
        l = lb / a.B;
        b = lb - l * a.B;
    }
    __device__ __forceinline__ void carry(const PageArgs& a)
    {
        while (b >= a.B) {
            b -= a.B;
            ++l;
        }
    }
    __device__ __forceinline__ void next(const PageArgs& a)
    {
        if (++g == a.Hkv) {
            g = 0;
            ++b;
            carry(a);
        }
    }
    // 128 slabs on (a.skip_b slots and a.skip_g heads).
    __device__ __forceinline__ void skip(const PageArgs& a)
    {
        b += a.skip_b;
        g += a.skip_g;
        if (g >= a.Hkv) {
            g -= a.Hkv;
            ++b;
        }
        carry(a);
    }
    // Rows that the slab gains (grow; negative: out of range), or whether it ends (release).
    // per_slot: new tokens, ended flags or the plan's sequence (-1: none) of each slot.
    __device__ __forceinline__ int rows(const PageArgs& a, const int32_t* per_slot) const
    {
        const int x = per_slot[b];
        if (a.mode != kGrowPlan) return x;
        return x < 0 ? 0 : a.plan_len[((int64_t)l * a.planB + x) * a.Hkv + g];
    }
};

// Pages that a slab of len rows takes (n new rows) or gives back (n: it ends).
__device__ __forceinline__ int slab_pages(const PageArgs& a, int len, int n)
{
    if (a.mode == kRelease) return n ? pages_of(a, len) : 0;
    return pages_of(a, len + n) - pages_of(a, len);
}

__device__ __forceinline__ int slab_after(const PageArgs& a, int len, int n)
{
    return a.mode == kRelease ? (n ? 0 : len) : len + n;
}

struct ScanShared {
    int64_t sums[32];
    int32_t per_slot[kMaxSlots];
    int32_t cu[kMaxSlots + 1];
    int bad;
};

// One CTA's scan of all slabs: first[h] = pages of the slabs before h. Returns whether all is in
// range; then *head and, in token mode, sh->cu hold. Reads nothing that a commit writes after it.
__device__ __forceinline__ bool scan_slabs(const PageArgs& a, ScanShared* sh, int32_t* first, PageHead* head)
{
    const int tid = threadIdx.x;
    if (tid == 0) sh->bad = 0;
    // A contiguous piece of the slabs a warp, 128 at a time, four neighbours a lane; the first
    // lengths are on their way at once.
    const int lane = tid & 31, warp = tid >> 5, per = (a.NH + 128 * (kThreads / 32) - 1) / (128 * (kThreads / 32)) * 128;
    const int h0 = (int)min((int64_t)a.NH, (int64_t)warp * per), h1 = (int)min((int64_t)a.NH, (int64_t)h0 + per);
    int lens[4];
    auto fetch = [&](int h) {
#pragma unroll
        for (int i = 0; i < 4; ++i) lens[i] = h + i < h1 ? a.len[h + i] : 0;
    };
    fetch(h0 + 4 * lane);
    const int count = *a.free_count;
    for (int b = tid; b < a.B; b += kThreads) sh->per_slot[b] = a.mode == kGrowPlan ? -1 : a.tokens[b];
    __syncthreads();
    int flags = 0;
    if (a.mode == kGrowPlan) {
        for (int i = tid; i < a.planB; i += kThreads) {
            const int b = a.seq ? a.seq[i] : i;
            if (b < 0 || b >= a.B || (a.seq && i > 0 && a.seq[i - 1] >= b))
                flags |= kDevRange;  // slots ascend, so that no slot is named twice
            else
                sh->per_slot[b] = i;
        }
        __syncthreads();
    }
    if (a.mode == kGrowTokens && warp == kThreads / 32 - 1) {
        // The last warp scans the tokens.
        int64_t sum = 0;
        for (int b0 = 0; b0 < a.B; b0 += 32) {
            const int n = b0 + lane < a.B ? sh->per_slot[b0 + lane] : 0;
            if (n < 0) flags |= kDevRange;
            int64_t up = max(n, 0);
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int64_t y = __shfl_up_sync(kFull, up, o);
                if (lane >= o) up += y;
            }
            if (b0 + lane < a.B) sh->cu[b0 + lane + 1] = (int)min(sum + up, (int64_t)INT32_MAX);
            sum += __shfl_sync(kFull, up, 31);
        }
        if (lane == 0) sh->cu[0] = 0;
        if (sum > (a.slots ? a.max_tokens : (int64_t)INT32_MAX)) flags |= kDevRange;
    }
    const int cap = a.max_pages << a.log_P;
    int64_t mine = 0;  // this lane's pages; `run`: the warp's so far (32 bits do: it is used only if the sum fits)
    int run = 0;
    const bool quads = a.Hkv % 4 == 0;
    Slab s;
    s.at(a, h0 + 4 * lane);
#pragma unroll 1
    for (int h = h0; h < h1; h += 128) {
        const int x = h + 4 * lane;
        int v[4], sum = 0;
        Slab one = s;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int len = lens[i];
            v[i] = sum;
            if (x + i < h1) {
                const int n = one.rows(a, sh->per_slot);
                if (len < 0 || len > cap || (a.mode != kRelease && (n < 0 || n > cap - len)))
                    flags |= kDevRange;
                else
                    sum += slab_pages(a, len, n);
            }
            if (quads)
                ++one.g;  // four neighbours of one slot
            else
                one.next(a);
        }
        s.skip(a);
        if (h + 128 < h1) fetch(x + 128);
        mine += sum;  // four slabs: at most 2^29
        int up = sum;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int y = __shfl_up_sync(kFull, up, o);
            if (lane >= o) up += y;
        }
        const int before = run + up - sum;
        if (x + 3 < h1)
            *reinterpret_cast<int4*>(first + x) = make_int4(before + v[0], before + v[1], before + v[2], before + v[3]);
        else
            for (int i = 0; x + i < h1; ++i) first[x + i] = before + (i == 0 ? v[0] : i == 1 ? v[1] : v[2]);
        run += __shfl_sync(kFull, up, 31);
    }
#pragma unroll
    for (int o = 16; o >= 1; o >>= 1) mine += __shfl_xor_sync(kFull, mine, o);
    int64_t pages;
    const int64_t at = block_scan(lane == 31 ? mine : 0, sh->sums, &pages);
    if (count < 0 || count > a.num_pages)
        flags |= kDevRange;
    else if (a.mode == kRelease ? count + pages > a.num_pages : pages > count)
        flags |= a.mode == kRelease ? kDevRange : kDevExhausted;
    if (flags) atomicOr(&sh->bad, flags);
    const int base = __shfl_sync(kFull, (int)at, 0);  // pages of the warps before
    for (int h = h0 + lane; h < h1; h += 32) first[h] += base;
    __syncthreads();
    *head = PageHead{sh->bad == 0, count, a.mode == kGrowTokens ? sh->cu[a.B] : 0, (int)pages};
    return sh->bad == 0;
}

// What one CTA of the call writes besides pages and slots: status, token offsets, counts.
__device__ __forceinline__ void write_totals(const PageArgs& a, const ScanShared* sh, const PageHead& head, int32_t* new_count)
{
    const int tid = threadIdx.x;
    if (a.cu)
        for (int b = tid; b <= a.B; b += kThreads) a.cu[b] = head.ok ? sh->cu[b] : 0;
    if (tid == 0) {
        if (!head.ok && a.status) atomicOr(a.status, sh->bad);
        *new_count = !head.ok ? head.count : a.mode == kRelease ? head.count + head.pages : head.count - head.pages;
    }
}

// A load that stays ahead of what follows it (volatile).
__device__ __forceinline__ int load_now(const int32_t* p)
{
    int v;
    asm volatile("ld.global.s32 %0, [%1];" : "=r"(v) : "l"(p));
    return v;
}

// Whether all N page numbers that move are in range; if not, those that are none become -1 (reported). A
// compare of the largest: 12.8 M pages given back take 29.3 us (28.6 without any look, 31.4 with one at each),
// 4.1 M slots 12.2 (11.6, 14.7).
template <int N>
__device__ __forceinline__ bool pages_hold(const PageArgs& a, int (&page)[N])
{
    unsigned most = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) most = max(most, (unsigned)page[i]);
    if (most < (unsigned)a.num_pages) return true;
#pragma unroll
    for (int i = 0; i < N; ++i)
        if ((unsigned)page[i] >= (unsigned)a.num_pages) page[i] = -1;
    if (a.status) atomicOr(a.status, kDevRange);
    return false;
}

// Bounds-checked build: whether entries [e, e + n) are a slab's, and places [x, x + n) the free list's.
__device__ __forceinline__ bool entries_hold(const PageArgs& a, int h, int e, int n)
{
    return in_bounds(h >= 0 && h < a.NH && e >= 0 && n <= a.max_pages - e, a.status);
}
__device__ __forceinline__ bool list_holds(const PageArgs& a, int x, int n) { return in_bounds(x >= 0 && n <= a.num_pages - x, a.status); }

// For N values j[]: the last slab h in [lo, hi] with first[h] <= j, the one that page j belongs to.
template <int N>
__device__ __forceinline__ void slabs_of_pages(const int32_t* first, int lo, int hi, const int (&j)[N], int (&h)[N])
{
#pragma unroll
    for (int i = 0; i < N; ++i) h[i] = lo;
    int step = 1;
    while (step <= hi - lo) step <<= 1;
#pragma unroll 1
    for (step >>= 1; step >= 1; step >>= 1)
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (h[i] + step <= hi && first[min(h[i] + step, hi)] <= j[i]) h[i] += step;
}

// The same for one value, all lanes of a warp together: 32 probes a round.
__device__ __forceinline__ int slab_of_page(const int32_t* first, int NH, int j)
{
    const int lane = threadIdx.x & 31;
    int lo = 0, n = NH;  // in [lo, lo + n)
    while (n > 1) {
        const int step = (n + 31) >> 5, x = lane * step;
        const int k = 31 - __clz(__ballot_sync(kFull, x < n && first[lo + x] <= j) | 1u);
        lo += k * step;
        n = min(step, n - k * step);
    }
    return lo;
}

// Pages c0 + 32 i + lane (i < N; up to `end`) of the call, of slabs ha .. hb (one warp).
template <int N>
__device__ __forceinline__ void fill_pages(const PageArgs& a, const PageHead& head, const int32_t* first, const int32_t* len, int c0, int end, int ha, int hb)
{
    const int lane = threadIdx.x & 31;
    int j[N], h[N], page[N];
#pragma unroll
    for (int i = 0; i < N; ++i) j[i] = min(end - 1, c0 + 32 * i + lane);
    slabs_of_pages(first, ha, hb, j, h);
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int k = j[i] - first[h[i]];
        if (!entries_hold(a, h[i], a.mode == kRelease ? k : pages_of(a, len[h[i]]) + k, 1) ||
            !list_holds(a, a.mode == kRelease ? head.count + j[i] : head.count - 1 - j[i], 1))
            return;
    }
#pragma unroll
    for (int i = 0; i < N; ++i)
        page[i] = a.mode == kRelease ? a.table[(int64_t)h[i] * a.max_pages + (j[i] - first[h[i]])] : a.free_pages[head.count - 1 - j[i]];
    pages_hold(a, page);
#pragma unroll
    for (int i = 0; i < N; ++i) {
        if (c0 + 32 * i + lane >= end) continue;
        if (a.mode == kRelease)
            a.free_pages[head.count + j[i]] = page[i];
        else
            a.table[(int64_t)h[i] * a.max_pages + pages_of(a, len[h[i]]) + (j[i] - first[h[i]])] = page[i];
    }
}

constexpr int kLong = 8;  // pages of a lane on their way at once in a run of one slab

// Chunk after chunk of 32 kLong pages (one warp): a run of one slab, as most are when there are so
// many pages, is copied as it is.
__device__ __forceinline__ void fill_chunks(const PageArgs& a, const PageHead& head, const int32_t* first, const int32_t* len, int64_t c0, int64_t stride)
{
    const int lane = threadIdx.x & 31;
#pragma unroll 1
    for (; c0 < head.pages; c0 += stride) {
        const int j0 = (int)c0, end = (int)min((int64_t)head.pages, c0 + 32 * kLong);
        const int ha = slab_of_page(first, a.NH, j0);
        if (ha + 1 < a.NH && first[ha + 1] < end) {
            const int hb = ha + slab_of_page(first + ha, a.NH - ha, end - 1);
            fill_pages<kLong>(a, head, first, len, j0, end, ha, hb);
            continue;
        }
        if (!entries_hold(a, ha, j0 - first[ha] + (a.mode == kRelease ? 0 : pages_of(a, len[ha])), end - j0) ||
            !list_holds(a, a.mode == kRelease ? head.count + j0 : head.count - end, end - j0))
            continue;
        const int32_t* from = a.mode == kRelease ? a.table + ((int64_t)ha * a.max_pages + (j0 - first[ha])) : a.free_pages + (head.count - 1 - j0);
        int32_t* to = a.mode == kRelease ? a.free_pages + head.count + j0 : a.table + ((int64_t)ha * a.max_pages + pages_of(a, len[ha]) + (j0 - first[ha]));
        const int step = a.mode == kRelease ? 1 : -1, n = end - j0;
        int page[kLong];
#pragma unroll
        for (int i = 0; i < kLong; ++i) page[i] = 32 * i + lane < n ? load_now(from + step * (32 * i + lane)) : 0;
        pages_hold(a, page);
#pragma unroll
        for (int i = 0; i < kLong; ++i)
            if (32 * i + lane < n) to[32 * i + lane] = page[i];
    }
}

// a / b of numbers that are not negative; in 32 bits where they fit.
__device__ __forceinline__ int64_t quotient(int64_t a, int64_t b)
{
    return ((a | b) >> 32) == 0 ? (int64_t)((uint32_t)a / (uint32_t)b) : a / b;
}

// Slot map [L][t][Hkv], V neighbouring heads a lane. A warp takes a contiguous piece of the map, a unit of 32 / (Hkv / V)
// tokens (of one token's 32 V heads, where it has more) after the other, and looks sequence, lengths and
// scan up again only where they change (all of it for each entry: 14.3 us instead of the 11.6 before pages were looked at, for 4.1 M
// entries). Pages that this call takes are read from the free list: their table entries may not be
// written yet.
template <int V>
__device__ __forceinline__ void fill_slots(const PageArgs& a, const PageHead& head, const int32_t* first, const int32_t* len, const int32_t* cu, int warp, int warps)
{
    const int lane = threadIdx.x & 31, row = a.Hkv / V, width = min(row, 32), per = 32 / width, parts = (row + 31) / 32;
    const int groups = (int)(((uint32_t)head.total + per - 1) / per);
    const int64_t per_layer = (int64_t)groups * parts, units = per_layer * a.L;
    const int64_t each = quotient(units, warps), more = units - each * warps;  // `more` warps take one unit more
    const int count = (int)each + (warp < more);
    if (count == 0) return;
    const int64_t u0 = each * warp + min((int64_t)warp, more);
    int l = (int)quotient(u0, per_layer);
    const int64_t rest = u0 - l * per_layer;
    int group = (int)quotient(rest, parts), part = (int)(rest - (int64_t)group * parts);
    const int tk = lane / width, sub = lane - tk * width;
    int until = 0;  // the tokens that what follows holds for end here
    int shift[V], had[V], from_free[V];  // row of token t; pages before the call; place of page p in the free list, less p
    const int32_t* table = nullptr;
#pragma unroll 1
    for (int n = 0; n < count; ++n) {
        const uint32_t place = (uint32_t)group * per + tk;
        const int t = (int)place, x = part * 32 + sub;
        if (tk < per && place < (uint32_t)head.total && x < row) {
            const int g = x * V;
            if (t >= until) {
                int lo = 0, hi = a.B - 1;  // the last sequence that starts at t or before
                while (lo < hi) {
                    const int mid = (lo + hi + 1) >> 1;
                    if (cu[mid] <= t)
                        lo = mid;
                    else
                        hi = mid - 1;
                }
                until = parts == 1 ? cu[lo + 1] : 0;
                const int h = (l * a.B + lo) * a.Hkv + g;
                table = a.table + (int64_t)h * a.max_pages;
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const int before = len[h + i];
                    shift[i] = before - cu[lo];
                    had[i] = pages_of(a, before);
                    from_free[i] = head.count - 1 - first[h + i] + had[i];
                }
            }
            int page[V], slot[V];
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const int r = shift[i] + t, p = r >> a.log_P;
                const int32_t* from = p < had[i] ? table + ((int64_t)i * a.max_pages + p) : a.free_pages + (from_free[i] - p);
                const bool there = p < had[i] ? entries_hold(a, l * a.B * a.Hkv + g + i, p, 1) : list_holds(a, from_free[i] - p, 1);
                page[i] = there ? *from : -1;
                slot[i] = (int)((unsigned)page[i] << a.log_P) + (r & (a.P - 1));
            }
            if (!pages_hold(a, page))
#pragma unroll
                for (int i = 0; i < V; ++i)
                    if (page[i] < 0) slot[i] = -1;
            int32_t* to = a.slots + ((int64_t)l * a.max_tokens + t) * a.Hkv + g;
            if (!in_bounds(l < a.L && t < a.max_tokens && g + V <= a.Hkv, a.status))
                ;
            else if (V == 4)
                *reinterpret_cast<int4*>(to) = make_int4(slot[0], slot[1 % V], slot[2 % V], slot[3 % V]);
            else
                to[0] = slot[0];
        }
        if (++part == parts) {
            part = 0;
            if (++group == groups) {
                group = 0;
                ++l;
                until = 0;
            }
        }
    }
}

// This CTA's share of the table entries (or of the free list's) and of the slot map. first: the
// scan (shared or global); len: rows of the slabs before the call; cu: token offsets.
__device__ __forceinline__ void fill(const PageArgs& a, const PageHead& head, const int32_t* first, const int32_t* len, const int32_t* cu)
{
    const int warps = gridDim.x * (kThreads / 32), warp = (threadIdx.x >> 5) * gridDim.x + blockIdx.x;
    if (a.slots) {
        const int w = warps - 1 - warp;  // a small call's slots from the last warp on, its pages from the first: 6.9 us against 7.8
        if (a.slot_vec == 4)
            fill_slots<4>(a, head, first, len, cu, w, warps);
        else
            fill_slots<1>(a, head, first, len, cu, w, warps);
    }
    // One page a lane while that is enough (latency counts). Chunks of neighbouring warps lie side by side:
    // a contiguous piece a warp took 37 us where this took 28.5, for the release of 12.8 M pages.
    if (head.pages > warps * 32)
        fill_chunks(a, head, first, len, (int64_t)warp * 32 * kLong, (int64_t)warps * 32 * kLong);
    else if (warp * 32 < head.pages)
        fill_pages<1>(a, head, first, len, warp * 32, head.pages, 0, a.NH - 1);
}

// The whole call. new_len: the caller's, or the workspace's where that is len itself (then
// page_commit_kernel follows); new_count the same.
__global__ void __launch_bounds__(kThreads, 1) page_fused_kernel(const __grid_constant__ PageArgs a, int32_t* new_len, int32_t* new_count)
{
    extern __shared__ __align__(16) int32_t first[];
    __shared__ ScanShared sh;
    pdl_wait();
    pdl_launch_dependents();
    PageHead head;
    const bool ok = scan_slabs(a, &sh, first, &head);
    if (blockIdx.x == 0) write_totals(a, &sh, head, new_count);
    if (ok) fill(a, head, first, a.len, sh.cu);
    for (int h = blockIdx.x * kThreads + threadIdx.x; h < a.NH; h += gridDim.x * kThreads) {
        Slab s;
        s.at(a, h);
        const int len = a.len[h];
        new_len[h] = ok ? slab_after(a, len, s.rows(a, sh.per_slot)) : len;
    }
}

__global__ void __launch_bounds__(kThreads) page_commit_kernel(const __grid_constant__ PageArgs a, const int32_t* from_len, const int32_t* from_count)
{
    pdl_wait();
    const int h = blockIdx.x * kThreads + threadIdx.x;
    if (a.new_len != from_len && h < a.NH) a.new_len[h] = from_len[h];
    if (h == 0 && a.new_count != from_count) *a.new_count = *from_count;
}

// Many slabs: one CTA scans into the workspace and writes lengths and counts; then all fill.
__global__ void __launch_bounds__(kThreads, 1) page_scan_kernel(const __grid_constant__ PageArgs a)
{
    __shared__ ScanShared sh;
    pdl_wait();
    pdl_launch_dependents();
    PageHead head;
    const bool ok = scan_slabs(a, &sh, a.first, &head);
    write_totals(a, &sh, head, a.new_count);
    if (threadIdx.x == 0) *a.head = head;
    for (int h = threadIdx.x; h < a.NH; h += kThreads) {
        Slab s;
        s.at(a, h);
        const int len = a.len[h];
        a.before[h] = len;
        a.new_len[h] = ok ? slab_after(a, len, s.rows(a, sh.per_slot)) : len;
    }
}

__global__ void __launch_bounds__(kThreads, 1) page_fill_kernel(const __grid_constant__ PageArgs a)
{
    __shared__ int32_t cu[kMaxSlots + 1];
    pdl_wait();
    const PageHead head = *a.head;
    if (!head.ok) return;
    if (a.slots)
        for (int b = threadIdx.x; b <= a.B; b += kThreads) cu[b] = a.cu[b];
    __syncthreads();
    fill(a, head, a.first, a.before, cu);
}

// ---------------------------------------------------------------- prune-and-pack into pages
// pool[row(h, len_h - n_h + r)] = K[h'][idx[ioff[h'] + r]] for the n_h kept rows of plan slab h'
// = (l, i, g) and pool slab h = (l, seq[i], g); the same for V. A copy of bytes, bound by HBM.
//
// A warp takes a contiguous piece of the kept rows, 32 at a time, one row's places a lane. Kept
// rows come in runs (a bin's positions, a window's) and pages are runs too, so a group is few
// segments whose source and destination are both contiguous: one bulk copy into shared memory
// and one out again for each, no data through registers. Two groups a warp (16 KB each, K and V) are
// on their way, 192 KB an SM. 16K prompt,
// 32 layers: 265 us, 6.3 TB/s of the 6.8 of a plain copy (rows through registers, a warp 8 rows with
// the look-ups of each: 299).
constexpr int kPcWarps = 6;
constexpr int kPcSlots = 2;
constexpr int kPcSlotBytes = 2 * 32 * kRowBytes;  // 32 rows of K, then of V
constexpr int kPcSmem = kPcWarps * kPcSlots * kPcSlotBytes;

__device__ __forceinline__ void bulk_s2g(void* dst, uint32_t src, uint32_t bytes)
{
    asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;" ::"l"(dst), "r"(src), "r"(bytes) : "memory");
}

// The last slab h with ioff[h] <= row (one warp: 32 probes a round).
__device__ __forceinline__ int slab_of_row(const int64_t* ioff, int NH, int64_t row)
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

__global__ void __launch_bounds__(kPcWarps * 32, 1) page_compact_kernel(const __grid_constant__ PageCompactArgs a, int64_t rows_per_warp)
{
    extern __shared__ __align__(128) unsigned char buffer[];
    __shared__ uint64_t landed[kPcWarps][kPcSlots];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int64_t first = ((int64_t)blockIdx.x * kPcWarps + warp) * rows_per_warp, end = min(a.plan.kept, first + rows_per_warp);
    if (first >= end) return;
    const int NH = a.plan.L * a.plan.B * a.plan.Hkv;
    if (lane < kPcSlots) mbar_init(smem_u32(&landed[warp][lane]), 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    fence_proxy_async_smem();
    __syncwarp();
    const uint64_t pol = evict_first_policy();
    const uint32_t base = smem_u32(buffer) + warp * kPcSlots * kPcSlotBytes;
    // The lane's slab: its kept rows end at n1; row r lies at position r + shift of its pool slab.
    int hr = slab_of_row(a.plan.ioff, NH, first) - 1;
    int64_t n1 = first, shift = 0, entries = 0;  // (no slab yet)
    bool ok = true, slot_ok = true;
    int32_t next = first + lane < end ? a.plan.idx[first + lane] : 0;
    // The group before this one, waiting for its rows: the lane's segment (0 rows: none).
    int seg = 0;
    int64_t seg_to = 0;
#pragma unroll 1
    for (int it = 0; ok; ++it) {
        const int64_t r0 = first + (int64_t)it * 32, r = r0 + lane;
        const bool more = r0 < end;
        int rows = 0;
        int64_t from = -2 - 2 * lane, to = from;  // no neighbour of another lane's
        const uint32_t slot = base + (it & 1) * kPcSlotBytes;
        if (more) {
            const int32_t ix = next;
            if (r + 32 < end) next = a.plan.idx[r + 32];
            if (r < end) {
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
                    atomicOr(a.status, kDevRange);
                }
            }
            // Segments: a lane that does not continue the one before it starts a segment.
            const int64_t f0 = __shfl_up_sync(kFull, from, 1), t0 = __shfl_up_sync(kFull, to, 1);
            const bool starts = lane == 0 || from < 0 || f0 + 1 != from || t0 + 1 != to;
            const unsigned heads = __ballot_sync(kFull, starts), valid = __ballot_sync(kFull, from >= 0);
            if (starts && from >= 0) {
                const unsigned later = lane == 31 ? 0u : heads >> (lane + 1);
                rows = later ? __ffs(later) : 32 - lane;
            }
            // The slot's copies out, of two groups ago (the latest that were issued), have read it.
            static_assert(kPcSlots == 2, "else not all copies out need have read");
            asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
            __syncwarp();
            const uint32_t bar = smem_u32(&landed[warp][it & 1]);
            if (lane == 0) mbar_arrive_expect_tx(bar, __popc(valid) * 2 * kRowBytes);
            __syncwarp();
            if (rows > 0) {
                bulk_g2s(slot + lane * kRowBytes, a.K + from * kHeadDim, rows * kRowBytes, bar, pol);
                bulk_g2s(slot + 32 * kRowBytes + lane * kRowBytes, a.V + from * kHeadDim, rows * kRowBytes, bar, pol);
            }
        }
        if (it > 0) {
            const uint32_t before = base + ((it - 1) & 1) * kPcSlotBytes;
            ok = __all_sync(kFull, mbar_wait(smem_u32(&landed[warp][(it - 1) & 1]), ((it - 1) >> 1) & 1));
            if (ok && seg > 0) {
                bulk_s2g(a.Kp + seg_to * kHeadDim, before + lane * kRowBytes, seg * kRowBytes);
                bulk_s2g(a.Vp + seg_to * kHeadDim, before + 32 * kRowBytes + lane * kRowBytes, seg * kRowBytes);
            }
        }
        asm volatile("cp.async.bulk.commit_group;" ::: "memory");
        if (!more) break;
        seg = rows;
        seg_to = to;
    }
    if (!ok) {
        if (lane == 0 && a.status) atomicOr(a.status, DKV_DEV_TMA_TIMEOUT);
        for (int s = 0; s < kPcSlots; ++s)  // copies in flight land, or run out of time, before the CTA exits
            for (int parity = 0; parity < 2; ++parity) mbar_wait(smem_u32(&landed[warp][s]), parity);
    }
    asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
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
    if ((e = cudaFuncSetAttribute(page_fused_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kFusedSlabs * 4)) != cudaSuccess) return e;
    if ((e = cudaFuncSetAttribute(page_compact_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kPcSmem)) != cudaSuccess) return e;
    if (count < kMost) known[count++] = Known{id, *sms};
    return cudaSuccess;
}

cudaError_t launch_page_tables(const PageArgs& a, cudaStream_t st)
{
    int sms = 0;
    cudaError_t e = page_setup(&sms);
    if (e != cudaSuccess) return e;
    if (a.NH > kFusedSlabs) {
        if ((e = launch_pdl(page_scan_kernel, 1, kThreads, 0, st, a)) != cudaSuccess) return e;
        return launch_pdl(page_fill_kernel, sms, kThreads, 0, st, a);
    }
    const bool len_in_place = a.new_len == a.len, count_in_place = a.new_count == a.free_count;
    int32_t* new_len = len_in_place ? a.before : a.new_len;
    int32_t* new_count = count_in_place ? &a.head->count : a.new_count;
    if ((e = launch_pdl(page_fused_kernel, sms, kThreads, a.NH * 4, st, a, new_len, new_count)) != cudaSuccess) return e;
    if (!len_in_place && !count_in_place) return cudaSuccess;
    const int32_t *from_len = new_len, *from_count = new_count;
    return launch_pdl(page_commit_kernel, len_in_place ? (a.NH + kThreads - 1) / kThreads : 1, kThreads, 0, st, a, from_len, from_count);
}

cudaError_t launch_page_compact(const PageCompactArgs& a, cudaStream_t st)
{
    if (a.plan.kept == 0) return cudaSuccess;
    int sms = 0;
    const cudaError_t e = page_setup(&sms);
    if (e != cudaSuccess) return e;
    const int64_t groups = (a.plan.kept + 31) / 32, warps = std::min<int64_t>(groups, (int64_t)sms * kPcWarps);
    const int64_t rows_per_warp = (groups + warps - 1) / warps * 32;
    page_compact_kernel<<<(unsigned)((warps + kPcWarps - 1) / kPcWarps), kPcWarps * 32, kPcSmem, st>>>(a, rows_per_warp);
    return cudaGetLastError();
}

}  // namespace dkv
