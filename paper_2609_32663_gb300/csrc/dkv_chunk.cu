// Attention of a ragged chunk of new tokens over a paged cache: the new tokens' K and V
// rows are appended to their slabs' pages, then token i of the n new ones of sequence b
// attends, per query head, to the first len - n + i + 1 rows of its slab (causal) or to
// all len rows:  o = sum_r softmax_r(scale q.k_r) v_r.
//
// Unit of work: up to 2 TQ tokens of one sequence and KV head (TQ = 128 / G tokens x G heads
// fill a 128-row tile of queries, row = token G + head), against the cache rows that its last
// token sees, in tiles of 128 rows. All (unit, cache tile) pairs, unit after unit, are cut into
// contiguous shares of equal cost, one a CTA, one CTA an SM, so ragged lengths leave no SM idle; a
// unit that lies in several CTAs is joined by the one that finishes last.
//
//   chunk_append_kernel  appends the rows.
//   chunk_attn_kernel    starts beside it, finds its shares, and waits for the append only where a
//                        tile holds new rows. Two pipelines of S = Q K^T, softmax, O += P V, one a softmax group:
//     pair units (more than TQ tokens): group p has query tile p; both use the same K and V tile.
//     split units (decode, drafts, the rest of a turn): one query tile; group p takes the cache
//     tiles of parity p, and the groups' (m, l, O) are joined at the unit's end.
//     warps 0-3, 4-7  softmax groups; thread = query row = TMEM lane. S is read from TMEM, P goes
//                     back over it as the A operand of the second product.
//     warp 8          MMA: S(0), S(1), then PV(s), S(s + 2) of step s (group s % 2), in one order, so
//                     that the tensor pipe itself keeps S(s + 2) behind the PV(s) whose P it overwrites.
//     warp 9          TMA: Q tiles, and K and V tiles page by page into one ring in the order of use.
//     warp 10         walks the CTA's share and describes its units to the others (11 is idle).
//
// What bounds it. Next tokens stream the cache: 16 sequences of 3K-24K rows, 847 MB, in 131 us, 6.5
// TB/s of the 6.8 of a plain copy. Turns and queries: a pair unit's tile (four products, 2,048 cycles
// of the tensor pipe at its best) takes 1.52 us, 2,900 cycles. Q K^T reads both operands from shared
// memory, 8 KB a 64-cycle instruction and so the 128 B a cycle that it gives, beside the copies into
// the ring: about 630 cycles instead of 512, so the pipe is busy for 2,280. What bounds it is each
// group's chain, as TMEM holds one S a group: 950 cycles from S to the first half of P, P V and the
// next Q K^T behind it, and four hand-offs of 100 to 150 cycles. 200-777 queries over 5K-13K rows: 127.7 us, 1.24 PFLOP/s, 100 us of it in the loop;
// 4K tokens over 45K rows: 1,730 us, 1.43 PFLOP/s, 0.85 of what the library's matrix product sustains
// (1,531 us before the clocks fall under the power limit). One token over 1.8K rows: 15.1 us, all of
// it latency: two launches, the count of the cost, one tile, the join (0.3 us of it the looks at offsets and
// lengths, and the fence).
//
// Scores, their max and sum and O are fp32. The weights P are rounded to the inputs' type, as both operands of
// the second product have it: half a step of each weight, of either sign, so that errors against 64 bits go from
// the 0.0017 of the output's own rounding to 0.0019 (next tokens, queries) and 0.0021 (the turn) in bf16, from 0.00021 to
// 0.00022 in fp16. P as a high and a low part would take another P V beside each, 1,024 more cycles for a pair
// unit's 2,048.
// Two MMA warps, a group each, took 173 us for the queries where one took 137 (their products alternate on
// the pipe), four softmax warpgroups 152; stages freed by the softmax warps instead of by commits 136.
//
// Every wait is bounded (polls and 2 s), and so are the softmax warps' meetings (Waits::meet); one
// that runs out sets DKV_DEV_TMA_TIMEOUT, the roles leave, copies and products in flight are
// drained, and the outputs of the CTA's unfinished units stay unwritten.
#include "dkv_pages.cuh"
#include "dkv_tcgen05.cuh"

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cudaTypedefs.h>

#include <mutex>

namespace dkv {
namespace {

constexpr int kTile = 128;                 // query rows and cache rows of a tile
constexpr int kHalf = kTile * 128;         // one 64-dim half of a tile (16 KB)
constexpr int kOperand = 2 * kHalf;        // a tile: dims 0-63, then 64-127
constexpr int kStages = 5;                 // ring of K and V tiles
constexpr int kThreads = 384;
constexpr int kRegsSoft = 216, kRegsRest = 72;  // a thread's registers after the split; launched with 168
static_assert(2 * kRegsSoft + kRegsRest <= 3 * 168, "three warpgroups share what they were launched with");
constexpr int kSoft = 256;                 // threads of the softmax groups
constexpr int kMaxCtas = 160;              // CTAs of the largest grid (the workspace's size)
constexpr int kPieceRows = 2 * kTile;      // rows of a piece in the workspace
constexpr int kTmemCols = 512;             // S of group p at 128 p (P over its first half), O at 256 + 128 p

// Shared memory, from its 1024-byte aligned start (there is no room to align it by hand).
constexpr int kOffQ = 0;
constexpr int kOffRing = kOffQ + 2 * kOperand;
constexpr int kOffBars = kOffRing + kStages * kOperand;
constexpr int kAhead = 4;                  // ring of unit descriptors
constexpr int kNumBars = 2 * kStages + 3 * kAhead + 11;  // full[], empty[], said[], q_full[], late[], q_empty[2], s_full[2], p_half[2], p_full[2], o_done[2], fin
constexpr int kOffMisc = kOffBars + (kNumBars + 1) / 2 * 16;  // int[4]: TMEM address, abort, last
constexpr int kOffPieces = kOffMisc + 16;                      // Piece[kAhead]
constexpr int kOffMl = kOffPieces + kAhead * 64;                           // float2[128]: group 1's (m, l), then group 0's
constexpr int kSmemBytes = kOffMl + 2 * kTile * 8;
static_assert(kSmemBytes <= 227 * 1024, "fits one CTA");

// Workspace.
struct ChunkWork {
    int32_t* done;      // [kMaxCtas] finished pieces of the unit that starts in CTA c and ends in a later one
    float2* ml;         // [kMaxCtas][2][256]
    float4* o;          // [kMaxCtas][2][128 / 4][256]: a warp's rows side by side
};
constexpr int64_t kOffPieceMl = (kMaxCtas * 4 + 255) / 256 * 256, kOffPieceO = kOffPieceMl + (int64_t)kMaxCtas * 2 * kPieceRows * 8,
                  kWorkBytes = kOffPieceO + (int64_t)kMaxCtas * 2 * kPieceRows * kHeadDim * 4;

struct ChunkMaps {
    CacheMaps cache;
    CUtensorMap q;
};

__device__ __forceinline__ int cu_at(const ChunkArgs& a, int b) { return min(max(a.cu[b], 0), a.T); }

// ---------------------------------------------------------------- units
struct Unit {
    int h;       // slab
    int t0;      // first token (row of q)
    int tokens;  // 1 .. 2 TQ
    int row0;    // rows that the first token sees (causal), before the clamp to [0, len]
    int len;     // rows of the slab
    int kv;      // rows that the last token sees
    int fresh;   // rows that this call appends to the slab
    bool pair;   // two query tiles
    __device__ __forceinline__ int tiles() const { return max(1, (kv + kTile - 1) / kTile); }
};

// Rows of slab h; none if its length is out of range.
__device__ __forceinline__ int slab_len(const ChunkArgs& a, int h)
{
    const int len = a.len[h];
    return len >= 0 && len <= a.max_pages * a.P ? len : 0;  // (the product is below 2^31)
}

// Unit i of the n tokens from row t of q on, over a slab of len rows.
__device__ __forceinline__ Unit make_unit(const ChunkArgs& a, int h, int t, int n, int len, int i)
{
    const int TQ = kTile / a.G, w = 2 * TQ;
    Unit u;
    u.h = h;
    u.t0 = t + i * w;
    u.tokens = min(w, n - i * w);
    u.len = len;
    u.row0 = a.causal ? len - n + i * w + 1 : len;
    u.kv = a.causal ? max(0, u.row0 + u.tokens - 1) : len;
    u.pair = u.tokens > TQ;
    u.fresh = n;
    return u;
}

// What a cache tile costs: a pair unit's has twice the products, a split unit's waits for its rows.
// In shares of one kind a pair unit's takes 1.52 us, a split unit's 1.14, so 4 : 3, but a step of two turns and ten
// next tokens takes 308 us with 3 : 2 and 311 with 4 : 3 (queries 127.1 and 126.7, next tokens 130.4 and 130.0). With
// one weight for both, the SMs with next tokens only were done at 225 us of 320.
constexpr int kPairCost = 3, kSplitCost = 2;

// The share of one CTA, unit by unit. Units lie end to end on a line of costs; a tile is the
// CTA's in whose part of the line it starts.
struct Walk {
    int b, g, i, t, n, j0, j1, tiles;
    int64_t start, end;  // of the unit, of the share
    Unit u;
    __device__ __forceinline__ int cost() const { return kSplitCost + (int)u.pair; }
    // Tiles that start before point x of the unit (a unit costs less than 2^26).
    __device__ __forceinline__ int before(unsigned x) const
    {
        const unsigned w = cost();
        return (int)((x + w - 1) / w);
    }
    // The unit (b, g, i), its start set, from its tile at `off` behind its start.
    __device__ __forceinline__ void enter(const ChunkArgs& a, int len, int off)
    {
        u = make_unit(a, b * a.Hkv + g, t, n, len, i);
        tiles = u.tiles();
        j0 = min(tiles, before((unsigned)off));
        j1 = min(tiles, before((unsigned)min(end - start, (int64_t)1 << 28)));
    }
    __device__ __forceinline__ bool more() const { return j1 == tiles && start + tiles * cost() < end; }
    __device__ __forceinline__ void next(const ChunkArgs& a)
    {
        start += tiles * cost();
        if (++i * 2 * (kTile / a.G) >= n) {
            i = 0;
            if (++g == a.Hkv) {
                g = 0;
                do ++b;
                while (b < a.B - 1 && cu_at(a, b + 1) <= cu_at(a, b));
                t = cu_at(a, b);
                n = cu_at(a, b + 1) - t;
            }
        }
        enter(a, slab_len(a, b * a.Hkv + g), 0);
    }
    __device__ __forceinline__ bool whole() const { return j0 == 0 && j1 == tiles; }
};

// What the other roles need of a CTA's part of a unit, described by the walking warp.
struct alignas(16) Piece {
    int t0, tokens, row0, len;  // as in Unit
    int kv, h, g, j0;
    int j1, flags, fresh, pad0;
    int c0, pieces, pad1, pad2;  // CTAs c0 .. c0 + pieces - 1 hold the unit (written after the rest: `late`)
    static constexpr int kPair = 1, kWhole = 2, kMore = 4;
    __device__ __forceinline__ bool pair() const { return flags & kPair; }
    __device__ __forceinline__ bool whole() const { return flags & kWhole; }
    __device__ __forceinline__ bool more() const { return flags & kMore; }  // the CTA has a unit after this
    __device__ __forceinline__ int steps() const { return pair() ? 2 * (j1 - j0) : j1 - j0; }
    __device__ __forceinline__ int tile(int s) const { return j0 + (pair() ? s >> 1 : s); }
};
static_assert(sizeof(Piece) == 64, "four 16-byte words, of which read_piece reads three");

__device__ __forceinline__ Piece read_piece(const unsigned char* at)
{
    union {
        uint4 u[4];
        Piece p;
    } x;
#pragma unroll
    for (int i = 0; i < 3; ++i)
        asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];"
                     : "=r"(x.u[i].x), "=r"(x.u[i].y), "=r"(x.u[i].z), "=r"(x.u[i].w)
                     : "r"(smem_u32(at) + 16 * i)
                     : "memory");
    return x.p;
}

// The whole call: the cost of all units, and CTAs with a share of it.
struct Extent {
    int64_t cost;
    int parts;
};

// x / y of values >= 0 (most calls are small enough for the short division).
__device__ __forceinline__ int64_t divide(int64_t x, int64_t y)
{
    return x <= UINT32_MAX && y <= UINT32_MAX ? (int64_t)((uint32_t)x / (uint32_t)y) : x / y;
}

// Where share c starts, and the CTA whose share holds point x of the line.
__device__ __forceinline__ int64_t share_start(const Extent& e, int c) { return divide(e.cost * c, e.parts); }
__device__ __forceinline__ int cta_of(const Extent& e, int64_t x) { return (int)divide((x + 1) * e.parts - 1, e.cost); }

__device__ __forceinline__ void report(const ChunkArgs& a, int bits)
{
    if (a.status) atomicOr(a.status, bits);
}

// Token offsets hold if they start at 0, ascend and end within the batch; whether the pair (b, b + 1) breaks
// that. Every CTA of both kernels looks at all pairs: with one that breaks it the call does nothing (followed
// as far as they go, such offsets would lead to rows of earlier tokens).
__device__ __forceinline__ bool bad_offsets(const ChunkArgs& a, int b)
{
    const int t0 = a.cu[b], t1 = a.cu[b + 1];
    return t1 < t0 || t1 > a.T || (b == 0 && t0 != 0);
}

// ---------------------------------------------------------------- append
constexpr int kAppThreads = 512;

__global__ void __launch_bounds__(kAppThreads) chunk_append_kernel(const __grid_constant__ ChunkArgs a, const __grid_constant__ ChunkWork w)
{
    __shared__ int32_t cu[kMaxSlots + 1];
    static_assert(kMaxSlots <= kAppThreads && kMaxCtas <= kAppThreads, "one thread each");
    const int tid = threadIdx.x;
    pdl_wait();
    pdl_launch_dependents();
    if (blockIdx.x == 0) {
        // The attention kernel's counters, and the checks of what lives on the device.
        if (tid < kMaxCtas) w.done[tid] = 0;
        if (tid < a.B && bad_offsets(a, tid)) report(a, DKV_DEV_PAGE_RANGE);
        for (int h = tid; h < a.B * a.Hkv; h += kAppThreads) {
            const int b = h / a.Hkv, n = cu_at(a, b + 1) - cu_at(a, b), len = a.len[h];
            if (n > 0 && (len != slab_len(a, h) || (a.k_new && len < n))) report(a, DKV_DEV_PAGE_RANGE);
        }
        return;
    }
    const bool bad = tid < a.B && bad_offsets(a, tid);
    if (tid < a.B) cu[tid] = a.cu[tid];
    if (tid == 0) cu[a.B] = a.cu[a.B];
    // A half-warp a row (K and V).
    const int64_t i = (int64_t)(blockIdx.x - 1) * (kAppThreads / 16) + (tid >> 4);
    const int sub = tid & 15, t = (int)(i / a.Hkv), g = (int)(i - (int64_t)t * a.Hkv);
    const int64_t src = t * a.kv_stride + g * kHeadDim;
    uint4 kv, vv;
    if (t < a.T) {
        kv = __ldcs(reinterpret_cast<const uint4*>(a.k_new + src) + sub);
        vv = __ldcs(reinterpret_cast<const uint4*>(a.v_new + src) + sub);
    }
    if (__syncthreads_or(bad) || t >= cu[a.B]) return;
    int lo = 0, hi = a.B - 1;  // the last sequence that starts at t or before
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (cu[mid] <= t)
            lo = mid;
        else
            hi = mid - 1;
    }
    const int h = lo * a.Hkv + g;
    const int r = slab_len(a, h) - cu[lo + 1] + t;  // below the slab's length
    int page = -1;
    if (r >= 0 && in_bounds(h < a.B * a.Hkv && r / a.P < a.max_pages, a.status)) page = a.table[(int64_t)h * a.max_pages + r / a.P];
    if (page < 0 || page >= a.num_pages) {
        if (sub == 0) report(a, DKV_DEV_PAGE_RANGE);
        return;
    }
    const int64_t row = (int64_t)page * a.P + r % a.P;
    reinterpret_cast<uint4*>(a.Kp + row * kHeadDim)[sub] = kv;
    reinterpret_cast<uint4*>(a.Vp + row * kHeadDim)[sub] = vv;
}

// ---------------------------------------------------------------- schedule
constexpr int kMaxGroups = kStages * kOperand / 8;  // prefix sums in the ring before its first use

// Cost of a unit, and of slab h. any_pair is set if there is a pair unit.
__device__ __forceinline__ int unit_cost(const Unit& u) { return u.tiles() * (kSplitCost + (int)u.pair); }
__device__ __forceinline__ int64_t slab_cost(const ChunkArgs& a, int h, int& any_pair)
{
    const int b = h / a.Hkv, t = cu_at(a, b), n = cu_at(a, b + 1) - t, len = slab_len(a, h), TQ = kTile / a.G;
    any_pair |= n > TQ;
    int64_t sum = 0;
#pragma unroll 1
    for (int i = 0; i * 2 * TQ < n; ++i) sum += unit_cost(make_unit(a, h, t, n, len, i));
    return sum;
}

// All threads of the CTA: the cost of every slab (or group of slabs, where there are more than
// fit), summed into `before`. Every CTA does it for itself, beside the append: as a kernel's
// job in front of this one it was 2 us on the way of a small call.
__device__ __forceinline__ Extent count_cost(const ChunkArgs& a, int64_t* before, int64_t* sums, int nctas, int& group)
{
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, slabs = a.B * a.Hkv;
    group = (slabs + kMaxGroups - 1) / kMaxGroups;
    const int groups = (slabs + group - 1) / group, per = (groups + kThreads - 1) / kThreads;
    const int g0 = min(groups, tid * per), g1 = min(groups, g0 + per);
    int64_t mine = 0;
    int any_pair = 0;
#pragma unroll 1
    for (int x = g0; x < g1; ++x) {
        before[x] = mine;
#pragma unroll 1
        for (int h = x * group; h < min(slabs, (x + 1) * group); ++h) mine += slab_cost(a, h, any_pair);
    }
    int64_t up = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int64_t y = __shfl_up_sync(kFull, up, o);
        if (lane >= o) up += y;
    }
    // Whether there is a pair unit, and whether the offsets are bad, goes along in the sums' upper bits (a
    // barrier that votes, instead, cost the whole kernel 5 %). The cost itself is below 2^52: at most 2^26
    // slabs' last units and 2^23 full ones, 2^24 tiles each.
    constexpr int kFlag = 52, kBad = kFlag + 4;
    static_assert(kThreads / 32 < 16, "a field of 4 bits counts the warps");
    bool bad = false;
#pragma unroll 1
    for (int b = tid; b < a.B; b += kThreads) bad |= bad_offsets(a, b);
    const int64_t flags = (__any_sync(kFull, any_pair) ? (int64_t)1 << kFlag : 0) + (__any_sync(kFull, bad) ? (int64_t)1 << kBad : 0);
    if (lane == 31) sums[warp] = up + flags;
    __syncthreads();
    int64_t base = up - mine, total = 0;
#pragma unroll
    for (int k = 0; k < kThreads / 32; ++k) {
        if (k < warp) base += sums[k] & (((int64_t)1 << kFlag) - 1);
        total += sums[k];
    }
    const bool skip = total >> kBad;
    const int dearest = (total >> kFlag) & 15 ? kPairCost : kSplitCost;
    total &= ((int64_t)1 << kFlag) - 1;
#pragma unroll 1
    for (int x = g0; x < g1; ++x) before[x] += base;
    __syncthreads();
    if (skip) return Extent{0, 0};
    // A share is at least as long as the dearest tile, so that one starts in every share of a unit.
    static_assert(kPairCost >= kSplitCost, "the dearest tile");
    return Extent{total, total >= (int64_t)nctas * dearest ? nctas : (int)((unsigned)total / (unsigned)dearest)};
}

// Where the share of CTA c (which has one) starts.
__device__ __forceinline__ void seek(const ChunkArgs& a, const Extent& e, const int64_t* before, int group, int c, Walk& k)
{
    const int64_t pos = share_start(e, c);
    k.end = share_start(e, c + 1);
    int lo = 0, hi = (a.B * a.Hkv + group - 1) / group - 1;  // the last group that starts at `pos` or before (it has units)
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (before[mid] <= pos)
            lo = mid;
        else
            hi = mid - 1;
    }
    int64_t off = pos - before[lo];
    int h = lo * group, any = 0;
    if (group > 1)
        for (int64_t x; off >= (x = slab_cost(a, h, any)); ++h) off -= x;
    k.b = h / a.Hkv;
    k.g = h - k.b * a.Hkv;
    k.t = cu_at(a, k.b);
    k.n = cu_at(a, k.b + 1) - k.t;
    const int len = slab_len(a, h);
    k.i = 0;
#pragma unroll 1
    for (int x; off >= (x = unit_cost(make_unit(a, h, k.t, k.n, len, k.i))); ++k.i) off -= x;
    k.start = pos - off;
    k.enter(a, len, (int)off);
    if (k.j0 == k.tiles) k.next(a);  // the unit's last tile starts before this share
}

// ---------------------------------------------------------------- attention
__device__ __forceinline__ bool wait_more(uint32_t bar, uint32_t parity, volatile int* abort, int32_t* status)
{
    const unsigned long long t0 = global_ns();
    for (int i = 1; i < kWaitSpins; ++i) {
        if (mbar_try_wait(bar, parity)) return true;
        if ((i & 15) == 0 && (*abort || global_ns() - t0 > kWaitNs)) break;
    }
    if (!*abort) {
        *abort = 1;
        if (status) atomicOr(status, DKV_DEV_TMA_TIMEOUT);
    }
    return false;
}

// The drain after a wait that ran out: the phase completes, or the bound passes (in line: a warp
// whose registers were split calls no function).
__device__ __forceinline__ void land(uint64_t* bar, uint32_t parity)
{
    const unsigned long long t0 = global_ns();
    for (int i = 1; i < kWaitSpins && !mbar_try_wait(smem_u32(bar), parity); ++i)
        if ((i & 63) == 0 && global_ns() - t0 > kWaitNs) break;
}

// Bounded waits of a whole warp. After one that ran out (here or in another role) every wait
// of the CTA returns false at once.
struct Waits {
    volatile int* abort;
    int32_t* status;
    bool ok;
    bool left;  // this softmax warp goes to no further meeting
    __device__ __forceinline__ bool operator()(uint64_t* b, uint32_t parity)
    {
        if (!ok) return false;
        const uint32_t bar = smem_u32(b);
        if (__all_sync(kFull, mbar_try_wait(bar, parity))) return true;
        ok = __all_sync(kFull, wait_more(bar, parity, abort, status));
        return ok;
    }
    // All softmax warps meet at a named barrier, which has no bound: a warp whose wait ran out
    // still goes to one more meeting and says so there, to whichever the others come next (all
    // go to one after their last unit); every warp then leaves.
    __device__ __forceinline__ bool meet()
    {
        if (left) return false;
        uint32_t r;
        asm volatile(
            "{\n\t.reg .pred p, q;\n\tsetp.ne.b32 q, %1, 0;\n\t"
            "bar.red.or.pred p, 1, %2, q;\n\t"
            "selp.u32 %0, 1, 0, p;\n\t}"
            : "=r"(r)
            : "r"(ok ? 0 : 1), "n"(kSoft)
            : "memory");
        if (r) {
            ok = false;
            left = true;
        }
        return r == 0;
    }
};

template <bool F16>
__device__ __forceinline__ uint32_t pack16(float lo, float hi)
{
    if (F16) {
        const __half2 x = __floats2half2_rn(lo, hi);
        return *reinterpret_cast<const uint32_t*>(&x);
    }
    return pack_bf16(lo, hi);
}

// Zeroes rows [first, 128) of a V tile (one warp).
__device__ __forceinline__ void zero_rows(unsigned char* v, int first, int lane)
{
    for (int e = lane; e < (kTile - first) * 16; e += 32)
        *reinterpret_cast<uint4*>(v + ((e & 15) >> 3) * kHalf + (first + (e >> 4)) * 128 + (e & 7) * 16) = make_uint4(0u, 0u, 0u, 0u);
    fence_proxy_async_smem();
    __syncwarp();
}

// Two fp32 values in a register pair, one instruction for both.
__device__ __forceinline__ uint64_t pack2(float x, float y)
{
    uint64_t v;
    asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "f"(x), "f"(y));
    return v;
}
__device__ __forceinline__ void unpack2(uint64_t v, float& x, float& y) { asm("mov.b64 {%0, %1}, %2;" : "=f"(x), "=f"(y) : "l"(v)); }
__device__ __forceinline__ uint64_t fma2(uint64_t x, uint64_t y, uint64_t z)
{
    uint64_t v;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(v) : "l"(x), "l"(y), "l"(z));
    return v;
}
__device__ __forceinline__ uint64_t add2(uint64_t x, uint64_t y)
{
    uint64_t v;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(v) : "l"(x), "l"(y));
    return v;
}

// The larger of three, NaN only if all are.
__device__ __forceinline__ float max3(float x, float y, float z)
{
    float v;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(v) : "f"(x), "f"(y), "f"(z));
    return v;
}

// P of a score s is 2^(s c - origin(m, c)).
template <bool F16>
__device__ __forceinline__ float origin(float m, float c)
{
    constexpr float kShift = F16 ? 7.f : 0.f;
    return (m == -INFINITY ? 0.f : m * c) - kShift;
}

// P of 32 scores as 16 packed words; their sums are added to sum[].
template <bool F16>
__device__ __forceinline__ void exponentials(const uint32_t (&x)[32], uint64_t c2, uint64_t o2, uint32_t (&p)[16], uint64_t (&sum)[4])
{
#pragma unroll
    for (int e = 0; e < 16; ++e) {
        float p0, p1;
        unpack2(fma2(pack2(__uint_as_float(x[2 * e]), __uint_as_float(x[2 * e + 1])), c2, o2), p0, p1);
        p0 = ex2(p0);
        p1 = ex2(p1);
        sum[e & 3] = add2(sum[e & 3], pack2(p0, p1));
        p[e] = pack16<F16>(p0, p1);
    }
}

// One step of a softmax group's warp: scores of 32 query rows x 128 cache rows (TMEM columns of
// `s`) to P over them, with the running max m (of raw scores), sum l and output `o`. lim: the
// cache rows of this tile that the thread's query sees (may be outside 0 .. 128).
// The max moves only when a score tops it by 2^kSlack (then O is rescaled, so `rescale` says
// whether it holds anything): P stays below 2^kSlack. fp16 P is scaled by 2^7 more, which l shares: the
// smallest normal P is then 2^-21 of the largest score's. The first half of P is signalled alone, so that
// its products run beside the second half's exponentials (signalled at 96 of the 128 columns: 144 us
// instead of 141 for 777 queries over 13K rows; with that half computed by the old max, beside the tile's own
// max: 163 instead of 145).
template <bool F16>
__device__ __forceinline__ void softmax_step(uint32_t s, uint32_t o, int lim, bool rescale, float c, float& m, float& l, uint32_t half_bar)
{
    uint32_t x[4][32];
#pragma unroll
    for (int k = 0; k < 4; ++k) tmem_ld32_async(s + 32 * k, x[k]);
    tmem_wait_ld();
#pragma unroll
    for (int k = 0; k < 4; ++k) tmem_fence_regs(x[k]);
    if (__any_sync(kFull, lim < kTile)) {
#pragma unroll
        for (int k = 0; k < 4; ++k)
#pragma unroll
            for (int e = 0; e < 32; ++e)
                if (32 * k + e >= lim) x[k][e] = 0xff800000u;  // -inf: also over NaN
    }
    // Two warps share a scheduler, so the step is latency: independent chains for max and sum.
    float mxs[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) mxs[e] = -INFINITY;
#pragma unroll
    for (int k = 0; k < 4; ++k)
#pragma unroll
        for (int e = 0; e < 32; e += 2)
            mxs[(e >> 1) & 7] = max3(mxs[(e >> 1) & 7], __uint_as_float(x[k][e]), __uint_as_float(x[k][e + 1]));
    const float mx = max3(max3(mxs[0], mxs[1], mxs[2]), max3(mxs[3], mxs[4], mxs[5]), fmaxf(mxs[6], mxs[7]));
    const bool move = (mx - m) * c > kSlack;
    if (__any_sync(kFull, move)) {
        const float alpha = move ? ex2((m - mx) * c) : 1.f;
        if (move) m = mx;
        l *= alpha;
        if (rescale) {
#pragma unroll 1
            for (int k = 0; k < 8; ++k) {
                uint32_t v[16];
                tmem_ld16_async(o + 16 * k, v);
                tmem_wait_ld();
                tmem_fence_regs(v);
#pragma unroll
                for (int e = 0; e < 16; ++e) v[e] = __float_as_uint(__uint_as_float(v[e]) * alpha);
                tmem_st16_async(o + 16 * k, v);
            }
        }
    }
    const float mc = origin<F16>(m, c);
    const uint64_t c2 = pack2(c, c), o2 = pack2(-mc, -mc);
    uint64_t sum[4] = {0, 0, 0, 0};
    uint32_t p[16];
    exponentials<F16>(x[0], c2, o2, p, sum);
    tmem_st16_async(s, p);
    exponentials<F16>(x[1], c2, o2, p, sum);
    tmem_st16_async(s + 16, p);
    tmem_wait_st();
    tc_fence_before();
    __syncwarp();
    if ((threadIdx.x & 31) == 0) mbar_arrive(half_bar);
    exponentials<F16>(x[2], c2, o2, p, sum);
    tmem_st16_async(s + 32, p);
    exponentials<F16>(x[3], c2, o2, p, sum);
    tmem_st16_async(s + 48, p);
    float s0, s1;
    unpack2(add2(add2(sum[0], sum[1]), add2(sum[2], sum[3])), s0, s1);
    l += s0 + s1;
    tmem_wait_st();
}

// Elements 32 k .. 32 k + 31 of an output row.
template <bool F16>
__device__ __forceinline__ void store_out(uint16_t* row, const float (&v)[32], float z)
{
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        uint4 u;
        u.x = pack16<F16>(v[8 * k] * z, v[8 * k + 1] * z);
        u.y = pack16<F16>(v[8 * k + 2] * z, v[8 * k + 3] * z);
        u.z = pack16<F16>(v[8 * k + 4] * z, v[8 * k + 5] * z);
        u.w = pack16<F16>(v[8 * k + 6] * z, v[8 * k + 7] * z);
        reinterpret_cast<uint4*>(row)[k] = u;
    }
}

// Elements 32 k .. 32 k + 31 of a row of a piece (at: its element 32 k).
__device__ __forceinline__ void store_piece(float4* at, const float (&v)[32])
{
#pragma unroll
    for (int k = 0; k < 8; ++k) __stcg(at + k * kPieceRows, make_float4(v[4 * k], v[4 * k + 1], v[4 * k + 2], v[4 * k + 3]));
}

// 1 / l; a sum of 0 (no rows) gives 0, NaN stays.
__device__ __forceinline__ float inverse(float l) { return l == 0.f ? 0.f : 1.f / l; }

template <bool F16>
__device__ __forceinline__ float2 widen(uint32_t u)
{
    if (F16) return __half22float2(*reinterpret_cast<const __half2*>(&u));
    return make_float2(__uint_as_float(u << 16), __uint_as_float(u & 0xffff0000u));
}

// Pool row of row r of the unit's slab, or -1.
__device__ __forceinline__ int64_t pool_row(const ChunkArgs& a, int h, int r)
{
    if (!in_bounds(r >= 0 && r / a.P < a.max_pages, a.status)) return -1;
    const int page = a.table[(int64_t)h * a.max_pages + r / a.P];
    return page < 0 || page >= a.num_pages ? -1 : (int64_t)page * a.P + r % a.P;
}

// A value of V that is not finite, in a later token's row, spoils the rows of the same tile
// that do not see it (0 NaN is NaN). Rows whose result is not finite (`odd`) and that have
// such a value in a masked place, rows [lim, end), are computed again without the tensor cores:
// o = sum over rows [first, lim) of 2^(s - mc) v, dims [d0, d0 + nd). Slow and rare: 4 rows at
// once, 8 lanes and 16 dims a lane each.
template <bool F16>
__device__ __forceinline__ void mend_rows(const ChunkArgs& a, int h, bool odd, int first, int lim, int end, float mc, float z,
                                          const uint16_t* q, uint16_t* out, float4* piece, int d0, int nd)
{
    const int lane = threadIdx.x & 31, sub = lane & 7, dim = 16 * sub;
    const bool mine = dim >= d0 && dim < d0 + nd;
    __syncwarp();  // the rows' first results are stored
    pdl_wait();    // the appended rows are read from the pools
    unsigned todo = __ballot_sync(kFull, odd);
#pragma unroll 1
    while (todo) {
        const int src = __ffs(todo) - 1;
        todo &= todo - 1;
        const int L = __shfl_sync(kFull, lim, src);
        const float m1 = __shfl_sync(kFull, mc, src), z1 = __shfl_sync(kFull, z, src);
        const uint16_t* q1 = reinterpret_cast<const uint16_t*>(__shfl_sync(kFull, reinterpret_cast<unsigned long long>(q), src));
        uint16_t* out1 = reinterpret_cast<uint16_t*>(__shfl_sync(kFull, reinterpret_cast<unsigned long long>(out), src));
        float4* piece1 = reinterpret_cast<float4*>(__shfl_sync(kFull, reinterpret_cast<unsigned long long>(piece), src));
        float spoilt = 0.f;
#pragma unroll 1
        for (int r = max(L, first) + (lane >> 3); r < end; r += 4) {
            const int64_t row = pool_row(a, h, r);
            if (row < 0 || !mine) continue;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float2 v = widen<F16>(reinterpret_cast<const uint32_t*>(a.Vp + row * kHeadDim + dim)[e]);
                spoilt += 0.f * v.x + 0.f * v.y;
            }
        }
        if (!__any_sync(kFull, spoilt != spoilt)) continue;
        float o[16];
#pragma unroll
        for (int e = 0; e < 16; ++e) o[e] = 0.f;
        const int last = min(L, end);
#pragma unroll 1
        for (int r0 = first; r0 < last; r0 += 4) {
            const int r = r0 + (lane >> 3);
            const int64_t row = r < last ? pool_row(a, h, r) : -1;
            float s = 0.f;
            if (row >= 0)
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float2 x = widen<F16>(reinterpret_cast<const uint32_t*>(q1 + dim)[e]);
                    const float2 k = widen<F16>(reinterpret_cast<const uint32_t*>(a.Kp + row * kHeadDim + dim)[e]);
                    s = fmaf(x.x, k.x, fmaf(x.y, k.y, s));
                }
#pragma unroll
            for (int x = 4; x >= 1; x >>= 1) s += __shfl_xor_sync(kFull, s, x);
            if (row >= 0) {
                const float p = ex2(fmaf(s, a.qscale, -m1));
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float2 v = widen<F16>(reinterpret_cast<const uint32_t*>(a.Vp + row * kHeadDim + dim)[e]);
                    o[2 * e] = fmaf(p, v.x, o[2 * e]);
                    o[2 * e + 1] = fmaf(p, v.y, o[2 * e + 1]);
                }
            }
        }
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            o[e] += __shfl_xor_sync(kFull, o[e], 8);
            o[e] += __shfl_xor_sync(kFull, o[e], 16);
        }
        if (lane < 8 && mine) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                if (piece1)
                    __stcg(reinterpret_cast<float2*>(piece1 + (dim / 4 + e / 2) * kPieceRows) + (e & 1), make_float2(o[2 * e], o[2 * e + 1]));
                else
                    reinterpret_cast<uint32_t*>(out1 + dim)[e] = pack16<F16>(o[2 * e] * z1, o[2 * e + 1] * z1);
            }
        }
        __syncwarp();
    }
}

// Loads from L2 that stay ahead of their use, a batch together (volatile).
__device__ __forceinline__ float4 load_l2(const float4* p)
{
    float4 v;
    asm volatile("ld.global.cg.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "l"(p));
    return v;
}
__device__ __forceinline__ float2 load_l2(const float2* p)
{
    float2 v;
    asm volatile("ld.global.cg.v2.f32 {%0, %1}, [%2];" : "=f"(v.x), "=f"(v.y) : "l"(p));
    return v;
}

__device__ __forceinline__ int load_acquire(const int32_t* p)
{
    int v;
    asm volatile("ld.acquire.gpu.global.s32 %0, [%1];" : "=r"(v) : "l"(p) : "memory");
    return v;
}

// A row's max and sum over the pieces of its unit, one after the other. (The roundings are written out:
// what joins the pieces must not show in the result.)
struct RowSum {
    float M, L;
    __device__ __forceinline__ void add(float2 ml, float c)
    {
        if (ml.x == -INFINITY && ml.y == 0.f) return;  // a piece that the row does not see
        const float M1 = fmaxf(M, ml.x);
        const float of_ml = __fmul_rn(ml.y, ml.x == -INFINITY ? 0.f : ex2((ml.x - M1) * c));
        L = __fmaf_rn(L, M == -INFINITY ? 0.f : ex2((M - M1) * c), of_ml);
        M = M1;
    }
};

// Pieces that one thread adds up, in their order. A turn's units are cut in two or three, all but the last stored
// long before; with that one stored and all read again as items of join_items the last CTAs took 9 to 17 us
// longer (200-777 queries over 5K-13K rows: 137 us, and 125.5 so).
constexpr int kFew = 3;

// Where piece k of the unit that starts in CTA c0 lies.
__device__ __forceinline__ int64_t piece_at(int c0, int k) { return (int64_t)(c0 + k) * 2 + (k == 0); }

// Joining a pair unit's few pieces, this CTA's (`own`) still in TMEM: the thread of each row adds the
// others to it. The sums are those of join_items.
template <bool F16>
__device__ __forceinline__ void join_own(const ChunkArgs& a, const ChunkWork& w, int c0, int pieces, int own, int prow, bool live, float2 mine,
                                         uint32_t o_at, uint16_t* out)
{
    const float c = a.qscale;
    float2 ml[kFew];
#pragma unroll
    for (int k = 0; k < kFew; ++k) {
        ml[k] = k == own ? mine : make_float2(-INFINITY, 0.f);
        if (k < pieces && k != own && live) ml[k] = load_l2(w.ml + piece_at(c0, k) * kPieceRows + prow);
    }
    RowSum sum{-INFINITY, 0.f};
#pragma unroll
    for (int k = 0; k < kFew; ++k) sum.add(ml[k], c);
    const float z = inverse(sum.L);
#pragma unroll 1
    for (int e = 0; e < kHeadDim / 32; ++e) {
        float acc[32];
#pragma unroll
        for (int d = 0; d < 32; ++d) acc[d] = 0.f;
#pragma unroll
        for (int k = 0; k < kFew; ++k) {
            if (k >= pieces) continue;
            __syncwarp();
            const bool seen = live && !(ml[k].x == -INFINITY && ml[k].y == 0.f);
            const float f = ex2((ml[k].x - sum.M) * c);
            if (k == own) {
                float v[32];
                tmem_ld32(o_at + 32 * e, v);
                if (seen)
#pragma unroll
                    for (int d = 0; d < 32; ++d) acc[d] = fmaf(v[d], f, acc[d]);
            } else if (seen) {
                const float4* o = w.o + (piece_at(c0, k) * (kHeadDim / 4) + 8 * e) * kPieceRows + prow;
                float4 u[8];
#pragma unroll
                for (int d = 0; d < 8; ++d) u[d] = load_l2(o + d * kPieceRows);
#pragma unroll
                for (int d = 0; d < 8; ++d) {
                    acc[4 * d] = fmaf(u[d].x, f, acc[4 * d]);
                    acc[4 * d + 1] = fmaf(u[d].y, f, acc[4 * d + 1]);
                    acc[4 * d + 2] = fmaf(u[d].z, f, acc[4 * d + 2]);
                    acc[4 * d + 3] = fmaf(u[d].w, f, acc[4 * d + 3]);
                }
            }
        }
        if (live) store_out<F16>(out + 32 * e, acc, z);
    }
}

// Joining the pieces of a unit: eight elements of a row an item, neighbouring rows in
// neighbouring lanes, the sums in the order of the CTAs. Loads are most of it, so ITEMS items of
// a thread and PIECES of their pieces are on the way at once (16 loads of 16 bytes).
template <bool F16, int ITEMS, int PIECES>
__device__ __forceinline__ void join_items(const ChunkArgs& a, const ChunkWork& w, const float2* scale, int t0, int rows, int g, int c0, int pieces)
{
    const int low = kTile / a.G * a.G, items = rows * (kHeadDim / 8);
    const float c = a.qscale;
#pragma unroll 1
    for (int i0 = threadIdx.x; i0 < items; i0 += ITEMS * kSoft) {
        int x[ITEMS], ch[ITEMS], at[ITEMS];
        float4 A[ITEMS], B[ITEMS];
        float2 mz[ITEMS];
#pragma unroll
        for (int y = 0; y < ITEMS; ++y) {
            const int i = min(i0 + y * kSoft, items - 1);
            ch[y] = i / rows;
            x[y] = i - ch[y] * rows;
            at[y] = x[y] < low ? x[y] : x[y] - low + kTile;
            mz[y] = scale[x[y]];
            A[y] = B[y] = make_float4(0.f, 0.f, 0.f, 0.f);
        }
#pragma unroll 1
        for (int k0 = 0; k0 < pieces; k0 += PIECES) {
            float2 ml[ITEMS][PIECES];
            float4 u[ITEMS][PIECES], v[ITEMS][PIECES];
#pragma unroll
            for (int z = 0; z < PIECES; ++z) {
                const int k = min(k0 + z, pieces - 1);
                const int64_t piece = piece_at(c0, k);
#pragma unroll
                for (int y = 0; y < ITEMS; ++y) {
                    const float4* o = w.o + (piece * (kHeadDim / 4) + 2 * ch[y]) * kPieceRows + at[y];
                    ml[y][z] = load_l2(w.ml + piece * kPieceRows + at[y]);
                    u[y][z] = load_l2(o);
                    v[y][z] = load_l2(o + kPieceRows);
                }
            }
#pragma unroll
            for (int z = 0; z < PIECES; ++z)
#pragma unroll
                for (int y = 0; y < ITEMS; ++y) {
                    const float2 m = ml[y][z];
                    if (k0 + z >= pieces || (m.x == -INFINITY && m.y == 0.f)) continue;  // a piece that the row does not see
                    const float f = ex2((m.x - mz[y].x) * c);
                    const float4 p = u[y][z], q = v[y][z];
                    A[y] = make_float4(fmaf(p.x, f, A[y].x), fmaf(p.y, f, A[y].y), fmaf(p.z, f, A[y].z), fmaf(p.w, f, A[y].w));
                    B[y] = make_float4(fmaf(q.x, f, B[y].x), fmaf(q.y, f, B[y].y), fmaf(q.z, f, B[y].z), fmaf(q.w, f, B[y].w));
                }
        }
#pragma unroll
        for (int y = 0; y < ITEMS; ++y) {
            if (i0 + y * kSoft >= items) break;
            const int token = x[y] / a.G, j = x[y] - token * a.G;
            const float z = mz[y].y;
            *reinterpret_cast<uint4*>(a.out + ((int64_t)(t0 + token) * a.H + g * a.G + j) * kHeadDim + 8 * ch[y]) =
                make_uint4(pack16<F16>(A[y].x * z, A[y].y * z), pack16<F16>(A[y].z * z, A[y].w * z), pack16<F16>(B[y].x * z, B[y].y * z),
                           pack16<F16>(B[y].z * z, B[y].w * z));
        }
    }
}

// The last piece's CTA joins the pieces. `scale` (shared): each row's max and 1 / sum over them.
template <bool F16>
__device__ __forceinline__ void join_pieces(const ChunkArgs& a, const ChunkWork& w, Waits& wait, float2* scale, int t0, int tokens, int g, int c0, int pieces)
{
    const bool ok = in_bounds(t0 >= 0 && t0 + tokens <= a.T && tokens * a.G <= kPieceRows, a.status);
    const int tid = threadIdx.x, rows = ok ? tokens * a.G : 0, low = kTile / a.G * a.G;
    const float c = a.qscale;
    // As many lanes a row as there are threads for (a power of 2), one for few pieces.
    int lanes = pieces <= kFew ? 1 : 32;
    while (lanes > 1 && lanes * rows > kSoft) lanes >>= 1;
    const int x = tid / lanes, first = tid & (lanes - 1), at = x < low ? x : x - low + kTile;
    RowSum sum{-INFINITY, 0.f};
    if (x < rows) {
#pragma unroll 4
        for (int k = first; k < pieces; k += lanes) sum.add(__ldcg(w.ml + piece_at(c0, k) * kPieceRows + at), c);
    }
    float M = sum.M, L = sum.L;
#pragma unroll 1
    for (int o = lanes >> 1; o >= 1; o >>= 1) {
        const float M0 = __shfl_xor_sync(kFull, M, o), L0 = __shfl_xor_sync(kFull, L, o), M1 = fmaxf(M, M0);
        L = (L == 0.f ? 0.f : L * ex2((M - M1) * c)) + (L0 == 0.f ? 0.f : L0 * ex2((M0 - M1) * c));
        M = M1;
    }
    if (x < rows && first == 0) scale[x] = make_float2(M, inverse(L));
    if (!wait.meet()) return;
    if (pieces <= 2)
        join_items<F16, 4, 2>(a, w, scale, t0, rows, g, c0, pieces);
    else if (rows > 16)
        join_items<F16, 2, 4>(a, w, scale, t0, rows, g, c0, pieces);
    else
        join_items<F16, 1, 8>(a, w, scale, t0, rows, g, c0, pieces);
}

template <bool F16>
__global__ void __launch_bounds__(kThreads, 1)
    chunk_attn_kernel(const __grid_constant__ ChunkArgs a, const __grid_constant__ ChunkMaps maps, const __grid_constant__ ChunkWork w, int nctas)
{
    extern __shared__ __align__(1024) unsigned char sm[];
    if (smem_u32(sm) & 1023) {  // never: the swizzled tiles need it
        if (threadIdx.x == 0) report(a, DKV_DEV_TMA_TIMEOUT);
        return;
    }
    uint64_t* full = reinterpret_cast<uint64_t*>(sm + kOffBars);  // [kStages] the stage's rows landed
    uint64_t* empty = full + kStages;                              // [kStages] its products are done
    uint64_t* said = empty + kStages;                              // [kAhead] the unit is described
    uint64_t* q_full = said + kAhead;                              // [kAhead] its Q landed
    uint64_t* late = q_full + kAhead;                              // [kAhead] the unit's CTAs are described
    uint64_t* q_empty = late + kAhead;                             // [2] the unit's score products are done
    uint64_t* s_full = q_empty + 2;                                // [2] S of the group's next step is done
    uint64_t* p_half = s_full + 2;                                 // [2] the first half of its P is written
    uint64_t* p_full = p_half + 2;                                 // [2] all of it
    uint64_t* o_done = p_full + 2;                                 // [2] the group's last product of the unit is done
    uint64_t* fin = o_done + 2;                                    // drain after a timeout
    volatile int* misc = reinterpret_cast<volatile int*>(sm + kOffMisc);
    float2* sh_ml = reinterpret_cast<float2*>(sm + kOffMl);        // [2][128]

    const int tid = threadIdx.x, warp = uniform(tid >> 5), lane = tid & 31, c = blockIdx.x;
    if (warp == 8) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(sm + kOffMisc)),
                     "r"(kTmemCols));
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    }
    if (tid == 0) {
        misc[1] = 0;
        for (int i = 0; i < kNumBars; ++i) mbar_init(smem_u32(full + i), full + i >= p_half && full + i < p_full + 2 ? 4 : 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        fence_proxy_async_smem();
    }
    // The append kernel started only after every kernel before it had completed, and this one after
    // that: what those wrote (lengths, tables, q, earlier rows) is in L2 and may be read now. The fence drops
    // what this SM's L1 holds from before, as lengths and tables are updated in place (0.1 us; loads past L1
    // instead took 145 us for the queries' 126, since a tile's page numbers lie in a line of L1). The appended rows and the
    // counters may not be read before pdl_wait().
    asm volatile("fence.acq_rel.gpu;" ::: "memory");
    int64_t* before = reinterpret_cast<int64_t*>(sm + kOffRing);
    int group;
    tc_fence_before();
    const Extent head = count_cost(a, before, reinterpret_cast<int64_t*>(sm + kOffMl), nctas, group);
    tc_fence_after();
    const uint32_t tmem = (uint32_t)uniform(misc[0]);
    const bool work = c < head.parts;
    Waits wait{misc + 1, a.status, true, false};
    const int TQ = kTile / a.G;
    if (warp >= 8) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsRest));
    if (work && warp == 10) {
        // ---------------------------------------------------------------- walk
        Walk k;
        seek(a, head, before, group, c, k);
        fence_proxy_async_smem();  // `before` lies in the ring, which the copies write next
        __syncwarp();
#pragma unroll 1
        for (int unit = 0;; ++unit) {
            // Two units ahead of the score products at most: the slot's readers are past it.
            if (unit > 1 && !wait(&q_empty[unit & 1], (unit / 2 - 1) & 1)) break;
            const bool whole = k.whole(), more = k.more();
            Piece* d = reinterpret_cast<Piece*>(sm + kOffPieces) + unit % kAhead;
            if (lane == 0) {
                *reinterpret_cast<int4*>(&d->t0) = make_int4(k.u.t0, k.u.tokens, k.u.row0, k.u.len);
                *reinterpret_cast<int4*>(&d->kv) = make_int4(k.u.kv, k.u.h, k.g, k.j0);
                *reinterpret_cast<int4*>(&d->j1) = make_int4(
                    k.j1, (k.u.pair ? Piece::kPair : 0) | (whole ? Piece::kWhole : 0) | (more ? Piece::kMore : 0), k.u.fresh, 0);
                mbar_arrive(smem_u32(&said[unit % kAhead]));
            }
            const int c0 = whole ? c : cta_of(head, k.start), last = whole ? c : cta_of(head, k.start + (k.tiles - 1) * k.cost());
            if (lane == 0) {
                d->c0 = c0;
                d->pieces = last - c0 + 1;
                mbar_arrive(smem_u32(&late[unit % kAhead]));
            }
            if (!more) break;
            k.next(a);
        }
    } else if (work && warp == 9) {
        // ---------------------------------------------------------------- TMA
        const int ppt = kTile / a.P;  // pages a tile
        bool appended = !a.k_new, pair_before = false;
        int pos = 0, unit = 0;
        Piece k;
        // Pages of tile j, and the lane's page number.
        auto pages_in = [&](int j) { return (min(max(k.kv - j * kTile, 0), kTile) + a.P - 1) / a.P; };
        auto page_of = [&](int j) {
            return lane < pages_in(j) && in_bounds(k.h >= 0 && k.h < a.B * a.Hkv && j >= 0 && j * ppt + lane < a.max_pages, a.status)
                       ? a.table[(int64_t)k.h * a.max_pages + j * ppt + lane]
                       : 0;
        };
        auto load = [&](const CUtensorMap* map, int j, int page) {
            const int s = pos % kStages, np = pages_in(j);
            const bool good = page >= 0 && page < a.num_pages;
            if (!good) report(a, DKV_DEV_PAGE_RANGE);
            const int y = (good ? page : a.num_pages) * a.P;  // behind the pool: zeros
            if (!appended && (j + 1) * kTile > k.len - k.fresh) {
                pdl_wait();
                asm volatile("fence.proxy.async.global;" ::: "memory");  // the rows were written by ordinary stores
                appended = true;
            }
            if (pos >= kStages && !wait(&empty[s], (pos / kStages - 1) & 1)) return;
            const uint32_t bar = smem_u32(&full[s]), dst = smem_u32(sm + kOffRing + s * kOperand);
            if (lane == 0) mbar_arrive_expect_tx(bar, np * a.P * kRowBytes);
            __syncwarp();
            // Rows that one unit streams once leave L2 first; a turn's units share theirs.
            uint64_t pol;
            if (k.pair())
                asm volatile("createpolicy.fractional.L2::evict_normal.b64 %0, 1.0;" : "=l"(pol));
            else
                pol = evict_first_policy();
            if (lane < np) {
                tma_box(dst + lane * a.P * 128, map, 0, y, bar, pol);
                tma_box(dst + kHalf + lane * a.P * 128, map, 64, y, bar, pol);
            }
            __syncwarp();
            ++pos;
        };
        do {
            if (!wait(&said[unit % kAhead], (unit / kAhead) & 1)) break;
            k = read_piece(sm + kOffPieces + unit % kAhead * sizeof(Piece));
            const bool pair = k.pair();
            // Q buffers: both for a pair unit, the unit's parity's for a split one, so that these run ahead.
            if (unit > 1 && !wait(&q_empty[unit & 1], (unit / 2 - 1) & 1)) break;
            if (unit > 0 && (pair || pair_before) && !wait(&q_empty[(unit - 1) & 1], ((unit - 1) / 2) & 1)) break;
            pair_before = pair;
            const int page = page_of(k.j0);  // on its way while Q is
            if (lane == 0) {
                const uint32_t bar = smem_u32(&q_full[unit % kAhead]), box = 2u * 64 * a.G * TQ;
                mbar_arrive_expect_tx(bar, (pair ? 4 : 2) * box);
                for (int p = 0; p < (pair ? 2 : 1); ++p)
                    for (int half = 0; half < 2; ++half)
                        tma_box3(smem_u32(sm + kOffQ + (pair ? p : unit & 1) * kOperand + half * kHalf), &maps.q, 64 * half, k.g * a.G,
                                 k.t0 + p * TQ, bar);
            }
            ++unit;
            __syncwarp();
            const int steps = k.steps();
            // K(0), K(1), then V(s), K(s + 2); pair units have one K and one V a pair of steps.
            load(&maps.cache.k, k.tile(0), page);
#pragma unroll 1
            for (int x = -1; x < 2 * steps && wait.ok; ++x) {
                const int s = (x >> 1) + 2 * (x & 1);  // even x: V of step x / 2; odd x: K of step x / 2 + 2
                if (s >= steps || (pair && (s & 1))) continue;
                const int j = k.tile(s);
                load(x & 1 ? &maps.cache.k : &maps.cache.v, j, page_of(j));
            }
        } while (wait.ok && k.more());
        if (!wait.ok) {
            // Copies in flight land (or run out of time) before the CTA exits.
            for (int x = max(0, pos - kStages); x < pos; ++x) land(&full[x % kStages], (x / kStages) & 1);
            for (int x = max(0, unit - 2); x < unit; ++x) land(&q_full[x % kAhead], (x / kAhead) & 1);
        }
    } else if (work && warp == 8) {
        // ---------------------------------------------------------------- MMA
        const bool leads = elect_one();
        const uint32_t id_s = idesc(kTile, kTile, 0, 0, !F16), id_o = idesc(kTile, kTile, 0, 1, !F16);
        // Operand descriptors: a stride byte offset of 1 KB, version 1, 128-byte swizzle in the high
        // word; stages and k-steps add to the address field of the low one (16-byte units).
        const uint32_t dhi = (uint32_t)(sdesc(0, 0, 1024) >> 32);
        const uint32_t dQ = (uint32_t)sdesc(smem_u32(sm + kOffQ), 16, 1024), dK = (uint32_t)sdesc(smem_u32(sm + kOffRing), 16, 1024),
                       dV = (uint32_t)sdesc(smem_u32(sm + kOffRing), kHalf, 1024);
        auto desc = [dhi](uint32_t lo) { return ((uint64_t)dhi << 32) | lo; };
        Piece k;
        int pos = 0, unit = 0, curK = 0, curV = 0;
        uint32_t phases = 0;  // bit p: parity of the P tiles taken of group p
        bool issued = false;
        do {
            if (!wait(&q_full[unit % kAhead], (unit / kAhead) & 1)) break;
            k = read_piece(sm + kOffPieces + unit % kAhead * sizeof(Piece));
            const int steps = k.steps();
            const bool pair = k.pair();
            const uint32_t qbuf = dQ + (pair ? 0 : unit & 1) * (kOperand >> 4);
#pragma unroll 1
            for (int x = -2; x < steps; ++x) {
                const int p = x & 1;
                if (x >= 0) {  // PV(x)
                    if (!pair || p == 0) {
                        curV = pos % kStages;
                        if (!wait(&full[curV], (pos / kStages) & 1)) break;
                        ++pos;
                        // Rows past the unit's last (another token's, or never written) are zeroed: 0 NaN is NaN.
                        const int valid = max(k.kv - k.tile(x) * kTile, 0);
                        if (valid < kTile) zero_rows(sm + kOffRing + curV * kOperand, valid, lane);
                    }
                    if (!wait(&p_half[p], (phases >> p) & 1)) break;
                    tc_fence_after();
                    const uint32_t v = dV + curV * (kOperand >> 4), o = tmem + 256 + p * kTile, pt = tmem + p * kTile;
                    if (leads) {
#pragma unroll
                        for (int e = 0; e < 4; ++e) umma_ts(o, pt + 8 * e, desc(v + e * (2048 >> 4)), id_o, x > 1 || e > 0);
                    }
                    __syncwarp();
                    if (!wait(&p_full[p], (phases >> p) & 1)) break;
                    phases ^= 1u << p;
                    tc_fence_after();
                    if (leads) {
#pragma unroll
                        for (int e = 4; e < 8; ++e) umma_ts(o, pt + 8 * e, desc(v + e * (2048 >> 4)), id_o, x > 1 || e > 0);
                        if (!pair || p == 1) umma_commit(smem_u32(&empty[curV]));
                        if (x + 2 >= steps) umma_commit(smem_u32(&o_done[p]));
                    }
                    __syncwarp();
                }
                if (x + 2 < steps) {  // S(x + 2)
                    if (!pair || p == 0) {
                        curK = pos % kStages;
                        if (!wait(&full[curK], (pos / kStages) & 1)) break;
                        ++pos;
                    }
                    tc_fence_after();
                    if (leads) {
                        const uint32_t q = qbuf + (pair ? p : 0) * (kOperand >> 4), kt = dK + curK * (kOperand >> 4), d = tmem + p * kTile;
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            const uint32_t off = ((e >> 2) * kHalf + (e & 3) * 32) >> 4;
                            umma(d, desc(q + off), desc(kt + off), id_s, e > 0);
                        }
                        umma_commit(smem_u32(&s_full[p]));
                        if (!pair || p == 1) umma_commit(smem_u32(&empty[curK]));
                        if (x + 2 == steps - 1) umma_commit(smem_u32(&q_empty[unit & 1]));
                    }
                    issued = true;
                    __syncwarp();
                }
            }
            ++unit;
        } while (wait.ok && k.more());
        if (!wait.ok && issued) {
            if (leads) {
                umma_commit(smem_u32(fin));
                land(fin, 0);
            }
            __syncwarp();
        }
    }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegsSoft));
        if (work) {
        // ---------------------------------------------------------------- softmax groups
        const int p = warp >> 2, r = tid & 127;
        const uint32_t lanes = (uint32_t)(32 * (warp & 3)) << 16;
        const uint32_t s_at = tmem + lanes + p * kTile, o_at = tmem + lanes + 256;
        const int token = r / a.G, j = r - token * a.G;
        const float cs = a.qscale;
        Piece k;
        int ns = 0, no = 0;  // S tiles and O accumulators taken
        int unit = 0;
        do {
            if (!wait(&said[unit % kAhead], (unit / kAhead) & 1)) break;
            k = read_piece(sm + kOffPieces + unit % kAhead * sizeof(Piece));
            const int steps = k.steps();
            const bool pair = k.pair(), whole = k.whole();
            const int tok = token + (pair ? p * TQ : 0);
            const bool live = token < TQ && tok < k.tokens && in_bounds(k.t0 >= 0 && k.t0 + tok < a.T && k.g * a.G + j < a.H, a.status);
            const int lim = !live ? 0x3fffffff : a.causal ? min(max(k.row0 + tok, 0), k.len) : k.len;
            const bool any = __any_sync(kFull, live);
            float m = -INFINITY, l = 0.f;
#pragma unroll 1
            for (int s = p; s < steps; s += 2) {
                if (!wait(&s_full[p], ns++ & 1)) break;
                if (any) {
                    tc_fence_after();
                    softmax_step<F16>(s_at, o_at + p * kTile, lim - k.tile(s) * kTile, s > 1, cs, m, l, smem_u32(&p_half[p]));
                    tc_fence_before();
                } else if (lane == 0) {
                    mbar_arrive(smem_u32(&p_half[p]));
                }
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&p_full[p]));
            }
            if (!wait.ok) break;
            if (steps > p && !wait(&o_done[p], no++ & 1)) break;
            tc_fence_after();
            uint16_t* out = a.out + ((int64_t)(k.t0 + tok) * a.H + k.g * a.G + j) * kHeadDim;
            // Of a pair unit with few pieces, all others may be done: then this one is not stored. (Not if some of
            // its rows may have to be mended.)
            int c0 = c, pieces = 1;
            bool few = false, last = false;
            if (!whole) {
                if (!wait(&late[unit % kAhead], (unit / kAhead) & 1)) break;
                const volatile Piece* d = reinterpret_cast<const volatile Piece*>(sm + kOffPieces) + unit % kAhead;
                c0 = d->c0;
                pieces = d->pieces;
                if (!in_bounds(c0 >= 0 && c0 <= c && pieces > c - c0 && c0 + pieces <= nctas, a.status)) c0 = c, pieces = 1;
                few = pair && pieces <= kFew && min(k.kv, k.j1 * kTile) <= k.row0;
                if (few) {
                    if (tid == 0) {
                        pdl_wait();  // the counters are cleared
                        misc[2] = load_acquire(w.done + c0) == pieces - 1;
                    }
                    if (!wait.meet()) break;
                    last = misc[2];
                    if (last) __threadfence();
                }
            }
            const int64_t slot = (int64_t)c * 2 + (k.j0 == 0);
            const int prow = (pair ? p * kTile : 0) + r;
            // Cache rows of this piece, and whether some of them are hidden from the thread's query.
            const int first = k.j0 * kTile, end = min(k.kv, k.j1 * kTile);
            const bool hidden = live && lim < end;
            const uint16_t* q = a.q + (int64_t)(k.t0 + tok) * a.q_stride + (k.g * a.G + j) * kHeadDim;
            float4* o_piece = whole ? nullptr : w.o + slot * (kHeadDim / 4) * kPieceRows + prow;
            float odd = 0.f;  // NaN if a result is not finite
            if (pair) {
                if (any && !last) {
                    const float z = inverse(l);
#pragma unroll 1
                    for (int e = 0; e < 4; ++e) {
                        float v[32];
                        tmem_ld32(o_at + p * kTile + 32 * e, v);
#pragma unroll
                        for (int d = 0; d < 32; ++d) odd = fmaf(v[d], 0.f, odd);
                        if (live && whole) store_out<F16>(out + 32 * e, v, z);
                        if (live && !whole) store_piece(o_piece + 8 * e * kPieceRows, v);
                    }
                    if (__any_sync(kFull, hidden && odd != odd))
                        mend_rows<F16>(a, k.h, hidden && odd != odd, first, lim, end, origin<F16>(m, cs), z, q, out, o_piece, 0, kHeadDim);
                    if (live && !whole) __stcg(w.ml + slot * kPieceRows + prow, make_float2(m, l));
                }
            } else {
                // The groups' halves of the cache rows: each group joins 64 of the dimensions.
                sh_ml[p * kTile + r] = make_float2(m, l);
                tc_fence_before();
                if (!wait.meet()) break;
                tc_fence_after();
                const float2 x = sh_ml[r], y = sh_ml[kTile + r];
                const float M = fmaxf(x.x, y.x);
                const float fx = x.x == -INFINITY ? 0.f : ex2((x.x - M) * cs), fy = y.x == -INFINITY ? 0.f : ex2((y.x - M) * cs);
                const float L = x.y * fx + y.y * fy, z = inverse(L);
                const bool two = steps > 1;
                if (any) {
#pragma unroll 1
                    for (int e = 2 * p; e < 2 * p + 2; ++e) {
                        float v[32], v1[32];
                        tmem_ld32(o_at + 32 * e, v);
                        if (two) tmem_ld32(o_at + kTile + 32 * e, v1);
#pragma unroll
                        for (int d = 0; d < 32; ++d) {
                            v[d] = v[d] * fx + (two ? v1[d] * fy : 0.f);
                            odd = fmaf(v[d], 0.f, odd);
                        }
                        if (live && whole) store_out<F16>(out + 32 * e, v, z);
                        if (live && !whole) store_piece(o_piece + 8 * e * kPieceRows, v);
                    }
                    if (__any_sync(kFull, hidden && odd != odd))
                        mend_rows<F16>(a, k.h, hidden && odd != odd, first, lim, end, origin<F16>(M, cs), z, q, out, o_piece, 64 * p, 64);
                    if (live && !whole && p == 0) __stcg(w.ml + slot * kPieceRows + prow, make_float2(M, L));
                }
            }
            if (!whole && !last) {
                __threadfence();
                if (!wait.meet()) break;
                if (tid == 0) {
                    pdl_wait();  // the counters are cleared
                    misc[2] = atomicAdd(w.done + c0, 1) == pieces - 1;
                }
                if (!wait.meet()) break;
                last = misc[2];
                if (last) __threadfence();
                if (last && !few) join_pieces<F16>(a, w, wait, sh_ml, k.t0, k.tokens, k.g, c0, pieces);
            }
            if (few && last && any) join_own<F16>(a, w, c0, pieces, c - c0, prow, live, make_float2(m, l), o_at + p * kTile, out);
            if (!pair || !whole) {
                tc_fence_before();
                if (!wait.meet()) break;  // O of the other group, sh_ml and misc[2] are read
            }
            ++unit;
        } while (k.more());
        wait.meet();
        }
    }
    // ---------------------------------------------------------------- teardown
    pdl_wait();  // the call is not over before its append
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == 8)
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmemCols));
}

PFN_cuTensorMapEncodeTiled_v12000 encode_tiled()
{
    static std::once_flag once;
    static PFN_cuTensorMapEncodeTiled_v12000 fn = nullptr;
    std::call_once(once, [] {
        void* p = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &q) == cudaSuccess &&
            q == cudaDriverEntryPointSuccess)
            fn = reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(p);
    });
    return fn;
}

// q as [T][H][128] with its token stride; a box is 64 dims x the heads of a group x TQ tokens.
cudaError_t make_q_map(const ChunkArgs& a, CUtensorMap* map)
{
    PFN_cuTensorMapEncodeTiled_v12000 enc = encode_tiled();
    if (!enc) return cudaErrorNotSupported;
    const cuuint64_t dim[3] = {(cuuint64_t)kHeadDim, (cuuint64_t)a.H, (cuuint64_t)a.T};
    const cuuint64_t stride[2] = {(cuuint64_t)kRowBytes, (cuuint64_t)a.q_stride * 2};
    const cuuint32_t box[3] = {64, (cuuint32_t)a.G, (cuuint32_t)(kTile / a.G)};
    const cuuint32_t elem[3] = {1, 1, 1};
    return enc(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<uint16_t*>(a.q), dim, stride, box, elem,
               CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
               CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS
               ? cudaSuccess
               : cudaErrorInvalidValue;
}

template <bool F16>
cudaError_t launch_attn(const ChunkArgs& a, const ChunkMaps& maps, const ChunkWork& w, int nctas, cudaStream_t st)
{
    return launch_pdl(chunk_attn_kernel<F16>, nctas, kThreads, kSmemBytes, st, a, maps, w, nctas);
}

}  // namespace

int64_t chunk_workspace_bytes() { return kWorkBytes; }

cudaError_t chunk_setup()
{
    cudaError_t e = cudaFuncSetAttribute(chunk_attn_kernel<false>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemBytes);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(chunk_attn_kernel<true>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemBytes);
    return e;
}

cudaError_t launch_chunk(const ChunkArgs& a, bool short_boxes, cudaStream_t st)
{
    int sms = 0;
    cudaError_t e = page_setup(&sms);
    if (e != cudaSuccess) return e;
    const int nctas = sms < kMaxCtas ? sms : kMaxCtas;
    ChunkMaps maps;
    if ((e = make_cache_maps(a.Kp, a.Vp, (int64_t)a.num_pages * a.P, &maps.cache, short_boxes, a.P, false)) != cudaSuccess) return e;
    if ((e = make_q_map(a, &maps.q)) != cudaSuccess) return e;
    unsigned char* base = static_cast<unsigned char*>(a.work);
    ChunkWork w;
    w.done = reinterpret_cast<int32_t*>(base);
    w.ml = reinterpret_cast<float2*>(base + kOffPieceMl);
    w.o = reinterpret_cast<float4*>(base + kOffPieceO);
    const int64_t rows = a.k_new ? (int64_t)a.T * a.Hkv : 0;
    const int blocks = 1 + (int)((rows + kAppThreads / 16 - 1) / (kAppThreads / 16));
    if ((e = launch_pdl(chunk_append_kernel, blocks, kAppThreads, 0, st, a, w)) != cudaSuccess) return e;
    return a.fp16 ? launch_attn<true>(a, maps, w, nctas, st) : launch_attn<false>(a, maps, w, nctas, st);
}

}  // namespace dkv
