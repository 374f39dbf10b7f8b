// Attention of a step's new tokens over 8-bit pages: token i of the n new ones of sequence b attends,
// per query head, to the first len - n + i + 1 rows of its slab (causal) or to all len rows,
//   o = sum_r softmax_r(scale 2^ek_r q.k_r) 2^ev_r v_r,   k_r, v_r e4m3 values, 2^ek_r, 2^ev_r their rows' scales.
// Here: sequences of few columns (column = token G + head of the group), at most 16; those of more go to
// chunk_attn_kernel (dkv_chunk.cu), which turns 8-bit tiles into 16-bit ones for the tensor memory's products.
//
// Unit of work: a slab, its columns against the cache rows that its last token sees, in tiles of 32 rows. Units lie end to
// end on a line of costs, a tile each and kStart for a unit's start, that is cut into equal shares, one a CTA, one CTA an SM;
// a CTA's warps take the tiles of its part of a unit in turn, each through a ring of its own, and are joined at its end. A unit
// that lies in several CTAs is joined by the one that finishes last, in the order of the CTAs. Behind chunk_attn_kernel this one also
// joins what that left in many pieces, a warp 8 rows and 16 dims (join_chunks; it waits for that kernel's end anyway): 3 us for
// the drafts of four sequences, 17 where a unit's last CTA did it.
//
//   quant_begin_kernel  clears the counters.
//   quant_attn_kernel   the rest.
//
// A warp multiplies with the warp-level fp16 products (m16n8k16), whose values e4m3 values are among: 16 cache rows x 8
// columns x 16 dims for the scores, 16 dims x 8 columns x 16 rows for O. The dims of a product may be any order that
// both operands share, so a lane takes 32 dims of K that lie together, and 16 of V: K's bytes convert in place, V's
// pairs of rows after a byte permutation, and the weights come to the second product's order by an 8 x 8 transposition.
// Tiles lie in shared memory as TMA's 128-byte swizzle puts them, which makes these 16-byte reads free of conflicts.
//
// A row's V scale goes into its weight's exponent: O goes by 2^(top + scale), the running maxima of the scores and of the V
// scales that the column has seen (of those alone: a later token's row may hold anything), the sum of weights by 2^top.
// Scores, statistics and O are fp32; the weights, times V's scales, are rounded to fp16, as the products take them: half a
// step is 2^-11 of a weight, an eighth of the rounding of a bf16 output.
//
// What bounds it. 16 sequences' next tokens over 3K-24K rows, 386 MB: 68 us, 5.7 TB/s of a plain copy's 6.7; about 700
// instructions a tile and warp, 0.43 a cycle and scheduler, more than half of them the conversion (two values an
// instruction). With the columns as the products' 16-row operand, half of whose rows were then of no column, it took 82 us with 12 warps
// and 96 with 8; with a share of tiles alone, and not of a unit's start, 70.5. One token over 1.5K rows: 11.5 us, all latency, 8 of
// it here (count 1.7, walk 0.7, page table and copy 1.9, a tile 1.2, joins 2.3), where shares of a unit and a half took 17.6.
#include "dkv_quant.cuh"

#include "dkv_tcgen05.cuh"

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cudaTypedefs.h>

#include <algorithm>
#include <mutex>

namespace dkv {
namespace {

constexpr int kMostCols = 16;              // columns of a unit, at most
constexpr int kRows = 32;                  // cache rows of a tile
constexpr int kTileBytes = kRows * kHeadDim;
constexpr int kStageBytes = 2 * kTileBytes;  // K, then V
constexpr int kMaxCtas = 160;              // CTAs of the largest grid (the workspace's size)
constexpr float kShift = 7.f;              // weights for the second product are 2^7 larger: fp16 has 2^15 above the slack

// Z: 8-column halves of a unit's columns. One half takes half of the registers, so a CTA has more warps.
template <int Z>
struct Cfg {
    static constexpr int kCols = 8 * Z;
    static constexpr int kWarps = Z == 1 ? 12 : 8;
    static constexpr int kThreads = 32 * kWarps;
    static constexpr int kStages = Z == 1 ? 2 : 3;  // ring of a warp
    // Shared memory, from its 1024-byte aligned start.
    static constexpr int kOffSum = kWarps * kStages * kStageBytes;            // float[kWarps][kCols][64], before that State[kWarps][kCols]
    static constexpr int kOffScales = kOffSum + kWarps * kCols * 64 * 4;      // a stage's scale bytes: of K, of V
    static constexpr int kOffFactors = kOffScales + kWarps * kStages * 2 * kRows;  // uint32[kWarps][kRows]: a tile's scales
    static constexpr int kOffBars = kOffFactors + kWarps * kRows * 4;
    static constexpr int kOffMisc = kOffBars + kWarps * kStages * 8;          // int[4]: abort, last
    static constexpr int kSmemBytes = kOffMisc + 16;
    static constexpr int kMaxGroups = kOffSum / 8;                            // prefix sums in the rings before their first use
    static_assert(kSmemBytes <= 227 * 1024, "fits one CTA");
    static_assert(kChunkCounters * 20 + 20 <= kOffScales - kOffSum && kOffSum % 16 == 0, "join_chunks's units fit");
    static_assert(kOffBars % 8 == 0 && kOffScales % 16 == 0, "aligned");
};

// A column's softmax over some rows: max of x, sum of 2^(x - top), and the V scale (its exponent) that O goes by.
struct State {
    float top, sum, scale, pad;
};

// Workspace.
struct QuantWork {
    int32_t* done;  // [kMaxCtas] finished pieces of the unit that starts in CTA c and ends in a later one
    State* state;   // [kMaxCtas][2][16]
    float4* o;      // [kMaxCtas][2][16][32]
    int4* jobs;     // [kChunkCounters] what the kernel of many tokens leaves to this one
    int32_t* chunk; // that kernel's workspace, its counters first
};
constexpr int64_t kOffJobs = (kMaxCtas * 4 + 255) / 256 * 256, kOffState = kOffJobs + (kChunkCounters * 16 + 255) / 256 * 256, kOffO = kOffState + (int64_t)kMaxCtas * 2 * kMostCols * sizeof(State),
                  kWorkBytes = kOffO + (int64_t)kMaxCtas * 2 * kMostCols * kHeadDim * 4;
static_assert(kWorkBytes % 256 == 0, "the other kernel's workspace lies behind it");

__device__ __forceinline__ void report(const QuantAttnArgs& a, int bits)
{
    if (a.status) atomicOr(a.status, bits);
}

__device__ __forceinline__ int cu_at(const QuantAttnArgs& a, int b) { return min(max(a.cu[b], 0), a.T); }

__device__ __forceinline__ bool bad_offsets(const QuantAttnArgs& a, int b)
{
    const int t0 = a.cu[b], t1 = a.cu[b + 1];
    return t1 < t0 || t1 > a.T || (b == 0 && t0 != 0);
}

// Tokens of sequence b that quant_attn_kernel deals with.
__device__ __forceinline__ int tokens_of(const QuantAttnArgs& a, int b)
{
    const int n = cu_at(a, b + 1) - cu_at(a, b);
    return n > a.few ? 0 : n;
}

// Rows of slab h; none if its length is out of range.
__device__ __forceinline__ int slab_len(const QuantAttnArgs& a, int h)
{
    const int len = a.len[h];
    return len >= 0 && len <= a.max_pages * a.P ? len : 0;  // (the product is below 2^31)
}

// Rows that token i of n sees.
__device__ __forceinline__ int sees(const QuantAttnArgs& a, int len, int n, int i) { return a.causal ? min(max(len - n + i + 1, 0), len) : len; }

__device__ __forceinline__ int tiles_of(int rows) { return max(1, (int)(((unsigned)rows + kRows - 1) / kRows)); }

// What slab h's unit costs: its tiles, and as much as kStart of them for its start (the join of the warps, a fence, a count:
// 3 us, in which a CTA has its share of 16 tiles from memory).
constexpr int kStart = 16;
__device__ __forceinline__ int slab_cost(const QuantAttnArgs& a, int h)
{
    const int n = tokens_of(a, h / a.Hkv), len = slab_len(a, h);  // (both loads at once)
    return n == 0 ? 0 : kStart + tiles_of(sees(a, len, n, n - 1));
}

// Clears the counters of both kernels. `early`: the next kernel is started at once and waits for this one before it reads
// anything; else it is started once every kernel before this one has completed, and waits only for the counters.
__global__ void __launch_bounds__(256) quant_begin_kernel(const __grid_constant__ QuantWork w, int early)
{
    if (early) pdl_launch_dependents();
    pdl_wait();
    if (!early) pdl_launch_dependents();
    for (int i = threadIdx.x; i < kMaxCtas; i += 256) w.done[i] = 0;
    for (int i = threadIdx.x; i < kChunkCounters; i += 256) w.chunk[i] = 0;
}

// Reports what lives on the device and is out of range (one CTA).
__device__ __forceinline__ void check(const QuantAttnArgs& a)
{
    for (int b = threadIdx.x; b < a.B; b += blockDim.x)
        if (bad_offsets(a, b) || cu_at(a, b + 1) - cu_at(a, b) > a.most) report(a, DKV_DEV_PAGE_RANGE);
    for (int h = threadIdx.x; h < a.B * a.Hkv; h += blockDim.x) {
        const int b = h / a.Hkv;
        if (cu_at(a, b + 1) > cu_at(a, b) && a.len[h] != slab_len(a, h)) report(a, DKV_DEV_PAGE_RANGE);
    }
}

// ---------------------------------------------------------------- schedule
// Units lie end to end on a line of costs, kStart before the tiles of each; a tile is the CTA's in whose part of the line it
// lies. Shares are not shorter than kLeast, where a CTA's warps would not all have a tile.
constexpr int kLeast = 8;
struct Extent {
    int64_t cost;
    int parts;
};
__device__ __forceinline__ int64_t divide(int64_t x, int64_t y)
{
    return x <= UINT32_MAX && y <= UINT32_MAX ? (int64_t)((uint32_t)x / (uint32_t)y) : x / y;
}
__device__ __forceinline__ int64_t share_start(const Extent& e, int c) { return divide(e.cost * c, e.parts); }
__device__ __forceinline__ int cta_of(const Extent& e, int64_t x) { return (int)divide((x + 1) * e.parts - 1, e.cost); }

// All threads of the CTA: the cost before every slab (or group of slabs, where there are more than fit), into `before`.
template <int Z>
__device__ __forceinline__ Extent count_cost(const QuantAttnArgs& a, int64_t* before, int64_t* sums, int nctas, int& group)
{
    constexpr int kMaxGroups = Cfg<Z>::kMaxGroups, kThreads = Cfg<Z>::kThreads, kWarps = Cfg<Z>::kWarps;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, slabs = a.B * a.Hkv;
    group = (slabs + kMaxGroups - 1) / kMaxGroups;
    const int groups = (slabs + group - 1) / group, per = (groups + kThreads - 1) / kThreads;
    const int g0 = min(groups, tid * per), g1 = min(groups, g0 + per);
    int64_t mine = 0;
#pragma unroll 1
    for (int x = g0; x < g1; ++x) {
        before[x] = mine;
#pragma unroll 1
        for (int h = x * group; h < min(slabs, (x + 1) * group); ++h) mine += slab_cost(a, h);
    }
    int64_t up = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int64_t y = __shfl_up_sync(kFull, up, o);
        if (lane >= o) up += y;
    }
    if (lane == 31) sums[warp] = up;
    bool bad = false;
#pragma unroll 1
    for (int b = tid; b < a.B; b += kThreads) bad |= bad_offsets(a, b);
    bad = __syncthreads_or(bad);
    int64_t base = up - mine, total = 0;
#pragma unroll
    for (int k = 0; k < kWarps; ++k) {
        if (k < warp) base += sums[k];
        total += sums[k];
    }
#pragma unroll 1
    for (int x = g0; x < g1; ++x) before[x] += base;
    __syncthreads();
    return bad ? Extent{0, 0} : Extent{total, (int)min((int64_t)nctas, (total + kLeast - 1) / kLeast)};
}

// The share of one CTA, unit by unit.
struct Walk {
    int b, g, t, n, len;       // sequence, head; the sequence's first token, its tokens, the slab's rows
    int rows, tiles, j0, j1;   // of the unit; the CTA's tiles of it
    int64_t start, end;        // where the unit's tiles start, where the share ends
    __device__ __forceinline__ void sequence(const QuantAttnArgs& a)
    {
        t = cu_at(a, b);
        n = tokens_of(a, b);
    }
    // The unit (b, g), from its tile j on; `start` is set.
    __device__ __forceinline__ void enter(const QuantAttnArgs& a, int j)
    {
        len = slab_len(a, b * a.Hkv + g);
        rows = sees(a, len, n, n - 1);
        tiles = tiles_of(rows);
        j0 = j;
        j1 = (int)min((int64_t)tiles, end - start);
    }
    __device__ __forceinline__ bool more() const { return start + tiles + kStart < end; }
    __device__ __forceinline__ void next(const QuantAttnArgs& a)
    {
        start += tiles + kStart;
        if (++g == a.Hkv) {
            g = 0;
            do ++b;
            while (b < a.B - 1 && tokens_of(a, b) == 0);
            sequence(a);
        }
        enter(a, 0);
    }
    __device__ __forceinline__ bool whole() const { return j0 == 0 && j1 == tiles; }
};

// Where the share of CTA c starts; false if no tile lies in it.
__device__ __forceinline__ bool seek(const QuantAttnArgs& a, const Extent& e, const int64_t* before, int group, int c, Walk& k)
{
    if (c >= e.parts) return false;
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
    int h = lo * group;
    if (group > 1)
        for (int x; off >= (x = slab_cost(a, h)); ++h) off -= x;
    k.start = pos - off + kStart;
    if (k.start >= k.end) return false;
    k.b = h / a.Hkv;
    k.g = h - k.b * a.Hkv;
    k.sequence(a);
    k.enter(a, (int)max(off - kStart, (int64_t)0));
    return true;
}

// ---------------------------------------------------------------- products
__device__ __forceinline__ void mma(float (&d)[4], const uint32_t (&x)[4], uint32_t y0, uint32_t y1)
{
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(x[0]), "r"(x[1]), "r"(x[2]), "r"(x[3]), "r"(y0), "r"(y1));
}

__device__ __forceinline__ uint32_t half2_of(float x, float y)
{
    const __half2 v = __floats2half2_rn(x, y);
    return *reinterpret_cast<const uint32_t*>(&v);
}

// 2^x, 0 below 2^-126; x <= 127.
__device__ __forceinline__ float exp2i(int x) { return __uint_as_float((uint32_t)max(x + 127, 0) << 23); }

// Bytes of a word that are NaN, as 0xff.
__device__ __forceinline__ uint32_t nan_bytes(uint32_t w) { return __vcmpeq4(w & 0x7f7f7f7fu, 0x7f7f7f7fu); }

__device__ __forceinline__ uint4 lds128(const unsigned char* p)
{
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(smem_u32(p)) : "memory");
    return v;
}

// A lane's quarter of a column of q (elements 32 t .. 32 t + 31 of 128), zeros if there is none.
__device__ __forceinline__ void load_column(const uint16_t* src, bool live, uint4 (&x)[4])
{
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = live ? ld_prev(reinterpret_cast<const uint4*>(src) + i) : make_uint4(0u, 0u, 0u, 0u);
}

// The same as fp16 pairs, scaled by a power of two that takes the column's largest element to 2^14 .. 2^15; `back`: its
// inverse.
template <bool F16>
__device__ __forceinline__ void scale_column(const uint4 (&x)[4], uint32_t (&q)[16], float& back)
{
    float f[32], most = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const uint32_t w = i & 2 ? (i & 1 ? x[i >> 2].w : x[i >> 2].z) : (i & 1 ? x[i >> 2].y : x[i >> 2].x);
        if (F16) {
            const float2 v = __half22float2(*reinterpret_cast<const __half2*>(&w));
            f[2 * i] = v.x;
            f[2 * i + 1] = v.y;
        } else {
            f[2 * i] = __uint_as_float(w << 16);
            f[2 * i + 1] = __uint_as_float(w & 0xffff0000u);
        }
    }
#pragma unroll
    for (int i = 0; i < 32; ++i) most = fmaxf(most, fabsf(f[i]) < INFINITY ? fabsf(f[i]) : 0.f);
    most = fmaxf(most, __shfl_xor_sync(kFull, most, 1));
    most = fmaxf(most, __shfl_xor_sync(kFull, most, 2));
    const uint32_t e = max(__float_as_uint(most) >> 23, 15u);
    const float scale = __uint_as_float((268u - e) << 23);
    back = __uint_as_float((e - 14u) << 23);
#pragma unroll
    for (int i = 0; i < 16; ++i) q[i] = half2_of(f[2 * i] * scale, f[2 * i + 1] * scale);
}

// An 8 x 8 matrix of 16-bit values, row lane / 4, columns 2 (lane % 4) and the next: transposed.
__device__ __forceinline__ uint32_t transposed(uint32_t x)
{
    uint32_t y;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}

// What a lane (g = lane / 4, t = lane % 4) has of its warp's columns 8 z + 2 t + e.
template <int Z>
struct Acc {
    float o[8][Z][4];         // dims 16 g + 2 i of columns e = 0, 1, then dims 16 g + 2 i + 1
    float top[Z][2], l[Z][2]; // in units of 1 / cs; l: of the lane's rows
    int scale[Z][2];          // byte of the largest V scale that the column has seen, which its O goes by
};

// One tile: scores, softmax, O += P V. lim: the tile's rows that the columns see; rows: those of the unit; `shown`: rows
// that all columns see.
template <int Z>
__device__ __forceinline__ void tile_step(Acc<Z>& c, const uint32_t (&q)[Z][16], const float (&cs)[Z][2], const unsigned char* k, const unsigned char* v,
                                          const unsigned char* scales, uint32_t* factors, const int (&lim)[Z][2], int shown, int rows)
{
    const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const bool edge = shown < kRows;
    // A row a lane: K's scale as a factor, V's as an exponent. A column's O goes by the largest V scale that it has seen so far;
    // where a larger one comes, it is brought to that.
    {
        const int ku = scales[lane], vu = scales[kRows + lane];
        // (a power of two, and a whole number below 256: the upper half of each has all of it)
        factors[lane] = __float_as_uint(scale_of(ku)) | __float_as_uint((float)(vu - 127)) >> 16;
        int most = lane < shown ? vu : 0;
        bool more = false;
#pragma unroll
        for (int z = 0; z < Z; ++z) more |= most > min(c.scale[z][0], c.scale[z][1]);
        if (edge || __any_sync(kFull, more)) {
            most = __reduce_max_sync(kFull, most);
            int own[Z][2];
#pragma unroll
            for (int z = 0; z < Z; ++z) own[z][0] = own[z][1] = most;
            if (edge) {  // rows that not all columns see: the lane's columns' own
                for (int row = max(shown, 0); row < min(rows, kRows); ++row) {
                    const int u = scales[kRows + row];
#pragma unroll
                    for (int z = 0; z < Z; ++z)
#pragma unroll
                        for (int e = 0; e < 2; ++e)
                            if (row < lim[z][e]) own[z][e] = max(own[z][e], u);
                }
            }
#pragma unroll
            for (int z = 0; z < Z; ++z)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int to = max(own[z][e], c.scale[z][e]);
                    const float down = exp2i(c.scale[z][e] - to);
                    c.scale[z][e] = to;
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        c.o[i][z][e] *= down;
                        c.o[i][z][2 + e] *= down;
                    }
                }
        }
    }
    // Rows 16 m + g and 16 m + g + 8 of columns 2 t and 2 t + 1.
    float s[2][Z][4];
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int z = 0; z < Z; ++z)
#pragma unroll
            for (int e = 0; e < 4; ++e) s[m][z][e] = 0.f;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        uint32_t w[4][4];
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            const uint4 u = lds128(k + (8 * x + g) * kHeadDim + (((2 * t + i) ^ g) << 4));
            w[x][0] = u.x;
            w[x][1] = u.y;
            w[x][2] = u.z;
            w[x][3] = u.w;
        }
#pragma unroll
        for (int y = 0; y < 4; ++y) {
            const int ks = 4 * i + y;  // dims 32 t + 4 ks .. + 3 of every t
#pragma unroll
            for (int m = 0; m < 2; ++m) {
                uint32_t A[4];
                widen_e4m3(w[2 * m][y], A[0], A[2]);
                widen_e4m3(w[2 * m + 1][y], A[1], A[3]);
#pragma unroll
                for (int z = 0; z < Z; ++z) mma(s[m][z], A, q[z][2 * ks], q[z][2 * ks + 1]);
            }
        }
    }
    __syncwarp();  // the factors are there
    // Scores by their rows' scales; f: the exponents of the rows' V scales.
    float f[4];
#pragma unroll
    for (int x = 0; x < 4; ++x) {
        const uint32_t u = factors[8 * x + g];
        f[x] = __uint_as_float(u << 16);
        const float kf = __uint_as_float(u & 0xffff0000u);
#pragma unroll
        for (int z = 0; z < Z; ++z)
#pragma unroll
            for (int e = 0; e < 2; ++e) s[x >> 1][z][2 * (x & 1) + e] *= kf;
    }
    if (edge) {
#pragma unroll
        for (int x = 0; x < 4; ++x)
#pragma unroll
            for (int z = 0; z < Z; ++z)
#pragma unroll
                for (int e = 0; e < 2; ++e)
                    if (8 * x + g >= lim[z][e]) s[x >> 1][z][2 * (x & 1) + e] = -INFINITY;  // also over NaN
    }
    // The maxima move only when a score tops them by 2^kSlack (they are then found over the lanes of a column).
    float mx[Z][2];
    bool any = false;
#pragma unroll
    for (int z = 0; z < Z; ++z)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            mx[z][e] = fmaxf(fmaxf(s[0][z][e], s[0][z][2 + e]), fmaxf(s[1][z][e], s[1][z][2 + e]));
            any |= (mx[z][e] - c.top[z][e]) * cs[z][e] > kSlack;
        }
    if (__any_sync(kFull, any)) {
#pragma unroll
        for (int z = 0; z < Z; ++z) {
            float alpha[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
#pragma unroll
                for (int o = 4; o < 32; o <<= 1) mx[z][e] = fmaxf(mx[z][e], __shfl_xor_sync(kFull, mx[z][e], o));
                const bool up = (mx[z][e] - c.top[z][e]) * cs[z][e] > kSlack;  // (a column's own, whatever the others hold)
                alpha[e] = up ? ex2((c.top[z][e] - mx[z][e]) * cs[z][e]) : 1.f;
                if (up) c.top[z][e] = mx[z][e];
                c.l[z][e] *= alpha[e];
            }
#pragma unroll
            for (int i = 0; i < 8; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) c.o[i][z][e] *= alpha[e & 1];
        }
    }
    uint32_t p[4][Z];
#pragma unroll
    for (int z = 0; z < Z; ++z) {
        float top[2], ref[2];  // origins of the weights, and of the weights times V's scales
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            top[e] = c.top[z][e] == -INFINITY ? 0.f : c.top[z][e] * cs[z][e];
            ref[e] = top[e] + ((float)(c.scale[z][e] - 127) - kShift);
        }
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            const float x0 = s[x >> 1][z][2 * (x & 1)], x1 = s[x >> 1][z][2 * (x & 1) + 1];
            c.l[z][0] += ex2(fmaf(x0, cs[z][0], -top[0]));
            c.l[z][1] += ex2(fmaf(x1, cs[z][1], -top[1]));
            p[x][z] = transposed(half2_of(ex2(fmaf(x0, cs[z][0], f[x] - ref[0])), ex2(fmaf(x1, cs[z][1], f[x] - ref[1]))));
        }
    }
    bool odd = false;  // NaN in a row of V that not all columns see
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
        uint32_t w[4][4];
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            const int row = 16 * kb + 2 * t + (x & 1) + 8 * (x >> 1);
            const uint4 u = lds128(v + row * kHeadDim + ((g ^ (row & 7)) << 4));
            w[x][0] = u.x;
            w[x][1] = u.y;
            w[x][2] = u.z;
            w[x][3] = u.w;
            if (edge && row >= shown) {  // 0 NaN is NaN
#pragma unroll
                for (int y = 0; y < 4; ++y) {
                    const uint32_t bad = nan_bytes(w[x][y]);
                    odd |= bad != 0 && row < rows;
                    w[x][y] = row < rows ? w[x][y] & ~bad : 0u;
                }
            }
        }
#pragma unroll
        for (int y = 0; y < 4; ++y)
#pragma unroll
            for (int x = 0; x < 2; ++x) {  // dims 16 g + 4 y + 2 x and the next
                uint32_t A[4];
                widen_e4m3(__byte_perm(w[0][y], w[1][y], x ? 0x7362 : 0x5140), A[0], A[1]);
                widen_e4m3(__byte_perm(w[2][y], w[3][y], x ? 0x7362 : 0x5140), A[2], A[3]);
#pragma unroll
                for (int z = 0; z < Z; ++z) mma(c.o[2 * y + x][z], A, p[2 * kb][z], p[2 * kb + 1][z]);
            }
    }
    if (edge && __any_sync(kFull, odd)) {
        // The columns that do see such a row are NaN in its dims.
#pragma unroll 1
        for (int row = max(shown, 0); row < min(rows, kRows); ++row)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const uint32_t code = v[row * kHeadDim + ((g ^ (row & 7)) << 4) + i];
                if ((code & 0x7fu) == 0x7fu) {
#pragma unroll
                    for (int z = 0; z < Z; ++z)
#pragma unroll
                        for (int e = 0; e < 2; ++e)
                            if (row < lim[z][e]) c.o[i >> 1][z][2 * (i & 1) + e] = __uint_as_float(0x7fffffffu);
                }
            }
    }
}

// Factor that joins a state to others of this maximum; of its O besides 2^(scale - the largest scale).
__device__ __forceinline__ float factor(float x, float most) { return x == -INFINITY ? 0.f : ex2(x - most); }

// What turns O into the output: 1 / sum times 2^(scale - 127 - kShift), 0 for no rows. That power may be 2^-133, below the
// least normal number, where O / sum times it is a normal bf16 value: it is two factors of about its root, and O is multiplied by
// `first` and then by `last`. (A sum is 1 to 2^39, so both are normal.)
struct Final {
    float first, last;
};
__device__ __forceinline__ Final final_scale(float scale, float sum)
{
    const int e = (int)scale - 127 - (int)kShift, half = e / 2;
    return Final{sum == 0.f ? 0.f : exp2i(half) / sum, exp2i(e - half)};
}
__device__ __forceinline__ float4 final4(float4 x, Final z)
{
    return make_float4(x.x * z.first * z.last, x.y * z.first * z.last, x.z * z.first * z.last, x.w * z.first * z.last);
}

template <bool F16>
__device__ __forceinline__ uint2 pack4(float4 x, float z)
{
    if (F16) return make_uint2(half2_of(x.x * z, x.y * z), half2_of(x.z * z, x.w * z));
    return make_uint2(pack_bf16(x.x * z, x.y * z), pack_bf16(x.z * z, x.w * z));
}

__device__ __forceinline__ int bank_of(int t) { return (t & 1) | (t & 2) << 1; }

// Where piece k of the unit that starts in CTA c0 lies.
__device__ __forceinline__ int64_t piece_at(int c0, int k) { return (int64_t)(c0 + k) * 2 + (k == 0); }

// The cut units of the kernel of many tokens, after it (all threads of all CTAs): a warp has 8 rows and 16 dims of a unit at
// once, a lane 4 dims of a row; kJoin pieces on the way at once, in their order. `units`: shared.
template <bool F16, int kThreads>
__device__ __forceinline__ void join_chunks(const QuantAttnArgs& a, const ChunkJobs& x, int nctas, int4* units)
{
    constexpr int kUnits = kChunkCounters, kJoin = 8, kWarps = kThreads / 32;
    static_assert(kUnits % 32 == 0 && kUnits <= kThreads, "a thread a unit");
    const int tid = threadIdx.x, warp = uniform(tid >> 5), lane = tid & 31;
    int* ends = reinterpret_cast<int*>(units + kUnits);  // [kUnits] the tasks up to a unit's last; then its warps' sums
    int* sums = ends + kUnits;
    int tasks = 0;
    if (tid < kUnits) {
        const int n = tid < nctas ? __ldcg(x.done + tid) : 0;
        int4 u = make_int4(0, 0, 0, 0);
        if (n >= kJobStarts) u = __ldcg(x.jobs + tid);
        if (n >= kJobStarts && n == u.w + kJobStarts &&
            in_bounds(u.x >= 0 && u.x + u.y <= a.T && u.y * a.G <= kChunkRows && u.z < a.Hkv && tid + u.w <= nctas, a.status))
            tasks = (u.y * a.G + 7) / 8 * 8;
        units[tid] = u;
        int up = tasks;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int y = __shfl_up_sync(kFull, up, o);
            if (lane >= o) up += y;
        }
        ends[tid] = up;
        if (lane == 31) sums[warp] = up;
    }
    __syncthreads();
    int before = 0, total = 0;
#pragma unroll
    for (int i = 0; i < kUnits / 32; ++i) {
        before += i < warp ? sums[i] : 0;
        total += sums[i];
    }
    if (total == 0) return;
    __syncthreads();
    if (tid < kUnits) ends[tid] += before;
    __syncthreads();
    const int low = kChunkTile / a.G * a.G;
#pragma unroll 1
    for (int task = warp * nctas + blockIdx.x; task < total; task += kWarps * nctas) {
        int c0 = 0, hi = kUnits - 1;  // the first unit that ends after the task
        while (c0 < hi) {
            const int mid = (c0 + hi) >> 1;
            if (ends[mid] > task)
                hi = mid;
            else
                c0 = mid + 1;
        }
        const int4 u = units[c0];
        const int rows = u.y * a.G, i = task - (ends[c0] - (rows + 7) / 8 * 8), row = (i >> 3) * 8 + (lane & 7), dim4 = (i & 7) * 4 + (lane >> 3);
        if (row >= rows) continue;
        const int at = row < low ? row : row - low + kChunkTile;
        float top = -INFINITY, sum = 0.f;
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 1
        for (int k0 = 0; k0 < u.w; k0 += kJoin) {
            float2 ml[kJoin];
            float4 o[kJoin];
#pragma unroll
            for (int k = 0; k < kJoin; ++k) {
                const int64_t piece = piece_at(c0, min(k0 + k, u.w - 1));
                ml[k] = __ldcg(x.ml + piece * kChunkRows + at);
                o[k] = __ldcg(x.o + (piece * (kHeadDim / 4) + dim4) * kChunkRows + at);
            }
            float now = top;
#pragma unroll
            for (int k = 0; k < kJoin; ++k) now = fmaxf(now, ml[k].x);
            const float old = top == -INFINITY ? 0.f : ex2((top - now) * x.qscale);
            sum *= old;
            v = make_float4(v.x * old, v.y * old, v.z * old, v.w * old);
#pragma unroll
            for (int k = 0; k < kJoin; ++k) {
                if (k0 + k >= u.w || (ml[k].x == -INFINITY && ml[k].y == 0.f)) continue;  // a piece that the row does not see
                const float f = ml[k].x == -INFINITY ? 0.f : ex2((ml[k].x - now) * x.qscale);
                sum = fmaf(ml[k].y, f, sum);
                v = make_float4(fmaf(o[k].x, f, v.x), fmaf(o[k].y, f, v.y), fmaf(o[k].z, f, v.z), fmaf(o[k].w, f, v.w));
            }
            top = now;
        }
        const int token = row / a.G;
        const int64_t to = ((int64_t)(u.x + token) * a.H + u.z * a.G + (row - token * a.G)) * kHeadDim + 4 * dim4;
        *reinterpret_cast<uint2*>(a.out + to) = pack4<F16>(v, sum == 0.f ? 0.f : x.back / sum);
    }
}

template <bool F16, int Z>
__global__ void __launch_bounds__(Cfg<Z>::kThreads, 1)
    quant_attn_kernel(const __grid_constant__ QuantAttnArgs a, const __grid_constant__ CacheMaps maps, const __grid_constant__ QuantWork w, int nctas,
                      int alone, const __grid_constant__ ChunkJobs chunks)
{
    using C = Cfg<Z>;
    constexpr int kWarps = C::kWarps, kStages = C::kStages, kCols = C::kCols;
    extern __shared__ __align__(1024) unsigned char sm[];
    if (smem_u32(sm) & 1023) {  // never: the swizzled tiles need it
        if (threadIdx.x == 0) report(a, DKV_DEV_TMA_TIMEOUT);
        return;
    }
    const int tid = threadIdx.x, warp = uniform(tid >> 5), lane = tid & 31, c = blockIdx.x, g = lane >> 2, t = lane & 3;
    uint64_t* full = reinterpret_cast<uint64_t*>(sm + C::kOffBars) + warp * kStages;
    volatile int* misc = reinterpret_cast<volatile int*>(sm + C::kOffMisc);
    float* sums = reinterpret_cast<float*>(sm + C::kOffSum);
    State* states = reinterpret_cast<State*>(sm + C::kOffSum);
    unsigned char* ring = sm + warp * kStages * kStageBytes;
    unsigned char* scales = sm + C::kOffScales + warp * kStages * 2 * kRows;
    uint32_t* factors = reinterpret_cast<uint32_t*>(sm + C::kOffFactors) + warp * kRows;
    if (lane == 0)
        for (int s = 0; s < kStages; ++s) mbar_init(smem_u32(full + s), 1);
    if (tid == 0) misc[0] = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    // alone: this kernel was started before the ones before it had completed, and waits for them (and the begin
    // kernel). Else it follows the kernel of many tokens, which started after the ones before the call had: what they
    // wrote may be read, and the wait is for the counters. The fence drops what this SM's L1 holds from before.
    if (alone) pdl_wait();
    asm volatile("fence.acq_rel.gpu;" ::: "memory");
    pdl_launch_dependents();
    if (c == nctas - 1) check(a);
    int group;
    const Extent head = count_cost<Z>(a, reinterpret_cast<int64_t*>(sm), reinterpret_cast<int64_t*>(sm + C::kOffSum), nctas, group);
    Walk k;
    if (seek(a, head, reinterpret_cast<const int64_t*>(sm), group, c, k)) {
        fence_proxy_async_smem();  // the sums of tiles lie in the rings, which the copies write next
        __syncthreads();
        Walk f = k;              // ahead of k by the ring's stages
        int fj = f.j0 + warp, stage = 0, used = 0, fetched = 0, rows0 = 0, rows1 = 0, ahead = 0;  // ahead: tiles of f since its pages were read
        bool left = true, ok = true;
        const uint64_t pol = evict_first_policy();
        const int log_P = 31 - __clz(a.P), box = min(a.P, kRows);
        uint4 qx[Z][4];  // the unit's columns as they lie in memory
        auto load_q = [&] {
#pragma unroll
            for (int z = 0; z < Z; ++z) {
                const int x = 8 * z + g, token = x / a.G, j = x - token * a.G;
                const bool live = token < k.n && in_bounds(k.t + token < a.T && k.g * a.G + j < a.H, a.status);
                load_column(a.q + (int64_t)(k.t + token) * a.q_stride + (k.g * a.G + j) * kHeadDim + 32 * t, live, qx[z]);
            }
        };
        load_q();
        // The next tile on its way. Each lane knows the pool rows of one of the next 32 tiles (of its two halves, where pages have
        // 16 rows); a bad page's are behind the pool, from where zeros come.
        auto fetch = [&] {
            if (!left) return;
            while (fj >= f.j1) {
                left = f.more();
                if (!left) return;
                f.next(a);
                fj = f.j0 + warp;
                ahead = 0;
            }
            if ((ahead & 31) == 0) {
                const int h = f.b * a.Hkv + f.g;
                const int64_t row = ((int64_t)fj + (int64_t)kWarps * lane) * kRows;
                const bool mine = row < f.rows && in_bounds(h >= 0 && h < a.B * a.Hkv && row / a.P < a.max_pages, a.status);
                const bool second = mine && a.P < kRows && row + a.P < f.rows;
                const int32_t* at = a.table + (int64_t)h * a.max_pages + (mine ? (int)row >> log_P : 0);
                const int p0 = mine ? at[0] : 0, p1 = second ? at[1] : 0;
                const bool bad0 = p0 < 0 || p0 >= a.num_pages, bad1 = p1 < 0 || p1 >= a.num_pages;
                if (bad0 || bad1) report(a, DKV_DEV_PAGE_RANGE);
                rows0 = bad0 ? -1 : (p0 << log_P) + ((int)row & (a.P - 1));
                rows1 = bad1 ? -1 : p1 << log_P;
            }
            const int r0 = __shfl_sync(kFull, rows0, ahead & 31), r1 = __shfl_sync(kFull, rows1, ahead & 31);
            ++ahead;
            const int rows = f.rows - fj * kRows, boxes = rows <= 0 ? 0 : a.P < kRows && rows > a.P ? 2 : 1;
            fj += kWarps;
            ++fetched;
            if (lane == 0) {
                const uint32_t bar = smem_u32(full + stage), dst = smem_u32(ring + stage * kStageBytes);
                unsigned char* sc = scales + stage * 2 * kRows;
                mbar_arrive_expect_tx(bar, boxes * 2 * box * kHeadDim + ((boxes > 0 && r0 >= 0) + (boxes > 1 && r1 >= 0)) * 2 * box);
#pragma unroll 1
                for (int x = 0; x < boxes; ++x) {
                    const int r = x ? r1 : r0, y = r < 0 ? a.num_pages * a.P : r;
                    tma_box(dst + x * box * kHeadDim, &maps.k, 0, y, bar, pol);
                    tma_box(dst + kTileBytes + x * box * kHeadDim, &maps.v, 0, y, bar, pol);
                    if (r >= 0) {
                        bulk_g2s(smem_u32(sc) + x * box, a.Ks + y, box, bar, pol);
                        bulk_g2s(smem_u32(sc) + kRows + x * box, a.Vs + y, box, bar, pol);
                    } else {
                        for (int i = 0; i < box; ++i) sc[x * box + i] = sc[kRows + x * box + i] = 1;
                    }
                }
            }
            stage = stage + 1 == kStages ? 0 : stage + 1;
            __syncwarp();
        };
        for (int s = 0; s < kStages; ++s) fetch();
        int at_stage = 0;
        uint32_t phases = 0;  // bit s: the parity of stage s's next tile
#pragma unroll 1
        for (;;) {
            const int cols = k.n * a.G;
            Acc<Z> acc;
            uint32_t q[Z][16];
            float cs[Z][2];
            int lim[Z][2];
#pragma unroll
            for (int z = 0; z < Z; ++z) {
                float back;  // (of column g)
                scale_column<F16>(qx[z], q[z], back);
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int y = 8 * z + 2 * t + e;
                    // Positive and finite, whatever q's size and the scale are (their product may pass fp32's range while the
                    // scores do not, as those of a q or K of zeros): 0 or infinity times an infinite or a zero score were NaN. At the least
                    // number, 2^-149, scores are below 2^-21, as they should be; at the largest those above the others have all weight.
                    cs[z][e] = fminf(fmaxf(__shfl_sync(kFull, back, 8 * t + 4 * e) * a.qscale, 0x1p-149f), 0x1.fffffep127f);
                    lim[z][e] = y < cols ? sees(a, k.len, k.n, y / a.G) : k.rows;
                    acc.top[z][e] = -INFINITY;
                    acc.scale[z][e] = 0;
                    acc.l[z][e] = 0.f;
                }
            }
#pragma unroll
            for (int i = 0; i < 8; ++i)
#pragma unroll
                for (int z = 0; z < Z; ++z)
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc.o[i][z][e] = 0.f;
            const int shown = sees(a, k.len, k.n, 0);
#pragma unroll 1
            for (int j = k.j0 + warp; j < k.j1; j += kWarps) {
                if (ok && !__all_sync(kFull, mbar_wait(smem_u32(full + at_stage), (phases >> at_stage) & 1))) {
                    ok = false;
                    misc[0] = 1;
                    if (lane == 0) report(a, DKV_DEV_TMA_TIMEOUT);
                }
                if (!ok) break;
                ++used;
                phases ^= 1u << at_stage;
                const int r0 = j * kRows;
                int tl[Z][2];
#pragma unroll
                for (int z = 0; z < Z; ++z)
#pragma unroll
                    for (int e = 0; e < 2; ++e) tl[z][e] = lim[z][e] - r0;
                const unsigned char* tile = ring + at_stage * kStageBytes;
                tile_step<Z>(acc, q, cs, tile, tile + kTileBytes, scales + at_stage * 2 * kRows, factors, tl, shown - r0, k.rows - r0);
                at_stage = at_stage + 1 == kStages ? 0 : at_stage + 1;
                __syncwarp();
                fetch();
            }
            // The warps' states: joined in the order of the warps, 64 dims at a time.
            const int active = min(kWarps, k.j1 - k.j0);
#pragma unroll
            for (int z = 0; z < Z; ++z)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
#pragma unroll
                    for (int o = 4; o < 32; o <<= 1) acc.l[z][e] += __shfl_xor_sync(kFull, acc.l[z][e], o);
                    if (g == 0) states[warp * kCols + 8 * z + 2 * t + e] = State{acc.top[z][e] * cs[z][e], acc.l[z][e], (float)acc.scale[z][e], 0.f};
                }
            __syncthreads();
            const bool aborted = misc[0];
            const int mine = tid >> 4, chunk = tid & 15;  // this thread sums 4 dims of column `mine`: chunk 2 g + i of lane g's 8
            State total{-INFINITY, 0.f, 0.f, 0.f};
            float f0[Z][2], up[Z][2];  // of this lane's columns: what joins its O; the largest scale
#pragma unroll
            for (int z = 0; z < Z; ++z) f0[z][0] = f0[z][1] = -INFINITY, up[z][0] = up[z][1] = 0.f;
#pragma unroll 4
            for (int x = 0; x < active; ++x) {
                if (mine < kCols) {
                    total.top = fmaxf(total.top, states[x * kCols + mine].top);
                    total.scale = fmaxf(total.scale, states[x * kCols + mine].scale);
                }
#pragma unroll
                for (int z = 0; z < Z; ++z)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const State y = states[x * kCols + 8 * z + 2 * t + e];
                        f0[z][e] = fmaxf(f0[z][e], y.top);
                        up[z][e] = fmaxf(up[z][e], y.scale);
                    }
            }
            if (mine < kCols)
#pragma unroll 4
                for (int x = 0; x < active; ++x) {
                    const State y = states[x * kCols + mine];
                    total.sum += y.sum * factor(y.top, total.top);
                }
#pragma unroll
            for (int z = 0; z < Z; ++z)
#pragma unroll
                for (int e = 0; e < 2; ++e) f0[z][e] = factor(acc.top[z][e] * cs[z][e], f0[z][e]) * ex2((float)acc.scale[z][e] - up[z][e]);
            const bool whole = k.whole(), live = mine < cols && !aborted;
            const int token = mine / a.G, head_j = mine - token * a.G;
            uint16_t* out = a.out + ((int64_t)(k.t + token) * a.H + k.g * a.G + head_j) * kHeadDim;
            const int64_t slot = (int64_t)c * 2 + (k.j0 == 0);
            const Final z = final_scale(total.scale, total.sum);
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                __syncthreads();
                if (warp < active) {
#pragma unroll
                    for (int z = 0; z < Z; ++z)
#pragma unroll
                        for (int e = 0; e < 2; ++e)
#pragma unroll
                            for (int i = 0; i < 2; ++i) {
                                // (chunks are permuted so that a quarter-warp's eight lie in different banks)
                                const float f1 = f0[z][e], *x = acc.o[4 * half + 2 * i][z], *y = acc.o[4 * half + 2 * i + 1][z];
                                reinterpret_cast<float4*>(sums + (warp * kCols + 8 * z + 2 * t + e) * 64)[(2 * g + i) ^ bank_of(t)] =
                                    make_float4(x[e] * f1, x[2 + e] * f1, y[e] * f1, y[2 + e] * f1);
                            }
                }
                __syncthreads();
                if (live) {
                    const int at = chunk ^ bank_of((mine >> 1) & 3);
                    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
                    for (int x = 0; x < active; ++x) {
                        const float4 y = reinterpret_cast<const float4*>(sums + (x * kCols + mine) * 64)[at];
                        v = make_float4(v.x + y.x, v.y + y.y, v.z + y.z, v.w + y.w);
                    }
                    const int dim = 16 * (chunk >> 1) + 8 * half + 4 * (chunk & 1);
                    if (whole)
                        *reinterpret_cast<uint2*>(out + dim) = pack4<F16>(final4(v, z), 1.f);
                    else
                        __stcg(w.o + (slot * kMostCols + mine) * (kHeadDim / 4) + dim / 4, v);
                }
            }
            if (!whole) {
                if (live && chunk == 0) __stcg(reinterpret_cast<float4*>(w.state + slot * kMostCols + mine), make_float4(total.top, total.sum, total.scale, 0.f));
                const int c0 = cta_of(head, k.start), pieces = cta_of(head, k.start + k.tiles - 1) - c0 + 1;
                __threadfence();
                __syncthreads();
                if (tid == 0) {
                    pdl_wait();  // the counters are cleared
                    misc[1] = !aborted && atomicAdd(w.done + c0, 1) == pieces - 1;
                }
                __syncthreads();
                if (misc[1] && mine < cols && in_bounds(c0 >= 0 && c0 + pieces <= nctas, a.status)) {
                    // kJoin pieces on the way at once, in the order of the CTAs.
                    __threadfence();
                    constexpr int kJoin = 8;
                    State all{-INFINITY, 0.f, 0.f, 0.f};
                    float4 v[2] = {make_float4(0.f, 0.f, 0.f, 0.f), make_float4(0.f, 0.f, 0.f, 0.f)};
#pragma unroll 1
                    for (int x0 = 0; x0 < pieces; x0 += kJoin) {
                        float4 y[kJoin], u[kJoin][2];
#pragma unroll
                        for (int x = 0; x < kJoin; ++x) {
                            const int64_t piece = piece_at(c0, min(x0 + x, pieces - 1)) * kMostCols + mine;
                            y[x] = __ldcg(reinterpret_cast<const float4*>(w.state + piece));
                            u[x][0] = __ldcg(w.o + piece * (kHeadDim / 4) + 2 * chunk);
                            u[x][1] = __ldcg(w.o + piece * (kHeadDim / 4) + 2 * chunk + 1);
                        }
                        State now = all;
#pragma unroll
                        for (int x = 0; x < kJoin; ++x) {
                            now.top = fmaxf(now.top, y[x].x);
                            now.scale = fmaxf(now.scale, y[x].z);
                        }
                        const float old = factor(all.top, now.top), old_o = old * ex2(all.scale - now.scale);
                        now.sum *= old;
#pragma unroll
                        for (int i = 0; i < 2; ++i) v[i] = make_float4(v[i].x * old_o, v[i].y * old_o, v[i].z * old_o, v[i].w * old_o);
#pragma unroll
                        for (int x = 0; x < kJoin; ++x) {
                            if (x0 + x >= pieces) break;
                            const float fl = factor(y[x].x, now.top), fo = fl * ex2(y[x].z - now.scale);
                            now.sum += y[x].y * fl;
#pragma unroll
                            for (int i = 0; i < 2; ++i)
                                v[i] = make_float4(fmaf(u[x][i].x, fo, v[i].x), fmaf(u[x][i].y, fo, v[i].y), fmaf(u[x][i].z, fo, v[i].z),
                                                   fmaf(u[x][i].w, fo, v[i].w));
                        }
                        all = now;
                    }
                    const Final y = final_scale(all.scale, all.sum);
                    const uint2 lo = pack4<F16>(final4(v[0], y), 1.f), hi = pack4<F16>(final4(v[1], y), 1.f);
                    *reinterpret_cast<uint4*>(out + 8 * chunk) = make_uint4(lo.x, lo.y, hi.x, hi.y);
                }
            }
            __syncthreads();  // sums and misc[1] are read
            if (!k.more()) break;
            k.next(a);
            load_q();
        }
        // Copies in flight land (or run out of time) before the CTA exits.
        for (; used < fetched; ++used) {
            mbar_wait(smem_u32(full + at_stage), (phases >> at_stage) & 1);
            phases ^= 1u << at_stage;
            at_stage = at_stage + 1 == kStages ? 0 : at_stage + 1;
        }
    }
    pdl_wait();  // the call is not over before its begin kernel, and the one of many tokens
    if (!alone) {
        __syncthreads();
        join_chunks<F16, C::kThreads>(a, chunks, nctas, reinterpret_cast<int4*>(sm + C::kOffSum));  // (where no copy writes)
    }
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

// A pool of bytes: boxes of up to kRows rows of 128, in one page.
cudaError_t make_pool_map(const QuantAttnArgs& a, const uint8_t* pool, bool short_boxes, CUtensorMap* map)
{
    PFN_cuTensorMapEncodeTiled_v12000 enc = encode_tiled();
    if (!enc) return cudaErrorNotSupported;
    const cuuint32_t rows = (cuuint32_t)std::min(a.P, kRows);
    const cuuint64_t dim[2] = {(cuuint64_t)kHeadDim, (cuuint64_t)a.num_pages * a.P};
    const cuuint64_t stride[1] = {(cuuint64_t)kHeadDim};
    const cuuint32_t box[2] = {(cuuint32_t)kHeadDim, short_boxes ? rows / 2 : rows};
    const cuuint32_t elem[2] = {1, 1};
    return enc(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<uint8_t*>(pool), dim, stride, box, elem, CU_TENSOR_MAP_INTERLEAVE_NONE,
               CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS
               ? cudaSuccess
               : cudaErrorInvalidValue;
}

template <bool F16, int Z>
cudaError_t setup_few()
{
    return cudaFuncSetAttribute(quant_attn_kernel<F16, Z>, cudaFuncAttributeMaxDynamicSharedMemorySize, Cfg<Z>::kSmemBytes);
}

template <bool F16>
cudaError_t launch_few(const QuantAttnArgs& a, const CacheMaps& maps, const QuantWork& w, int nctas, int alone,
                       const ChunkJobs& chunks, cudaStream_t st)
{
    if (a.few * a.G <= Cfg<1>::kCols)
        return launch_pdl(quant_attn_kernel<F16, 1>, nctas, Cfg<1>::kThreads, Cfg<1>::kSmemBytes, st, a, maps, w, nctas, alone, chunks);
    return launch_pdl(quant_attn_kernel<F16, 2>, nctas, Cfg<2>::kThreads, Cfg<2>::kSmemBytes, st, a, maps, w, nctas, alone, chunks);
}

}  // namespace

int64_t quant_workspace_bytes() { return kWorkBytes + chunk_workspace_bytes(); }

cudaError_t quant_setup()
{
    cudaError_t e = setup_few<false, 1>();
    if (e == cudaSuccess) e = setup_few<true, 1>();
    if (e == cudaSuccess) e = setup_few<false, 2>();
    if (e == cudaSuccess) e = setup_few<true, 2>();
    return e;
}

cudaError_t launch_quant_attn(const QuantAttnArgs& a, bool short_boxes, cudaStream_t st)
{
    int sms = 0;
    cudaError_t e = page_setup(&sms);
    if (e != cudaSuccess) return e;
    const int nctas = std::min(sms, kMaxCtas);
    CacheMaps maps;
    if ((e = make_pool_map(a, a.Kp, short_boxes, &maps.k)) != cudaSuccess) return e;
    if ((e = make_pool_map(a, a.Vp, short_boxes, &maps.v)) != cudaSuccess) return e;
    unsigned char* base = static_cast<unsigned char*>(a.work);
    QuantWork w;
    w.done = reinterpret_cast<int32_t*>(base);
    w.jobs = reinterpret_cast<int4*>(base + kOffJobs);
    w.state = reinterpret_cast<State*>(base + kOffState);
    w.o = reinterpret_cast<float4*>(base + kOffO);
    w.chunk = reinterpret_cast<int32_t*>(base + kWorkBytes);
    QuantAttnArgs few = a;
    // Sequences of up to 16 columns; beside the kernel of many tokens, of up to 8, which take a faster form of this one (the
    // step of turns and next tokens of 4 columns: 140 us with 16, 134 with 8).
    few.few = std::min(a.most, (a.most * a.G <= kMostCols ? kMostCols : Cfg<1>::kCols) / a.G);
    const int alone = a.most <= few.few;
    if ((e = launch_pdl(quant_begin_kernel, 1, 256, 0, st, w, alone)) != cudaSuccess) return e;
    ChunkJobs chunks{};
    if (!alone) {
        ChunkArgs c{};
        c.q = a.q;
        c.q_stride = a.q_stride;
        c.cu = a.cu;
        c.table = a.table;
        c.len = a.len;
        c.Kp = reinterpret_cast<uint16_t*>(const_cast<uint8_t*>(a.Kp));
        c.Vp = reinterpret_cast<uint16_t*>(const_cast<uint8_t*>(a.Vp));
        c.out = a.out;
        c.status = a.status;
        c.work = w.chunk;
        c.T = a.T;
        c.B = a.B;
        c.H = a.H;
        c.Hkv = a.Hkv;
        c.G = a.G;
        c.P = a.P;
        c.num_pages = a.num_pages;
        c.max_pages = a.max_pages;
        c.causal = a.causal;
        c.fp16 = a.fp16;
        c.qscale = a.fp16 ? 2 * a.qscale : a.qscale;  // (fp16 keys enter at half their value)
        c.Ks = a.Ks;
        c.Vs = a.Vs;
        c.least = few.few + 1;
        c.most = a.most;
        c.jobs = w.jobs;
        chunks = chunk_jobs(c);
        if ((e = launch_chunk8(c, nctas, short_boxes, st)) != cudaSuccess) return e;
    }
    return a.fp16 ? launch_few<true>(few, maps, w, nctas, alone, chunks, st) : launch_few<false>(few, maps, w, nctas, alone, chunks, st);
}

}  // namespace dkv
