// Attention of a step's new tokens over 8-bit pages: token i of the n new ones of sequence b attends,
// per query head, to the first len - n + i + 1 rows of its slab (causal) or to all len rows,
//   o = sum_r softmax_r(scale 2^ek_r q.k_r) 2^ev_r v_r,   k_r, v_r e4m3 values, 2^ek_r, 2^ev_r their rows' scales.
//
// Unit of work: 16 columns (token x head of the group, column = token G + head) of one sequence and KV
// head, against the cache rows that its last token sees, in tiles of 32 rows. All (unit, tile) pairs,
// unit after unit, are cut into contiguous equal shares, one a CTA, one CTA an SM; a CTA's 8 warps take the tiles
// of its part of a unit in turn, each through a ring of its own, and are joined at its end. A unit that
// lies in several CTAs is joined by the one that finishes last.
//
//   quant_begin_kernel  clears the counters, checks what lives on the device.
//   quant_attn_kernel   starts beside it, and waits for it only where it counts.
//
// A warp multiplies with the warp-level fp16 products (m16n8k16: 16 columns x 8 rows x 16 dims, then 16
// columns x 8 dims x 16 rows): e4m3 values are fp16 values. The dims of a product may be any order that both
// operands share, so a lane takes 32 dims of K that lie together, and 16 of V: K's bytes convert in place, V's
// pairs of rows after a byte permutation. Tiles lie in shared memory as TMA's 128-byte swizzle puts them, which makes
// these 16-byte reads free of conflicts.
//
// A row's V scale goes into its weight's exponent, x_r + ev_r, so O has a running maximum of its own beside that of the
// scores x_r, which the sum of weights goes by.
#include "dkv_quant.cuh"

#include "dkv_tcgen05.cuh"

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cudaTypedefs.h>

#include <algorithm>
#include <mutex>

namespace dkv {
namespace {

constexpr int kWarps = 8;
constexpr int kThreads = 32 * kWarps;
constexpr int kCols = 16;                  // columns of a unit
constexpr int kRows = 32;                  // cache rows of a tile
constexpr int kTileBytes = kRows * kHeadDim;
constexpr int kStages = 3;                 // ring of a warp
constexpr int kMaxCtas = 160;              // CTAs of the largest grid (the workspace's size)
constexpr float kShift = 7.f;              // weights for the second product are 2^7 larger: fp16 has 2^15 above the slack

// Shared memory, from its 1024-byte aligned start.
constexpr int kStageBytes = 2 * kTileBytes;                            // K, then V
constexpr int kOffSum = kWarps * kStages * kStageBytes;                // float[kWarps][16][64], before that State[kWarps][16]
constexpr int kOffScales = kOffSum + kWarps * kCols * 64 * 4;          // a stage's scale bytes: of K, of V
constexpr int kOffBars = kOffScales + kWarps * kStages * 2 * kRows;
constexpr int kOffMisc = kOffBars + kWarps * kStages * 8;              // int[4]: abort, last
constexpr int kSmemBytes = kOffMisc + 16;
static_assert(kSmemBytes <= 227 * 1024, "fits one CTA");
constexpr int kMaxGroups = kOffSum / 8;    // prefix sums in the rings before their first use

// A column's softmax over some rows: max of x + ev, max of x, sum of 2^(x - top).
struct State {
    float reach, top, sum, pad;
};

// Workspace.
struct QuantWork {
    int32_t* done;  // [kMaxCtas] finished pieces of the unit that starts in CTA c and ends in a later one
    State* state;   // [kMaxCtas][2][16]
    float4* o;      // [kMaxCtas][2][16][32]
    int32_t* chunk; // the workspace of the kernel of many tokens, its counters first
};
constexpr int64_t kOffState = (kMaxCtas * 4 + 255) / 256 * 256, kOffO = kOffState + (int64_t)kMaxCtas * 2 * kCols * sizeof(State),
                  kWorkBytes = kOffO + (int64_t)kMaxCtas * 2 * kCols * kHeadDim * 4;
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

__device__ __forceinline__ int blocks_of(const QuantAttnArgs& a, int n) { return (int)(((int64_t)n * a.G + kCols - 1) / kCols); }

// Cache rows, and tiles, of block i of n tokens over a slab of len rows.
__device__ __forceinline__ int block_rows(const QuantAttnArgs& a, int len, int n, int i)
{
    return sees(a, len, n, min(n, (int)((i * (int64_t)kCols + kCols - 1) / a.G + 1)) - 1);
}
__device__ __forceinline__ int tiles_of(int rows) { return max(1, (int)(((unsigned)rows + kRows - 1) / kRows)); }

__global__ void __launch_bounds__(512) quant_begin_kernel(const __grid_constant__ QuantAttnArgs a, const __grid_constant__ QuantWork w)
{
    const int tid = threadIdx.x;
    pdl_wait();
    pdl_launch_dependents();
    if (tid < kMaxCtas) w.done[tid] = 0;
    if (tid < kChunkCounters) w.chunk[tid] = 0;
    static_assert(kMaxSlots <= 512 && kChunkCounters <= 512, "a thread each");
    if (tid < a.B && (bad_offsets(a, tid) || cu_at(a, tid + 1) - cu_at(a, tid) > a.most)) report(a, DKV_DEV_PAGE_RANGE);
    for (int h = tid; h < a.B * a.Hkv; h += 512) {
        const int b = h / a.Hkv;
        if (cu_at(a, b + 1) > cu_at(a, b) && a.len[h] != slab_len(a, h)) report(a, DKV_DEV_PAGE_RANGE);
    }
}

// ---------------------------------------------------------------- schedule
__device__ __forceinline__ int64_t slab_tiles(const QuantAttnArgs& a, int h)
{
    const int n = tokens_of(a, h / a.Hkv), len = slab_len(a, h);
    int64_t sum = 0;
#pragma unroll 1
    for (int i = 0, nb = blocks_of(a, n); i < nb; ++i) sum += tiles_of(block_rows(a, len, n, i));
    return sum;
}

struct Extent {
    int64_t tiles;
    int parts;
};
__device__ __forceinline__ int64_t divide(int64_t x, int64_t y)
{
    return x <= UINT32_MAX && y <= UINT32_MAX ? (int64_t)((uint32_t)x / (uint32_t)y) : x / y;
}
__device__ __forceinline__ int64_t share_start(const Extent& e, int c) { return divide(e.tiles * c, e.parts); }
__device__ __forceinline__ int cta_of(const Extent& e, int64_t x) { return (int)divide((x + 1) * e.parts - 1, e.tiles); }

// All threads of the CTA: the tiles before every slab (or group of slabs, where there are more than fit), into `before`.
__device__ __forceinline__ Extent count_tiles(const QuantAttnArgs& a, int64_t* before, int64_t* sums, int nctas, int& group)
{
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, slabs = a.B * a.Hkv;
    group = (slabs + kMaxGroups - 1) / kMaxGroups;
    const int groups = (slabs + group - 1) / group, per = (groups + kThreads - 1) / kThreads;
    const int g0 = min(groups, tid * per), g1 = min(groups, g0 + per);
    int64_t mine = 0;
#pragma unroll 1
    for (int x = g0; x < g1; ++x) {
        before[x] = mine;
#pragma unroll 1
        for (int h = x * group; h < min(slabs, (x + 1) * group); ++h) mine += slab_tiles(a, h);
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
    return bad ? Extent{0, 0} : Extent{total, (int)min((int64_t)nctas, total)};
}

// The share of one CTA, unit by unit.
struct Walk {
    int b, g, i, t, n, len;    // sequence, head, block; the sequence's first token, its tokens, the slab's rows
    int rows, tiles, j0, j1;   // of the unit; the CTA's tiles of it
    int64_t start, end;        // of the unit, of the share
    __device__ __forceinline__ void enter(const QuantAttnArgs& a, int64_t off)
    {
        rows = block_rows(a, len, n, i);
        tiles = tiles_of(rows);
        j0 = (int)off;
        j1 = (int)min((int64_t)tiles, end - start);
    }
    __device__ __forceinline__ bool more() const { return start + tiles < end; }
    __device__ __forceinline__ void sequence(const QuantAttnArgs& a)
    {
        t = cu_at(a, b);
        n = tokens_of(a, b);
    }
    __device__ __forceinline__ void next(const QuantAttnArgs& a)
    {
        start += tiles;
        if (++i >= blocks_of(a, n)) {
            i = 0;
            if (++g == a.Hkv) {
                g = 0;
                do ++b;
                while (b < a.B - 1 && tokens_of(a, b) == 0);
                sequence(a);
            }
            len = slab_len(a, b * a.Hkv + g);
        }
        enter(a, 0);
    }
    __device__ __forceinline__ bool whole() const { return j0 == 0 && j1 == tiles; }
};

__device__ __forceinline__ void seek(const QuantAttnArgs& a, const Extent& e, const int64_t* before, int group, int c, Walk& k)
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
    int h = lo * group;
    if (group > 1)
        for (int64_t x; off >= (x = slab_tiles(a, h)); ++h) off -= x;
    k.b = h / a.Hkv;
    k.g = h - k.b * a.Hkv;
    k.sequence(a);
    k.len = slab_len(a, h);
    k.i = 0;
#pragma unroll 1
    for (int x; off >= (x = tiles_of(block_rows(a, k.len, k.n, k.i))); ++k.i) off -= x;
    k.start = pos - off;
    k.enter(a, off);
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

// Bytes of a word that are NaN, as 0xff.
__device__ __forceinline__ uint32_t nan_bytes(uint32_t w) { return __vcmpeq4(w & 0x7f7f7f7fu, 0x7f7f7f7fu); }

__device__ __forceinline__ uint4 lds128(const unsigned char* p)
{
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(smem_u32(p)) : "memory");
    return v;
}

// A lane's half of a column of q (elements 32 t .. 32 t + 31 of 128) as fp16 pairs, scaled by a power of two that
// takes the column's largest element to 2^14 .. 2^15; `back`: its inverse.
template <bool F16>
__device__ __forceinline__ void load_column(const uint16_t* src, bool live, uint32_t (&q)[16], float& back)
{
    uint4 x[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = live ? ld_prev(reinterpret_cast<const uint4*>(src) + i) : make_uint4(0u, 0u, 0u, 0u);
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

// What a lane has of its warp's columns lane / 4 and lane / 4 + 8.
struct Acc {
    float o[16][4];               // dims 32 t + i and 32 t + 16 + i of the one column, then of the other (t = lane % 4)
    float reach[2], top[2], l[2]; // l: of the lane's rows
};

// One tile: scores, softmax, O += P V. lim: the tile's rows that the columns see; rows: those of the unit; `shown`: rows
// that all columns see.
__device__ __forceinline__ void tile_step(Acc& c, const uint32_t (&q)[2][16], const float (&cs)[2], const unsigned char* k, const unsigned char* v,
                                          const unsigned char* scales, const int (&lim)[2], int shown, int rows)
{
    const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    float s[4][4];
#pragma unroll
    for (int nt = 0; nt < 4; ++nt) {
#pragma unroll
        for (int e = 0; e < 4; ++e) s[nt][e] = 0.f;
        const unsigned char* row = k + (8 * nt + g) * kHeadDim;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const uint4 x = lds128(row + (((2 * t + i) ^ g) << 4));
            const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
            for (int y = 0; y < 4; ++y) {
                const int ks = 4 * i + y;  // dims 32 t + 4 ks .. + 3 of every t
                uint32_t b0, b1;
                widen_e4m3(w[y], b0, b1);
                const uint32_t A[4] = {q[0][2 * ks], q[1][2 * ks], q[0][2 * ks + 1], q[1][2 * ks + 1]};
                mma(s[nt], A, b0, b1);
            }
        }
    }
    // Scores in units of the base-2 softmax, and with V's exponents.
    float r[4][4];
#pragma unroll
    for (int nt = 0; nt < 4; ++nt) {
        const uint32_t ku = *reinterpret_cast<const uint16_t*>(scales + 8 * nt + 2 * t), vu = *reinterpret_cast<const uint16_t*>(scales + kRows + 8 * nt + 2 * t);
        const float k0 = scale_of(ku & 255u), k1 = scale_of(ku >> 8);
        const float v0 = (float)(vu & 255u) - 127.f, v1 = (float)(vu >> 8) - 127.f;
#pragma unroll
        for (int z = 0; z < 2; ++z) {
            s[nt][2 * z] *= cs[z] * k0;
            s[nt][2 * z + 1] *= cs[z] * k1;
            r[nt][2 * z] = s[nt][2 * z] + v0;
            r[nt][2 * z + 1] = s[nt][2 * z + 1] + v1;
        }
    }
    if (shown < kRows) {
#pragma unroll
        for (int nt = 0; nt < 4; ++nt)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (8 * nt + 2 * t + (e & 1) >= lim[e >> 1]) s[nt][e] = r[nt][e] = -INFINITY;  // also over NaN
    }
    float mx[2], mr[2];
#pragma unroll
    for (int z = 0; z < 2; ++z) {
        mx[z] = mr[z] = -INFINITY;
#pragma unroll
        for (int nt = 0; nt < 4; ++nt) {
            mx[z] = fmaxf(mx[z], fmaxf(s[nt][2 * z], s[nt][2 * z + 1]));
            mr[z] = fmaxf(mr[z], fmaxf(r[nt][2 * z], r[nt][2 * z + 1]));
        }
#pragma unroll
        for (int o = 1; o < 4; o <<= 1) {
            mx[z] = fmaxf(mx[z], __shfl_xor_sync(kFull, mx[z], o));
            mr[z] = fmaxf(mr[z], __shfl_xor_sync(kFull, mr[z], o));
        }
    }
    // The maxima move only when a score tops them by 2^kSlack.
    const bool up0 = mx[0] - c.top[0] > kSlack, up1 = mx[1] - c.top[1] > kSlack, out0 = mr[0] - c.reach[0] > kSlack, out1 = mr[1] - c.reach[1] > kSlack;
    if (__any_sync(kFull, up0 || up1 || out0 || out1)) {
        if (up0) c.l[0] *= ex2(c.top[0] - mx[0]), c.top[0] = mx[0];
        if (up1) c.l[1] *= ex2(c.top[1] - mx[1]), c.top[1] = mx[1];
        const float a0 = out0 ? ex2(c.reach[0] - mr[0]) : 1.f, a1 = out1 ? ex2(c.reach[1] - mr[1]) : 1.f;
        if (out0) c.reach[0] = mr[0];
        if (out1) c.reach[1] = mr[1];
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            c.o[i][0] *= a0;
            c.o[i][1] *= a0;
            c.o[i][2] *= a1;
            c.o[i][3] *= a1;
        }
    }
    uint32_t p[2][4];
#pragma unroll
    for (int z = 0; z < 2; ++z) {
        const float top = c.top[z] == -INFINITY ? 0.f : c.top[z], reach = (c.reach[z] == -INFINITY ? 0.f : c.reach[z]) - kShift;
#pragma unroll
        for (int nt = 0; nt < 4; ++nt) {
            c.l[z] += ex2(s[nt][2 * z] - top) + ex2(s[nt][2 * z + 1] - top);
            p[nt >> 1][2 * (nt & 1) + z] = half2_of(ex2(r[nt][2 * z] - reach), ex2(r[nt][2 * z + 1] - reach));
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
            if (shown < kRows && row >= shown) {  // 0 NaN is NaN
#pragma unroll
                for (int y = 0; y < 4; ++y) {
                    const uint32_t bad = nan_bytes(w[x][y]);
                    odd |= bad != 0 && row < rows;
                    w[x][y] = row < rows ? w[x][y] & ~bad : 0u;
                }
            }
        }
#pragma unroll
        for (int y = 0; y < 4; ++y) {
            uint32_t b[4], d[4];
            widen_e4m3(__byte_perm(w[0][y], w[1][y], 0x5140), b[0], b[1]);
            widen_e4m3(__byte_perm(w[0][y], w[1][y], 0x7362), b[2], b[3]);
            widen_e4m3(__byte_perm(w[2][y], w[3][y], 0x5140), d[0], d[1]);
            widen_e4m3(__byte_perm(w[2][y], w[3][y], 0x7362), d[2], d[3]);
#pragma unroll
            for (int i = 0; i < 4; ++i) mma(c.o[4 * y + i], p[kb], b[i], d[i]);
        }
    }
    if (shown < kRows && __any_sync(kFull, odd)) {
        // The columns that do see such a row are NaN in its dims.
#pragma unroll 1
        for (int row = max(shown, 0); row < min(rows, kRows); ++row)
#pragma unroll
            for (int i = 0; i < 32; ++i) {
                const uint32_t code = v[row * kHeadDim + (((2 * t + (i >> 4)) ^ (row & 7)) << 4) + (i & 15)];
                if ((code & 0x7fu) == 0x7fu) {
                    if (row < lim[0]) c.o[i & 15][i >> 4] = __uint_as_float(0x7fffffffu);
                    if (row < lim[1]) c.o[i & 15][2 + (i >> 4)] = __uint_as_float(0x7fffffffu);
                }
            }
    }
}

// Factors that join states: that of O, 2^(reach - R), and that of the sum, 2^(top - M).
__device__ __forceinline__ float factor(float x, float most) { return x == -INFINITY ? 0.f : ex2(x - most); }

// What turns O (relative to reach) into the output: 2^(reach - kShift - top) / sum; 0 for no rows.
__device__ __forceinline__ float final_scale(float reach, float top, float sum) { return sum == 0.f ? 0.f : ex2(reach - kShift - top) / sum; }

template <bool F16>
__device__ __forceinline__ uint2 pack4(float4 x, float z)
{
    if (F16) return make_uint2(half2_of(x.x * z, x.y * z), half2_of(x.z * z, x.w * z));
    return make_uint2(pack_bf16(x.x * z, x.y * z), pack_bf16(x.z * z, x.w * z));
}

// Where piece k of the unit that starts in CTA c0 lies.
__device__ __forceinline__ int64_t piece_at(int c0, int k) { return (int64_t)(c0 + k) * 2 + (k == 0); }

template <bool F16>
__global__ void __launch_bounds__(kThreads, 1)
    quant_attn_kernel(const __grid_constant__ QuantAttnArgs a, const __grid_constant__ CacheMaps maps, const __grid_constant__ QuantWork w, int nctas)
{
    extern __shared__ __align__(1024) unsigned char sm[];
    if (smem_u32(sm) & 1023) {  // never: the swizzled tiles need it
        if (threadIdx.x == 0) report(a, DKV_DEV_TMA_TIMEOUT);
        return;
    }
    const int tid = threadIdx.x, warp = uniform(tid >> 5), lane = tid & 31, c = blockIdx.x, g = lane >> 2, t = lane & 3;
    uint64_t* full = reinterpret_cast<uint64_t*>(sm + kOffBars) + warp * kStages;
    volatile int* misc = reinterpret_cast<volatile int*>(sm + kOffMisc);
    float* sums = reinterpret_cast<float*>(sm + kOffSum);
    State* states = reinterpret_cast<State*>(sm + kOffSum);
    unsigned char* ring = sm + warp * kStages * kStageBytes;
    unsigned char* scales = sm + kOffScales + warp * kStages * 2 * kRows;
    if (lane == 0)
        for (int s = 0; s < kStages; ++s) mbar_init(smem_u32(full + s), 1);
    if (tid == 0) misc[0] = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    // What the kernels before the begin kernel wrote may be read (it started after they had completed, and
    // this one after that); the fence drops what this SM's L1 holds from before. The counters may not, before pdl_wait().
    asm volatile("fence.acq_rel.gpu;" ::: "memory");
    int group;
    const Extent head = count_tiles(a, reinterpret_cast<int64_t*>(sm), reinterpret_cast<int64_t*>(sm + kOffSum), nctas, group);
    if (c < head.parts) {
        Walk k;
        seek(a, head, reinterpret_cast<const int64_t*>(sm), group, c, k);
        fence_proxy_async_smem();  // the sums of tiles lie in the rings, which the copies write next
        __syncthreads();
        Walk f = k;                 // ahead of k by the ring's stages
        int fj = f.j0 + warp, fetched = 0, used = 0, page0 = 0, page1 = 0, ahead = 0;  // ahead: tiles of f since its pages were read
        bool left = true, ok = true;
        const uint64_t pol = evict_first_policy();
        auto fetch = [&] {
            while (left && fj >= f.j1) {
                left = f.more();
                if (left) {
                    f.next(a);
                    fj = f.j0 + warp;
                    ahead = 0;
                }
            }
            if (!left) return;
            const int h = f.b * a.Hkv + f.g;
            if ((ahead & 31) == 0) {
                const int64_t row = ((int64_t)fj + (int64_t)kWarps * lane) * kRows;
                const bool mine = row < f.rows && in_bounds(h >= 0 && h < a.B * a.Hkv && row / a.P < a.max_pages, a.status);
                const int32_t* at = a.table + (int64_t)h * a.max_pages + (mine ? (int)row / a.P : 0);
                page0 = mine ? at[0] : 0;
                page1 = mine && a.P < kRows && row + a.P < f.rows ? at[1] : 0;
            }
            const int p0 = __shfl_sync(kFull, page0, ahead & 31), p1 = __shfl_sync(kFull, page1, ahead & 31);
            ++ahead;
            const int s = fetched % kStages, rows = f.rows - fj * kRows, box = min(a.P, kRows);
            ++fetched;
            const int boxes = rows <= 0 ? 0 : a.P < kRows && rows > a.P ? 2 : 1;
            __syncwarp();
            if (lane == 0) {
                const uint32_t bar = smem_u32(full + s), dst = smem_u32(ring + s * kStageBytes);
                unsigned char* sc = scales + s * 2 * kRows;
                const bool good0 = p0 >= 0 && p0 < a.num_pages, good1 = p1 >= 0 && p1 < a.num_pages;
                mbar_arrive_expect_tx(bar, boxes * 2 * box * kHeadDim + ((boxes > 0 && good0) + (boxes > 1 && good1)) * 2 * box);
                for (int x = 0; x < boxes; ++x) {
                    const bool good = x ? good1 : good0;
                    const int y = good ? (x ? p1 : p0) * a.P + (x ? 0 : fj * kRows % a.P) : a.num_pages * a.P;  // behind the pool: zeros
                    tma_box(dst + x * box * kHeadDim, &maps.k, 0, y, bar, pol);
                    tma_box(dst + kTileBytes + x * box * kHeadDim, &maps.v, 0, y, bar, pol);
                    if (good) {
                        bulk_g2s(smem_u32(sc) + x * box, a.Ks + y, box, bar, pol);
                        bulk_g2s(smem_u32(sc) + kRows + x * box, a.Vs + y, box, bar, pol);
                    } else {
                        report(a, DKV_DEV_PAGE_RANGE);
                        for (int i = 0; i < box; ++i) sc[x * box + i] = sc[kRows + x * box + i] = 127;
                    }
                }
            }
            fj += kWarps;
            __syncwarp();
        };
        for (int s = 0; s < kStages; ++s) fetch();
#pragma unroll 1
        for (;;) {
            // The unit's columns of this lane.
            const int col0 = k.i * kCols, cols = min((int64_t)kCols, (int64_t)k.n * a.G - col0);
            Acc acc;
            uint32_t q[2][16];
            float cs[2];
            int lim[2];
#pragma unroll
            for (int z = 0; z < 2; ++z) {
                const int x = g + 8 * z, token = (col0 + x) / a.G, j = col0 + x - token * a.G;
                const bool live = x < cols && in_bounds(k.t + token < a.T && k.g * a.G + j < a.H, a.status);
                load_column<F16>(a.q + (int64_t)(k.t + token) * a.q_stride + (k.g * a.G + j) * kHeadDim + 32 * t, live, q[z], cs[z]);
                cs[z] *= a.qscale;
                lim[z] = live ? sees(a, k.len, k.n, token) : k.rows;
                acc.reach[z] = acc.top[z] = -INFINITY;
                acc.l[z] = 0.f;
            }
#pragma unroll
            for (int i = 0; i < 16; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) acc.o[i][e] = 0.f;
            const int shown = sees(a, k.len, k.n, col0 / a.G);
#pragma unroll 1
            for (int j = k.j0 + warp; j < k.j1; j += kWarps) {
                const int s = used % kStages;
                if (ok && !__all_sync(kFull, mbar_wait(smem_u32(full + s), (used / kStages) & 1))) {
                    ok = false;
                    misc[0] = 1;
                    if (lane == 0) report(a, DKV_DEV_TMA_TIMEOUT);
                }
                if (!ok) break;
                ++used;
                const int r0 = j * kRows, tl[2] = {lim[0] - r0, lim[1] - r0};
                const unsigned char* tile = ring + s * kStageBytes;
                tile_step(acc, q, cs, tile, tile + kTileBytes, scales + s * 2 * kRows, tl, shown - r0, k.rows - r0);
                __syncwarp();
                fetch();
            }
            // The warps' states: joined in the order of the warps, 64 dims at a time.
            const int active = min(kWarps, k.j1 - k.j0);
#pragma unroll
            for (int z = 0; z < 2; ++z) {
                acc.l[z] += __shfl_xor_sync(kFull, acc.l[z], 1);
                acc.l[z] += __shfl_xor_sync(kFull, acc.l[z], 2);
                if (t == 0) states[warp * kCols + g + 8 * z] = State{acc.reach[z], acc.top[z], acc.l[z], 0.f};
            }
            __syncthreads();
            const bool aborted = misc[0];
            const int mine = tid >> 4, chunk = tid & 15;  // this thread sums 4 dims of column `mine`: chunk 4 t + i of lane t's 16
            State total{-INFINITY, -INFINITY, 0.f, 0.f};
            float f0 = -INFINITY, f1 = -INFINITY;
            for (int x = 0; x < active; ++x) {
                const State y = states[x * kCols + mine];
                total.reach = fmaxf(total.reach, y.reach);
                total.top = fmaxf(total.top, y.top);
                f0 = fmaxf(f0, states[x * kCols + g].reach);
                f1 = fmaxf(f1, states[x * kCols + g + 8].reach);
            }
            for (int x = 0; x < active; ++x) {
                const State y = states[x * kCols + mine];
                total.sum += y.sum * factor(y.top, total.top);
            }
            f0 = factor(acc.reach[0], f0);
            f1 = factor(acc.reach[1], f1);
            const bool whole = k.whole(), live = mine < cols && !aborted;
            const int token = (col0 + mine) / a.G, head_j = col0 + mine - token * a.G;
            uint16_t* out = a.out + ((int64_t)(k.t + token) * a.H + k.g * a.G + head_j) * kHeadDim;
            const int64_t slot = (int64_t)c * 2 + (k.j0 == 0);
            const float z = final_scale(total.reach, total.top, total.sum);
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                __syncthreads();
                if (warp < active) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        // (chunks are permuted so that a quarter-warp's eight lie in different banks)
                        const int at = (4 * t + i) ^ (t >> 1) ^ (2 * (g & 1));
                        float4* to = reinterpret_cast<float4*>(sums + (warp * kCols + g) * 64) + at;
                        to[0] = make_float4(acc.o[4 * i][half] * f0, acc.o[4 * i + 1][half] * f0, acc.o[4 * i + 2][half] * f0, acc.o[4 * i + 3][half] * f0);
                        to[8 * 16] = make_float4(acc.o[4 * i][2 + half] * f1, acc.o[4 * i + 1][2 + half] * f1, acc.o[4 * i + 2][2 + half] * f1,
                                                 acc.o[4 * i + 3][2 + half] * f1);
                    }
                }
                __syncthreads();
                if (live) {
                    const int at = chunk ^ (chunk >> 3) ^ (2 * (mine & 1));
                    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
                    for (int x = 0; x < active; ++x) {
                        const float4 y = reinterpret_cast<const float4*>(sums + (x * kCols + mine) * 64)[at];
                        v = make_float4(v.x + y.x, v.y + y.y, v.z + y.z, v.w + y.w);
                    }
                    const int dim = 32 * (chunk >> 2) + 16 * half + 4 * (chunk & 3);
                    if (whole)
                        *reinterpret_cast<uint2*>(out + dim) = pack4<F16>(v, z);
                    else
                        __stcg(w.o + (slot * kCols + mine) * (kHeadDim / 4) + dim / 4, v);
                }
            }
            if (!whole) {
                if (live && chunk == 0) __stcg(reinterpret_cast<float4*>(w.state + slot * kCols + mine), make_float4(total.reach, total.top, total.sum, 0.f));
                const int c0 = cta_of(head, k.start), pieces = cta_of(head, k.start + k.tiles - 1) - c0 + 1;
                __threadfence();
                __syncthreads();
                if (tid == 0) {
                    pdl_wait();  // the counters are cleared
                    misc[1] = !aborted && atomicAdd(w.done + c0, 1) == pieces - 1;
                }
                __syncthreads();
                if (misc[1] && mine < cols && in_bounds(c0 >= 0 && c0 + pieces <= nctas, a.status)) {
                    __threadfence();
                    State all{-INFINITY, -INFINITY, 0.f, 0.f};
#pragma unroll 4
                    for (int x = 0; x < pieces; ++x) {
                        const float4 y = __ldcg(reinterpret_cast<const float4*>(w.state + piece_at(c0, x) * kCols + mine));
                        all.reach = fmaxf(all.reach, y.x);
                        all.top = fmaxf(all.top, y.y);
                    }
                    float4 v[2] = {make_float4(0.f, 0.f, 0.f, 0.f), make_float4(0.f, 0.f, 0.f, 0.f)};
#pragma unroll 4
                    for (int x = 0; x < pieces; ++x) {
                        const int64_t piece = piece_at(c0, x) * kCols + mine;
                        const float4 y = __ldcg(reinterpret_cast<const float4*>(w.state + piece));
                        const float fo = factor(y.x, all.reach);
                        all.sum += y.z * factor(y.y, all.top);
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            const float4 u = __ldcg(w.o + piece * (kHeadDim / 4) + 2 * chunk + i);
                            v[i] = make_float4(fmaf(u.x, fo, v[i].x), fmaf(u.y, fo, v[i].y), fmaf(u.z, fo, v[i].z), fmaf(u.w, fo, v[i].w));
                        }
                    }
                    const float y = final_scale(all.reach, all.top, all.sum);
                    const uint2 lo = pack4<F16>(v[0], y), hi = pack4<F16>(v[1], y);
                    *reinterpret_cast<uint4*>(out + 8 * chunk) = make_uint4(lo.x, lo.y, hi.x, hi.y);
                }
            }
            __syncthreads();  // sums and misc[1] are read
            if (!k.more()) break;
            k.next(a);
        }
        // Copies in flight land (or run out of time) before the CTA exits.
        for (; used < fetched; ++used) mbar_wait(smem_u32(full + used % kStages), (used / kStages) & 1);
    }
    pdl_wait();  // the call is not over before its begin kernel
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

}  // namespace

int64_t quant_workspace_bytes() { return kWorkBytes + chunk_workspace_bytes(); }

cudaError_t quant_setup()
{
    cudaError_t e = cudaFuncSetAttribute(quant_attn_kernel<false>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemBytes);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(quant_attn_kernel<true>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemBytes);
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
    w.state = reinterpret_cast<State*>(base + kOffState);
    w.o = reinterpret_cast<float4*>(base + kOffO);
    w.chunk = reinterpret_cast<int32_t*>(base + kWorkBytes);
    QuantAttnArgs few = a;
    few.few = std::min(a.most, kCols / a.G);
    if ((e = launch_pdl(quant_begin_kernel, 1, 512, 0, st, few, w)) != cudaSuccess) return e;
    if (a.most > few.few) {
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
        if ((e = launch_chunk8(c, nctas, short_boxes, st)) != cudaSuccess) return e;
    }
    return a.fp16 ? launch_pdl(quant_attn_kernel<true>, nctas, kThreads, kSmemBytes, st, few, maps, w, nctas)
                  : launch_pdl(quant_attn_kernel<false>, nctas, kThreads, kSmemBytes, st, few, maps, w, nctas);
}

}  // namespace dkv
