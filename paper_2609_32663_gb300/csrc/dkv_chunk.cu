// Attention of a ragged chunk of new tokens over a paged cache: the new tokens' K and V
// rows are appended to their slabs' pages, then token i of the n new ones of sequence b
// attends, per query head, to the first len - n + i + 1 rows of its slab (causal) or to
// all len rows:  o = sum_r softmax_r(scale q.k_r) v_r.
#include "dkv_decode_common.cuh"
#include "dkv_pages.cuh"

#include <cuda_bf16.h>
#include <cuda_fp16.h>

namespace dkv {
namespace {

__device__ __forceinline__ int cu_at(const ChunkArgs& a, int b) { return min(max(a.cu[b], 0), a.T); }

// The sequence of token t, or -1 behind the last one.
__device__ __forceinline__ int seq_of(const ChunkArgs& a, int t)
{
    if (t >= cu_at(a, a.B)) return -1;
    int lo = 0, hi = a.B - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (cu_at(a, mid) <= t)
            lo = mid;
        else
            hi = mid - 1;
    }
    return lo;
}

// Pool row of row r of slab h, or -1.
__device__ __forceinline__ int64_t pool_row(const ChunkArgs& a, int h, int64_t r)
{
    if (r < 0 || r >= (int64_t)a.max_pages * a.P) return -1;
    const int page = a.table[(int64_t)h * a.max_pages + r / a.P];
    return page < 0 || page >= a.num_pages ? -1 : (int64_t)page * a.P + r % a.P;
}

__global__ void __launch_bounds__(256) chunk_append_kernel(const ChunkArgs a)
{
    const int i = blockIdx.x * 16 + (threadIdx.x >> 4), sub = threadIdx.x & 15;
    const int t = i / a.Hkv, g = i - t * a.Hkv;
    if (t >= a.T) return;
    const int b = seq_of(a, t);
    if (b < 0) return;
    const int h = b * a.Hkv + g, n = cu_at(a, b + 1) - cu_at(a, b);
    const int64_t row = pool_row(a, h, (int64_t)a.len[h] - n + (t - cu_at(a, b)));
    if (row < 0) {
        if (sub == 0 && a.status) atomicOr(a.status, DKV_DEV_PAGE_RANGE);
        return;
    }
    const int64_t src = t * a.kv_stride + g * kHeadDim;
    reinterpret_cast<uint4*>(a.Kp + row * kHeadDim)[sub] = reinterpret_cast<const uint4*>(a.k_new + src)[sub];
    reinterpret_cast<uint4*>(a.Vp + row * kHeadDim)[sub] = reinterpret_cast<const uint4*>(a.v_new + src)[sub];
}

template <bool F16>
__device__ __forceinline__ float4 load4(const uint16_t* p)
{
    const uint2 u = *reinterpret_cast<const uint2*>(p);
    if (F16) {
        const float2 x = __half22float2(*reinterpret_cast<const __half2*>(&u.x)), y = __half22float2(*reinterpret_cast<const __half2*>(&u.y));
        return make_float4(x.x, x.y, y.x, y.y);
    }
    return make_float4(__uint_as_float(u.x << 16), __uint_as_float(u.x & 0xffff0000u), __uint_as_float(u.y << 16),
                       __uint_as_float(u.y & 0xffff0000u));
}

// One warp a (token, query head): 4 dimensions a lane, one row after another.
template <bool F16>
__global__ void __launch_bounds__(256) chunk_rows_kernel(const ChunkArgs a)
{
    const int64_t w = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
    const int lane = threadIdx.x & 31, t = (int)(w / a.H), head = (int)(w - (int64_t)t * a.H);
    if (t >= a.T) return;
    const int b = seq_of(a, t);
    if (b < 0) return;
    const int h = b * a.Hkv + head / a.G, t0 = cu_at(a, b), n = cu_at(a, b + 1) - t0;
    const int64_t len = a.len[h], rows = a.causal ? len - n + (t - t0) + 1 : len;
    const float4 q = load4<F16>(a.q + t * a.q_stride + head * kHeadDim + 4 * lane);
    float m = -INFINITY, l = 0.f;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int64_t r = 0; r < rows; ++r) {
        const int64_t row = pool_row(a, h, r);
        if (row < 0) {
            if (lane == 0 && a.status) atomicOr(a.status, DKV_DEV_PAGE_RANGE);
            break;
        }
        const float4 k = load4<F16>(a.Kp + row * kHeadDim + 4 * lane), v = load4<F16>(a.Vp + row * kHeadDim + 4 * lane);
        float s = q.x * k.x + q.y * k.y + q.z * k.z + q.w * k.w;
#pragma unroll
        for (int x = 16; x >= 1; x >>= 1) s += __shfl_xor_sync(kFull, s, x);
        s *= a.qscale;
        const float m1 = fmaxf(m, s), f = ex2(m - m1), p = ex2(s - m1);
        m = m1;
        l = l * f + p;
        o = make_float4(o.x * f + p * v.x, o.y * f + p * v.y, o.z * f + p * v.z, o.w * f + p * v.w);
    }
    const float z = l > 0.f ? 1.f / l : (l == l ? 0.f : l);
    uint2 u;
    if (F16) {
        const __half2 x = __floats2half2_rn(o.x * z, o.y * z), y = __floats2half2_rn(o.z * z, o.w * z);
        u = make_uint2(*reinterpret_cast<const uint32_t*>(&x), *reinterpret_cast<const uint32_t*>(&y));
    } else {
        const __nv_bfloat162 x = __floats2bfloat162_rn(o.x * z, o.y * z), y = __floats2bfloat162_rn(o.z * z, o.w * z);
        u = make_uint2(*reinterpret_cast<const uint32_t*>(&x), *reinterpret_cast<const uint32_t*>(&y));
    }
    *reinterpret_cast<uint2*>(a.out + ((int64_t)t * a.H + head) * kHeadDim + 4 * lane) = u;
}

}  // namespace

int64_t chunk_workspace_bytes() { return 256; }

cudaError_t launch_chunk(const ChunkArgs& a, cudaStream_t st)
{
    if (a.k_new) {
        chunk_append_kernel<<<(unsigned)(((int64_t)a.T * a.Hkv + 15) / 16), 256, 0, st>>>(a);
        const cudaError_t e = cudaGetLastError();
        if (e != cudaSuccess) return e;
    }
    const unsigned grid = (unsigned)(((int64_t)a.T * a.H + 7) / 8);
    if (a.fp16)
        chunk_rows_kernel<true><<<grid, 256, 0, st>>>(a);
    else
        chunk_rows_kernel<false><<<grid, 256, 0, st>>>(a);
    return cudaGetLastError();
}

}  // namespace dkv
