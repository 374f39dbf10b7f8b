// Host side of the paged cache's entry points (include/dkv.h): argument checks and
// launches.
#include "dkv_pages.cuh"

#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <cstdlib>
#include <cstring>

namespace {

dkv_status refuse(const char* fmt, ...)
{
    char msg[256];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(msg, sizeof msg, fmt, ap);
    va_end(ap);
    return dkv::set_error(DKV_ERR_INVALID_ARG, msg);
}

// DKV_FAULT as for the other entry points: "launch" makes launches report failure, "copy" makes
// every wait for a page copy of dkv_chunk_attn run out.
bool fault(const char* what)
{
    const char* f = std::getenv("DKV_FAULT");
    return f && std::strcmp(f, what) == 0;
}

dkv_status launched(cudaError_t e, const char* where)
{
    char msg[256];
    if (fault("launch")) {
        snprintf(msg, sizeof msg, "%s: injected launch failure", where);
        return dkv::set_error(DKV_ERR_CUDA, msg);
    }
    if (e == cudaSuccess) return dkv::set_error(DKV_OK, "");
    snprintf(msg, sizeof msg, "%s: %s", where, cudaGetErrorString(e));
    return dkv::set_error(DKV_ERR_CUDA, msg);
}

bool aligned(const void* p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

// Slabs of a geometry; -1 (with the error set) for a bad one.
int64_t check_pages(const dkv_pages* g)
{
    if (!g) return refuse("pages is NULL"), -1;
    if (g->L < 1 || g->H < 1 || g->H_kv < 1) return refuse("bad pages: L=%d H=%d H_kv=%d", g->L, g->H, g->H_kv), -1;
    if (g->B < 1 || g->B > dkv::kMaxSlots) return refuse("B=%d out of [1, %d]", g->B, dkv::kMaxSlots), -1;
    if (g->H % g->H_kv != 0) return refuse("H=%d is not a multiple of H_kv=%d", g->H, g->H_kv), -1;
    if (g->H / g->H_kv > 8) return refuse("group size H/H_kv=%d > 8 is not supported", g->H / g->H_kv), -1;
    if (g->head_dim != dkv::kHeadDim) return refuse("head_dim=%d: only 128 is supported", g->head_dim), -1;
    if (g->page_rows != 16 && g->page_rows != 32 && g->page_rows != 64 && g->page_rows != 128)
        return refuse("page_rows=%d: 16, 32, 64 or 128", g->page_rows), -1;
    if (g->num_pages < 1 || (int64_t)g->num_pages * g->page_rows >= dkv::kMaxMmaRows)
        return refuse("num_pages=%d of %d rows: need 1 to 2^31 - 17 rows", g->num_pages, g->page_rows), -1;
    if (g->max_pages < 1 || (int64_t)g->max_pages * g->page_rows > 0x7fffff00LL)
        return refuse("max_pages=%d of %d rows: need 1 to 2^31 - 256 rows", g->max_pages, g->page_rows), -1;
    // (The product of three large factors passes 64 bits.)
    if (g->L > (1 << 20) || g->H_kv > (1 << 20) || (int64_t)g->L * g->B * g->H_kv > (1 << 26))
        return refuse("L=%d B=%d H_kv=%d: more than 2^26 slabs", g->L, g->B, g->H_kv), -1;
    return (int64_t)g->L * g->B * g->H_kv;
}

dkv_status check_plan(const dkv_pages* g, const dkv_plan* plan, const int32_t* seq, dkv::PlanView* v)
{
    *v = dkv::plan_view(plan);
    if (v->dense) return refuse("the plan is of an uncompressed cache");
    if (v->L != g->L || v->Hkv != g->H_kv)
        return refuse("the plan has L=%d H_kv=%d, the pages L=%d H_kv=%d", v->L, v->Hkv, g->L, g->H_kv);
    if (v->B > g->B) return refuse("the plan has %d sequences, the pages %d slots", v->B, g->B);
    if (!aligned(seq, 4)) return refuse("seq must be 4-byte aligned");
    return DKV_OK;
}

// What dkv_page_tables and dkv_page_release share.
dkv_status page_args(const dkv_pages* g, const int32_t* len, int32_t* new_len, const int32_t* table,
                     const int32_t* free_pages, const int32_t* free_count, int32_t* new_count, void* workspace,
                     int64_t workspace_bytes, int32_t* status, dkv::PageArgs* a)
{
    const int64_t NH = check_pages(g);
    if (NH < 0) return DKV_ERR_INVALID_ARG;
    if (!len || !new_len || !table || !free_pages || !free_count || !new_count)
        return refuse("NULL len/new_len/table/free_pages/free_count/new_count");
    if (!aligned(len, 4) || !aligned(new_len, 4) || !aligned(table, 4) || !aligned(free_pages, 4) ||
        !aligned(free_count, 4) || !aligned(new_count, 4) || !aligned(status, 4))
        return refuse("int32 arrays must be 4-byte aligned");
    if (!workspace || !aligned(workspace, 16) || workspace_bytes < dkv::page_workspace_bytes(NH))
        return refuse("workspace: need %lld bytes, 16-byte aligned", (long long)dkv::page_workspace_bytes(NH));
    *a = dkv::PageArgs{};
    a->L = g->L;
    a->B = g->B;
    a->Hkv = g->H_kv;
    a->NH = (int)NH;
    a->P = g->page_rows;
    while ((1 << a->log_P) < a->P) ++a->log_P;
    a->skip_b = 128 / g->H_kv;
    a->skip_g = 128 % g->H_kv;
    a->num_pages = g->num_pages;
    a->max_pages = g->max_pages;
    a->len = len;
    a->new_len = new_len;
    a->table = const_cast<int32_t*>(table);
    a->free_pages = const_cast<int32_t*>(free_pages);
    a->free_count = free_count;
    a->new_count = new_count;
    a->status = status;
    unsigned char* w = static_cast<unsigned char*>(workspace);
    a->head = reinterpret_cast<dkv::PageHead*>(w);
    a->first = reinterpret_cast<int32_t*>(w + dkv::kPageHeadBytes);
    a->before = reinterpret_cast<int32_t*>(w + dkv::kPageHeadBytes + (NH * 4 + 255) / 256 * 256);
    return DKV_OK;
}

}  // namespace

extern "C" {

int64_t dkv_page_workspace_bytes(const dkv_pages* g)
{
    const int64_t NH = check_pages(g);
    return NH < 0 ? -1 : dkv::page_workspace_bytes(NH);
}

dkv_status dkv_page_tables(const dkv_pages* g, const int32_t* tokens, const dkv_plan* plan, const int32_t* seq,
                           const int32_t* len, int32_t* new_len, int32_t* table, const int32_t* free_pages,
                           const int32_t* free_count, int32_t* new_count, int32_t* cu_tokens, int32_t* slots,
                           int64_t max_tokens, void* workspace, int64_t workspace_bytes, int32_t* status,
                           cudaStream_t stream)
{
    dkv::PageArgs a;
    const dkv_status st = page_args(g, len, new_len, table, free_pages, free_count, new_count, workspace, workspace_bytes,
                                    status, &a);
    if (st != DKV_OK) return st;
    if ((tokens != nullptr) == (plan != nullptr)) return refuse("exactly one of tokens and plan is given");
    if (seq && !plan) return refuse("seq goes with a plan");
    if (plan && (cu_tokens || slots)) return refuse("cu_tokens and slots go with tokens, not with a plan");
    if (slots && !cu_tokens) return refuse("slots needs cu_tokens");
    if (slots && (max_tokens < 0 || max_tokens > 0x7fffffffLL))
        return refuse("max_tokens=%lld out of [0, 2^31)", (long long)max_tokens);
    if (!aligned(tokens, 4) || !aligned(cu_tokens, 4) || !aligned(slots, 4))
        return refuse("int32 arrays must be 4-byte aligned");
    a.mode = plan ? dkv::kGrowPlan : dkv::kGrowTokens;
    a.tokens = tokens;
    if (plan) {
        dkv::PlanView v;
        const dkv_status sp = check_plan(g, plan, seq, &v);
        if (sp != DKV_OK) return sp;
        a.plan_len = v.len;
        a.planB = v.B;
        a.seq = seq;
    }
    a.cu = cu_tokens;
    a.slots = slots;
    a.max_tokens = max_tokens;
    a.slot_vec = g->H_kv % 4 == 0 && aligned(slots, 16) ? 4 : 1;
    return launched(dkv::launch_page_tables(a, stream), "page table kernels");
}

dkv_status dkv_page_release(const dkv_pages* g, const int32_t* ended, const int32_t* len, int32_t* new_len,
                            const int32_t* table, int32_t* free_pages, const int32_t* free_count, int32_t* new_count,
                            void* workspace, int64_t workspace_bytes, int32_t* status, cudaStream_t stream)
{
    dkv::PageArgs a;
    const dkv_status st = page_args(g, len, new_len, table, free_pages, free_count, new_count, workspace, workspace_bytes,
                                    status, &a);
    if (st != DKV_OK) return st;
    if (!ended || !aligned(ended, 4)) return refuse("ended is NULL or not 4-byte aligned");
    a.mode = dkv::kRelease;
    a.tokens = ended;
    return launched(dkv::launch_page_tables(a, stream), "page release kernels");
}

dkv_status dkv_page_compact(const dkv_pages* g, const dkv_plan* plan, const int32_t* seq, const void* K, const void* V,
                            int64_t T_stride, const int32_t* table, const int32_t* len, void* Kp, void* Vp,
                            int32_t* status, cudaStream_t stream)
{
    if (check_pages(g) < 0) return DKV_ERR_INVALID_ARG;
    if (!plan) return refuse("plan is NULL");
    dkv::PageCompactArgs a{};
    const dkv_status st = check_plan(g, plan, seq, &a.plan);
    if (st != DKV_OK) return st;
    if (!K || !V || !Kp || !Vp || !table || !len) return refuse("NULL K/V/Kp/Vp/table/len");
    if (!aligned(K, 16) || !aligned(V, 16) || !aligned(Kp, 16) || !aligned(Vp, 16))
        return refuse("K/V/Kp/Vp must be 16-byte aligned");
    if (Kp == Vp) return refuse("Kp and Vp must be different buffers");
    if (!aligned(table, 4) || !aligned(len, 4) || !aligned(status, 4)) return refuse("int32 arrays must be 4-byte aligned");
    if (T_stride < 1) return refuse("T_stride=%lld < 1", (long long)T_stride);
    a.B = g->B;
    a.P = g->page_rows;
    a.num_pages = g->num_pages;
    a.max_pages = g->max_pages;
    a.seq = seq;
    a.K = static_cast<const uint16_t*>(K);
    a.V = static_cast<const uint16_t*>(V);
    a.T_stride = T_stride;
    a.table = table;
    a.len = len;
    a.Kp = static_cast<uint16_t*>(Kp);
    a.Vp = static_cast<uint16_t*>(Vp);
    a.status = status;
    return launched(dkv::launch_page_compact(a, stream), "paged compact kernel");
}

int64_t dkv_chunk_workspace_bytes(const dkv_pages* g) { return check_pages(g) < 0 ? -1 : dkv::chunk_workspace_bytes(); }

dkv_status dkv_chunk_attn(const dkv_pages* g, int32_t layer, int32_t dtype, int32_t num_tokens, const void* q,
                          int64_t q_stride, const void* k_new, const void* v_new, int64_t kv_stride,
                          const int32_t* cu_tokens, const int32_t* table, const int32_t* len, void* Kp, void* Vp,
                          int32_t causal, float scale, void* out, void* workspace, int64_t workspace_bytes,
                          int32_t* status, cudaStream_t stream)
{
    if (check_pages(g) < 0) return DKV_ERR_INVALID_ARG;
    if (layer < 0 || layer >= g->L) return refuse("layer=%d out of [0, %d)", layer, g->L);
    if (dtype != DKV_BF16 && dtype != DKV_FP16) return refuse("dtype=%d: DKV_BF16 or DKV_FP16", dtype);
    if (num_tokens < 0 || (int64_t)num_tokens * g->H > (1 << 30))
        return refuse("num_tokens=%d: need 0 <= num_tokens and num_tokens*H <= 2^30", num_tokens);
    const float sc = scale > 0.f ? scale : 1.0f / std::sqrt((float)dkv::kHeadDim);
    const float qscale = sc * 1.4426950408889634f;  // base-2 softmax: exp(x) = exp2(x log2 e)
    if (!std::isfinite(scale) || !std::isfinite(qscale)) return refuse("scale=%g is not finite, or too large", scale);
    if ((k_new == nullptr) != (v_new == nullptr)) return refuse("k_new and v_new must both be given or both be NULL");
    if (num_tokens == 0) return dkv::set_error(DKV_OK, "");
    if (!q || !cu_tokens || !table || !len || !Kp || !Vp || !out) return refuse("NULL q/cu_tokens/table/len/Kp/Vp/out");
    if (!aligned(q, 16) || !aligned(k_new, 16) || !aligned(v_new, 16) || !aligned(Kp, 16) || !aligned(Vp, 16) ||
        !aligned(out, 16))
        return refuse("q/k_new/v_new/Kp/Vp/out must be 16-byte aligned");
    if (Kp == Vp) return refuse("Kp and Vp must be different buffers");
    if (!aligned(cu_tokens, 4) || !aligned(table, 4) || !aligned(len, 4) || !aligned(status, 4))
        return refuse("int32 arrays must be 4-byte aligned");
    const int64_t most = (int64_t)1 << 36;  // a tensor map's strides are below 2^40 bytes
    if (q_stride % 8 != 0 || q_stride < (int64_t)g->H * dkv::kHeadDim || q_stride > most)
        return refuse("q_stride=%lld: a multiple of 8, at least H*128=%lld", (long long)q_stride,
                      (long long)g->H * dkv::kHeadDim);
    if (k_new && (kv_stride % 8 != 0 || kv_stride < (int64_t)g->H_kv * dkv::kHeadDim || kv_stride > most))
        return refuse("kv_stride=%lld: a multiple of 8, at least H_kv*128=%lld", (long long)kv_stride,
                      (long long)g->H_kv * dkv::kHeadDim);
    if (!workspace || !aligned(workspace, 16) || workspace_bytes < dkv::chunk_workspace_bytes())
        return refuse("workspace: need %lld bytes, 16-byte aligned", (long long)dkv::chunk_workspace_bytes());
    dkv::ChunkArgs a{};
    const int64_t slabs = (int64_t)g->B * g->H_kv;
    a.q = static_cast<const uint16_t*>(q);
    a.k_new = static_cast<const uint16_t*>(k_new);
    a.v_new = static_cast<const uint16_t*>(v_new);
    a.q_stride = q_stride;
    a.kv_stride = kv_stride;
    a.cu = cu_tokens;
    a.table = table + layer * slabs * g->max_pages;
    a.len = len + layer * slabs;
    a.Kp = static_cast<uint16_t*>(Kp);
    a.Vp = static_cast<uint16_t*>(Vp);
    a.out = static_cast<uint16_t*>(out);
    a.status = status;
    a.work = workspace;
    a.T = num_tokens;
    a.B = g->B;
    a.H = g->H;
    a.Hkv = g->H_kv;
    a.G = g->H / g->H_kv;
    a.P = g->page_rows;
    a.num_pages = g->num_pages;
    a.max_pages = g->max_pages;
    a.causal = causal != 0;
    a.fp16 = dtype == DKV_FP16;
    a.qscale = qscale;
    return launched(dkv::launch_chunk(a, fault("copy"), stream), "chunk attention kernels");
}

}  // extern "C"
