// Declarations of the paged cache (dkv_pages.cu, dkv_chunk.cu), shared with the host
// side of the C ABI (dkv_pages_api.cu).
#pragma once

#include "dkv.h"
#include "dkv_internal.cuh"

namespace dkv {

constexpr int kMaxSlots = 512;  // sequence slots of a page geometry (dkv_pages.B), as sequences of a plan

// What the page kernels read of a plan made by dkv_map_pattern (dkv_api.cu).
struct PlanView {
    int L, B, Hkv;
    bool dense;
    int64_t kept;
    const int32_t* len;
    const int64_t* ioff;
    const int32_t* idx;
};
PlanView plan_view(const dkv_plan* p);

// Reports through dkv_last_error() (dkv_api.cu).
dkv_status set_error(dkv_status st, const char* msg);

// Workspace of dkv_page_tables and dkv_page_release: a header, then for every slab the
// position of its first page among the pages that the call moves, and its rows before (or,
// where the lengths are updated in place by one kernel and committed by another, after).
struct PageHead {
    int32_t ok;      // 0: the call changes nothing
    int32_t count;   // free pages before the call
    int32_t total;   // new tokens of the call
    int32_t pages;   // pages that the call moves
};
constexpr int64_t kPageHeadBytes = 256;
inline int64_t page_workspace_bytes(int64_t NH) { return kPageHeadBytes + 2 * ((NH * 4 + 255) / 256 * 256); }

enum PageMode { kGrowTokens, kGrowPlan, kRelease };

struct PageArgs {
    int L, B, Hkv, NH, P, log_P, num_pages, max_pages;
    int skip_b, skip_g;        // 128 slabs as slots and heads: 128 / Hkv and the rest
    int slot_vec;              // entries of the slot map a thread writes at once: 4 where they are aligned, else 1
    int mode;                  // PageMode
    const int32_t* tokens;     // [B] new tokens (kGrowTokens) or ended flags (kRelease)
    const int32_t* plan_len;   // kGrowPlan: [L][planB][Hkv] kept rows
    int planB;
    const int32_t* seq;        // kGrowPlan: slot of each plan sequence, or null (the same index)
    const int32_t* len;
    int32_t* new_len;
    int32_t* table;            // [NH][max_pages]
    int32_t* free_pages;       // [num_pages]
    const int32_t* free_count;
    int32_t* new_count;
    int32_t* cu;               // [B + 1] or null
    int32_t* slots;            // [L][max_tokens][Hkv] or null
    int64_t max_tokens;
    int32_t* status;           // or null
    PageHead* head;
    int32_t* first;            // [NH]
    int32_t* before;           // [NH]
};
cudaError_t launch_page_tables(const PageArgs& a, cudaStream_t st);

struct PageCompactArgs {
    PlanView plan;
    int B, P, num_pages, max_pages;
    const int32_t* seq;
    const uint16_t* K;
    const uint16_t* V;
    int64_t T_stride;
    const int32_t* table;
    const int32_t* len;
    uint16_t* Kp;
    uint16_t* Vp;
    int32_t* status;
};
cudaError_t launch_page_compact(const PageCompactArgs& a, cudaStream_t st);

struct ChunkArgs {
    const uint16_t* q;      // [T] rows of q_stride elements, H x 128 used
    const uint16_t* k_new;  // [T] rows of kv_stride elements, Hkv x 128 used, or null
    const uint16_t* v_new;
    int64_t q_stride, kv_stride;
    const int32_t* cu;      // [B + 1]
    const int32_t* table;   // the layer's slabs: [B * Hkv][max_pages]
    const int32_t* len;     // [B * Hkv]
    uint16_t* Kp;
    uint16_t* Vp;
    uint16_t* out;          // [T][H][128]
    int32_t* status;
    void* work;
    int T, B, H, Hkv, G, P, num_pages, max_pages;
    int causal, fp16;
    float qscale;           // softmax scale * log2(e)
};
int64_t chunk_workspace_bytes();
cudaError_t chunk_setup();  // the kernels' attributes in the current context
// SMs of the current device; the kernels' attributes are set once a context (a lock and a
// look-up, where the runtime calls take microseconds).
cudaError_t page_setup(int* sms);
// short_boxes (fault injection): page copies deliver half the bytes that a stage expects,
// inside the stage, so that every wait for them runs out.
cudaError_t launch_chunk(const ChunkArgs& a, bool short_boxes, cudaStream_t st);

}  // namespace dkv
