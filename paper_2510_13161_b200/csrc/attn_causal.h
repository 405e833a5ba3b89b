// Definitions shared by the two kernels of mirror_attn_causal (attn_causal.cu: single tokens, attn_prompt.cu: longer rows).
#pragma once
#include "attn_common.h"

struct CausalParams {
    int L, B, R, Hq, Hkv, G;
    int max_rows, window, n_sink;
    int max_pages, num_pages, layer_pages;
    float scale_log2e;
    const int32_t* row_start;
    const int32_t* page_table;
    const int32_t* prefix_len;
    const __nv_bfloat16* q;
    const __nv_bfloat16* v_pool;
    __nv_bfloat16* out;
    float* lse_out;
    float* partial;                       // records of the units that the partition cut
    attn::GroupBegin* begins;             // [CTAs]
    int* status;
    long long wait_limit;                 // SM cycles after which a wait gives up
};

// How long a request can be, as far as the host knows: 16-token slots that its rows see.
static inline long long causal_most_slots(const CausalParams& p, int rows) {       // of `rows` neighbouring rows
    long long s = p.max_pages;
    if (p.window > 0) {
        const long long w = ((long long)p.window + rows + 14) / 16 + 1 + ((long long)p.n_sink + 15) / 16;
        if (w < s) s = w;
    }
    return s;
}
mirror_status mirror_attn_prompt_launch(mirror_ctx* ctx, const mirror_kv* kv, const CausalParams& p, void* plan, cudaStream_t stream);
size_t mirror_attn_prompt_plan_bytes(const mirror_ctx* ctx);
// pool as (64 columns, 8 tokens, D/64 halves, 2 token groups, (layer*page)*head): one box is one page of one head, landing as
// [token / 8][half][token % 8][128 B]
mirror_status mirror_attn_pool_tmap(const mirror_ctx* ctx, const mirror_kv* kv, const void* pool, CUtensorMap* map);

#ifdef __CUDACC__
namespace causal {

__device__ __forceinline__ void report(int* status, int code, int detail) {
    if (atomicCAS(status, 0, code) == 0) atomicExch(status + 1, detail);
}

// The tokens that some row of a request sees: [0, sink) and [lo, len), in 16-token slots: the first sink_slots of the request, then
// those from slot `from` on.
struct Request {
    int row0, n;                          // its rows
    int prefix;                           // position of the first
    int len, lo, sink;
    int sink_slots, from, slots;
    __device__ __forceinline__ int slot_page(int t) const { return t < sink_slots ? t : t - sink_slots + from; }
};
// Row start, rows and prefix as they are usable: within the tensors and the page table whatever the device arrays hold.  (Past L1, which
// may hold what a look ahead of the kernel in front has seen.)
__device__ __forceinline__ void load_request(const CausalParams& p, int b, int& row0, int& n, int& prefix, bool report_it) {
    int r0, r1;
    if (p.row_start) {
        r0 = __ldcg(p.row_start + b);
        r1 = __ldcg(p.row_start + b + 1);
    } else {
        r0 = b * p.max_rows;
        r1 = r0 + p.max_rows;
    }
    row0 = min(max(r0, 0), p.R);
    n = min(max(min(r1, p.R) - row0, 0), p.max_rows);
    const int raw = __ldcg(p.prefix_len + b), cap = p.max_pages * kAttnSlotTok;
    prefix = min(max(raw, 0), cap);
    if (report_it) {
        if (r0 < 0 || r1 > p.R || r1 - r0 > p.max_rows || r1 < r0) report(p.status, MIRROR_DEV_CHECK, 830);
        if (raw < 0 || (long long)raw + n > cap) report(p.status, MIRROR_DEV_CHECK, 831);
    }
    n = min(n, cap - prefix);
}
__device__ __forceinline__ Request make_request(const CausalParams& p, int row0, int n, int prefix) {
    Request r;
    r.row0 = row0;
    r.n = n;
    r.prefix = prefix;
    r.len = prefix + n;
    r.lo = p.window > 0 ? min(max(0, prefix - p.window + 1), r.len) : 0;
    r.sink = min(p.n_sink, r.lo);
    r.from = r.lo / kAttnSlotTok;
    r.sink_slots = min((r.sink + kAttnSlotTok - 1) / kAttnSlotTok, r.from);
    r.slots = n > 0 ? r.sink_slots + (r.len + kAttnSlotTok - 1) / kAttnSlotTok - r.from : 0;
    return r;
}

}  // namespace causal
#endif
