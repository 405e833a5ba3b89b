// Causal attention of new rows over the paged cache (mirror_attn_causal): the entry point, and the kernel for few rows.
//
// attn_token_kernel: requests with at most 16 rows per KV head (rows x query heads of the group), single tokens above all.  Each byte of the
// cache is used for 16 rows at most, so HBM bounds it, and what counts is that every SM always has enough bytes on the way (45 KB,
// Little's law at 6.5 TB/s and ~1 us).  The 16-token slots (one page of one head: 4 KB of K and of V at d = 128) of all (layer, request, head)
// units form one sequence that is split evenly over the CTAs by what units cost.  Within a CTA every warp streams for itself: of each unit it
// takes every fourth slot (or twelfth), keeps two on the way with TMA (a ring of its own: no barrier but its own), multiplies them with
// mma.sync (16 rows are what it has; a tcgen05 tile would be 128) and holds its running maximum, sum and accumulator in registers.  At the
// end of a unit the warps' accumulators are added up in shared memory, one after the other; three or four CTAs share an SM, so that one's
// chains of dependent steps, and its merges, hide behind the others' streams.  A unit that the partition cut leaves a record per part for
// attn_token_merge_kernel.  Tried and no faster: two slots at a time (the same instructions, less overlap), and ranges of whole warps
// without barriers between units (more parts).
//
// Neither kernel lets the one behind it start early: CTAs of the next call that find room beside the last ones of this call leave the SMs
// with unequal numbers of equal shares (48 requests under a window, call after call: 178 us, else 130).
// (Letting only the merge kernel start early costs 2 us where its time counts: 32768 tokens 35 -> 38.)
// Measured on a B200: 64 requests of 130 to 8191 tokens, 40 / 8 heads of 128: 180 us (6.1 TB/s); one of 32768 tokens, 64 / 8 heads: 35 us, of which 21 are
// bytes and the rest the two launches' fixed parts.
// P is multiplied as the sum of two bf16 (its rounding and what that left): the tensor cores have the time, and the output then carries no
// rounding but its own.
#include <math.h>

#include <algorithm>

#include "attn_causal.h"

namespace {

using causal::Request;

constexpr int kStages = 2;                          // slots a warp has on the way
constexpr int kRows = 16;
constexpr int kMaxCtas = 768;                       // (notes of 16 bytes each, in 12 KB)
constexpr int kMergeThreads = 256;
constexpr size_t kSmemPerSm = 233472;               // 228 KB, of which every CTA takes 1 KB more than it asks for
constexpr float kLazy = 8.f;                        // the running maximum moves when a score passes it by this (log2): P stays below 2^8
constexpr int kUnitSlots = 10;                      // what a unit costs beside its slots (queries, the merge of the warps, the output)
constexpr int kMinShare = 16;                       // slots of a CTA at least, where units are cut

template <int D, int kWarps>
struct Cfg {
    static constexpr int kThreads = 32 * kWarps;
    static constexpr int kAreas = kWarps / 4;                       // where four warps each add up what they have
    static constexpr int kHalves = D / 64;
    static constexpr int kSlotBytes = kAttnSlotTok * D * 2;
    static constexpr int kRec = kRows * D + 2 * kRows;              // record: accumulators, maxima, sums
    static constexpr int kPitch = D + 4;                            // floats of a row in the merge area
    static constexpr int kRing = kWarps * kStages * 2 * kSlotBytes;
    static constexpr int kMerge = kAreas * kRows * kPitch * 4 + kWarps * kRows * 2 * 4;
    static constexpr int kCtas = kWarps > 4 ? 1 : D == 128 ? 3 : 4; // of an SM, by registers
    static constexpr int kBars = kWarps * kStages * 8;
    static size_t smem(int B) { return (size_t)kRing + kMerge + kBars + 64 + (5 * (size_t)B + 2) * 4; }
};

struct TokenMaps {
    CUtensorMap k, v;
};

struct Begin {
    long long x;                          // slots ahead of it
    int layer, b, h, t;
};
// Slots of a head's units, and how many units have any, summed over the requests.
struct Sums {
    const int *slots, *units;             // [B + 1] each
    int of_slot, of_unit;                 // what a slot and a unit cost
    __device__ __forceinline__ int cost(int b) const { return of_slot * slots[b] + of_unit * units[b]; }
};
// Where CTA c's range begins.  The sequence is split evenly by cost.  never_cut: a range
// begins with a unit; else a boundary close to a unit's is moved there (a cut costs a record and a merge).
__device__ Begin range_begin(const CausalParams& p, const Sums& s, long long total, int ctas, int c, bool never_cut) {
    const long long per_layer = (long long)p.Hkv * s.slots[p.B];
    Begin u = {c <= 0 ? 0 : per_layer * p.L, 0, 0, 0, 0};
    if (c <= 0 || c >= ctas) return u;
    const long long cost_layer = (long long)p.Hkv * s.cost(p.B), x = total * c / ctas;
    u.layer = (int)(x / cost_layer);
    const long long rem = x - u.layer * cost_layer;
    int lo = 0, hi = p.B - 1;                                      // the first b with Hkv * cost(b + 1) > rem
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if ((long long)p.Hkv * s.cost(mid + 1) > rem) hi = mid; else lo = mid + 1;
    }
    u.b = lo;
    const int T = s.slots[lo + 1] - s.slots[lo], per = s.of_slot * T + s.of_unit;
    const long long in = rem - (long long)p.Hkv * s.cost(lo);
    u.h = (int)(in / per);
    const int in_unit = (int)(in - (long long)u.h * per);
    u.t = max(0, in_unit - s.of_unit);
    const int tol = (int)min(8ll, total / ctas >> 2);
    if (!never_cut && u.t <= tol) u.t = 0;
    // (never cut: the unit belongs to the CTA that has its larger part)
    if (u.t > 0 && (never_cut ? 2ll * in_unit > per : T - u.t <= tol)) u.t = T;
    if (never_cut && u.t < T) u.t = 0;
    u.x = u.layer * per_layer + (long long)p.Hkv * s.slots[lo] + (long long)u.h * T + u.t;
    if (u.t == T) {
        u.t = 0;
        if (++u.h == p.Hkv) {
            u.h = 0;
            do {
                if (++u.b == p.B) { u.b = 0; ++u.layer; }
            } while (u.layer < p.L && s.slots[u.b + 1] == s.slots[u.b]);
        }
    }
    return u;
}

__device__ __forceinline__ void ldmatrix4(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldmatrix4t(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void mma16816(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// A warp's way through the CTA's slots: every kWarps-th of each unit's part.
struct Cursor {
    int layer, b, h;
    int t, t_end;                         // this warp's slot, end of the part
    long long left;                       // slots of the range behind this part
    Request r;
};

template <int D, int kWarps>
__global__ void __launch_bounds__(32 * kWarps, Cfg<D, kWarps>::kCtas) attn_token_kernel(const __grid_constant__ TokenMaps tm, const __grid_constant__ CausalParams p, const int never_cut) {
    using C = Cfg<D, kWarps>;
    constexpr int kThreads = C::kThreads;
    extern __shared__ __align__(1024) uint8_t smem[];
    float* const s_o = (float*)(smem + C::kRing);                   // [areas][16][pitch], then [warps][16][max, sum]
    float* const s_ml = s_o + C::kAreas * kRows * C::kPitch;
    uint64_t* const bars = (uint64_t*)(smem + C::kRing + C::kMerge);
    Begin* const s_begin = (Begin*)(bars + kWarps * kStages);       // 2 x 24 bytes
    int* const cum = (int*)((uint8_t*)bars + C::kBars + 64);        // [B + 1] slots of a head's units, summed over the requests
    int* const cum_units = cum + p.B + 1;                           // [B + 1] units that have any
    int* const s_row0 = cum_units + p.B + 1;                        // [B] each
    int* const s_n = s_row0 + p.B;
    int* const s_prefix = s_n + p.B;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;

    if (lane == 0) {
        for (int s = 0; s < kStages; ++s) ptx::mbar_init(&bars[warp * kStages + s], 1);
        ptx::fence_mbar_init();
        if (warp == 0) { ptx::prefetch_tmap(&tm.k); ptx::prefetch_tmap(&tm.v); }
    }
    ptx::grid_dep_wait();
    if (warp == 0) {
        int acc = 0, units = 0;
        if (lane == 0) cum[0] = cum_units[0] = 0;
        for (int b0 = 0; b0 < p.B; b0 += 32) {
            const int b = b0 + lane;
            int row0 = 0, n = 0, prefix = 0, sum = 0;
            if (b < p.B) {
                causal::load_request(p, b, row0, n, prefix, blockIdx.x == 0);
                sum = max(causal::make_request(p, row0, n, prefix).slots, 0);
                s_row0[b] = row0; s_n[b] = n; s_prefix[b] = prefix;
            }
            const uint32_t some = __ballot_sync(0xffffffffu, sum > 0);
            if (b < p.B) cum_units[b + 1] = units + __popc(some & (0xffffffffu >> (31 - lane)));
            units += __popc(some);
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int v = __shfl_up_sync(0xffffffffu, sum, o);
                if (lane >= o) sum += v;
            }
            if (b < p.B) cum[b + 1] = acc + sum;
            acc += __shfl_sync(0xffffffffu, sum, 31);
        }
        __syncwarp();
        // kUnitSlots for a unit and one for each of its slots; whole units that are no more than the CTAs get one each, whatever their
        // lengths (by cost the shorter ones shared: 159 units of 1 to 3 slots 17.0 -> 10.2 us)
        const long long lh = (long long)p.L * p.Hkv;
        const bool one_each = never_cut && lh * units <= (long long)gridDim.x;
        const Sums sums = {cum, cum_units, one_each ? 0 : 1, one_each ? 1 : kUnitSlots};
        const long long total = lh * sums.cost(p.B), most = one_each ? lh * units : max(lh * units, lh * acc / kMinShare);
        const int ctas = (int)min((long long)gridDim.x, max(most, 1ll));
        if (lane < 2) {
            s_begin[lane] = range_begin(p, sums, total, ctas, (int)blockIdx.x + lane, never_cut != 0);
            if (lane == 0 && !never_cut) {
                const Begin& u = s_begin[0];
                p.begins[blockIdx.x] = {u.t > 0 ? 1 : 0, u.layer, u.b, u.h};
            }
        }
    }
    __syncthreads();
    const Begin from = s_begin[0];
    const long long n_slots = s_begin[1].x - from.x;
    if (n_slots <= 0) return;

    bool dead = false;                                              // a wait ran out: on to the end without waiting
    auto open = [&](Cursor& c) {                                    // the request of a new unit, and the unit's part
        c.r = causal::make_request(p, s_row0[c.b], s_n[c.b], s_prefix[c.b]);
    };
    auto start = [&](Cursor& c) {
        c.layer = from.layer; c.b = from.b; c.h = from.h;
        open(c);
        const long long m = min((long long)(c.r.slots - from.t), n_slots);
        c.t_end = from.t + (int)m;
        c.left = n_slots - m;
        c.t = from.t + warp;
    };
    auto next_unit = [&](Cursor& c) {                               // (left > 0)
        const int b_was = c.b;
        if (++c.h == p.Hkv) {
            c.h = 0;
            do {
                if (++c.b == p.B) { c.b = 0; ++c.layer; }
            } while (cum[c.b + 1] == cum[c.b]);
        }
        if (c.b != b_was) open(c);
        const long long m = min((long long)c.r.slots, c.left);
        c.t_end = (int)m;
        c.left -= m;
        c.t = warp;
    };
    auto settle = [&](Cursor& c) -> bool {                          // on to a part that has a slot for this warp
        while (c.t >= c.t_end) {
            if (c.left <= 0) return false;
            next_unit(c);
        }
        return true;
    };

    // ---- this warp's copies
    uint8_t* const ring = smem + warp * (kStages * 2 * C::kSlotBytes);
    uint64_t* const bar = bars + warp * kStages;
    Cursor ci;
    start(ci);
    bool more = settle(ci);
    int page = 0;
    auto fetch = [&]() { if (more) page = p.page_table[(size_t)ci.b * p.max_pages + ci.r.slot_page(ci.t)]; };
    fetch();
    uint32_t issued = 0, taken = 0;
    auto issue = [&]() {
        if (!more || dead) return;
        const uint32_t s = issued % kStages;
        if (page < 0 || page >= p.num_pages) {
            if (lane == 0) causal::report(p.status, MIRROR_DEV_CHECK, 832);
            page = 0;
        }
        if (lane == 0) {
            const int row = (ci.layer * p.layer_pages + page) * p.Hkv + ci.h;
            ptx::mbar_arrive_expect_tx(&bar[s], 2 * C::kSlotBytes);
            ptx::tma_load_5d(ring + s * 2 * C::kSlotBytes, &tm.k, &bar[s], 0, 0, 0, 0, row);
            ptx::tma_load_5d(ring + (s * 2 + 1) * C::kSlotBytes, &tm.v, &bar[s], 0, 0, 0, 0, row);
        }
        __syncwarp();
        ++issued;
        ci.t += kWarps;
        more = settle(ci);
        fetch();
    };
    for (int s = 0; s < kStages; ++s) issue();

    // ---- this warp's products.  Thread (g, c) = (lane / 4, lane % 4) has rows g and g + 8, columns 2c and 2c + 1 of every eight.
    const int g = lane >> 2, c2 = (lane & 3) * 2;
    // rows of ldmatrix: K slot as two blocks of eight tokens by two 16-byte chunks; V likewise, transposed
    const int k_tok = (lane & 7) + ((lane >> 4) << 3), k_chunk = (lane >> 3) & 1;
    const int v_tok = lane & 15, v_chunk = lane >> 4;
    Cursor cc;
    start(cc);
    uint32_t qf[D / 16][4];
    const int i0 = g / p.G, i1 = (g + 8) / p.G;
    auto load_q = [&](const Cursor& c) {                            // a unit's queries
        const int rows = c.r.n * p.G;
        const __nv_bfloat16* const qb = p.q + (((size_t)c.layer * p.R + c.r.row0) * p.Hq + c.h * p.G) * D + c2;
        const __nv_bfloat16* const q0 = qb + ((size_t)i0 * p.Hq + (g - i0 * p.G)) * D;
        const __nv_bfloat16* const q1 = qb + ((size_t)i1 * p.Hq + (g + 8 - i1 * p.G)) * D;
#pragma unroll
        for (int k = 0; k < D / 16; ++k) {
            qf[k][0] = g < rows ? *reinterpret_cast<const uint32_t*>(q0 + k * 16) : 0u;
            qf[k][1] = g + 8 < rows ? *reinterpret_cast<const uint32_t*>(q1 + k * 16) : 0u;
            qf[k][2] = g < rows ? *reinterpret_cast<const uint32_t*>(q0 + k * 16 + 8) : 0u;
            qf[k][3] = g + 8 < rows ? *reinterpret_cast<const uint32_t*>(q1 + k * 16 + 8) : 0u;
        }
    };
    load_q(cc);
    for (;;) {
        // a unit's part
        const int rows = cc.r.n * p.G;
        float o[D / 8][4];
#pragma unroll
        for (int j = 0; j < D / 8; ++j) o[j][0] = o[j][1] = o[j][2] = o[j][3] = 0.f;
        float m0 = -INFINITY, m1 = -INFINITY, l0 = 0.f, l1 = 0.f;
        const int pos0 = cc.r.prefix + i0, pos1 = cc.r.prefix + i1, pos_last = cc.r.prefix + cc.r.n - 1;
        const int t_first = cc.t - warp;
        for (; cc.t < cc.t_end; cc.t += kWarps) {
            const uint32_t s = taken % kStages;
            if (!dead && !ptx::mbar_wait(&bar[s], (taken / kStages) & 1, p.wait_limit)) {
                if (lane == 0) causal::report(p.status, MIRROR_DEV_TIMEOUT, 50);
                dead = true;
            }
            dead = __any_sync(0xffffffffu, dead);
            if (dead) continue;
            ++taken;
            uint8_t* const ks = ring + s * 2 * C::kSlotBytes;
            uint8_t* const vs = ks + C::kSlotBytes;
            const uint32_t ka = ptx::smem_u32(ks), va = ptx::smem_u32(vs);
            const int key0 = cc.r.slot_page(cc.t) * kAttnSlotTok;
            // V rows that no row of the request sees may hold anything: zeros, since 0 times infinity is not
            if (key0 + kAttnSlotTok > cc.r.len || (key0 < cc.r.lo && key0 + kAttnSlotTok > cc.r.sink)) {
                for (int tok = 0; tok < kAttnSlotTok; ++tok) {
                    const int key = key0 + tok;
                    if (key < cc.r.len && (key >= cc.r.lo || key < cc.r.sink)) continue;
                    if (lane < D / 8) *reinterpret_cast<uint4*>(vs + attn::kv_slot_off<C::kHalves>(tok, lane)) = make_uint4(0, 0, 0, 0);
                }
                ptx::fence_proxy_async();                           // (the stage's next copy comes behind these)
                __syncwarp();
            }
            // (all of a slot's loads are issued ahead of the products that wait for them)
            float sc[2][4] = {}, sd[2][4] = {};
            uint32_t kf[D / 16][4];
#pragma unroll
            for (int k = 0; k < D / 16; ++k) ldmatrix4(kf[k], ka + attn::kv_slot_off<C::kHalves>(k_tok, 2 * k + k_chunk));
#pragma unroll
            for (int k = 0; k < D / 16; k += 2) {
                mma16816(sc[0], qf[k], kf[k][0], kf[k][1]);
                mma16816(sc[1], qf[k], kf[k][2], kf[k][3]);
                mma16816(sd[0], qf[k + 1], kf[k + 1][0], kf[k + 1][1]);
                mma16816(sd[1], qf[k + 1], kf[k + 1][2], kf[k + 1][3]);
            }
            uint32_t vf[D / 32][4];
#pragma unroll
            for (int j = 0; j < D / 32; ++j) ldmatrix4t(vf[j], va + attn::kv_slot_off<C::kHalves>(v_tok, 2 * j + v_chunk));
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) sc[j][e] += sd[j][e];
            const bool all_seen = key0 + kAttnSlotTok - 1 <= cc.r.prefix &&
                                  (p.window == 0 || key0 > pos_last - p.window || key0 + kAttnSlotTok <= p.n_sink);
            if (!all_seen) {
#pragma unroll
                for (int j = 0; j < 2; ++j)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const int key = key0 + j * 8 + c2 + e;
                        const bool sink = key < p.n_sink || p.window == 0;
                        if (key > pos0 || !(sink || key > pos0 - p.window)) sc[j][e] = -INFINITY;
                        if (key > pos1 || !(sink || key > pos1 - p.window)) sc[j][2 + e] = -INFINITY;
                    }
            }
            float x0 = fmaxf(fmaxf(sc[0][0], sc[0][1]), fmaxf(sc[1][0], sc[1][1])) * p.scale_log2e;
            float x1 = fmaxf(fmaxf(sc[0][2], sc[0][3]), fmaxf(sc[1][2], sc[1][3])) * p.scale_log2e;
            if (__any_sync(0xffffffffu, x0 > m0 + kLazy || x1 > m1 + kLazy)) {
                x0 = fmaxf(x0, __shfl_xor_sync(0xffffffffu, x0, 1)); x1 = fmaxf(x1, __shfl_xor_sync(0xffffffffu, x1, 1));
                x0 = fmaxf(x0, __shfl_xor_sync(0xffffffffu, x0, 2)); x1 = fmaxf(x1, __shfl_xor_sync(0xffffffffu, x1, 2));
                const bool up0 = x0 > m0 + kLazy, up1 = x1 > m1 + kLazy;
                const float a0 = up0 ? exp2f(m0 - x0) : 1.f, a1 = up1 ? exp2f(m1 - x1) : 1.f;
                if (up0) m0 = x0;
                if (up1) m1 = x1;
                l0 *= a0;
                l1 *= a1;
#pragma unroll
                for (int j = 0; j < D / 8; ++j) { o[j][0] *= a0; o[j][1] *= a0; o[j][2] *= a1; o[j][3] *= a1; }
            }
            const float n0 = m0 == -INFINITY ? 0.f : -m0, n1 = m1 == -INFINITY ? 0.f : -m1;
            uint32_t ph[4], pl[4];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const float e0 = ptx::ex2_approx(fmaf(sc[j][0], p.scale_log2e, n0)), e1 = ptx::ex2_approx(fmaf(sc[j][1], p.scale_log2e, n0));
                const float e2 = ptx::ex2_approx(fmaf(sc[j][2], p.scale_log2e, n1)), e3 = ptx::ex2_approx(fmaf(sc[j][3], p.scale_log2e, n1));
                l0 += e0 + e1;
                l1 += e2 + e3;
                ph[2 * j] = attn::pack_bf16(e0, e1);
                ph[2 * j + 1] = attn::pack_bf16(e2, e3);
                pl[2 * j] = attn::pack_bf16(e0 - __uint_as_float(ph[2 * j] << 16), e1 - __uint_as_float(ph[2 * j] & 0xffff0000u));
                pl[2 * j + 1] = attn::pack_bf16(e2 - __uint_as_float(ph[2 * j + 1] << 16), e3 - __uint_as_float(ph[2 * j + 1] & 0xffff0000u));
            }
#pragma unroll
            for (int j0 = 0; j0 < D / 16; j0 += D / 32) {
#pragma unroll
                for (int j = 0; j < D / 32; ++j) {
                    mma16816(o[2 * (j0 + j)], ph, vf[j][0], vf[j][1]);
                    mma16816(o[2 * (j0 + j) + 1], ph, vf[j][2], vf[j][3]);
                }
#pragma unroll
                for (int j = 0; j < D / 32; ++j) {
                    mma16816(o[2 * (j0 + j)], pl, vf[j][0], vf[j][1]);
                    mma16816(o[2 * (j0 + j) + 1], pl, vf[j][2], vf[j][3]);
                }
                if (j0 == 0) {
#pragma unroll
                    for (int j = 0; j < D / 32; ++j) ldmatrix4t(vf[j], va + attn::kv_slot_off<C::kHalves>(v_tok, 2 * (D / 32 + j) + v_chunk));
                }
            }
            __syncwarp();
            issue();
        }
        // ---- the part's end: the warps' accumulators are merged (the next unit's queries are on the way meanwhile)
        const Cursor was = cc;
        const bool last = cc.left <= 0;
        if (!last) {
            next_unit(cc);
            load_q(cc);
        }
        l0 += __shfl_xor_sync(0xffffffffu, l0, 1); l1 += __shfl_xor_sync(0xffffffffu, l1, 1);
        l0 += __shfl_xor_sync(0xffffffffu, l0, 2); l1 += __shfl_xor_sync(0xffffffffu, l1, 2);
        if (c2 == 0) {
            float* const ml = s_ml + warp * kRows * 2;
            ml[g * 2] = m0; ml[g * 2 + 1] = l0;
            ml[(g + 8) * 2] = m1; ml[(g + 8) * 2 + 1] = l1;
        }
        __syncthreads();
        // the warps bring their accumulators to the common maximum and add them up, one after the other
        float M0 = -INFINITY, M1 = -INFINITY;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
            M0 = fmaxf(M0, s_ml[(w * kRows + g) * 2]);
            M1 = fmaxf(M1, s_ml[(w * kRows + g + 8) * 2]);
        }
        const float f0 = m0 == -INFINITY ? 0.f : exp2f(m0 - M0), f1 = m1 == -INFINITY ? 0.f : exp2f(m1 - M1);
#pragma unroll 1
        for (int w = 0; w < 4; ++w) {
            if (w == (warp & 3)) {
                float* const area = s_o + (warp >> 2) * kRows * C::kPitch;
#pragma unroll
                for (int j = 0; j < D / 8; ++j) {
                    float2* const a = reinterpret_cast<float2*>(area + g * C::kPitch + j * 8 + c2);
                    float2* const b = reinterpret_cast<float2*>(area + (g + 8) * C::kPitch + j * 8 + c2);
                    const float2 x = w ? *a : make_float2(0.f, 0.f);
                    if (g < rows) *a = make_float2(fmaf(f0, o[j][0], x.x), fmaf(f0, o[j][1], x.y));
                    const float2 y = w ? *b : make_float2(0.f, 0.f);
                    if (g + 8 < rows) *b = make_float2(fmaf(f1, o[j][2], y.x), fmaf(f1, o[j][3], y.y));
                }
            }
            __syncthreads();
        }
        const bool whole = t_first == 0 && was.t_end == was.r.slots;
        float* const rec = p.partial + ((size_t)blockIdx.x * 2 + (t_first > 0 ? 0 : 1)) * C::kRec;
        for (int i = tid; i < rows * (D / 4); i += kThreads) {
            const int row = i / (D / 4), col = (i % (D / 4)) * 4;
            float M = -INFINITY, Ls = 0.f;
#pragma unroll
            for (int w = 0; w < kWarps; ++w) M = fmaxf(M, s_ml[(w * kRows + row) * 2]);
#pragma unroll
            for (int w = 0; w < kWarps; ++w) {
                const float mw = s_ml[(w * kRows + row) * 2];
                Ls = fmaf(mw == -INFINITY ? 0.f : exp2f(mw - M), s_ml[(w * kRows + row) * 2 + 1], Ls);     // (0 times a sum that is no number is none)
            }
            float4 acc = *reinterpret_cast<const float4*>(s_o + row * C::kPitch + col);
#pragma unroll
            for (int a = 1; a < C::kAreas; ++a) {
                const float4 v = *reinterpret_cast<const float4*>(s_o + (a * kRows + row) * C::kPitch + col);
                acc.x += v.x; acc.y += v.y; acc.z += v.z; acc.w += v.w;
            }
            if (whole) {
                const float inv = 1.f / Ls;
                const int it = row / p.G, head = was.h * p.G + row - it * p.G;
                const size_t at = ((size_t)was.layer * p.R + was.r.row0 + it) * p.Hq + head;
                *reinterpret_cast<uint2*>(p.out + at * D + col) = make_uint2(attn::pack_bf16(acc.x * inv, acc.y * inv), attn::pack_bf16(acc.z * inv, acc.w * inv));
                if (p.lse_out && col == 0) p.lse_out[at] = M * kAttnLn2 + logf(Ls);
            } else {
                *reinterpret_cast<float4*>(rec + row * D + col) = acc;
                if (col == 0) { rec[kRows * D + row] = M; rec[kRows * D + kRows + row] = Ls; }
            }
        }
        if (last) break;
        __syncthreads();                                            // (the merge area is written again)
    }
    if (dead) {
        // copies on the way land before the CTA's shared memory goes away
        for (; taken < issued; ++taken) ptx::mbar_wait(&bar[taken % kStages], (taken / kStages) & 1, 20000000ll);
    }
}

// The units that the partition cut.  A block per boundary; the blocks whose boundaries cut one unit share its merge by runs of four
// columns, a thread to each.  What takes the time is one trip to L2 after another, so a thread asks for kMergeBatch parts at once.
constexpr int kMergeBatch = 4;
template <int D>
__global__ void __launch_bounds__(kMergeThreads) attn_token_merge_kernel(const __grid_constant__ CausalParams p, const int ctas) {
    constexpr int kRec = kRows * D + 2 * kRows;
    __shared__ attn::GroupBegin s_begin[kMaxCtas];
    const int tid = threadIdx.x, at = blockIdx.x + 1;
    ptx::grid_dep_wait();
    for (int i = tid; i < ctas; i += kMergeThreads) s_begin[i] = p.begins[i];
    __syncthreads();
    const attn::GroupBegin u = s_begin[at];
    if (!u.part) return;
    auto same = [&](int i) { const attn::GroupBegin& v = s_begin[i]; return v.part && v.layer == u.layer && v.b == u.b && v.g == u.g; };
    int ga = at - 1, gb = at;
    while (ga > 0 && same(ga)) --ga;
    while (gb + 1 < ctas && same(gb + 1)) ++gb;
    const int parts = gb - ga + 1, blocks = parts - 1, mine = at - (ga + 1);
    int row0, n, prefix;
    causal::load_request(p, u.b, row0, n, prefix, false);
    // lanes to a run of columns: as many as there are threads for, each with every S-th part
    const int items = n * p.G * (D / 4);
    int S = 1;
    while (S < 32 && 2 * S <= parts && 2 * S * items <= blocks * kMergeThreads) S <<= 1;
    const int lane_s = tid & (S - 1), per_block = kMergeThreads / S;
    for (int i0 = mine * per_block; i0 < items; i0 += blocks * per_block) {
        const int i = min(i0 + tid / S, items - 1);                 // (groups behind the last one do its work, too)
        const int row = i / (D / 4), col = (i % (D / 4)) * 4;
        float M = -INFINITY, L = 0.f;
        float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int k0 = lane_s; k0 < parts; k0 += kMergeBatch * S) {
            float m[kMergeBatch], l[kMergeBatch];
            float4 v[kMergeBatch];
#pragma unroll
            for (int k = 0; k < kMergeBatch; ++k) {                 // (all loads of a batch are on the way at once)
                const int part = k0 + k * S;
                const float* rec = p.partial + ((size_t)(ga + part) * 2 + (part == 0)) * kRec;
                const bool in = part < parts;
                m[k] = in ? rec[kRows * D + row] : -INFINITY;
                l[k] = in ? rec[kRows * D + kRows + row] : 0.f;
                v[k] = in ? *reinterpret_cast<const float4*>(rec + row * D + col) : make_float4(0.f, 0.f, 0.f, 0.f);
            }
            float top = M;
#pragma unroll
            for (int k = 0; k < kMergeBatch; ++k) top = fmaxf(top, m[k]);
            const float keep = M == -INFINITY ? 0.f : exp2f(M - top);
            M = top;
            L *= keep;
            acc.x *= keep; acc.y *= keep; acc.z *= keep; acc.w *= keep;
#pragma unroll
            for (int k = 0; k < kMergeBatch; ++k) {
                const float f = m[k] == -INFINITY ? 0.f : exp2f(m[k] - top);         // (a part that saw nothing)
                L = fmaf(f, l[k], L);
                acc.x = fmaf(f, v[k].x, acc.x); acc.y = fmaf(f, v[k].y, acc.y); acc.z = fmaf(f, v[k].z, acc.z); acc.w = fmaf(f, v[k].w, acc.w);
            }
        }
        if (S > 1) {
            float top = M;
            for (int d = 1; d < S; d <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
            const float f = M == -INFINITY ? 0.f : exp2f(M - top);
            M = top;
            L *= f;
            acc.x *= f; acc.y *= f; acc.z *= f; acc.w *= f;
            for (int d = 1; d < S; d <<= 1) {
                L += __shfl_xor_sync(0xffffffffu, L, d);
                acc.x += __shfl_xor_sync(0xffffffffu, acc.x, d); acc.y += __shfl_xor_sync(0xffffffffu, acc.y, d);
                acc.z += __shfl_xor_sync(0xffffffffu, acc.z, d); acc.w += __shfl_xor_sync(0xffffffffu, acc.w, d);
            }
        }
        if (lane_s != 0 || i0 + tid / S >= items) continue;
        const float inv = 1.f / L;
        const int it = row / p.G, head = u.g * p.G + row - it * p.G;
        const size_t o = ((size_t)u.layer * p.R + row0 + it) * p.Hq + head;
        *reinterpret_cast<uint2*>(p.out + o * D + col) = make_uint2(attn::pack_bf16(acc.x * inv, acc.y * inv), attn::pack_bf16(acc.z * inv, acc.w * inv));
        if (p.lse_out && col == 0) p.lse_out[o] = M * kAttnLn2 + logf(L);
    }
}

template <int D, int kWarps>
mirror_status token_launch(mirror_ctx* ctx, const mirror_kv* kv, const CausalParams& p, size_t records_bytes, cudaStream_t stream) {
    using C = Cfg<D, kWarps>;
    TokenMaps tm;
    mirror_status st = mirror_attn_pool_tmap(ctx, kv, kv->k_pool, &tm.k);
    if (st == MIRROR_OK) st = mirror_attn_pool_tmap(ctx, kv, kv->v_pool, &tm.v);
    if (st != MIRROR_OK) return st;
    // Units of at most 32 slots take a CTA less time whole (8 slots a warp) than a launch that merges their parts.
    const int never_cut = causal_most_slots(p, p.max_rows) <= 32;
    const size_t smem = C::smem(p.B);
    const int ctas = ctx->num_sms * std::max(1, std::min((int)C::kCtas, (int)(kSmemPerSm / (smem + 1024))));
    static_assert(sizeof(attn::GroupBegin) == 16, "notes");
    if (ctas > kMaxCtas || (size_t)ctas * 2 * C::kRec * sizeof(float) > records_bytes) return MIRROR_ERR_SHAPE;
    MIRROR_CUDA_OK(mirror_allow_smem(ctx, kRowsToken + (D == 128) + (kWarps > 4 ? 2 : 0), attn_token_kernel<D, kWarps>, 232448));
    MIRROR_CUDA_OK(mirror_launch_pdl(attn_token_kernel<D, kWarps>, dim3((unsigned)ctas), dim3(C::kThreads), smem, stream, tm, p, never_cut));
    ctx->launches += 1;
    if (!never_cut) {
        MIRROR_CUDA_OK(mirror_launch_pdl(attn_token_merge_kernel<D>, dim3((unsigned)(ctas - 1)), dim3(kMergeThreads), 0, stream, p, ctas));
        ctx->launches += 1;
    }
    MIRROR_CUDA_OK(cudaGetLastError());
    return MIRROR_OK;
}

}  // namespace

mirror_status mirror_attn_pool_tmap(const mirror_ctx* ctx, const mirror_kv* kv, const void* pool, CUtensorMap* map) {
    const uint64_t Hkv = (uint64_t)ctx->desc.n_kv_heads, row = (uint64_t)ctx->desc.head_dim * 2;
    const uint64_t layer_pages = (uint64_t)kv->layer_stride / (Hkv * kAttnSlotTok * (uint64_t)ctx->desc.head_dim);
    const uint64_t rows = ((uint64_t)(kv->num_layers - 1) * layer_pages + (uint64_t)kv->num_pages) * Hkv;
    if (rows >= (1ull << 31)) return MIRROR_ERR_SHAPE;               // (a box's coordinates are 32 bits)
    const uint64_t dims[5] = {64, 8, row / 128, 2, rows};
    const uint64_t strides[4] = {row, 128, 8 * row, kAttnSlotTok * row};
    const uint32_t box[5] = {64, 8, (uint32_t)(row / 128), 2, 1};
    return mirror_make_tmap(ctx, map, pool, 5, dims, strides, box);
}


extern "C" mirror_status mirror_rows_workspace_bytes(const mirror_ctx* ctx, const mirror_rows* rows, size_t* bytes) {
    if (!ctx || !bytes) return MIRROR_ERR_ARG;
    const mirror_status st = mirror_check_rows(rows);
    if (st != MIRROR_OK) return st;
    MirrorWsLayout L;
    mirror_ws_layout(ctx, 1, &L);
    *bytes = align_up(L.end_attn, 256) + std::max(mirror_attn_prompt_plan_bytes(ctx), kMaxCtas * sizeof(attn::GroupBegin));
    return MIRROR_OK;
}

extern "C" mirror_status mirror_attn_causal(mirror_ctx* ctx, const mirror_kv* kv, const mirror_rows* rows, int window, int n_sink,
                                            const void* q, void* out, float* lse_out, void* stream) {
    if (!ctx || !kv || !rows || window < 0 || n_sink < 0) return MIRROR_ERR_ARG;
    mirror_status st = mirror_check_rows(rows);
    if (st != MIRROR_OK || rows->n_rows == 0) return st;
    if (!q || !out) return MIRROR_ERR_ARG;
    st = mirror_check_kv(ctx, kv);
    if (st != MIRROR_OK) return st;
    if (((uintptr_t)q & 15) || ((uintptr_t)out & 15)) return MIRROR_ERR_ARG;
    size_t need = 0;
    st = mirror_rows_workspace_bytes(ctx, rows, &need);
    if (st != MIRROR_OK) return st;
    if (!ctx->ws || ctx->ws_bytes < need) return MIRROR_ERR_WORKSPACE;
    // (positions, and the slots of a layer's units, are counted in 31 bits)
    if (kv->max_pages_per_req > (1 << 26) || (int64_t)rows->batch * kv->max_pages_per_req > (1 << 30)) return MIRROR_ERR_SHAPE;
    MIRROR_CUDA_OK(cudaSetDevice(ctx->device));
    MirrorWsLayout L;
    mirror_ws_layout(ctx, 1, &L);
    CausalParams p;
    p.L = kv->num_layers; p.B = rows->batch; p.R = rows->n_rows; p.Hq = ctx->desc.n_q_heads; p.Hkv = ctx->desc.n_kv_heads;
    p.G = p.Hq / p.Hkv;
    p.max_rows = std::min(rows->max_rows, rows->n_rows);
    p.window = window; p.n_sink = window > 0 ? n_sink : 0;
    p.max_pages = kv->max_pages_per_req; p.num_pages = kv->num_pages;
    p.layer_pages = (int)(kv->layer_stride / ((int64_t)p.Hkv * kAttnSlotTok * ctx->desc.head_dim));
    p.scale_log2e = ctx->scale * 1.4426950408889634f;
    p.row_start = rows->row_start; p.page_table = kv->page_table; p.prefix_len = kv->prefix_len;
    p.q = (const __nv_bfloat16*)q; p.v_pool = (const __nv_bfloat16*)kv->v_pool;
    p.out = (__nv_bfloat16*)out; p.lse_out = lse_out;
    uint8_t* const ws = (uint8_t*)ctx->ws;
    p.begins = (attn::GroupBegin*)(ws + L.notes);
    p.partial = (float*)(ws + L.attn_partial);
    p.status = ctx->d_status;
    p.wait_limit = ctx->tune.wait_limit_cycles;
    void* const notes = ws + align_up(L.end_attn, 256);
    if ((int64_t)p.max_rows * p.G <= kRows) {
        p.begins = (attn::GroupBegin*)notes;
        // Units that are few, a quarter of the SMs at most, get one CTA of twelve warps per SM: a third of the parts to merge, and a short unit
        // is over sooner (32768 tokens x 8 heads 39.6 -> 35.0 us, 300 tokens 11.2 -> 10.1).  Else three or four CTAs of four warps, of which
        // some stream while others merge (96 units of up to 66 slots: 20.4 against 28.2 us).
        const bool few = (int64_t)p.L * p.B * p.Hkv * 4 <= ctx->num_sms;
        auto launch = ctx->desc.head_dim == 128 ? (few ? token_launch<128, 12> : token_launch<128, 4>) : (few ? token_launch<64, 12> : token_launch<64, 4>);
        return launch(ctx, kv, p, L.attn_partial_bytes, (cudaStream_t)stream);
    }
    return mirror_attn_prompt_launch(ctx, kv, p, notes, (cudaStream_t)stream);
}
