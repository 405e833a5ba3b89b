// Causal attention of prompts (mirror_attn_causal with more than 16 rows per KV head), on the tensor cores.
//
// Rows that share one KV head's stream, the gs query heads of the group times tokens, are cut in tiles of at most 128 rows (whole tokens).  A
// unit is (layer, KV head, two neighbouring row tiles of one request); a CTA works on both tiles as two streams over the same K/V tiles in
// shared memory, since one stream alone is a chain (Q K^T -> softmax -> P V) that leaves the tensor cores idle for as long as its
// softmax takes.  A unit's keys are the 16-token slots that some row of it sees: the first slots that stay visible (sinks), then from
// the window of its first row to its last row; eight slots to a tile of 128 keys.  What no row of a stream sees of a tile is neither
// multiplied nor exponentiated.
//
// Units are of any length (prompts are causal), and how many tiles they have only the device knows.  Every CTA, one per SM, makes the same
// plan for itself, in the ring's shared memory, and takes its part:
//   whole  units sorted by length are dealt out in turns, there and back (the longest go with the shortest): nothing is cut
//   cut    the tiles of all units form one sequence that is split evenly.  A unit that a boundary cuts leaves a (max, sum,
//          accumulator) record per part and stream, which attn_prompt_merge_kernel combines in the order of the parts
// whichever ends sooner, a cut counted as kCutTiles and a unit's start and end as kUnitTiles.
//
// Per CTA, 12 warps (as in attn_verify.cu, whose softmax this shares; see there for the offset that stands in for a running maximum):
//   warps 0, 3   stage K and V tiles into one ring; the V warp stages Q too
//   warps 1, 2   issue, one stream each and in turns, P V of one tile and Q K^T of the next.  Warp 1 owns tensor memory
//   warps 4..7, 8..11  softmax of stream 0 and of stream 1, a thread per row
// TMEM: S0 | S1 (128 columns each) | O0 | O1 (d columns each).
// Every mbarrier wait is bounded; on expiry the kernel records MIRROR_DEV_TIMEOUT and unwinds.
//
// What bounds it: the chain of a step (4000 cycles for two streams' 128 x 128 at d = 128, 3430 at d = 64; the tensor pipe is busy for half of them), units'
// starts and ends (4 to 5 thousand cycles each) where prompts are short, and power where they are long.  Measured on a B200: 2048 rows behind
// 30720 tokens, 64 / 8 heads of 128: 1.9 ms (1140 TFLOP/s), 2.2 run back to back; 2048 rows from 0, 40 / 8 heads of 128: 62 us; seven ragged chunks, 32 / 8
// heads of 64 under a window of 1000: 175 to 183 us, from run to run.
// P is one bf16 here (single tokens take two): against 64 bits outputs are 0.0020 to 0.0023 off where their own rounding alone gives 0.0016.
#include <math.h>

#include <algorithm>

#include "attn_causal.h"
#include "attn_softmax.h"

namespace {

using namespace attn;

constexpr int kThreads = 384;
constexpr int kSlotTok = kAttnSlotTok;
constexpr int kTileSlots = 8;
constexpr int kTileTok = kSlotTok * kTileSlots;     // 128
constexpr int kRows = 128;                          // UMMA M: rows of a stream
constexpr int kMaxStages = 10;
constexpr int kTmemCols = 512;
constexpr int kTmemO = 2 * kTileTok;
constexpr int kCtrlBytes = 1536;
constexpr size_t kSmemLimit = 232448;               // 227 KB
constexpr int kSnapTiles = 2;                       // a boundary moves to a unit boundary that is at most this many tiles away
constexpr int kUnitTiles = 1;                       // what a unit costs beside its tiles
constexpr int kCutTiles = 6;                        // what cutting costs: a record, a unit more, the merge behind
constexpr int kMaxList = 24;                        // whole units of a CTA
constexpr int kMaxSorted = kThreads;                // pairs that are sorted
constexpr int kMergeSlotsPrompt = 8;                // (most calls have nothing to merge, or two parts: small blocks, all resident at once)

// A unit: a pair of row tiles of one request, of one layer and head.
struct Unit {
    int row0, n, prefix;                  // the request's rows
    int tok;                              // the pair's first token
    int b, layer, hs, tiles;              // hs: KV head (x share of its query heads); K/V tiles
};
static_assert(sizeof(Unit) == 32, "32 bytes");

struct PromptParams {
    CausalParams c;
    int gs, shares;                       // query heads of a row tile; shares of a group's heads (1 unless G > 128)
    int nt;                               // tokens of a row tile
    int n_hs;                             // KV heads x shares
    int n_cta;
    int wide_out;                         // out on a 32-byte boundary
    int never_cut;                        // units are dealt out whole whatever their lengths: no merge is launched
    Unit* firsts;                         // [n_cta] the unit that each CTA's range begins in, for the merge
};

struct Maps {
    CUtensorMap k, v, q;
};

// The keys of a pair: [0, sink) and [lo, end), in slots as in causal::Request.
struct Keys {
    int lo, sink, end, sink_slots, from, slots;
    __device__ __forceinline__ int page(int t) const { return t < sink_slots ? t : t - sink_slots + from; }
};
__device__ __forceinline__ Keys pair_keys(const PromptParams& p, int n, int prefix, int tok) {
    Keys k;
    k.end = prefix + min(tok + 2 * p.nt, n);
    k.lo = p.c.window > 0 ? min(max(0, prefix + tok - p.c.window + 1), k.end) : 0;
    k.sink = min(p.c.n_sink, k.lo);
    k.from = k.lo / kSlotTok;
    k.sink_slots = min((k.sink + kSlotTok - 1) / kSlotTok, k.from);
    k.slots = k.sink_slots + (k.end + kSlotTok - 1) / kSlotTok - k.from;
    return k;
}

// ---- a CTA's way through its units -----------------------------------------------------------------------------
struct Segment {
    Unit u;
    int t_first, t_last;                  // tiles [t_first, t_last) of the unit
    int k;                                // (whole units) place in the CTA's list
    Keys keys;
};
__device__ __forceinline__ int tiles_of(const PromptParams& p, int n, int prefix, int tok) {
    return (pair_keys(p, n, prefix, tok).slots + kTileSlots - 1) / kTileSlots;
}
__device__ __forceinline__ void fill_segment(Segment& s, const PromptParams& p, int left) {
    s.t_last = min(s.u.tiles, s.t_first + left);
    s.keys = pair_keys(p, s.u.n, s.u.prefix, s.u.tok);
}
// Does some row of stream g see something of tile t?  (Its tokens are tok + g nt and the nt - 1 behind it, as far as they exist.)
struct StreamRows {
    int first, last;                      // positions; last < first: no rows
};
__device__ __forceinline__ StreamRows stream_rows(const PromptParams& p, const Segment& s, int g) {
    const int t0 = s.u.tok + g * p.nt, t1 = min(t0 + p.nt, s.u.n) - 1;
    return {s.u.prefix + t0, s.u.prefix + t1};
}
// (Segments go to a function out of line by their address, so what is read of them again comes from local memory: Keys and StreamRows are
// passed as values, which stay in registers.)
__device__ __forceinline__ bool tile_seen(const PromptParams& p, Keys k, StreamRows r, int t) {
    const int key0 = k.page(t * kTileSlots) * kSlotTok, key1 = k.page(min(t * kTileSlots + kTileSlots, k.slots) - 1) * kSlotTok + kSlotTok - 1;
    return r.last >= r.first && key0 <= r.last && (p.c.window == 0 || key1 > r.first - p.c.window || key0 < p.c.n_sink);
}

// ... and of how many of the tile's slots, from its first?  (What lies behind the stream's last row is not multiplied.)
__device__ __forceinline__ int slots_seen(Keys k, StreamRows r, int t) {
    const int most = min(kTileSlots, k.slots - t * kTileSlots), page0 = k.page(t * kTileSlots);
    const int jump = k.sink_slots > t * kTileSlots ? k.from - k.sink_slots : 0;         // (sinks and window in one tile: by its last slot)
    return max(1, min(most, r.last / kSlotTok + 1 - page0 + (jump > 0 ? most : 0)));
}

struct Ctrl {
    uint64_t full[kMaxStages], empty[kMaxStages];
    uint64_t q_full[2], q_empty[2];                     // per stream: one is through with a unit long before the other
    uint64_t s_full[2], p_full[2][2], o_full[2];        // per stream (P: per half of the tile)
    uint64_t pv_half[2];
    uint64_t turn[2];                                   // the issuing warps take turns
    uint64_t exp_turn[2][4];                            // the two softmax warps of a scheduler take turns
    Unit first;                                         // where this CTA begins
    int first_t, n_tiles, whole;
    int cut, too_long;                                  // it begins inside a unit; more tiles than 31 bits count
    int makespan, ends[2];
    uint32_t scan[kThreads / 32];
    int* status;
    long long wait_limit;
    uint32_t tmem_base;
    volatile int abort;
    Unit list[kMaxList];                                // its units, where they are dealt out whole
};
static_assert(sizeof(Ctrl) <= kCtrlBytes, "control block");

// On to the next unit (there is one).
__device__ __noinline__ void next_segment(Segment& s, const PromptParams& p, const Ctrl* ctrl, int left) {
    s.t_first = 0;
    if (ctrl->whole) {
        s.u = ctrl->list[++s.k];
    } else {
        s.u.tok += 2 * p.nt;
        while (s.u.tok >= s.u.n) {                       // (requests without rows are passed over)
            s.u.tok = 0;
            if (++s.u.b == p.c.B) {
                s.u.b = 0;
                if (++s.u.hs == p.n_hs) {
                    s.u.hs = 0;
                    if (++s.u.layer >= p.c.L) break;     // (the lengths have been changed under the call)
                }
            }
            causal::load_request(p.c, s.u.b, s.u.row0, s.u.n, s.u.prefix, false);
        }
        s.u.tiles = max(tiles_of(p, s.u.n, s.u.prefix, s.u.tok), 1);
    }
    fill_segment(s, p, left);
}

// ---- the plan: every CTA for itself ----------------------------------------------------------------------------
// It is made twice as far as its inputs are concerned: ahead of the kernel in front, from whatever the lengths are then (nothing but this
// CTA's shared memory is written), and once that kernel is through the lengths are read again: hardly ever has one changed, and then the
// plan is made anew.  (It takes 4 us, most of them for code that runs once.)

// Tiles, inclusive over the block.  (A page table has at most 2^26 entries, a pair at most 2^23 tiles: those of a block fit 32 bits.)
__device__ uint32_t block_scan(uint32_t v, uint32_t* s_warp, uint32_t* total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const uint32_t t = __shfl_up_sync(0xffffffffu, v, o);
        if (lane >= o) v += t;
    }
    __syncthreads();
    if (lane == 31) s_warp[warp] = v;
    __syncthreads();
    uint32_t before = 0, all = 0;
    for (int w = 0; w < kThreads / 32; ++w) {
        if (w < warp) before += s_warp[w];
        all += s_warp[w];
    }
    *total = all;
    return v + before;
}
// Scratch in shared memory: pairs summed over the requests, and the requests' rows.
struct Scratch {
    int *base, *row0, *n, *prefix;        // [B + 1], [B] each
    int *sorted, *sorted_tiles;           // [kMaxSorted]: pairs by length
    __device__ Scratch(int* mem, int B) : base(mem + 2 * kMaxSorted), row0(base + B + 1), n(row0 + B), prefix(n + B), sorted(mem), sorted_tiles(mem + kMaxSorted) {}
};
// The requests' rows; has one changed?
__device__ __forceinline__ bool load_rows(const PromptParams& p, const Scratch& x, bool report_it) {
    bool changed = false;
    for (int b = threadIdx.x; b < p.c.B; b += kThreads) {
        int row0, n, prefix;
        causal::load_request(p.c, b, row0, n, prefix, report_it);
        changed |= x.row0[b] != row0 || x.n[b] != n || x.prefix[b] != prefix;
        x.row0[b] = row0; x.n[b] = n; x.prefix[b] = prefix;
    }
    return changed;
}
__device__ __noinline__ void make_plan(const PromptParams& p, Ctrl* ctrl, int* mem) {
    const int tid = threadIdx.x, lane = tid & 31, B = p.c.B, cta = blockIdx.x;
    const Scratch x(mem, B);
    // (sums stop one above what rows in ascending order come to, of which each belongs to one request)
    const int most_pairs = p.c.R / (2 * p.nt) + B + 1;
    for (int b = tid; b < B; b += kThreads) x.base[b + 1] = (x.n[b] + 2 * p.nt - 1) / (2 * p.nt);
    if (tid == 0) { x.base[0] = 0; ctrl->makespan = 0; ctrl->n_tiles = 0; ctrl->whole = 0; ctrl->cut = 0; ctrl->too_long = 0; }
    __syncthreads();
    if (tid < 32) {
        int acc = 0;
        for (int b0 = 0; b0 < B; b0 += 32) {
            int v = b0 + lane < B ? x.base[b0 + lane + 1] : 0;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int t = __shfl_up_sync(0xffffffffu, v, o);
                if (lane >= o) v = min(v + t, most_pairs);
            }
            v = min(acc + v, most_pairs);
            if (b0 + lane < B) x.base[b0 + lane + 1] = v;
            acc = __shfl_sync(0xffffffffu, v, 31);
        }
    }
    __syncthreads();
    const int pairs = x.base[B];
    if (pairs == 0 || pairs == most_pairs) return;       // (rows that are not in order have been reported)
    auto pair = [&](int c) {                             // pair number c, in the order of the rows
        int lo = 0, hi = B - 1;                          // the first b with base[b + 1] > c
        while (lo < hi) {
            const int mid = (lo + hi) >> 1;
            if (x.base[mid + 1] > c) hi = mid; else lo = mid + 1;
        }
        Unit u;
        u.b = lo; u.row0 = x.row0[lo]; u.n = x.n[lo]; u.prefix = x.prefix[lo];
        u.tok = (c - x.base[lo]) * 2 * p.nt;
        u.layer = u.hs = 0;
        u.tiles = tiles_of(p, u.n, u.prefix, u.tok);
        return u;
    };
    Unit mine = {};
    long long total = 0, cum = 0;                        // tiles of all pairs; of those before `mine`
    for (int c0 = 0; c0 < pairs; c0 += kThreads) {
        mine = {};
        if (c0 + tid < pairs) mine = pair(c0 + tid);
        uint32_t all;
        cum = total + block_scan((uint32_t)mine.tiles, ctrl->scan, &all) - mine.tiles;
        total += all;
    }
    const int lh = p.c.L * p.n_hs;
    const long long seq = lh * total, units = (long long)lh * pairs;
    if (seq >= (1ll << 31)) {
        if (tid == 0) ctrl->too_long = 1;
        return;
    }
    const int rounds = (int)min((units + p.n_cta - 1) / p.n_cta, 1000ll);
    auto dealt = [&](int k, int c) -> int { return k * p.n_cta + ((k & 1) ? p.n_cta - 1 - c : c); };          // (few rounds)
    if (pairs <= kMaxSorted && rounds <= kMaxList) {
        if (tid < pairs) {
            x.sorted[tid] = tid;
            x.sorted_tiles[tid] = mine.tiles;
        }
        bool whole = p.never_cut != 0;
        if (rounds == 1) {                               // (nothing to sort: a CTA has one unit at most)
            if (!whole) {
                const int load = __reduce_max_sync(0xffffffffu, mine.tiles + kUnitTiles);
                if (lane == 0) atomicMax(&ctrl->makespan, load);
            }
            __syncthreads();
        } else {
            // longest first; of equals the first
            __syncthreads();
            int at = 0;
            if (tid < pairs)
#pragma unroll 8
                for (int c = 0; c < pairs; ++c) at += x.sorted_tiles[c] > mine.tiles || (x.sorted_tiles[c] == mine.tiles && c < tid);
            __syncthreads();
            if (tid < pairs) { x.sorted[at] = tid; x.sorted_tiles[at] = mine.tiles; }
            __syncthreads();
            if (!whole) {
                int load = 0;
                if (tid < p.n_cta) {
#pragma unroll 4
                    for (int k = 0; k < rounds; ++k) {
                        const uint32_t v = (uint32_t)dealt(k, tid);
                        if (v < (uint32_t)units) load += x.sorted_tiles[v / (uint32_t)lh] + kUnitTiles;
                    }
                }
                load = __reduce_max_sync(0xffffffffu, load);
                if (lane == 0) atomicMax(&ctrl->makespan, load);
                __syncthreads();
            }
        }
        whole |= ctrl->makespan <= (int)((seq + units * kUnitTiles) / p.n_cta) + kCutTiles;
        if (whole) {
            int tiles = 0;
            if (tid < rounds) {
                const int v = dealt(tid, cta);
                if (v < units) {
                    const int r = v / lh, l = v - r * lh;
                    Unit u = pair(x.sorted[r]);
                    u.layer = l / p.n_hs;
                    u.hs = l - u.layer * p.n_hs;
                    ctrl->list[tid] = u;
                    tiles = u.tiles;
                    if (tid == 0) { ctrl->first = u; ctrl->first_t = 0; }
                }
            }
            if (tid < 32) {
                tiles = __reduce_add_sync(0xffffffffu, tiles);
                if (lane == 0) {
                    ctrl->n_tiles = tiles;
                    ctrl->whole = 1;
                }
            }
            return;
        }
    }
    // ---- an even split: where this CTA's range begins and ends
    const int used = (int)min((long long)p.n_cta, seq);
    const int tol = (int)min((long long)kSnapTiles, seq / used >> 2);
    long long x0 = cta >= used ? seq : seq * cta / used, x1 = cta + 1 >= used ? seq : seq * (cta + 1) / used;
    const int per = (int)total;                          // tiles of one (layer, head)
    const int lh0 = (int)(x0 / per), rem0 = (int)(x0 - (long long)lh0 * per), rem1 = (int)(x1 % per);
    int* const s_ends = ctrl->ends;
    if (tid == 0) { s_ends[0] = (int)x0; s_ends[1] = (int)x1; }
    long long seen = 0;
    for (int c0 = 0; c0 < pairs; c0 += kThreads) {
        if (pairs > kThreads) {                          // (a second time: the first kept the last pairs only)
            mine = {};
            if (c0 + tid < pairs) mine = pair(c0 + tid);
            uint32_t all;
            cum = seen + block_scan((uint32_t)mine.tiles, ctrl->scan, &all) - mine.tiles;
            seen += all;
        }
        __syncthreads();
        if (c0 + tid < pairs) {
            // (this pair's tiles lie in front of both boundaries' places within their head, or hold them)
            if (x0 < seq && rem0 >= cum && rem0 < cum + mine.tiles) {
                Unit u = mine;
                int t = rem0 - (int)cum, at = lh0;
                if (t <= tol) {
                    s_ends[0] = (int)x0 - t;
                    t = 0;
                } else if (mine.tiles - t <= tol) {      // (to the next unit)
                    s_ends[0] = (int)x0 + mine.tiles - t;
                    t = 0;
                    const int c = c0 + tid + 1;
                    u = pair(c < pairs ? c : 0);
                    at += c == pairs;
                }
                u.layer = at / p.n_hs;
                u.hs = at - u.layer * p.n_hs;
                ctrl->first = u;
                ctrl->first_t = t;
            }
            if (x1 < seq && rem1 >= cum && rem1 < cum + mine.tiles) {
                const int t = rem1 - (int)cum;
                if (t <= tol) s_ends[1] = (int)x1 - t;
                else if (mine.tiles - t <= tol) s_ends[1] = (int)x1 + mine.tiles - t;
            }
        }
    }
    __syncthreads();
    if (tid == 0) {
        const int n = s_ends[1] - s_ends[0];
        ctrl->n_tiles = n;
        ctrl->cut = n > 0 && ctrl->first_t > 0;
    }
}

template <int D>
struct Cfg {
    static constexpr int kHalves = D / 64;
    static constexpr int kSlotBytes = kHalves * kSlotTok * 128;
    static constexpr int kGroupStride = kHalves * 1024;
    static constexpr int kStageBytes = kTileSlots * kSlotBytes;
    static constexpr int kQHalfBytes = kRows * 128;
    static constexpr int kQBytes = kHalves * kQHalfBytes;
};

// Scores of tokens that the row at position `pos` does not see become -inf, in TMEM; `rows` are the stream's positions.  A slot at a time,
// and little code: most of a tile's slots are seen by all rows, or by none, and what runs once per unit is bound by the fetch of its
// instructions (32 columns at a time, unrolled, with the maximum taken on the way: 4400 cycles, this and tile_max 2500).
__device__ __noinline__ void mask_tile(uint32_t s_addr, int slot0, int slots, int sink_slots, int from, int n_slots, int pos, int row_first, int row_last, int window, int n_sink) {
    // (what lies up to there is out of the window; without one, or with one past all positions, nothing does)
    window = window == 0 ? 1 << 30 : min(window, 1 << 30);
    const int first_lo = row_first - window, last_lo = row_last - window;
    auto bits = [](int n) { return 1u << min(max(n, 0), 16); };
#pragma unroll 1
    for (int c = 0; c < slots; ++c, s_addr += 16) {
        const int sl = slot0 + c, key0 = (sl < sink_slots ? sl : sl - sink_slots + from) * kSlotTok, key1 = key0 + kSlotTok - 1;
        const bool there = sl < n_slots;
        if (there && key1 <= row_first && (key0 > last_lo || key1 < n_sink)) continue;
        uint32_t r[16], m = 0;
        if (there && key0 <= row_last && (key1 > first_lo || key0 < n_sink)) {
            ptx::tmem_ld_32x32b_x16(s_addr, r);
            const int n = pos + 1 - key0;                                                  // of the slot's tokens those ahead of the row's, and its own
            m = (bits(n) - 1u) & (0u - bits(n - window) | (bits(n_sink - key0) - 1u));
            tmem_ld_wait16(r);
        }
#pragma unroll
        for (int j = 0; j < 16; ++j) r[j] = (m & (1u << j)) ? r[j] : 0xff800000u;
        tmem_st_32x32b_x16(s_addr, r);
    }
    tmem_st_wait();
}

// 32 bytes of a row
__device__ __forceinline__ void store32(__nv_bfloat16* dst, const uint32_t* a, float f, bool wide) {
    uint32_t w[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) w[j] = pack_bf16(f * __uint_as_float(a[2 * j]), f * __uint_as_float(a[2 * j + 1]));
    if (wide) {
        asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
                     ::"l"(dst), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7]) : "memory");
    } else {
        *reinterpret_cast<uint4*>(dst) = make_uint4(w[0], w[1], w[2], w[3]);
        *reinterpret_cast<uint4*>(dst + 8) = make_uint4(w[4], w[5], w[6], w[7]);
    }
}

template <int D>
__global__ void __launch_bounds__(kThreads, 1) attn_prompt_kernel(const __grid_constant__ Maps tm, const __grid_constant__ PromptParams p, const int n_stages) {
    using C = Cfg<D>;
    extern __shared__ __align__(1024) uint8_t smem[];
    uint8_t* const sQ = smem;                                            // [2 streams]
    uint8_t* const ring = sQ + 2 * C::kQBytes;                           // [n_stages] K or V tiles: K of a tile, V of it, K of the next
    Ctrl* const ctrl = (Ctrl*)(ring + (size_t)n_stages * C::kStageBytes);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;

    // ---- prologue, while the kernel ahead is still running: of global memory the lengths alone are read (and again behind the wait)
    if (tid == 0) {
        for (int s = 0; s < n_stages; ++s) { ptx::mbar_init(&ctrl->full[s], 1); ptx::mbar_init(&ctrl->empty[s], 2); }
        for (int g = 0; g < 2; ++g) {
            ptx::mbar_init(&ctrl->q_full[g], 1); ptx::mbar_init(&ctrl->q_empty[g], 1);
            ptx::mbar_init(&ctrl->s_full[g], 1); ptx::mbar_init(&ctrl->p_full[g][0], 4); ptx::mbar_init(&ctrl->p_full[g][1], 4);
            ptx::mbar_init(&ctrl->o_full[g], 1); ptx::mbar_init(&ctrl->turn[g], 1); ptx::mbar_init(&ctrl->pv_half[g], 1);
            for (int s = 0; s < 4; ++s) ptx::mbar_init(&ctrl->exp_turn[g][s], 1);
        }
        ctrl->abort = 0;
        ctrl->status = p.c.status;
        ctrl->wait_limit = p.c.wait_limit;
        ptx::fence_mbar_init();
        ptx::prefetch_tmap(&tm.k); ptx::prefetch_tmap(&tm.v); ptx::prefetch_tmap(&tm.q);
    }
    // rows that the Q copies do not fill are zeros
    const int q_rows = p.gs * p.nt, pad = kRows - q_rows;
    for (int i = tid; i < 2 * C::kHalves * pad * 8; i += kThreads) {
        const int half = i / (pad * 8), c = i - half * pad * 8;
        *reinterpret_cast<uint4*>(sQ + half * C::kQHalfBytes + q_rows * 128 + c * 16) = make_uint4(0, 0, 0, 0);
    }
    ptx::fence_proxy_async();
    if (warp == 1) {
        ptx::tmem_alloc(&ctrl->tmem_base, kTmemCols);
        ptx::tmem_relinquish();
    }
    const Scratch lengths((int*)ring, p.c.B);
    load_rows(p, lengths, false);
    ptx::tc_fence_before();
    __syncthreads();
    ptx::tc_fence_after();
    make_plan(p, ctrl, (int*)ring);
    ptx::grid_dep_wait();
    ptx::grid_dep_launch();
    if (__syncthreads_or(load_rows(p, lengths, blockIdx.x == 0))) make_plan(p, ctrl, (int*)ring);
    ptx::fence_proxy_async();                            // (the ring is filled by copies from here on)
    __syncthreads();
    if (tid == 0) {
        if (ctrl->too_long) causal::report(p.c.status, MIRROR_DEV_CHECK, 833);
        if (!p.never_cut) {
            const Unit& u = ctrl->first;
            p.c.begins[blockIdx.x] = ctrl->cut ? GroupBegin{1, u.layer, u.row0 + u.tok, u.hs} : GroupBegin{0, 0, 0, 0};
            if (ctrl->cut) p.firsts[blockIdx.x] = u;
        }
    }
    const uint32_t tmem_base = ctrl->tmem_base;
    const int n_tiles = ctrl->n_tiles;
    auto first_segment = [&](Segment& s) {
        s.u = ctrl->first;
        s.t_first = ctrl->first_t;
        s.k = 0;
        fill_segment(s, p, n_tiles);
    };

    if (n_tiles <= 0) {
        // (no tiles: nothing to do)
    } else if (warp == 0 || warp == 3) {
        // ======================================================================= K and V producers, Q with V
        const bool V = warp == 3;
        const CUtensorMap* const map = V ? &tm.v : &tm.k;
        Segment sg;
        first_segment(sg);
        int left = n_tiles, t = sg.t_first;
        uint32_t seq = V ? 1 : 0, n_seg = 0;
        bool ok = true;
        int pg = 0, pg_next = 0;
        Keys keys = sg.keys;
        const int32_t* table = nullptr;                              // the request's pages
        int row0 = 0, kvh = 0, t_last = 0;                           // the layer's first page
        auto fetch = [&](int tt) -> int {                            // physical pages of a tile, one per lane (0..7)
            const int sl = tt * kTileSlots + lane;
            return (lane < kTileSlots && sl < keys.slots) ? table[keys.page(sl)] : 0;
        };
        auto load_q = [&]() {
            const int head = kvh * p.c.G + (sg.u.hs - kvh * p.shares) * p.gs;
            for (int g = 0; g < 2; ++g) {
                if (!ptx::warp_wait(ctrl, &ctrl->q_empty[g], (n_seg & 1) ^ 1, 61)) { ok = false; return; }
                if (ptx::elect_one()) {
                    ptx::mbar_arrive_expect_tx(&ctrl->q_full[g], (uint32_t)(C::kHalves * q_rows * 128));
                    for (int h = 0; h < C::kHalves; ++h)
                        ptx::tma_load_5d(sQ + g * C::kQBytes + h * C::kQHalfBytes, &tm.q, &ctrl->q_full[g], 0, head, sg.u.layer * p.c.R + sg.u.row0 + sg.u.tok + g * p.nt, h, 0);
                }
                __syncwarp();
            }
            ++n_seg;
        };
        // what some row of the request sees (see causal::Request); the rest of V may be anything, and is taken as zeros
        int req_lo = 0, req_sink = 0, req_len = 0;
        auto unit = [&]() {
            keys = sg.keys;
            t_last = sg.t_last;
            table = p.c.page_table + (size_t)sg.u.b * p.c.max_pages;
            row0 = sg.u.layer * p.c.layer_pages;
            kvh = sg.u.hs / p.shares;
            req_len = sg.u.prefix + sg.u.n;
            req_lo = p.c.window > 0 ? min(max(0, sg.u.prefix - p.c.window + 1), req_len) : 0;
            req_sink = min(p.c.n_sink, req_lo);
        };
        unit();
        pg_next = fetch(t);
        if (V) load_q();
#pragma unroll 1
        while (left > 0 && ok) {
            pg = pg_next;
            if (t + 1 < t_last) pg_next = fetch(t + 1);
            const uint32_t st = seq % (uint32_t)n_stages;
            if (!ptx::warp_wait(ctrl, &ctrl->empty[st], ((seq / (uint32_t)n_stages) & 1) ^ 1, 60)) { ok = false; break; }
            uint8_t* const dst = ring + (size_t)st * C::kStageBytes;
            uint64_t* const bar = &ctrl->full[st];
            const int sl0 = t * kTileSlots, n_sl = min(kTileSlots, keys.slots - sl0);
            if (pg < 0 || pg >= p.c.num_pages) { causal::report(p.c.status, MIRROR_DEV_CHECK, 832); pg = 0; }
            uint32_t partial = 0;                                    // V: slots with tokens that no row of the request sees
            if (V) {
                const int key0 = keys.page(sl0 + (lane & 7)) * kSlotTok;
                partial = __ballot_sync(0xffffffffu, lane < n_sl && (key0 + kSlotTok > req_len || (key0 < req_lo && key0 + kSlotTok > req_sink)));
                if (partial) {
                    for (int k = 0; k < n_sl; ++k) {
                        if (!(partial >> k & 1)) continue;
                        const int page = __shfl_sync(0xffffffffu, pg, k), base = keys.page(sl0 + k) * kSlotTok;
                        const uint8_t* const src = (const uint8_t*)p.c.v_pool + ((size_t)(row0 + page) * p.c.Hkv + kvh) * (size_t)C::kSlotBytes;
                        constexpr int kRowChunks = D / 8;
#pragma unroll 1
                        for (int c = lane; c < kSlotTok * kRowChunks; c += 32) {
                            const int tr = c / kRowChunks, cc = c % kRowChunks, key = base + tr;
                            const bool seen = key < req_len && (key >= req_lo || key < req_sink);
                            asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;"
                                         ::"r"(ptx::smem_u32(dst + k * C::kSlotBytes + kv_slot_off<C::kHalves>(tr, cc))), "l"(src + c * 16), "r"(seen ? 16u : 0u) : "memory");
                        }
                    }
                    asm volatile("cp.async.wait_all;" ::: "memory");
                    ptx::fence_proxy_async();
                    __syncwarp();
                }
            }
            // (the barrier's one arrival is its arming, so copies that land before it cannot complete the phase)
            if (n_sl == kTileSlots && !partial) {
                int row[kTileSlots];
#pragma unroll
                for (int k = 0; k < kTileSlots; ++k) row[k] = (row0 + __shfl_sync(0xffffffffu, pg, k)) * p.c.Hkv + kvh;
                if (ptx::elect_one()) {
                    ptx::mbar_arrive_expect_tx(bar, (uint32_t)C::kStageBytes);
#pragma unroll
                    for (int k = 0; k < kTileSlots; ++k) ptx::tma_load_5d(dst + k * C::kSlotBytes, map, bar, 0, 0, 0, 0, row[k]);
                }
            } else {
                const bool leader = ptx::elect_one();
                if (leader) ptx::mbar_arrive_expect_tx(bar, (uint32_t)((n_sl - __popc(partial)) * C::kSlotBytes));
#pragma unroll 1
                for (int k = 0; k < n_sl; ++k) {
                    const int page = __shfl_sync(0xffffffffu, pg, k);
                    if (leader && !(partial >> k & 1)) ptx::tma_load_5d(dst + k * C::kSlotBytes, map, bar, 0, 0, 0, 0, (row0 + page) * p.c.Hkv + kvh);
                }
            }
            __syncwarp();
            seq += 2;
            --left;
            if (++t == t_last && left > 0) {
                next_segment(sg, p, ctrl, left);
                t = 0;
                unit();
                pg_next = fetch(0);
                if (V) load_q();
            }
        }
        if (!ok) {
            // let copies already on the way land before the CTA's shared memory goes away
            for (int k = 0; k <= n_stages / 2 + 1 && seq >= 2; ++k) {
                seq -= 2;
                ptx::mbar_wait(&ctrl->full[seq % (uint32_t)n_stages], (seq / (uint32_t)n_stages) & 1, 20000000ll);
            }
            // (of a unit whose second Q was not asked for the wait runs out: it is bounded)
            if (V && n_seg > 0)
                for (int g = 0; g < 2; ++g) ptx::mbar_wait(&ctrl->q_full[g], (n_seg - 1) & 1, 20000000ll);
        }
    } else if (warp < 4) {
        // ======================================================================= tensor-core issuers (see attn_verify.cu)
        const uint32_t hi_q = ptx::umma_desc_hi_sw128(1024), hi_k = ptx::umma_desc_hi_sw128(C::kGroupStride), hi_v = hi_k;
        const int g = warp - 1;
        const uint32_t q_lo = ptx::umma_desc_lo(ptx::smem_u32(sQ + g * C::kQBytes), 16);
        const uint32_t k_lo = ptx::umma_desc_lo(ptx::smem_u32(ring), 16);
        const uint32_t v_lo = ptx::umma_desc_lo(ptx::smem_u32(ring), 1024);        // MN-major: LBO = next 64-column atom
        const uint32_t idesc_pv = ptx::umma_idesc_bf16(kRows, D) | (1u << 16);
        const uint32_t q_half = (uint32_t)(C::kQHalfBytes >> 4);
        const uint32_t s_d = tmem_base + (uint32_t)(g * kTileTok), o_d = tmem_base + kTmemO + (uint32_t)(g * D);
        bool ok = true;
        auto wait = [&](uint64_t* bar, uint32_t parity, int where) { ok = ok && ptx::warp_wait(ctrl, bar, parity, where); };
        uint32_t st = 0, ph = 0;
        auto take = [&]() -> uint32_t {
            const uint32_t s = st;
            wait(&ctrl->full[s], ph, 62);
            if (++st == (uint32_t)n_stages) { st = 0; ph ^= 1; }
            return s;
        };
        uint32_t p_par = 0, q_par = 0, turn_par = g == 0 ? 1 : 0;
        Segment sg;
        first_segment(sg);
        StreamRows rows = stream_rows(p, sg, g);
        Keys keys = sg.keys;
        int t_first = sg.t_first, t_last = sg.t_last;
        int left = n_tiles, t = t_first;                          // the tile whose Q K^T comes next
        bool has_pv = false, pv_on = false, pv_last = false, started = false;
        int pv_sl = 0;
#pragma unroll 1
        while (ok) {
            const bool has_qk = left > 0, qk_on = has_qk && tile_seen(p, keys, rows, t), qk_last = has_qk && t + 1 == t_last;
            const int qk_sl = has_qk ? slots_seen(keys, rows, t) : 0;
            const uint32_t idesc_qk = ptx::umma_idesc_bf16(kRows, qk_sl * kSlotTok);
            uint32_t vst = 0, kst = 0;
            if (has_pv) vst = take();
            if (has_qk) {
                kst = take();
                if (t == t_first) { wait(&ctrl->q_full[g], q_par, 63); q_par ^= 1; }
            }
            const uint32_t vb = v_lo + vst * (uint32_t)(C::kStageBytes >> 4);
            auto pv = [&](int k0, int k1) {
#pragma unroll 1
                for (int k = k0; k < k1; ++k)
                    ptx::umma_f16_tmem_a(o_d, s_d + (uint32_t)(k * 8), vb + (uint32_t)(k * (C::kSlotBytes / 16)), hi_v, idesc_pv, k > 0 || started);
            };
            if (has_pv) {
                wait(&ctrl->p_full[g][0], p_par, 64);
                if (!ok) break;
                ptx::tc_fence_after();
                if (ptx::elect_one()) {
                    if (pv_on) pv(0, min(pv_sl, kTileSlots / 2));
                    ptx::umma_commit(&ctrl->pv_half[g]);
                }
                __syncwarp();
                wait(&ctrl->p_full[g][1], p_par, 65);
                p_par ^= 1;
            }
            wait(&ctrl->turn[g], turn_par, 66);
            turn_par ^= 1;
            if (!ok) break;
            ptx::tc_fence_after();
            const uint32_t kb = k_lo + kst * (uint32_t)(C::kStageBytes >> 4);
            if (ptx::elect_one()) {
                if (has_pv) {
                    if (pv_on) pv(kTileSlots / 2, pv_sl);
                    ptx::umma_commit(&ctrl->empty[vst]);
                    if (pv_last) ptx::umma_commit(&ctrl->o_full[g]);
                }
                if (has_qk) {
                    if (qk_on) {
#pragma unroll 1
                        for (int kk = 0; kk < D / 16; ++kk)
                            ptx::umma_f16_lohi(s_d, q_lo + (kk >> 2) * q_half + (uint32_t)((kk & 3) * 2), hi_q, kb + (uint32_t)((kk >> 2) * 64 + (kk & 3) * 2), hi_k, idesc_qk, kk != 0);
                    }
                    ptx::umma_commit(&ctrl->s_full[g]);
                    ptx::umma_commit(&ctrl->empty[kst]);
                    if (qk_last) ptx::umma_commit(&ctrl->q_empty[g]);
                }
                ptx::mbar_arrive(&ctrl->turn[g ^ 1]);
            }
            __syncwarp();
            if (!has_qk) break;
            if (has_pv) started = pv_last ? false : started || pv_on;
            has_pv = true;
            pv_on = qk_on;
            pv_last = qk_last;
            pv_sl = qk_sl;
            --left;
            if (++t == t_last && left > 0) {
                next_segment(sg, p, ctrl, left);
                rows = stream_rows(p, sg, g);
                keys = sg.keys;
                t_last = sg.t_last;
                t = t_first = 0;
            }
        }
    } else {
        // ======================================================================= softmax
        const int grp = (warp - 4) >> 2, w4 = warp & 3, row = w4 * 32 + lane;
        const int it = row / p.gs, hl = row - it * p.gs;             // token of the tile, head of the share
        const uint32_t lane_base = tmem_base + ((uint32_t)(w4 * 32) << 16);
        const uint32_t s_addr = lane_base + (uint32_t)(grp * kTileTok), o_addr = lane_base + kTmemO + (uint32_t)(grp * D);
        constexpr int kRowW = D + 4;                                 // record: D accumulator columns, then (max, sum)
        const float sc = p.c.scale_log2e;
        const uint64_t sc2 = pack2(sc, sc);
        uint32_t t_par = grp == 0 ? 1 : 0, s_par = 0, o_par = 0;
        auto take_turn = [&]() -> bool {
            const bool r = ptx::warp_wait(ctrl, &ctrl->exp_turn[grp][w4], t_par, 67);
            t_par ^= 1;
            return r;
        };
        auto pass_turn = [&]() {
            __syncwarp();
            if (lane == 0) ptx::mbar_arrive(&ctrl->exp_turn[grp ^ 1][w4]);
        };
        bool ok = true;
        int left = n_tiles;
        Segment sg;
        first_segment(sg);
#pragma unroll 1
        while (left > 0 && ok) {
            const StreamRows rows = stream_rows(p, sg, grp);
            const int kvh = sg.u.hs / p.shares, hg = (sg.u.hs - kvh * p.shares) * p.gs + hl;                     // head within the group
            const int tok = sg.u.tok + grp * p.nt + it, pos = sg.u.prefix + tok;
            const bool row_ok = it < p.nt && tok < sg.u.n && hg < p.c.G;
            const bool warp_has_rows = __any_sync(0xffffffffu, row_ok);
            float off = row_ok ? -INFINITY : 1e30f, l_run = 0.f;
            const Keys keys = sg.keys;
            const int t_last = sg.t_last;
            bool redone = false, any_tile = false;                   // any_tile: the accumulator holds something
#pragma unroll 1
            for (int t = sg.t_first; t < t_last; ++t) {
                const bool on = tile_seen(p, keys, rows, t);
                if (!ptx::warp_wait(ctrl, &ctrl->s_full[grp], s_par, 68)) { ok = false; break; }
                s_par ^= 1;
                ptx::tc_fence_after();
                if (warp_has_rows && on) {
                    const int key0 = keys.page(t * kTileSlots) * kSlotTok;
                    const bool whole_tile = (t + 1) * kTileSlots <= keys.slots && keys.page(t * kTileSlots + kTileSlots - 1) * kSlotTok + kSlotTok - 1 <= rows.first &&
                                            (p.c.window == 0 || key0 > rows.last - p.c.window);
                    // Two halves of 64 scores, one copy of the code (the second left out where no row sees it).  P of a half goes over S columns
                    // that have been read.
                    const int halves = slots_seen(keys, rows, t) > kTileSlots / 2 ? 2 : 1;
                    // The offset is set by the first tile in which the row sees anything (before that every P was 0).
                    if (!whole_tile) mask_tile(s_addr, t * kTileSlots, halves * (kTileSlots / 2), keys.sink_slots, keys.from, keys.slots, pos, rows.first, rows.last, p.c.window, p.c.n_sink);
                    if (__any_sync(0xffffffffu, off == -INFINITY)) {
                        const float mx = tile_max(s_addr, 2 * halves);
                        if (off == -INFINITY) off = mx * sc;       // (-inf when nothing is visible yet)
                    }
                    float sum = 0.f;
                    uint32_t ra[32];
                    ptx::tmem_ld_32x32b_x32(s_addr, ra);
                    if (!take_turn()) { ok = false; break; }
#pragma unroll 1
                    for (int h = 0; h < halves;) {
                        uint32_t pk[32], rb[32];
                        const float o = (off == -INFINITY) ? 0.f : -off;
                        const uint64_t no2 = pack2(o, o);
                        uint64_t s0 = 0, s1 = 0;
                        tmem_ld_wait32(ra);
                        ptx::tmem_ld_32x32b_x32(s_addr + (uint32_t)(h * 64 + 32), rb);
                        exp_chunk<false>(ra, sc2, no2, pk, s0, s1);
                        tmem_ld_wait32(rb);
                        ptx::tmem_ld_32x32b_x32(s_addr + 64, ra);    // (of no use to the second half)
                        exp_chunk<false>(rb, sc2, no2, pk + 16, s0, s1);
                        float a, b;
                        unpack2(add2(s0, s1), a, b);
                        const float half_sum = a + b;
                        if (h == halves - 1 && !redone) pass_turn();
                        const bool grow = half_sum > kSumLimit && !redone;
                        if (__any_sync(0xffffffffu, grow)) {
                            tmem_ld_wait32(ra);
                            if (h == 1) {
                                if (!ptx::warp_wait(ctrl, &ctrl->pv_half[grp], s_par ^ 1, 69)) { ok = false; break; }
                                ptx::tc_fence_after();
                            }
                            const float2 m = move_offset(s_addr + (uint32_t)(h * 64), o_addr, any_tile || h > 0 ? D : 0, grow, off, sc);
                            off = m.x;
                            l_run *= m.y;
                            sum *= m.y;
                            redone = true;
                            ptx::tmem_ld_32x32b_x32(s_addr + (uint32_t)(h * 64), ra);
                            continue;
                        }
                        redone = false;
                        sum += half_sum;
                        tmem_st_32x32b_x32(s_addr + (uint32_t)(h * 32), pk);
                        tmem_st_wait();
                        ptx::tc_fence_before();
                        __syncwarp();
                        if (lane == 0) ptx::mbar_arrive(&ctrl->p_full[grp][h]);
                        ++h;
                    }
                    if (!ok) break;
                    tmem_ld_wait32(ra);
                    if (halves == 1 && lane == 0) ptx::mbar_arrive(&ctrl->p_full[grp][1]);
                    l_run += sum;
                } else {
                    if (!take_turn()) { ok = false; break; }
                    pass_turn();
                    if (lane == 0) { ptx::mbar_arrive(&ctrl->p_full[grp][0]); ptx::mbar_arrive(&ctrl->p_full[grp][1]); }
                }
                any_tile |= on;
            }
            if (!ok) break;
            // ---- end of this CTA's part of the unit
            const bool whole = sg.t_first == 0 && sg.t_last == sg.u.tiles;
            const size_t at = ((size_t)sg.u.layer * p.c.R + sg.u.row0 + tok) * p.c.Hq + kvh * p.c.G + hg;
            __nv_bfloat16* const orow = p.c.out + at * D;
            const int slot = sg.t_first > 0 ? 0 : 1;                 // a unit that began before this CTA's range uses slot 0
            float* const rec = p.c.partial + (((size_t)blockIdx.x * 2 + slot) * 2 + grp) * kRowW * kRows + row;
            left -= sg.t_last - sg.t_first;
            if (left > 0) next_segment(sg, p, ctrl, left);           // (while the last P V is running)
            if (!ptx::warp_wait(ctrl, &ctrl->o_full[grp], o_par, 70)) { ok = false; break; }
            o_par ^= 1;
            ptx::tc_fence_after();
            if (warp_has_rows) {
                // (a sum that is no number, or 0 where every score is -inf, makes the row NaN, as in the merge and for single tokens)
                const float inv = 1.f / l_run;
                // An accumulator that no P V wrote may hold anything, and a part in which the row saw nothing has no weight: neither is read.
                const bool nothing = !any_tile || (!whole && off == -INFINITY);
#pragma unroll 1
                for (int c = 0; c < D; c += 32) {
                    uint32_t r[32];
                    ptx::tmem_ld_32x32b_x32(o_addr + (uint32_t)c, r);
                    tmem_ld_wait32(r);
                    if (nothing) {
#pragma unroll
                        for (int j = 0; j < 32; ++j) r[j] = 0u;
                    }
                    if (!whole) {
#pragma unroll
                        for (int j = 0; j < 32; ++j) rec[(size_t)(c + j) * kRows] = __uint_as_float(r[j]);
                    } else if (row_ok) {
                        store32(orow + c, r, inv, p.wide_out != 0);
                        store32(orow + c + 16, r + 16, inv, p.wide_out != 0);
                    }
                }
                if (!whole) {
                    rec[(size_t)D * kRows] = any_tile ? off : -INFINITY;
                    rec[(size_t)(D + 1) * kRows] = l_run;
                } else if (p.c.lse_out && row_ok) {
                    p.c.lse_out[at] = off * kAttnLn2 + logf(l_run);
                }
            }
            // (the stream's next P V waits for a P that its own warps write after this)
            ptx::tc_fence_before();
        }
    }

    ptx::tc_fence_before();
    __syncthreads();
    if (warp == 1) {
        ptx::tc_fence_after();
        ptx::tmem_dealloc(tmem_base, kTmemCols);
    }
}

// The units that the partition cut: one block per (inner boundary, stream).
template <int D>
__global__ void __launch_bounds__(kMergeThreads) attn_prompt_merge_kernel(const __grid_constant__ PromptParams p) {
    const int grp = blockIdx.y;
    ptx::grid_dep_wait();
    ptx::grid_dep_launch();
    merge_boundary<D, kMergeSlotsPrompt>(
        p.c.begins, p.n_cta, p.c.out, p.c.lse_out, p.c.status, p.c.wait_limit, 0,
        [&](int row, const GroupBegin& u, size_t& place, size_t& lse_place) {
            const Unit c = p.firsts[blockIdx.x + 1];                 // (the boundary's unit)
            const int it = row / p.gs, hl = row - it * p.gs, kvh = u.g / p.shares, hg = (u.g - kvh * p.shares) * p.gs + hl, tok = c.tok + grp * p.nt + it;
            place = lse_place = ((size_t)u.layer * p.c.R + c.row0 + tok) * p.c.Hq + kvh * p.c.G + hg;
            return it < p.nt && tok < c.n && hg < p.c.G;
        },
        [&](int cta, int slot) { return p.c.partial + (((size_t)cta * 2 + slot) * 2 + grp) * (D + 4) * kRows; });
}

// Tokens of a row tile, and query heads: a group's heads, or (more than 128) an even share of them.
void row_tile(int G, int* gs, int* shares, int* nt) {
    *shares = (G + kRows - 1) / kRows;
    *gs = (G + *shares - 1) / *shares;
    *nt = kRows / *gs;
}
}  // namespace

size_t mirror_attn_prompt_plan_bytes(const mirror_ctx* ctx) {
    return align_up((size_t)ctx->num_sms * sizeof(Unit), 256);
}

mirror_status mirror_attn_prompt_launch(mirror_ctx* ctx, const mirror_kv* kv, const CausalParams& cp, void* plan, cudaStream_t stream) {
    const int D = ctx->desc.head_dim;
    PromptParams p;
    p.c = cp;
    row_tile(cp.G, &p.gs, &p.shares, &p.nt);
    p.n_hs = cp.Hkv * p.shares;
    p.n_cta = ctx->num_sms;
    p.firsts = (Unit*)plan;
    p.wide_out = ((uintptr_t)cp.out & 31) == 0;
    // No unit is cut where even the longest that the page table allows is over before a cut would pay (and the CTAs' lists hold them all).
    const int64_t pairs = cp.R / (2 * p.nt) + cp.B, most_tiles = (causal_most_slots(cp, 2 * p.nt) + kTileSlots - 1) / kTileSlots;
    p.never_cut = most_tiles <= kCutTiles && pairs <= kMaxSorted && (pairs * cp.L * p.n_hs + ctx->num_sms - 1) / ctx->num_sms <= kMaxList;
    if (p.n_cta > kThreads || (size_t)p.n_cta * sizeof(GroupBegin) > kWsNotesBytes) return MIRROR_ERR_SHAPE;
    if ((int64_t)cp.L * cp.R > 0x7fffffff) return MIRROR_ERR_SHAPE;
    Maps tm;
    mirror_status st = mirror_attn_pool_tmap(ctx, kv, kv->k_pool, &tm.k);
    if (st == MIRROR_OK) st = mirror_attn_pool_tmap(ctx, kv, kv->v_pool, &tm.v);
    if (st != MIRROR_OK) return st;
    {
        // Q as (64 columns, heads, rows of all layers, D/64 halves): one box is one half of a row tile
        const uint64_t row = (uint64_t)D * 2, rows = (uint64_t)cp.L * cp.R;
        const uint64_t dims[5] = {64, (uint64_t)cp.Hq, rows, row / 128, 1};
        const uint64_t strides[4] = {row, cp.Hq * row, 128, rows * cp.Hq * row};
        const uint32_t box[5] = {64, (uint32_t)p.gs, (uint32_t)p.nt, 1, 1};
        st = mirror_make_tmap(ctx, &tm.q, cp.q, 5, dims, strides, box);
        if (st != MIRROR_OK) return st;
    }
    auto launch = [&](auto cfg, auto kern, auto merge) -> mirror_status {
        using C = decltype(cfg);
        const size_t fixed = 2 * (size_t)C::kQBytes + kCtrlBytes;
        const int stages = std::min((int)((kSmemLimit - fixed) / C::kStageBytes), kMaxStages);
        MIRROR_CUDA_OK(mirror_allow_smem(ctx, kRowsPrompt + (D == 128), kern, (int)kSmemLimit));
        MIRROR_CUDA_OK(mirror_launch_pdl(kern, dim3((unsigned)p.n_cta), dim3(kThreads), fixed + (size_t)stages * C::kStageBytes, stream, tm, p, stages));
        ctx->launches += 1;
        if (p.never_cut) return MIRROR_OK;
        constexpr int kSmem = merge_smem(kMergeSlotsPrompt);
        MIRROR_CUDA_OK(mirror_allow_smem(ctx, kRowsPromptMerge + (D == 128), merge, kSmem));
        MIRROR_CUDA_OK(mirror_launch_pdl(merge, dim3((unsigned)(p.n_cta - 1), 2), dim3(kMergeThreads), kSmem, stream, p));
        ctx->launches += 1;
        return MIRROR_OK;
    };
    st = D == 128 ? launch(Cfg<128>{}, attn_prompt_kernel<128>, attn_prompt_merge_kernel<128>) : launch(Cfg<64>{}, attn_prompt_kernel<64>, attn_prompt_merge_kernel<64>);
    if (st != MIRROR_OK) return st;
    MIRROR_CUDA_OK(cudaGetLastError());
    return MIRROR_OK;
}
