// One token per row of logits under temperature, Top-k, Top-p and Min-p, from a given uniform (mirror_sample).
//
// With z = (logit - max) / T the weight of an id is exp(z).  Each filter keeps a front of the ranks (logit descending, id ascending), so
// the kept set is the shortest of three fronts, and no sort of the row is needed: only where the front ends has to be found.  What
// decides are sums of weights, and a sum that is off by 10^-7 moves the end of a Top-p front by an id in one row of a hundred (an id's
// share is 10^-5 where the row is open).  Weights are therefore 64-bit integers, round(exp(z) 2^S) with S = 62 - ceil(log2 V) (at most 51), from a
// double-precision exponential: their sums are exact, and the same in whatever order threads and CTAs take them.
//
// A cluster of CTAs has one row, each a contiguous part of it, each warp a contiguous part of that, so that sums in the order of the ids
// are sums over warps.  With few rows a part is kept in shared memory.  With many it is read again from L2 by every pass: what takes
// the time then is the steps that one CTA, or one thread, takes for its row while the others wait, so four small CTAs an SM, each with
// more of a row, get more rows through than two large ones (520 rows x 128256 ids: 435 us against 541 when this was changed).
//   1  load, maximum over the cluster (the logits leave HBM once)
//   2  (rows of up to kList ids go to 4 as they are, Top-k of one asks for the maximum alone)
//      Top-k of up to kQuickK: a histogram of the largest logits of groups of 16 (or of every four, where groups are few) says down to which
//      logit at least k ids lie; Min-p says so by itself.  Top-p of the whole row: a histogram of z in 2048 bins of 1/64, how many ids each holds and where in the bin they lie on
//      average, packed in one word, which gives a bin's mass to 10^-3
//   3  the leading CTA adds the histograms up and reads off the bin in which each filter's front ends, Top-p's by estimate
//   4  if at most kList ids lie ahead of a logit that surely lies behind the end of the front, they go to the leader, which ranks them and
//      does the rest, while the others fill the distribution's rows.  Top-p's exact total is taken in the same pass
//   4' otherwise only the bin in which the front ends goes to the leader; what lies ahead of it is counted and summed by all.  (A bin
//      of more than kList ids, many equal logits above all, is bisected by key, with exact counts and masses of each half.)
//   5  the drawn token, by the warps' masses, and the filtered distribution
// What bounds it: where Top-p or a draw takes the whole row, instructions (147 an id, a thread each, over all passes) that leave at 42% of the
// issue slots, and barriers, a third of the stalls: CTAs of a cluster wait for the leading one, and one row's steps hide behind three others' at
// most.  The double-precision pipe is busy for 9% of the time only.  Where Top-k goes ahead, the leader's ranking; for a row alone the cluster's
// barriers and code that runs once.  Both instances have 64 registers a thread and spill (900 and 540 bytes of loads in all of the code).
// Measured on a B200: one row of 152064 ids under all three filters 15 us (0.1 us of bytes); 64 rows x 128256 under Top-p 0.9,
// probabilities written, 97 to 101 us; 520 rows x 128256 under Top-k 1000 and Top-p 0.98, logits written, 180 us (3.0 TB/s).
#include <cooperative_groups.h>
#include <math.h>

#include <type_traits>
#include <utility>

#include "mirror_internal.h"

namespace cg = cooperative_groups;

namespace {

using u64 = unsigned long long;

constexpr int kMaxWarps = 16;                 // 512 threads a CTA, or 256
constexpr int kBins = 2048;
constexpr float kBinsPerNat = 64.f;
constexpr int kList = 2048;                   // candidates that the leader ranks
constexpr int kShort = 256;                   // so few that each is compared with each
constexpr int kDeep = 48;                     // ids of a bin, above which pairs are sorted
constexpr int kMaxCluster = 16;
constexpr int kGroup = 4;                     // a group: this many of a thread's loads, 16 ids
constexpr int kTable = 64;
constexpr int kQuickK = 1400;                 // (the largest of every four: hardly more than k candidates then)
constexpr int kMaxPart = 40960;               // ids of a CTA
static_assert(kMaxPart / (4 * kGroup) <= 2 * kList && kMaxPart % (1024 * kGroup) == 0, "a part's groups have their place");
static_assert(kBins == kList, "a thread has as many bins as candidates");

struct SampleParams {
    int V, part;                           // part: ids of a CTA, a multiple of 128 per warp
    int shift;                                // S
    int id_shift;                             // ids >> id_shift are less than kList
    int off_bits, off_shift;                  // of a histogram word: see pack_off
    int vec_in, vec_probs, vec_logits;        // rows begin on 16-byte boundaries
    float temperature;                        // of the ctx
    long long ld;
    const float* logits;
    const float* temperatures;
    const int32_t* top_k;
    const float* top_p;
    const float* min_p;
    const float* u;
    int32_t* token;
    float* logprob;
    int32_t* n_kept;
    float* probs;
    float* logits_out;
    double two_s, two_ms;                     // 2^S, 2^-S
    double table[kTable];                     // 2^(j / 64)
};

struct Sums {
    u64 n, m, o, t;
};
struct Drawn {
    u64 w;
    uint32_t id, pad;
};

// What the CTAs of a cluster tell one another, and what a CTA's warps share.
struct alignas(16) Shared {
    float max[kMaxCluster];
    u64 sum[2][kMaxCluster][4];               // sums of the CTAs, for steps in turns
    u64 warp_sum[kMaxWarps][4];
    u64 warp_mass[kMaxWarps];                    // kept mass of the warps' parts
    u64 cut_key;                              // composite key of the last kept id
    u64 kept, kept_mass;                      // ids of its front, their mass
    u64 base;
    uint32_t key_first, key_last;             // of the list that is sorted: logits
    int last_bin, list_at;                    // written by the leader
    int n_list, n_all;                        // ids up to last_bin, and in all bins
    int bin_k, bin_p;                         // ... the bins in which Top-k and (estimated) Top-p end
    int bucket;
    float row_mass;
    alignas(16) double table[kTable];         // 2^(j / 64)
    double shares[kTable];                    // the same over the kept mass
    union alignas(16) {
        uint32_t hist[kBins];                 // counts and offsets; the leader's: then where each bin's candidates go
        Drawn drawn[kBins / 4];               // (the candidates that the draw has to look at one by one)
    };
    u64 list[kList];                          // composite keys: ~order key, id; then the masses of buckets of ids
    union {
        u64 ranked[kList];                    // the same in the order of the ranks
        float tops[2 * kList];                // (before there is a list) the largest logit of every group
    };
};
static_assert(sizeof(Shared) % 16 == 0, "the logits behind it are read 16 bytes at a time");

__device__ __forceinline__ float unkey(uint32_t k) { return __uint_as_float((k & 0x80000000u) ? k & 0x7fffffffu : ~k); }
__device__ __forceinline__ float logit_of(u64 key) { return unkey(~(uint32_t)(key >> 32)); }

// round(2^S exp((l - max) / T)): y = (l - max) log2(e) / T = n / 64 + f with |f| <= 1/128; 2^(n / 64) from a table, 2^f by its Taylor series to
// f^4 (the next term is below 4e-14), or to f^3 (4e-11) where the result is rounded to fp32.  (Against a table of sixteenths and f^6 the
// table's bank conflicts cost less than the operations, of which double precision has 64 a cycle and SM.)
struct Weigh {
    double max, c;                            // c: log2(e) / T, as far as weights can tell (the next number below the maximum at 2^-900)
    float lo, hi;                             // l is taken between them: 2^-900 is nothing, and a maximum of +inf counts as a number (c = 0)
    int shift;
    const double* table;
    __device__ __forceinline__ double y_of(float l) const { return ((double)fminf(fmaxf(l, lo), hi) - max) * c; }
    template <int kDegree>
    __device__ __forceinline__ double exp2_scaled(double y, int s, const double* of) const {      // of[0] 2^(y + s)
        const double magic = 105553116266496.0;                  // 1.5 * 2^46: the sum's low bits are the nearest 64th
        const double t = y + magic;
        const int n = __double2loint(t);
        const double f = y - (t - magic);
        double r = 5.55041086648215762e-02;                        // ln(2)^k / k!, k = 4 or 3 .. 0
        if (kDegree == 4) r = fma(9.61812910762847688e-03, f, r);
        r = fma(r, f, 2.40226506959100694e-01);
        r = fma(r, f, 6.93147180559945286e-01);
        r = fma(r, f, 1.0);
        r *= of[n & (kTable - 1)];
        return __hiloint2double(__double2hiint(r) + (((n >> 6) + s) << 20), __double2loint(r));
    }
    // (of an id that may be kept)
    __device__ __forceinline__ double unrounded(float l) const { return exp2_scaled<4>(y_of(l), shift, table); }
    __device__ __forceinline__ u64 operator()(float l) const {
        return (u64)__double_as_longlong(unrounded(l) + 4503599627370496.0) & 0xfffffffffffffull;         // + 2^52: the low bits are the integer
    }
    __device__ __forceinline__ double share(float l, const double* shares) const { return exp2_scaled<3>(y_of(l), 0, shares); }
};

__device__ __forceinline__ u64 warp_sum64(u64 v) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}
__device__ __forceinline__ u64 warp_incl64(u64 v) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const u64 t = __shfl_up_sync(0xffffffffu, v, o);
        if (lane >= o) v += t;
    }
    return v;
}

// A thread's w[], inclusive over the block: what lies before it, and all.
template <int kThreads, int kPer>
__device__ __forceinline__ u64 block_scan(Shared& s, const u64 (&w)[kPer], u64& before) {
    constexpr int kWarps = kThreads / 32;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    u64 mine = 0;
#pragma unroll
    for (int j = 0; j < kPer; ++j) mine += w[j];
    const u64 in = warp_incl64(mine);
    __syncthreads();
    if (lane == 31) s.warp_sum[warp][0] = in;
    __syncthreads();
    u64 all = lane < kWarps ? s.warp_sum[lane][0] : 0ull;
    all = warp_incl64(all);
    before = in - mine + (warp ? __shfl_sync(0xffffffffu, all, warp - 1) : 0ull);
    return __shfl_sync(0xffffffffu, all, kWarps - 1);
}

// list[0 .. n) in ascending order, whatever it holds: log2(n)^2 / 2 rounds of compared pairs.
template <int kThreads>
__device__ __noinline__ void sort_pairs(Shared& s, int n) {
    const int tid = threadIdx.x;
    int N = 2;
    while (N < n) N <<= 1;
    for (int i = n + tid; i < N; i += kThreads) s.list[i] = ~0ull;
    __syncthreads();
    for (int k = 2; k <= N; k <<= 1)
        for (int d = k >> 1; d > 0; d >>= 1) {
            for (int i = tid; i < N / 2; i += kThreads) {
                const int a = 2 * i - (i & (d - 1));
                const u64 x = s.list[a], y = s.list[a + d];
                if ((x > y) == ((a & k) == 0)) { s.list[a] = y; s.list[a + d] = x; }
            }
            __syncthreads();
        }
}
// The same: sorted into bins over the logits' range, and within a bin by comparing all with all.  (Many equal logits, or one far away from
// the others, make bins so deep that pairs are sooner.)
template <int kThreads, int kPer>
__device__ __noinline__ void sort_list(Shared& s, int n) {
    constexpr int kBinsPer = kBins / kThreads;
    const int tid = threadIdx.x, lane = tid & 31;
    __syncthreads();
    for (int i = tid; i < kBins; i += kThreads) s.hist[i] = 0;
    if (tid == 0) { s.key_first = ~0u; s.key_last = 0; }
    u64 key[kPer];
    uint32_t k0 = ~0u, k1 = 0;
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
        key[j] = tid + j * kThreads < n ? s.list[tid + j * kThreads] : ~0ull;
        if (tid + j * kThreads < n) { k0 = min(k0, (uint32_t)(key[j] >> 32)); k1 = max(k1, (uint32_t)(key[j] >> 32)); }
    }
    __syncthreads();
    k0 = __reduce_min_sync(0xffffffffu, k0);
    k1 = __reduce_max_sync(0xffffffffu, k1);
    if (lane == 0) { atomicMin(&s.key_first, k0); atomicMax(&s.key_last, k1); }
    __syncthreads();
    const float hi = logit_of((u64)s.key_first << 32), span = hi - logit_of((u64)s.key_last << 32);
    const float scale = span > 0.f && span < INFINITY ? (float)(kBins - 1) / span : 0.f;
    auto place = [&](u64 k) { return (int)fminf(fmaxf((hi - logit_of(k)) * scale, 0.f), (float)(kBins - 1)); };
#pragma unroll
    for (int j = 0; j < kPer; ++j)
        if (tid + j * kThreads < n) atomicAdd(&s.hist[place(key[j])], 1u);
    __syncthreads();
    {
        u64 cnt[kBinsPer], before;
        u64 most = 0;
#pragma unroll
        for (int j = 0; j < kBinsPer; ++j) {
            cnt[j] = s.hist[tid * kBinsPer + j];
            most = max(most, cnt[j]);
        }
        if (__syncthreads_or(most > (u64)kDeep)) {
            sort_pairs<kThreads>(s, n);
            return;
        }
        block_scan<kThreads>(s, cnt, before);
#pragma unroll
        for (int j = 0; j < kBinsPer; ++j) {
            s.hist[tid * kBinsPer + j] = (uint32_t)before;
            before += cnt[j];
        }
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kPer; ++j)
        if (tid + j * kThreads < n) s.ranked[atomicAdd(&s.hist[place(key[j])], 1u)] = key[j];
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
        if (tid + j * kThreads >= n) break;
        const int b = place(key[j]), lo = b ? (int)s.hist[b - 1] : 0, end = (int)s.hist[b];
        int ahead = 0;
        for (int q = lo; q < end; ++q) ahead += s.ranked[q] < key[j];
        s.list[lo + ahead] = key[j];
    }
    __syncthreads();
}

// The same for up to kShort of them: all with all.
__device__ __forceinline__ void sort_short(Shared& s, int n) {
    const int tid = threadIdx.x;
    __syncthreads();
    const u64 key = tid < n ? s.list[tid] : ~0ull;
    int ahead = 0;
    if (tid < n)
#pragma unroll 4
        for (int q = 0; q < n; ++q) ahead += s.list[q] < key;
    __syncthreads();
    if (tid < n) s.list[ahead] = key;
    __syncthreads();
}

template <bool kResident, int kThreads>
__global__ void __launch_bounds__(kThreads, 1024 / kThreads) sample_kernel(const __grid_constant__ SampleParams p) {
    constexpr int kWarps = kThreads / 32, kPer = kList / kThreads;
    extern __shared__ __align__(16) uint8_t smem_raw[];
    Shared& s = *reinterpret_cast<Shared*>(smem_raw);
    float* const z = reinterpret_cast<float*>(smem_raw + sizeof(Shared));         // (resident)
    cg::cluster_group cluster = cg::this_cluster();
    const int C = (int)cluster.num_blocks(), rank = (int)cluster.block_rank(), row = blockIdx.x / C;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int first = rank * p.part;                             // the part's first id
    const int n_mine = max(0, min(p.part, p.V - first));
    const int per_warp = p.part / kWarps, w0 = warp * per_warp, w1 = min(w0 + per_warp, (n_mine + 3) & ~3);
    Shared* const lead = cluster.map_shared_rank(&s, 0);
    auto started = cluster.barrier_arrive();

    ptx::grid_dep_wait();
    ptx::grid_dep_launch();
    // ---- 1: load, maximum.  (What cannot be kept, NaN and the part's end, becomes -inf.)
    const float* const in = p.logits + (long long)row * p.ld + first;
    float mx = -INFINITY;
    auto numbers = [](float4 v) { return make_float4(v.x == v.x ? v.x : -INFINITY, v.y == v.y ? v.y : -INFINITY, v.z == v.z ? v.z : -INFINITY, v.w == v.w ? v.w : -INFINITY); };
    auto fetch = [&](int i) -> float4 {                          // four ids' logits from memory
        float v[4];
        if (p.vec_in && i + 4 <= n_mine) {
            *reinterpret_cast<float4*>(v) = kResident ? __ldcs(reinterpret_cast<const float4*>(in + i)) : *reinterpret_cast<const float4*>(in + i);
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] = i + j < n_mine ? in[i + j] : -INFINITY;
        }
        return numbers(make_float4(v[0], v[1], v[2], v[3]));
    };
    const int n_groups = (per_warp + kGroup * 128 - 1) / (kGroup * 128);          // of a thread: kGroup of its loads each
    float* const tops = s.tops + warp * n_groups * 32 + lane;
    auto take_group = [&](int g, const float4 (&v)[kGroup]) {
        float top = -INFINITY;
#pragma unroll
        for (int j = 0; j < kGroup; ++j) {
            const int i = w0 + (g * kGroup + j) * 128 + lane * 4;
            if (kResident && i < w1) *reinterpret_cast<float4*>(z + i) = v[j];
            top = fmaxf(fmaxf(top, fmaxf(v[j].x, v[j].y)), fmaxf(v[j].z, v[j].w));
        }
        tops[g * 32] = top;
        mx = fmaxf(mx, top);
    };
    int g0 = 0;
    if (p.vec_in) {                                              // (groups within the part: two on the way at once)
        const int n_whole = max(0, min(w1, n_mine & ~3) - w0) / (kGroup * 128);
        for (; g0 + 2 <= n_whole; g0 += 2) {
            float4 v[2][kGroup];
#pragma unroll
            for (int j = 0; j < 2 * kGroup; ++j) {
                const float4* const at = reinterpret_cast<const float4*>(in + w0 + (g0 * kGroup + j) * 128 + lane * 4);
                v[j / kGroup][j % kGroup] = kResident ? __ldcs(at) : *at;
            }
#pragma unroll
            for (int j = 0; j < 2 * kGroup; ++j) v[j / kGroup][j % kGroup] = numbers(v[j / kGroup][j % kGroup]);
            take_group(g0, v[0]);
            take_group(g0 + 1, v[1]);
        }
    }
    for (; g0 < n_groups; ++g0) {
        float4 v[kGroup];
#pragma unroll
        for (int j = 0; j < kGroup; ++j) {
            const int i = w0 + (g0 * kGroup + j) * 128 + lane * 4;
            v[j] = i < w1 ? fetch(i) : make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY);
        }
        take_group(g0, v);
    }
    auto load = [&](int i) -> float4 { return kResident ? *reinterpret_cast<const float4*>(z + i) : fetch(i); };
    for (int i = tid; i < kBins; i += kThreads) s.hist[i] = 0;
    if (tid < kTable) s.table[tid] = p.table[tid];
#pragma unroll
    for (int o = 16; o; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
    if (lane == 0) s.warp_sum[warp][0] = __float_as_uint(mx);
    __syncthreads();
    // (every CTA of the cluster has started: its shared memory may be written to.  One without ids is here long before the others.)
    cluster.barrier_wait(std::move(started));
    if (tid < kWarps) {
        mx = __uint_as_float((uint32_t)s.warp_sum[tid][0]);
#pragma unroll
        for (int o = kWarps / 2; o; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync((1u << kWarps) - 1u, mx, o));
        if (tid == 0)
            for (int c = 0; c < C; ++c) cluster.map_shared_rank(&s, c)->max[rank] = mx;
    }
    cluster.sync();
    mx = -INFINITY;
    for (int c = 0; c < C; ++c) mx = fmaxf(mx, s.max[c]);

    // ---- the row's settings
    float T = p.temperatures ? p.temperatures[row] : p.temperature;
    const bool first_only = !(T > 0.f);
    if (first_only) T = 1.f;
    const double min_p = p.min_p && !first_only ? (double)p.min_p[row] : 0.0;
    const bool by_m = min_p > 0.0 && min_p <= 1.0;
    int k = p.top_k ? p.top_k[row] : 0;
    if (first_only || min_p > 1.0) k = 1;                        // (no id has more than the largest probability: the first alone, of equals, too)
    const bool by_k = k > 0 && k < p.V;
    const double top_p = p.top_p && !first_only ? (double)p.top_p[row] : 1.0;
    const bool by_p = top_p < 1.0;
    const bool whole_total = by_p && !by_k;                      // Top-p of the whole row
    const bool max_inf = mx == INFINITY, none = mx == -INFINITY; // (none: nothing to keep)
    Weigh weigh;
    weigh.hi = fminf(fmaxf(mx, -3.4028235e38f), 3.4028235e38f);
    weigh.max = (double)weigh.hi;
    const double c = max_inf || none ? 0.0 : 1.4426950408889634074 / (double)T;
    const float below = nextafterf(weigh.hi, -INFINITY);
    weigh.c = fmin(c, below > -INFINITY ? 900.0 / (weigh.max - (double)below) : 1e300);
    weigh.lo = fmaxf(fminf((float)fmax(weigh.max - 900.0 / weigh.c, -3.4e38), below), -3.4028235e38f);
    weigh.shift = p.shift;
    weigh.table = s.table;
    const double ln2T = 0.69314718055994530942 * (double)p.temperature;
    // ids that may be kept: neither NaN nor -inf, and where the maximum is +inf only those
    const float least = max_inf ? INFINITY : -3.4028235e38f;
    auto may = [&](float l) { return l >= least; };
    const double min_w = min_p * p.two_s;             // (not rounded to steps: what weighs less than one may be kept, too)
    // composite key of an id: smaller is ahead
    auto key_of = [&](float l, int id) { return ((u64)~mirror_order_key(l + 0.f) << 32) | (uint32_t)id; };      // (-0 and 0 are equal)
    const float inv_T = 1.f / T;
    auto bin_of = [&](float l, float& at) {
        at = max_inf || l == mx ? 0.f : fminf((mx - l) * inv_T * kBinsPerNat, (float)(kBins - 1));        // (what is no number: the last bin)
        return (int)at;
    };
    int turn = 0;
    // a word of every CTA's for every CTA, by way of s.warp_sum
    auto exchange = [&]() -> Sums {
        __syncthreads();
        if (tid < 4 * C) {
            const int c = tid >> 2, q = tid & 3;
            u64 t = 0;
            for (int w = 0; w < kWarps; ++w) t += s.warp_sum[w][q];
            cluster.map_shared_rank(&s, c)->sum[turn][rank][q] = t;
        }
        cluster.sync();
        Sums a = {0, 0, 0, 0};
        for (int c = 0; c < C; ++c) { a.n += s.sum[turn][c][0]; a.m += s.sum[turn][c][1]; a.o += s.sum[turn][c][2]; a.t += s.sum[turn][c][3]; }
        turn ^= 1;                                               // (read before the other turn's barrier: rewritten after it)
        return a;
    };
    // what f(l, i, sums) adds for the ids of the warp's part
    auto warp_part = [&](auto f) -> Sums {
        Sums a = {0, 0, 0, 0};
        for (int i = w0 + lane * 4; i < w1; i += 128) {
            const float4 v = load(i);
            f(v.x, i, a); f(v.y, i + 1, a); f(v.z, i + 2, a); f(v.w, i + 3, a);
        }
        return {warp_sum64(a.n), warp_sum64(a.m), warp_sum64(a.o), warp_sum64(a.t)};
    };
    // ... summed over the cluster; every thread gets the sums
    auto all_sums = [&](auto f) -> Sums {
        const Sums a = warp_part(f);
        __syncthreads();
        if (lane == 0) { s.warp_sum[warp][0] = a.n; s.warp_sum[warp][1] = a.m; s.warp_sum[warp][2] = a.o; s.warp_sum[warp][3] = a.t; }
        return exchange();
    };

    u64 cut = ~0ull;                                             // composite key of the last id of the front
    int ahead_bin = -1;                                          // >= 0: the warps' masses ahead of that bin are in s.warp_mass
    bool known = false;                                          // all of the front's are, and how many ids it has
    u64 n_known = 0, m_known = 0;
    u64 Z = 0;
    if (!none && (by_k || by_p || by_m)) {
        const float parts = (float)(1 << p.off_bits);
        // ---- 3: the leader's reading of the histograms.  `masses`: the words hold offsets, too.
        auto read_bins = [&](bool masses) {
            cluster.sync();
            if (rank == 0) {
                uint32_t cnt[kPer] = {}, off[kPer] = {};
                const uint32_t low = (1u << p.off_shift) - 1u;
#pragma unroll 4
                for (int c = 0; c < C; ++c) {
#pragma unroll
                    for (int j = 0; j < kPer; j += 4) {
                        const uint4 h = *reinterpret_cast<const uint4*>(&cluster.map_shared_rank(&s, c)->hist[tid * kPer + j]);
                        cnt[j] += h.x >> p.off_shift; cnt[j + 1] += h.y >> p.off_shift; cnt[j + 2] += h.z >> p.off_shift; cnt[j + 3] += h.w >> p.off_shift;
                        off[j] += h.x & low; off[j + 1] += h.y & low; off[j + 2] += h.z & low; off[j + 3] += h.w & low;
                    }
                }
                uint32_t n = 0;
                float m = 0.f, ms[kPer];
#pragma unroll
                for (int j = 0; j < kPer; ++j) {
                    // (the mean of exp(-x) over a 64th is exp(-mean) but for a relative 10^-4; the last bin is open: no mass)
                    const int b = tid * kPer + j;
                    const float mean = ((float)b + __fdividef((float)off[j] + 0.5f * (float)cnt[j], parts * fmaxf((float)cnt[j], 1.f))) * (1.f / kBinsPerNat);
                    ms[j] = b == kBins - 1 ? 0.f : (float)cnt[j] * __expf(-mean);
                    n += cnt[j];
                    m += ms[j];
                }
                // exclusive sums over the threads
                uint32_t n_in = n;
                float m_in = m;
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) {
                    const uint32_t a = __shfl_up_sync(0xffffffffu, n_in, o);
                    const float b = __shfl_up_sync(0xffffffffu, m_in, o);
                    if (lane >= o) { n_in += a; m_in += b; }
                }
                if (lane == 31) s.warp_sum[warp][0] = ((u64)n_in << 32) | __float_as_uint(m_in);
                if (tid == 0) s.last_bin = s.bin_k = s.bin_p = kBins - 1;
                __syncthreads();
                float m_all = 0.f;
                uint32_t n_before = n_in - n;
                float m_before = m_in - m;
#pragma unroll
                for (int w = 0; w < kWarps; ++w) {
                    const u64 t = s.warp_sum[w][0];
                    if (w < warp) { n_before += (uint32_t)(t >> 32); m_before += __uint_as_float((uint32_t)t); }
                    m_all += __uint_as_float((uint32_t)t);
                }
                if (tid == 0) s.row_mass = m_all;
                __syncthreads();
                // Top-k's bin, and about what its front weighs
                if (by_k) {
                    uint32_t nb = n_before;
                    float mb = m_before;
#pragma unroll
                    for (int j = 0; j < kPer; ++j) {
                        if (nb < (uint32_t)k && nb + cnt[j] >= (uint32_t)k) {
                            s.bin_k = tid * kPer + j;
                            s.row_mass = mb + ms[j] * (float)((uint32_t)k - nb) / (float)cnt[j];
                        }
                        nb += cnt[j];
                        mb += ms[j];
                    }
                    __syncthreads();
                }
                if (masses && by_p) {
                    const float about = (float)top_p * s.row_mass;
                    float mb = m_before;
                    int end = kBins - 1, end_p = kBins - 1;
#pragma unroll
                    for (int j = 0; j < kPer; ++j) {
                        const int b = tid * kPer + j;
                        mb += ms[j];
                        // the first bin at which Top-p is surely through, and where it ends by estimate
                        if (mb >= 1.01f * about) end = min(end, b);
                        if (mb >= about) end_p = min(end_p, b);
                    }
                    end = __reduce_min_sync(0xffffffffu, end);
                    end_p = __reduce_min_sync(0xffffffffu, end_p);
                    if (lane == 0) {
                        atomicMin(&s.last_bin, end);
                        atomicMin(&s.bin_p, end_p);
                    }
                    __syncthreads();
                }
                // how many ids that is
                uint32_t nb = n_before;
#pragma unroll
                for (int j = 0; j < kPer; ++j) {
                    nb += cnt[j];
                    if (tid * kPer + j == s.last_bin) s.n_list = (int)nb;
                }
                if (tid == kThreads - 1) s.n_all = (int)nb;
                // (Top-p behind Top-k is a share of all that Top-k leaves, so Top-k's end counts alone)
                if (tid == 0 && by_k) s.last_bin = s.bin_k;
                __syncthreads();
                if (tid < C) {
                    Shared* const o = cluster.map_shared_rank(&s, tid);
                    o->last_bin = s.last_bin;
                    o->bin_k = s.bin_k;
                    o->bin_p = s.bin_p;
                    o->n_list = s.n_list;
                    o->n_all = s.n_all;
                }
            }
            cluster.sync();
        };
        // a logit below all of the bins up to b, and one that Min-p surely leaves out
        const float slack = fabsf(weigh.hi) * 1e-6f;
        auto below_bin = [&](int b) { return b >= kBins - 1 || max_inf ? least : weigh.hi - (float)(b + 1) * T * (1.00002f / kBinsPerNat) - slack; };
        const float below_m = by_m && !max_inf ? weigh.hi + T * (logf((float)min_p) * 1.00002f - 1e-5f) - slack : least;
        // Candidates: into the CTA's own list (an atomic of another CTA's memory is a trip of a thousand cycles), and once the exchange has
        // told how many every CTA has, count(c) of them, one behind the other into the leader's.
        auto gather = [&](auto count) {
            if (rank != 0) {
                int at = 0;
                for (int c = 0; c < rank; ++c) at += count(c);
                const int n = count(rank);
                for (int i = tid; i < n; i += kThreads) lead->list[at + i] = s.list[i];
            }
            cluster.sync();
        };
        // ---- 4: the ids from `from` on to the leader, and (of_all) the mass of all.  How many they are:
        u64 total = 0;
        auto push = [&](float from, bool of_all) -> int {
            if (tid == 0) s.list_at = 0;
            __syncthreads();
            u64 m = 0;
            if (of_all)
                for (int i = w0 + lane * 4; i < w1; i += 128) {
                    const float4 v = load(i);
                    if (may(v.x)) m += weigh(v.x);
                    if (may(v.y)) m += weigh(v.y);
                    if (may(v.z)) m += weigh(v.z);
                    if (may(v.w)) m += weigh(v.w);
                }
            // groups that have such ids, in the place of their largest logits, then a lane to a group
            int* const groups = reinterpret_cast<int*>(tops - lane);
            int n_hit = 0;
            for (int g = 0; g < n_groups; ++g) {
                const bool hit = tops[g * 32] >= from;
                const uint32_t hits = __ballot_sync(0xffffffffu, hit);
                if (hit) groups[n_hit + __popc(hits & ((1u << lane) - 1u))] = w0 + g * (kGroup * 128) + lane * 4;
                n_hit += __popc(hits);
            }
            __syncwarp();
            int n = 0;
            for (int q = 0; q < n_hit; q += 32) {
                const int i0 = q + lane < n_hit ? groups[q + lane] : w1;
                float v[4 * kGroup];
#pragma unroll
                for (int j = 0; j < kGroup; ++j)
                    *reinterpret_cast<float4*>(v + 4 * j) = i0 + j * 128 < w1 ? load(i0 + j * 128) : make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY);
                int mine = 0;
#pragma unroll
                for (int j = 0; j < 4 * kGroup; ++j) mine += v[j] >= from;
                int in = mine;
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) {
                    const int t = __shfl_up_sync(0xffffffffu, in, o);
                    if (lane >= o) in += t;
                }
                int at = 0;
                if (lane == 31) at = atomicAdd(&s.list_at, in);
                at = __shfl_sync(0xffffffffu, at, 31) + in - mine;
                n += mine;
#pragma unroll
                for (int j = 0; j < 4 * kGroup; ++j)
                    if (v[j] >= from) {
                        if (at < kList) s.list[at] = key_of(v[j], first + i0 + j / 4 * 128 + j % 4);
                        ++at;
                    }
            }
            Sums a = {(u64)n, m, 0, 0};
            a.n = warp_sum64(a.n);
            a.m = warp_sum64(a.m);
            __syncthreads();
            if (lane == 0) { s.warp_sum[warp][0] = a.n; s.warp_sum[warp][1] = a.m; s.warp_sum[warp][2] = s.warp_sum[warp][3] = 0; }
            const int was = turn;
            a = exchange();
            total = a.m;
            if (a.n > (u64)kList) return kList + 1;
            gather([&](int c) { return (int)s.sum[was][c][0]; });
            return (int)a.n;
        };
        float from = least;
        int n_list = kList + 1;
        const bool all = p.V <= kList;                           // (then the list takes the row)
        const bool quick = all || (by_k ? k <= kQuickK : by_m && !by_p);
        // ---- 2: histograms.  A word counts in its upper bits and sums in its lower ones in which part of the bin the ids lie: neither half
        // outgrows its bits over a part's ids.
        if (quick) {
            if (by_k && k == 1) {
                from = mx;
            } else if (by_k && !all) {
                auto count = [&](float top) {
                    float at;
                    if (may(top)) atomicAdd(&s.hist[bin_of(top, at)], 1u << p.off_shift);
                };
                if ((int64_t)k * 8 * kGroup <= p.V) {            // (half of the groups hold k ids, and hardly more than 1.4 k where they lie anyhow)
                    for (int g = 0; g < n_groups; ++g) count(tops[g * 32]);
                } else {
                    for (int i = w0 + lane * 4; i < w1; i += 128) {
                        const float4 v = load(i);
                        count(fmaxf(fmaxf(v.x, v.y), fmaxf(v.z, v.w)));
                    }
                }
                read_bins(false);
                from = below_bin(s.last_bin);
            }
            if (!(by_k && by_p)) from = fmaxf(from, below_m);
            from = from >= least ? from : least;
            n_list = push(from, whole_total);
        }
        if (n_list > kList) {
            __syncthreads();
            for (int i = tid; i < kBins; i += kThreads) s.hist[i] = 0;
            __syncthreads();
            for (int i = w0 + lane * 4; i < w1; i += 128) {
                const float4 v4 = load(i);
                const float v[4] = {v4.x, v4.y, v4.z, v4.w};
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    if (!may(v[j])) continue;
                    float at;
                    const int bin = bin_of(v[j], at);
                    atomicAdd(&s.hist[bin], (1u << p.off_shift) + (uint32_t)((at - (float)bin) * parts));
                }
            }
            read_bins(true);
            if (!by_k && by_p && (by_m || s.n_list <= kList)) {  // (the others have been tried, or have no list that is short enough)
                from = fmaxf(below_bin(s.last_bin), below_m);
                from = from >= least ? from : least;
                n_list = push(from, whole_total);
            }
        }
        if (n_list <= kList) {
            // the distribution's rows: the others fill them while the leader ranks (nobody reads the logits any more)
            if (rank != 0 || C == 1) {
                auto fill = [&](float* out, float what, bool vec) {
                    const int workers = C == 1 ? 1 : C - 1, me = C == 1 ? 0 : rank - 1;
                    if (vec) {
                        float4* const o = reinterpret_cast<float4*>(out);
                        for (int i = me * kThreads + tid; i < p.V / 4; i += workers * kThreads) __stcs(o + i, make_float4(what, what, what, what));
                    } else {
                        for (int i = me * kThreads + tid; i < p.V; i += workers * kThreads) out[i] = what;
                    }
                };
                if (p.probs) fill(p.probs + (size_t)row * p.V, 0.f, p.vec_probs);
                if (p.logits_out) fill(p.logits_out + (size_t)row * p.V, -INFINITY, p.vec_logits);
            }
            if (rank != 0) {
                // (the rows are filled: the leader waits for those that are still there)
                if (p.probs || p.logits_out) cluster.barrier_arrive();
                return;
            }
            auto finish = [&](auto per) {
                constexpr int P = decltype(per)::value;          // ids of a thread
                if (P == 1) sort_short(s, n_list);
                else sort_list<kThreads, P>(s, n_list);
                int n_m = n_list;                                // of the ranks those that Min-p keeps
                if (by_m) {
                    n_m = 0;
#pragma unroll 1
                    for (int r = tid; r - tid < n_list; r += kThreads) n_m += __syncthreads_count(r < n_list && weigh.unrounded(logit_of(s.list[r])) >= min_w);
                }
                u64 key[P], w[P], sel[P], before;
#pragma unroll
                for (int j = 0; j < P; ++j) {
                    const int r = tid * P + j;
                    key[j] = r < n_list ? s.list[r] : ~0ull;
                    w[j] = r < n_list ? weigh(logit_of(key[j])) : 0ull;
                    sel[j] = by_k && r >= k ? 0ull : w[j];
                }
                const u64 part = block_scan<kThreads>(s, sel, before);
                const double want = top_p * (double)(whole_total ? total : part);
                int kept = 0;
                u64 kept_mass = 0;
#pragma unroll
                for (int j = 0; j < P; ++j) {
                    const int r = tid * P + j;
                    const bool stays = r < n_list && (r == 0 || ((!by_k || r < k) && (!by_p || (double)before < want) && r < n_m));
                    kept += stays;
                    if (stays) {
                        kept_mass += w[j];
                        if (P == 1) s.drawn[tid] = {w[j], (uint32_t)key[j], 0u};
                    }
                    before += sel[j];
                }
                kept = __reduce_add_sync(0xffffffffu, kept);
                kept_mass = warp_sum64(kept_mass);
                if (lane == 0) { s.warp_sum[warp][2] = (u64)kept; s.warp_sum[warp][3] = kept_mass; }
                if (P > 1) {
#pragma unroll
                    for (int j = 0; j < kPer; ++j) s.ranked[tid * kPer + j] = 0;     // (from here on: masses of buckets of ids)
                    if (tid == 0) s.list_at = 0;
                }
                __syncthreads();
                int n = 0;
                Z = 0;
#pragma unroll
                for (int q = 0; q < kWarps; ++q) { n += (int)s.warp_sum[q][2]; Z += s.warp_sum[q][3]; }
                const double t = fmax((double)p.u[row], 0.0) * (double)Z;
                const u64 target = t >= (double)Z ? Z - 1 : (u64)t;                 // the first id whose inclusive sum is above it
                // the draw: of few, each adds up those of the lower ids; of many the bucket of ids in which the sum over ids passes the target, then
                // the id within it
                auto draw = [&](const Drawn& d, u64 sum, int of) {
                    for (int q = 0; q < of; ++q)
                        if (s.drawn[q].id < d.id) sum += s.drawn[q].w;
                    if (sum <= target && sum + d.w > target) {
                        p.token[row] = (int32_t)d.id;
                        if (p.logprob) p.logprob[row] = (float)log((double)d.w / (double)Z);
                        if (p.n_kept) p.n_kept[row] = n;
                    }
                };
                if (P == 1) {
                    if (tid < n) draw({w[0], (uint32_t)key[0], 0u}, 0, n);
                } else {
#pragma unroll
                    for (int j = 0; j < P; ++j)
                        if (tid * P + j < n) atomicAdd(&s.ranked[(uint32_t)key[j] >> p.id_shift], w[j]);
                    __syncthreads();
                    u64 bucket[kPer];
#pragma unroll
                    for (int j = 0; j < kPer; ++j) bucket[j] = s.ranked[tid * kPer + j];
                    block_scan<kThreads>(s, bucket, before);
#pragma unroll
                    for (int j = 0; j < kPer; ++j) {
                        if (before <= target && before + bucket[j] > target) {
                            s.bucket = tid * kPer + j;
                            s.base = before;
                        }
                        before += bucket[j];
                    }
                    __syncthreads();
#pragma unroll
                    for (int j = 0; j < P; ++j)
                        if (tid * P + j < n && (int)((uint32_t)key[j] >> p.id_shift) == s.bucket) s.drawn[atomicAdd(&s.list_at, 1)] = {w[j], (uint32_t)key[j], 0u};
                    __syncthreads();
                    for (int q = tid; q < s.list_at; q += kThreads) draw(s.drawn[q], s.base, s.list_at);
                }
                if (!p.probs && !p.logits_out) return;
                cluster.sync();                                  // (the rows are filled)
                const double unit = (double)Z * p.two_ms, ln_z = log(unit);
                if (tid < kTable) s.shares[tid] = s.table[tid] / unit;
                __syncthreads();
#pragma unroll
                for (int j = 0; j < P; ++j) {
                    if (tid * P + j >= n) break;
                    const float l = logit_of(key[j]);
                    const size_t at = (size_t)row * p.V + (uint32_t)key[j];
                    if (p.probs) p.probs[at] = (float)weigh.share(l, s.shares);
                    if (p.logits_out) p.logits_out[at] = (float)((max_inf ? 0.0 : ((double)l - weigh.max) * c) * ln2T - ln_z * (double)p.temperature);
                }
            };
            if (n_list <= kShort) finish(std::integral_constant<int, 1>());
            else if (n_list <= kList / 2) finish(std::integral_constant<int, kPer / 2>());
            else if (n_list <= kList / 4 * 3) finish(std::integral_constant<int, kPer / 4 * 3>());
            else finish(std::integral_constant<int, kPer>());
            return;
        }
        {
            // ---- 4': the bin in which each filter's front ends, and where in it
            auto front = [&](u64 at) {                           // (count, mass) of the ids up to the composite key `at`
                return all_sums([&](float l, int i, Sums& a) {
                    if (may(l) && key_of(l, first + i) <= at) { ++a.n; a.m += weigh(l); }
                });
            };
            // the least order key that lies in bin b or ahead of it (no data takes part)
            auto edge = [&](int b) -> uint32_t {
                uint32_t lo = 0, hi = mirror_order_key(mx);
                while (lo < hi) {
                    const uint32_t mid = lo + ((hi - lo) >> 1);
                    float at;
                    if (bin_of(unkey(mid), at) <= b) hi = mid; else lo = mid + 1;
                }
                return lo;
            };
            // The smallest key whose front (count, mass, and the mass of all ids where that is asked for) fulfils `done`, which is monotone;
            // guessed to lie in bin `b`.
            auto end_of = [&](int b, bool of_all, auto done) -> u64 {
                u64 n0, m0, n_in, all = 0;
                u64 lo = 0, hi = ~0ull;                          // (what is known of the key where the guess is off again and again)
                bool far = false, early = false;
                int was = 0;
                for (int again = 0;; ++again) {
                    // what lies ahead of the bin, and the bin itself into the leader's list
                    if (tid == 0) s.list_at = 0;
                    __syncthreads();
                    const bool rest = of_all && again == 0;
                    uint32_t n_ahead = 0, n_bin = 0;
                    u64 m_ahead = 0, m_bin = 0, m_all = 0;
                    for (int i = w0 + lane * 4; i < w1; i += 128) {
                        const float4 v4 = load(i);
                        const float v[4] = {v4.x, v4.y, v4.z, v4.w};
                        int bin[4];
                        float at;
#pragma unroll
                        for (int j = 0; j < 4; ++j) bin[j] = may(v[j]) ? bin_of(v[j], at) : kBins;
                        const int least_bin = min(min(bin[0], bin[1]), min(bin[2], bin[3]));
                        if (least_bin > (rest ? kBins - 1 : b)) continue;
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const u64 any = weigh(v[j]), w = bin[j] < kBins ? any : 0ull;
                            m_all += w;
                            m_ahead += bin[j] < b ? w : 0ull;
                            n_ahead += bin[j] < b;
                            if (bin[j] == b) {
                                ++n_bin;
                                m_bin += w;
                                const int slot = atomicAdd(&s.list_at, 1);
                                if (slot < kList) s.list[slot] = key_of(v[j], first + i + j);
                            }
                        }
                    }
                    const Sums mine = {warp_sum64(((u64)n_bin << 32) | n_ahead), warp_sum64(m_ahead), warp_sum64(m_bin), warp_sum64(m_all)};
                    __syncthreads();
                    if (lane == 0) {
                        s.warp_sum[warp][0] = mine.n; s.warp_sum[warp][1] = mine.m; s.warp_sum[warp][2] = mine.o; s.warp_sum[warp][3] = mine.t;
                        s.warp_mass[warp] = mine.m;
                    }
                    was = turn;
                    const Sums a = exchange();
                    n0 = a.n & 0xffffffffull;
                    n_in = a.n >> 32;
                    m0 = a.m;
                    if (rest) all = a.t;
                    ahead_bin = b;
                    known = false;
                    early = n0 > 0 && done(n0, m0, all);
                    const bool late = b < kBins - 1 && !done(n0 + n_in, m0 + a.o, all);
                    far = (early || late) && again >= 3;
                    // (the bin's own keys, or all ahead of it, or all behind it)
                    if (far || n_in > (u64)kList) {
                        lo = early || b == 0 ? 0ull : (u64)~(edge(b - 1) - 1) << 32;
                        hi = late ? ~0ull : ((u64)~edge(b) << 32) | 0xffffffffull;
                    }
                    if (far || !(early || late)) break;
                    b += early ? -1 : 1;                         // it ends ahead of this bin, or behind it
                }
                if (far) ahead_bin = -1;
                if (far || n_in > (u64)kList) {
                    // the logit first, then the id; what lies ahead of `lo` is known, so few ids are weighed
                    u64 n_lo = early ? 0ull : n0, m_lo = early ? 0ull : m0;
                    while (lo < hi) {
                        const uint32_t l0 = (uint32_t)(lo >> 32), l1 = (uint32_t)(hi >> 32);
                        if (l0 == l1) hi = min(hi, ((u64)l0 << 32) | (uint32_t)(p.V - 1));
                        const u64 mid = l0 < l1 ? ((u64)(l0 + ((l1 - l0) >> 1)) << 32) | 0xffffffffull : lo + ((hi - lo) >> 1);
                        const Sums a = all_sums([&](float l, int i, Sums& a) {
                            if (!may(l)) return;
                            const u64 key = key_of(l, first + i);
                            if (key >= lo && key <= mid) { ++a.n; a.m += weigh(l); }
                        });
                        if (done(n_lo + a.n, m_lo + a.m, all)) {
                            hi = mid;
                        } else {
                            lo = mid + 1;
                            n_lo += a.n;
                            m_lo += a.m;
                        }
                    }
                    return lo;
                }
                gather([&](int c) { return (int)(s.sum[was][c][0] >> 32); });
                if (rank == 0) {
                    const int n = (int)n_in;
                    sort_list<kThreads, kPer>(s, n);
                    if (tid == 0) s.list_at = n - 1;
                    u64 w[kPer], before;
#pragma unroll
                    for (int j = 0; j < kPer; ++j) {
                        const int r = tid * kPer + j;
                        w[j] = r < n ? weigh(logit_of(s.list[r])) : 0ull;
                    }
                    block_scan<kThreads>(s, w, before);
                    u64 at = before + m0;
#pragma unroll
                    for (int j = 0; j < kPer; ++j) {
                        const int r = tid * kPer + j;
                        at += w[j];
                        if (r < n && done(n0 + r + 1, at, all)) { atomicMin(&s.list_at, r); break; }
                    }
                    __syncthreads();
                    if (tid < C) {
                        Shared* const o = cluster.map_shared_rank(&s, tid);
                        o->cut_key = s.list[s.list_at];
                        o->kept = n0 + s.list_at + 1;
                    }
                    // (what stays of the bin belongs to warps' parts, too)
                    at = before + m0;
#pragma unroll
                    for (int j = 0; j < kPer; ++j) {
                        const int r = tid * kPer + j;
                        if (r > s.list_at) break;
                        at += w[j];
                        if (r == s.list_at)
                            for (int c = 0; c < C; ++c) cluster.map_shared_rank(&s, c)->kept_mass = at;
                        const int id = (int)(uint32_t)s.list[r], of = id / p.part;
                        atomicAdd(&cluster.map_shared_rank(&s, of)->warp_mass[(id - of * p.part) / per_warp], w[j]);
                    }
                }
                known = true;
                cluster.sync();
                const u64 c = s.cut_key;
                n_known = s.kept;
                m_known = s.kept_mass;
                cluster.sync();                                  // (the next one may be written)
                return c;
            };
            total = 0;
            const bool cuts_k = by_k && k < s.n_all;             // (there may be fewer that may be kept)
            if (cuts_k) {
                cut = end_of(s.bin_k, false, [&](u64 n, u64, u64) { return n >= (u64)k; });
                if (by_p) total = known ? m_known : front(cut).m;
            }
            if (by_p) {
                const u64 c = end_of(s.bin_p, !cuts_k, [&](u64 n, u64 m, u64 all) { return n >= 1 && (double)m >= top_p * (double)(cuts_k ? total : all); });
                cut = min(cut, c);
            }
            if (by_m) {
                // the last logit of at least min_w, by its key (no data takes part)
                __syncthreads();
                if (warp == 0) {
                    uint32_t lo = 0, hi = mirror_order_key(mx);  // weight(hi) >= min_w
                    while (lo < hi) {
                        const uint32_t mid = lo + ((hi - lo) >> 1);
                        const float l = unkey(mid);
                        if (l > -INFINITY && weigh.unrounded(l) >= min_w) hi = mid; else lo = mid + 1;
                    }
                    if (lane == 0) s.base = ((u64)~hi << 32) | 0xffffffffull;
                }
                __syncthreads();
                if (s.base < cut) { cut = s.base; ahead_bin = -1; known = false; }
            }
        }
    }
    // ---- 5: the warps' kept masses, the draw, the distribution
    const float cut_l = cut == ~0ull ? least : fmaxf(logit_of(cut), least);
    const int cut_i = cut == ~0ull ? 0x7fffffff : (int)min((uint32_t)cut, 0x7fffffffu) - first;
    auto kept = [&](float l, int i) { return l > cut_l || (l == cut_l && i <= cut_i); };
    {
        // (ahead of the bin in which the front ends the masses are known)
        Sums mine = {rank == 0 && warp == 0 ? n_known : 0ull, 0, 0, 0};
        if (!known)
            mine = warp_part([&](float l, int i, Sums& a) {
                if (!kept(l, i)) return;
                ++a.n;
                float at;
                if (ahead_bin < 0 || bin_of(l, at) >= ahead_bin) a.m += weigh(l);
            });
        const u64 mass = mine.m + (known || ahead_bin >= 0 ? s.warp_mass[warp] : 0ull);
        __syncthreads();
        if (lane == 0) {
            s.warp_sum[warp][0] = mine.n; s.warp_sum[warp][1] = mass; s.warp_sum[warp][2] = s.warp_sum[warp][3] = 0;
            s.warp_mass[warp] = mass;
        }
        const int was = turn;
        const Sums all = exchange();
        Z = all.m;
        if (all.n == 0) {
            if (rank == 0 && tid == 0) {
                p.token[row] = -1;
                if (p.logprob) p.logprob[row] = -INFINITY;
                if (p.n_kept) p.n_kept[row] = 0;
            }
        } else {
            if (rank == 0 && tid == 0 && p.n_kept) p.n_kept[row] = (int32_t)all.n;
            const double t = fmax((double)p.u[row], 0.0) * (double)Z;
            const u64 target = t >= (double)Z ? Z - 1 : (u64)t;
            u64 before = 0;
            for (int c = 0; c < rank; ++c) before += s.sum[was][c][1];
            for (int w = 0; w < warp; ++w) before += s.warp_mass[w];
            if (before <= target && before + mass > target) {
                for (int i0 = w0; i0 < w1; i0 += 128) {          // (this warp's ids in order, four to a lane)
                    const int i = i0 + lane * 4;
                    u64 w[4] = {};
                    if (i < w1) {
                        const float4 v4 = load(i);
                        const float v[4] = {v4.x, v4.y, v4.z, v4.w};
#pragma unroll
                        for (int j = 0; j < 4; ++j)
                            if (kept(v[j], i + j)) w[j] = weigh(v[j]);
                    }
                    const u64 four = w[0] + w[1] + w[2] + w[3], in_ = before + warp_incl64(four);
                    const uint32_t over = __ballot_sync(0xffffffffu, in_ > target);
                    if (over) {
                        if (lane == __ffs(over) - 1) {
                            u64 at = in_ - four;
#pragma unroll
                            for (int j = 0; j < 4; ++j) {
                                if (at <= target && at + w[j] > target) {
                                    p.token[row] = first + i + j;
                                    if (p.logprob) p.logprob[row] = (float)log((double)w[j] / (double)Z);
                                }
                                at += w[j];
                            }
                        }
                        break;
                    }
                    before = __shfl_sync(0xffffffffu, in_, 31);
                }
            }
        }
    }
    if (p.probs || p.logits_out) {
        const double unit = (double)Z * p.two_ms, ln_z = log(unit);
        if (tid < kTable) s.shares[tid] = s.table[tid] / unit;   // (nothing kept: not read)
        __syncthreads();
        float* const probs = p.probs ? p.probs + (size_t)row * p.V + first : nullptr;
        float* const lg = p.logits_out ? p.logits_out + (size_t)row * p.V + first : nullptr;
        for (int i = w0 + lane * 4; i < w1; i += 128) {
            const float4 v4 = load(i);
            const float v[4] = {v4.x, v4.y, v4.z, v4.w};
            float a[4], b[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const bool in_front = kept(v[j], i + j);
                a[j] = in_front && probs ? (float)weigh.share(v[j], s.shares) : 0.f;
                b[j] = in_front && lg ? (float)((max_inf ? 0.0 : ((double)v[j] - weigh.max) * c) * ln2T - ln_z * (double)p.temperature) : -INFINITY;
            }
            const bool whole = i + 4 <= n_mine;
            if (probs) {
                if (p.vec_probs && whole) {
                    __stcs(reinterpret_cast<float4*>(probs + i), make_float4(a[0], a[1], a[2], a[3]));
                } else {
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        if (i + j < n_mine) probs[i + j] = a[j];
                }
            }
            if (lg) {
                if (p.vec_logits && whole) {
                    __stcs(reinterpret_cast<float4*>(lg + i), make_float4(b[0], b[1], b[2], b[3]));
                } else {
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        if (i + j < n_mine) lg[i + j] = b[j];
                }
            }
        }
    }
}

}  // namespace

extern "C" mirror_status mirror_sample(mirror_ctx* ctx, const float* logits, int64_t ld, int M, const float* temperature,
                                       const int32_t* top_k, const float* top_p, const float* min_p, const float* u, int32_t* token,
                                       float* logprob, int32_t* n_kept, float* probs, float* logits_out, void* stream) {
    if (!ctx || M < 0) return MIRROR_ERR_ARG;
    if (M == 0) return MIRROR_OK;
    if (!logits || !u || !token) return MIRROR_ERR_ARG;
    const int V = ctx->desc.vocab;
    if (ld < V || V > kMaxCluster * kMaxPart || (int64_t)M * kMaxCluster > 0x7fffffff) return MIRROR_ERR_SHAPE;
    // (the row is read before its outputs are written, so they may be the logits themselves where the rows lie alike)
    if ((((uintptr_t)logits | (uintptr_t)probs | (uintptr_t)logits_out) & 3) || (probs && (const float*)probs == logits && ld != V) ||
        (logits_out && (const float*)logits_out == logits && ld != V) || (probs && probs == logits_out))
        return MIRROR_ERR_ARG;
    MIRROR_CUDA_OK(cudaSetDevice(ctx->device));
    SampleParams p;
    p.V = V; p.ld = ld;
    int bits = 0;
    while ((1ll << bits) < V) ++bits;
    p.shift = 62 - bits < 51 ? 62 - bits : 51;                   // (a weight has to fit a double's 52 bits)
    p.id_shift = bits > 11 ? bits - 11 : 0;
    p.two_s = ldexp(1.0, p.shift);
    p.two_ms = ldexp(1.0, -p.shift);
    for (int j = 0; j < kTable; ++j) p.table[j] = exp2((double)j / kTable);
    p.temperature = ctx->temperature;
    p.logits = logits; p.temperatures = temperature; p.top_k = top_k; p.top_p = top_p; p.min_p = min_p; p.u = u;
    p.token = token; p.logprob = logprob; p.n_kept = n_kept; p.probs = probs; p.logits_out = logits_out;
    p.vec_in = ((uintptr_t)logits & 15) == 0 && ld % 4 == 0;
    p.vec_probs = ((uintptr_t)probs & 15) == 0 && V % 4 == 0;
    p.vec_logits = ((uintptr_t)logits_out & 15) == 0 && V % 4 == 0;
    // CTAs of a row.  Few rows (two large CTAs an SM hold them all, up to eight to a row): parts of at most 16384 ids in shared memory, and
    // more CTAs where rows are fewer still.  (50 rows x 6519 ids 18.6 us, as many rows 28.4; 204 x 1228 18.1 and 24.3; 205 x 431 10.6 and 9.4.)
    // Many: as many small CTAs to a row as four to an SM allow at once.
    const int sms = ctx->num_sms;
    int most = V > 2 * kShort ? 1 : 8;                           // CTAs that a row has work for (short rows: 512 threads have none)
    while (most < 8 && most * 4 * 512 < V) most <<= 1;
    const bool resident = (int64_t)M * most <= 2 * sms && V <= kMaxCluster * 16384;
    const int threads = resident ? 512 : 256;
    auto part = [&](int c) { return (int)(align_up((size_t)((V + c - 1) / c), (size_t)4 * threads)); };
    int C = 1;
    if (resident)
        while (C < kMaxCluster && (part(C) > 16384 || (part(C) > 4 * threads && (int64_t)2 * C * M <= sms))) C <<= 1;
    else
        while (C < kMaxCluster && (part(C) > kMaxPart || (C < 8 && part(C) > 4 * threads && (int64_t)2 * C * M <= 4 * sms))) C <<= 1;
    p.part = part(C);
    // a histogram word: up to `part` ids counted above, their places of three bits (or one) summed below
    p.off_bits = p.part <= 16384 ? 3 : 1;
    p.off_shift = p.part <= 16384 ? 17 : 16;
    const size_t smem = sizeof(Shared) + (resident ? (size_t)p.part * sizeof(float) : 0);
    auto kernel = resident ? sample_kernel<true, 512> : sample_kernel<false, 256>;
    const int bit = kRowsSample + (resident ? 2 : 0);
    MIRROR_CUDA_OK(mirror_allow_smem(ctx, bit, kernel, (int)(sizeof(Shared) + (resident ? 16384 * sizeof(float) : 0))));
    if (C > 8 && !(ctx->rows_attr_set >> (bit + 1) & 1u)) {
        MIRROR_CUDA_OK(cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1));
        ctx->rows_attr_set |= 1u << (bit + 1);
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)C * (unsigned)M);
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = (cudaStream_t)stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)C;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    MIRROR_CUDA_OK(cudaLaunchKernelEx(&cfg, kernel, p));
    ctx->launches += 1;
    MIRROR_CUDA_OK(cudaGetLastError());
    return MIRROR_OK;
}
