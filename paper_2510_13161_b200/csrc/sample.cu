// One token per row of logits under temperature, Top-k, Top-p and Min-p, from a given uniform (mirror_sample).
//
// With z = (logit - max) / T the weight of an id is exp(z).  Each filter keeps a front of the ranks (logit descending, id ascending), so
// the kept set is the shortest of three fronts, and no sort of the row is needed: only where the front ends has to be found.  What
// decides are sums of weights, and a sum that is off by 10^-7 moves the end of a Top-p front by an id in one row of a hundred (an id's
// share is 10^-5 where the row is open).  Weights are therefore 64-bit integers, round(exp(z) 2^S) with S = 62 - ceil(log2 V), from a
// double-precision exponential: their sums are exact, and the same in whatever order threads and CTAs take them.
//
// A cluster of CTAs has one row, each a contiguous part of it in shared memory (the logits leave HBM once), each warp a contiguous part of
// that, so that sums in the order of the ids are sums over warps.
//   1  load, maximum over the cluster
//   2  a histogram of z in 2048 bins of 1/64: how many ids each holds, and, for Top-p, where in the bin they lie on average, which gives a
//      bin's mass to 10^-4.  With Top-p over the whole row also the exact total
//   3  the leading CTA reads off a bin that surely lies behind the end of the front
//   4  if at most kList ids lie ahead of that, they all go to the leader, which sorts them and does the rest: the usual case
//   4' otherwise only the bin in which the front ends goes to the leader, which sorts it; what lies ahead of it is counted and summed by all.
//      (A bin of more than kList ids, many equal logits above all, is bisected by key, with exact counts and masses of each half.)
//   5  the drawn token, by the warps' masses, and the filtered distribution
// What bounds it: double-precision arithmetic (18 operations an id, 64 a cycle and SM) where Top-p or a draw takes the whole row, the
// bytes otherwise; for a row alone the cluster's barriers.
#include <cooperative_groups.h>
#include <math.h>

#include "mirror_internal.h"

namespace cg = cooperative_groups;

namespace {

using u64 = unsigned long long;

constexpr int kThreads = 512;
constexpr int kWarps = kThreads / 32;
constexpr int kBins = 2048;
constexpr float kBinsPerNat = 64.f;
constexpr int kList = 2048;                   // candidates that the leader sorts
constexpr int kMaxCluster = 16;
constexpr int kMaxPart = 40960;               // ids of a CTA (160 KB)

struct SampleParams {
    int V, M, part;                           // part: ids of a CTA, a multiple of 4 * kThreads
    int shift;                                // S
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
};

// What the CTAs of a cluster tell one another, and what a CTA's warps share.
struct alignas(16) Shared {
    float max[kMaxCluster];
    u64 sum[2][kMaxCluster][3];               // sums of the CTAs, for steps in turns
    u64 warp_sum[kWarps][3];
    u64 warp_mass[kWarps];                    // kept mass of the warps' parts
    u64 total;                                // the row's mass
    int last_bin, n_list, list_at;            // written by the leader
    int bin_k, bin_p;                         // ... the bins in which Top-k and (estimated) Top-p end
    u64 cut_key;                              // composite key of the last kept id
    u64 kept;                                 // its front's mass
    int drawn, n;
    union {
        struct {
            uint32_t hist[kBins];
            uint32_t off[kBins];
        };
        u64 list[kList];                      // (the histogram is no longer needed) composite keys: ~order key, id; ascending in rank
    };
    u64 mass[kList];
};

static_assert(sizeof(Shared) % 16 == 0, "the logits behind it are read 16 bytes at a time");

__device__ __forceinline__ float unkey(uint32_t k) { return __uint_as_float((k & 0x80000000u) ? k & 0x7fffffffu : ~k); }

// round(2^S exp((l - max) / T)): y = (l - max) log2(e) / T = n + f with |f| <= 1/2, and 2^f by its Taylor series to f^11 (the next term
// is below 7e-15).
struct Weigh {
    double max, c;                            // c = log2(e) / T
    int shift;
    bool max_inf;
    __device__ __forceinline__ double exp2_scaled(double y, int s) const {      // 2^(y + s), 0 where that is below 2^-1000
        const double magic = 6755399441055744.0;                 // 1.5 * 2^52: the sum's low bits are the nearest integer
        const double t = y + magic;
        const int n = __double2loint(t);
        const double f = y - (t - magic);
        double r = 4.4455382718708116e-10;                       // ln(2)^k / k!, k = 11 .. 0
        r = fma(r, f, 7.0549116208011234e-09);
        r = fma(r, f, 1.0178086009239699e-07);
        r = fma(r, f, 1.3215486790144307e-06);
        r = fma(r, f, 1.5252733804059840e-05);
        r = fma(r, f, 1.5403530393381609e-04);
        r = fma(r, f, 1.3333558146428443e-03);
        r = fma(r, f, 9.6181291076284772e-03);
        r = fma(r, f, 5.5504108664821580e-02);
        r = fma(r, f, 2.4022650695910071e-01);
        r = fma(r, f, 6.9314718055994531e-01);
        r = fma(r, f, 1.0);
        const int e = n + s;
        if (!(y > -1000.0)) return 0.0;
        return __hiloint2double(__double2hiint(r) + (e << 20), __double2loint(r));
    }
    __device__ __forceinline__ double y_of(float l) const { return max_inf ? 0.0 : ((double)l - max) * c; }
    // (of an id that may be kept: neither NaN nor -inf; where the maximum is +inf only ids of +inf may)
    __device__ __forceinline__ u64 operator()(float l) const {
        const double w = exp2_scaled(y_of(l), shift);
        return (u64)__double_as_longlong(w + 4503599627370496.0) & 0xfffffffffffffull;          // + 2^52: the low bits are the integer
    }
    __device__ __forceinline__ double exact(float l) const { return exp2_scaled(y_of(l), 0); }
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

// The first n entries of the list in ascending order (bitonic, by the whole block).
__device__ __noinline__ void sort_list(Shared& s, int n) {
    const int tid = threadIdx.x;
    int n2 = 32;
    while (n2 < n) n2 <<= 1;
    __syncthreads();
    for (int i = n + tid; i < n2; i += kThreads) s.list[i] = ~0ull;
    for (int size = 2; size <= n2; size <<= 1)
        for (int d = size >> 1; d; d >>= 1) {
            __syncthreads();
            for (int t = tid; t < n2 / 2; t += kThreads) {
                const int i = ((t & ~(d - 1)) << 1) | (t & (d - 1)), j = i | d;
                const u64 a = s.list[i], b = s.list[j];
                if ((a > b) == ((i & size) == 0)) { s.list[i] = b; s.list[j] = a; }
            }
        }
    __syncthreads();
}

__global__ void __launch_bounds__(kThreads) sample_kernel(const __grid_constant__ SampleParams p) {
    extern __shared__ __align__(16) uint8_t smem_raw[];
    Shared& s = *reinterpret_cast<Shared*>(smem_raw);
    float* const z = reinterpret_cast<float*>(smem_raw + sizeof(Shared));
    cg::cluster_group cluster = cg::this_cluster();
    const int C = (int)cluster.num_blocks(), rank = (int)cluster.block_rank(), row = blockIdx.x / C;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int first = rank * p.part;                             // the part's first id
    const int n_mine = max(0, min(p.part, p.V - first));
    const int per_warp = p.part / kWarps, w0 = warp * per_warp, w1 = min(w0 + per_warp, (n_mine + 3) & ~3);
    Shared* const lead = cluster.map_shared_rank(&s, 0);

    ptx::grid_dep_wait();
    ptx::grid_dep_launch();
    // ---- 1: load, maximum.  (What cannot be kept, NaN and the part's end, becomes -inf.)
    const float* const in = p.logits + (long long)row * p.ld + first;
    float mx = -INFINITY;
    if (p.vec_in) {
#pragma unroll 4
        for (int i = w0 + lane * 4; i < w1; i += 128) {
            float v[4];
            if (i + 4 <= n_mine) {
                *reinterpret_cast<float4*>(v) = __ldcs(reinterpret_cast<const float4*>(in + i));
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j) v[j] = i + j < n_mine ? in[i + j] : -INFINITY;
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) { v[j] = v[j] == v[j] ? v[j] : -INFINITY; mx = fmaxf(mx, v[j]); }
            *reinterpret_cast<float4*>(z + i) = *reinterpret_cast<float4*>(v);
        }
    } else {
#pragma unroll 8
        for (int i = w0 + lane; i < w1; i += 32) {
            float v = i < n_mine ? __ldcs(in + i) : -INFINITY;
            v = v == v ? v : -INFINITY;
            mx = fmaxf(mx, v);
            z[i] = v;
        }
    }
    for (int i = tid; i < kBins; i += kThreads) s.hist[i] = s.off[i] = 0;
    if (tid == 0) { s.n_list = 0; s.list_at = 0; }
#pragma unroll
    for (int o = 16; o; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
    if (lane == 0) s.warp_sum[warp][0] = __float_as_uint(mx);
    __syncthreads();
    if (tid < kWarps) {
        mx = __uint_as_float((uint32_t)s.warp_sum[tid][0]);
#pragma unroll
        for (int o = 8; o; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffu, mx, o));
        if (tid < C) cluster.map_shared_rank(&s, tid)->max[rank] = mx;
    }
    cluster.sync();
    mx = -INFINITY;
    for (int c = 0; c < C; ++c) mx = fmaxf(mx, s.max[c]);

    // ---- the row's settings
    float T = p.temperatures ? p.temperatures[row] : p.temperature;
    const bool first_only = !(T > 0.f);
    if (first_only) T = 1.f;
    int k = p.top_k ? p.top_k[row] : 0;
    if (first_only) k = 1;
    const bool by_k = k > 0 && k < p.V;
    const double top_p = p.top_p && !first_only ? (double)p.top_p[row] : 1.0;
    const bool by_p = top_p < 1.0;
    const double min_p = p.min_p && !first_only ? (double)p.min_p[row] : 0.0;
    const bool by_m = min_p > 0.0;
    Weigh weigh;
    weigh.max = (double)mx;
    weigh.c = 1.4426950408889634074 / (double)T;
    weigh.shift = p.shift;
    weigh.max_inf = mx == INFINITY;
    auto may = [&](float l) { return weigh.max_inf ? l == INFINITY : l > -INFINITY; };
    const bool none = mx == -INFINITY;                           // (nothing to keep)
    const u64 min_w = by_m ? (u64)fmin(ceil(min_p * exp2((double)p.shift)), exp2((double)p.shift)) : 0ull;
    // composite key of an id: smaller is ahead
    auto key_of = [&](float l, int id) { return ((u64)~mirror_order_key(l + 0.f) << 32) | (uint32_t)id; };      // (-0 and 0 are equal)
    int turn = 0;
    // Sums over the cluster of what f(l, i, sums) adds for the ids of the part; every thread gets them.
    struct Sums {
        u64 n, m, o;
    };
    auto all_sums = [&](auto f) -> Sums {
        Sums a = {0, 0, 0};
        for (int i = w0 + lane * 4; i < w1; i += 128) {
            const float4 v = *reinterpret_cast<const float4*>(z + i);
            f(v.x, i, a); f(v.y, i + 1, a); f(v.z, i + 2, a); f(v.w, i + 3, a);
        }
        a.n = warp_sum64(a.n);
        a.m = warp_sum64(a.m);
        a.o = warp_sum64(a.o);
        __syncthreads();
        if (lane == 0) { s.warp_sum[warp][0] = a.n; s.warp_sum[warp][1] = a.m; s.warp_sum[warp][2] = a.o; }
        __syncthreads();
        if (tid < 3 * C) {
            const int c = tid / 3, k = tid - c * 3;
            u64 t = 0;
            for (int w = 0; w < kWarps; ++w) t += s.warp_sum[w][k];
            cluster.map_shared_rank(&s, c)->sum[turn][rank][k] = t;
        }
        cluster.sync();
        a = {0, 0, 0};
        for (int c = 0; c < C; ++c) { a.n += s.sum[turn][c][0]; a.m += s.sum[turn][c][1]; a.o += s.sum[turn][c][2]; }
        turn ^= 1;                                               // (read before the other turn's barrier: rewritten after it)
        return a;
    };

    u64 cut = ~0ull;                                             // composite key of the last id of the front
    u64 total = 0;
    if (!none && (by_k || by_p || by_m)) {
        // ---- 2: histogram
        const float inv_T = 1.f / T;
        auto bin_of = [&](float l, float& at) {
            at = weigh.max_inf ? 0.f : fminf((mx - l) * inv_T * kBinsPerNat, (float)(kBins - 1));
            return (int)at;
        };
        const bool whole_total = by_p && !by_k;                  // Top-p of the whole row
        for (int i = w0 + lane * 4; i < w1; i += 128) {
            const float4 v4 = *reinterpret_cast<const float4*>(z + i);
            const float v[4] = {v4.x, v4.y, v4.z, v4.w};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (!may(v[j])) continue;
                float at;
                const int bin = bin_of(v[j], at);
                atomicAdd(&s.hist[bin], 1u);
                if (by_p) atomicAdd(&s.off[bin], (uint32_t)((at - (float)bin) * 1024.f));
                if (whole_total) total += weigh(v[j]);
            }
        }
        total = warp_sum64(total);
        if (lane == 0) s.warp_sum[warp][0] = total;
        __syncthreads();
        if (tid == 0) {
            u64 a = 0;
            for (int w = 0; w < kWarps; ++w) a += s.warp_sum[w][0];
            lead->sum[0][rank][0] = a;
        }
        if (rank != 0)
            for (int i = tid; i < kBins; i += kThreads) {
                const uint32_t n = s.hist[i];
                if (n) {
                    atomicAdd(&lead->hist[i], n);
                    if (by_p) atomicAdd(&lead->off[i], s.off[i]);
                }
            }
        cluster.sync();
        // ---- 3: a bin behind the front's end
        if (rank == 0) {
            constexpr int kPer = kBins / kThreads;
            u64 n = 0;
            double m = 0.0;
            uint32_t cnt[kPer];
            double ms[kPer];
#pragma unroll
            for (int j = 0; j < kPer; ++j) {
                const int b = tid * kPer + j;
                cnt[j] = s.hist[b];
                ms[j] = 0.0;
                if (cnt[j] && by_p) {
                    // (the mean of exp(-x) over a 64th is exp(-mean) but for a relative x^2 / 2 of 10^-4; the last bin is open: no mass)
                    const float mean = ((float)b + (float)s.off[b] * (1.f / 1024.f) / (float)cnt[j]) * (1.f / kBinsPerNat);
                    ms[j] = b == kBins - 1 ? 0.0 : (double)cnt[j] * (double)expf(-mean);
                }
                n += cnt[j];
                m += ms[j];
            }
            // exclusive sums over the threads
            u64 n_in = warp_incl64(n);
            double m_in = m;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const double t = __shfl_up_sync(0xffffffffu, m_in, o);
                if (lane >= o) m_in += t;
            }
            if (lane == 31) { s.warp_sum[warp][0] = n_in; s.warp_sum[warp][1] = (u64)__double_as_longlong(m_in); }
            if (tid == 0) {
                s.last_bin = s.bin_k = s.bin_p = kBins - 1;
                u64 a = 0;
                for (int c = 0; c < C; ++c) a += s.sum[0][c][0];
                s.total = a;
            }
            __syncthreads();
            for (int w = 0; w < warp; ++w) { n_in += s.warp_sum[w][0]; m_in += __longlong_as_double((long long)s.warp_sum[w][1]); }
            u64 nb = n_in - n;
            double mb = m_in - m;
            // Top-k's bin, and about what its front weighs
            if (by_k) {
#pragma unroll
                for (int j = 0; j < kPer; ++j) {
                    if (nb < (u64)k && nb + cnt[j] >= (u64)k) {
                        s.bin_k = tid * kPer + j;
                        s.warp_mass[0] = (u64)__double_as_longlong(mb + ms[j] * (double)(k - (int)nb) / (double)cnt[j]);
                    }
                    nb += cnt[j];
                    mb += ms[j];
                }
                if (tid == kThreads - 1 && nb < (u64)k) s.warp_mass[0] = (u64)__double_as_longlong(mb);
                __syncthreads();
                nb = n_in - n;
                mb = m_in - m;
            }
            const double row_mass = by_k ? __longlong_as_double((long long)s.warp_mass[0]) : (double)s.total * exp2(-(double)p.shift);
            const double about = by_p ? top_p * row_mass : 0.0, want = whole_total ? about * 1.002 : 0.0;
            // (Top-p behind Top-k is a share of all that Top-k leaves: then Min-p does not shorten the list)
            const float m_at = -logf((float)fmin(min_p, 1.0)) * kBinsPerNat + 1.f;
            const bool m_ends = by_m && !(by_k && by_p);
#pragma unroll
            for (int j = 0; j < kPer; ++j) {
                nb += cnt[j];
                mb += ms[j];
                // the first bin at which one of the filters is surely through
                if ((by_k && nb >= (u64)k) || (whole_total && mb >= want) || (m_ends && (float)(tid * kPer + j) >= m_at)) {
                    atomicMin(&s.last_bin, tid * kPer + j);
                    break;
                }
            }
            mb = m_in - m;
            if (by_p) {
#pragma unroll
                for (int j = 0; j < kPer; ++j) {
                    mb += ms[j];
                    if (mb >= about) { atomicMin(&s.bin_p, tid * kPer + j); break; }
                }
            }
            __syncthreads();
            // how many ids that is
            nb = n_in - n;
#pragma unroll
            for (int j = 0; j < kPer; ++j) {
                nb += cnt[j];
                if (tid * kPer + j == s.last_bin) s.n_list = (int)min(nb, (u64)0x7fffffff);
            }
            __syncthreads();
            if (tid < C) {
                Shared* const o = cluster.map_shared_rank(&s, tid);
                o->last_bin = s.last_bin;
                o->bin_k = s.bin_k;
                o->bin_p = s.bin_p;
                o->n_list = s.n_list;
                o->total = s.total;
            }
        }
        cluster.sync();
        const int n_list = s.n_list, last_bin = s.last_bin;
        total = s.total;
        if (n_list <= kList) {
            // ---- 4: the leader's list
            for (int i = w0 + lane * 4; i < w1; i += 128) {
                const float4 v4 = *reinterpret_cast<const float4*>(z + i);
                const float v[4] = {v4.x, v4.y, v4.z, v4.w};
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    if (!may(v[j])) continue;
                    float at;
                    if (bin_of(v[j], at) > last_bin) continue;
                    const int slot = atomicAdd(&lead->list_at, 1);
                    if (slot < kList) lead->list[slot] = key_of(v[j], first + i + j);
                }
            }
            cluster.sync();
            if (rank == 0) {
                sort_list(s, n_list);
                constexpr int kPer = kList / kThreads;
                // inclusive sums of mass[] over the list: a thread has neighbours
                auto scan = [&](u64 (&w)[kPer], u64& before) -> u64 {
                    u64 mine = 0;
#pragma unroll
                    for (int j = 0; j < kPer; ++j) mine += w[j];
                    const u64 in_ = warp_incl64(mine);
                    __syncthreads();
                    if (lane == 31) s.warp_sum[warp][0] = in_;
                    __syncthreads();
                    before = in_ - mine;
                    u64 all = 0;
                    for (int q = 0; q < kWarps; ++q) {
                        if (q < warp) before += s.warp_sum[q][0];
                        all += s.warp_sum[q][0];
                    }
                    return all;
                };
                u64 w[kPer], before;
#pragma unroll
                for (int j = 0; j < kPer; ++j) {
                    const int r = tid * kPer + j;
                    w[j] = r < n_list ? weigh(unkey(~(uint32_t)(s.list[r] >> 32))) : 0ull;
                    if (r < n_list) s.mass[r] = w[j];
                }
                u64 sel[kPer];
#pragma unroll
                for (int j = 0; j < kPer; ++j) sel[j] = by_k && tid * kPer + j >= k ? 0ull : w[j];
                const u64 part = scan(sel, before);
                const double want = top_p * (double)(whole_total ? total : part);
                int kept = 0;
                u64 kept_mass = 0;
#pragma unroll
                for (int j = 0; j < kPer; ++j) {
                    const int r = tid * kPer + j;
                    const bool stays = r < n_list && (r == 0 || ((!by_k || r < k) && (!by_p || (double)before < want) && (!by_m || w[j] >= min_w)));
                    kept += stays;
                    if (stays) kept_mass += w[j];
                    before += sel[j];
                }
                kept = __reduce_add_sync(0xffffffffu, kept);
                kept_mass = warp_sum64(kept_mass);
                __syncthreads();
                if (lane == 0) { s.warp_sum[warp][0] = (u64)kept; s.warp_sum[warp][1] = kept_mass; }
                __syncthreads();
                int n = 0;
                u64 Z = 0;
                for (int q = 0; q < kWarps; ++q) { n += (int)s.warp_sum[q][0]; Z += s.warp_sum[q][1]; }
                const u64 last = s.list[n - 1];
                if (tid < C && (p.probs || p.logits_out)) {
                    Shared* const o = cluster.map_shared_rank(&s, tid);
                    o->cut_key = last;
                    o->kept = Z;
                }
                // the draw: the kept ids in their own order (id, then the key's place in the list)
                __syncthreads();
                u64 by_id[kPer];
#pragma unroll
                for (int j = 0; j < kPer; ++j) {
                    const int r = tid + j * kThreads;
                    by_id[j] = r < n ? ((s.list[r] & 0xffffffffull) << 32) | (uint32_t)r : ~0ull;
                }
                __syncthreads();
#pragma unroll
                for (int j = 0; j < kPer; ++j) s.list[tid + j * kThreads] = by_id[j];
                sort_list(s, n);
#pragma unroll
                for (int j = 0; j < kPer; ++j) {
                    const int r = tid * kPer + j;
                    w[j] = r < n ? s.mass[(uint32_t)s.list[r]] : 0ull;
                }
                scan(w, before);
                const float u = p.u[row];
                const double t = fmax((double)u, 0.0) * (double)Z;
                const u64 target = t >= (double)Z ? Z - 1 : (u64)t;          // the first id whose inclusive sum is above it
#pragma unroll
                for (int j = 0; j < kPer; ++j) {
                    const int r = tid * kPer + j;
                    if (r < n && before <= target && before + w[j] > target) {
                        p.token[row] = (int32_t)(s.list[r] >> 32);
                        if (p.logprob) p.logprob[row] = (float)log((double)w[j] / (double)Z);
                        if (p.n_kept) p.n_kept[row] = n;
                    }
                    before += w[j];
                }
            }
            if (!p.probs && !p.logits_out) return;
            cluster.sync();
            cut = s.cut_key;
            total = s.kept;
        } else {
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
            // The smallest key whose front (count, mass) fulfils `done`, which is monotone; guessed to lie in bin `b`.
            auto end_of = [&](int b, bool by_mass, auto done) -> u64 {
                u64 n0, m0, n_in;
                for (;;) {
                    // what lies ahead of the bin, and the bin itself into the leader's list
                    if (rank == 0 && tid == 0) s.list_at = 0;
                    cluster.sync();
                    const Sums a = all_sums([&](float l, int i, Sums& a) {
                        if (!may(l)) return;
                        float at;
                        const int bin = bin_of(l, at);
                        if (bin > b) return;
                        const u64 w = by_mass ? weigh(l) : 0ull;
                        if (bin < b) {
                            ++a.n;
                            a.m += w;
                        } else {
                            a.n += 1ull << 32;
                            a.o += w;
                            const int slot = atomicAdd(&lead->list_at, 1);
                            if (slot < kList) lead->list[slot] = key_of(l, first + i);
                        }
                    });
                    n0 = a.n & 0xffffffffull;
                    n_in = a.n >> 32;
                    m0 = a.m;
                    if (n0 > 0 && done(n0, m0)) { --b; continue; }                                // it ends ahead of this bin
                    if (b < kBins - 1 && !done(n0 + n_in, m0 + a.o)) { ++b; continue; }           // ... or behind it
                    break;
                }
                if (n_in > (u64)kList) {
                    u64 lo = b > 0 ? (u64)~(edge(b - 1) - 1) << 32 : 0ull, hi = ((u64)~edge(b) << 32) | 0xffffffffull;
                    while (lo < hi) {
                        const u64 mid = lo + ((hi - lo) >> 1);
                        const Sums a = front(mid);
                        if (done(a.n, a.m)) hi = mid; else lo = mid + 1;
                    }
                    return lo;
                }
                if (rank == 0) {
                    const int n = (int)n_in;
                    sort_list(s, n);
                    constexpr int kPer = kList / kThreads;
                    u64 w[kPer], mine = 0;
#pragma unroll
                    for (int j = 0; j < kPer; ++j) {
                        const int r = tid * kPer + j;
                        w[j] = by_mass && r < n ? weigh(unkey(~(uint32_t)(s.list[r] >> 32))) : 0ull;
                        mine += w[j];
                    }
                    u64 at = warp_incl64(mine);
                    __syncthreads();
                    if (lane == 31) s.warp_sum[warp][0] = at;
                    if (tid == 0) s.list_at = n - 1;
                    __syncthreads();
                    at += m0 - mine;
                    for (int q = 0; q < warp; ++q) at += s.warp_sum[q][0];
#pragma unroll
                    for (int j = 0; j < kPer; ++j) {
                        const int r = tid * kPer + j;
                        at += w[j];
                        if (r < n && done(n0 + r + 1, at)) { atomicMin(&s.list_at, r); break; }
                    }
                    __syncthreads();
                    if (tid < C) cluster.map_shared_rank(&s, tid)->cut_key = s.list[s.list_at];
                }
                cluster.sync();
                const u64 c = s.cut_key;
                cluster.sync();                                  // (the next one may be written)
                return c;
            };
            if (by_k) {
                cut = end_of(s.bin_k, false, [&](u64 n, u64) { return n >= (u64)k; });
                if (by_p) total = front(cut).m;
            }
            if (by_p) {
                const double want = top_p * (double)total;
                const u64 c = end_of(s.bin_p, true, [&](u64 n, u64 m) { return n >= 1 && (double)m >= want; });
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
                        if (l > -INFINITY && weigh(l) >= min_w) hi = mid; else lo = mid + 1;
                    }
                    if (lane == 0) s.warp_mass[0] = ((u64)~hi << 32) | 0xffffffffull;
                }
                __syncthreads();
                cut = min(cut, s.warp_mass[0]);
                __syncthreads();
            }
        }
    }
    // ---- 5: the warps' kept masses, the draw, the distribution
    auto kept = [&](float l, int i) { return may(l) && key_of(l, first + i) <= cut; };
    const bool listed = !none && (by_k || by_p || by_m) && s.n_list <= kList;
    u64 Z = total;
    if (!listed) {
        u64 n = 0, m = 0;
        for (int i = w0 + lane * 4; i < w1; i += 128) {
            const float4 v4 = *reinterpret_cast<const float4*>(z + i);
            const float v[4] = {v4.x, v4.y, v4.z, v4.w};
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (kept(v[j], i + j)) { ++n; m += weigh(v[j]); }
        }
        n = warp_sum64(n);
        m = warp_sum64(m);
        __syncthreads();
        if (lane == 0) { s.warp_sum[warp][0] = n; s.warp_mass[warp] = m; }
        __syncthreads();
        if (tid < C) {
            u64 a = 0, b = 0;
            for (int w = 0; w < kWarps; ++w) { a += s.warp_sum[w][0]; b += s.warp_mass[w]; }
            Shared* const o = cluster.map_shared_rank(&s, tid);
            o->sum[turn][rank][0] = a;
            o->sum[turn][rank][1] = b;
        }
        cluster.sync();
        n = 0;
        Z = 0;
        u64 before = 0;                                          // mass of the CTAs ahead
        for (int c = 0; c < C; ++c) {
            n += s.sum[turn][c][0];
            if (c < rank) before += s.sum[turn][c][1];
            Z += s.sum[turn][c][1];
        }
        if (n == 0) {
            if (rank == 0 && tid == 0) {
                p.token[row] = -1;
                if (p.logprob) p.logprob[row] = -INFINITY;
                if (p.n_kept) p.n_kept[row] = 0;
            }
        } else {
            if (rank == 0 && tid == 0 && p.n_kept) p.n_kept[row] = (int32_t)n;
            const double t = fmax((double)p.u[row], 0.0) * (double)Z;
            const u64 target = t >= (double)Z ? Z - 1 : (u64)t;
            for (int w = 0; w < warp; ++w) before += s.warp_mass[w];
            if (before <= target && before + s.warp_mass[warp] > target) {
                for (int i0 = w0; i0 < w1; i0 += 32) {           // (this warp's ids in order)
                    const int i = i0 + lane;
                    const float l = i < w1 ? z[i] : -INFINITY;
                    const u64 w = i < w1 && kept(l, i) ? weigh(l) : 0ull, in_ = before + warp_incl64(w);
                    const uint32_t over = __ballot_sync(0xffffffffu, in_ > target);
                    if (over) {
                        if (lane == __ffs(over) - 1) {
                            p.token[row] = first + i;
                            if (p.logprob) p.logprob[row] = (float)log((double)w / (double)Z);
                        }
                        break;
                    }
                    before = __shfl_sync(0xffffffffu, in_, 31);
                }
            }
        }
    }
    if (p.probs || p.logits_out) {
        const double unit = (double)Z * exp2(-(double)p.shift), inv = 1.0 / unit, ln_z = log(unit);
        const double ln2T = 0.69314718055994530942 * (double)p.temperature;
        float* const probs = p.probs ? p.probs + (size_t)row * p.V + first : nullptr;
        float* const lg = p.logits_out ? p.logits_out + (size_t)row * p.V + first : nullptr;
        for (int i = w0 + lane * 4; i < w1; i += 128) {
            const float4 v4 = *reinterpret_cast<const float4*>(z + i);
            const float v[4] = {v4.x, v4.y, v4.z, v4.w};
            float a[4], b[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const bool in_front = kept(v[j], i + j);
                a[j] = in_front && probs ? (float)(weigh.exact(v[j]) * inv) : 0.f;
                b[j] = in_front ? (float)(weigh.y_of(v[j]) * ln2T - ln_z * (double)p.temperature) : -INFINITY;
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
    if (ld < V || V > kMaxCluster * kMaxPart) return MIRROR_ERR_SHAPE;
    // (the row is read before its outputs are written, so they may be the logits themselves where the rows lie alike)
    if ((((uintptr_t)logits | (uintptr_t)probs | (uintptr_t)logits_out) & 3) || (probs && (const float*)probs == logits && ld != V) ||
        (logits_out && (const float*)logits_out == logits && ld != V) || (probs && probs == logits_out))
        return MIRROR_ERR_ARG;
    MIRROR_CUDA_OK(cudaSetDevice(ctx->device));
    SampleParams p;
    p.V = V; p.M = M; p.ld = ld;
    int bits = 0;
    while ((1ll << bits) < V) ++bits;
    p.shift = 62 - bits < 51 ? 62 - bits : 51;                   // (a weight has to fit a double's 52 bits)
    p.temperature = ctx->temperature;
    p.logits = logits; p.temperatures = temperature; p.top_k = top_k; p.top_p = top_p; p.min_p = min_p; p.u = u;
    p.token = token; p.logprob = logprob; p.n_kept = n_kept; p.probs = probs; p.logits_out = logits_out;
    p.vec_in = ((uintptr_t)logits & 15) == 0 && ld % 4 == 0;
    p.vec_probs = ((uintptr_t)probs & 15) == 0 && V % 4 == 0;
    p.vec_logits = ((uintptr_t)logits_out & 15) == 0 && V % 4 == 0;
    // CTAs of a row: parts of at most 16384 ids, so that two or three CTAs share an SM; more CTAs where rows are few
    int C = 1;
    auto part = [&](int c) { return (int)(align_up((size_t)((V + c - 1) / c), 4 * kThreads)); };
    while (C < kMaxCluster && (part(C) > 16384 || (part(C) > 4 * kThreads && (int64_t)2 * C * M <= ctx->num_sms))) C <<= 1;
    p.part = part(C);
    const size_t smem = sizeof(Shared) + (size_t)p.part * sizeof(float);
    MIRROR_CUDA_OK(cudaFuncSetAttribute(sample_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
    if (C > 8) MIRROR_CUDA_OK(cudaFuncSetAttribute(sample_kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1));
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)C * (unsigned)M);
    cfg.blockDim = dim3(kThreads);
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
    MIRROR_CUDA_OK(cudaLaunchKernelEx(&cfg, sample_kernel, p));
    ctx->launches += 1;
    MIRROR_CUDA_OK(cudaGetLastError());
    return MIRROR_OK;
}
