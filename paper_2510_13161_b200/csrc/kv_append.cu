// New rows into the paged cache, turned to their positions on the way (mirror_kv_append), and the frequencies of the rotation
// (mirror_rope_init).
//
// Pair i of a head's first rotary_dim elements turns by the angle a = position * f_i:  (x, y) -> (x cos a - y sin a, y cos a + x sin a).
// Positions reach 10^6, where a product in fp32 would be off by a tenth of a radian: the angle is taken in turns in double precision, its
// whole turns are dropped there, and what is left is within half a turn, which fp32 sine and cosine take.  An angle belongs to a row and
// not to its heads, so a block computes those of its rows once, in shared memory, and reads them for all heads.
//
// What bounds it: bytes (2 * rows * (Hq + 2 Hkv) * d * 2), and for single tokens the launch.  A thread moves 16 elements of a head at a time,
// either 8 pairs or 16 elements that only pass through: two 16-byte loads and stores.
// Measured on a B200: 5.6 TB/s over prompts of 11 k rows (0.45 GB: 80 us), 3.5 us for a token.  Tried and no faster: two or four items
// of a thread on the way at once, eight rows or 512 threads to a block (79.5 to 97 us).
#include <math.h>

#include "mirror_internal.h"

namespace {

constexpr int kThreads = 256;
constexpr int kMaxRowsPerBlock = 4;
constexpr int kMaxBatch = 1024;

struct AppendParams {
    int L, B, R, Hq, Hkv, d, max_rows, max_pages, num_pages;
    int rows_per_block, half, interleaved;   // half: pairs of a head
    int q_heads;                             // 0 without queries
    float amplitude;
    long long q_row, q_layer, kv_row, kv_layer, layer_stride;
    const int32_t* row_start;
    const int32_t* page_table;
    const int32_t* prefix_len;
    const __nv_bfloat16* q;
    const __nv_bfloat16* k;
    const __nv_bfloat16* v;
    __nv_bfloat16* q_out;
    __nv_bfloat16* k_pool;
    __nv_bfloat16* v_pool;
    int* status;
    double turns[64];                        // turns per position of every pair
};

__device__ __forceinline__ void report(int* status, int detail) {
    if (atomicCAS(status, 0, MIRROR_DEV_CHECK) == 0) atomicExch(status + 1, detail);
}

// Whose row is it?  By a warp: two rounds of 32 probes cover 1025 starts.  (A row that belongs to nobody: -1.)
__device__ __forceinline__ int request_of(const int32_t* start, int B, int row, int* first) {
    const int lane = threadIdx.x & 31, step = (B + 32) >> 5;
    int at = lane * step;
    int n = __popc(__ballot_sync(0xffffffffu, at <= B && start[min(at, B)] <= row));
    if (n == 0) return -1;
    const int lo = (n - 1) * step;
    int found = lo;
    for (int k0 = 1; k0 < step; k0 += 32) {                    // (step <= 33)
        at = lo + k0 + lane;
        found += __popc(__ballot_sync(0xffffffffu, k0 + lane < step && at <= B && start[min(at, B)] <= row));
    }
    if (found >= B) return -1;
    *first = start[found];
    return found;
}

__device__ __forceinline__ float2 unpack(uint32_t w) { return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u)); }
__device__ __forceinline__ uint32_t pack(float lo, float hi) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
}

// grid (row groups, shares of a row's heads, layers)
__global__ void __launch_bounds__(kThreads) kv_append_kernel(const __grid_constant__ AppendParams p) {
    __shared__ float2 s_cs[kMaxRowsPerBlock * 64];
    __shared__ int s_pos[kMaxRowsPerBlock];                    // -1: nobody's row
    __shared__ long long s_slot[kMaxRowsPerBlock];             // where the row's first KV head lies in a layer's pool; -1: nowhere
    ptx::grid_dep_wait();
    ptx::grid_dep_launch();
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, row0 = blockIdx.x * p.rows_per_block, layer = blockIdx.z;
    if (warp < p.rows_per_block) {
        const int row = row0 + warp;
        int b = -1, first = 0;
        if (row < p.R) {
            if (p.row_start) {
                b = request_of(p.row_start, p.B, row, &first);
            } else if (row / p.max_rows < p.B) {
                b = row / p.max_rows;
                first = b * p.max_rows;
            }
        }
        if (lane == 0) {
            int pos = -1;
            long long slot = -1;
            if (b >= 0) {
                // (32 bits: with 64 the kernel takes 37 registers instead of 31, and prompts of 11 k rows 85 us instead of 82)
                const int i = row - first, at = (int)min((long long)p.prefix_len[b] + i, 0x7fffffffll);
                const bool within = i < p.max_rows;              // (mirror_attn_causal sees no others)
                if (within && at >= 0 && at < 0x7fffffff && at / 16 < p.max_pages) {
                    const int page = p.page_table[(size_t)b * p.max_pages + at / 16];
                    if (page >= 0 && page < p.num_pages) slot = ((long long)page * p.Hkv * 16 + at % 16) * p.d;
                }
                if (slot < 0) report(p.status, within ? 820 : 830);
                pos = within ? max(at, 0) : -1;
            }
            s_pos[warp] = pos;
            s_slot[warp] = slot;
        }
    }
    __syncthreads();
    for (int i = tid; i < p.rows_per_block * p.half; i += kThreads) {
        const int r = i / p.half, f = i - r * p.half;
        double t = (double)max(s_pos[r], 0) * p.turns[f];
        t -= rint(t);
        float s, c;
        sincospif(2.f * (float)t, &s, &c);
        s_cs[r * 64 + f] = make_float2(c * p.amplitude, s * p.amplitude);
    }
    __syncthreads();
    const int per_head = p.d >> 4, per_row = (p.q_heads + 2 * p.Hkv) * per_head, pair_items = p.half >> 3;
    for (int i = blockIdx.y * kThreads + tid; i < p.rows_per_block * per_row; i += gridDim.y * kThreads) {
        const int r = i / per_row, at = i - r * per_row, head = at / per_head, item = at - head * per_head, row = row0 + r;
        if (s_pos[r] < 0) continue;
        const __nv_bfloat16* src;
        __nv_bfloat16* dst;
        const bool values = head >= p.q_heads + p.Hkv;
        if (head < p.q_heads) {
            src = p.q + layer * p.q_layer + row * p.q_row + head * p.d;
            dst = p.q_out + (((size_t)layer * p.R + row) * p.Hq + head) * p.d;
        } else {
            const int h = head - p.q_heads - (values ? p.Hkv : 0);
            if (s_slot[r] < 0) continue;
            src = (values ? p.v : p.k) + layer * p.kv_layer + row * p.kv_row + h * p.d;
            dst = (values ? p.v_pool : p.k_pool) + layer * p.layer_stride + s_slot[r] + (long long)h * 16 * p.d;
        }
        // the item's two runs of 8 elements: neighbours, or half a rotation apart
        const bool turn = item < pair_items && !values, split = turn && !p.interleaved;
        const int e0 = split ? item * 8 : item * 16, e1 = e0 + (split ? p.half : 8);
        uint4 a = *reinterpret_cast<const uint4*>(src + e0), b = *reinterpret_cast<const uint4*>(src + e1);
        if (turn) {
            uint32_t* const wa = &a.x;
            uint32_t* const wb = &b.x;
            const float2* cs = s_cs + r * 64 + item * 8;
            if (split) {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float2 x = unpack(wa[j]), y = unpack(wb[j]), c0 = cs[2 * j], c1 = cs[2 * j + 1];
                    wa[j] = pack(x.x * c0.x - y.x * c0.y, x.y * c1.x - y.y * c1.y);
                    wb[j] = pack(y.x * c0.x + x.x * c0.y, y.y * c1.x + x.y * c1.y);
                }
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float2 x = unpack(wa[j]), y = unpack(wb[j]), c0 = cs[j], c1 = cs[j + 4];
                    wa[j] = pack(x.x * c0.x - x.y * c0.y, x.y * c0.x + x.x * c0.y);
                    wb[j] = pack(y.x * c1.x - y.y * c1.y, y.y * c1.x + y.x * c1.y);
                }
            }
        }
        *reinterpret_cast<uint4*>(dst + e0) = a;
        *reinterpret_cast<uint4*>(dst + e1) = b;
    }
}

}  // namespace

mirror_status mirror_check_rows(const mirror_rows* rows) {
    if (!rows) return MIRROR_ERR_ARG;
    if (rows->batch <= 0 || rows->n_rows < 0 || rows->max_rows <= 0) return MIRROR_ERR_ARG;
    if (rows->batch > kMaxBatch || rows->n_rows > (1 << 30)) return MIRROR_ERR_SHAPE;
    if (!rows->row_start && (int64_t)rows->batch * rows->max_rows > rows->n_rows) return MIRROR_ERR_SHAPE;
    return MIRROR_OK;
}

extern "C" mirror_status mirror_rope_init(mirror_rope* out, int head_dim, int rotary_dim, int interleaved, double theta,
                                          mirror_rope_scaling scaling, double factor, double original_len, double low, double high,
                                          double amplitude) {
    if (!out) return MIRROR_ERR_ARG;
    if (head_dim != 64 && head_dim != 128) return MIRROR_ERR_UNSUPPORTED;
    if (rotary_dim == 0) rotary_dim = head_dim;
    if (rotary_dim < 0 || rotary_dim > head_dim || rotary_dim % 16 != 0) return MIRROR_ERR_SHAPE;
    if (!(theta > 1.0) || !isfinite(theta) || !(amplitude >= 0.0) || !isfinite(amplitude)) return MIRROR_ERR_ARG;
    if (scaling < MIRROR_ROPE_PLAIN || scaling > MIRROR_ROPE_PAIRS) return MIRROR_ERR_ARG;
    if (scaling != MIRROR_ROPE_PLAIN && (!(factor > 0.0) || !isfinite(factor))) return MIRROR_ERR_ARG;
    const bool blend = scaling == MIRROR_ROPE_TURNS || scaling == MIRROR_ROPE_PAIRS;
    if (blend && (!(original_len > 0.0) || !isfinite(original_len) || !(low > 0.0) || !(high > low) || !isfinite(high))) return MIRROR_ERR_ARG;
    const double two_pi = 6.283185307179586476925286766559;
    const double r = (double)rotary_dim;
    auto clamp01 = [](double x) { return x < 0.0 ? 0.0 : x > 1.0 ? 1.0 : x; };
    double first = 0.0, last = 0.0;
    if (scaling == MIRROR_ROPE_PAIRS) {
        auto pair_at = [&](double turns) { return r * log(original_len / (two_pi * turns)) / (2.0 * log(theta)); };
        first = fmax(floor(pair_at(high)), 0.0);
        last = fmin(ceil(pair_at(low)), r - 1.0);
    }
    out->rotary_dim = rotary_dim;
    out->interleaved = interleaved != 0;
    out->amplitude = amplitude > 0.0 ? amplitude : 1.0;
    for (int i = 0; i < 64; ++i) {
        out->freq[i] = 0.0;
        if (i >= rotary_dim / 2) continue;
        const double f = pow(theta, -2.0 * i / r);
        double w = 1.0;
        if (scaling == MIRROR_ROPE_LINEAR) w = 0.0;
        if (scaling == MIRROR_ROPE_TURNS) w = clamp01((original_len * f / two_pi - low) / (high - low));
        if (scaling == MIRROR_ROPE_PAIRS) w = 1.0 - clamp01((i - first) / fmax(last - first, 0.001));
        out->freq[i] = scaling == MIRROR_ROPE_PLAIN ? f : f * w + f * (1.0 - w) / factor;
    }
    return MIRROR_OK;
}

extern "C" mirror_status mirror_kv_append(mirror_ctx* ctx, const mirror_kv* kv, const mirror_rows* rows, const mirror_rope* rope,
                                          const void* q, int64_t q_row, int64_t q_layer, void* q_out, const void* k, const void* v,
                                          int64_t kv_row, int64_t kv_layer, void* stream) {
    if (!ctx || !kv || !rows) return MIRROR_ERR_ARG;
    mirror_status st = mirror_check_rows(rows);
    if (st != MIRROR_OK || rows->n_rows == 0) return st;
    if (!k || !v || (q != nullptr) != (q_out != nullptr)) return MIRROR_ERR_ARG;
    st = mirror_check_kv(ctx, kv);
    if (st != MIRROR_OK) return st;
    const int d = ctx->desc.head_dim, Hq = ctx->desc.n_q_heads, Hkv = ctx->desc.n_kv_heads;
    if (((uintptr_t)k & 15) || ((uintptr_t)v & 15) || ((uintptr_t)q & 15) || ((uintptr_t)q_out & 15)) return MIRROR_ERR_ARG;
    if (kv_row % 8 || kv_layer % 8 || (q && (q_row % 8 || q_layer % 8))) return MIRROR_ERR_SHAPE;
    // (layers may share their rows, which are only read; rows that are closer than they are long are nobody's layout)
    if (kv_row < (int64_t)Hkv * d || (q && q_row < (int64_t)Hq * d) || kv_layer < 0 || q_layer < 0) return MIRROR_ERR_SHAPE;
    // In place an element is read and written by one thread only where both tensors lie alike; else a row may be turned after another
    // block has overwritten it.
    if (q && q == q_out && ((rows->n_rows > 1 && q_row != (int64_t)Hq * d) || (kv->num_layers > 1 && q_layer != (int64_t)rows->n_rows * Hq * d)))
        return MIRROR_ERR_ARG;
    if (rope) {
        if (rope->rotary_dim <= 0 || rope->rotary_dim > d || rope->rotary_dim % 16 != 0) return MIRROR_ERR_SHAPE;
        if (!isfinite(rope->amplitude)) return MIRROR_ERR_ARG;
    }
    if (kv->num_layers > 65535) return MIRROR_ERR_SHAPE;
    MIRROR_CUDA_OK(cudaSetDevice(ctx->device));
    AppendParams p;
    p.L = kv->num_layers; p.B = rows->batch; p.R = rows->n_rows; p.Hq = Hq; p.Hkv = Hkv; p.d = d;
    p.max_rows = rows->max_rows; p.max_pages = kv->max_pages_per_req; p.num_pages = kv->num_pages;
    p.q_heads = q ? Hq : 0;
    p.half = rope ? rope->rotary_dim / 2 : 0;
    p.interleaved = rope && rope->interleaved;
    p.amplitude = rope ? (float)rope->amplitude : 1.f;
    for (int i = 0; i < 64; ++i) p.turns[i] = rope ? rope->freq[i] * 0.15915494309189533577 : 0.0;
    p.q_row = q_row; p.q_layer = q_layer; p.kv_row = kv_row; p.kv_layer = kv_layer; p.layer_stride = kv->layer_stride;
    p.row_start = rows->row_start; p.page_table = kv->page_table; p.prefix_len = kv->prefix_len;
    p.q = (const __nv_bfloat16*)q; p.k = (const __nv_bfloat16*)k; p.v = (const __nv_bfloat16*)v;
    p.q_out = (__nv_bfloat16*)q_out;
    p.k_pool = (__nv_bfloat16*)const_cast<void*>(kv->k_pool);
    p.v_pool = (__nv_bfloat16*)const_cast<void*>(kv->v_pool);
    p.status = ctx->d_status;
    // Few rows: one to a block and its heads over several blocks, so that all of a token's loads are in flight at once.  Many: four
    // rows to a block, which share its set-up.
    const int items = (p.q_heads + 2 * Hkv) * (d / 16);
    const bool few = (int64_t)p.R * p.L <= 4 * ctx->num_sms;
    p.rows_per_block = few ? 1 : kMaxRowsPerBlock;
    const dim3 grid((unsigned)((p.R + p.rows_per_block - 1) / p.rows_per_block), (unsigned)(few ? (items + kThreads - 1) / kThreads : 1), (unsigned)p.L);
    MIRROR_CUDA_OK(mirror_launch_pdl(kv_append_kernel, grid, dim3(kThreads), 0, (cudaStream_t)stream, p));
    ctx->launches += 1;
    MIRROR_CUDA_OK(cudaGetLastError());
    return MIRROR_OK;
}
