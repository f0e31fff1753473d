// evict.hip -- which cached tokens to keep, and moving them to the front.
//
// Selection.  A row of weights is mapped to 32-bit keys in the order of the
// numbers (NaN lowest, -0 as +0).  The smallest key that is kept, and how many
// of the tokens at exactly that key, follow from four counts of eight bits
// each, from the top byte down; the kept indices then come out in order by a
// prefix sum over the row.
//
// Compaction.  Row keep[i] >= i moves to row i, in place: a tile of rows is
// read before it is written, and what a tile writes (rows below its end) no
// later tile reads.  So one workgroup takes one head's rows of a plane in
// order; heads, planes, layers and requests are independent.

#include <math.h>

#include "paged.h"

namespace tkv {
namespace {

constexpr int kThreads = 256;

struct SelectParams {
    const float *weights;
    const int32_t *len;
    int32_t *keep, *new_len;
    int64_t weight_stride;
    int32_t num_reqs, heads, budget, sink, recent;
};

// A float's bits as a number in the same order.
__device__ __forceinline__ uint32_t ordered(float x) {
    if (x != x) return 0;
    const uint32_t b = __builtin_bit_cast(uint32_t, x == 0.0f ? 0.0f : x);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}

// Sum over the lanes before this one in the workgroup, and the total.
__device__ __forceinline__ int prefix(int x, int *scratch, int &total) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int y = x;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const int z = __shfl_up(y, d);
        if (lane >= d) y += z;
    }
    if (lane == 63) scratch[wave] = y;
    __syncthreads();
    int before = 0;
    total = 0;
#pragma unroll
    for (int w = 0; w < kThreads / 64; ++w) {
        if (w < wave) before += scratch[w];
        total += scratch[w];
    }
    __syncthreads();
    return before + y - x;
}

__global__ __launch_bounds__(kThreads) void evict_select_kernel(SelectParams p) {
    __shared__ int hist[256];
    __shared__ int scratch[kThreads / 64];
    __shared__ uint32_t found[2];          // the byte, and how many are still to be taken below it
    const int tid = threadIdx.x;
    const int64_t g = blockIdx.x;          // (layer * num_reqs + request) * heads + head
    const int r = (int)(g / p.heads % p.num_reqs);
    const int32_t raw = p.len[r];
    const int n = (int)min((int64_t)(raw < 0 ? 0 : raw), p.weight_stride);
    const int m = min(n, p.budget);
    int32_t *keep = p.keep + g * p.budget;
    if (g < (int64_t)p.num_reqs * p.heads && g % p.heads == 0 && tid == 0) p.new_len[r] = m;
    for (int i = m + tid; i < p.budget; i += kThreads) keep[i] = -1;
    if (n <= p.budget) {
        for (int i = tid; i < n; i += kThreads) keep[i] = i;
        return;
    }
    const float *w = p.weights + g * p.weight_stride;
    const int lo = p.sink, hi = n - p.recent;                 // candidates
    int want = p.budget - p.sink - p.recent;                  // of them, so many
    uint32_t known = 0, mask = 0;
    if (want > 0)
        for (int shift = 24; shift >= 0; shift -= 8) {
            hist[tid] = 0;
            __syncthreads();
            for (int i = lo + tid; i < hi; i += kThreads) {
                const uint32_t k = ordered(w[i]);
                if ((k & mask) == known) atomicAdd(&hist[(k >> shift) & 255], 1);
            }
            __syncthreads();
            // from the top byte down: where the wanted number is reached
            int total;
            const int mine = hist[255 - tid], before = prefix(mine, scratch, total);
            if (before < want && before + mine >= want) {
                found[0] = 255 - tid;
                found[1] = (uint32_t)(want - before);
            }
            __syncthreads();
            known |= found[0] << shift;
            mask |= 255u << shift;
            want = (int)found[1];
            __syncthreads();
        }
    // kept: above `known`, and the first `want` at it
    int at = 0, ties = 0;
    for (int base = 0; base < n; base += kThreads) {
        const int i = base + tid;
        const bool safe = i < n && (i < lo || i >= hi), cand = i < n && !safe && p.budget > p.sink + p.recent;
        const uint32_t k = cand ? ordered(w[i]) : 0;
        int total;
        const bool tie = cand && k == known;
        const int rank = ties + prefix(tie ? 1 : 0, scratch, total);
        ties += total;
        const bool kept = safe || (cand && k > known) || (tie && rank < want);
        const int to = at + prefix(kept ? 1 : 0, scratch, total);
        at += total;
        if (kept) keep[to] = i;
    }
}

struct CompactParams {
    Paged cache;
    char *layers[KV_MAX_LAYERS];
    const int32_t *keep, *new_len;
    float *weights;
    int64_t weight_stride;
    int32_t num_layers, heads, kv_heads, budget;
    int32_t vecs;          // 16-byte vectors that move together for a token: a head's row, or all heads'
};

// One workgroup: a (layer, request, head, plane), a tile of kThreads vectors
// at a time.
__global__ __launch_bounds__(kThreads) void evict_compact_kernel(CompactParams p) {
    const int tid = threadIdx.x;
    int64_t x = blockIdx.x;
    const int plane = (int)(x & 1);
    x >>= 1;
    const int64_t g = x;                   // (layer * num_reqs + request) * heads + head
    const int h = (int)(g % p.heads), r = (int)(g / p.heads % p.cache.num_reqs), l = (int)(g / p.heads / p.cache.num_reqs);
    const int n = min(max(p.new_len[r], 0), p.budget);
    const int32_t *keep = p.keep + g * p.budget;
    char *base = p.layers[l] + plane * p.cache.kv_stride + (int64_t)h * p.cache.head_bytes;
    const int64_t total = (int64_t)n * p.vecs;
    for (int64_t at = 0; at < total; at += kThreads) {
        const int64_t v = at + tid;
        const int i = (int)(v / p.vecs), vec = (int)(v % p.vecs);
        char *to = nullptr;
        u32x4 y = {0, 0, 0, 0};
        if (v < total) {
            const int32_t src = keep[i];
            if (src > i) {
                uint32_t ra, rb;
                const int32_t a = block_of(p.cache, r, (uint32_t)src, ra), b = block_of(p.cache, r, (uint32_t)i, rb);
                if (a >= 0 && b >= 0) {
                    y = *(const u32x4 *)(base + (((int64_t)a * p.cache.block16 + (int64_t)ra * p.cache.row16 + vec) << 4));
                    to = base + (((int64_t)b * p.cache.block16 + (int64_t)rb * p.cache.row16 + vec) << 4);
                }
            }
        }
        __syncthreads();
        if (to) *(u32x4 *)to = y;
    }
    if (plane == 0 && p.weights) {
        float *w = p.weights + g * p.weight_stride;
        __syncthreads();
        for (int at = 0; at < n; at += kThreads) {
            const int i = at + tid;
            const int32_t src = i < n ? keep[i] : -1;
            const bool moves = src > i && src < p.weight_stride;
            const float y = moves ? w[src] : 0.0f;
            __syncthreads();
            if (moves) w[i] = y;
        }
    }
}

}  // namespace
}  // namespace tkv

extern "C" {

int kv_evict_select(const float *d_weights, int64_t weight_stride, const int32_t *d_len, int32_t num_layers,
                    int32_t num_reqs, int32_t heads, int32_t budget, int32_t sink, int32_t recent, int32_t *d_keep,
                    int32_t *d_new_len, void *stream) {
    if (num_layers <= 0 || num_reqs < 0 || heads <= 0 || budget <= 0 || sink < 0 || recent < 0 || weight_stride < 0)
        return KV_EINVAL;
    if ((int64_t)sink + recent > budget || weight_stride > INT32_MAX) return KV_EINVAL;
    if (num_reqs > 0 && ((!d_weights && weight_stride > 0) || !d_len || !d_keep || !d_new_len)) return KV_EINVAL;
    if (((uintptr_t)d_weights & 3u) || ((uintptr_t)d_len & 3u) || ((uintptr_t)d_keep & 3u) || ((uintptr_t)d_new_len & 3u))
        return KV_EALIGN;
    const int64_t rows = (int64_t)num_layers * num_reqs;
    if (rows >= (int64_t(1) << 31) / heads) return KV_ELIMIT;
    if (num_reqs == 0) return KV_OK;
    const tkv::SelectParams p = {d_weights, d_len, d_keep, d_new_len, weight_stride, num_reqs, heads, budget, sink, recent};
    (void)hipGetLastError();
    hipLaunchKernelGGL(tkv::evict_select_kernel, dim3((unsigned)(rows * heads)), dim3(tkv::kThreads), 0,
                       (hipStream_t)stream, p);
    return hipGetLastError() == hipSuccess ? KV_OK : KV_EHIP;
}

int kv_evict_compact(const kv_layout *layout, void *const *h_layer_ptrs, const int32_t *d_block_tables,
                     int32_t bt_stride, int32_t num_reqs, int32_t heads, const int32_t *d_keep, int32_t budget,
                     const int32_t *d_new_len, float *d_weights, int64_t weight_stride, void *stream) {
    int rc = tkv::check_layout(layout);
    if (rc == KV_OK) rc = tkv::check_span(layout);
    if (rc != KV_OK) return rc;
    if (!h_layer_ptrs || bt_stride <= 0 || num_reqs < 0 || budget <= 0 || (heads != 1 && heads != layout->kv_heads))
        return KV_EINVAL;
    if (num_reqs > 0 && (!d_block_tables || !d_keep || !d_new_len || (d_weights && weight_stride < 0))) return KV_EINVAL;
    if ((int64_t)layout->head_dim * layout->elem_bytes % 16 != 0 || ((uintptr_t)d_block_tables & 3u) ||
        ((uintptr_t)d_keep & 3u) || ((uintptr_t)d_new_len & 3u) || ((uintptr_t)d_weights & 3u))
        return KV_EALIGN;
    tkv::CompactParams p;
    for (int l = 0; l < layout->num_layers; ++l) {
        if (!h_layer_ptrs[l]) return KV_EINVAL;
        if ((uintptr_t)h_layer_ptrs[l] & 15u) return KV_EALIGN;
        p.layers[l] = (char *)h_layer_ptrs[l];
    }
    const int64_t rows = (int64_t)layout->num_layers * num_reqs;
    if (rows >= (int64_t(1) << 30) / heads) return KV_ELIMIT;
    if (num_reqs == 0) return KV_OK;
    kv_batch b = {};
    b.num_reqs = num_reqs;
    b.bt_stride = bt_stride;
    b.d_block_tables = d_block_tables;
    p.cache = tkv::make_paged(layout, nullptr, &b);
    p.keep = d_keep;
    p.new_len = d_new_len;
    p.weights = d_weights;
    p.weight_stride = weight_stride;
    p.num_layers = layout->num_layers;
    p.heads = heads;
    p.kv_heads = layout->kv_heads;
    p.budget = budget;
    p.vecs = p.cache.head_bytes / 16 * (heads == 1 ? layout->kv_heads : 1);
    (void)hipGetLastError();
    hipLaunchKernelGGL(tkv::evict_compact_kernel, dim3((unsigned)(rows * heads * 2)), dim3(tkv::kThreads), 0,
                       (hipStream_t)stream, p);
    return hipGetLastError() == hipSuccess ? KV_OK : KV_EHIP;
}

}  // extern "C"
