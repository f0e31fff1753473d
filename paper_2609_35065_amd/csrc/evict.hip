// evict.hip -- which cached tokens to keep, and moving them to the front.
//
// Selection.  A row of weights is mapped to 32-bit keys in the order of the
// numbers (NaN lowest, -0 as +0, what is kept in any case above all).  The
// smallest key that is kept, and how many of the tokens at exactly that key,
// follow from counts of 10, 11 and 11 bits, from the top down.  Weights share
// few exponents and have ties, so each bin is counted in eight or four copies,
// by lane.  Each wave owns a stretch of the row, so that after one
// exchange of counts the kept indices come out in order without another.
//
// Compaction.  Row keep[i] >= i moves to row i, in place: what a tile of rows
// writes (rows below its end) no later tile reads, so that a tile may be
// written once its own reads and those before it are on their way.  One
// workgroup takes a head's rows of a plane (or a slice of their bytes) in
// order; heads, planes, layers and requests are independent.

#include <math.h>

#include <type_traits>

#include "paged.h"

namespace tkv {
namespace {

constexpr int kThreads = 256;            // of a compaction
constexpr int kWords = 8192;               // of a count: bins times copies

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

// Sum over the lanes before this one in the workgroup.
template <int WAVES> __device__ __forceinline__ int prefix(int x, int *scratch) {
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
#pragma unroll
    for (int w = 0; w < WAVES; ++w)
        if (w < wave) before += scratch[w];
    return before + y - x;
}

// One workgroup a row.  ITEMS > 0: the row has at most ITEMS * THREADS
// tokens and is read once, into registers; 0: any length, read again from the
// caches in each pass.  Reading is an eighth of it: 8 ragged requests around 4,096
// tokens (2,048 rows, 46 MB) take 62 us, 32 layers x 8 heads of 1,001 tokens 9.4
// us.  Vector instructions are busy for 48 % of that, LDS for 26 % (a third of it
// conflicts between lanes that count one bin); the rest are the waits between the
// passes, which depend on one another.
template <int THREADS, int ITEMS>
__global__ __launch_bounds__(THREADS, THREADS == 256 ? 4 : 6) void evict_select_kernel(SelectParams p) {
    constexpr int kWaves = THREADS / 64, kBatch = 8;          // loads on their way together
    __shared__ __align__(16) int hist[kWords];
    __shared__ int scratch[kWaves], above[kWaves], level[kWaves];
    __shared__ int found[2];               // the bin, and how many are still to be taken from it
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int64_t g = blockIdx.x;          // (layer * num_reqs + request) * heads + head
    const int r = (int)(g / p.heads % p.num_reqs);
    const int32_t raw = p.len[r];
    const int n = (int)min((int64_t)(raw < 0 ? 0 : raw), p.weight_stride);
    const int m = min(n, p.budget);
    int32_t *keep = p.keep + g * p.budget;
    if (g < (int64_t)p.num_reqs * p.heads && g % p.heads == 0 && tid == 0) p.new_len[r] = m;
    for (int i = m + tid; i < p.budget; i += THREADS) keep[i] = -1;
    if (n <= p.budget) {
        for (int i = tid; i < n; i += THREADS) keep[i] = i;
        return;
    }
    const float *w = p.weights + g * p.weight_stride;
    const int lo = p.sink, hi = n - p.recent;                 // candidates
    // (what lies past the end has the lowest key and the highest indices: it is never among `budget` < n)
    const auto key_of = [&](int i) { return i >= n ? 0u : (i < lo || i >= hi ? 0xffffffffu : ordered(w[i])); };
    // this wave's stretch, 64 tokens at a time
    const int rounds = (n + THREADS - 1) / THREADS, start = wave * rounds * 64 + lane;
    uint32_t mine[ITEMS > 0 ? ITEMS : 1];
    if constexpr (ITEMS > 0) {
#pragma unroll
        for (int x = 0; x < ITEMS; ++x) mine[x] = x < rounds ? key_of(start + x * 64) : 0u;
    }
    const auto each = [&](auto body) {     // body(index, key) over the stretch; uniform in the wave
        if constexpr (ITEMS > 0) {
#pragma unroll
            for (int x = 0; x < ITEMS; ++x)
                if (x < rounds) body(start + x * 64, mine[x]);
        } else {
            for (int x0 = 0; x0 < rounds; x0 += kBatch) {
                uint32_t k[kBatch];
#pragma unroll
                for (int x = 0; x < kBatch; ++x) k[x] = x0 + x < rounds ? key_of(start + (x0 + x) * 64) : 0u;
#pragma unroll
                for (int x = 0; x < kBatch; ++x)
                    if (x0 + x < rounds) body(start + (x0 + x) * 64, k[x]);
            }
        }
    };
    int want = p.budget;
    uint32_t known = 0, mask = 0;
    // one count: the keys that agree with `known` so far, by their next bits
    const auto count = [&](auto shift_, auto bits_) {
        constexpr int shift = shift_, bins = 1 << bits_, copies = kWords / bins, per = (bins + THREADS - 1) / THREADS;
        for (int i = tid; i < kWords / 4; i += THREADS) ((i32x4 *)hist)[i] = i32x4{0, 0, 0, 0};
        __syncthreads();
        int *const own = hist + (lane & (copies - 1));
        each([&](int, uint32_t k) {
            if ((k & mask) == known) atomicAdd(own + ((k >> shift) & (bins - 1)) * copies, 1);
        });
        __syncthreads();
        // from the top bin down: where the wanted number is reached
        int c[per], sum = 0;
#pragma unroll
        for (int i = 0; i < per; ++i) {
            const int bin = bins - 1 - (tid * per + i);
            c[i] = 0;
            if (bin >= 0)
#pragma unroll
                for (int y = 0; y < copies; y += 4) {
                    const i32x4 z = *(const i32x4 *)(hist + bin * copies + y);
                    c[i] += (z[0] + z[1]) + (z[2] + z[3]);
                }
            sum += c[i];
        }
        int before = prefix<kWaves>(sum, scratch);
#pragma unroll
        for (int i = 0; i < per; ++i) {
            if (before < want && before + c[i] >= want) {
                found[0] = bins - 1 - (tid * per + i);
                found[1] = want - before;
            }
            before += c[i];
        }
        __syncthreads();
        known |= (uint32_t)found[0] << shift;
        mask |= (uint32_t)(bins - 1) << shift;
        want = found[1];
    };
    count(std::integral_constant<int, 22>{}, std::integral_constant<int, 10>{});
    count(std::integral_constant<int, 11>{}, std::integral_constant<int, 11>{});
    count(std::integral_constant<int, 0>{}, std::integral_constant<int, 11>{});
    // kept: above `known`, and the first `want` at it
    int over = 0, ties = 0;
    each([&](int, uint32_t k) {
        over += __popcll(__ballot(k > known));
        ties += __popcll(__ballot(k == known));
    });
    if (lane == 0) {
        above[wave] = over;
        level[wave] = ties;
    }
    __syncthreads();
    int at = 0, tied = 0;                  // kept, and met at the level, before this wave's stretch
    for (int x = 0; x < wave; ++x) {
        at += above[x];
        tied += level[x];
    }
    at += min(tied, want);
    const auto lanes_below = [](uint64_t x) { return (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(x >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)x, 0)); };
    each([&](int i, uint32_t k) {
        const uint64_t level_mask = __ballot(k == known);
        bool kept = k > known;
        if (level_mask) {
            if (k == known) kept = tied + lanes_below(level_mask) < want;
            tied += __popcll(level_mask);
        }
        const uint64_t kept_mask = __ballot(kept);
        if (kept) keep[at + lanes_below(kept_mask)] = i;
        at += __popcll(kept_mask);
    });
}

struct CompactParams {
    Paged cache;
    char *layers[KV_MAX_LAYERS];
    const int32_t *keep, *new_len;
    float *weights;
    int64_t weight_stride;
    Divider by_vecs;
    int32_t heads, budget;
    int32_t vecs;          // 16-byte vectors of a row's slice: a head's row, or all heads', or a part
    int32_t slices;
};

constexpr int kMoves = 2048;               // rows whose places are looked up at a time
constexpr int kAhead = 4;                  // vectors of a lane in a tile

// One workgroup: a (layer, request, head, plane, slice).  A row already in its
// place is neither read nor written.  Bound by memory, and by the two barriers
// of a tile, at which its workgroup has only the next tile's reads on their way:
// 8 ragged requests around 4,096 tokens, 32 layers, a quarter kept, 2.16 GB read
// and written in 458 us (4.7 TB/s) where nearly all kept rows move; 1,001 tokens,
// half kept, 0.13 GB in 30 us (4.4 TB/s).
__global__ __launch_bounds__(kThreads) void evict_compact_kernel(CompactParams p) {
    __shared__ uint32_t from[kMoves], to[kMoves];      // 16-byte units from the plane's start; from = to: no move
    const int tid = threadIdx.x;
    uint32_t x = blockIdx.x;
    const int plane = (int)(x & 1);
    x >>= 1;
    const int slice = (int)(x % p.slices);
    const int64_t g = x / p.slices;                    // (layer * num_reqs + request) * heads + head
    const int h = (int)(g % p.heads), r = (int)(g / p.heads % p.cache.num_reqs), l = (int)(g / p.heads / p.cache.num_reqs);
    const int n = min(max(p.new_len[r], 0), p.budget);
    const int32_t *keep = p.keep + g * p.budget;
    char *base = p.layers[l] + plane * p.cache.kv_stride + (int64_t)h * p.cache.head_bytes + (int64_t)slice * p.vecs * 16;
    const bool with_weights = plane == 0 && slice == 0 && p.weights;
    float *w = p.weights + g * p.weight_stride;
    for (int row0 = 0; row0 < n; row0 += kMoves) {
        const int rows = min(kMoves, n - row0);
        __syncthreads();                   // the chunk before is read
        for (int i = tid; i < rows; i += kThreads) {
            const int32_t src = keep[row0 + i];
            uint32_t a = 0, b = 0, ra, rb;
            if (src > row0 + i) {
                const int32_t ida = block_of(p.cache, r, (uint32_t)src, ra), idb = block_of(p.cache, r, (uint32_t)(row0 + i), rb);
                if (ida >= 0 && idb >= 0) {
                    a = (uint32_t)ida * p.cache.block16 + ra * p.cache.row16;
                    b = (uint32_t)idb * p.cache.block16 + rb * p.cache.row16;
                }
            }
            from[i] = a;
            to[i] = b;
        }
        if (with_weights)                  // (a lane's places are those that it looked up above)
            for (int at = 0; at < rows; at += kThreads) {
                const int i = row0 + at + tid;
                const int32_t src = at + tid < rows && from[at + tid] != to[at + tid] ? keep[i] : -1;
                const bool moves = src > i && src < p.weight_stride;
                const float y = moves ? w[src] : 0.0f;
                __syncthreads();
                if (moves) w[i] = y;
            }
        __syncthreads();
        // tiles of kAhead * kThreads vectors: the next one's are read before this one's are written
        const int total = rows * p.vecs;   // at most 2,048 * 2^15
        u32x4 y[kAhead], z[kAhead];
        const auto read = [&](int at, u32x4 *v) {
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                const int e = at + i * kThreads + tid, row = (int)divide(min(e, total - 1), p.by_vecs);
                if (e < total && from[row] != to[row])
                    v[i] = *(const u32x4 *)(base + ((int64_t)from[row] + e - row * p.vecs) * 16);
            }
        };
        const auto write = [&](int at, const u32x4 *v) {
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                const int e = at + i * kThreads + tid, row = (int)divide(min(e, total - 1), p.by_vecs);
                if (e < total && from[row] != to[row])
                    *(u32x4 *)(base + ((int64_t)to[row] + e - row * p.vecs) * 16) = v[i];
            }
        };
        constexpr int kTile = kAhead * kThreads;
        read(0, y);
        for (int at = 0; at < total; at += 2 * kTile) {
            if (at + kTile < total) read(at + kTile, z);
            __syncthreads();
            write(at, y);
            if (at + 2 * kTile < total) read(at + 2 * kTile, y);
            __syncthreads();
            if (at + kTile < total) write(at + kTile, z);
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
    if (rows >= (int64_t(1) << 31) / heads || weight_stride > (int64_t(1) << 30)) return KV_ELIMIT;   // indices and rounds in 32 bits
    if (num_reqs == 0) return KV_OK;
    const tkv::SelectParams p = {d_weights, d_len, d_keep, d_new_len, weight_stride, num_reqs, heads, budget, sink, recent};
    (void)hipGetLastError();
    // Rows of up to 4,096 and 16,384 tokens stay in registers.
    const int threads = weight_stride <= 4096 ? 256 : 512;
    auto kernel = threads == 256 ? tkv::evict_select_kernel<256, 16>
                                 : (weight_stride <= 16384 ? tkv::evict_select_kernel<512, 32> : tkv::evict_select_kernel<512, 0>);
    hipLaunchKernelGGL(kernel, dim3((unsigned)(rows * heads)), dim3(threads), 0, (hipStream_t)stream, p);
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
    p.heads = heads;
    p.budget = budget;
    p.vecs = p.cache.head_bytes / 16 * (heads == 1 ? layout->kv_heads : 1);
    // Bytes of a row are independent: where there are few rows' workgroups, slices of at least 64 bytes give each
    // compute unit four.
    p.slices = 1;
    while (rows * heads * 2 * p.slices < 1024 && p.vecs % 2 == 0 && p.vecs >= 8) {
        p.vecs /= 2;
        p.slices *= 2;
    }
    if (p.vecs > 32768 || rows * heads * p.slices >= (int64_t(1) << 30)) return KV_ELIMIT;
    p.by_vecs = tkv::make_divider((uint32_t)p.vecs);
    (void)hipGetLastError();
    hipLaunchKernelGGL(tkv::evict_compact_kernel, dim3((unsigned)(rows * heads * 2 * p.slices)), dim3(tkv::kThreads), 0,
                       (hipStream_t)stream, p);
    return hipGetLastError() == hipSuccess ? KV_OK : KV_EHIP;
}

}  // extern "C"
