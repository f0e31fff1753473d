// weights.hip -- attention weight that cached tokens received, accumulated.
//
// W[h][j] = decay W[h][j] + sum over rows i that see j of exp(s_ij - lse_i).
// With lse known nothing depends on other keys, so a workgroup owns the sums
// of some keys of one KV head and passes the request's rows, with no atomics.
// S = Q K^T leaves a lane with one key (lane % 32) and 16 of 32 rows, so that
// the sum over rows stays in the lane: one register a key.

#include <math.h>

#include "mfma.h"
#include "paged.h"

namespace tkv {
namespace {

constexpr int kWaves = 4;
constexpr int kThreads = 64 * kWaves;
constexpr int kWaveKeys = 64;               // keys of a wave, held as matrix operands in registers
constexpr float kLog2e = 1.44269504088896340736f;

struct WeightParams {
    Paged cache;
    const char *q;
    int64_t q_ts, q_hs;    // bytes
    const float *lse;
    const float *k_scale;
    float *weights;
    int64_t weight_stride;
    float scale, decay;    // scale times log2 e
    Divider by_group;
    int32_t q_heads, kv_heads, group, head_dim;
    int32_t window;
    bool causal;
};

// What a staged row is to its keys: those it sees, lo <= j < hi, and its
// lse in units of log 2.
struct __align__(16) RowInfo {
    float base[32];
    int lo[32], hi[32];
};

template <int DP> constexpr int kQueryRow = DP * 2 + 16;     // bytes of an LDS row: 8 rows on different banks

// The four waves take KW groups of 64 keys and 4 / KW groups of 32 rows at a
// time; the rows go through LDS, one step ahead, for all of them.  Chunks of
// 1,000 tokens over 4,000 in 4 requests, 32 heads on 8 of 128, 115 GFLOP in 168 to
// 176 us (650 to 680 TFLOP/s).  A wave's products and exponentials take turns,
// with two waves on each SIMD to overlap them: the matrix units are busy for 27 %
// of the time, the vector units for 44 %.  And all 512 workgroups run at once,
// those of the last quarter of the keys with half the rows.
template <class T, bool F8, int DP, int KW>
__global__ __launch_bounds__(kThreads, DP > 128 ? 1 : 2) void attention_weights_kernel(WeightParams p) {
    constexpr int KS = DP / 16, RW = kWaves / KW, RT = KW > 1 ? 2 : 1, kRows = 32 * RW * RT, VPR = DP / 8, VL = kRows * VPR / kThreads;
    constexpr int kKeys = kWaveKeys * KW;
    __shared__ __align__(16) char rows[2][kRows * kQueryRow<DP>];
    __shared__ RowInfo info[2][RW * RT];
    __shared__ float parts[kWaves][kWaveKeys];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, col = lane & 31, half = lane >> 5;
    const int kw = wave % KW, rw = wave / KW;
    const int h = (int)(blockIdx.x % p.kv_heads), r = (int)(blockIdx.x / p.kv_heads);
    const int len_raw = min(max(p.cache.kv_len[r], 0), kMaxLength);
    const int64_t first = clamp_row(p.cache, p.cache.q_off[r]);
    const int ntok = (int)max((int64_t)0, clamp_row(p.cache, p.cache.q_off[r + 1]) - first);
    const int64_t len = min((int64_t)len_raw, p.weight_stride), ahead = len_raw - ntok;
    const float c = p.scale * (F8 && p.k_scale ? p.k_scale[h] : 1.0f);
    float *out = p.weights + ((int64_t)r * p.kv_heads + h) * p.weight_stride;

    for (int64_t tile = blockIdx.y; tile * kKeys < len; tile += gridDim.y) {
        const int tile0 = (int)tile * kKeys, t0 = tile0 + kw * kWaveKeys;      // t0 + 63 may pass 2^31 - 1: no key is there
        // this lane's two keys, as operands; the element order follows the rows'
        u32x4 kf[2][KS];
        bool there[2];
        uint64_t all = ~uint64_t(0);
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            const int64_t t = (int64_t)t0 + x * 32 + col;
            uint32_t row = 0;
            const int32_t blk = t < len ? block_of(p.cache, r, (uint32_t)t, row) : -1;
            there[x] = blk >= 0;
            all &= __ballot(there[x]);
            const char *at = p.cache.layer + (int64_t)h * p.cache.head_bytes +
                             ((int64_t)(blk < 0 ? 0u : (uint32_t)blk * p.cache.block16 + row * p.cache.row16) << 4);
            if constexpr (F8) {
                // 16 elements at a time: a lane holds other elements than in order, as the rows are read below
#pragma unroll
                for (int ks = 0; ks < KS; ks += 2) {
                    const int d = ks * 16 + half * 16;
                    const u32x4 y = d < p.head_dim ? *(const u32x4 *)(at + d) : u32x4{0, 0, 0, 0};
                    kf[x][ks] = unpack8<T>(y[0], y[1]);
                    kf[x][ks + 1] = unpack8<T>(y[2], y[3]);
                }
            } else {
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) {
                    const int d = ks * 16 + half * 8;
                    kf[x][ks] = d < p.head_dim ? *(const u32x4 *)(at + d * 2) : u32x4{0, 0, 0, 0};
                }
            }
        }
        // rows that may see a key of the tile: from the token at its first key on (causal), to the one whose window
        // ends at its last key
        int tok0 = 0, tok1 = ntok;
        if (p.causal) tok0 = (int)min((int64_t)ntok, max((int64_t)0, (int64_t)tile0 - ahead));
        if (p.window > 0) tok1 = (int)max((int64_t)0, min((int64_t)ntok, (int64_t)tile0 + kKeys - 1 + p.window - ahead));
        const int row_begin = tok0 * p.group, row_end = tok1 * p.group;

        u32x4 qreg[VL];
        float base = 0.0f;
        int lo = 0, hi = 0;
        const auto load = [&](int row0) {
#pragma unroll
            for (int i = 0; i < VL; ++i) {
                const int x = i * kThreads + tid, vec = x % VPR;
                const int row = row0 + x / VPR;
                qreg[i] = u32x4{0, 0, 0, 0};
                if (row < row_end && vec * 8 < p.head_dim) {
                    const int token = (int)divide(row, p.by_group), head = h * p.group + row - token * p.group;
                    qreg[i] = *(const u32x4 *)(p.q + (first + token) * p.q_ts + head * p.q_hs + vec * 16);
                }
            }
            if (tid < kRows) {
                const int row = row0 + tid, token = (int)divide(row, p.by_group);
                base = lo = hi = 0;
                if (row < row_end) {
                    base = p.lse[(first + token) * p.q_heads + h * p.group + row - token * p.group];
                    const int64_t pos = ahead + token;
                    if (base != -INFINITY) hi = (int)max((int64_t)0, p.causal ? min(len, pos + 1) : len);
                    else base = 0.0f;
                    lo = (int)(p.window > 0 ? max((int64_t)0, pos - p.window + 1) : 0);
                }
            }
        };
        const auto stage = [&](int buf) {
#pragma unroll
            for (int i = 0; i < VL; ++i) {
                const int x = i * kThreads + tid;
                *(u32x4 *)(rows[buf] + x / VPR * kQueryRow<DP> + x % VPR * 16) = qreg[i];
            }
            if (tid < kRows) {
                info[buf][tid / 32].base[tid % 32] = base * kLog2e;
                info[buf][tid / 32].lo[tid % 32] = lo;
                info[buf][tid / 32].hi[tid % 32] = hi;
            }
        };
        float sum[2] = {0.0f, 0.0f};
        if (row_begin < row_end) load(row_begin);
        int buf = 0;
        for (int row0 = row_begin; row0 < row_end; row0 += kRows, buf ^= 1) {
            stage(buf);
            __syncthreads();
            if (row0 + kRows < row_end) load(row0 + kRows);
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) {
                const int rg = rw * RT + rt;
                if (row0 + rg * 32 >= row_end) continue;
                const char *at = rows[buf] + (rg * 32 + col) * kQueryRow<DP>;
                const RowInfo &y = info[buf][rg];
                u32x4 qf[KS];
                f32x4 b[4];
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) {
                    const int d = F8 ? (ks / 2) * 32 + half * 16 + (ks & 1) * 8 : ks * 16 + half * 8;
                    qf[ks] = *(const u32x4 *)(at + d * 2);
                }
#pragma unroll
                for (int g = 0; g < 4; ++g) b[g] = *(const f32x4 *)&y.base[g * 8 + half * 4];
                // whether every row sees every key of the wave
                const bool whole = __all(y.lo[col] <= t0 && y.hi[col] >= t0 + kWaveKeys) && all == ~uint64_t(0);
                __builtin_amdgcn_sched_barrier(0);     // all reads are on their way before the first product waits
                f32x16 s[2];
#pragma unroll
                for (int x = 0; x < 2; ++x)
#pragma unroll
                    for (int e = 0; e < 16; ++e) s[x][e] = 0.0f;
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) {
                    s[0] = T::mfma32(qf[ks], kf[0][ks], s[0]);
                    s[1] = T::mfma32(qf[ks], kf[1][ks], s[1]);
                }
                float part[2] = {0.0f, 0.0f};          // of these rows, so that long sums stay exact
                if (whole) {
#pragma unroll
                    for (int g = 0; g < 16; ++g)
#pragma unroll
                        for (int x = 0; x < 2; ++x) part[x] += exp2_(__builtin_fmaf(s[x][g], c, -b[g / 4][g % 4]));
                } else {
#pragma unroll
                    for (int g = 0; g < 16; g += 4) {
                        const i32x4 l = *(const i32x4 *)&y.lo[g * 2 + half * 4], u = *(const i32x4 *)&y.hi[g * 2 + half * 4];
#pragma unroll
                        for (int e = 0; e < 4; ++e)
#pragma unroll
                            for (int x = 0; x < 2; ++x) {
                                const int t = t0 + x * 32 + col;
                                const float v = exp2_(__builtin_fmaf(s[x][g + e], c, -b[g / 4][e]));
                                part[x] += there[x] && t >= l[e] && t < u[e] ? v : 0.0f;
                            }
                    }
                }
                sum[0] += part[0];
                sum[1] += part[1];
            }
        }
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            const f32x2 y = both_halves(sum[x]);
            sum[x] = y[0] + y[1];
        }
        // lane i has the sum of key 32 x + i % 32 in sum[x]
        float got = half ? sum[1] : sum[0];
        if constexpr (RW > 1) {
            parts[wave][lane] = got;
            __syncthreads();
            if (rw == 0)
#pragma unroll
                for (int i = 1; i < RW; ++i) got += parts[i * KW + kw][lane];
            __syncthreads();
        } else {
            __syncthreads();      // the rows' buffers are free for the next tile
        }
        const int64_t key = (int64_t)t0 + lane;
        if (rw == 0 && key < len) out[key] = p.decay == 0.0f ? got : __builtin_fmaf(p.decay, out[key], got);
    }
}

// Few rows (a decoded token's heads): nothing to share, so that each wave works
// alone on 64 keys, 16 rows at a time, and all its loads are on their way at
// once.  A lane has one key (lane % 16) and 4 of 16 rows.  Bound by the reads of
// K: 64 requests of 4,096 tokens, 8 KV heads of 128, 0.54 GB in 123 us (4.5
// TB/s).  Keys loaded as half cache lines, without the exchange of columns,
// take 31 against 28.7 us for 32 requests of 4,000 at head size 64, 48 against
// 42 us at 80 and 96, 124.8 us where 128 takes 125.4.
template <class T, bool F8, int DP>
__global__ __launch_bounds__(kThreads) void attention_weights_few_kernel(WeightParams p) {
    constexpr int KS = DP / 32, LD = F8 ? KS / 2 : KS, KT = kWaveKeys / 16;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = lane & 15, quad = lane >> 4;
    const int h = (int)(blockIdx.x % p.kv_heads), r = (int)(blockIdx.x / p.kv_heads);
    const int len_raw = min(max(p.cache.kv_len[r], 0), kMaxLength);
    const int64_t first = clamp_row(p.cache, p.cache.q_off[r]);
    const int ntok = (int)max((int64_t)0, clamp_row(p.cache, p.cache.q_off[r + 1]) - first), nrows = ntok * p.group;
    const int64_t len = min((int64_t)len_raw, p.weight_stride), ahead = len_raw - ntok;
    const float c = p.scale * (F8 && p.k_scale ? p.k_scale[h] : 1.0f);
    float *out = p.weights + ((int64_t)r * p.kv_heads + h) * p.weight_stride;

    for (int64_t tile = (int64_t)blockIdx.y * kWaves + wave; tile * kWaveKeys < len; tile += (int64_t)gridDim.y * kWaves) {
        const int t0 = (int)tile * kWaveKeys;
        uint32_t row = 0;
        const int32_t blk = t0 + lane < len ? block_of(p.cache, r, (uint32_t)(t0 + lane), row) : -1;
        const uint64_t there = __ballot(blk >= 0);
        const uint32_t off = blk < 0 ? 0u : (uint32_t)blk * p.cache.block16 + row * p.cache.row16;
        const float old = p.decay != 0.0f && t0 + lane < len ? out[t0 + lane] : 0.0f;
        u32x4 kf[KT][LD];
#pragma unroll
        for (int x = 0; x < KT; ++x)
            load_rows(kf[x], p.cache.head_bytes, [&](int row) {
                return p.cache.layer + (int64_t)h * p.cache.head_bytes + ((int64_t)(uint32_t)__shfl((int)off, x * 16 + row) << 4);
            });
        bool arranged = false;
        float sum[KT];
#pragma unroll
        for (int x = 0; x < KT; ++x) sum[x] = 0.0f;
        for (int row0 = 0; row0 < nrows; row0 += 16) {
            const int mine = min(row0 + col, nrows - 1), token = (int)divide(mine, p.by_group);
            const char *qat = p.q + (first + token) * p.q_ts + (int64_t)(h * p.group + mine - token * p.group) * p.q_hs;
            u32x4 qf[KS];
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                const int d = F8 ? (ks / 2) * 64 + quad * 16 + (ks & 1) * 8 : ks * 32 + quad * 8;
                qf[ks] = d < p.head_dim ? *(const u32x4 *)(qat + d * 2) : u32x4{0, 0, 0, 0};
            }
            // this lane's four rows of the result
            float base[4];
            int lo[4], hi[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int rr = row0 + quad * 4 + i, tok = (int)divide(min(rr, nrows - 1), p.by_group);
                const float lse = p.lse[(first + tok) * p.q_heads + h * p.group + min(rr, nrows - 1) - tok * p.group];
                const int64_t pos = ahead + tok;
                const bool on = rr < nrows && lse != -INFINITY;
                base[i] = on ? lse * kLog2e : 0.0f;
                hi[i] = on ? (int)max((int64_t)0, p.causal ? min(len, pos + 1) : len) : 0;
                lo[i] = (int)(p.window > 0 ? max((int64_t)0, pos - p.window + 1) : 0);
            }
            if (!arranged) {                   // here, so that the rows above are on their way with the keys
#pragma unroll
                for (int x = 0; x < KT; ++x) arrange_rows(kf[x]);
                arranged = true;
            }
#pragma unroll
            for (int x = 0; x < KT; ++x) {
                f32x4 s = {0, 0, 0, 0};
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) {
                    if constexpr (F8) s = T::mfma16(qf[ks], unpack8<T>(kf[x][ks / 2][ks % 2 * 2], kf[x][ks / 2][ks % 2 * 2 + 1]), s);
                    else s = T::mfma16(qf[ks], kf[x][ks], s);
                }
                const int t = t0 + x * 16 + col;
                const bool in = (there >> (x * 16 + col)) & 1;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float v = exp2_(__builtin_fmaf(s[i], c, -base[i]));
                    sum[x] += in && t >= lo[i] && t < hi[i] ? v : 0.0f;
                }
            }
        }
        // over the four groups of rows; lane i then takes key i
        float got = 0.0f;
#pragma unroll
        for (int x = 0; x < KT; ++x) {
            float y = sum[x];
            y += __shfl_xor(y, 16);
            const f32x2 z = both_halves(y);
            got = quad == x ? z[0] + z[1] : got;
        }
        if (t0 + lane < len) out[t0 + lane] = p.decay == 0.0f ? got : __builtin_fmaf(p.decay, old, got);
    }
}

template <class T, bool F8> void (*weights_few_kernel(int head_dim))(WeightParams) {
    if (head_dim <= 64) return attention_weights_few_kernel<T, F8, 64>;
    if constexpr (!F8) {
        if (head_dim <= 96) return attention_weights_few_kernel<T, F8, 96>;
    }
    if (head_dim <= 128) return attention_weights_few_kernel<T, F8, 128>;
    return attention_weights_few_kernel<T, F8, 256>;
}

template <class T, bool F8, int KW> void (*weights_kernel(int head_dim))(WeightParams) {
    if (head_dim <= 64) return attention_weights_kernel<T, F8, 64, KW>;
    if (head_dim <= 96) return attention_weights_kernel<T, F8, 96, KW>;
    if (head_dim <= 128) return attention_weights_kernel<T, F8, 128, KW>;
    return attention_weights_kernel<T, F8, 256, KW>;
}

template <int KW> auto weights_kernel(bool bf16, bool f8, int d) {
    return bf16 ? (f8 ? weights_kernel<Bf16, true, KW>(d) : weights_kernel<Bf16, false, KW>(d))
                : (f8 ? weights_kernel<F16, true, KW>(d) : weights_kernel<F16, false, KW>(d));
}

}  // namespace
}  // namespace tkv

extern "C" {

int kv_attention_weights(const kv_layout *layout, const void *d_layer, const kv_batch *batch, const kv_rows *q,
                         const float *d_lse, float scale, int32_t causal, int32_t window, int32_t cache_dtype,
                         const float *d_k_scale, float decay, float *d_weights, int64_t weight_stride, void *stream) {
    int rc = tkv::check_cache(layout, cache_dtype);
    if (rc == KV_OK) rc = tkv::check_batch(batch);
    if (rc == KV_OK) rc = tkv::check_rows(q, batch->num_q, layout->head_dim, false);
    if (rc != KV_OK) return rc;
    if (!d_layer || weight_stride < 0 || window < 0 || q->heads % layout->kv_heads != 0) return KV_EINVAL;
    if (cache_dtype != KV_F8E4M3 && cache_dtype != q->dtype) return KV_EINVAL;
    if (!(scale > 0.0f) || !isfinite(scale) || !isfinite(decay)) return KV_EINVAL;
    if (batch->num_reqs > 0 && weight_stride > 0 &&
        (!d_weights || !batch->d_q_off || !batch->d_kv_len || !batch->d_block_tables))
        return KV_EINVAL;
    if (batch->num_q > 0 && !d_lse) return KV_EINVAL;
    if (((uintptr_t)d_layer & 15u) || ((uintptr_t)d_lse & 3u) || ((uintptr_t)d_weights & 3u)) return KV_EALIGN;
    if (batch->num_reqs == 0 || weight_stride == 0) return KV_OK;
    if ((int64_t)batch->num_reqs * layout->kv_heads >= (int64_t(1) << 31)) return KV_ELIMIT;
    if (batch->num_q >= (int64_t(1) << 30) / q->heads) return KV_ELIMIT;
    tkv::WeightParams p;
    p.cache = tkv::make_paged(layout, d_layer, batch);
    p.q = (const char *)q->d_data;
    p.q_ts = q->token_stride * 2, p.q_hs = q->head_stride * 2;
    p.lse = d_lse;
    p.k_scale = cache_dtype == KV_F8E4M3 ? d_k_scale : nullptr;
    p.weights = d_weights;
    p.weight_stride = weight_stride;
    p.scale = scale * tkv::kLog2e;
    p.decay = decay;
    p.q_heads = q->heads;
    p.kv_heads = layout->kv_heads;
    p.group = q->heads / layout->kv_heads;
    p.by_group = tkv::make_divider((uint32_t)p.group);
    p.head_dim = layout->head_dim;
    p.window = window < tkv::kMaxLength ? window : 0;
    p.causal = causal != 0;
    // Keys of a workgroup: 256, each wave 64 of its own, or 64, with the waves sharing the rows, where that is needed to
    // give each compute unit two workgroups.  Up to 16 rows take a kernel of their own.
    const int64_t heads = (int64_t)batch->num_reqs * layout->kv_heads;
    const bool few = (int64_t)batch->max_q_len * p.group <= 16;
    const bool share = !few && heads * ((batch->max_kv_len + 255) / 256) < 512;
    const int keys = share ? 64 : 256, d = layout->head_dim;
    const bool bf16 = q->dtype == KV_BF16, f8 = cache_dtype == KV_F8E4M3;
    auto kernel = few ? (bf16 ? (f8 ? tkv::weights_few_kernel<tkv::Bf16, true>(d) : tkv::weights_few_kernel<tkv::Bf16, false>(d))
                              : (f8 ? tkv::weights_few_kernel<tkv::F16, true>(d) : tkv::weights_few_kernel<tkv::F16, false>(d)))
                      : (share ? tkv::weights_kernel<1>(bf16, f8, d) : tkv::weights_kernel<4>(bf16, f8, d));
    int64_t tiles = ((int64_t)batch->max_kv_len + keys - 1) / keys;
    tiles = tiles < 1 ? 1 : (tiles > 65535 ? 65535 : tiles);
    (void)hipGetLastError();
    hipLaunchKernelGGL(kernel, dim3((unsigned)heads, (unsigned)tiles),
                       dim3(tkv::kThreads), 0, (hipStream_t)stream, p);
    return hipGetLastError() == hipSuccess ? KV_OK : KV_EHIP;
}

}  // extern "C"
