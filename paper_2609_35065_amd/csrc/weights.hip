// weights.hip -- attention weight that cached tokens received, accumulated.
//
// W[h][j] = decay W[h][j] + sum over rows i that see j of exp(s_ij - lse_i).
// With lse known nothing depends on other keys, so a workgroup owns 128 keys
// of one KV head, holds them as matrix operands in registers (32 keys a wave)
// and passes the request's rows; a lane's sums stay in its registers and are
// added across lanes once at the end, in a fixed order, with no atomics.

#include <math.h>

#include "mfma.h"
#include "paged.h"

namespace tkv {
namespace {

constexpr int kWaves = 4;
constexpr int kThreads = 64 * kWaves;
constexpr int kKeys = 32 * kWaves;
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
    int32_t q_heads, kv_heads, group, head_dim;
    int32_t window;
    bool causal;
};

template <class T, bool F8, int DP>
__global__ __launch_bounds__(kThreads) void attention_weights_kernel(WeightParams p) {
    constexpr int KS = DP / 16;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = lane & 31, half = lane >> 5;
    const int h = (int)(blockIdx.x % p.kv_heads), r = (int)(blockIdx.x / p.kv_heads);
    const int32_t len_raw = p.cache.kv_len[r];
    const int64_t first = clamp_row(p.cache, p.cache.q_off[r]);
    const int64_t ntok = max((int64_t)0, clamp_row(p.cache, p.cache.q_off[r + 1]) - first), nrows = ntok * p.group;
    const int64_t len = min((int64_t)(len_raw < 0 ? 0 : len_raw), p.weight_stride);
    const float c = p.scale * (F8 && p.k_scale ? p.k_scale[h] : 1.0f);
    float *out = p.weights + ((int64_t)r * p.kv_heads + h) * p.weight_stride;

    for (int64_t tile = blockIdx.y; tile * kKeys < len; tile += gridDim.y) {
        const int64_t t0 = tile * kKeys + wave * 32;
        if (t0 >= len) continue;
        // this lane's key, as an operand row
        const int64_t t = t0 + col;
        uint32_t row = 0;
        const int32_t blk = t < len ? block_of(p.cache, r, (uint32_t)t, row) : -1;
        const uint32_t there = (uint32_t)__ballot(blk >= 0);
        const char *at = p.cache.layer + (int64_t)h * p.cache.head_bytes +
                         ((int64_t)(blk < 0 ? 0u : (uint32_t)blk * p.cache.block16 + row * p.cache.row16) << 4);
        u32x4 kf[KS];
        // an 8-bit cache is loaded 16 elements at a time: lanes hold the head's elements in another order
        if constexpr (F8) {
#pragma unroll
            for (int ks = 0; ks < KS; ks += 2) {
                const int d = ks * 16 + half * 16;
                const u32x4 y = d < p.head_dim ? *(const u32x4 *)(at + d) : u32x4{0, 0, 0, 0};
                kf[ks] = unpack8<T>(y[0], y[1]);
                kf[ks + 1] = unpack8<T>(y[2], y[3]);
            }
        } else {
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                const int d = ks * 16 + half * 8;
                kf[ks] = d < p.head_dim ? *(const u32x4 *)(at + d * 2) : u32x4{0, 0, 0, 0};
            }
        }
        float sum[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) sum[i] = 0.0f;
        // rows that may see one of these keys: from the token at t0 on (causal), to the one whose window ends here
        int64_t tok0 = 0, tok1 = ntok;
        if (p.causal) tok0 = max((int64_t)0, t0 - (len_raw - ntok));
        if (p.window > 0) tok1 = min(ntok, t0 + 31 + p.window - (len_raw - ntok));
        for (int64_t row0 = tok0 * p.group; row0 < tok1 * p.group; row0 += 32) {
            const int64_t myrow = row0 + col;
            const bool have = myrow < nrows;
            const int64_t token = have ? myrow / p.group : 0;
            const int head = h * p.group + (int)(have ? myrow % p.group : 0);
            const char *qat = p.q + (first + token) * p.q_ts + head * p.q_hs;
            f32x16 s;
#pragma unroll
            for (int i = 0; i < 16; ++i) s[i] = 0.0f;
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                const int d = F8 ? (ks / 2) * 32 + half * 16 + (ks & 1) * 8 : ks * 16 + half * 8;
                u32x4 qf = {0, 0, 0, 0};
                if (have && d < p.head_dim) qf = *(const u32x4 *)(qat + d * 2);
                s = T::mfma32(kf[ks], qf, s);
            }
            const float lse = have ? p.lse[(first + token) * p.q_heads + head] : -INFINITY;
            const int64_t pos = len_raw - ntok + token;
            const int64_t hi = !have || lse == -INFINITY ? 0 : (p.causal ? pos + 1 : len);
            const int64_t lo = p.window > 0 ? pos - p.window + 1 : 0;
            const float base = lse * kLog2e;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int k = 8 * (i / 4) + 4 * half + i % 4;
                const bool seen = ((there >> k) & 1) && t0 + k >= lo && t0 + k < hi;
                if (seen) sum[i] += exp2_(__builtin_fmaf(s[i], c, -base));
            }
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) {
#pragma unroll
            for (int x = 1; x < 32; x *= 2) sum[i] += __shfl_xor(sum[i], x);
        }
        // lane 32 half + i writes the key of its sum i
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const int64_t key = t0 + 8 * (i / 4) + 4 * half + i % 4;
            if (col == i && key < len) out[key] = p.decay == 0.0f ? sum[i] : __builtin_fmaf(p.decay, out[key], sum[i]);
        }
    }
}

template <class T, bool F8> void (*weights_kernel(int head_dim))(WeightParams) {
    if (head_dim <= 64) return attention_weights_kernel<T, F8, 64>;
    if (head_dim <= 96) return attention_weights_kernel<T, F8, 96>;
    if (head_dim <= 128) return attention_weights_kernel<T, F8, 128>;
    return attention_weights_kernel<T, F8, 256>;
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
    p.head_dim = layout->head_dim;
    p.window = window;
    p.causal = causal != 0;
    const bool bf16 = q->dtype == KV_BF16, f8 = cache_dtype == KV_F8E4M3;
    const int d = layout->head_dim;
    auto kernel = bf16 ? (f8 ? tkv::weights_kernel<tkv::Bf16, true>(d) : tkv::weights_kernel<tkv::Bf16, false>(d))
                       : (f8 ? tkv::weights_kernel<tkv::F16, true>(d) : tkv::weights_kernel<tkv::F16, false>(d));
    int64_t tiles = ((int64_t)batch->max_kv_len + tkv::kKeys - 1) / tkv::kKeys;
    tiles = tiles < 1 ? 1 : (tiles > 65535 ? 65535 : tiles);
    (void)hipGetLastError();
    hipLaunchKernelGGL(kernel, dim3((unsigned)(batch->num_reqs * layout->kv_heads), (unsigned)tiles),
                       dim3(tkv::kThreads), 0, (hipStream_t)stream, p);
    return hipGetLastError() == hipSuccess ? KV_OK : KV_EHIP;
}

}  // extern "C"
