// rope.hip -- rotary positions and the append to the paged cache.
//
// A row at position p has pair i turned by u = p * f_i:
//     (a, b) -> (a cos u - b sin u, a sin u + b cos u) * magnitude.
// The angle needs more than 32 bits (position 100,000 times 1 radian leaves
// 2^-7 radians of a float's mantissa), so the product and its remainder by a
// turn are formed in 64 bits, once per (token, pair), and shared by all heads.

#include "paged.h"

namespace tkv {
namespace {

constexpr int kThreads = 256;

struct RopeParams {
    Paged cache;
    const char *q, *k, *v;
    char *q_out;
    int64_t q_ts, q_hs, o_ts, o_hs, k_ts, k_hs, v_ts, v_hs;   // bytes
    const double *freqs;
    const int32_t *positions;
    const float *k_scale, *v_scale;
    int32_t q_heads, kv_heads;
    int32_t vecs;          // 16-byte vectors (8 elements) of a row
    int32_t half;          // rotated pairs
    int32_t per_block;     // tokens a workgroup takes
    float magnitude, sign;
    bool interleaved;
};

template <bool BF16> __device__ __forceinline__ float to_f32(uint32_t bits16) {
    if constexpr (BF16) return __builtin_bit_cast(float, bits16 << 16);
    return (float)__builtin_bit_cast(_Float16, (uint16_t)bits16);
}

template <bool BF16> __device__ __forceinline__ uint32_t pack2(float a, float b) {
    if constexpr (BF16) {
        typedef __bf16 bf2 __attribute__((ext_vector_type(2)));
        const bf2 x = {(__bf16)a, (__bf16)b};
        return __builtin_bit_cast(uint32_t, x);
    }
    typedef _Float16 h2 __attribute__((ext_vector_type(2)));
    const h2 x = {(_Float16)a, (_Float16)b};
    return __builtin_bit_cast(uint32_t, x);
}

// To the 8-bit type: largest value 448, NaN stays.
__device__ __forceinline__ float clamp_f8(float x) { return x != x ? x : fminf(fmaxf(x, -448.0f), 448.0f); }

__device__ __forceinline__ uint32_t pack4_f8(float a, float b, float c, float d) {
    int x = __builtin_amdgcn_cvt_pk_fp8_f32(clamp_f8(a), clamp_f8(b), 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(clamp_f8(c), clamp_f8(d), x, true);
}

// A workgroup takes per_block consecutive tokens: their angles first (one
// lane per token and pair), then every row of q, k and v.  A row lies in one
// wave (8 elements a lane, 64 / vecs rows a wave), which reads all of it
// before it writes, so q may be rotated in place.
template <bool BF16, bool F8>
__global__ __launch_bounds__(kThreads) void rope_append_kernel(RopeParams p) {
    extern __shared__ float trig[];                        // [per_block][half] cos, then sin
    __shared__ int32_t where_req[16], where_index[16];
    __shared__ uint32_t rows[kThreads / 64][64 * 4];       // a wave's rows, for partners in other lanes
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int64_t t0 = (int64_t)blockIdx.x * p.per_block;
    const int n = (int)(p.cache.num_q - t0 < p.per_block ? p.cache.num_q - t0 : p.per_block);
    for (int i = wave; i < n; i += kThreads / 64) {
        // request of the token: how many requests end at or before it
        int r = 0;
        for (int base = 0; base < p.cache.num_reqs; base += 64) {
            const bool before = base + lane < p.cache.num_reqs && p.cache.q_off[base + lane + 1] <= t0 + i;
            const int c = __popcll(__ballot(before));
            r += c;
            if (c < 64) break;
        }
        if (lane == 0) {
            const bool known = r < p.cache.num_reqs;
            where_req[i] = known ? r : -1;
            where_index[i] = known ? p.cache.kv_len[r] - (int32_t)(p.cache.q_off[r + 1] - (t0 + i)) : -1;
        }
    }
    __syncthreads();
    for (int x = tid; x < n * p.half; x += kThreads) {
        const int i = x / p.half, j = x - i * p.half;
        const double pos = p.positions ? p.positions[t0 + i] : where_index[i];
        double u = pos * p.freqs[j];
        u -= rint(u * 0.15915494309189533577) * 6.283185307179586476925;
        float s, c;
        sincosf((float)u, &s, &c);
        trig[x] = c * p.magnitude;
        trig[n * p.half + x] = s * p.magnitude * p.sign;
    }
    __syncthreads();
    const int nq = p.q ? p.q_heads : 0, nk = p.k ? p.kv_heads : 0;
    const int per_token = nq + 2 * nk, per_wave = 64 / p.vecs;
    const int sub = lane / p.vecs, vec = lane - sub * p.vecs;
    const int total = n * per_token;
    for (int first = wave * per_wave; first < total; first += (kThreads / 64) * per_wave) {
        const int item = first + sub;
        const bool on = sub < per_wave && item < total;
        const int i = on ? item / per_token : 0, h = on ? item - i * per_token : 0;
        const int64_t t = t0 + i;
        const bool is_q = h < nq, is_k = !is_q && h < nq + nk;
        const int kh = is_q ? 0 : (is_k ? h - nq : h - nq - nk);
        const char *src = is_q ? p.q + t * p.q_ts + h * p.q_hs
                               : (is_k ? p.k + t * p.k_ts + kh * p.k_hs : p.v + t * p.v_ts + kh * p.v_hs);
        u32x4 raw = {0, 0, 0, 0};
        if (on) raw = *(const u32x4 *)(src + vec * 16);
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = to_f32<BF16>((raw[e / 2] >> (16 * (e & 1))) & 0xffff);
        const bool turned = on && (is_q || is_k);
        const float *c = trig + i * p.half, *s = c + n * p.half;
        if (p.interleaved) {
            if (turned)
#pragma unroll
                for (int e = 0; e < 8; e += 2) {
                    const int j = vec * 4 + e / 2;
                    if (j < p.half) {
                        const float a = x[e], b = x[e + 1];
                        x[e] = __builtin_fmaf(a, c[j], -b * s[j]);
                        x[e + 1] = __builtin_fmaf(a, s[j], b * c[j]);
                    }
                }
        } else {
            // partners half a rotated part away, by way of LDS (the wave's own rows)
            uint16_t *mine = (uint16_t *)rows[wave] + sub * p.vecs * 8;
            if (on) *(u32x4 *)(mine + vec * 8) = raw;
            __builtin_amdgcn_wave_barrier();
            if (turned)
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int d = vec * 8 + e;
                    if (d < p.half) {
                        x[e] = __builtin_fmaf(x[e], c[d], -to_f32<BF16>(mine[d + p.half]) * s[d]);
                    } else if (d < 2 * p.half) {
                        const int j = d - p.half;
                        x[e] = __builtin_fmaf(to_f32<BF16>(mine[j]), s[j], x[e] * c[j]);
                    }
                }
            __builtin_amdgcn_wave_barrier();
        }
        if (!on) continue;
        if (is_q) {
            const u32x4 y = {pack2<BF16>(x[0], x[1]), pack2<BF16>(x[2], x[3]), pack2<BF16>(x[4], x[5]),
                             pack2<BF16>(x[6], x[7])};
            *(u32x4 *)(p.q_out + t * p.o_ts + h * p.o_hs + vec * 16) = y;
            continue;
        }
        const int32_t r = where_req[i], index = where_index[i];
        if (r < 0 || index < 0) continue;
        uint32_t row;
        const int32_t id = block_of(p.cache, r, (uint32_t)index, row);
        if (id < 0) continue;
        char *dst = p.cache.layer + (is_k ? 0 : p.cache.kv_stride) +
                    (((int64_t)id * p.cache.block16 + (int64_t)row * p.cache.row16) << 4) +
                    (int64_t)kh * p.cache.head_bytes;
        if constexpr (F8) {
            const float *scale = is_k ? p.k_scale : p.v_scale;
            if (scale) {
                const float by = scale[kh];
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] /= by;
            }
            const u32x2 y = {pack4_f8(x[0], x[1], x[2], x[3]), pack4_f8(x[4], x[5], x[6], x[7])};
            *(u32x2 *)(dst + vec * 8) = y;
        } else {
            const u32x4 y = {pack2<BF16>(x[0], x[1]), pack2<BF16>(x[2], x[3]), pack2<BF16>(x[4], x[5]),
                             pack2<BF16>(x[6], x[7])};
            *(u32x4 *)(dst + vec * 16) = is_k ? y : raw;
        }
    }
}

}  // namespace
}  // namespace tkv

extern "C" {

int kv_rope_append(const kv_layout *layout, void *d_layer, const kv_batch *batch, const kv_rows *q,
                   const kv_rows *q_out, const kv_rows *k, const kv_rows *v, const double *d_freqs, int32_t rot_dim,
                   int32_t flags, float magnitude, const int32_t *d_positions, int32_t cache_dtype,
                   const float *d_k_scale, const float *d_v_scale, void *stream) {
    int rc = tkv::check_cache(layout, cache_dtype);
    if (rc == KV_OK) rc = tkv::check_batch(batch);
    if (rc != KV_OK) return rc;
    const int32_t d = layout->head_dim;
    if ((!q && !k) || !q != !q_out || !k != !v || (k && !d_layer)) return KV_EINVAL;
    if (q && ((rc = tkv::check_rows(q, batch->num_q, d, false)) != KV_OK ||
              (rc = tkv::check_rows(q_out, batch->num_q, d, true)) != KV_OK))
        return rc;
    if (k && ((rc = tkv::check_rows(k, batch->num_q, d, false)) != KV_OK ||
              (rc = tkv::check_rows(v, batch->num_q, d, false)) != KV_OK))
        return rc;
    const int32_t dtype = q ? q->dtype : k->dtype;
    if (q && (q_out->dtype != dtype || q_out->heads != q->heads)) return KV_EINVAL;
    if (k && (k->dtype != dtype || v->dtype != dtype || k->heads != layout->kv_heads || v->heads != layout->kv_heads))
        return KV_EINVAL;
    if (k && cache_dtype != KV_F8E4M3 && cache_dtype != dtype) return KV_EINVAL;
    if (rot_dim < 0 || rot_dim % 2 != 0 || rot_dim > d || (rot_dim > 0 && !d_freqs)) return KV_EINVAL;
    if (flags & ~(KV_ROPE_INTERLEAVED | KV_ROPE_INVERSE)) return KV_EINVAL;
    if (((uintptr_t)d_layer & 15u) || ((uintptr_t)d_freqs & 7u) || ((uintptr_t)d_positions & 3u)) return KV_EALIGN;
    if (batch->num_q == 0) return KV_OK;
    tkv::RopeParams p;
    p.cache = tkv::make_paged(layout, d_layer, batch);
    p.q = q ? (const char *)q->d_data : nullptr;
    p.q_out = q ? (char *)const_cast<void *>(q_out->d_data) : nullptr;
    p.k = k ? (const char *)k->d_data : nullptr;
    p.v = k ? (const char *)v->d_data : nullptr;
    p.q_ts = q ? q->token_stride * 2 : 0, p.q_hs = q ? q->head_stride * 2 : 0;
    p.o_ts = q ? q_out->token_stride * 2 : 0, p.o_hs = q ? q_out->head_stride * 2 : 0;
    p.k_ts = k ? k->token_stride * 2 : 0, p.k_hs = k ? k->head_stride * 2 : 0;
    p.v_ts = k ? v->token_stride * 2 : 0, p.v_hs = k ? v->head_stride * 2 : 0;
    p.freqs = d_freqs;
    p.positions = d_positions;
    p.k_scale = d_k_scale;
    p.v_scale = d_v_scale;
    p.q_heads = q ? q->heads : 0;
    p.kv_heads = layout->kv_heads;
    p.vecs = d / 8;
    p.half = rot_dim / 2;
    p.per_block = 4;
    p.magnitude = magnitude;
    p.sign = (flags & KV_ROPE_INVERSE) ? -1.0f : 1.0f;
    p.interleaved = (flags & KV_ROPE_INTERLEAVED) != 0;
    const int64_t blocks = (batch->num_q + p.per_block - 1) / p.per_block;
    if (blocks >= (int64_t(1) << 31)) return KV_ELIMIT;
    const size_t lds = (size_t)p.per_block * p.half * 2 * sizeof(float);
    const bool f8 = cache_dtype == KV_F8E4M3;
    auto kernel = dtype == KV_BF16 ? (f8 ? tkv::rope_append_kernel<true, true> : tkv::rope_append_kernel<true, false>)
                                   : (f8 ? tkv::rope_append_kernel<false, true> : tkv::rope_append_kernel<false, false>);
    (void)hipGetLastError();
    hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(tkv::kThreads), lds, (hipStream_t)stream, p);
    return hipGetLastError() == hipSuccess ? KV_OK : KV_EHIP;
}

}  // extern "C"
