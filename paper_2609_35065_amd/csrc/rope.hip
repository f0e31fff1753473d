// rope.hip -- rotary positions and the append to the paged cache.
//
// A row at position p has pair i turned by u = p * f_i:
//     (a, b) -> (a cos u - b sin u, a sin u + b cos u) * magnitude.
// The angle needs more than 32 bits (position 100,000 times 1 radian leaves
// 2^-7 radians of a float's mantissa), so the product and its remainder by a
// turn are formed in 64 bits, once per (token, pair), and shared by all heads.
// With several axes p is the row's position on the pair's axis.

#include "paged.h"

namespace tkv {
namespace {

constexpr int kThreads = 256, kMaxTokens = 4;
constexpr int64_t kStream = int64_t(1) << 28;          // bytes from which rows pass the caches by

struct RopeParams {
    Paged cache;
    const char *q, *k, *v;
    char *q_out;
    int64_t q_ts, q_hs, o_ts, o_hs, k_ts, k_hs, v_ts, v_hs;   // bytes
    const double *freqs;
    const int32_t *positions;
    int64_t position_stride;                                  // between the positions of one axis and the next
    const float *k_scale, *v_scale;
    int32_t q_heads, kv_heads;
    Divider by_token, by_row, by_half;
    int32_t vecs;          // 16-byte vectors (8 elements) of a row
    int32_t half;          // rotated pairs
    int32_t row_units, token_units;
    int32_t per_block;     // tokens a workgroup takes
    float magnitude, sign;
    uint8_t axis[kMaxHeadDim / 2];                            // of each pair
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

// A token's angles are shared by its rows, so a workgroup takes per_block
// tokens: where each goes and its angles first (one lane per token and pair),
// then the rows, in units of two 16-byte vectors that need nothing else:
//   HALF         vectors v and v + half/8, whose elements are each other's partners (half a multiple of 8)
//   INTERLEAVED  neighbouring vectors
//   ODD          half not a multiple of 8: neighbouring vectors, partners by way of LDS
// What is not rotated (the rest of a row, v) comes in neighbouring vectors.
// A row lies in one wave, which reads all of it before it writes, so q may be
// rotated in place.  A lane's first unit is loaded before the angles.
// Bound by memory: 32,768 tokens of 32 + 2 x 8 heads of 128, 0.81 GB read and
// written in 143 us (5.6 TB/s); ragged, head size 80, an 8-bit cache: 0.25 GB in
// 54 us (4.6 TB/s).  STREAM passes the caches by, which a large batch's rows do
// not fit: 143 against 157 us by itself.  What follows an append is attention,
// which reads its rows.  The two together, into rows of their own, take 273
// against 283 us at 403 MB (32 prompts of 512 tokens) and 226 against 238 at 270
// MB (11 of 1,000), in place the same within 1 %; but at 201 MB (16 of 512) in
// place 144 against 138, as much of it is still in the memory-side cache of 256
// MB.  That is for units of whole cache lines (64 pairs of 16 bits); the narrow
// rows of the 8-bit batch take 69 us that way.
enum Pairing { HALF, INTERLEAVED, ODD };

template <bool STREAM, class V> __device__ __forceinline__ V read_row(const V *at) {
    if constexpr (STREAM) return __builtin_nontemporal_load(at);
    return *at;
}

template <bool STREAM, class V> __device__ __forceinline__ void write_row(V x, V *at) {
    if constexpr (STREAM) __builtin_nontemporal_store(x, at);
    else *at = x;
}

template <bool BF16, bool F8, Pairing PAIR, bool AXES, bool STREAM>
__global__ __launch_bounds__(kThreads) void rope_append_kernel(RopeParams p) {
    extern __shared__ __align__(16) float trig[];                       // [per_block][half4] cos, then sin
    __shared__ int32_t where_index[kMaxTokens];
    __shared__ uint32_t where_row[kMaxTokens];             // 16-byte units from the plane's start
    __shared__ bool where_in[kMaxTokens];
    __shared__ uint32_t rows[PAIR == ODD ? kThreads / 64 : 1][PAIR == ODD ? 64 * 8 : 1];   // a wave's rows
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int64_t t0 = (int64_t)blockIdx.x * p.per_block;
    const int n = (int)(p.cache.num_q - t0 < p.per_block ? p.cache.num_q - t0 : p.per_block);
    const int half4 = (p.half + 3) & ~3;
    const int total = n * p.token_units;

    // unit x: its row, and its vectors a and b (b = -1: none)
    struct Unit {
        int token, head, a, b;     // head: of q, then k, then v
        bool on;
    };
    const int per_wave = PAIR == ODD ? 64 / p.row_units * p.row_units : 64;    // whole rows where LDS is in between
    const int stride = kThreads / 64 * per_wave, start = wave * per_wave + lane;
    const auto unit_of = [&](int x) {
        Unit u;
        u.on = x < total && lane < per_wave;
        if (!u.on) x = 0;
        u.token = (int)divide(x, p.by_token);
        const int y = x - u.token * p.token_units;
        u.head = (int)divide(y, p.by_row);
        const int z = y - u.head * p.row_units, hv = p.half / 8;
        const bool partners = PAIR == HALF && z < hv;
        u.a = partners ? z : 2 * z;          // past the partners' units: 2 hv + 2 (z - hv)
        u.b = partners ? z + hv : u.a + 1;
        if (u.b >= p.vecs) u.b = -1;
        return u;
    };
    const int nq = p.q_heads, nk = p.k ? p.kv_heads : 0;
    const auto source = [&](const Unit &u) {
        const int64_t t = t0 + u.token;
        if (u.head < nq) return p.q + t * p.q_ts + u.head * p.q_hs;
        if (u.head < nq + nk) return p.k + t * p.k_ts + (u.head - nq) * p.k_hs;
        return p.v + t * p.v_ts + (u.head - nq - nk) * p.v_hs;
    };
    const auto fetch = [&](const Unit &u, u32x4 &a, u32x4 &b) {
        if (!u.on) return;
        const char *src = source(u);
        a = read_row<STREAM>((const u32x4 *)(src + u.a * 16));
        if (u.b >= 0) b = read_row<STREAM>((const u32x4 *)(src + u.b * 16));
    };
    u32x4 ra = {0, 0, 0, 0}, rb = {0, 0, 0, 0};
    Unit u = unit_of(start);
    fetch(u, ra, rb);

    for (int i = wave; i < n; i += kThreads / 64) {
        // the token's request: how many requests end at or before it
        int r = 0;
        for (int base = 0; base < p.cache.num_reqs; base += 64) {
            const bool before = base + lane < p.cache.num_reqs && p.cache.q_off[base + lane + 1] <= t0 + i;
            const int c = __popcll(__ballot(before));
            r += c;
            if (c < 64) break;
        }
        if (lane == 0) {
            const bool known = r < p.cache.num_reqs && p.cache.q_off[r] <= t0 + i;     // (of no request: the rows before the first)
            const int32_t index = known ? p.cache.kv_len[r] - (int32_t)(p.cache.q_off[r + 1] - (t0 + i)) : -1;
            uint32_t row = 0;
            const int32_t id = index >= 0 ? block_of(p.cache, r, (uint32_t)index, row) : -1;
            where_index[i] = index;
            where_in[i] = id >= 0;
            where_row[i] = id < 0 ? 0u : (uint32_t)id * p.cache.block16 + row * p.cache.row16;
        }
    }
    __syncthreads();
    for (int x = tid; x < n * p.half; x += kThreads) {
        const int i = (int)divide(x, p.by_half), j = x - i * p.half;
        double pos;
        if constexpr (AXES) pos = p.positions[p.axis[j] * p.position_stride + t0 + i];
        else pos = p.positions ? p.positions[t0 + i] : where_index[i];
        double angle = pos * p.freqs[j];
        angle -= rint(angle * 0.15915494309189533577) * 6.283185307179586476925;
        float s, c;
        sincosf((float)angle, &s, &c);
        trig[i * half4 + j] = c * p.magnitude;
        trig[(n + i) * half4 + j] = s * p.magnitude * p.sign;
    }
    __syncthreads();
    // (uniform in the wave: the LDS of ODD is its own)
    for (int x = start; x - lane < total; x += stride) {
        u32x4 na = {0, 0, 0, 0}, nb = {0, 0, 0, 0};
        const Unit next = unit_of(x + stride);
        fetch(next, na, nb);
        const bool is_q = u.head < nq, is_k = !is_q && u.head < nq + nk;
        const float *c = trig + u.token * half4, *s = c + n * half4;
        float xa[8], xb[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            xa[e] = to_f32<BF16>((ra[e / 2] >> (16 * (e & 1))) & 0xffff);
            xb[e] = to_f32<BF16>((rb[e / 2] >> (16 * (e & 1))) & 0xffff);
        }
        const bool turned = u.on && (is_q || is_k);
        if constexpr (PAIR == HALF) {
            if (turned && u.a < p.half / 8) {
                f32x4 cc[2], ss[2];
#pragma unroll
                for (int g = 0; g < 2; ++g) {
                    cc[g] = *(const f32x4 *)(c + u.a * 8 + g * 4);
                    ss[g] = *(const f32x4 *)(s + u.a * 8 + g * 4);
                }
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float a = xa[e], b = xb[e], co = cc[e / 4][e % 4], si = ss[e / 4][e % 4];
                    xa[e] = __builtin_fmaf(a, co, -b * si);
                    xb[e] = __builtin_fmaf(a, si, b * co);
                }
            }
        } else if constexpr (PAIR == INTERLEAVED) {
            if (turned)
#pragma unroll
                for (int v = 0; v < 2; ++v) {
                    const int j0 = (v ? u.b : u.a) * 4;
                    if (j0 < 0 || j0 >= p.half) continue;
                    const f32x4 co = *(const f32x4 *)(c + j0), si = *(const f32x4 *)(s + j0);
                    float *y = v ? xb : xa;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float a = y[2 * e], b = y[2 * e + 1];
                        if (j0 + e < p.half) {
                            y[2 * e] = __builtin_fmaf(a, co[e], -b * si[e]);
                            y[2 * e + 1] = __builtin_fmaf(a, si[e], b * co[e]);
                        }
                    }
                }
        } else {
            const int first = lane / p.row_units * p.row_units;            // lane of the row's first unit
            uint16_t *mine = (uint16_t *)rows[wave] + first * 16;
            // (the wave's own rows: its LDS accesses are in order, and the fences keep them so in the code)
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
            if (u.on) {
                *(u32x4 *)(mine + u.a * 8) = ra;
                if (u.b >= 0) *(u32x4 *)(mine + u.b * 8) = rb;
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
            if (turned)
#pragma unroll
                for (int v = 0; v < 2; ++v) {
                    float *y = v ? xb : xa;
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const int d = (v ? u.b : u.a) * 8 + e;
                        if (d < 0) continue;
                        if (d < p.half) {
                            y[e] = __builtin_fmaf(y[e], c[d], -to_f32<BF16>(mine[d + p.half]) * s[d]);
                        } else if (d < 2 * p.half) {
                            const int j = d - p.half;
                            y[e] = __builtin_fmaf(to_f32<BF16>(mine[j]), s[j], y[e] * c[j]);
                        }
                    }
                }
        }
        if (u.on && (is_q || where_in[u.token])) {
            const int kh = is_k ? u.head - nq : u.head - nq - nk;
            char *dst = is_q ? p.q_out + (t0 + u.token) * p.o_ts + u.head * p.o_hs
                             : p.cache.layer + (is_k ? 0 : p.cache.kv_stride) + ((int64_t)where_row[u.token] << 4) +
                                   (int64_t)kh * p.cache.head_bytes;
            const float *scale = is_k ? p.k_scale : p.v_scale;
            const float by = F8 && !is_q && scale ? 1.0f / scale[kh] : 1.0f;
#pragma unroll
            for (int v = 0; v < 2; ++v) {
                const int vec = v ? u.b : u.a;
                const float *y = v ? xb : xa;
                if (vec < 0) continue;
                if (F8 && !is_q) {
                    const u32x2 z = {pack4_f8(y[0] * by, y[1] * by, y[2] * by, y[3] * by),
                                     pack4_f8(y[4] * by, y[5] * by, y[6] * by, y[7] * by)};
                    *(u32x2 *)(dst + vec * 8) = z;
                } else {
                    const u32x4 z = {pack2<BF16>(y[0], y[1]), pack2<BF16>(y[2], y[3]), pack2<BF16>(y[4], y[5]),
                                     pack2<BF16>(y[6], y[7])};
                    write_row<STREAM>(is_q || is_k ? z : (v ? rb : ra), (u32x4 *)(dst + vec * 16));
                }
            }
        }
        u = next;
        ra = na;
        rb = nb;
    }
}

template <bool BF16, bool F8, bool AXES> void (*rope_kernel(Pairing pair, bool stream))(RopeParams) {
    if constexpr (!F8) {
        if (stream) return rope_append_kernel<BF16, F8, HALF, AXES, true>;
    }
    return pair == HALF ? rope_append_kernel<BF16, F8, HALF, AXES, false>
                        : (pair == INTERLEAVED ? rope_append_kernel<BF16, F8, INTERLEAVED, AXES, false>
                                               : rope_append_kernel<BF16, F8, ODD, AXES, false>);
}

template <bool AXES> auto rope_kernel(bool bf16, bool f8, Pairing pair, bool stream) {
    return bf16 ? (f8 ? rope_kernel<true, true, AXES>(pair, stream) : rope_kernel<true, false, AXES>(pair, stream))
                : (f8 ? rope_kernel<false, true, AXES>(pair, stream) : rope_kernel<false, false, AXES>(pair, stream));
}

// The append with one position a row (num_axes 0), or several and the axis of each pair.
int rope_append(const kv_layout *layout, void *d_layer, const kv_batch *batch, const kv_rows *q, const kv_rows *q_out,
                const kv_rows *k, const kv_rows *v, const double *d_freqs, int32_t rot_dim, int32_t flags,
                float magnitude, const int32_t *d_positions, int64_t position_stride, int32_t num_axes,
                const uint8_t *h_axis, int32_t cache_dtype, const float *d_k_scale, const float *d_v_scale,
                void *stream) {
    int rc = check_cache(layout, cache_dtype);
    if (rc == KV_OK) rc = check_batch(batch);
    if (rc != KV_OK) return rc;
    const int32_t d = layout->head_dim;
    if ((!q && !k) || !q != !q_out || !k != !v || (k && !d_layer)) return KV_EINVAL;
    if (q && ((rc = check_rows(q, batch->num_q, d, false)) != KV_OK ||
              (rc = check_rows(q_out, batch->num_q, d, true)) != KV_OK))
        return rc;
    if (k && ((rc = check_rows(k, batch->num_q, d, false)) != KV_OK ||
              (rc = check_rows(v, batch->num_q, d, false)) != KV_OK))
        return rc;
    const int32_t dtype = q ? q->dtype : k->dtype;
    if (q && (q_out->dtype != dtype || q_out->heads != q->heads)) return KV_EINVAL;
    if (k && (k->dtype != dtype || v->dtype != dtype || k->heads != layout->kv_heads || v->heads != layout->kv_heads))
        return KV_EINVAL;
    if (k && cache_dtype != KV_F8E4M3 && cache_dtype != dtype) return KV_EINVAL;
    if (rot_dim < 0 || rot_dim % 2 != 0 || rot_dim > d || (rot_dim > 0 && !d_freqs)) return KV_EINVAL;
    if (flags & ~(KV_ROPE_INTERLEAVED | KV_ROPE_INVERSE)) return KV_EINVAL;
    RopeParams p;
    if (num_axes > 0) {
        if (rot_dim > 0 && !h_axis) return KV_EINVAL;
        for (int32_t i = 0; i < rot_dim / 2; ++i) {
            if (h_axis[i] >= num_axes) return KV_EINVAL;
            p.axis[i] = h_axis[i];
        }
        if (batch->num_q > 0 && rot_dim > 0 && (!d_positions || position_stride < batch->num_q)) return KV_EINVAL;
    }
    if (((uintptr_t)d_layer & 15u) || ((uintptr_t)d_freqs & 7u) || ((uintptr_t)d_positions & 3u)) return KV_EALIGN;
    if (batch->num_q == 0) return KV_OK;
    p.cache = make_paged(layout, d_layer, batch);
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
    p.position_stride = position_stride;
    p.k_scale = d_k_scale;
    p.v_scale = d_v_scale;
    p.q_heads = q ? q->heads : 0;
    p.kv_heads = layout->kv_heads;
    p.vecs = d / 8;
    p.half = rot_dim / 2;
    p.magnitude = magnitude;
    p.sign = (flags & KV_ROPE_INVERSE) ? -1.0f : 1.0f;
    const Pairing pair = (flags & KV_ROPE_INTERLEAVED) ? INTERLEAVED : (p.half % 8 ? ODD : HALF);
    const int hv = pair == HALF ? p.half / 8 : 0;
    p.row_units = hv + (p.vecs - 2 * hv + 1) / 2;
    p.token_units = p.row_units * (p.q_heads + (k ? 2 * p.kv_heads : 0));
    p.by_row = make_divider((uint32_t)p.row_units);
    p.by_token = make_divider((uint32_t)p.token_units);
    p.by_half = make_divider((uint32_t)(p.half ? p.half : 1));
    const bool f8 = cache_dtype == KV_F8E4M3;
    // Rows of a batch that pass the caches by; and four tokens (of those two) that share a workgroup's start where there
    // are workgroups enough, while few tokens take one each.
    const int64_t moved = batch->num_q * 4 * d * (p.q_heads + (k ? 2 * p.kv_heads : 0));      // bytes
    const bool stream_rows = !f8 && pair == HALF && p.half > 0 && p.half % 64 == 0 && 2 * p.half == d && moved >= kStream;
    const int64_t share = batch->num_q / 1024, most = stream_rows ? 2 : kMaxTokens;
    p.per_block = share < 1 ? 1 : (share > most ? (int)most : (int)share);
    const int64_t blocks = (batch->num_q + p.per_block - 1) / p.per_block;
    if (blocks >= (int64_t(1) << 31)) return KV_ELIMIT;
    const size_t lds = (size_t)p.per_block * ((p.half + 3) & ~3) * 2 * sizeof(float);
    auto kernel = num_axes > 0 ? rope_kernel<true>(dtype == KV_BF16, f8, pair, stream_rows)
                               : rope_kernel<false>(dtype == KV_BF16, f8, pair, stream_rows);
    (void)hipGetLastError();
    hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(kThreads), lds, (hipStream_t)stream, p);
    return hipGetLastError() == hipSuccess ? KV_OK : KV_EHIP;
}

}  // namespace
}  // namespace tkv

extern "C" {

int kv_rope_append(const kv_layout *layout, void *d_layer, const kv_batch *batch, const kv_rows *q,
                   const kv_rows *q_out, const kv_rows *k, const kv_rows *v, const double *d_freqs, int32_t rot_dim,
                   int32_t flags, float magnitude, const int32_t *d_positions, int32_t cache_dtype,
                   const float *d_k_scale, const float *d_v_scale, void *stream) {
    return tkv::rope_append(layout, d_layer, batch, q, q_out, k, v, d_freqs, rot_dim, flags, magnitude, d_positions, 0, 0,
                            nullptr, cache_dtype, d_k_scale, d_v_scale, stream);
}

int kv_rope_append_axes(const kv_layout *layout, void *d_layer, const kv_batch *batch, const kv_rows *q,
                        const kv_rows *q_out, const kv_rows *k, const kv_rows *v, const double *d_freqs,
                        int32_t rot_dim, int32_t flags, float magnitude, const int32_t *d_positions,
                        int64_t position_stride, int32_t num_axes, const uint8_t *h_axis, int32_t cache_dtype,
                        const float *d_k_scale, const float *d_v_scale, void *stream) {
    if (num_axes <= 0 || num_axes > KV_MAX_AXES) return KV_EINVAL;
    return tkv::rope_append(layout, d_layer, batch, q, q_out, k, v, d_freqs, rot_dim, flags, magnitude, d_positions,
                            position_stride, num_axes, h_axis, cache_dtype, d_k_scale, d_v_scale, stream);
}

}  // extern "C"
