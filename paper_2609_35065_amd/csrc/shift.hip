// shift.hip -- keys that lie in the paged cache turned to other positions.
//
// Rotations add: a key turned by p f_i that is turned again by s f_i is one of
// position p + s.  Pair (a, b) becomes (a cos u - b sin u, a sin u + b cos u),
// u = s f_i, the product and its remainder by a turn in 64 bits.  Bound by
// memory: 32 layers of 8 requests of 2,048 tokens, 8 KV heads of 128, 2.15 GB read
// and written in 376 to 385 us (5.6 to 5.7 TB/s); in 8 bits, where each head's
// tokens have shifts of their own, by the vector units too (60 % of the time): 0.93
// GB in 204 to 211 us (4.5 TB/s).

#include "mfma.h"
#include "paged.h"

namespace tkv {
namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr int kHeads = 16;                     // of a workgroup's tile
// Tokens of a tile, and units that a lane has on their way.  Small tiles keep what all workgroups move at a time spread
// evenly: 32 layers of 8 x 2,048 tokens in 16 bits take 376 us with 16, 390 with 32, 408 with 64; 8-bit rows, whose
// angles cost as much for half the bytes, amortise a start over 32 (207 us; 214 with 16, 210 with 64).
template <bool F8> constexpr int kTokens = F8 ? 32 : 16;
template <bool F8> constexpr int kAhead = F8 ? 2 : 4;
constexpr int kPairs = 8;                      // of a lane's unit
constexpr int64_t kMaxBlocks = 1 << 23;        // of a launch, which may have 2^32 lanes

struct ShiftParams {
    Paged cache;
    char *layers[KV_MAX_LAYERS];
    const int32_t *len, *shift;
    int64_t shift_stride;
    const double *freqs;
    int32_t shift_layers, shift_heads;         // 1: one shift for all
    int32_t kv_heads, groups;                  // groups of kHeads heads
    int32_t half, units;                       // pairs of a row, and units
    int32_t tiles;                             // of a request's tokens: workgroups for each layer, request and group
    Divider by_heads;                          // of a group that is not full
    double sign;
};

// What a workgroup takes.  Tiles of one request are next to one another: they go to all XCDs in turn, where ragged
// requests side by side left some of them idle.
struct Place {
    int l, r, head0;
    int64_t tile;
};

__device__ __forceinline__ Place find_place(const ShiftParams &p) {
    const uint32_t x = blockIdx.x / (uint32_t)p.tiles, lr = x / (uint32_t)p.groups;
    Place y;
    y.tile = blockIdx.x - x * p.tiles;
    y.head0 = (int)(x - lr * p.groups) * kHeads;
    y.l = (int)(lr / (uint32_t)p.cache.num_reqs);
    y.r = (int)(lr - (uint32_t)y.l * p.cache.num_reqs);
    return y;
}

// Elements at any alignment.
typedef u32x4 __attribute__((aligned(1))) u32x4_any;
typedef u32x2 __attribute__((aligned(1))) u32x2_any;

template <bool STREAM, class V> __device__ __forceinline__ V read_some(const V *at) {
    if constexpr (STREAM) return __builtin_nontemporal_load(at);
    return *at;
}

template <bool STREAM, class V> __device__ __forceinline__ void write_some(V x, V *at) {
    if constexpr (STREAM) __builtin_nontemporal_store(x, at);
    else *at = x;
}

// N elements of the cache's type, and as 32-bit values.
template <class T, bool F8, int N> struct Elements {
    uint32_t raw[F8 ? N / 4 : N / 2];
    template <bool STREAM> __device__ __forceinline__ void load(const char *at) {
        constexpr int kWords = F8 ? N / 4 : N / 2;
        if constexpr (kWords == 2) {
            const u32x2 x = read_some<STREAM>((const u32x2_any *)at);
            raw[0] = x[0], raw[1] = x[1];
        } else {
#pragma unroll
            for (int i = 0; i < kWords; i += 4) {
                const u32x4 x = read_some<STREAM>((const u32x4_any *)(at + i * 4));
#pragma unroll
                for (int e = 0; e < 4; ++e) raw[i + e] = x[e];
            }
        }
    }
    template <bool STREAM> __device__ __forceinline__ void store(char *at) const {
        constexpr int kWords = F8 ? N / 4 : N / 2;
        if constexpr (kWords == 2) {
            write_some<STREAM, u32x2_any>(u32x2{raw[0], raw[1]}, (u32x2_any *)at);
        } else {
#pragma unroll
            for (int i = 0; i < kWords; i += 4)
                write_some<STREAM, u32x4_any>(u32x4{raw[i], raw[i + 1], raw[i + 2], raw[i + 3]}, (u32x4_any *)(at + i * 4));
        }
    }
    __device__ __forceinline__ void get(float (&x)[N]) const {
#pragma unroll
        for (int i = 0; i < N; i += 2) {
            if constexpr (F8) {
                const f32x2 y = i & 2 ? __builtin_amdgcn_cvt_pk_f32_fp8((int)raw[i / 4], true)
                                      : __builtin_amdgcn_cvt_pk_f32_fp8((int)raw[i / 4], false);
                x[i] = y[0], x[i + 1] = y[1];
            } else {
                x[i] = T::to_f32(raw[i / 2] & 0xffffu), x[i + 1] = T::to_f32(raw[i / 2] >> 16);
            }
        }
    }
    // rounded once, to nearest even; in 8 bits (saturating, see saturate_f8) values beyond 448 become 448, NaN stays
    __device__ __forceinline__ void set(const float (&x)[N]) {
        if constexpr (F8) {
#pragma unroll
            for (int i = 0; i < N; i += 4) {
                const int y = __builtin_amdgcn_cvt_pk_fp8_f32(x[i], x[i + 1], 0, false);
                raw[i / 4] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x[i + 2], x[i + 3], y, true);
            }
        } else {
#pragma unroll
            for (int i = 0; i < N; i += 2) raw[i / 2] = pack2<T>(x[i], x[i + 1]);
        }
    }
};

// From here on the wave's conversions to 8 bits give the largest value, 448, for finite values beyond it (the mode
// register's bit 23; infinities, which an 8-bit cache does not hold, would become NaN).  As a clamp, with NaN kept, it
// would be three instructions an element.
__device__ __forceinline__ void saturate_f8() { __builtin_amdgcn_s_setreg(1 | 23 << 6, 1); }

// Sine and cosine of the angles s f_i, f in turns below 1/2 in size.  Added to 1.5 x 2^20 in 64 bits, a number of turns
// leaves its fraction in the low 32 bits, in units of 2^-32: one operation for the product and the remainder, where the
// turns stay below 2^19.  The sines of the unit are off by up to 1.3e-7 (2^-22.9) of their size-1 range.
template <int N> __device__ __forceinline__ void sincos_turns(int s, const double (&f)[N], float (&c)[N], float (&si)[N]) {
    float u[N];
    if (__any((uint32_t)s + (1u << 20) >= 1u << 21)) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const double turns = s * f[i];
            u[i] = (float)(turns - rint(turns));
        }
    } else {
        const double x = s;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const double y = __builtin_fma(x, f[i], 0x1.8p20);
            u[i] = (float)(int32_t)__builtin_bit_cast(uint64_t, y) * 0x1p-32f;
        }
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
        c[i] = __builtin_amdgcn_cosf(u[i]);
        si[i] = __builtin_amdgcn_sinf(u[i]);
    }
}

// A frequency in turns a position, without its whole turns (a shift is a whole number), backwards if asked.
__device__ __forceinline__ double to_turns(const ShiftParams &p, int pair) {
    const double f = p.freqs[pair] * 0.15915494309189533577;
    return (f - rint(f)) * p.sign;
}

// One workgroup: a layer, a request, up to 16 heads and a tile of tokens.  Where the
// tokens lie and their shifts go to LDS first.  A lane takes eight pairs of a
// row, always the same ones, so that it holds their frequencies; a row's last
// unit ends at its last pair and may overlap the one before.  A row lies in one
// wave, which reads all of it before it writes.  STREAM passes the caches by:
// for halves of a row that are whole cache lines (376 against 412 us for the
// 16-bit keys above; halves of 16 and 48 bytes would take twice as long as they do).
template <class T, bool F8, bool INTERLEAVED, bool STREAM>
__global__ __launch_bounds__(kThreads) void rope_shift_kernel(ShiftParams p) {
    constexpr int kElem = F8 ? 1 : 2, kTok = kTokens<F8>, kNext = kAhead<F8>;
    __shared__ uint32_t where[kTok];            // 16-byte units from the plane's start
    __shared__ int32_t by[kHeads][kTok];        // 0: left as it is
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const Place at0 = find_place(p);
    const int r = at0.r, l = at0.l, head0 = at0.head0, heads = min(kHeads, p.kv_heads - head0);
    const int64_t len = min((int64_t)max(p.len[r], 0), p.shift_stride);
    const int32_t *shift = p.shift + ((int64_t)(p.shift_layers > 1 ? l : 0) * p.cache.num_reqs + r) * p.shift_heads * p.shift_stride;
    char *base = p.layers[l];

    const int slot = lane / p.units, unit = lane - slot * p.units, rows = 64 / p.units;     // of a wave
    const bool on = slot < rows;
    const int pair0 = min(unit * kPairs, p.half - kPairs);
    double f[kPairs];
#pragma unroll
    for (int i = 0; i < kPairs; ++i) f[i] = to_turns(p, pair0 + i);
    if constexpr (F8) saturate_f8();
    const int first = (INTERLEAVED ? 2 * pair0 : pair0) * kElem, second = (p.half + pair0) * kElem;     // bytes

    for (int64_t t0 = at0.tile * kTok; t0 < len; t0 += (int64_t)p.tiles * kTok) {
        const int n = (int)min((int64_t)kTok, len - t0);
        __syncthreads();                           // the tile before is done
        for (int x = tid; x < heads * kTok; x += kThreads) {
            const int t = x % kTok, h = x / kTok;
            uint32_t row = 0;
            const int32_t id = t < n ? block_of(p.cache, r, (uint32_t)(t0 + t), row) : -1;
            if (h == 0) where[t] = id < 0 ? 0u : (uint32_t)id * p.cache.block16 + row * p.cache.row16;
            by[h][t] = id < 0 ? 0 : shift[(p.shift_heads > 1 ? (int64_t)(head0 + h) * p.shift_stride : 0) + t0 + t];
        }
        __syncthreads();
        const int total = n * heads, step = kWaves * rows;
        for (int x0 = wave * rows; x0 < total; x0 += kNext * step) {
            Elements<T, F8, INTERLEAVED ? 16 : 8> a[kNext], b[kNext];
            int s[kNext];
            char *at[kNext];
#pragma unroll
            for (int i = 0; i < kNext; ++i) {
                const int x = x0 + i * step + slot;
                s[i] = 0;
                if (!on || x >= total) continue;
                const int t = heads == kHeads ? x / kHeads : (int)divide(x, p.by_heads), h = x - t * heads;
                s[i] = by[h][t];
                at[i] = base + ((int64_t)where[t] << 4) + (int64_t)(head0 + h) * p.cache.head_bytes;
                if (s[i] == 0) continue;
                a[i].template load<STREAM>(at[i] + first);
                if constexpr (!INTERLEAVED) b[i].template load<STREAM>(at[i] + second);
            }
            // units of a row overlap, in the same instructions of a wave: all are read here
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
#pragma unroll
            for (int i = 0; i < kNext; ++i) {
                if (s[i] == 0) continue;
                float xa[INTERLEAVED ? 16 : 8], xb[8], c[kPairs], si[kPairs];
                sincos_turns(s[i], f, c, si);
                a[i].get(xa);
                if constexpr (!INTERLEAVED) b[i].get(xb);
#pragma unroll
                for (int e = 0; e < kPairs; ++e) {
                    float &ra = xa[INTERLEAVED ? 2 * e : e], &rb = INTERLEAVED ? xa[(2 * e + 1) % (INTERLEAVED ? 16 : 8)] : xb[e];
                    const float va = ra, vb = rb;
                    ra = __builtin_fmaf(va, c[e], -vb * si[e]);
                    rb = __builtin_fmaf(va, si[e], vb * c[e]);
                }
                a[i].set(xa);
                a[i].template store<STREAM>(at[i] + first);
                if constexpr (!INTERLEAVED) {
                    b[i].set(xb);
                    b[i].template store<STREAM>(at[i] + second);
                }
            }
        }
    }
}

// Rows of fewer than eight pairs: a lane takes one.
template <class T, bool F8, bool INTERLEAVED>
__global__ __launch_bounds__(kThreads) void rope_shift_short_kernel(ShiftParams p) {
    const Place at0 = find_place(p);
    const int r = at0.r, l = at0.l, head0 = at0.head0;
    if constexpr (F8) saturate_f8();
    const int heads = min(kHeads, p.kv_heads - head0), per_token = heads * p.half;
    const int64_t len = min((int64_t)max(p.len[r], 0), p.shift_stride);
    const int32_t *shift = p.shift + ((int64_t)(p.shift_layers > 1 ? l : 0) * p.cache.num_reqs + r) * p.shift_heads * p.shift_stride;
    for (int64_t t0 = at0.tile * kTokens<F8>; t0 < len; t0 += (int64_t)p.tiles * kTokens<F8>) {
        const int n = (int)min((int64_t)kTokens<F8>, len - t0);
        for (int x = threadIdx.x; x < n * per_token; x += kThreads) {
            const int t = x / per_token, y = x - t * per_token, h = y / p.half, i = y - h * p.half;
            uint32_t row = 0;
            const int32_t id = block_of(p.cache, r, (uint32_t)(t0 + t), row);
            const int s = id < 0 ? 0 : shift[(p.shift_heads > 1 ? (int64_t)(head0 + h) * p.shift_stride : 0) + t0 + t];
            if (s == 0) continue;
            char *at = p.layers[l] + ((int64_t)((uint32_t)id * p.cache.block16 + row * p.cache.row16) << 4) +
                       (int64_t)(head0 + h) * p.cache.head_bytes;
            const int ia = INTERLEAVED ? 2 * i : i, ib = INTERLEAVED ? 2 * i + 1 : i + p.half;
            const double f[1] = {to_turns(p, i)};
            float c[1], si[1];
            sincos_turns(s, f, c, si);
            Elements<T, F8, 4> one;
            float v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
            float w[4];
            if constexpr (F8) {
                one.raw[0] = ((const uint8_t *)at)[ia] | (uint32_t)((const uint8_t *)at)[ib] << 8;
            } else {
                one.raw[0] = ((const uint16_t *)at)[ia] | (uint32_t)((const uint16_t *)at)[ib] << 16;
                one.raw[1] = 0;
            }
            one.get(w);
            v[0] = __builtin_fmaf(w[0], c[0], -w[1] * si[0]);
            v[1] = __builtin_fmaf(w[0], si[0], w[1] * c[0]);
            one.set(v);
            if constexpr (F8) {
                ((uint8_t *)at)[ia] = (uint8_t)one.raw[0];
                ((uint8_t *)at)[ib] = (uint8_t)(one.raw[0] >> 8);
            } else {
                ((uint16_t *)at)[ia] = (uint16_t)one.raw[0];
                ((uint16_t *)at)[ib] = (uint16_t)(one.raw[0] >> 16);
            }
        }
    }
}

template <class T, bool F8> void (*shift_kernel(bool interleaved, bool small, bool stream))(ShiftParams) {
    if (small) return interleaved ? rope_shift_short_kernel<T, F8, true> : rope_shift_short_kernel<T, F8, false>;
    if (interleaved) return rope_shift_kernel<T, F8, true, false>;
    return stream ? rope_shift_kernel<T, F8, false, true> : rope_shift_kernel<T, F8, false, false>;
}

}  // namespace
}  // namespace tkv

extern "C" {

int kv_rope_shift(const kv_layout *layout, void *const *h_layer_ptrs, const int32_t *d_block_tables, int32_t bt_stride,
                  int32_t num_reqs, const int32_t *d_len, int32_t max_len, int32_t layers, int32_t heads,
                  const int32_t *d_shift, int64_t shift_stride, const double *d_freqs, int32_t rot_dim, int32_t flags,
                  int32_t cache_dtype, void *stream) {
    int rc = tkv::check_cache(layout, cache_dtype);
    if (rc != KV_OK) return rc;
    if (!h_layer_ptrs || bt_stride <= 0 || num_reqs < 0 || max_len < 0 || shift_stride < 0) return KV_EINVAL;
    if ((layers != 1 && layers != layout->num_layers) || (heads != 1 && heads != layout->kv_heads)) return KV_EINVAL;
    if (rot_dim < 0 || rot_dim % 2 != 0 || rot_dim > layout->head_dim || (rot_dim > 0 && !d_freqs)) return KV_EINVAL;
    if (flags & ~(KV_ROPE_INTERLEAVED | KV_ROPE_INVERSE)) return KV_EINVAL;
    if (num_reqs > 0 && (!d_block_tables || !d_len || (!d_shift && shift_stride > 0))) return KV_EINVAL;
    if (((uintptr_t)d_block_tables & 3u) || ((uintptr_t)d_len & 3u) || ((uintptr_t)d_shift & 3u) || ((uintptr_t)d_freqs & 7u))
        return KV_EALIGN;
    tkv::ShiftParams p;
    for (int l = 0; l < layout->num_layers; ++l) {
        if (!h_layer_ptrs[l]) return KV_EINVAL;
        if ((uintptr_t)h_layer_ptrs[l] & 15u) return KV_EALIGN;
        p.layers[l] = (char *)h_layer_ptrs[l];
    }
    p.groups = (layout->kv_heads + tkv::kHeads - 1) / tkv::kHeads;
    const int64_t places = (int64_t)layout->num_layers * num_reqs * p.groups;
    if (layout->kv_heads > tkv::kMaxHeads || places >= tkv::kMaxBlocks) return KV_ELIMIT;
    if (num_reqs == 0 || shift_stride == 0 || rot_dim == 0) return KV_OK;
    kv_batch b = {};
    b.num_reqs = num_reqs;
    b.bt_stride = bt_stride;
    b.d_block_tables = d_block_tables;
    p.cache = tkv::make_paged(layout, nullptr, &b);
    p.len = d_len;
    p.shift = d_shift;
    p.shift_stride = shift_stride;
    p.freqs = d_freqs;
    p.shift_layers = layers;
    p.shift_heads = heads;
    p.kv_heads = layout->kv_heads;
    p.half = rot_dim / 2;
    p.units = (p.half + tkv::kPairs - 1) / tkv::kPairs;
    p.by_heads = tkv::make_divider((uint32_t)(layout->kv_heads % tkv::kHeads ? layout->kv_heads % tkv::kHeads : tkv::kHeads));
    p.sign = (flags & KV_ROPE_INVERSE) ? -1.0 : 1.0;
    const bool small = p.half < tkv::kPairs, inter = flags & KV_ROPE_INTERLEAVED;
    const bool lines = p.half * layout->elem_bytes % 128 == 0 && p.cache.head_bytes % 128 == 0;
    auto kernel = cache_dtype == KV_F8E4M3 ? tkv::shift_kernel<tkv::Bf16, true>(inter, small, lines)
                                           : (cache_dtype == KV_BF16 ? tkv::shift_kernel<tkv::Bf16, false>(inter, small, lines)
                                                                     : tkv::shift_kernel<tkv::F16, false>(inter, small, lines));
    const int tokens = cache_dtype == KV_F8E4M3 ? tkv::kTokens<true> : tkv::kTokens<false>;
    const int64_t tiles = ((int64_t)max_len + tokens - 1) / tokens;
    const int64_t most = tkv::kMaxBlocks / places;
    p.tiles = (int32_t)(tiles < 1 ? 1 : (tiles > most ? most : tiles));
    (void)hipGetLastError();
    hipLaunchKernelGGL(kernel, dim3((unsigned)(places * p.tiles)), dim3(tkv::kThreads), 0, (hipStream_t)stream, p);
    return hipGetLastError() == hipSuccess ? KV_OK : KV_EHIP;
}

}  // extern "C"
