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
    int32_t window, sink;
    bool causal;
    bool steady;               // 64 rows are whole tokens, and 128 span less than 2^30 bytes
    float *sums;               // [num_reqs * kv_heads][sink_tiles][parts][64], where a sink's rows are cut into parts
    int32_t sink_tiles, parts;
};

template <int DP> constexpr int kQueryRow = DP * 2 + 16;     // bytes of an LDS row: 8 rows on different banks

// A request's rows for one KV head.
struct Span {
    int64_t first, len;        // its first row of q; keys that have a sum
    int ntok;
    int64_t ahead;             // cache index of its first token
};

__device__ __forceinline__ Span find_span(const WeightParams &p, int r) {
    const int len = min(max(p.cache.kv_len[r], 0), kMaxLength);
    Span x;
    x.first = clamp_row(p.cache, p.cache.q_off[r]);
    x.ntok = (int)max((int64_t)0, clamp_row(p.cache, p.cache.q_off[r + 1]) - x.first);
    x.len = min((int64_t)len, p.weight_stride), x.ahead = len - x.ntok;
    return x;
}

constexpr uint32_t kNothing = 0xffc0deadu;     // a NaN that no lse is

template <int DP, int KW> struct Shape {
    static constexpr int RW = kWaves / KW, RT = KW > 2 ? 2 : 1, kRows = 32 * RW * RT, kKeys = kWaveKeys * KW;
};
template <int DP, int KW> struct __align__(16) TileLds {
    char rows[2][Shape<DP, KW>::kRows * kQueryRow<DP>];
    float base[2][Shape<DP, KW>::kRows];       // lse in units of log 2; kNothing for a row that adds nothing
    float parts[kWaves][kWaveKeys];
};

// What the keys tile0 .. tile0 + 64 KW - 1 receive from rows row_begin .. row_end - 1: of key t0 + lane of the wave's
// 64 keys, in the waves of the first group of rows.  The four waves take KW groups of 64 keys and 4 / KW groups of 32
// rows at a time; the rows go through LDS, one step ahead, for all of them.  A wave's products and exponentials take
// turns, with two waves on each SIMD to overlap them.  Chunks of 1,000 tokens over 4,000 in 4 requests, 32 heads on 8 of
// 128, 115 GFLOP in 154 to 156 us (740 TFLOP/s); of 2,000 over 6,000 with a window of 1,024 and 4 sinks, 67 GFLOP in 127
// to 130 us (520): the matrix units busy for 24 % of the time, the vector units for 41 %.  Products of the next rows
// beside the exponentials of these, with two sets of accumulators, need more registers than two waves on a SIMD leave.
template <class T, bool F8, int DP, int KW, bool SINK>
__device__ __forceinline__ float weigh_tile(const WeightParams &p, const Span &span, int r, int h, int tile0, int row_begin,
                                            int row_end, TileLds<DP, KW> &lds) {
    constexpr int KS = DP / 16, RW = Shape<DP, KW>::RW, RT = Shape<DP, KW>::RT, kRows = Shape<DP, KW>::kRows, VPR = DP / 8,
                  VL = kRows * VPR / kThreads;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, col = lane & 31, half = lane >> 5;
    const int kw = wave % KW, rw = wave / KW;
    const int64_t first = span.first, len = span.len, ahead = span.ahead;
    const float c = p.scale * (F8 && p.k_scale ? p.k_scale[h] : 1.0f);
    const int t0 = tile0 + kw * kWaveKeys;     // t0 + 63 may pass 2^31 - 1: no key is there
    u32x4 qreg[VL];
    float base = 0.0f;
    // Where this lane's vectors of a step lie behind the step's first token.  Where each pass of the lanes takes whole
    // rows and those are whole tokens, a pass lies as far behind the one before for all; else each has a place of its own.
    constexpr bool kWholeRows = kThreads % VPR == 0;
    constexpr int kOffsets = kWholeRows ? 1 : VL;
    const bool steady = p.steady && (!kWholeRows || kThreads / VPR % p.group == 0);
    const int64_t apart = kWholeRows ? (int64_t)divide(kThreads / VPR, p.by_group) * p.q_ts : 0;
    uint32_t off[kOffsets];
#pragma unroll
    for (int i = 0; i < kOffsets; ++i) {
        const uint32_t x = i * kThreads + tid, row = x / VPR, token = divide(row, p.by_group);
        off[i] = token * (uint32_t)p.q_ts + (row - token * p.group) * (uint32_t)p.q_hs + x % VPR * 16;
    }
    const auto load = [&](int row0) {
        if (steady && row0 + kRows <= row_end) {
            const char *at = p.q + (first + divide((uint32_t)row0, p.by_group)) * p.q_ts + (int64_t)h * p.group * p.q_hs;
            if (p.head_dim == DP) {
#pragma unroll
                for (int i = 0; i < VL; ++i) qreg[i] = *(const u32x4 *)(at + i * apart + off[i % kOffsets]);
            } else {
#pragma unroll
                for (int i = 0; i < VL; ++i) {
                    qreg[i] = u32x4{0, 0, 0, 0};
                    if ((i * kThreads + tid) % VPR * 8 < p.head_dim) qreg[i] = *(const u32x4 *)(at + i * apart + off[i % kOffsets]);
                }
            }
        } else {
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
        }
        if (tid < kRows) {
            const int row = row0 + tid, token = (int)divide(row, p.by_group);
            base = -INFINITY;
            if (row < row_end) base = p.lse[(first + token) * p.q_heads + h * p.group + row - token * p.group];
            base = base == -INFINITY ? __builtin_bit_cast(float, kNothing) : (base != base ? NAN : base * kLog2e);
        }
    };
    const auto stage = [&](int buf) {
#pragma unroll
        for (int i = 0; i < VL; ++i) {
            const int x = i * kThreads + tid;
            *(u32x4 *)(lds.rows[buf] + x / VPR * kQueryRow<DP> + x % VPR * 16) = qreg[i];
        }
        if (tid < kRows) lds.base[buf][tid] = base;
    };
    // The first rows are on their way while the keys are looked up and, of 8 bits, unpacked (64 requests of 20 rows over 4,000
    // tokens 158 us, 166 with them behind the keys).
    if (row_begin < row_end) load(row_begin);
    // this lane's two keys, as operands; the element order follows the rows'
    u32x4 kf[2][KS];
    int from[2], to[2];
#pragma unroll
    for (int x = 0; x < 2; ++x) {
        const int64_t t = (int64_t)t0 + x * 32 + col;
        uint32_t row = 0;
        const int32_t blk = t < len ? block_of(p.cache, r, (uint32_t)t, row) : -1;
        // the rows that see the key, causal from its own token on and up to the one whose window ends at it
        const int64_t tok = t - ahead;
        from[x] = blk < 0 ? 0 : (p.causal ? (int)min((int64_t)span.ntok, max((int64_t)0, tok)) * p.group : 0);
        to[x] = blk < 0 ? 0 : span.ntok * p.group;
        if (p.window > 0 && !(SINK && t < p.sink)) to[x] = min(to[x], (int)min((int64_t)span.ntok, max((int64_t)0, tok + p.window)) * p.group);
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
    // Of 32 rows the operands are read while the exponentials of the 32 before are taken, and their lse after that: from
    // the next step's buffer too, which is filled, with the step's one barrier, between the products and exponentials of
    // its last rows.
    u32x4 qf[KS];
    f32x4 b[4];
    float mark = 0.0f;                             // lse of row col
    const auto read = [&](int buf, int at) {
        const char *from = lds.rows[buf] + (at + col) * kQueryRow<DP>;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            const int d = F8 ? (ks / 2) * 32 + half * 16 + (ks & 1) * 8 : ks * 16 + half * 8;
            qf[ks] = *(const u32x4 *)(from + d * 2);
        }
    };
    const auto read_lse = [&](int buf, int at) {
#pragma unroll
        for (int g = 0; g < 4; ++g) b[g] = *(const f32x4 *)&lds.base[buf][at + g * 8 + half * 4];
        mark = lds.base[buf][at + col];
    };
    const auto below = [](int n) { return n >= 32 ? ~0u : (1u << max(n, 0)) - 1; };
    float sum[2] = {0.0f, 0.0f};
    f32x16 s[2];
    const auto products = [&]() {
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int e = 0; e < 16; ++e) s[x][e] = 0.0f;
        __builtin_amdgcn_sched_barrier(0);         // all reads are on their way before the first product waits
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            s[0] = T::mfma32(qf[ks], kf[0][ks], s[0]);
            s[1] = T::mfma32(qf[ks], kf[1][ks], s[1]);
        }
        __builtin_amdgcn_sched_barrier(0);
    };
    const auto exponentials = [&](int row0) {
        __builtin_amdgcn_sched_barrier(0);
        // which of the rows the lane's keys see
        const uint32_t add = (uint32_t)__ballot(__builtin_bit_cast(uint32_t, mark) != kNothing);
        uint32_t bits[2];
#pragma unroll
        for (int x = 0; x < 2; ++x) bits[x] = below(to[x] - row0) & ~below(from[x] - row0) & add;
        float part[2] = {0.0f, 0.0f};              // of these rows, so that long sums stay exact
        if (__all((bits[0] & bits[1]) == ~0u)) {
#pragma unroll
            for (int g = 0; g < 16; ++g)
#pragma unroll
                for (int x = 0; x < 2; ++x) part[x] += exp2_(__builtin_fmaf(s[x][g], c, -b[g / 4][g % 4]));
        } else if (__any((bits[0] | bits[1]) != 0u)) {
            bits[0] >>= 4 * half;                  // element g has bit 8 (g / 4) + g % 4
            bits[1] >>= 4 * half;
#pragma unroll
            for (int g = 0; g < 16; ++g)
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    const float v = exp2_(__builtin_fmaf(s[x][g], c, -b[g / 4][g % 4]));
                    const uint32_t on = (uint32_t)((int)(bits[x] << (31 - (8 * (g / 4) + g % 4))) >> 31);
                    part[x] += __builtin_bit_cast(float, __builtin_bit_cast(uint32_t, v) & on);
                }
        }
        sum[0] += part[0];
        sum[1] += part[1];
    };
    const int mine = rw * RT * 32;
    if (row_begin < row_end) {
        stage(0);
        __syncthreads();
        if (row_begin + kRows < row_end) load(row_begin + kRows);
        read(0, mine);
        read_lse(0, mine);
    }
    // Up to 32 rows, a request's that decodes in a batch of many rows, take one group: the others' products are left out
    // (these 64 requests: 4 us).
    const bool one = row_end - row_begin <= 32;
    if (one && row_begin < row_end && mine == 0) {
        products();
        exponentials(row_begin);
    }
    int buf = 0;
    for (int row0 = one ? row_end : row_begin; row0 < row_end; row0 += kRows, buf ^= 1) {
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            const int at = mine + rt * 32;
            products();
            int next = buf, next_at = at + 32;
            if (rt + 1 == RT) {
                next = buf ^ 1, next_at = mine;
                if (row0 + kRows < row_end) {
                    stage(next);
                    __syncthreads();
                    if (row0 + 2 * kRows < row_end) load(row0 + 2 * kRows);
                }
            }
            read(next, next_at);                   // (past the last step what an older one left, not used)
            exponentials(row0 + at);
            read_lse(next, next_at);
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
        lds.parts[wave][lane] = got;
        __syncthreads();
        if (rw == 0)
#pragma unroll
            for (int i = 1; i < RW; ++i) got += lds.parts[i * KW + kw][lane];
        __syncthreads();
    } else {
        __syncthreads();      // the rows' buffers are free for the next tile
    }
    return got;
}

template <class T, bool F8, int DP, int KW>
__global__ __launch_bounds__(kThreads, DP > 128 ? 1 : 2) void attention_weights_kernel(WeightParams p) {
    constexpr int kKeys = Shape<DP, KW>::kKeys;
    __shared__ TileLds<DP, KW> lds;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int h = (int)(blockIdx.x % p.kv_heads), r = (int)(blockIdx.x / p.kv_heads);
    const Span span = find_span(p, r);
    const int64_t len = span.len, ahead = span.ahead;
    const int ntok = span.ntok;
    float *out = p.weights + ((int64_t)r * p.kv_heads + h) * p.weight_stride;

    for (int64_t tile = blockIdx.y; tile * kKeys < len; tile += gridDim.y) {
        const int tile0 = (int)tile * kKeys;
        // rows that may see a key of the tile: from the token at its first key on (causal), to the one whose window
        // ends at its last key
        int tok0 = 0, tok1 = ntok;
        if (p.causal) tok0 = (int)min((int64_t)ntok, max((int64_t)0, (int64_t)tile0 - ahead));
        if (p.window > 0) tok1 = (int)max((int64_t)0, min((int64_t)ntok, (int64_t)tile0 + kKeys - 1 + p.window - ahead));
        float got = 0.0f;                          // (a window may have left all of them behind)
        if (tok0 < tok1) got = weigh_tile<T, F8, DP, KW, false>(p, span, r, h, tile0, tok0 * p.group, tok1 * p.group, lds);
        const int64_t key = (int64_t)tile0 + wave % KW * kWaveKeys + lane;
        if (wave / KW == 0 && key < len) out[key] = p.decay == 0.0f ? got : __builtin_fmaf(p.decay, out[key], got);
    }
}

// With a window only some of a request's keys have a row that sees them: the first `sink`, and those from `start` on.
// Of the others the sums only fade.
struct SinkKeys {
    int64_t sink, start;
};

__device__ __forceinline__ SinkKeys find_keys(const WeightParams &p, const Span &x) {
    if (x.ntok == 0) return {0, x.len};
    const int64_t sink = min((int64_t)p.sink, x.len);
    return {sink, min(x.len, max(sink, x.ahead - p.window + 1))};
}

// `threads` threads, this one the i-th: sums of keys that no row sees.
__device__ __forceinline__ void fade(const WeightParams &p, float *out, const SinkKeys &keys, int64_t i, int64_t threads) {
    if (p.decay == 1.0f) return;
    for (int64_t t = keys.sink + i; t < keys.start; t += threads) out[t] = p.decay == 0.0f ? 0.0f : p.decay * out[t];
}

// The keys of a window as above, each tile with the rows whose window reaches it.  All of a chunk's rows see the sinks:
// those are tiles of 64 keys of their own, whose rows four waves share and p.parts workgroups, which leave their sums
// to be joined; so that no workgroup passes many more rows than a window has.
template <class T, bool F8, int DP, int KW>
__global__ __launch_bounds__(kThreads, DP > 128 ? 1 : 2) void sink_weights_kernel(WeightParams p) {
    constexpr int kKeys = Shape<DP, KW>::kKeys;
    __shared__ union { TileLds<DP, KW> keys; TileLds<DP, 1> sinks; } lds;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int h = (int)(blockIdx.x % p.kv_heads), r = (int)(blockIdx.x / p.kv_heads);
    const Span span = find_span(p, r);
    const SinkKeys keys = find_keys(p, span);
    float *out = p.weights + ((int64_t)r * p.kv_heads + h) * p.weight_stride;
    const int own = p.sink_tiles * p.parts;
    if ((int)blockIdx.y < own) {
        const int part = (int)blockIdx.y % p.parts;
        for (int64_t tile = blockIdx.y / p.parts; tile * kWaveKeys < keys.sink; tile += p.sink_tiles) {
            const int tile0 = (int)tile * kWaveKeys;
            const int tok0 = p.causal ? (int)min((int64_t)span.ntok, max((int64_t)0, (int64_t)tile0 - span.ahead)) : 0;
            // whole tokens, so that parts hold whole rows of the group
            const int64_t n = span.ntok - tok0;
            const int from = tok0 + (int)(n * part / p.parts), to = tok0 + (int)(n * (part + 1) / p.parts);
            const float got = weigh_tile<T, F8, DP, 1, true>(p, span, r, h, tile0, from * p.group, to * p.group, lds.sinks);
            const int64_t key = (int64_t)tile0 + lane;
            if (wave != 0 || key >= keys.sink) continue;
            if (p.parts > 1) p.sums[(((int64_t)blockIdx.x * p.sink_tiles + tile) * p.parts + part) * kWaveKeys + lane] = got;
            else out[key] = p.decay == 0.0f ? got : __builtin_fmaf(p.decay, out[key], got);
        }
        return;
    }
    const int y = (int)blockIdx.y - own, blocks = (int)gridDim.y - own;
    fade(p, out, keys, (int64_t)y * kThreads + threadIdx.x, (int64_t)blocks * kThreads);
    for (int64_t tile = y; keys.start + tile * kKeys < span.len; tile += blocks) {
        const int64_t at = keys.start + tile * kKeys;
        const int tile0 = (int)at;
        int tok0 = 0;
        if (p.causal) tok0 = (int)min((int64_t)span.ntok, max((int64_t)0, at - span.ahead));
        const int tok1 = (int)max((int64_t)0, min((int64_t)span.ntok, at + kKeys - 1 + p.window - span.ahead));
        const float got = weigh_tile<T, F8, DP, KW, false>(p, span, r, h, tile0, tok0 * p.group, tok1 * p.group, lds.keys);
        const int64_t key = at + wave % KW * kWaveKeys + lane;
        if (wave / KW == 0 && key < span.len) out[key] = p.decay == 0.0f ? got : __builtin_fmaf(p.decay, out[key], got);
    }
}

// Sums over the parts of a sink's rows, in their order: one wave a tile of 64 sinks.
__global__ __launch_bounds__(64) void sink_weights_join_kernel(WeightParams p) {
    const int r = (int)(blockIdx.x / p.kv_heads);
    const SinkKeys keys = find_keys(p, find_span(p, r));
    const int64_t key = (int64_t)blockIdx.y * kWaveKeys + threadIdx.x;
    if (key >= keys.sink) return;
    const float *at = p.sums + ((int64_t)blockIdx.x * p.sink_tiles + blockIdx.y) * p.parts * kWaveKeys + threadIdx.x;
    float got = 0.0f;
    for (int i = 0; i < p.parts; ++i) got += at[(int64_t)i * kWaveKeys];
    float *out = p.weights + (int64_t)blockIdx.x * p.weight_stride + key;
    *out = p.decay == 0.0f ? got : __builtin_fmaf(p.decay, *out, got);
}

// Few rows (a decoded token's heads): nothing to share, so that each wave works
// alone on 64 keys, 16 rows at a time.  A lane has one key (lane % 16) and 4 of
// 16 rows.  Bound by the reads of K: the last 2,048 and first 4 tokens of 64
// requests, 8 KV heads of 128, 0.28 GB in 62 us (4.5 TB/s; 8 bits 32 us).
// AHEAD: a wave passes several tiles, the next one in a second set of registers
// on its way beside this one (where two fit: not 16-bit rows beyond 128 columns),
// its places looked up (64 requests of 4,096 tokens 111 us, 122 without).  Else
// most waves have one tile, whose keys are asked for before the rows: 512
// requests of 64 tokens 19 us, 35 with AHEAD; 1,024 of 100 72 and 98.  16-bit rows
// of up to 96 columns, of three pieces, are fastest that way also in long caches:
// 64 requests of 4,096 at head size 80 87 us, 91 with AHEAD, ragged ones around
// 4,000 93 and 109.  Heads of one block on one XCD are no faster.
template <class T, bool F8, int DP, bool SINK, bool AHEAD>
__global__ __launch_bounds__(kThreads, AHEAD && DP <= 128 ? 2 : 1) void attention_weights_few_kernel(WeightParams p) {
    constexpr int KS = DP / 32, LD = F8 ? KS / 2 : KS, KT = kWaveKeys / 16;
    constexpr int kSets = AHEAD && LD <= 4 ? 2 : 1;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = lane & 15, quad = lane >> 4;
    const int h = (int)(blockIdx.x % p.kv_heads), r = (int)(blockIdx.x / p.kv_heads);
    const Span span = find_span(p, r);
    const int64_t first = span.first, len = span.len, ahead = span.ahead;
    const int nrows = span.ntok * p.group;
    const float c = p.scale * (F8 && p.k_scale ? p.k_scale[h] : 1.0f);
    float *out = p.weights + ((int64_t)r * p.kv_heads + h) * p.weight_stride;

    // with a window, tiles of places: the sinks and, next to them, the keys from `start` on
    const SinkKeys keys = SINK ? find_keys(p, span) : SinkKeys{0, 0};
    const int places = (int)(len - (keys.start - keys.sink)), gap = (int)(keys.start - keys.sink);
    if constexpr (SINK) fade(p, out, keys, (int64_t)blockIdx.y * kThreads + threadIdx.x, (int64_t)gridDim.y * kThreads);
    const auto key_at = [&](int place) { return SINK && place >= (int)keys.sink ? place + gap : place; };
    // (places are at most 2^30, and the grid's tiles 2^23 apart: 32 bits)
    const int stride = (int)gridDim.y * kWaves * kWaveKeys, start = ((int)blockIdx.y * kWaves + wave) * kWaveKeys;

    // 16 rows: operands, and for this lane's four rows of the result what they see
    u32x4 qf[KS];
    float base[4];
    int lo[4], hi[4];
    const auto rows = [&](int row0) {
        const int mine = min(row0 + col, nrows - 1), token = (int)divide(mine, p.by_group);
        const char *qat = p.q + (first + token) * p.q_ts + (int64_t)(h * p.group + mine - token * p.group) * p.q_hs;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            const int d = F8 ? (ks / 2) * 64 + quad * 16 + (ks & 1) * 8 : ks * 32 + quad * 8;
            qf[ks] = d < p.head_dim ? *(const u32x4 *)(qat + d * 2) : u32x4{0, 0, 0, 0};
        }
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
    };
    int32_t id = -1;
    uint32_t id_row = 0;
    const auto look_up = [&](int t0) {
        id = t0 < places - lane ? block_of(p.cache, r, (uint32_t)key_at(t0 + lane), id_row) : -1;
    };
    u32x4 sets[kSets][KT][LD];
    uint64_t there[kSets];
    float old[kSets];
    const auto fetch = [&](int set, int t0) {
        there[set] = __ballot(id >= 0);
        const uint32_t off = id < 0 ? 0u : (uint32_t)id * p.cache.block16 + id_row * p.cache.row16;
        old[set] = p.decay != 0.0f && t0 < places - lane ? out[key_at(t0 + lane)] : 0.0f;
#pragma unroll
        for (int x = 0; x < KT; ++x)
            load_rows(sets[set][x], p.cache.head_bytes, [&](int row) {
                return p.cache.layer + (int64_t)h * p.cache.head_bytes + ((int64_t)(uint32_t)__shfl((int)off, x * 16 + row) << 4);
            });
    };
    const auto weigh = [&](int set, int t0) {
        u32x4(&kf)[KT][LD] = sets[set];
        float sum[KT];
#pragma unroll
        for (int x = 0; x < KT; ++x) sum[x] = 0.0f;
        if constexpr (AHEAD) {
#pragma unroll
            for (int x = 0; x < KT; ++x) arrange_rows(kf[x]);
        }
        for (int row0 = 0; row0 < nrows; row0 += 16) {
            if (!AHEAD || nrows > 16) rows(row0);
            if constexpr (!AHEAD) {
                if (row0 == 0) {                   // here, so that the rows above are on their way with the keys
#pragma unroll
                    for (int x = 0; x < KT; ++x) arrange_rows(kf[x]);
                }
            }
#pragma unroll
            for (int x = 0; x < KT; ++x) {
                f32x4 s = {0, 0, 0, 0};
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) {
                    if constexpr (F8) s = T::mfma16(qf[ks], unpack8<T>(kf[x][ks / 2][ks % 2 * 2], kf[x][ks / 2][ks % 2 * 2 + 1]), s);
                    else s = T::mfma16(qf[ks], kf[x][ks], s);
                }
                const int t = key_at(t0 + x * 16 + col);
                const bool in = (there[set] >> (x * 16 + col)) & 1;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float v = exp2_(__builtin_fmaf(s[i], c, -base[i]));
                    sum[x] += in && (t >= lo[i] || (SINK && t < p.sink)) && t < hi[i] ? v : 0.0f;
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
        if (t0 < places - lane) out[key_at(t0 + lane)] = p.decay == 0.0f ? got : __builtin_fmaf(p.decay, old[set], got);
    };
    if constexpr (!AHEAD) {
        for (int t0 = start; t0 < places; t0 += stride) {
            look_up(t0);
            fetch(0, t0);
            weigh(0, t0);
        }
    } else if constexpr (kSets == 1) {
        look_up(start);
        if (nrows > 0) rows(0);
        for (int t0 = start; t0 < places; t0 += stride) {
            fetch(0, t0);
            look_up(t0 + stride);
            weigh(0, t0);
        }
    } else {
        look_up(start);
        if (nrows > 0) rows(0);
        if (start < places) fetch(0, start);
        look_up(start + stride);
        for (int t0 = start; t0 < places; t0 += 2 * stride) {
            const int t1 = t0 + stride;
            if (t1 < places) fetch(1, t1);
            look_up(t1 + stride);
            weigh(0, t0);
            if (t1 >= places) break;
            if (t1 + stride < places) fetch(0, t1 + stride);
            look_up(t1 + 2 * stride);
            weigh(1, t1);
        }
    }
}

template <class T, bool F8, bool SINK, int DP> void (*weights_few_kernel_for(bool ahead))(WeightParams) {
    if constexpr (F8 || DP != 96) {
        if (ahead) return attention_weights_few_kernel<T, F8, DP, SINK, true>;
    }
    return attention_weights_few_kernel<T, F8, DP, SINK, false>;
}

template <class T, bool F8, bool SINK> auto weights_few_kernel(int head_dim, bool ahead) {
    if (head_dim <= 64) return weights_few_kernel_for<T, F8, SINK, 64>(ahead);
    if constexpr (!F8) {
        if (head_dim <= 96) return weights_few_kernel_for<T, F8, SINK, 96>(ahead);
    }
    if (head_dim <= 128) return weights_few_kernel_for<T, F8, SINK, 128>(ahead);
    return weights_few_kernel_for<T, F8, SINK, 256>(ahead);
}

template <bool SINK> auto weights_few_kernel(bool bf16, bool f8, int d, bool ahead) {
    return bf16 ? (f8 ? weights_few_kernel<Bf16, true, SINK>(d, ahead) : weights_few_kernel<Bf16, false, SINK>(d, ahead))
                : (f8 ? weights_few_kernel<F16, true, SINK>(d, ahead) : weights_few_kernel<F16, false, SINK>(d, ahead));
}

template <class T, bool F8, int KW, bool SINK, int DP> void (*weights_kernel_for())(WeightParams) {
    if constexpr (SINK) return sink_weights_kernel<T, F8, DP, KW>;
    else return attention_weights_kernel<T, F8, DP, KW>;
}

template <class T, bool F8, int KW, bool SINK> void (*weights_kernel(int head_dim))(WeightParams) {
    if (head_dim <= 64) return weights_kernel_for<T, F8, KW, SINK, 64>();
    if (head_dim <= 96) return weights_kernel_for<T, F8, KW, SINK, 96>();
    if (head_dim <= 128) return weights_kernel_for<T, F8, KW, SINK, 128>();
    return weights_kernel_for<T, F8, KW, SINK, 256>();
}

template <int KW, bool SINK> auto weights_kernel(bool bf16, bool f8, int d) {
    return bf16 ? (f8 ? weights_kernel<Bf16, true, KW, SINK>(d) : weights_kernel<Bf16, false, KW, SINK>(d))
                : (f8 ? weights_kernel<F16, true, KW, SINK>(d) : weights_kernel<F16, false, KW, SINK>(d));
}

template <bool SINK> auto weights_kernel(const WeightPlan &plan, bool bf16, bool f8, int d) {
    if (plan.few) return weights_few_kernel<SINK>(bf16, f8, d, plan.ahead);
    if constexpr (SINK) {
        if (plan.keys == 128) return weights_kernel<2, SINK>(bf16, f8, d);
    }
    return plan.keys == 64 ? weights_kernel<1, SINK>(bf16, f8, d) : weights_kernel<4, SINK>(bf16, f8, d);
}

int attention_weights(const kv_layout *layout, const void *d_layer, const kv_batch *batch, const kv_rows *q,
                      const float *d_lse, float scale, int32_t causal, int32_t window, int32_t sink,
                      int32_t cache_dtype, const float *d_k_scale, float decay, float *d_weights,
                      int64_t weight_stride, void *d_workspace, int64_t workspace_bytes, void *stream) {
    int rc = check_cache(layout, cache_dtype);
    if (rc == KV_OK) rc = check_batch(batch);
    if (rc == KV_OK) rc = check_rows(q, batch->num_q, layout->head_dim, false);
    if (rc != KV_OK) return rc;
    if (!d_layer || weight_stride < 0 || window < 0 || q->heads % layout->kv_heads != 0) return KV_EINVAL;
    if (cache_dtype != KV_F8E4M3 && cache_dtype != q->dtype) return KV_EINVAL;
    if (!(scale > 0.0f) || !isfinite(scale) || !isfinite(decay)) return KV_EINVAL;
    if (batch->num_reqs > 0 && weight_stride > 0 &&
        (!d_weights || !batch->d_q_off || !batch->d_kv_len || !batch->d_block_tables))
        return KV_EINVAL;
    if (batch->num_q > 0 && !d_lse) return KV_EINVAL;
    if (((uintptr_t)d_layer & 15u) || ((uintptr_t)d_lse & 3u) || ((uintptr_t)d_weights & 3u) || ((uintptr_t)d_workspace & 15u))
        return KV_EALIGN;
    WeightPlan plan;
    rc = plan_weights(layout, batch, q->heads, window, sink, &plan);
    if (rc != KV_OK) return rc;
    if (plan.workspace > 0 && !d_workspace) return KV_EINVAL;
    if (plan.workspace > workspace_bytes) return KV_ELIMIT;
    if (batch->num_reqs == 0 || weight_stride == 0) return KV_OK;
    WeightParams p;
    p.cache = make_paged(layout, d_layer, batch);
    p.q = (const char *)q->d_data;
    p.q_ts = q->token_stride * 2, p.q_hs = q->head_stride * 2;
    p.lse = d_lse;
    p.k_scale = cache_dtype == KV_F8E4M3 ? d_k_scale : nullptr;
    p.weights = d_weights;
    p.weight_stride = weight_stride;
    p.scale = scale * kLog2e;
    p.decay = decay;
    p.q_heads = q->heads;
    p.kv_heads = layout->kv_heads;
    p.group = q->heads / layout->kv_heads;
    p.by_group = make_divider((uint32_t)p.group);
    p.head_dim = layout->head_dim;
    p.window = window < kMaxLength ? window : 0;
    p.causal = causal != 0;
    p.steady = 64 % p.group == 0 && p.q_ts < (int64_t(1) << 22) && p.q_hs < (int64_t(1) << 22);
    p.sink = sink < kMaxLength ? sink : kMaxLength;
    p.sums = (float *)d_workspace;
    p.sink_tiles = plan.sink_tiles;
    p.parts = plan.parts;
    const int d = layout->head_dim;
    const bool bf16 = q->dtype == KV_BF16, f8 = cache_dtype == KV_F8E4M3;
    auto kernel = plan.windowed ? weights_kernel<true>(plan, bf16, f8, d) : weights_kernel<false>(plan, bf16, f8, d);
    const unsigned heads = (unsigned)(batch->num_reqs * layout->kv_heads);
    (void)hipGetLastError();
    hipLaunchKernelGGL(kernel, dim3(heads, (unsigned)(plan.tiles + plan.sink_tiles * plan.parts)), dim3(kThreads), 0,
                       (hipStream_t)stream, p);
    if (plan.parts > 1)
        hipLaunchKernelGGL(sink_weights_join_kernel, dim3(heads, (unsigned)plan.sink_tiles), dim3(64), 0, (hipStream_t)stream, p);
    return hipGetLastError() == hipSuccess ? KV_OK : KV_EHIP;
}

}  // namespace
}  // namespace tkv

extern "C" {

int kv_attention_weights(const kv_layout *layout, const void *d_layer, const kv_batch *batch, const kv_rows *q,
                         const float *d_lse, float scale, int32_t causal, int32_t window, int32_t cache_dtype,
                         const float *d_k_scale, float decay, float *d_weights, int64_t weight_stride, void *stream) {
    return tkv::attention_weights(layout, d_layer, batch, q, d_lse, scale, causal, window, -1, cache_dtype, d_k_scale, decay,
                                  d_weights, weight_stride, nullptr, 0, stream);
}

int kv_sink_weights(const kv_layout *layout, const void *d_layer, const kv_batch *batch, const kv_rows *q,
                    const float *d_lse, float scale, int32_t causal, int32_t window, int32_t sink, int32_t cache_dtype,
                    const float *d_k_scale, float decay, float *d_weights, int64_t weight_stride, void *d_workspace,
                    int64_t workspace_bytes, void *stream) {
    if (sink < 0) return KV_EINVAL;
    return tkv::attention_weights(layout, d_layer, batch, q, d_lse, scale, causal, window, sink, cache_dtype, d_k_scale,
                                  decay, d_weights, weight_stride, d_workspace, workspace_bytes, stream);
}

}  // extern "C"
