// attention.hip -- attention of new tokens over the paged cache.
//
// For a row i and the keys j it sees, s_ij = scale q_i.k_j, out_i = sum_j
// exp(s_ij - lse_i) v_j.  The keys are passed once, with the running maximum
// m and sum l of a softmax: adding keys with scores s makes
//     m' = max(m, s),  l' = l 2^(m-m') + sum 2^(s-m'),  o' = o 2^(m-m') + sum 2^(s-m') v
// (scores in units of log 2), and parts taken over different keys join by the
// same rule.  A row is a (token, head) pair: the heads that share a KV head
// are packed into one tile, so that K and V are read once for all of them.

#include <math.h>

#include <algorithm>
#include <type_traits>

#include "mfma.h"
#include "paged.h"

namespace tkv {
namespace {

constexpr int kWaves = 4;                  // of a workgroup that takes few rows, and of a join
constexpr int kThreads = 64 * kWaves;
constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;
static_assert(kSplitStep == 32 * kWaves, "a wave takes 32 keys a step");
static_assert(kTileStep == 64, "a lane looks up one key");

struct AttentionParams {
    Paged cache;
    const char *q;
    char *out;
    int64_t q_ts, q_hs, o_ts, o_hs;    // bytes
    float *lse;
    float *part_o;                     // [splits][num_q * q_heads][head_dim], then
    float *part_ml;                    // [splits][num_q * q_heads][2]: maximum (log 2) and sum
    const float *k_scale, *v_scale;
    int64_t tiles;
    float scale;                       // times log2 e
    Divider by_group;
    int32_t q_heads, kv_heads, group, head_dim;
    int32_t splits, window, sink;
    bool causal;
};

// The request, and the tile within it, of row tile `tile` for tiles of `rows`
// rows.  Request r starts at tile floor(q_off[r] * group / rows) + r, which
// leaves it at least ceil(n_r * group / rows) tiles: a map from the offsets
// alone, with at most one idle tile for each request.
struct Tile {
    int32_t req;
    int64_t first;      // the request's first row of q
    int row0;           // the tile's first row within the request (token * group + head)
    int rows;           // rows of the request
    int kv_len;
};

template <int ROWS> __device__ __forceinline__ Tile find_tile(const Paged &c, int tile, int group) {
    const int lane = threadIdx.x & 63;
    Tile t = {0, 0, 0, 0, 0};
    for (int base = 0; base < c.num_reqs; base += 64) {
        const int r = min(base + lane, c.num_reqs - 1);
        const int64_t first = clamp_row(c, c.q_off[r]), next = clamp_row(c, c.q_off[r + 1]);
        const int len = min(max(c.kv_len[r], 0), kMaxLength), tile0 = (int)first * group / ROWS + base + lane;
        // the last request that starts at or before the tile
        const int n = __popcll(__ballot(base + lane < c.num_reqs && tile0 <= tile));
        if (n == 0) break;
        const int at = n - 1;
        t.req = base + at;
        t.first = (int64_t)__builtin_amdgcn_readlane((int)first, at);    // below 2^30, as all rows together
        t.rows = max(0, __builtin_amdgcn_readlane((int)(next - first), at)) * group;
        t.row0 = (tile - __builtin_amdgcn_readlane(tile0, at)) * ROWS;
        t.kv_len = __builtin_amdgcn_readlane(len, at);
        if (n < 64) break;
    }
    return t;
}

__device__ __forceinline__ void store_out(const AttentionParams &p, int64_t row, int head, int d, f32x4 x, bool bf16) {
    char *to = p.out + row * p.o_ts + head * p.o_hs + d * 2;
    const u32x2 y = bf16 ? u32x2{pack2<Bf16>(x[0], x[1]), pack2<Bf16>(x[2], x[3])}
                         : u32x2{pack2<F16>(x[0], x[1]), pack2<F16>(x[2], x[3])};
    *(u32x2 *)to = y;
}

// One element of the cache.
template <class T, bool F8> __device__ __forceinline__ float load_one(const char *row, int d) {
    if constexpr (F8) return T::to_f32(T::from_f8(*(const uint8_t *)(row + d), false));
    return T::to_f32(*(const uint16_t *)(row + d * 2));
}

// A value that is the same in all lanes, as a scalar.
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ uint64_t uniform(uint64_t x) {
    return (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(x >> 32)) << 32 |
           (uint32_t)__builtin_amdgcn_readfirstlane((int)x);
}

// Start of part i of n steps cut into `parts`.
__device__ __forceinline__ int part_of(int n, int i, int parts) {
    return uniform(parts == 1 ? n * i : (int)((uint64_t)n * i / parts));
}

// LDS that the lanes of a wave exchange without a barrier: its accesses are in order, and this keeps them so in the code.
__device__ __forceinline__ void wave_fence() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront", "local");
    __builtin_amdgcn_wave_barrier();
}

// The keys that the rows of a tile see with a window and sinks: the request's first `sink` and, from the first key of
// the first row's window on, all up to the last row's last.  A body passes them as one run of places, so that the keys
// between cost no steps and neither range is rounded to whole steps: key t is place t below `sink` and place t - gap
// behind the gap, which is empty where the window begins among the sinks.
struct Run {
    int sink, gap;
};

__device__ __forceinline__ Run find_run(int sink, int first) { return {sink, max(0, first - sink)}; }
// The key at a place, and of a row's bound (its first key in the window, or one past its last) the place.
__device__ __forceinline__ int key_at(const Run &x, int place) { return place + (place < x.sink ? 0 : x.gap); }
__device__ __forceinline__ int place_of(const Run &x, int key) { return max(key - x.gap, min(key, x.sink)); }

// Columns that few_rows takes for a head of up to `dim`: of an 8-bit cache whole vectors of 16 elements for all lanes.
template <bool F8> constexpr int few_dim(int dim) { return F8 && dim == 96 ? 128 : dim; }

// Bytes of LDS that a body needs.
template <int DP, int W> constexpr int kSplitLds = W * 32 * (DP * 2 + 32);

// Tiles of 16 rows; the keys of a tile are cut into p.splits parts, one
// workgroup each, and a part's steps of 32 keys go to its waves in turn.
// S^T = K Q^T leaves a lane with the scores of one row (lane % 16) for the
// keys 4 (lane / 16) + i of either half of the step, which is where the
// second product, O^T = V^T P^T, wants them if V's keys are taken in the same
// order; so P never leaves its registers.  K is loaded from memory as the
// matrix operand itself; V goes through LDS, the wave's own, to be read
// transposed.  Waves share nothing until the end, so that there is no barrier
// in the loop and each keeps the next step's K and V on their way.
// Bound by the reads of the cache: 64 requests of 4,096 tokens, 8 KV heads of
// 128, 1.07 GB in 207 us (5.2 TB/s); 8 of 32,768 in 8 bits, 0.54 GB in 128 us
// (4.2 TB/s); the last 4,096 and first 4 of 64 requests of 8,192, 1.08 GB in 205
// us (5.3 TB/s).  P is rounded to the type of the products, as the matrix units
// take it: relative to the running maximum, after its sum.  That adds 12 to 19 %
// to the error of results that are rounded to bf16 alone (0.0017 to 0.0020 of
// their size; chunks 0.0023).  Sums and statistics stay in 32 bits.
template <class T, bool F8, int DP, int W, bool SINK>
__device__ __forceinline__ void few_rows(const AttentionParams &p, const Tile &tile, int h, int split, char *lds,
                                         float (*part)[16][2], int *odd) {
    constexpr int KS = DP / 32, LD = F8 ? KS / 2 : KS, DT = DP / 16;
    constexpr int NS = F8 ? 2 : 1, kWide = 32 * NS;    // an 8-bit cache takes two steps at a time: as many bytes
    constexpr int kRow = DP * 2 + 32;          // bytes of an LDS row: 8 rows lie on different banks
    constexpr int VEC = F8 ? 16 : 8;           // elements of a 16-byte vector of the cache
    constexpr int VPR = DP / VEC;              // vectors of a row
    constexpr int VL = 32 * VPR / 64;          // vectors a lane stages
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = lane & 15, quad = lane >> 4;

    // this lane's row
    const int myrow = tile.row0 + col;
    const bool have = myrow < tile.rows;
    const int token = have ? (int)divide(myrow, p.by_group) : 0;
    const int head = h * p.group + (have ? myrow - token * p.group : 0);
    const int32_t len_raw = tile.kv_len;
    const int64_t len = min((int64_t)(len_raw < 0 ? 0 : len_raw), (int64_t)p.cache.bt_stride * p.cache.block_size);
    const int64_t ahead = (int64_t)len_raw - divide(tile.rows, p.by_group);    // cache index of the first token
    const int64_t pos = ahead + token, pos_first = ahead + divide(tile.row0, p.by_group);
    const int64_t pos_last = ahead + divide(min(tile.row0 + 15, tile.rows - 1), p.by_group);
    // keys this lane's row sees: lo <= j < hi; and those that some or all rows of the tile see
    const int64_t hi64 = p.causal ? min(len, pos + 1) : len, lo64 = p.window > 0 ? max((int64_t)0, pos - p.window + 1) : 0;
    int hi = have ? (int)max((int64_t)0, hi64) : 0, lo = (int)lo64;
    int end = (int)max((int64_t)0, p.causal ? min(len, pos_last + 1) : len);
    int begin = (int)(p.window > 0 ? max((int64_t)0, pos_first - p.window + 1) : 0);
    int all_hi = (int)max((int64_t)0, p.causal ? min(len, pos_first + 1) : len);
    int all_lo = (int)(p.window > 0 ? max((int64_t)0, pos_last - p.window + 1) : 0);
    Run run = {0, 0};
    if constexpr (SINK) {                      // from here on all of these, and t, are places
        run = find_run(p.sink, begin);
        hi = place_of(run, hi), lo -= run.gap, end = place_of(run, end);
        all_hi = place_of(run, all_hi), all_lo -= run.gap, begin = 0;
    }
    begin &= ~(kWide - 1);
    const int steps = end > begin ? (end - begin + kWide - 1) / kWide : 0;
    const int step0 = part_of(steps, split, p.splits), step1 = part_of(steps, split + 1, p.splits);

    const float c = p.scale * (F8 && p.k_scale ? p.k_scale[h] : 1.0f);
    const char *kbase = p.cache.layer + (int64_t)h * p.cache.head_bytes;
    const char *vbase = kbase + p.cache.kv_stride;
    char *mine = lds + wave * 32 * kRow;
    const auto is_mixed = [&](uint32_t there, int t0) {
        return there != 0xffffffffu || (t0 < all_lo && !(SINK && t0 + 32 <= run.sink)) || t0 + 32 > all_hi;
    };
    if (threadIdx.x == 0) *odd = 0;
    __syncthreads();

    // one step ahead: a lane looks up a key (lanes 32..63 those of the other half, or the same ones), then all load
    int32_t id = -1;
    uint32_t id_row = 0;
    uint64_t there_next = 0;
    u32x4 kreg[2 * NS][LD], vreg[VL * NS];
    const auto look_up = [&](int step) {
        const int t = begin + step * kWide + (lane & (kWide - 1));
        id = step < step1 && t < end ? block_of(p.cache, tile.req, (uint32_t)(SINK ? key_at(run, t) : t), id_row) : -1;
    };
    const auto offset = [&]() { return id < 0 ? 0u : (uint32_t)id * p.cache.block16 + id_row * p.cache.row16; };
    const auto load = [&]() {
        const uint32_t off = offset();
        there_next = __ballot(id >= 0);
#pragma unroll
        for (int x = 0; x < 2 * NS; ++x) {
            const char *at = kbase + ((int64_t)(uint32_t)__shfl((int)off, x * 16 + col) << 4) + quad * 16;
#pragma unroll
            for (int ks = 0; ks < LD; ++ks)
                kreg[x][ks] = ks * 64 + quad * 16 < p.cache.head_bytes ? *(const u32x4 *)(at + ks * 64) : u32x4{0, 0, 0, 0};
        }
#pragma unroll
        for (int i = 0; i < VL * NS; ++i) {
            const int x = i * 64 + lane, r = x / VPR, vec = x % VPR;
            const char *at = vbase + ((int64_t)(uint32_t)__shfl((int)off, r) << 4);
            vreg[i] = vec * 16 < p.cache.head_bytes ? *(const u32x4 *)(at + vec * 16) : u32x4{0, 0, 0, 0};
        }
    };
    look_up(step0 + wave);
    u32x4 qf[KS];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
        // an 8-bit cache is loaded 16 elements at a time, so its lanes hold the head's elements in another order
        const int d = F8 ? (ks / 2) * 64 + quad * 16 + (ks & 1) * 8 : ks * 32 + quad * 8;
        qf[ks] = u32x4{0, 0, 0, 0};
        if (have && d < p.head_dim) qf[ks] = *(const u32x4 *)(p.q + (tile.first + token) * p.q_ts + head * p.q_hs + d * 2);
    }
    if (step0 + wave < step1) load();
    look_up(step0 + wave + W);

    f32x4 o[DT];
#pragma unroll
    for (int i = 0; i < DT; ++i) o[i] = f32x4{0, 0, 0, 0};
    float m = -INFINITY, l = 0.0f;

    for (int step = step0 + wave; step < step1; step += W) {
        const uint64_t there_now = there_next;
#pragma unroll
        for (int n = 0; n < NS; ++n) {
        const int t0 = begin + step * kWide + n * 32;
        const uint32_t there = (uint32_t)(there_now >> (n * 32));
        // A value that is not finite must reach only the rows that see its key: 0 times it is NaN.  In a step that some
        // row does not see whole, such values are staged as 0, and added below to the results that do see them.
        const bool mixed = is_mixed(there, t0);
        wave_fence();                          // the step before is read
#pragma unroll
        for (int i = 0; i < VL; ++i) {
            const int x = i * 64 + lane, r = x / VPR, vec = x % VPR;
            u32x4 y[F8 ? 2 : 1];
            if constexpr (F8) {
                y[0] = unpack8<T>(vreg[n * VL + i][0], vreg[n * VL + i][1]);
                y[1] = unpack8<T>(vreg[n * VL + i][2], vreg[n * VL + i][3]);
            } else {
                y[0] = vreg[n * VL + i];
            }
#pragma unroll
            for (int j = 0; j < (F8 ? 2 : 1); ++j) {
                if (mixed && T::drop_nonfinite(y[j])) *odd = 1;
                *(u32x4 *)(mine + r * kRow + vec * VEC * 2 + j * 16) = y[j];
            }
        }
        wave_fence();
        f32x4 s[2];
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            s[x] = f32x4{0, 0, 0, 0};
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                if constexpr (F8) s[x] = T::mfma16(unpack8<T>(kreg[n * 2 + x][ks / 2][(ks & 1) * 2], kreg[n * 2 + x][ks / 2][(ks & 1) * 2 + 1]), qf[ks], s[x]);
                else s[x] = T::mfma16(kreg[n * 2 + x][ks], qf[ks], s[x]);
            }
        }
        if (n == NS - 1) {
            if (step + W < step1) load();
            look_up(step + 2 * W);
        }
        float top = -INFINITY;
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int k = x * 16 + quad * 4 + i;
                const bool see = !mixed || (((there >> k) & 1) && (t0 + k >= lo || (SINK && t0 + k < run.sink)) && t0 + k < hi);
                s[x][i] = see ? s[x][i] * c : -INFINITY;
                top = fmaxf(top, s[x][i]);
            }
        top = fmaxf(top, __shfl_xor(top, 16));
        const f32x2 tops = both_halves(top);
        const float m1 = fmaxf(m, fmaxf(tops[0], tops[1])), base = m1 == -INFINITY ? 0.0f : m1;
        const float fade = exp2_(m - base);
        m = m1;
        l *= fade;
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                s[x][i] = exp2_(s[x][i] - base);
                l += s[x][i];
            }
        const u32x4 pf = {pack2<T>(s[0][0], s[0][1]), pack2<T>(s[0][2], s[0][3]), pack2<T>(s[1][0], s[1][1]),
                          pack2<T>(s[1][2], s[1][3])};
#pragma unroll
        for (int i = 0; i < DT; ++i) {
            const char *at = mine + (quad * 4 + (col >> 2)) * kRow + i * 32 + (col & 3) * 8;
            const u32x2 a = read_transposed(at), b = read_transposed(at + 16 * kRow);
#pragma unroll
            for (int e = 0; e < 4; ++e) o[i][e] *= fade;
            o[i] = T::mfma16(u32x4{a[0], a[1], b[0], b[1]}, pf, o[i]);
        }
        }
    }
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);

    // join the waves' parts
    wave_fence();
    float *po = (float *)mine;                 // [16][DP + 4]
#pragma unroll
    for (int i = 0; i < DT; ++i) *(f32x4 *)(po + col * (DP + 4) + i * 16 + quad * 4) = o[i];
    if (quad == 0) {
        part[wave][col][0] = m;
        part[wave][col][1] = l;
    }
    __syncthreads();
    const int64_t all = p.cache.num_q * p.q_heads;
    for (int x = threadIdx.x; x < 16 * DP / 4; x += (64 * W)) {
        const int r = x / (DP / 4), d = x % (DP / 4) * 4;
        const int row = tile.row0 + r, tok = (int)divide(row, p.by_group);
        if (row >= tile.rows || d >= p.head_dim) continue;
        const int64_t q = tile.first + tok;
        const int hd = h * p.group + row - tok * p.group;
        float mm = -INFINITY, ll = 0.0f;
#pragma unroll
        for (int w = 0; w < W; ++w) mm = fmaxf(mm, part[w][r][0]);
        const float base = mm == -INFINITY ? 0.0f : mm;
        f32x4 acc = {0, 0, 0, 0};
#pragma unroll
        for (int w = 0; w < W; ++w) {
            const float by = exp2_(part[w][r][0] - base);
            ll += part[w][r][1] * by;
            const f32x4 y = *(const f32x4 *)((const float *)(lds + w * 32 * kRow) + r * (DP + 4) + d);
            if (by != 0.0f) acc += y * by;     // a part that saw nothing holds zeros
        }
        if (p.splits > 1) {
            *(f32x4 *)(p.part_o + ((int64_t)split * all + q * p.q_heads + hd) * p.head_dim + d) = acc;
            if (d == 0) {
                float *ml = p.part_ml + ((int64_t)split * all + q * p.q_heads + hd) * 2;
                ml[0] = mm;
                ml[1] = ll;
            }
            continue;
        }
        const bool empty = ll == 0.0f;         // (scores that are all NaN leave the maximum as it began, and a sum of NaN)
        const float by = empty ? 0.0f : (F8 && p.v_scale ? p.v_scale[h] : 1.0f) / ll;
        store_out(p, q, hd, d, empty ? f32x4{0, 0, 0, 0} : acc * by, T::kBf16);
        if (d == 0 && p.lse) p.lse[q * p.q_heads + hd] = empty ? -INFINITY : (mm + log2_(ll)) * kLn2;
    }
    if (!*odd) return;
    __syncthreads();
    // the values staged as 0, to the elements just written
    for (int step = step0; step < step1; ++step) {
        const int t0 = begin + step * kWide;
        look_up(step);
        const uint32_t off = offset();
        const uint64_t in = __ballot(id >= 0);
        if (!is_mixed((uint32_t)in, t0) && (NS == 1 || !is_mixed((uint32_t)(in >> 32), t0 + 32))) continue;
        for (int k = 0; k < kWide; ++k) {
            const char *v = vbase + ((int64_t)(uint32_t)__shfl((int)off, k) << 4);
            if (!((in >> k) & 1)) continue;
            for (int x = threadIdx.x; x < 16 * p.head_dim; x += (64 * W)) {
                const int r = x / p.head_dim, d = x - r * p.head_dim, row = tile.row0 + r, tok = (int)divide(row, p.by_group);
                const int64_t at = ahead + tok;
                const int t = SINK ? key_at(run, t0 + k) : t0 + k;
                if (row >= tile.rows || (p.causal && t > at)) continue;
                if (p.window > 0 && t <= at - p.window && !(SINK && t < p.sink)) continue;
                const float y = load_one<T, F8>(v, d);
                if (fabsf(y) < INFINITY) continue;
                const int64_t q = tile.first + tok;
                const int hd = h * p.group + row - tok * p.group;
                if (p.splits > 1) {
                    p.part_o[((int64_t)split * all + q * p.q_heads + hd) * p.head_dim + d] += y;
                } else {
                    uint16_t *to = (uint16_t *)(p.out + q * p.o_ts + hd * p.o_hs) + d;
                    *to = (uint16_t)pack2<T>(T::to_f32(*to) + y, 0.0f);
                }
            }
        }
    }
}

// Tiles of 32 rows a wave over steps of 64 keys.  K and V of a step go
// through LDS for all waves: loaded into registers one step ahead or two,
// written to the other buffer, one barrier a step.
// Again S^T = K Q^T and O^T = V^T P^T, with 32 x 32 products: a lane holds
// one row's scores for half of the keys, so that a row's maximum and sum need
// one exchange between lanes.  Steps are bound by the issue of exponentials,
// LDS reads and products beside one another: 8 chunks of 2,048 tokens over
// 4,096, 32 heads on 8 of 128, 825 GFLOP in 840 to 890 us (930 to 980 TFLOP/s,
// by card), the matrix units busy for 43 % of the time, the vector units for 45 %;
// head size 80 with a window of 1,024, ragged, 61 to 65 us (330 to 350 TFLOP/s of
// what the rows see).  Four prompts of 4,096 with a window of 1,024 and 4 sinks,
// 241 GFLOP in 324 to 340 us (710 to 745): of a workgroup's 47 us 4 go before its
// first step and 2 behind its last, and its 18 steps hold 1,152 keys, of which a
// row sees 1,028.  The scores of the next step beside the exponentials of this
// one take 3 % longer, 64 rows a wave (half of the LDS reads, one wave on a SIMD)
// half as long again.
//
// The running maximum may lag: o and l are only scaled when some row's
// maximum has grown by more than 2^kLag since it was last taken.  Until then
// exponentials reach 2^kLag instead of 1, which costs no precision, neither in
// l and o (32 bits) nor in P (a rounding relative to its size; 2^8 is far
// below the 16-bit types' ends).  P is rounded to the type of the products, as
// the matrix units take it, which adds about a third to the error of results that
// are rounded alone: 0.0022 against 0.0016 of their size in bf16, 0.00029 against
// 0.00021 in f16; l sums what was not rounded.
constexpr float kLag = 8.0f;
constexpr int kStep = kTileStep;
template <int DP> constexpr int kKeyRow = DP * 2 + 16;     // bytes of an LDS row of K: 8 rows on different banks
template <int DP> constexpr int kValueRow = DP * 2 + (DP * 2 % 128 ? 0 : 64);   // of V: 4 rows, 64 bytes of each
template <int DP> constexpr int kTileLds = 2 * kStep * (kKeyRow<DP> + kValueRow<DP>);

// Steps that a tile's loads are ahead: two of an 8-bit cache in 96 columns (a ragged batch at head size 80 with a window 52
// against 54 us, 4 chunks of 1,000 tokens over 4,000 at 96 213 and 217, though 8 of 2,048 over 4,096 692 and 688), else one:
// the second set of registers costs more than it gives (8 bits at 64 columns, 4 chunks of 1,000 over 4,000 165 against 158
// us; at 128, 64 chunks of 20 over 2,020 123 and 113, 8 of 2,048 over 4,096 813 and 806).
template <bool F8, int DP> constexpr int ahead_of = F8 && DP == 96 ? 2 : 1;

// Where a step's keys lie (16-byte units from a plane's start), and which of
// them are in the cache.
struct Places {
    uint32_t at[kStep];
    uint64_t there;
};

template <class T, bool F8, int DP, int W, bool SINK>
__device__ __forceinline__ void many_rows(const AttentionParams &p, const Tile &tile, int h, int split, char *lds,
                                          int *odd, Places *places) {
    constexpr int KS = DP / 16, DT = DP / 32, kThreads = 64 * W, kRows = 32 * W;
    constexpr int VEC = F8 ? 16 : 8, VPR = DP / VEC, kVecs = kStep * VPR, VL = (kVecs + kThreads - 1) / kThreads;
    constexpr int kAhead = ahead_of<F8, DP>;
    const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), col = lane & 31, half = lane >> 5;
    char *const kbuf = lds, *const vbuf = lds + 2 * kStep * kKeyRow<DP>;

    const int wrow = tile.row0 + wave * 32, myrow = wrow + col, last_row = tile.rows - 1;
    const bool have = myrow < tile.rows;
    const int token = have ? (int)divide(myrow, p.by_group) : 0;
    const int head = h * p.group + (have ? myrow - token * p.group : 0);
    const int len_raw = tile.kv_len;
    const int len = uniform((int)min((int64_t)len_raw, (int64_t)p.cache.bt_stride * p.cache.block_size));
    const int ahead = len_raw - (int)divide(tile.rows, p.by_group);    // cache index of the first token
    // keys that rows see, lo <= j < hi: this lane's, those that all of the wave's rows see, and all of the tile's
    const auto hi_of = [&](int tok) { return max(0, p.causal ? min(len, ahead + tok + 1) : len); };
    const auto lo_of = [&](int tok) { return p.window > 0 ? max(0, ahead + tok - p.window + 1) : 0; };
    const auto token_of = [&](int row) { return uniform((int)divide(min(row, last_row), p.by_group)); };
    int hi = have ? hi_of(token) : 0, lo = lo_of(token);
    const int wfirst = token_of(wrow), wlast = token_of(wrow + 31), first = token_of(tile.row0), last = token_of(tile.row0 + kRows - 1);
    int all_hi = uniform(hi_of(wfirst)), all_lo = uniform(lo_of(wlast));
    int tile_hi = uniform(hi_of(first)), tile_lo = uniform(lo_of(last));
    int end = uniform(hi_of(last)), begin = uniform(lo_of(first));
    Run run = {0, 0};
    if constexpr (SINK) {                      // from here on all of these, and t, are places
        run = find_run(p.sink, begin);
        hi = place_of(run, hi), lo -= run.gap, end = place_of(run, end);
        all_hi = place_of(run, all_hi), all_lo -= run.gap;
        tile_hi = place_of(run, tile_hi), tile_lo -= run.gap, begin = 0;
    }
    begin &= ~(kStep - 1);
    const int steps = end > begin ? (end - begin + kStep - 1) / kStep : 0;
    const int step0 = part_of(steps, split, p.splits), step1 = part_of(steps, split + 1, p.splits);

    u32x4 qf[KS];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
        const int d = ks * 16 + half * 8;
        qf[ks] = u32x4{0, 0, 0, 0};
        if (have && d < p.head_dim) qf[ks] = *(const u32x4 *)(p.q + (tile.first + token) * p.q_ts + head * p.q_hs + d * 2);
    }
    const float c = p.scale * (F8 && p.k_scale ? p.k_scale[h] : 1.0f);
    const char *kbase = p.cache.layer + (int64_t)h * p.cache.head_bytes;
    const char *vbase = kbase + p.cache.kv_stride;

    uint64_t there = 0, there_next[kAhead];    // bit k: key k of the step is in the cache
    const auto is_mixed = [&](uint64_t there, int t0) {
        return there != ~uint64_t(0) || (t0 < tile_lo && !(SINK && t0 + kStep <= run.sink)) || t0 + kStep > tile_hi;
    };
    if (tid == 0) *odd = 0;

    // Staging.  One wave, in turn, looks up the keys of a step, a lane each, and leaves their places for all: the
    // table's entries are asked for kAhead + 2 steps ahead and looked at one step later.  kAhead steps ahead all load
    // the vectors x = i kThreads + tid.
    const int32_t *const table = p.cache.bt + (int64_t)tile.req * p.cache.bt_stride;
    u32x4 kregs[kAhead][VL], vregs[kAhead][VL];
    int32_t id = -1;
    uint32_t id_row = 0;
    const auto ask = [&](int step) {
        const uint32_t t = begin + step * kStep + lane, key = SINK ? key_at(run, t) : t, blk = divide(key, p.cache.by_block);
        id_row = key - blk * p.cache.block_size;
        id = -1;
        if (step < step1 && t < (uint32_t)end) id = table[blk];        // t < end <= the table's span
    };
    const auto leave = [&](int step) {
        const bool in = (uint32_t)id < p.cache.blocks;
        const uint64_t mask = __ballot(in);
        places[step & 3].at[lane] = in ? (uint32_t)id * p.cache.block16 + id_row * p.cache.row16 : 0u;
        if (lane == 0) places[step & 3].there = mask;
    };
    const auto load = [&](int slot, int step) {
        const Places &from = places[step & 3];
        u32x4(&kreg)[VL] = kregs[slot], (&vreg)[VL] = vregs[slot];
        there_next[slot] = uniform(from.there);
        uint32_t at[VL];
#pragma unroll
        for (int i = 0; i < VL; ++i) at[i] = from.at[(i * kThreads + tid) / VPR % kStep];
#pragma unroll
        for (int i = 0; i < VL; ++i) {
            // (past a head narrower than DP its last vector is read again, and dropped in stage)
            const int vec = min((i * kThreads + tid) % VPR, p.cache.head_bytes / 16 - 1);
            const uint64_t x = ((uint64_t)at[i] + vec) << 4;
            kreg[i] = *(const u32x4 *)(kbase + x);
            vreg[i] = *(const u32x4 *)(vbase + x);
        }
    };
    // A value that is not finite must reach only the rows that see its key: 0 times it is NaN.  In a step that some
    // row does not see whole, such values are staged as 0; below they are added to the results that do see them.
    const auto stage = [&](int buf, int slot, int step) {
        u32x4(&kreg)[VL] = kregs[slot], (&vreg)[VL] = vregs[slot];
        const bool mixed = is_mixed(there_next[slot], begin + step * kStep);
        if (p.head_dim < DP) {
#pragma unroll
            for (int i = 0; i < VL; ++i)
                if ((i * kThreads + tid) % VPR * VEC >= p.head_dim) kreg[i] = vreg[i] = u32x4{0, 0, 0, 0};
        }
#pragma unroll
        for (int i = 0; i < VL; ++i) {
            const int x = i * kThreads + tid, r = x / VPR, vec = x % VPR;
            if (kVecs % kThreads && x >= kVecs) break;         // (whole waves; what they loaded is not used)
            char *k = kbuf + (buf * kStep + r) * kKeyRow<DP> + vec * VEC * 2;
            char *v = vbuf + (buf * kStep + r) * kValueRow<DP> + vec * VEC * 2;
            u32x4 y[F8 ? 2 : 1];
            if constexpr (F8) {
                *(u32x4 *)k = unpack8<T>(kreg[i][0], kreg[i][1]);
                *(u32x4 *)(k + 16) = unpack8<T>(kreg[i][2], kreg[i][3]);
                y[0] = unpack8<T>(vreg[i][0], vreg[i][1]);
                y[1] = unpack8<T>(vreg[i][2], vreg[i][3]);
            } else {
                *(u32x4 *)k = kreg[i];
                y[0] = vreg[i];
            }
#pragma unroll
            for (int j = 0; j < (F8 ? 2 : 1); ++j) {
                if (mixed && T::drop_nonfinite(y[j])) *odd = 1;
                *(u32x4 *)(v + j * 16) = y[j];
            }
        }
    };

    f32x16 o[DT];
#pragma unroll
    for (int i = 0; i < DT; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[i][e] = 0.0f;
    float m = -INFINITY, base = 0.0f, l = 0.0f;

    if (wave < kAhead + 2) {
        ask(step0 + wave);
        leave(step0 + wave);
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kAhead; ++i)
        if (step0 + i < step1) load(i, step0 + i);
    const auto take = [&](auto buf, int step) {
        const int t0 = begin + step * kStep, slot = kAhead > 1 ? (int)buf : 0;
        stage(buf, slot, step);
        there = there_next[slot];
        __syncthreads();
        if (step + kAhead < step1) load(slot, step + kAhead);
        const int turn = (step - step0) % W;
        if (wave == (turn + kAhead + 1) % W && step > step0) leave(step + kAhead + 1);
        if (wave == (turn + kAhead + 2) % W) ask(step + kAhead + 2);

        // S: the reads of K are ahead of the products, of the second half among those of the first
        f32x16 s[2];
        const char *kat = kbuf + (buf * kStep + col) * kKeyRow<DP> + half * 16;
        u32x4 kf[2][KS];
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) kf[0][ks] = *(const u32x4 *)(kat + ks * 32);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int e = 0; e < 16; ++e) s[x][e] = 0.0f;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            s[0] = T::mfma32(kf[0][ks], qf[ks], s[0]);
            kf[1][ks] = *(const u32x4 *)(kat + 32 * kKeyRow<DP> + ks * 32);
            __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) s[1] = T::mfma32(kf[1][ks], qf[ks], s[1]);
        // V for the first 16 keys
        const char *vat = vbuf + (buf * kStep + half * 4 + (lane >> 2 & 3)) * kValueRow<DP> + (lane >> 4 & 1) * 32 + (lane & 3) * 8;
        u32x4 vf[2][DT];
        const auto read_v = [&](int kk) {
#pragma unroll
            for (int i = 0; i < DT; ++i) {
                const char *at = vat + kk * 16 * kValueRow<DP> + i * 64;
                const u32x2 a = read_transposed(at), b = read_transposed(at + 8 * kValueRow<DP>);
                vf[kk & 1][i] = u32x4{a[0], a[1], b[0], b[1]};
            }
        };
        read_v(0);
        __builtin_amdgcn_sched_barrier(0);
        if (there != ~uint64_t(0) || (t0 < all_lo && !(SINK && t0 + kStep <= run.sink)) || t0 + kStep > all_hi) {
            // bit k: this lane's row sees key 4 half + k, for the k below (x = 32, 8 and 1 times the indices)
            const int from = min(max(lo - t0, 0), kStep), to = min(max(hi - t0, 0), kStep);
            uint64_t see = there;
            uint64_t seen = from < kStep ? ~uint64_t(0) << from : 0;
            if constexpr (SINK) {
                const int sinks = max(run.sink - t0, 0);
                seen |= sinks < kStep ? (uint64_t(1) << sinks) - 1 : ~uint64_t(0);
            }
            see &= seen;
            see = to < kStep ? see & ((uint64_t(1) << to) - 1) : see;
            see >>= 4 * half;
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                const uint32_t bits = (uint32_t)(see >> (32 * x));
#pragma unroll
                for (int i = 0; i < 16; ++i) s[x][i] = bits & (1u << (8 * (i / 4) + i % 4)) ? s[x][i] : -INFINITY;
            }
        }
        float tops[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            tops[i] = fmaxf(s[i / 2][i % 2 * 8], s[i / 2][i % 2 * 8 + 1]);
#pragma unroll
            for (int e = 2; e < 8; ++e) tops[i] = fmaxf(tops[i], s[i / 2][i % 2 * 8 + e]);
        }
        const f32x2 both = both_halves(fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3])));
        const float top = fmaxf(both[0], both[1]) * c;
        if (__any(top > m + kLag)) {
            const float m1 = fmaxf(m, top), b1 = m1 == -INFINITY ? 0.0f : m1, fade = exp2_(m - b1);
            m = m1;
            base = b1;
            l *= fade;
#pragma unroll
            for (int i = 0; i < DT; ++i)
#pragma unroll
                for (int e = 0; e < 16; ++e) o[i][e] *= fade;
        }
        float sums[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        u32x4 pf[2];
        const auto exponentials = [&](int kk) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int i = (kk & 1) * 8 + e * 2;
                const float a = exp2_(__builtin_fmaf(s[kk / 2][i], c, -base)), b = exp2_(__builtin_fmaf(s[kk / 2][i + 1], c, -base));
                sums[kk] += a + b;
                pf[kk & 1][e] = pack2<T>(a, b);
            }
        };
        exponentials(0);
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) {
            if (kk < 3) read_v(kk + 1);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int i = 0; i < DT; ++i) o[i] = T::mfma32(vf[kk & 1][i], pf[kk & 1], o[i]);
            if (kk < 3) exponentials(kk + 1);
        }
        l += (sums[0] + sums[1]) + (sums[2] + sums[3]);
    };
    if constexpr (kAhead > 1) {
        for (int step = step0; step < step1; step += 2) {
            take(std::integral_constant<int, 0>{}, step);
            if (step + 1 < step1) take(std::integral_constant<int, 1>{}, step + 1);
        }
    } else {
        for (int step = step0; step < step1; ++step) take((step - step0) & 1, step);
    }
    const f32x2 ls = both_halves(l);
    l = ls[0] + ls[1];

    const int64_t row = tile.first + token, at = row * p.q_heads + head;
    float *const to32 = p.part_o + ((int64_t)split * p.cache.num_q * p.q_heads + at) * p.head_dim;
    char *const to = p.out + row * p.o_ts + head * p.o_hs;
    if (p.splits > 1) {
#pragma unroll
        for (int i = 0; i < DT; ++i)
#pragma unroll
            for (int e = 0; e < 16; e += 4) {
                const int d = i * 32 + e * 2 + half * 4;
                if (have && d < p.head_dim) *(f32x4 *)(to32 + d) = f32x4{o[i][e], o[i][e + 1], o[i][e + 2], o[i][e + 3]};
            }
        if (have && half == 0) {
            float *ml = p.part_ml + ((int64_t)split * p.cache.num_q * p.q_heads + at) * 2;
            ml[0] = m;
            ml[1] = l;
        }
    } else {
        const bool empty = l == 0.0f;
        const float by = empty ? 0.0f : (F8 && p.v_scale ? p.v_scale[h] : 1.0f) / l;
        if (empty)
#pragma unroll
            for (int i = 0; i < DT; ++i)
#pragma unroll
                for (int e = 0; e < 16; ++e) o[i][e] = 0.0f;
#pragma unroll
        for (int i = 0; i < DT; ++i)
#pragma unroll
            for (int e = 0; e < 16; e += 8) {
                // both halves' four elements of one group of eight to one lane
                const u32x2 a = swap_halves(pack2<T>(o[i][e] * by, o[i][e + 1] * by), pack2<T>(o[i][e + 4] * by, o[i][e + 5] * by));
                const u32x2 b = swap_halves(pack2<T>(o[i][e + 2] * by, o[i][e + 3] * by), pack2<T>(o[i][e + 6] * by, o[i][e + 7] * by));
                const int d = i * 32 + e * 2 + half * 8;
                if (have && d < p.head_dim) *(u32x4 *)(to + d * 2) = u32x4{a[0], b[0], a[1], b[1]};
            }
        if (have && half == 0 && p.lse) p.lse[at] = empty ? -INFINITY : (m + log2_(l)) * kLn2;
    }
    __syncthreads();
    if (!*odd) return;
    // add_nonfinite: the values staged as 0, to the elements just written (each lane to those of one half's, which no
    // other lane writes: the barrier is behind both halves' stores)
    for (int step = step0; step < step1; ++step) {
        const int t0 = begin + step * kStep;
        ask(step);
        const bool here = (uint32_t)id < p.cache.blocks;
        const uint32_t off = here ? (uint32_t)id * p.cache.block16 + id_row * p.cache.row16 : 0u;
        const uint64_t in = __ballot(here);
        if (!is_mixed(in, t0)) continue;
        for (int k = 0; k < kStep; ++k) {
            const char *v = vbase + ((int64_t)(uint32_t)__shfl((int)off, k) << 4);
            if (!((in >> k) & 1) || !have || (t0 + k < lo && !(SINK && t0 + k < run.sink)) || t0 + k >= hi) continue;
            for (int d = half; d < p.head_dim; d += 2) {
                const float x = load_one<T, F8>(v, d);
                if (fabsf(x) < INFINITY) continue;
                if (p.splits > 1) to32[d] += x;
                else ((uint16_t *)to)[d] = (uint16_t)pack2<T>(T::to_f32(((const uint16_t *)to)[d]) + x, 0.0f);
            }
        }
    }
}

// Every request in tiles of 16 rows.
template <class T, bool F8, int DP, bool SINK>
__global__ __launch_bounds__(kThreads) void attention_few_kernel(AttentionParams p) {
    __shared__ __align__(16) char lds[kSplitLds<DP, kWaves>];
    __shared__ float part[kWaves][16][2];
    __shared__ int odd;                        // some value that not all rows see is not finite
    const unsigned id = blockIdx.x;
    const int h = (int)(id % p.kv_heads), split = (int)(id / p.kv_heads % p.splits);
    const Tile tile = find_tile<kSplitRows>(p.cache, (int)(id / p.kv_heads / p.splits), p.group);
    if (tile.row0 < tile.rows) few_rows<T, F8, DP, kWaves, SINK>(p, tile, h, split, lds, part, &odd);
}

// Large tiles, from the last to the first (a request's last rows see most
// keys); a request with no more than 16 rows in all takes the other body.
template <class T, bool F8, int DP, int W, bool SINK>
__global__ __launch_bounds__(64 * W, DP > 128 ? 1 : 2) void attention_many_kernel(AttentionParams p) {
    constexpr int kFew = few_dim<F8>(DP);
    __shared__ __align__(16) char lds[kTileLds<DP> > kSplitLds<kFew, W> ? kTileLds<DP> : kSplitLds<kFew, W>];
    __shared__ float part[W][16][2];
    __shared__ int odd;                        // some value that not all rows see is not finite
    __shared__ Places places[4];
    const unsigned id = blockIdx.x;
    const int h = (int)(id % p.kv_heads), split = (int)(id / p.kv_heads % p.splits);
    const Tile tile = find_tile<32 * W>(p.cache, (int)p.tiles - 1 - (int)(id / p.kv_heads / p.splits), p.group);
    if (tile.row0 >= tile.rows) return;
    if (tile.rows <= kSplitRows) few_rows<T, F8, kFew, W, SINK>(p, tile, h, split, lds, part, &odd);
    else many_rows<T, F8, DP, W, SINK>(p, tile, h, split, lds, &odd, places);
}

// Join the parts of each row: one wave a row, each half of it every other
// part, eight elements a lane; the parts' sums and values are loaded together.
// Bound by latency: 3.5 to 5.5 us for the parts of few rows.
template <class T>
__global__ __launch_bounds__(kThreads) void attention_join_kernel(AttentionParams p) {
    const int lane = threadIdx.x & 63, half = lane >> 5, d = (lane & 31) * 8;
    const int64_t all = p.cache.num_q * p.q_heads, row = (int64_t)blockIdx.x * kWaves + (threadIdx.x >> 6);
    if (row >= all) return;
    const int64_t q = (uint32_t)row / (uint32_t)p.q_heads;
    const bool ours = q >= p.cache.q_off[0] && q < p.cache.q_off[p.cache.num_reqs];   // no part holds rows of no request
    f32x2 ml = {-INFINITY, 0.0f};
    if (lane < p.splits) ml = *(const f32x2 *)(p.part_ml + (lane * all + row) * 2);
    const float *at = p.part_o + row * p.head_dim + d;
    const bool in = d < p.head_dim;
    constexpr int kAhead = 4;
    f32x4 x[kAhead], y[kAhead];
    const auto load = [&](int s0) {
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int s = s0 + 2 * i + half;
            x[i] = y[i] = f32x4{0, 0, 0, 0};
            if (in && s < p.splits) {
                const f32x4 *from = (const f32x4 *)(at + s * all * p.head_dim);
                x[i] = from[0];
                y[i] = from[1];
            }
        }
    };
    load(0);
    float top = ml[0];
#pragma unroll
    for (int i = 1; i < 32; i *= 2) top = fmaxf(top, __shfl_xor(top, i));
    const f32x2 tops = both_halves(top);
    top = fmaxf(tops[0], tops[1]);
    const float base = top == -INFINITY ? 0.0f : top, by = exp2_(ml[0] - base);
    float l = ml[1] * by;
#pragma unroll
    for (int i = 1; i < 32; i *= 2) l += __shfl_xor(l, i);
    const f32x2 ls = both_halves(l);
    l = ls[0] + ls[1];
    f32x4 a = {0, 0, 0, 0}, b = {0, 0, 0, 0};
    for (int s0 = 0; s0 < p.splits; s0 += 2 * kAhead) {
        if (s0 > 0) load(s0);
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const float w = __shfl(by, s0 + 2 * i + half);     // 0 past the last part, and for one that saw nothing
            if (w != 0.0f) {
                a += x[i] * w;
                b += y[i] * w;
            }
        }
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const f32x2 u = both_halves(a[e]), v = both_halves(b[e]);
        a[e] = u[0] + u[1];
        b[e] = v[0] + v[1];
    }
    if (!ours) return;
    const int head = (int)(row - q * p.q_heads);
    const bool empty = l == 0.0f;
    const float inv = empty ? 0.0f : (p.v_scale ? p.v_scale[(int)divide(head, p.by_group)] : 1.0f) / l;
    if (half == 0 && in) {
        char *to = p.out + q * p.o_ts + head * p.o_hs + d * 2;
        if (empty) *(u32x4 *)to = u32x4{0, 0, 0, 0};
        else *(u32x4 *)to = u32x4{pack2<T>(a[0] * inv, a[1] * inv), pack2<T>(a[2] * inv, a[3] * inv),
                                  pack2<T>(b[0] * inv, b[1] * inv), pack2<T>(b[2] * inv, b[3] * inv)};
    }
    if (lane == 0 && p.lse) p.lse[row] = empty ? -INFINITY : (top + log2_(l)) * kLn2;
}

template <class T, bool F8, bool SINK, int DP> void (*attention_kernel_for(int rows))(AttentionParams) {
    if (rows == kSplitRows) return attention_few_kernel<T, F8, few_dim<F8>(DP), SINK>;
    if constexpr (DP <= 128) {
        if (rows == kLargeRows) return attention_many_kernel<T, F8, DP, kLargeRows / 32, SINK>;
    }
    return attention_many_kernel<T, F8, DP, kTileRows / 32, SINK>;
}

template <class T, bool F8, bool SINK> auto attention_kernel(int rows, int head_dim) {
    if (head_dim <= 64) return attention_kernel_for<T, F8, SINK, 64>(rows);
    if (head_dim <= 96) return attention_kernel_for<T, F8, SINK, 96>(rows);
    if (head_dim <= 128) return attention_kernel_for<T, F8, SINK, 128>(rows);
    return attention_kernel_for<T, F8, SINK, 256>(rows);
}

template <bool SINK> auto attention_kernel(bool bf16, bool f8, int rows, int d) {
    return bf16 ? (f8 ? attention_kernel<Bf16, true, SINK>(rows, d) : attention_kernel<Bf16, false, SINK>(rows, d))
                : (f8 ? attention_kernel<F16, true, SINK>(rows, d) : attention_kernel<F16, false, SINK>(rows, d));
}

int attention(const kv_layout *layout, const void *d_layer, const kv_batch *batch, const kv_rows *q, const kv_rows *out,
              float scale, int32_t causal, int32_t window, int32_t sink, int32_t cache_dtype, const float *d_k_scale,
              const float *d_v_scale, float *d_lse, void *d_workspace, int64_t workspace_bytes, void *stream) {
    int rc = check_cache(layout, cache_dtype);
    if (rc == KV_OK) rc = check_batch(batch);
    if (rc == KV_OK) rc = check_rows(q, batch->num_q, layout->head_dim, false);
    if (rc == KV_OK) rc = check_rows(out, batch->num_q, layout->head_dim, true);
    if (rc != KV_OK) return rc;
    if (!d_layer || out->dtype != q->dtype || out->heads != q->heads) return KV_EINVAL;
    if (cache_dtype != KV_F8E4M3 && cache_dtype != q->dtype) return KV_EINVAL;
    if (!(scale > 0.0f) || !isfinite(scale)) return KV_EINVAL;
    if (((uintptr_t)d_layer & 15u) || ((uintptr_t)d_lse & 3u) || ((uintptr_t)d_workspace & 15u)) return KV_EALIGN;
    AttentionPlan plan;
    rc = plan_attention(layout, batch, q->heads, window, sink, &plan);
    if (rc != KV_OK) return rc;
    if (plan.workspace > 0 && !d_workspace) return KV_EINVAL;
    if (plan.workspace > workspace_bytes) return KV_ELIMIT;
    if (batch->num_q == 0) return KV_OK;
    const int64_t all = batch->num_q * q->heads;
    AttentionParams p;
    p.cache = make_paged(layout, d_layer, batch);
    p.q = (const char *)q->d_data;
    p.out = (char *)const_cast<void *>(out->d_data);
    p.q_ts = q->token_stride * 2, p.q_hs = q->head_stride * 2;
    p.o_ts = out->token_stride * 2, p.o_hs = out->head_stride * 2;
    p.lse = d_lse;
    p.part_o = (float *)d_workspace;
    p.part_ml = p.part_o ? p.part_o + (int64_t)plan.splits * all * layout->head_dim : nullptr;
    p.k_scale = cache_dtype == KV_F8E4M3 ? d_k_scale : nullptr;
    p.v_scale = cache_dtype == KV_F8E4M3 ? d_v_scale : nullptr;
    p.tiles = plan.tiles;
    p.scale = scale * kLog2e;
    p.q_heads = q->heads;
    p.kv_heads = layout->kv_heads;
    p.group = q->heads / layout->kv_heads;
    p.by_group = make_divider((uint32_t)p.group);
    p.head_dim = layout->head_dim;
    p.splits = plan.splits;
    p.window = window < kMaxLength ? window : 0;
    p.sink = sink < kMaxLength ? sink : kMaxLength;
    p.causal = causal != 0;
    const bool bf16 = q->dtype == KV_BF16, f8 = cache_dtype == KV_F8E4M3;
    // Rows of an 8-bit cache of up to 96 elements take 128 columns where no request fills a tile and none is cut into parts:
    // 64 chunks of 20 tokens over 2,020 at head size 80 110 us, 122 in 96 columns; 16 of them, in parts, 45 and 44, 64 of 40
    // tokens 145 and 139.
    const bool short_tiles = f8 && layout->head_dim > 64 && plan.splits == 1 && (int64_t)batch->max_q_len * p.group < kTileRows;
    const int d = short_tiles ? std::max(layout->head_dim, 128) : layout->head_dim;
    // (without a window every key is in it)
    auto kernel = p.sink > 0 && p.window > 0 ? attention_kernel<true>(bf16, f8, plan.rows, d)
                                             : attention_kernel<false>(bf16, f8, plan.rows, d);
    const int threads = plan.rows == kSplitRows ? kThreads : 2 * plan.rows;
    hipStream_t s = (hipStream_t)stream;
    (void)hipGetLastError();
    hipLaunchKernelGGL(kernel, dim3((unsigned)(plan.tiles * p.kv_heads * p.splits)), dim3(threads), 0, s, p);
    if (p.splits > 1) {
        auto join = bf16 ? attention_join_kernel<Bf16> : attention_join_kernel<F16>;
        hipLaunchKernelGGL(join, dim3((unsigned)((all + kWaves - 1) / kWaves)), dim3(kThreads), 0, s, p);
    }
    return hipGetLastError() == hipSuccess ? KV_OK : KV_EHIP;
}

}  // namespace
}  // namespace tkv

extern "C" {

int kv_paged_attention(const kv_layout *layout, const void *d_layer, const kv_batch *batch, const kv_rows *q,
                       const kv_rows *out, float scale, int32_t causal, int32_t window, int32_t cache_dtype,
                       const float *d_k_scale, const float *d_v_scale, float *d_lse, void *d_workspace,
                       int64_t workspace_bytes, void *stream) {
    return tkv::attention(layout, d_layer, batch, q, out, scale, causal, window, 0, cache_dtype, d_k_scale, d_v_scale, d_lse,
                          d_workspace, workspace_bytes, stream);
}

int kv_sink_attention(const kv_layout *layout, const void *d_layer, const kv_batch *batch, const kv_rows *q,
                      const kv_rows *out, float scale, int32_t causal, int32_t window, int32_t sink,
                      int32_t cache_dtype, const float *d_k_scale, const float *d_v_scale, float *d_lse,
                      void *d_workspace, int64_t workspace_bytes, void *stream) {
    return tkv::attention(layout, d_layer, batch, q, out, scale, causal, window, sink, cache_dtype, d_k_scale, d_v_scale,
                          d_lse, d_workspace, workspace_bytes, stream);
}

}  // extern "C"
