// host.cpp -- the host-only calls of the C ABI: layout checks, the retrieve
// planner, host job build, job validation, the commitment rule, and the checks
// and launch plan of the operators over the paged cache.  Plain
// C++ with no HIP header, so that it can also be built and tested on its own
// (for instance under the address and undefined-behaviour sanitizers).

#include <math.h>

#include <algorithm>
#include <unordered_set>
#include <vector>

#include "host.h"

namespace tkv {

// Layout checks shared by the copy directions and staging.
int check_layout(const kv_layout *lo) {
    if (!lo) return KV_EINVAL;
    if (lo->num_layers <= 0 || lo->num_layers > KV_MAX_LAYERS || lo->kv_heads <= 0 || lo->head_dim <= 0 ||
        lo->block_size <= 0 || lo->chunk_tokens <= 0 || lo->num_blocks <= 0 || lo->num_slots <= 0)
        return KV_EINVAL;
    if (lo->elem_bytes != 1 && lo->elem_bytes != 2 && lo->elem_bytes != 4) return KV_EINVAL;
    if (lo->chunk_tokens % lo->block_size != 0) return KV_EINVAL;
    const int64_t seg = (int64_t)lo->block_size * lo->kv_heads * lo->head_dim * lo->elem_bytes;
    if (seg > (int64_t(1) << 40)) return KV_EINVAL;
    if (lo->paged_kv_stride <= 0 || lo->paged_block_stride <= 0) return KV_EINVAL;
    if (lo->paged_block_stride < seg || lo->paged_kv_stride < seg) return KV_EINVAL;
    if (seg % 16 != 0 || lo->paged_kv_stride % 16 != 0 || lo->paged_block_stride % 16 != 0) return KV_EALIGN;
    // slot_bytes * num_slots must stay well inside int64
    const int64_t slot = seg * (lo->chunk_tokens / lo->block_size) * 2 * lo->num_layers;
    if (slot <= 0 || lo->num_slots > (int64_t(1) << 62) / slot) return KV_EINVAL;
    return KV_OK;
}

// Checks shared by the operators over the paged cache.  They address rows in
// 32-bit units of 16 bytes, hence the limit on a layer's span.
int check_cache(const kv_layout *lo, int32_t cache_dtype) {
    const int rc = check_layout(lo);
    if (rc != KV_OK) return rc;
    if (cache_dtype != KV_BF16 && cache_dtype != KV_F16 && cache_dtype != KV_F8E4M3) return KV_EINVAL;
    if (lo->elem_bytes != (cache_dtype == KV_F8E4M3 ? 1 : 2)) return KV_EINVAL;
    if (lo->head_dim > kMaxHeadDim) return KV_ELIMIT;
    if (lo->head_dim % 8 != 0 || (lo->head_dim * lo->elem_bytes) % 16 != 0) return KV_EALIGN;
    return check_span(lo);
}

int check_span(const kv_layout *lo) {
    return lo->num_blocks > (int64_t(1) << 36) / lo->paged_block_stride ? KV_ELIMIT : KV_OK;
}

int check_batch(const kv_batch *b) {
    if (!b || b->num_reqs < 0 || b->bt_stride <= 0 || b->num_q < 0 || b->max_q_len < 0 || b->max_kv_len < 0)
        return KV_EINVAL;
    if (b->num_q > 0 && (b->num_reqs == 0 || !b->d_q_off || !b->d_kv_len || !b->d_block_tables)) return KV_EINVAL;
    if (((uintptr_t)b->d_q_off & 7u) || ((uintptr_t)b->d_kv_len & 3u) || ((uintptr_t)b->d_block_tables & 3u))
        return KV_EALIGN;
    return KV_OK;
}

// Whether rows of `dim` elements at t*ts + h*hs lie on one another (t < num,
// h < heads, strides >= 0).  Rows whose heads differ by a > 0 and tokens by b
// the other way are |a hs - b ts| apart, which is least for the two b beside
// a hs / ts; the usual layouts, one stride past all of the other's rows, need
// no search.
static bool rows_overlap(int64_t num, int64_t heads, int64_t ts, int64_t hs, int64_t dim) {
    typedef __int128 wide;
    if ((heads > 1 && hs < dim) || (num > 1 && ts < dim)) return true;
    if (heads <= 1 || num <= 1) return false;
    if ((wide)ts >= (wide)(heads - 1) * hs + dim || (wide)hs >= (wide)(num - 1) * ts + dim) return false;
    for (int64_t a = 1; a < heads; ++a) {
        const wide at = (wide)a * hs;
        wide b = at / ts;
        if (b >= num - 1) b = num - 1;
        if (at - b * ts < dim) return true;
        if (b + 1 < num && (b + 1) * ts - at < dim) return true;
    }
    return false;
}

int check_rows(const kv_rows *x, int64_t num, int32_t head_dim, bool written) {
    if (!x || x->heads <= 0 || (x->dtype != KV_BF16 && x->dtype != KV_F16)) return KV_EINVAL;
    if (num > 0 && !x->d_data) return KV_EINVAL;
    if (x->heads > kMaxHeads) return KV_ELIMIT;
    if (x->token_stride < 0 || x->head_stride < 0) return KV_EINVAL;
    if (written && rows_overlap(num, x->heads, x->token_stride, x->head_stride, head_dim)) return KV_EINVAL;
    if (((uintptr_t)x->d_data & 15u) || x->token_stride % 8 != 0 || x->head_stride % 8 != 0) return KV_EALIGN;
    return KV_OK;
}

// Into how many parts each tile's keys are cut: enough for two workgroups on
// each compute unit, but no part shorter than a step.  A batch of several
// requests may be ragged: there up to eight workgroups on each, as long as the
// longest request's parts keep 2,048 keys, so that it does not run on alone (32
// lognormal requests around 4,000 tokens: 136 against 295 us; 64 equal ones of
// 4,096: 207 against 203 us).
int32_t attention_splits(int64_t tiles, int32_t num_reqs, int32_t kv_heads, int64_t span, int32_t step) {
    const int64_t base = tiles * kv_heads, want = 512, most = (span + step - 1) / step;
    if (base <= 0) return 1;
    int64_t parts = want / base, ragged = num_reqs > 1 ? 4 * want / base : 1;
    if (ragged > span / 2048) ragged = span / 2048;
    if (parts > most) parts = most;
    if (parts < ragged) parts = ragged;
    if (parts > kMaxSplits) parts = kMaxSplits;
    return parts < 1 ? 1 : (int32_t)parts;
}

int plan_attention(const kv_layout *lo, const kv_batch *b, int32_t q_heads, int32_t window, int32_t sink,
                   AttentionPlan *plan) {
    if (q_heads <= 0 || q_heads % lo->kv_heads != 0 || window < 0 || sink < 0) return KV_EINVAL;
    const int64_t group = q_heads / lo->kv_heads;
    if (b->num_q >= (int64_t(1) << 30) / q_heads) return KV_ELIMIT;       // rows are counted in 32 bits
    int64_t span = b->max_kv_len;
    if (window > 0 && span > (int64_t)window + b->max_q_len + sink) span = (int64_t)window + b->max_q_len + sink;
    // Tiles of 256 rows read K and V half as often as those of 128, but take a compute unit each: where there are four
    // rounds of them (8 x 2,048 tokens of 32 heads: 859 against 917 us; a mixed batch of fewer: 77 against 61 us).  That is
    // without a window, at head size 128: with one of 1,024 or less, and at head size 64, 128 rows are the faster (4 x 4,096
    // tokens, a window of 512: 223 against 205 us).
    const bool many = b->max_q_len * group > kSplitRows;
    const bool large = lo->head_dim <= 128 && b->num_q * group / kLargeRows * lo->kv_heads >= 1024;
    plan->rows = !many ? kSplitRows : (large ? kLargeRows : kTileRows);
    plan->tiles = b->num_q * group / plan->rows + b->num_reqs;
    // (of the launched tiles, where all requests are small, one a request has rows)
    const int64_t real = !many && b->num_reqs < plan->tiles ? b->num_reqs : plan->tiles;
    plan->splits = attention_splits(real, b->num_reqs, lo->kv_heads, span, many ? kTileStep : kSplitStep);
    plan->workspace = plan->splits > 1 ? (int64_t)plan->splits * b->num_q * q_heads * (lo->head_dim + 2) * 4 : 0;
    if (plan->tiles * lo->kv_heads * plan->splits >= (int64_t(1) << 31)) return KV_ELIMIT;
    return KV_OK;
}

// sink < 0: the rule without sinks.
int plan_weights(const kv_layout *lo, const kv_batch *b, int32_t q_heads, int32_t window, int32_t sink, WeightPlan *plan) {
    const int64_t heads = (int64_t)b->num_reqs * lo->kv_heads, group = q_heads / lo->kv_heads;
    if (heads >= (int64_t(1) << 31) || b->num_q >= (int64_t(1) << 30) / q_heads) return KV_ELIMIT;
    plan->windowed = sink >= 0 && window > 0 && window < kMaxLength;
    // Keys of a workgroup: 256, each wave 64 of its own, or 64, with the waves sharing the rows, where that is needed to
    // give each compute unit two workgroups.  Up to 16 rows take a kernel of their own.
    plan->few = b->max_q_len * group <= 16;
    int64_t span = b->max_kv_len;
    if (plan->windowed && span > (int64_t)window + b->max_q_len) span = (int64_t)window + b->max_q_len;
    plan->keys = !plan->few && heads * ((span + 255) / 256) < 512 ? 64 : 256;
    // With a window, 128 in between: where the requests' mean gives five workgroups for two compute units (4 x 2,000 tokens
    // over 6,000, a window of 1,024: 127 us, 135 with 64 keys and 168 with 256; 8 of 512 over 2,512 75, 82 and 75; one of 4,096
    // over 8,192 112 against 79 with 64, 2 of 2,000 over 6,000 at 2,048 173 against 126).  Of 18 batches of 1 to 16 requests
    // and windows of 256 to 4,096 none is more than 11 % above the best of the three.
    if (plan->windowed && plan->keys == 64 && heads > 0) {
        const int64_t mean = (int64_t)window + b->num_q / b->num_reqs;
        if (heads * ((mean < span ? mean : span) / 128) >= 640) plan->keys = 128;
    }
    plan->sink_tiles = plan->parts = 0;
    if (plan->windowed && !plan->few) {
        // A sink's rows are all of a chunk's, a key's those of a window: as many parts as that is longer.  (Sums of
        // parts need memory for each sink: more than 1,024 are not cut.  Without sinks there is nothing to cut, or to join.)
        int64_t tiles = ((int64_t)sink + 63) / 64, parts = (b->max_q_len + (int64_t)window + 255) / ((int64_t)window + 256);
        parts = parts < 1 || tiles == 0 || tiles > 16 ? 1 : (parts > 64 ? 64 : parts);
        plan->sink_tiles = (int32_t)(tiles > 256 ? 256 : tiles);
        plan->parts = (int32_t)parts;
    }
    plan->workspace = plan->parts > 1 ? heads * plan->sink_tiles * plan->parts * 64 * 4 : 0;
    // (few rows: the sinks lie next to the window's keys)
    if (plan->windowed && plan->few) span += sink;
    if (span > b->max_kv_len) span = b->max_kv_len;
    int64_t tiles = (span + plan->keys - 1) / plan->keys;
    // Few rows: a wave for each tile, or a workgroup for each slot of the chip's, two on a compute unit (three at head sizes up
    // to 64), whose waves pass tile after tile with the next one on its way.  The second where one request, or a window that
    // cuts all to one length, leaves several tiles to a wave (one of 100,000 tokens 47 us, 51 a wave for each; 64 of 2,052
    // visible ones 62, 65).  Several requests may be ragged, and then some waves pass far more than others (16 lognormal ones
    // around 940 tokens 9.0 us a wave for each, 11 tile after tile): only where there are heads or keys enough for four
    // workgroups a slot, of 1,024 keys or more and up to 2,048 of the longest request's (64 of 4,096 111 us, 122 a wave for
    // each; 64 lognormal ones around 4,000 129 and 136).  16-bit rows of 72 to 96 columns always have a wave for each tile.
    plan->ahead = false;
    const bool pieces = lo->elem_bytes == 2 && lo->head_dim > 64 && lo->head_dim <= 96;
    if (plan->few && !pieces && heads > 0 && (heads <= 512 || span >= 512)) {
        const bool ragged = b->num_reqs > 1 && !(plan->windowed && (int64_t)window + b->max_q_len < b->max_kv_len);
        const int64_t slots = lo->head_dim <= 64 ? 768 : 512;
        int64_t most = slots / heads;
        if (ragged) most = std::max({most, std::min(4 * slots / heads, span / 1024), span / 2048});
        most = std::max(most, int64_t(1));
        plan->ahead = tiles > most && !(ragged && heads < 512 && heads * (span / 1024) < 4 * slots);
        if (plan->ahead) tiles = most;
    }
    plan->tiles = tiles < 1 ? 1 : (tiles > 32768 ? 32768 : tiles);
    return KV_OK;
}

}  // namespace tkv

using tkv::check_layout;

extern "C" {

int kv_rope_frequencies(int32_t rot_dim, double base, int32_t scaling, double factor, double context, double low,
                        double high, double *h_freqs, float *magnitude) {
    if (rot_dim < 0 || rot_dim % 2 != 0 || (rot_dim > 0 && !h_freqs) || !magnitude) return KV_EINVAL;
    if (!(base > 1.0) || !isfinite(base)) return KV_EINVAL;
    if (scaling < KV_ROPE_PLAIN || scaling > KV_ROPE_RAMP) return KV_EINVAL;
    if (scaling != KV_ROPE_PLAIN && (!(factor >= 1.0) || !isfinite(factor))) return KV_EINVAL;
    if (scaling == KV_ROPE_RAMP && (!(context > 0.0) || !isfinite(context) || !isfinite(low) || !(high > low) ||
                                    !isfinite(high)))
        return KV_EINVAL;
    if (scaling == KV_ROPE_BASE) {
        if (rot_dim <= 2) return KV_EINVAL;
        base *= pow(factor, (double)rot_dim / (rot_dim - 2));
    }
    const double two_pi = 6.283185307179586476925;
    for (int32_t i = 0; i < rot_dim / 2; ++i) {
        double f = pow(base, -2.0 * i / rot_dim);
        if (scaling == KV_ROPE_LINEAR) f /= factor;
        if (scaling == KV_ROPE_RAMP) {
            double keep = (context * f / two_pi - low) / (high - low);
            keep = keep < 0.0 ? 0.0 : (keep > 1.0 ? 1.0 : keep);
            f *= keep + (1.0 - keep) / factor;
        }
        h_freqs[i] = f;
    }
    *magnitude = scaling == KV_ROPE_RAMP ? (float)(0.1 * log(factor) + 1.0) : 1.0f;
    return KV_OK;
}

int kv_rope_axes(int32_t num_axes, const int32_t *h_sections, int32_t order, uint8_t *h_axis) {
    if (num_axes <= 0 || num_axes > KV_MAX_AXES || !h_sections) return KV_EINVAL;
    if (order != KV_AXES_SECTIONS && order != KV_AXES_IN_TURN) return KV_EINVAL;
    int64_t pairs = 0;
    int32_t longest = 0;
    for (int32_t a = 0; a < num_axes; ++a) {
        if (h_sections[a] < 0) return KV_EINVAL;
        pairs += h_sections[a];
        if (h_sections[a] > longest) longest = h_sections[a];
    }
    if (pairs > tkv::kMaxHeadDim / 2) return KV_ELIMIT;
    if (pairs > 0 && !h_axis) return KV_EINVAL;
    if (order == KV_AXES_SECTIONS) {
        for (int32_t a = 0; a < num_axes; ++a)
            for (int32_t i = 0; i < h_sections[a]; ++i) *h_axis++ = (uint8_t)a;
    } else {
        for (int32_t i = 0; i < longest; ++i)
            for (int32_t a = 0; a < num_axes; ++a)
                if (i < h_sections[a]) *h_axis++ = (uint8_t)a;
    }
    return KV_OK;
}

int kv_paged_attention_workspace(const kv_layout *layout, const kv_batch *batch, int32_t q_heads, int32_t window,
                                 int64_t *bytes) {
    return kv_sink_attention_workspace(layout, batch, q_heads, window, 0, bytes);
}

int kv_sink_attention_workspace(const kv_layout *layout, const kv_batch *batch, int32_t q_heads, int32_t window,
                                int32_t sink, int64_t *bytes) {
    int rc = check_layout(layout);
    if (rc == KV_OK) rc = tkv::check_batch(batch);
    if (rc != KV_OK) return rc;
    if (!bytes) return KV_EINVAL;
    tkv::AttentionPlan plan;
    rc = tkv::plan_attention(layout, batch, q_heads, window, sink, &plan);
    if (rc != KV_OK) return rc;
    *bytes = plan.workspace;
    return KV_OK;
}

int kv_sink_weights_workspace(const kv_layout *layout, const kv_batch *batch, int32_t q_heads, int32_t window,
                              int32_t sink, int64_t *bytes) {
    int rc = check_layout(layout);
    if (rc == KV_OK) rc = tkv::check_batch(batch);
    if (rc != KV_OK) return rc;
    if (!bytes || q_heads <= 0 || q_heads % layout->kv_heads != 0 || window < 0 || sink < 0) return KV_EINVAL;
    tkv::WeightPlan plan;
    rc = tkv::plan_weights(layout, batch, q_heads, window, sink, &plan);
    if (rc != KV_OK) return rc;
    *bytes = plan.workspace;
    return KV_OK;
}

int kv_retrieve_plan(const kv_layout *layout, const kv_job *h_jobs, int32_t num_jobs) {
    const int rc = check_layout(layout);
    if (rc != KV_OK) return rc;
    if (num_jobs < 0 || (num_jobs > 0 && !h_jobs)) return KV_EINVAL;
    if (num_jobs == 0) return KV_RETRIEVE_UNIT;
    int64_t runs = 0, pairs_shared = 0;
    for (int32_t i = 0; i < num_jobs; ++i) {
        if (i == 0 || h_jobs[i].slot != h_jobs[i - 1].slot) ++runs;
        if ((i & 1) && h_jobs[i].slot == h_jobs[i - 1].slot) ++pairs_shared;
    }
    if (runs == num_jobs) {
        // no slot twice in a row; streaming needs every slot once
        std::unordered_set<int32_t> seen;
        seen.reserve((size_t)num_jobs * 2);
        bool distinct = true;
        for (int32_t i = 0; i < num_jobs && distinct; ++i) distinct = seen.insert(h_jobs[i].slot).second;
        if (distinct) return KV_RETRIEVE_STREAM;
    }
    // Lists in which most pairs share their chunk and groups are small.  The
    // copy that runs is the same for PAIR and UNIT.
    const int64_t seg = (int64_t)layout->block_size * layout->kv_heads * layout->head_dim * layout->elem_bytes;
    if (seg == 32768 && 20 * pairs_shared >= 9 * (int64_t)num_jobs && num_jobs <= 16 * runs)
        return KV_RETRIEVE_PAIR;
    return KV_RETRIEVE_UNIT;
}

}  // extern "C"

namespace {

// Shared body of kv_build_jobs and kv_build_jobs_routed.  A request takes
// part when `requested` is null or requested[r] != 0; its matched chunks go to
// `ordinary` when decision[r] == KV_ORDINARY (and `ordinary` is given), else
// to `retrieve`.
int build_jobs(const int32_t *hit_chunks, const int32_t *chunk_slot, const uint64_t *block_hash,
               const int64_t *blk_off, const int64_t *chunk_off, int32_t num_reqs, int32_t bpc,
               const int32_t *free_slots, int32_t num_free, const uint8_t *requested, const int32_t *decision,
               kv_job *retrieve, int32_t *num_retrieve, kv_job *ordinary, int32_t *num_ordinary, kv_job *store,
               uint64_t *store_keys, int32_t *num_store, int32_t *dropped) {
    if (num_reqs < 0 || bpc <= 0 || num_free < 0) return KV_EINVAL;
    if (!num_retrieve || !num_store || !dropped) return KV_EINVAL;
    *num_retrieve = *num_store = *dropped = 0;
    if (num_ordinary) *num_ordinary = 0;
    if (num_reqs == 0) return KV_OK;
    if (!hit_chunks || !chunk_slot || !block_hash || !blk_off || !chunk_off || !retrieve || !store || !store_keys ||
        (num_free > 0 && !free_slots))
        return KV_EINVAL;
    for (int32_t r = 0; r < num_reqs; ++r) {
        const int64_t nb = blk_off[r + 1] - blk_off[r];
        const int64_t nc = chunk_off[r + 1] - chunk_off[r];
        if (nb < 0 || nc != nb / bpc || hit_chunks[r] < 0 || hit_chunks[r] > nc) return KV_EINVAL;
        if (decision && (!requested || requested[r]) && decision[r] != KV_COMMIT && decision[r] != KV_ORDINARY)
            return KV_EINVAL;
    }
    std::unordered_set<uint64_t> missing;   // distinct missing keys met so far
    int32_t nr = 0, no = 0, ns = 0, nd = 0;
    for (int32_t r = 0; r < num_reqs; ++r) {
        if (requested && !requested[r]) continue;
        const int64_t c0 = chunk_off[r];
        const int64_t nc = chunk_off[r + 1] - c0;
        const int32_t hit = hit_chunks[r];
        const bool ord = decision && decision[r] == KV_ORDINARY;
        for (int32_t j = 0; j < hit; ++j) {
            if (ord) ordinary[no++] = kv_job{chunk_slot[c0 + j], r, j, 0};
            else retrieve[nr++] = kv_job{chunk_slot[c0 + j], r, j, 0};
        }
        for (int64_t j = hit; j < nc; ++j) {
            if (chunk_slot[c0 + j] >= 0) continue;
            const uint64_t key = block_hash[blk_off[r] + (j + 1) * bpc - 1];
            if (!missing.insert(key).second) continue;
            if (ns >= num_free) {
                ++nd;
                continue;
            }
            store_keys[ns] = key;
            store[ns] = kv_job{free_slots[ns], r, (int32_t)j, 0};
            ++ns;
        }
    }
    *num_retrieve = nr;
    if (num_ordinary) *num_ordinary = no;
    *num_store = ns;
    *dropped = nd;
    return nd > 0 ? KV_ENOSPC : KV_OK;
}

}  // namespace

extern "C" {

int kv_build_jobs(const int32_t *h_hit_chunks, const int32_t *h_chunk_slot, const uint64_t *h_block_hash,
                  const int64_t *h_blk_off, const int64_t *h_chunk_off, int32_t num_reqs, int32_t blocks_per_chunk,
                  const int32_t *h_free_slots, int32_t num_free, kv_job *h_retrieve, int32_t *num_retrieve,
                  kv_job *h_store, uint64_t *h_store_keys, int32_t *num_store, int32_t *dropped) {
    return build_jobs(h_hit_chunks, h_chunk_slot, h_block_hash, h_blk_off, h_chunk_off, num_reqs, blocks_per_chunk,
                      h_free_slots, num_free, nullptr, nullptr, h_retrieve, num_retrieve, nullptr, nullptr, h_store,
                      h_store_keys, num_store, dropped);
}

int kv_chunk_keys(const uint64_t *h_block_hash, const int64_t *h_blk_off, int32_t num_reqs, int32_t blocks_per_chunk,
                  const int64_t *h_chunk_off, uint64_t *h_keys) {
    if (num_reqs < 0 || blocks_per_chunk <= 0) return KV_EINVAL;
    if (num_reqs == 0) return KV_OK;
    if (!h_block_hash || !h_blk_off || !h_chunk_off || !h_keys) return KV_EINVAL;
    for (int32_t r = 0; r < num_reqs; ++r) {
        const int64_t nb = h_blk_off[r + 1] - h_blk_off[r];
        const int64_t nc = h_chunk_off[r + 1] - h_chunk_off[r];
        if (nb < 0 || nc != nb / blocks_per_chunk) return KV_EINVAL;
        for (int64_t j = 0; j < nc; ++j)
            h_keys[h_chunk_off[r] + j] = h_block_hash[h_blk_off[r] + (j + 1) * blocks_per_chunk - 1];
    }
    return KV_OK;
}

int kv_decide_claims(int32_t num_reqs, const int32_t *h_hit_chunks, const int32_t *h_chunk_slot,
                     const int64_t *h_chunk_off, const double *h_ttu, const double *h_ttr,
                     const uint8_t *h_requested, uint64_t slot_bytes, uint64_t budget_bytes, int64_t num_slots,
                     uint8_t *h_protected, uint64_t *reserved_bytes, int32_t *h_decision) {
    if (num_reqs < 0 || num_slots <= 0 || !reserved_bytes) return KV_EINVAL;
    if (num_reqs == 0) return KV_OK;
    if (!h_hit_chunks || !h_chunk_slot || !h_chunk_off || !h_ttu || !h_ttr || !h_requested || !h_protected ||
        !h_decision)
        return KV_EINVAL;
    for (int32_t r = 0; r < num_reqs; ++r) {
        const int64_t nc = h_chunk_off[r + 1] - h_chunk_off[r];
        if (nc < 0 || h_hit_chunks[r] < 0 || h_hit_chunks[r] > nc) return KV_EINVAL;
        for (int32_t j = 0; j < h_hit_chunks[r]; ++j) {
            const int32_t s = h_chunk_slot[h_chunk_off[r] + j];
            if (s < 0 || s >= num_slots) return KV_ERANGE;
        }
    }
    // claims with a pending retrieval request first, then the others, each in request order
    std::vector<int32_t> order;
    order.reserve((size_t)num_reqs);
    for (int pass = 0; pass < 2; ++pass)
        for (int32_t r = 0; r < num_reqs; ++r)
            if ((h_requested[r] != 0) == (pass == 0)) order.push_back(r);
    std::unordered_set<int32_t> objs;
    for (int32_t r : order) {
        // the claim's KV objects: the distinct slots of its matched chunks
        objs.clear();
        uint64_t total = 0, fresh = 0;
        for (int32_t j = 0; j < h_hit_chunks[r]; ++j) {
            const int32_t s = h_chunk_slot[h_chunk_off[r] + j];
            if (!objs.insert(s).second) continue;
            total += slot_bytes;
            if (!h_protected[s]) fresh += slot_bytes;
        }
        const uint64_t free_bytes = budget_bytes > *reserved_bytes ? budget_bytes - *reserved_bytes : 0;
        const int d = kv_commit_should_stage(h_ttu[r], h_ttr[r], free_bytes, fresh, total, budget_bytes,
                                             h_requested[r] != 0);
        h_decision[r] = d;
        if (d == KV_COMMIT) {
            for (int32_t s : objs) h_protected[s] = 1;
            *reserved_bytes += fresh;
        }
    }
    return KV_OK;
}

int kv_build_jobs_routed(const int32_t *h_hit_chunks, const int32_t *h_chunk_slot, const uint64_t *h_block_hash,
                         const int64_t *h_blk_off, const int64_t *h_chunk_off, int32_t num_reqs,
                         int32_t blocks_per_chunk, const int32_t *h_free_slots, int32_t num_free,
                         const uint8_t *h_requested, const int32_t *h_decision, kv_job *h_retrieve,
                         int32_t *num_retrieve, kv_job *h_ordinary, int32_t *num_ordinary, kv_job *h_store,
                         uint64_t *h_store_keys, int32_t *num_store, int32_t *dropped) {
    if (num_reqs > 0 && (!h_requested || !h_decision || !h_ordinary)) return KV_EINVAL;
    if (!num_ordinary) return KV_EINVAL;
    return build_jobs(h_hit_chunks, h_chunk_slot, h_block_hash, h_blk_off, h_chunk_off, num_reqs, blocks_per_chunk,
                      h_free_slots, num_free, h_requested, h_decision, h_retrieve, num_retrieve, h_ordinary,
                      num_ordinary, h_store, h_store_keys, num_store, dropped);
}

int kv_group_jobs_by_slot(kv_job *h_jobs, int32_t num_jobs) {
    if (num_jobs < 0 || (num_jobs > 0 && !h_jobs)) return KV_EINVAL;
    std::stable_sort(h_jobs, h_jobs + num_jobs, [](const kv_job &a, const kv_job &b) { return a.slot < b.slot; });
    return KV_OK;
}

int kv_validate_jobs(const kv_layout *layout, const int32_t *h_block_tables, int32_t bt_stride, int32_t num_reqs,
                     const kv_job *h_jobs, int32_t num_jobs, int is_store) {
    int rc = check_layout(layout);
    if (rc != KV_OK) return rc;
    if (num_jobs < 0 || num_reqs < 0 || bt_stride <= 0) return KV_EINVAL;
    if (num_jobs == 0) return KV_OK;
    if (!h_block_tables || !h_jobs) return KV_EINVAL;
    const int32_t nseg = layout->chunk_tokens / layout->block_size;
    std::vector<uint8_t> seen(is_store ? (size_t)layout->num_slots : (size_t)layout->num_blocks, 0);
    for (int32_t q = 0; q < num_jobs; ++q) {
        const kv_job &jb = h_jobs[q];
        if (jb.reserved != 0 || jb.slot < 0 || jb.slot >= layout->num_slots || jb.req < 0 || jb.req >= num_reqs ||
            jb.chunk < 0 || ((int64_t)jb.chunk + 1) * nseg > bt_stride)
            return KV_ERANGE;
        for (int32_t i = 0; i < nseg; ++i) {
            const int32_t blk = h_block_tables[(int64_t)jb.req * bt_stride + (int64_t)jb.chunk * nseg + i];
            if (blk < 0 || blk >= layout->num_blocks) return KV_ERANGE;
        }
    }
    for (int32_t q = 0; q < num_jobs; ++q) {
        const kv_job &jb = h_jobs[q];
        if (is_store) {
            if (seen[jb.slot]++) return KV_EDUP;
        } else {
            for (int32_t i = 0; i < nseg; ++i) {
                const int32_t blk = h_block_tables[(int64_t)jb.req * bt_stride + (int64_t)jb.chunk * nseg + i];
                if (seen[blk]++) return KV_EDUP;
            }
        }
    }
    return KV_OK;
}

int kv_commit_should_stage(double ttu_s, double ttr_s, uint64_t free_protected_bytes, uint64_t claim_new_bytes,
                           uint64_t claim_total_bytes, uint64_t budget_bytes, int retrieval_requested) {
    if (isnan(ttu_s) || isnan(ttr_s) || claim_new_bytes > claim_total_bytes) return KV_EINVAL;
    const bool eligible = ttu_s <= ttr_s || retrieval_requested != 0;
    if (!eligible) return KV_DEFER;
    const bool fits = claim_total_bytes <= budget_bytes && claim_new_bytes <= free_protected_bytes;
    if (fits) return KV_COMMIT;
    return retrieval_requested ? KV_ORDINARY : KV_BLOCKED;
}

int kv_commit_should_stage_n(int32_t n, const double *h_ttu, const double *h_ttr, uint64_t free_protected_bytes,
                             const uint64_t *h_claim_new, const uint64_t *h_claim_total, uint64_t budget_bytes,
                             const uint8_t *h_requested, int32_t *h_out) {
    if (n < 0) return KV_EINVAL;
    if (n > 0 && (!h_ttu || !h_ttr || !h_claim_new || !h_claim_total || !h_requested || !h_out)) return KV_EINVAL;
    for (int32_t i = 0; i < n; ++i)
        h_out[i] = kv_commit_should_stage(h_ttu[i], h_ttr[i], free_protected_bytes, h_claim_new[i], h_claim_total[i],
                                          budget_bytes, h_requested[i] != 0);
    return KV_OK;
}

const char *kv_strerror(int status) {
    switch (status) {
    case KV_OK: return "ok";
    case KV_EINVAL: return "invalid argument";
    case KV_EALIGN: return "pointer or stride not 16-byte aligned";
    case KV_ERANGE: return "slot, request, chunk or block id out of range";
    case KV_ENOSPC: return "no free staging slot or index full";
    case KV_EHIP: return "HIP runtime error";
    case KV_EDUP: return "duplicate destination within one batch";
    case KV_ELIMIT: return "request exceeds a fixed capacity of the call";
    default: return "unknown status";
    }
}

const char *kv_version(void) { return "tempokv 0.1.0 gfx950"; }

}  // extern "C"
