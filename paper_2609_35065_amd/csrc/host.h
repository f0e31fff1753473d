// host.h -- declarations shared by the host-only code (host.cpp) and the
// GPU entry points; no HIP header.
#pragma once

#include <stdint.h>

#include "tempokv.h"

namespace tkv {

// Layout checks shared by the copy directions and staging.  Returns KV_OK or
// a negative kv_status.
int check_layout(const kv_layout *lo);

// Operators over the paged cache: checks of their arguments, and the launch
// plan of the attention.
constexpr int kMaxHeadDim = 256, kMaxHeads = 65536, kMaxLength = 1 << 30;
constexpr int kSplitRows = 16, kSplitStep = 128;   // rows (query, head of the group) of a small attention tile, and
                                                   // keys that its workgroup takes in one step
constexpr int kTileRows = 128, kLargeRows = 256, kTileStep = 64;   // the same of a tile for many rows, small or large
constexpr int kMaxSplits = 64;

struct AttentionPlan {
    int32_t rows;         // of a tile: kSplitRows, kTileRows or kLargeRows
    int64_t tiles;        // row tiles, each for every KV head
    int32_t splits;       // parts that a tile's keys are cut into
    int64_t workspace;    // bytes
};

struct WeightPlan {
    bool windowed;        // the kernels that know which keys a window leaves out
    bool few;             // no request has more than 16 rows a head
    bool ahead;           // of these: a wave passes several tiles of 64 keys
    int32_t keys;         // of a workgroup's tile of many rows: 64, 128 or 256
    int64_t tiles;        // workgroups for keys, each for every request and KV head
    int32_t sink_tiles;   // and for 64 sinks each,
    int32_t parts;        // times the parts that their rows are cut into
    int64_t workspace;    // bytes
};

int check_cache(const kv_layout *lo, int32_t cache_dtype);
int check_span(const kv_layout *lo);
int check_batch(const kv_batch *b);
int check_rows(const kv_rows *x, int64_t num, int32_t head_dim, bool written);
int plan_attention(const kv_layout *lo, const kv_batch *b, int32_t q_heads, int32_t window, int32_t sink, AttentionPlan *plan);
int plan_weights(const kv_layout *lo, const kv_batch *b, int32_t q_heads, int32_t window, int32_t sink, WeightPlan *plan);

}  // namespace tkv
