// paged.h -- device-side view of one layer's paged cache and of a ragged
// batch of new tokens, shared by the operators over the cache.
#pragma once

#include "internal.h"

namespace tkv {

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef int32_t i32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// Division of a non-negative 31-bit number by a fixed one: n / d =
// (n * mul) >> shift with mul = ceil(2^shift / d), shift = 31 + ceil(log2 d).
// The error n * (mul * d - 2^shift) / (d * 2^shift) stays below 1/d.
struct Divider {
    uint32_t mul;
    uint32_t shift;
};

inline Divider make_divider(uint32_t d) {
    uint32_t lg = 0;
    while ((uint64_t(1) << lg) < d) ++lg;
    const uint32_t shift = 31 + lg;
    return {(uint32_t)(((uint64_t(1) << shift) + d - 1) / d), shift};
}

__device__ __forceinline__ uint32_t divide(uint32_t n, Divider d) { return (uint32_t)(((uint64_t)n * d.mul) >> d.shift); }

// Rows are addressed in 32-bit units of 16 bytes from a plane's first block
// (the host refuses layers that span 64 GiB or more).
struct Paged {
    char *layer;
    const int32_t *bt;
    const int64_t *q_off;
    const int32_t *kv_len;
    int64_t kv_stride;
    int64_t num_blocks;
    int64_t num_q;
    uint32_t blocks;       // num_blocks, block ids being 31 bits
    uint32_t block16;      // 16-byte units between blocks of a plane
    uint32_t row16;        // and between the token rows of a block
    uint32_t block_size;
    Divider by_block;
    int32_t bt_stride;
    int32_t num_reqs;
    int32_t head_bytes;    // head_dim * elem_bytes
};

inline Paged make_paged(const kv_layout *lo, const void *layer, const kv_batch *b) {
    Paged p;
    p.layer = (char *)layer;
    p.bt = b->d_block_tables;
    p.q_off = b->d_q_off;
    p.kv_len = b->d_kv_len;
    p.kv_stride = lo->paged_kv_stride;
    p.num_blocks = lo->num_blocks;
    p.blocks = (uint32_t)(lo->num_blocks < INT32_MAX ? lo->num_blocks : INT32_MAX);
    p.num_q = b->num_q;
    p.block16 = (uint32_t)(lo->paged_block_stride / 16);
    p.head_bytes = lo->head_dim * lo->elem_bytes;
    p.row16 = (uint32_t)((int64_t)lo->kv_heads * p.head_bytes / 16);
    p.block_size = (uint32_t)lo->block_size;
    p.by_block = make_divider((uint32_t)lo->block_size);
    p.bt_stride = b->bt_stride;
    p.num_reqs = b->num_reqs;
    return p;
}

// Block id and row within the block of cache index t of request r; -1 where
// the block is missing or past the table.
__device__ __forceinline__ int32_t block_of(const Paged &p, int32_t r, uint32_t t, uint32_t &row) {
    const uint32_t b = divide(t, p.by_block);
    row = t - b * p.block_size;
    if (b >= (uint32_t)p.bt_stride) return -1;
    const int32_t id = p.bt[(int64_t)r * p.bt_stride + b];
    return id < 0 || id >= p.num_blocks ? -1 : id;
}

// Rows of request r, kept inside the buffers whatever the offsets hold.
__device__ __forceinline__ int64_t clamp_row(const Paged &p, int64_t x) {
    return x < 0 ? 0 : (x > p.num_q ? p.num_q : x);
}

}  // namespace tkv
