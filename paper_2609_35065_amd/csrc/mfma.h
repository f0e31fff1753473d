// mfma.h -- the two 16-bit element types as the matrix units take them.
#pragma once

#include "paged.h"

namespace tkv {

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

__device__ __forceinline__ float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ float log2_(float x) { return __builtin_amdgcn_logf(x); }

// Bits of the non-finite values among a register's two elements, `exponent`
// being all ones in each: 0xffff for an element that is not finite.
template <uint32_t kExponent> __device__ __forceinline__ uint32_t nonfinite_mask(uint32_t x) {
    const uint32_t lo = (x & (kExponent & 0xffffu)) == (kExponent & 0xffffu) ? 0xffffu : 0u;
    const uint32_t hi = (x & (kExponent & 0xffff0000u)) == (kExponent & 0xffff0000u) ? 0xffff0000u : 0u;
    return lo | hi;
}

// Set the non-finite elements to 0; whether there were any.
template <uint32_t kExponent> __device__ __forceinline__ bool drop_nonfinite_(u32x4 &v) {
    uint32_t any = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t bad = nonfinite_mask<kExponent>(v[i]);
        v[i] &= ~bad;
        any |= bad;
    }
    return any != 0;
}

struct Bf16 {
    static constexpr bool kBf16 = true;
    static __device__ __forceinline__ f32x4 mfma16(u32x4 a, u32x4 b, f32x4 c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c,
                                                       0, 0, 0);
    }
    static __device__ __forceinline__ f32x16 mfma32(u32x4 a, u32x4 b, f32x16 c) {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c,
                                                       0, 0, 0);
    }
    static __device__ __forceinline__ uint32_t pack(float a, float b) {   // to nearest even
        const bf16x2 x = {(__bf16)a, (__bf16)b};
        return __builtin_bit_cast(uint32_t, x);
    }
    static __device__ __forceinline__ uint32_t from_f8(uint32_t x, bool high) {   // exact
        return __builtin_bit_cast(uint32_t, high ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, 1.0f, true)
                                                 : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, 1.0f, false));
    }
    static __device__ __forceinline__ bool drop_nonfinite(u32x4 &v) { return drop_nonfinite_<0x7f807f80u>(v); }
    static __device__ __forceinline__ float to_f32(uint32_t x) { return __builtin_bit_cast(float, x << 16); }
};

struct F16 {
    static constexpr bool kBf16 = false;
    static __device__ __forceinline__ f32x4 mfma16(u32x4 a, u32x4 b, f32x4 c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0,
                                                      0, 0);
    }
    static __device__ __forceinline__ f32x16 mfma32(u32x4 a, u32x4 b, f32x16 c) {
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0,
                                                      0, 0);
    }
    static __device__ __forceinline__ uint32_t pack(float a, float b) {   // to nearest even
        const f16x2 x = {(_Float16)a, (_Float16)b};
        return __builtin_bit_cast(uint32_t, x);
    }
    static __device__ __forceinline__ uint32_t from_f8(uint32_t x, bool high) {   // exact
        return __builtin_bit_cast(uint32_t, high ? __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(x, 1.0f, true)
                                                 : __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(x, 1.0f, false));
    }
    static __device__ __forceinline__ bool drop_nonfinite(u32x4 &v) { return drop_nonfinite_<0x7c007c00u>(v); }
    static __device__ __forceinline__ float to_f32(uint32_t x) { return (float)__builtin_bit_cast(_Float16, (uint16_t)x); }
};

template <class T> __device__ __forceinline__ uint32_t pack2(float a, float b) { return T::pack(a, b); }

// Eight elements of the 8-bit type.
template <class T> __device__ __forceinline__ u32x4 unpack8(uint32_t a, uint32_t b) {
    return u32x4{T::from_f8(a, false), T::from_f8(a, true), T::from_f8(b, false), T::from_f8(b, true)};
}

// A value of both lanes 32 apart: lane i's (y[0]) and lane i + 32's (y[1]).
__device__ __forceinline__ f32x2 both_halves(float x) {
    const uint32_t b = __builtin_bit_cast(uint32_t, x);
    return __builtin_bit_cast(f32x2, __builtin_amdgcn_permlane32_swap(b, b, false, false));
}

// a with its upper 32 lanes exchanged for the lower 32 of b, and b likewise.
__device__ __forceinline__ u32x2 swap_halves(uint32_t a, uint32_t b) {
    return __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane32_swap(a, b, false, false));
}

// Sixteen rows of LD * 64 bytes as the 16 x 16 products take them: lane (col,
// quad) has of row `col` the bytes 64 ks + 16 quad on, in y[ks].  Loaded that
// way an instruction would take 64 bytes of each row, half a cache line.  So
// of each pair of pieces lanes load 128 bytes of eight rows at a time, and
// arrange_rows then exchanges columns eight apart.  `at_row(r)` is where row r
// starts; bytes from `bytes` on are zero.  All 64 lanes take part.
template <int LD, class F> __device__ __forceinline__ void load_rows(u32x4 (&y)[LD], int bytes, F at_row) {
    const int lane = threadIdx.x & 63, col = lane & 15, quad = lane >> 4;
    const int wide = (quad + 4 * (col >> 3)) * 16;
    if constexpr (LD > 1) {
        const char *a = at_row(col & 7), *b = at_row(8 + (col & 7));
#pragma unroll
        for (int ks = 0; ks + 1 < LD; ks += 2) {
            const bool in = ks * 64 + wide < bytes;
            y[ks] = in ? *(const u32x4 *)(a + ks * 64 + wide) : u32x4{0, 0, 0, 0};
            y[ks + 1] = in ? *(const u32x4 *)(b + ks * 64 + wide) : u32x4{0, 0, 0, 0};
        }
    }
    if constexpr (LD % 2) {
        const int at = (LD - 1) * 64 + quad * 16;
        const char *a = at_row(col);
        y[LD - 1] = at < bytes ? *(const u32x4 *)(a + at) : u32x4{0, 0, 0, 0};
    }
}

template <int LD> __device__ __forceinline__ void arrange_rows(u32x4 (&y)[LD]) {
    constexpr int kTurn8 = 0x128;          // rotate by 8 within 16 lanes; banks of four lanes
#pragma unroll
    for (int ks = 0; ks + 1 < LD; ks += 2)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int a = (int)y[ks][i], b = (int)y[ks + 1][i];
            y[ks][i] = (uint32_t)__builtin_amdgcn_update_dpp(a, b, kTurn8, 0xf, 0xc, false);
            y[ks + 1][i] = (uint32_t)__builtin_amdgcn_update_dpp(b, a, kTurn8, 0xf, 0x3, false);
        }
}

// Transposing read from LDS.  Of each 16 lanes, lane s gives the address of
// four consecutive 16-bit elements, 4 (s % 4) .. of row s / 4; lane s gets
// element s of the four rows.
__device__ __forceinline__ u32x2 read_transposed(const char *at) {
    const s16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
        (__attribute__((address_space(3))) s16x4 *)const_cast<char *>(at));
    return __builtin_bit_cast(u32x2, x);
}

}  // namespace tkv
