// Matrix-core building blocks shared by the prompt and attention kernels:
// binary16 planes of fp32 values, 16x16x32 products of them, transposing reads.
#pragma once

#include "stepq_seq.h"

namespace stepq {

using f16x2 = __attribute__((ext_vector_type(2))) _Float16;
using f16x8 = __attribute__((ext_vector_type(8))) _Float16;
using f32x2 = __attribute__((ext_vector_type(2))) float;
using f32x4 = __attribute__((ext_vector_type(4))) float;
using s16x4 = __attribute__((ext_vector_type(4))) short;
using u32x4 = __attribute__((ext_vector_type(4))) uint32_t;
using u32x2 = __attribute__((ext_vector_type(2))) uint32_t;

// Operand and result layout of the 16x16x32 block, lane = 16 g + n (checked
// on the device): operand A holds row n, operand B column n, 8 summation slots
// 8 g .. 8 g + 7 each; the result holds column n, rows 4 g .. 4 g + 3.
//
// The slots may stand for the 32 summands in any order as long as both
// operands agree.  Slot 8 g + 4 h + j is summand 16 h + 4 g + j here: the
// results of two blocks (rows 0-15 and 16-31, column n in lane n) then are
// operand B of the next product without a move between lanes.

// A power of two that brings values of magnitude up to m below 2^14, near it
// (binary16 then keeps 11 bits of everything down to 2^-28 of m), and its inverse.
struct Pow2 {
    float up, down;
};
__device__ __forceinline__ Pow2 scale_for(uint32_t m_bits)
{
    const uint32_t e = max(m_bits >> 23, 14u);
    return Pow2{__uint_as_float((267u - e) << 23), __uint_as_float((e - 13u) << 23)};
}

// N binary16 planes of 8 floats times a power of two: the value rounded to 11
// bits, then what that leaves, rounded to 11 more (22 bits; the difference is exact).
template <int N>
__device__ __forceinline__ void split(const float (&x)[8], float up, f16x8 (&p)[N])
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const f16x2 hi = __builtin_convertvector((f32x2{x[2 * i] * up, x[2 * i + 1] * up}), f16x2);
        p[0][2 * i] = hi[0], p[0][2 * i + 1] = hi[1];
        if constexpr (N > 1) {
            const f32x2 r = {fmaf(x[2 * i], up, -static_cast<float>(hi[0])), fmaf(x[2 * i + 1], up, -static_cast<float>(hi[1]))};
            const f16x2 lo = __builtin_convertvector(r, f16x2);
            p[1][2 * i] = lo[0], p[1][2 * i + 1] = lo[1];
        }
    }
}
template <int N>
__device__ __forceinline__ void split(const f32x4 &a, const f32x4 &b, float up, f16x8 (&p)[N])
{
    const float x[8] = {a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
    split(x, up, p);
}

// c += a b over planes, without the terms of order LIM and up (each order is
// 2^-11 of the one before it).
template <int LIM, int NA, int NB>
__device__ __forceinline__ void mma(f32x4 &c, const f16x8 (&a)[NA], const f16x8 (&b)[NB])
{
#pragma unroll
    for (int o = LIM - 1; o >= 0; --o)
#pragma unroll
        for (int i = 0; i < NA; ++i)
            if (o - i >= 0 && o - i < NB) c = __builtin_amdgcn_mfma_f32_16x16x32_f16(a[i], b[o - i], c, 0, 0, 0);
}

template <int CTRL>
__device__ __forceinline__ uint32_t max_dpp(uint32_t x)
{
    return max(x, static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(x), CTRL, 0xf, 0xf, false)));
}
// The largest of the wave's values (as unsigned: the order of non-negative floats).
__device__ __forceinline__ uint32_t wave_max(uint32_t x)
{
    x = max_dpp<0x121>(x), x = max_dpp<0x122>(x), x = max_dpp<0x124>(x), x = max_dpp<0x128>(x);   // row_ror 1, 2, 4, 8
    const auto at = [&](int l) { return static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(x), l)); };
    return max(max(at(0), at(16)), max(at(32), at(48)));
}
// The largest over the lanes n, n + 16, n + 32, n + 48: over a column of results.
__device__ __forceinline__ uint32_t column_max(uint32_t x)
{
    const auto a = __builtin_amdgcn_permlane16_swap(x, x, false, false);
    x = max(a[0], a[1]);
    const auto b = __builtin_amdgcn_permlane32_swap(x, x, false, false);
    return max(b[0], b[1]);
}

// Four rows of one column of 16-bit values in LDS: the 16 lanes of a group
// give the addresses of 4 rows x 16 columns (lane l: row l / 4, columns
// 4 (l % 4) .. + 3), and lane l receives column l.
__device__ __forceinline__ u32x2 read_columns(const uint8_t *lds)
{
    using P = __attribute__((address_space(3))) s16x4 *;
    return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((P)(lds)));
}

// The order of N steps of M products and the R reads of LDS that each needs: A steps are read ahead.
template <int N, int R, int M, int A>
__device__ __forceinline__ void reads_ahead()
{
    constexpr int product = 0x8, read = 0x100;
    __builtin_amdgcn_sched_group_barrier(read, R * A, 0);
#pragma unroll
    for (int i = 0; i < N - A; ++i) {
        __builtin_amdgcn_sched_group_barrier(product, M, 0);
        __builtin_amdgcn_sched_group_barrier(read, R, 0);
    }
    __builtin_amdgcn_sched_group_barrier(product, M * A, 0);
}

// A barrier that orders the waves' LDS accesses, and does not wait for copies and other global accesses under way.
__device__ __forceinline__ void lds_barrier()
{
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}
__device__ __forceinline__ float lower_bf16(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float upper_bf16(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

// Row-major tiles of 16-bit values in LDS, rows of BYTES = 128 or 256 bytes, their
// 16-byte slots exchanged within the row so that both the 16 rows of an
// operand read and the 4 x 4 slots of a transposing read fall on different banks.
template <int BYTES>
__device__ __forceinline__ int swizzle(int row)
{
    return BYTES == 256 ? ((row & 3) << 2) | ((row >> 2) & 3) : (((row >> 1) & 1) << 2) | ((row >> 2) & 3);
}

}  // namespace stepq
