// Matrix-core building blocks shared by the prompt and attention kernels:
// bfloat16 planes of fp32 values, 16x16x32 products of them, transposing reads.
#pragma once

#include "stepq_seq.h"

namespace stepq {

using bf16x2 = __attribute__((ext_vector_type(2))) __bf16;
using bf16x8 = __attribute__((ext_vector_type(8))) __bf16;
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

// Three bfloat16 planes of 8 floats, whose sum is the value itself: its upper
// half (8 bits, cut), what that leaves rounded to 8 bits, and the rest (at most
// 8 bits).  bfloat16 has fp32's exponents, so that a value keeps its bits whatever
// stands beside it in its row, column or tile.
__device__ __forceinline__ void split(const float (&x)[8], bf16x8 (&p)[3])
{
#pragma clang fp contract(off)              // of the value as rounded, whatever product it came from
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t a = __float_as_uint(x[2 * i]), b = __float_as_uint(x[2 * i + 1]);
        const bf16x2 hi = __builtin_bit_cast(bf16x2, __builtin_amdgcn_perm(b, a, 0x07060302u));
        const f32x2 r = {x[2 * i] - __uint_as_float(a & 0xffff0000u), x[2 * i + 1] - __uint_as_float(b & 0xffff0000u)};
        const bf16x2 mid = __builtin_convertvector(r, bf16x2);
        const bf16x2 lo = __builtin_convertvector((f32x2{r[0] - static_cast<float>(mid[0]), r[1] - static_cast<float>(mid[1])}), bf16x2);
        p[0][2 * i] = hi[0], p[0][2 * i + 1] = hi[1];
        p[1][2 * i] = mid[0], p[1][2 * i + 1] = mid[1];
        p[2][2 * i] = lo[0], p[2][2 * i + 1] = lo[1];
    }
}
__device__ __forceinline__ void split(const f32x4 &a, const f32x4 &b, bf16x8 (&p)[3])
{
    const float x[8] = {a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
    split(x, p);
}

// c += a b over planes, the smallest terms first, without those below 2^-22 of
// the product (a middle by a low plane, a low by a low).
template <int NA, int NB>
__device__ __forceinline__ void mma(f32x4 &c, const bf16x8 (&a)[NA], const bf16x8 (&b)[NB])
{
#pragma unroll
    for (int o = 2; o >= 0; --o)
#pragma unroll
        for (int i = 0; i < NA; ++i)
            if (o - i >= 0 && o - i < NB) c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[i], b[o - i], c, 0, 0, 0);
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
