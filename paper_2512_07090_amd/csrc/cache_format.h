// Rows of a cache in 4 or 8 bits: the bytes of a page, and rows to and from them.
//
// A row of 128 columns is four blocks of 32, each with one scale s = 2^(E - 127), E in a byte: the smallest
// power of two, E >= 1, with max|x| <= M s (M = 6, the largest e2m1 value, or 448, the largest e4m3 value).
// A code is x / s rounded to nearest even.  Dividing by a power of two is exact, so codes do not depend on
// how they are computed, nothing saturates, and both types convert in the hardware.  A block that holds a NaN or
// an infinity has E = 255, of which the hardware's conversions make a NaN whatever the code.
//
// A page holds 64 rows of one head: their codes, then 256 scale bytes.  Keys lie as rows (a lane of the
// attention reads one block of one key), their scales as [block][row % 16][row / 16], so that one dword is the
// scales of a lane's four keys.  Values lie as [row / 4][column / 8][row % 4][8 columns] and their scales as
// [row / 4 % 4][block][row / 16][row % 4]: what a lane needs of four keys is 16 (32) bytes in a row.
#pragma once

#include "tf_kernels.h"

namespace tf {

constexpr int kPageRows = 64, kBlockCols = 32;

// a row's place in its page: bytes to the codes of its eight columns 8 c, and to the scale of block blk
template <int BITS> __host__ __device__ constexpr int page_codes() { return kPageRows * kHeadDim * BITS / 8; }
template <int BITS> __host__ __device__ constexpr int page_bytes() { return page_codes<BITS>() + kPageRows * kHeadDim / kBlockCols; }
template <int BITS> __host__ __device__ constexpr int key_code_at(int row, int c) { return row * (16 * BITS) + c * BITS; }
template <int BITS> __host__ __device__ constexpr int value_code_at(int row, int c) { return (row >> 2) * (64 * BITS) + c * (4 * BITS) + (row & 3) * BITS; }
template <int BITS> __host__ __device__ constexpr int key_scale_at(int row, int blk) { return page_codes<BITS>() + (blk * 16 + (row & 15)) * 4 + (row >> 4); }
template <int BITS> __host__ __device__ constexpr int value_scale_at(int row, int blk) { return page_codes<BITS>() + (((row >> 2) & 3) * 4 + blk) * 16 + (row >> 4) * 4 + (row & 3); }

#ifdef __HIPCC__
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef short s16x2 __attribute__((ext_vector_type(2)));

// the larger magnitude, a NaN if either is one (fmaxf passes over it, and a 4-bit code cannot hold it)
__device__ __forceinline__ float larger(float a, float b) { return __builtin_elementwise_maximum(a, b); }
// exponent byte of a block whose largest magnitude is `top`: mantissas up to that of M keep the exponent
template <int BITS>
__device__ __forceinline__ int block_exponent(float top)
{
    const int e = (int)((__float_as_uint(top) + (BITS == 4 ? 0x3fffffu : 0x1fffffu)) >> 23) - (BITS == 4 ? 2 : 8);
    return top < INFINITY ? max(e, 1) : 255;
}
__device__ __forceinline__ float exponent_scale(int e) { return __uint_as_float((unsigned)e << 23); }

// two values to two codes, in the low 8 (16) bits
template <int BITS>
__device__ __forceinline__ unsigned codes_of2(float a, float b, float scale)
{
    if constexpr (BITS == 4) return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, a, b, scale, 0) & 0xffu;
    else return __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(s16x2{0, 0}, a, b, scale, false)) & 0xffffu;
}
// eight values to a dword (two) of codes
template <int BITS>
__device__ __forceinline__ void codes_of8(const float* x, float scale, unsigned* w)
{
    if constexpr (BITS == 4) {
        unsigned r = 0;
        r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[0], x[1], scale, 0);
        r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[2], x[3], scale, 1);
        r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[4], x[5], scale, 2);
        w[0] = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[6], x[7], scale, 3);
    } else {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            s16x2 r = {0, 0};
            r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(r, x[4 * i], x[4 * i + 1], scale, false);
            r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(r, x[4 * i + 2], x[4 * i + 3], scale, true);
            w[i] = __builtin_bit_cast(unsigned, r);
        }
    }
}
// the reverse, in fp32
template <int BITS>
__device__ __forceinline__ void values_of8(const unsigned* w, float scale, float* x)
{
    f32x2 r[4];
    if constexpr (BITS == 4) {
        r[0] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[0], scale, 0);
        r[1] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[0], scale, 1);
        r[2] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[0], scale, 2);
        r[3] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[0], scale, 3);
    } else {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            r[2 * i] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w[i], scale, false);
            r[2 * i + 1] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w[i], scale, true);
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) { x[2 * i] = r[i][0]; x[2 * i + 1] = r[i][1]; }
}
// ... and as four pairs of bf16 (exact: a code has at most four significant bits)
template <int BITS>
__device__ __forceinline__ void bf16_of8(const unsigned* w, float scale, unsigned* pair)
{
    if constexpr (BITS == 4) {
        pair[0] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[0], scale, 0));
        pair[1] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[0], scale, 1));
        pair[2] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[0], scale, 2));
        pair[3] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[0], scale, 3));
    } else {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            pair[2 * i] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[i], scale, false));
            pair[2 * i + 1] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[i], scale, true));
        }
    }
}

// four of them: the first or the second half of a dword of 4-bit codes, or a dword of 8-bit ones
template <int BITS>
__device__ __forceinline__ void bf16_of4(unsigned w, int half, float scale, unsigned* pair)
{
    if constexpr (BITS == 8) {
        pair[0] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, false));
        pair[1] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, true));
    } else if (half == 0) {
        pair[0] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0));
        pair[1] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1));
    } else {
        pair[0] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2));
        pair[1] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3));
    }
}

// Eight columns 8 c of one row into row `row` of a page, by lane c of a 16-lane group whose lanes all take part
// (`store`: whether this group's row is to be written).  value: the layout of values, not keys.
template <int BITS>
__device__ __forceinline__ void store_row8(uint8_t* page, int row, int c, const float* x, bool value, bool store)
{
    float top = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) top = larger(top, fabsf(x[i]));
    top = larger(top, dpp_mov<0xB1>(top));   // the four lanes of a block
    top = larger(top, dpp_mov<0x4E>(top));
    const int e = block_exponent<BITS>(top);
    unsigned w[BITS / 4];
    codes_of8<BITS>(x, exponent_scale(e), w);
    if (!store) return;
    uint8_t* at = page + (value ? value_code_at<BITS>(row, c) : key_code_at<BITS>(row, c));
    if constexpr (BITS == 4) *reinterpret_cast<unsigned*>(at) = w[0];
    else *reinterpret_cast<uint2*>(at) = make_uint2(w[0], w[1]);
    if ((c & 3) == 0) page[value ? value_scale_at<BITS>(row, c >> 2) : key_scale_at<BITS>(row, c >> 2)] = (uint8_t)e;
}
#endif

}  // namespace tf
