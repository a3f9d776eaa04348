// The 4-bit weights with group scales, as their writers and readers share them.
//
// Codes: blocks of 16 rows x 128 columns, 1 KB each, those of a row block one after the other.  The 64 places of a block are (c, r) = 16 c + r,
// 16 bytes each: word k of place (c, r) holds row r, columns 32 k + 8 c + 0..7.  A wavefront that gives lane 16 c + r place (c, r) reads whole
// blocks with one 16-byte load a lane, and word k is then, code by code, the lane's share of a matrix operand of 16 rows x 32 columns (lane 16 c
// + r: row r, 8 consecutive columns from 8 c on).
//
// A code is a whole number q of -7..7, kept as sign and size.  In a word the size of column b (b = 0..3) is in bits 8 b .. 8 b + 2 and its sign in
// bit 8 b + 7; the size of column 4 + b in bits 8 b + 4 .. 8 b + 6 and its sign in bit 8 ((b + 1) % 4) + 3.  So one mask over the word, and the
// same mask over the word rotated by 4, leave four bytes of sign and size each, and such a byte read as e4m3 is q 2^-9 exactly (the numbers below
// 2^-6 and those of the next binade are evenly spaced): the conversion instructions of 8-bit floats take codes apart.
//
// Scales: bfloat16 of 5 significant bits (the low 3 bits are 0), [groups][rows], rows and columns filled up to whole blocks (with scale 0, code
// 0).  A size of 3 bits times 5 bits has 8: q s is a bfloat16, exactly.
#pragma once

#include "skim_common.h"

#include <type_traits>

constexpr int GQ_ROWS = 16, GQ_COLS = 128;
constexpr uint32_t GQ_MASK = 0x87878787u;

typedef uint32_t gq_word4 __attribute__((ext_vector_type(4)));
typedef float gq_float2 __attribute__((ext_vector_type(2)));
typedef float gq_float4 __attribute__((ext_vector_type(4)));
typedef __bf16 gq_bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 gq_bf16x8 __attribute__((ext_vector_type(8)));

__host__ __device__ static inline int64_t gq_row_blocks(int64_t n) { return (n + GQ_ROWS - 1) / GQ_ROWS; }
__host__ __device__ static inline int64_t gq_col_blocks(int64_t m) { return (m + GQ_COLS - 1) / GQ_COLS; }

// Bytes of sign and size of columns 0..3 and 4..7 of a word.
__device__ __forceinline__ uint32_t gq_low(uint32_t w) { return w & GQ_MASK; }
__device__ __forceinline__ uint32_t gq_high(uint32_t w) { return __builtin_amdgcn_alignbit(w, w, 4) & GQ_MASK; }

// What every reader and writer of the format refuses.
skim_status skim_group_check(skim_ctx *ctx, const void *codes, const void *scales, int64_t n, int64_t m, int group, const char *who);

__device__ __forceinline__ float gq_scale(uint32_t bits) { return __uint_as_float(bits << 16); }

// f with the group as a constant.
template <typename F>
static inline void with_group(int group, F &&f) {
    if (group == 32) f(std::integral_constant<int, 32>{});
    else if (group == 64) f(std::integral_constant<int, 64>{});
    else f(std::integral_constant<int, 128>{});
}
