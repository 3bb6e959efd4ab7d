// The paged cache held in 4 bits: where a number's code lies, and how codes become numbers and back.
//
// A row of a kv head is cut into groups of 32 dims.  A group has a bf16 scale and 32 codes of 4 bits (sign, two exponent bits,
// one mantissa bit: 0, 0.5, 1, 1.5, 2, 3, 4, 6).  Two-bit mantissas times 8-bit scales are ten bits: exact in fp32, and the
// codes themselves exact in fp16, which is what the matrix instructions of the attention kernel take.
//   scale  the group's largest magnitude over 6, rounded to nearest even: 4.5 bits per number; no calibration, no second
//          scale, and any bf16 or fp32 input fits.  (Power-of-two scales would cost 0.25 bits less and have 14 % more error on
//          normal data; scales of 8 bits per 16 dims up to 7 % less, but they need a scale of their own.)
//   small  a scale below 2^-126 is stored as 0 and the group as zeros
//   NaN    a group with a number that is not finite has a NaN as its scale: all of it reads as NaN
// The pool of a layer is [n_pages][n_kv_heads][page_rows / 16] blocks of 18 D bytes.  A block holds the keys and the values of
// 16 rows, so that one bulk copy of 2304 bytes (D = 128) brings all that a warp needs for a step, in the order in which the
// lanes of its matrix instructions read it from shared memory without bank conflicts:
//   0     key codes    row r: D/2 bytes at r * D/2; dims 32 j + 8 t + i (j = group, t < 4, i < 8) at t * D/8 + 4 j + i / 2
//   8 D   value codes  row r = 8 h + 2 t + p: dims 32 j + 4 u + i (u < 8, i < 4) at h * 4 D + u * D/2 + t * D/8 + p * D/16 + 2 j + i / 2
//   16 D  key scales   bf16 [16][D/32]
//   17 D  value scales bf16 [16][D/32]
// The low half of a byte holds the even dim.
#pragma once

#include <cuda_fp16.h>

#include "cf_common.cuh"

namespace cf {
namespace kv4 {

constexpr int kBlockRows = 16;
constexpr int kGroup = 32;                       // dims that share a scale

__host__ __device__ constexpr int block_bytes(int head_dim) { return 18 * head_dim; }

// Where row `row` (0..15) of a block of head_dim D starts.
template <int D> __device__ __forceinline__ int key_code_at(int row) { return row * (D / 2); }
template <int D> __device__ __forceinline__ int value_code_at(int row, int u) {
    return 8 * D + (row >> 3) * (4 * D) + u * (D / 2) + ((row & 7) >> 1) * (D / 8) + (row & 1) * (D / 16);
}
template <int D> __device__ __forceinline__ int key_scale_at(int row) { return 16 * D + row * (D / 16); }
template <int D> __device__ __forceinline__ int value_scale_at(int row) { return 17 * D + row * (D / 16); }

// The two codes of byte I of a word as fp16 numbers, the low half of the byte in the low half.
template <int I>
__device__ __forceinline__ uint32_t two_numbers(uint32_t word) {
    uint32_t r;
    static_assert(I >= 0 && I < 4, "a byte of a word");
    if (I == 0) asm("{\n.reg .b8 b0, b1, b2, b3;\nmov.b32 {b0, b1, b2, b3}, %1;\ncvt.rn.f16x2.e2m1x2 %0, b0;\n}" : "=r"(r) : "r"(word));
    if (I == 1) asm("{\n.reg .b8 b0, b1, b2, b3;\nmov.b32 {b0, b1, b2, b3}, %1;\ncvt.rn.f16x2.e2m1x2 %0, b1;\n}" : "=r"(r) : "r"(word));
    if (I == 2) asm("{\n.reg .b8 b0, b1, b2, b3;\nmov.b32 {b0, b1, b2, b3}, %1;\ncvt.rn.f16x2.e2m1x2 %0, b2;\n}" : "=r"(r) : "r"(word));
    if (I == 3) asm("{\n.reg .b8 b0, b1, b2, b3;\nmov.b32 {b0, b1, b2, b3}, %1;\ncvt.rn.f16x2.e2m1x2 %0, b3;\n}" : "=r"(r) : "r"(word));
    return r;
}

// A byte with the codes of two numbers (`even` in its low half): nearest, ties to the even code, magnitudes above 6 to 6.
__device__ __forceinline__ uint32_t two_codes(float even, float odd) {
    uint32_t r;
    asm("{\n.reg .b8 b;\ncvt.rn.satfinite.e2m1x2.f32 b, %1, %2;\nmov.b32 %0, {b, 0, 0, 0};\n}" : "=r"(r) : "f"(odd), "f"(even));
    return r;
}

__device__ __forceinline__ float bf16_low(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_high(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

}  // namespace kv4

// A cf_pages descriptor as the kernels take it.
struct PagesView {
    int n_requests, page_rows, n_pages, table_cols;
    int* table;
    int* rows;
    int* free_pages;
    int* free_count;
    int* status;
};
// CF_OK, or what is wrong with the descriptor.
int check_pages(const cf_pages* p);
PagesView make_pages_view(const cf_pages* p);

}  // namespace cf
