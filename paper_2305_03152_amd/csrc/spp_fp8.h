// Hidden rows in 8 bits: what the kernels that write and read them share.
//
// A row of D columns is a byte of E4M3 code per column (sign, four bits of exponent with bias 7, three of fraction; 0x7F and 0xFF
// are NaN, there is no infinity), zeros up to a multiple of 16 bytes, one E8M0 byte per block of 128 columns, zeros up to a
// multiple of 16 bytes.  Codes before scales, so that lanes take codes in aligned 16-byte loads.
#pragma once

#include "spp_mx4.h"

namespace spp {

constexpr int kFp8Block = 128;           // columns that share a scale
static inline __host__ __device__ int fp8_blocks(int32_t D) { return (D + kFp8Block - 1) / kFp8Block; }
static inline __host__ __device__ int fp8_code_bytes(int32_t D) { return (D + 15) / 16 * 16; }
static inline __host__ __device__ int fp8_bytes(int32_t D) { return fp8_code_bytes(D) + (fp8_blocks(D) + 15) / 16 * 16; }

// Scales that quantising gives: every value is then a normal number of fp32 and of bf16, which have the same exponents (the smallest
// 2^-9 2^-117), and the largest, 448 2^119, is below 2^128.
constexpr int kFp8LeastScale = 127 - 117, kFp8MostScale = 127 + 119;
constexpr uint32_t kFp8Most = 0x7F600000u;      // 448 2^119 as an fp32: what is larger is held as this

}  // namespace spp
