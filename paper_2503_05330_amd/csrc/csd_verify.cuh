// csd — the cache of keys and values that a verifying pass works on: its layout in memory, and what its kernels share.
//
// Layout.  Keys and values are arrays [row][kv head][tokens][D] of their own, row: a prompt or a path, tokens rounded up to blocks of
// 32: a token that is written fills whole lines (8-bit heads of 128: one for its keys, one for its values), and no byte of
// another's.  (In the order of the matrix cores' operands, keys by eights of d's and values by eights of tokens, reads needed no
// turning, but a token lay in 17 lines: writing one of 64 x 16 paths of 8 heads took 12 us, and 9 tokens 21.)  The scales of
// an 8-bit cache lie in an array of their own, 64 bytes a block of 32 tokens: the biased exponents of the tokens' key scales,
// then of their value scales.
//
// Attention multiplies tiles of 32 tokens: scores S^T = K Q^T (rows: tokens, columns: query rows), then O^T += V^T P^T, both
// by v_mfma_f32_32x32x16, whose operands are 8 values of the contracted axis per lane.
#pragma once

#include <hip/hip_runtime.h>

#include "csd_verify.h"

namespace csd {
namespace verify {

constexpr int kBlock = 32;              // tokens of a block
constexpr int kScaleBytes = 2 * kBlock; // of a block's scales

typedef float Acc __attribute__((ext_vector_type(16)));
typedef uint32_t Words __attribute__((ext_vector_type(4)));   // 16 bytes
typedef uint32_t Pair __attribute__((ext_vector_type(2)));
typedef int16_t Codes __attribute__((ext_vector_type(2)));    // four of 8 bits

struct BF16 {
  typedef __bf16 One;
  typedef __bf16 Two __attribute__((ext_vector_type(2)));
  typedef __bf16 Eight __attribute__((ext_vector_type(8)));
  static constexpr uint32_t kExponent = 0x7f80;   // all ones: infinity or NaN
  static __device__ Acc mfma(Eight a, Eight b, Acc c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
  template <bool HIGH>
  static __device__ Two from_fp8(uint32_t codes, float scale) {
    return __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, HIGH);
  }
  // the codes of four values over scale, a power of two
  static __device__ uint32_t to_fp8(Two low, Two high, float scale) {
    Codes codes{};
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(codes, low, scale, false);
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(codes, high, scale, true));
  }
};
struct F16 {
  typedef _Float16 One;
  typedef _Float16 Two __attribute__((ext_vector_type(2)));
  typedef _Float16 Eight __attribute__((ext_vector_type(8)));
  static constexpr uint32_t kExponent = 0x7c00;
  static __device__ Acc mfma(Eight a, Eight b, Acc c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
  template <bool HIGH>
  static __device__ Two from_fp8(uint32_t codes, float scale) {
    return __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(codes, scale, HIGH);
  }
  // the codes of four values over scale, a power of two
  static __device__ uint32_t to_fp8(Two low, Two high, float scale) {
    Codes codes{};
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp8_f16(codes, low, scale, false);
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_fp8_f16(codes, high, scale, true));
  }
};

// Eight e4m3 codes as values, times a power of two (the conversion looks at the scale's exponent alone).
template <class T>
__device__ inline typename T::Eight from_fp8(Pair codes, float scale) {
  union {
    typename T::Two two[4];
    typename T::Eight eight;
  } x;
  x.two[0] = T::template from_fp8<false>(codes[0], scale);
  x.two[1] = T::template from_fp8<true>(codes[0], scale);
  x.two[2] = T::template from_fp8<false>(codes[1], scale);
  x.two[3] = T::template from_fp8<true>(codes[1], scale);
  return x.eight;
}

// One layer's prompts or paths.
struct Held {
  uint8_t *keys, *values;            // [row][kv head][blocks * 32][D]
  uint8_t* scale;                    // [row][kv head][blocks][64], 8-bit only
  int32_t cap;                       // tokens of a row
  int32_t blocks;                    // of a row and head
  __device__ __host__ int64_t first(int64_t row, int32_t head, int32_t heads) const { return (row * heads + head) * blocks; }
};

constexpr int64_t block_bytes(int64_t head_dim, bool fp8) { return kBlock * head_dim * (fp8 ? 1 : 2); }   // of the keys, of the values

// What a call of csd_attend hands to its kernels.
struct AttendArgs {
  Held prompt, path;
  csd_heads q;
  const int32_t *prompt_len, *path_len, *counts;
  int32_t P, N, n, H, Hk, G;         // G query heads to a kv head
  float scale;                       // times log2(e)
  void* out;
  float* lse;
  float* part_o;                     // [split][row][D] and [split][row]; split: the prompt's, then the paths'
  float* part_lse;                   // base 2
  int64_t rows;                      // P N n H
  int32_t prompt_splits, path_splits;
  int32_t prompt_tiles, path_tiles;  // tiles of query rows of a (problem, kv head), of a (path, kv head)
  int32_t prompt_groups;             // workgroups of the prompts' items, before those of the paths'
  int32_t solo;                      // a path's item is one wave's instead of a workgroup's
  int32_t paths_first;               // before the prompts'
  int32_t prompt_turns, path_turns;  // whether items that have tokens in common go to one XCD
  int32_t how;                       // one of these
};

// What the items of a launch do.
constexpr int32_t kParts = 0;            // prompts' and paths': parts, for attend_join_kernel
constexpr int32_t kDirect = 1;           // paths' alone, with the whole prompt each: results

// What a call of csd_cache_write or csd_cache_read hands to its kernel.
struct MoveArgs {
  Held held;
  csd_heads k, v;                    // (read: dense)
  const int32_t *start, *counts;
  int64_t rows;
  int32_t n, Hk, groups;             // groups of eight of the n tokens
  uint32_t* status;
};

// The shape of a call of csd_attend; every head_dim's kernels have a source of their own.
struct AttendLaunch {
  uint32_t groups;                   // workgroups of attend_rows_kernel
  bool join, f16, fp8;
};
void attend_64(const AttendArgs& a, const AttendLaunch& how, hipStream_t st);
void attend_96(const AttendArgs& a, const AttendLaunch& how, hipStream_t st);
void attend_128(const AttendArgs& a, const AttendLaunch& how, hipStream_t st);
void attend_256(const AttendArgs& a, const AttendLaunch& how, hipStream_t st);

// The bounds are of the lengths, 0 the capacities.  attend_form() sets a's sizes and form of launch for n tokens a path.
AttendLaunch attend_form(AttendArgs* a, const csd_cache_config& cfg, int32_t n, int32_t prompt_bound, int32_t path_bound);
void attend_any(const AttendArgs& a, const AttendLaunch& how, int32_t head_dim, hipStream_t st);
// How many parts calls of so many rows write at most.
int64_t parts_of_rows(int64_t rows, int32_t prompt_cap, int32_t path_cap);
void cache_write(const MoveArgs& a, int32_t head_dim, bool f16, bool fp8, hipStream_t st);
void cache_read(const MoveArgs& a, int32_t head_dim, bool f16, bool fp8, hipStream_t st);

}  // namespace verify
}  // namespace csd
