// csd — the cache of keys and values that a verifying pass works on: its layout in memory, and what its kernels share.
//
// Layout.  Attention multiplies tiles of 32 tokens on the matrix cores: scores S^T = K Q^T (rows: tokens, columns: query
// rows), then O^T += V^T P^T, both by v_mfma_f32_32x32x16, whose operands are 8 consecutive values of the contracted
// axis per lane.  The cache holds blocks of 32 tokens of one head in the order in which a wave's lanes take these
// operands, so that a copy to LDS is linear and the reads from there are without gaps (eight tokens' values lie together, so a
// token that is written alone touches the lines of seven others, not those of all 32):
//   keys    16-bit  [D/16][half][row m][8 d's]          d = 16 c + 8 half + i
//           8-bit   [D/32][half][row m][2][8 d's]       two operands in a lane's 16 bytes
//   values  either  [D/32][2][half][32 d's][8 tokens]   token = 16 u + 8 half + i
// The result S^T leaves tokens 8 j + 4 half + r of its 32 rows in register 4 j + r of a lane.  With keys in row
// m(token) = the token's bits 2 and 3 exchanged, the lane's registers 8 u .. 8 u + 7 are tokens 16 u + 8 half ..
// + 7: the operand P^T of the second product without moving anything between lanes.
// A block is its keys, then its values.  The scales of an 8-bit cache lie in an array of their own, 64 bytes a block: the
// biased exponents of the 32 tokens' key scales, then of their value scales.
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
  uint8_t* data;     // [row][kv head][blocks][block_bytes]
  uint8_t* scale;    // [row][kv head][blocks][64], 8-bit only
  int32_t cap;       // tokens of a row
  int32_t blocks;    // of a row and head
  int64_t block_bytes;
  __device__ __host__ int64_t first(int64_t row, int32_t head, int32_t heads) const { return (row * heads + head) * blocks; }
};

constexpr int64_t block_bytes(int64_t head_dim, bool fp8) { return 2 * kBlock * head_dim * (fp8 ? 1 : 2); }

__device__ inline int key_row(int token) { return (token & 19) | (token & 4) << 1 | (token & 8) >> 1; }

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
  int32_t n, Hk, groups;             // groups of eight cache positions that n tokens touch at most
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

// The bounds are of the lengths, parts: how many parts of rows a call may write.
void attend_any(AttendArgs a, const csd_cache_config& cfg, int32_t prompt_bound, int32_t path_bound, int64_t parts, hipStream_t st);
void cache_write(const MoveArgs& a, int32_t head_dim, bool f16, bool fp8, hipStream_t st);
void cache_read(const MoveArgs& a, int32_t head_dim, bool f16, bool fp8, hipStream_t st);

}  // namespace verify
}  // namespace csd
