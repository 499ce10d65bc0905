// How a paged key/value cache lies in memory, for the kernels that write and read it.
//
// The cache is [pages][key/value heads] blocks; a block is the page's tokens of one head in tiles of 16,
// each tile in the order in which the fragments of mma.m16n8k16 want it: a lane (g = lane / 4,
// t = lane % 4) finds its keys of tokens g and g + 8, and its values of tokens 2t, 2t + 1, 2t + 8 and 2t + 9, in
// 16-byte (D = 64: 8-byte) pieces that lie side by side for the lanes of a warp. So a tile is read without bank
// conflicts as it was copied, and a token is appended without touching another token's bytes.
//
// In 4 bits (tile of D = 64 or 128 channels, groups of 64 channels with a scale and a zero point, standing for
// scale (code - zero)):
//   keys    [token 16][t 4][group][16 channels], channel = 64 group + 16 t + i, low nibble first
//   values  [p 2][g 8][t 4][group][m 2][b 2][4 channels], token = 8 p + 2 t + b, channel = 64 group + 8 g + 4 m + i
//   scales  bf16 [g 8][h 2][key, value][group], token = 8 h + g
//   zeros of keys    u16 [g 8][h 2][group]
//   zeros of values  u16 [t 4][p 2][group][b 2];  both as 17 times the zero point: it is wanted at two places
// In bf16:
//   keys    [channel / 32][token 16][32]
//   values  [p 2][channel / 32][g 8][t 4][i 4][b 2], channel = 32 (channel / 32) + 4 g + i
#pragma once

#include <cuda_bf16.h>
#include <stdint.h>

#include "common.cuh"
#include "kernels.h"

namespace hydra {

constexpr int kKvTile = 16;    // tokens
constexpr int kKvGroup = 64;   // channels of a scale

template <int kDh, bool kInt4>
struct KvTile {
  static constexpr int kGroups = kDh / kKvGroup;
  static constexpr int kValues = kInt4 ? 8 * kDh : 32 * kDh;  // byte offsets within a tile
  static constexpr int kScales = 16 * kDh;
  static constexpr int kZerosK = kScales + 64 * kGroups;
  static constexpr int kZerosV = kZerosK + 32 * kGroups;
  static constexpr int kBytes = kInt4 ? 16 * kDh + 128 * kGroups : 64 * kDh;

  // 8 channels from d on (a multiple of 8) of a token's key: in 4 bits a word, in bf16 16 bytes
  static __host__ __device__ constexpr int key(int token, int d) {
    if constexpr (kInt4)
      return token * (kDh / 2) + ((d & 63) >> 4) * (8 * kGroups) + (d >> 6) * 8 + ((d >> 3) & 1) * 4;
    else
      return ((d >> 5) * kKvTile + token) * 64 + (d & 31) * 2;
  }
  // 4 channels from d on (a multiple of 4) of a token's value: in 4 bits two bytes, in bf16 every other of
  // the 8 bf16 from here on
  static __host__ __device__ constexpr int value(int token, int d) {
    const int p = token >> 3, t = (token & 7) >> 1, b = token & 1;
    if constexpr (kInt4)
      return kValues + ((p * 8 + ((d & 63) >> 3)) * 4 + t) * (8 * kGroups) + (d >> 6) * 8 + ((d >> 2) & 1) * 4 + b * 2;
    else
      return kValues + (((p * (kDh / 32) + (d >> 5)) * 8 + ((d & 31) >> 2)) * 4 + t) * 16 + b * 2;
  }
  static __host__ __device__ constexpr int scale(int token, bool of_value, int group) {
    return kScales + (((token & 7) * 2 + (token >> 3)) * 2 + (of_value ? 1 : 0)) * (2 * kGroups) + group * 2;
  }
  static __host__ __device__ constexpr int zero(int token, bool of_value, int group) {
    if (of_value)
      return kZerosV + ((((token & 7) >> 1) * 2 + (token >> 3)) * kGroups + group) * 4 + (token & 1) * 2;
    return kZerosK + ((token & 7) * 2 + (token >> 3)) * (2 * kGroups) + group * 2;
  }
};

// A sequence's part of a call: n new tokens (0..L) behind `cached` ones. A length outside [0, L] is clamped
// (0x202); a negative `cached`, or positions past what the table or the rotation table hold (0x204), leave nothing
// that could be addressed: ok is false and n counts the rows that the caller marks.
struct KvSeq {
  int cached, n;
  bool ok;
};
__device__ __forceinline__ KvSeq kv_seq(const KvBatch& b, int s, long long positions, int* err) {
  KvSeq q;
  q.cached = b.cached != nullptr ? b.cached[s] : 0;
  const int len = b.lengths != nullptr ? b.lengths[s] : static_cast<int>(b.L);
  q.n = min(max(len, 0), static_cast<int>(b.L));
  if (q.n != len) record_error(err, kDevBadLength);
  q.ok = q.cached >= 0 && static_cast<long long>(q.cached) + q.n <= positions;
  if (!q.ok && q.n > 0) record_error(err, kDevBadPosition);
  return q;
}

// The page of a position, or -1 (0x203) where the table's entry is none of the cache's.
__device__ __forceinline__ int kv_page(const KvBatch& b, const KvCache& c, int s, int pos, int* err) {
  const int page = b.table[static_cast<long long>(s) * b.ld_table + (pos >> c.page_bits)];
  if (page >= 0 && page < c.n_pages) return page;
  record_error(err, kDevBadPage);
  return -1;
}

// The tile of a position in a page, of one head.
template <typename Tile>
__device__ __forceinline__ uint8_t* kv_tile(const KvCache& c, int page, int head, int pos) {
  const int in_page = (pos & ((1 << c.page_bits) - 1)) / kKvTile;
  return static_cast<uint8_t*>(c.data) +
         (((static_cast<long long>(page) * c.kv_heads + head) << (c.page_bits - 4)) + in_page) * Tile::kBytes;
}

}  // namespace hydra
