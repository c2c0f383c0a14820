// The paged key/value cache in the microscaled 4-bit form (mx_format.cuh): uint8 [pages][2][heads][page * (d / 2 + d / 32)], a
// head's part of a page its tokens' codes, then their scales.  A token's codes lie in pieces: with B = d / 32 blocks, keys as
// [4][B] words (word p of a block holds channels 8 p .. 8 p + 7), values as [8][B] halfwords (halfword p channels 4 p .. 4 p + 3).
// So quarter p of a row, 4 B bytes, is of keys and values alike what holds channels 8 p .. 8 p + 7 of every block.
#pragma once
#include "mx_format.cuh"

namespace cat {

__host__ __device__ constexpr int64_t mx_page_bytes(int64_t page, int64_t d) { return page * (d / 2 + d / 32); }

// Where things are in a cache.
struct MxCache {
  uint8_t* base;
  int64_t rows;                             // pages * page
  int page, page_log, hkv;
  int64_t part;                             // bytes of a head's keys (or values) of a page
  // kind 0: keys, 1: values of head h of page p
  __device__ __forceinline__ uint8_t* at(int64_t p, int kind, int h) const { return base + ((p * 2 + kind) * hkv + h) * part; }
};

}  // namespace cat
