// Trees of drafted tokens: launch descriptions of their layout and verification.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/rq.h"

namespace rq {

struct TreeMaskLaunch {
  const int32_t* parents;   // [B][n]
  const int32_t* new_len;   // [B] or NULL
  uint32_t* mask;           // [B][n][words]
  int32_t* depth;           // [B][n] or NULL
  int B, n, words;
};

// Entries of a row that a workgroup takes at once, and the most parts of a row.
constexpr int kVerifyStep = 16384, kVerifyParts = 64;

struct TreeVerifyLaunch {
  const int32_t *tokens, *parents;   // [B][n]
  const int32_t* new_len;            // [B] or NULL
  const void *target, *draft;        // [B][n][vocab]; draft may be NULL
  int64_t t_sb, t_sn, d_sb, d_sn;
  const float* uniforms;             // [B][n]
  int B, n, vocab, dtype, n_path;
  int32_t *path, *count, *next;
  int part, parts;                   // a row's entries, in parts
  double* sums;                      // [B][parts]: of the residual
  double* inverse;                   // [B][n]: 1 / s before each of the node's rejections
  int32_t* found;                    // [B][4]: last node (-1: no nodes), rejections, path full
};

// Whether two arrays share memory (none shares with NULL).
inline bool overlap(const void* a, uint64_t a_bytes, const void* b, uint64_t b_bytes) {
  const uint64_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return a && b && (x < y ? y - x < a_bytes : x - y < b_bytes);
}

hipError_t launch_tree_mask(const TreeMaskLaunch& a, hipStream_t s);
hipError_t launch_tree_verify(const TreeVerifyLaunch& a, hipStream_t s);

}  // namespace rq
