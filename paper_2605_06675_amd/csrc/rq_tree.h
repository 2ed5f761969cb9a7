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

// Entries of a row that a workgroup takes at once, the most parts of a row, and of how
// many sums over a row the parts are shared.
constexpr int kVerifyStep = 8192, kVerifyParts = 64, kVerifySums = 16;

struct TreeVerifyLaunch {
  const int32_t *tokens, *parents;   // [B][n]
  const int32_t* new_len;            // [B] or NULL
  const void *target, *draft;        // [B][n][vocab]; draft may be NULL
  int64_t t_sb, t_sn, d_sb, d_sn;
  const float* uniforms;             // [B][n]
  int B, n, vocab, dtype, n_path;
  int32_t *path, *count, *next;
  int part, parts;                   // a row's entries, in parts, a workgroup each
  uint64_t* slots;                   // [B][kVerifySums][parts]: sums, or 0
  uint32_t* done;                    // [B]: workgroups that are
  int spread;                        // 2^spread threads look for a node's siblings
};

// Whether two arrays share memory (none shares with NULL).
inline bool overlap(const void* a, uint64_t a_bytes, const void* b, uint64_t b_bytes) {
  const uint64_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return a && b && (x < y ? y - x < a_bytes : x - y < b_bytes);
}

hipError_t launch_tree_mask(const TreeMaskLaunch& a, hipStream_t s);
hipError_t launch_tree_verify(const TreeVerifyLaunch& a, hipStream_t s);

}  // namespace rq
