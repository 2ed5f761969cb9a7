// The block-scaled 8-bit cache: launch descriptions and the device code that
// its kernels share.
//
// One unit is one (batch entry, kv-head) of one layer.  Its cache holds, for K
// and for V, [token][D] codes of 8 bits and one fp32 scale per 32 tokens; the
// tokens of the unfinished last block stay in the 16-bit tail.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/rq.h"
#include "rq_device.h"

namespace rq {

constexpr int kBlockTokens = 32;
// Splits of an attention tile that its last workgroup may add.
constexpr int kTicketSplits = 32;
// Eviction: units of at most this many slots are selected by one workgroup
// (up to 32 keys a thread); longer ones in parts of a multiple of kSelectPart, at
// most kSelectParts of them.
constexpr int kSelectShort = 32768, kSelectPart = 8192, kSelectParts = 32;
constexpr int kSelectState = 12;     // words a unit (three a launch)

// One layer of a cache, and its shape.
// A divisor d, for x / d with x (d - 1) < 2^32 by one product (the compiler's own
// division is a chain of some twenty instructions).
struct Divider {
  uint32_t mul, one;
};
inline Divider divider(uint32_t d) {
  return d == 1 ? Divider{0u, ~0u} : Divider{(uint32_t)(((1ull << 32) + d - 1) / d), 0u};
}

struct BlockLayer {
  uint8_t* codes;       // [B][H][2][cap][D]
  float* scales;        // [B][H][2][cap / 32]
  uint16_t* tail;       // [B][H][2][32][D]
  int32_t* positions;   // [B][H][cap]
  float* weights;       // [B][H][cap] or NULL
  uint32_t* counters;   // [B][H] or NULL
  int B, H, cap;
  Divider by_H;
  int D, fmt, is_bf16;  // select the kernels
};

// A strided 16-bit or fp32 tensor [B][heads][tokens][D] with contiguous rows.
struct BlockRows {
  const void* p;
  int64_t sb, sh, st;   // strides in elements
};

struct BlockAppendLaunch {
  BlockLayer c;
  const int32_t* past;     // [B]
  const int32_t* new_len;  // [B] or NULL
  BlockRows k, v;
  int n;
};

struct BlockAdvanceLaunch {
  int32_t* lengths;        // [B], as the following
  const int32_t* new_len;  // or NULL
  int32_t *past, *fitting, *dropped;   // each or NULL
  int B, cap, n;
};

struct BlockAttendLaunch {
  BlockLayer c;
  const int32_t* past;
  const int32_t* new_len;
  BlockRows q, out;
  int out_dtype;
  int G, n, max_tokens;
  int row_tiles;           // tiles of 16 rows (token-major, heads of a group together)
  int splits;              // workgroups that share a row tile's tokens
  Divider by_G, by_splits;
  float qscale;            // scale * log2(e); scale / cap where scores are capped
  float cap;               // cap * log2(e), or 0
  int fine;                // many rows: the cap's tanh relative to itself
  int window;
  const float* slopes;     // [H * G] or NULL
  int accumulate;
  int tickets;             // the last of a row tile's splits adds them all
  float* part;             // [unit][row tile][split][16][D]
  float* part_ml;          // [unit][row tile][split][16][2]: maximum (log2) and sum
  float* stats;            // [unit][row][2]: maximum and 1 / sum, where accumulate
  float* scores;           // [unit][block][row][32]: log2 scores, where accumulate
                           // and there are at most 32 rows; else NULL
  uint16_t* queries;       // else: [unit][row][D] queries as fp16 operands,
  float* factors;          // [unit][row] and the factor of their scores;
  int row_parts;           // workgroups that share a token's rows,
  Divider by_parts;
  float* sums;             // and, of more than one, [part][unit][token] sums
};

// A tree of drafted tokens that attends over the cache and itself: past tokens
// are cached, the call's own rows are not.
struct BlockTreeLaunch : BlockAttendLaunch {
  BlockRows k, v;          // [B][H][n][D]
  const uint32_t* mask;    // [B][n][words]: the nodes that each one sees
  const int32_t* depth;    // [B][n], where positions matter
  int words;
  int most;                // bound on the cached tokens (max_tokens: that and n)
  int group_rows, waves;   // of a workgroup, where there are more than 16 rows
  int plain;               // no cap, window or slopes
};

// The accepted path's rows of every layer.
struct BlockAcceptLaunch {
  BlockLayer c;            // of layer 0
  int layers, n, n_path;
  const int32_t* lengths;  // [layers][B], as new_lengths to dropped
  const int32_t* path;     // [B][n_path]
  const int32_t* count;    // [B]
  BlockRows k, v;          // of layer 0
  int64_t k_layer, v_layer;
  int32_t *new_lengths, *past, *fitting, *dropped;   // the last three or NULL
};

struct BlockEvictLaunch {
  BlockLayer src, dst;
  const int32_t* lengths;
  int32_t* new_lengths;
  int keep, n_sink, n_recent;
  int32_t* slots;          // [unit][keep] source slots, ascending
  // selection of units in several parts (parts > 1) of `part` tokens each
  int part, parts;
  uint32_t* state;         // [unit][kSelectState]: what each launch found
  uint32_t* before;        // [unit][parts]: kept keys of the parts before
  uint32_t* counts;        // [3][unit][parts][2048]
};

hipError_t launch_block_append(const BlockAppendLaunch& a, hipStream_t s);
hipError_t launch_block_advance(const BlockAdvanceLaunch& a, hipStream_t s);
hipError_t launch_block_attend(const BlockAttendLaunch& a, hipStream_t s);
hipError_t launch_block_prompt(const BlockAttendLaunch& a, hipStream_t s);
hipError_t launch_block_merge(const BlockAttendLaunch& a, hipStream_t s);
hipError_t launch_block_weigh(const BlockAttendLaunch& a, hipStream_t s);
hipError_t launch_tree_attend(const BlockTreeLaunch& a, hipStream_t s);
hipError_t launch_tree_rows(const BlockTreeLaunch& a, hipStream_t s);
hipError_t launch_block_accept(const BlockAcceptLaunch& a, hipStream_t s);
hipError_t launch_block_evict(const BlockEvictLaunch& a, hipStream_t s);

typedef uint32_t u2 __attribute__((ext_vector_type(2)));
typedef float f2 __attribute__((ext_vector_type(2)));
typedef __bf16 b8 __attribute__((ext_vector_type(8)));
typedef _Float16 h4 __attribute__((ext_vector_type(4)));
// callers' rows may begin at any element
typedef u4 u4_any __attribute__((aligned(2)));
typedef u2 u2_any __attribute__((aligned(2)));
typedef uint32_t u1_any __attribute__((aligned(2)));
typedef f4 f4_any __attribute__((aligned(4)));

// Memory that no kernel writes while this one runs: uniform addresses are
// scalar loads.
#define RQ_CONSTANT __attribute__((address_space(4)))
template <class T>
__device__ __forceinline__ const RQ_CONSTANT T* cptr(const T* p) {
  return (const RQ_CONSTANT T*)p;
}

// New tokens of batch entry b, whatever the device array holds: 0 <= new <= n, most.
__device__ __forceinline__ int new_tokens(const int32_t* new_len, int b, int n, int most) {
  int nw = new_len ? gptr(new_len)[b] : n;
  nw = nw < 0 ? 0 : (nw > n ? n : nw);
  return nw > most ? most : nw;
}

// Cached and new tokens of batch entry b: 0 <= past, past + new <= most.
__device__ __forceinline__ void block_lengths(const int32_t* past, const int32_t* new_len, int b,
                                              int n, int most, int* p, int* w) {
  const int nw = new_tokens(new_len, b, n, most);
  int ps = gptr(past)[b];
  ps = ps < 0 ? 0 : (ps > most - nw ? most - nw : ps);
  *p = __builtin_amdgcn_readfirstlane(ps);
  *w = __builtin_amdgcn_readfirstlane(nw);
}

__device__ __forceinline__ int over(int x, Divider d) {
  return (int)(__umulhi((uint32_t)x, d.mul) + ((uint32_t)x & d.one));
}

// Where part i of n things begins, in `parts` parts.
__device__ __forceinline__ int part_from(int n, int i, int parts, Divider by_parts) {
  const int each = over(n, by_parts), more = n - each * parts;
  return each * i + (i < more ? i : more);
}

// The lengths that a launch's rows attend with.  A tree's nodes are not cached:
// past does not count them, and is bounded by itself.
template <class Launch>
constexpr bool kIsTree = __is_same(Launch, BlockTreeLaunch);
template <class Launch>
__device__ __forceinline__ void launch_lengths(const Launch& a, int b, int* past, int* nnew) {
  block_lengths(a.past, a.new_len, b, a.n, a.max_tokens, past, nnew);
  if constexpr (kIsTree<Launch>) *past = *past < a.most ? *past : a.most;
}

// Blocks that rows first..last (tokens of the call) see: [lo, hi).
__device__ __forceinline__ void seen_blocks(int past, int first, int last, int window, int* lo,
                                            int* hi) {
  *hi = (past + last) / kBlockTokens + 1;
  const int slot = window ? past + first - window + 1 : 0;
  *lo = slot > 0 ? slot / kBlockTokens : 0;
}

// A float's maximum or sum over lanes, in all of them: of a row of 16 lanes, of a
// lane and the one 16 or 32 further.  Register moves, a few cycles each where an
// exchange through LDS takes a hundred.
struct Max {
  __device__ __forceinline__ float operator()(float a, float b) const { return __builtin_fmaxf(a, b); }
};
struct Sum {
  __device__ __forceinline__ float operator()(float a, float b) const { return a + b; }
};
template <int CTRL>
__device__ __forceinline__ float moved(float x) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, 0xf, 0xf, true));
}
template <class F>
__device__ __forceinline__ float row_all(float x) {
  x = F()(x, moved<0xb1>(x));           // lanes 1 and 2 further in a quad,
  x = F()(x, moved<0x4e>(x));
  x = F()(x, moved<0x141>(x));          // the other quad of eight,
  return F()(x, moved<0x140>(x));       // the other eight
}
template <class F>
__device__ __forceinline__ float pair_all(float x) {
  const u2 p = __builtin_bit_cast(u2, __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false));
  return F()(__uint_as_float(p.x), __uint_as_float(p.y));
}
template <class F>
__device__ __forceinline__ float half_all(float x) {
  const u2 p = __builtin_bit_cast(u2, __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false));
  return F()(__uint_as_float(p.x), __uint_as_float(p.y));
}
template <class F>
__device__ __forceinline__ float wave_all(float x) {
  return half_all<F>(pair_all<F>(row_all<F>(x)));
}

// ------------------------------------------------------------- quantization
// The scale of a block whose largest magnitude is amax, and its reciprocal.
// Scales below the smallest normal number become 0 (their reciprocal would
// not be finite) and all codes with them.
template <int FMT>
__device__ __forceinline__ float block_scale(float amax, float* inv) {
  float s = amax * (FMT == RQ_INT8 ? 1.0f / 127.0f : 1.0f / 448.0f);
  s = s < 1.17549435e-38f ? 0.0f : s;
  *inv = s > 0.0f ? 1.0f / s : 0.0f;
  return s;
}

// Four codes from four values (two separately rounded fp32 steps: the product,
// then half-even to the code).  |x inv| exceeds the largest code by rounding
// only, which falls back to it: 127.00002 rounds to 127, 448.00003 to 448.
template <int FMT>
__device__ __forceinline__ uint32_t block_codes(float x0, float x1, float x2, float x3, float inv) {
  x0 *= inv;
  x1 *= inv;
  x2 *= inv;
  x3 *= inv;
  if constexpr (FMT == RQ_INT8) {
    // adding 1.5 * 2^23 rounds to whole numbers; the low byte is the code
    const uint32_t a = __float_as_uint(x0 + 12582912.0f), b = __float_as_uint(x1 + 12582912.0f);
    const uint32_t c = __float_as_uint(x2 + 12582912.0f), d = __float_as_uint(x3 + 12582912.0f);
    const uint32_t ab = __builtin_amdgcn_perm(b, a, 0x0c0c0400u);
    return __builtin_amdgcn_perm(__builtin_amdgcn_perm(d, c, 0x0c0c0400u), ab, 0x05040100u);
  } else {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(x0, x1, 0, false);
    w = __builtin_amdgcn_cvt_pk_fp8_f32(x2, x3, w, true);
    return inv > 0.0f ? (uint32_t)w : 0u;      // (not the code of -0)
  }
}

// The value of code byte i of w.
template <int FMT>
__device__ __forceinline__ float block_value(uint32_t w, int i) {
  if constexpr (FMT == RQ_INT8) return (float)(int8_t)(w >> (8 * i));
  switch (i) {   // (the byte's number is an immediate)
    case 0: return __builtin_amdgcn_cvt_f32_fp8((int)w, 0);
    case 1: return __builtin_amdgcn_cvt_f32_fp8((int)w, 1);
    case 2: return __builtin_amdgcn_cvt_f32_fp8((int)w, 2);
    default: return __builtin_amdgcn_cvt_f32_fp8((int)w, 3);
  }
}

__device__ __forceinline__ uint16_t bf16_rne(float x) {
  const uint32_t u = __float_as_uint(x);
  return (uint16_t)((u + 0x7fffu + ((u >> 16) & 1u)) >> 16);
}
template <bool BF16>
__device__ __forceinline__ uint16_t narrow_t(float x) {
  if constexpr (BF16) return bf16_rne(x);
  return __builtin_bit_cast(uint16_t, (_Float16)x);
}

// ------------------------------------------------------------ matrix operands
// Codes enter the matrix cores as fp16, which holds every int8 and e4m3 value
// exactly.  int8: the byte plus 128 under the exponent of 1024, minus 1152;
// where two bytes of different words meet (values) there is no room for the
// exponent byte in one permute, and the zero-extended byte, a subnormal number
// u 2^-24, becomes (u - 128) 2^-9 by one fused multiply-add.
template <int FMT>
constexpr float kValueUnit = FMT == RQ_INT8 ? 0x1p-9f : 1.0f;

// codes 0,1 (hi = false) or 2,3 of a word
template <int FMT>
__device__ __forceinline__ uint32_t key_pair(uint32_t w, bool hi) {
  if constexpr (FMT == RQ_INT8) {
    const uint32_t x = __builtin_amdgcn_perm(0x64646464u, w ^ 0x80808080u,
                                             hi ? 0x04030402u : 0x04010400u);
    return as_u32(as_h2(x) + (h2){(_Float16)-1152.0f, (_Float16)-1152.0f});
  } else {
    return hi ? as_u32(__builtin_bit_cast(h2, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, true)))
              : as_u32(__builtin_bit_cast(h2, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, false)));
  }
}

// Four channels (the bytes of a word) of two tokens a, b -> four fp16 pairs
// (a, b), in units of kValueUnit.
template <int FMT>
__device__ __forceinline__ void value_pairs(uint32_t a, uint32_t b, uint32_t out[4]) {
  if constexpr (FMT == RQ_INT8) {
    a ^= 0x80808080u;
    b ^= 0x80808080u;
    const h2 k = {(_Float16)32768.0f, (_Float16)32768.0f}, z = {(_Float16)-0.25f, (_Float16)-0.25f};
    out[0] = as_u32(__builtin_elementwise_fma(as_h2(__builtin_amdgcn_perm(b, a, 0x0c040c00u)), k, z));
    out[1] = as_u32(__builtin_elementwise_fma(as_h2(__builtin_amdgcn_perm(b, a, 0x0c050c01u)), k, z));
    out[2] = as_u32(__builtin_elementwise_fma(as_h2(__builtin_amdgcn_perm(b, a, 0x0c060c02u)), k, z));
    out[3] = as_u32(__builtin_elementwise_fma(as_h2(__builtin_amdgcn_perm(b, a, 0x0c070c03u)), k, z));
  } else {
    const uint32_t x = __builtin_amdgcn_perm(b, a, 0x05010400u);   // a0 b0 a1 b1
    const uint32_t y = __builtin_amdgcn_perm(b, a, 0x07030602u);   // a2 b2 a3 b3
    out[0] = key_pair<FMT>(x, false);
    out[1] = key_pair<FMT>(x, true);
    out[2] = key_pair<FMT>(y, false);
    out[3] = key_pair<FMT>(y, true);
  }
}

__device__ __forceinline__ h8 as_h8(u4 x) { return __builtin_bit_cast(h8, x); }
__device__ __forceinline__ b8 as_b8(u4 x) { return __builtin_bit_cast(b8, x); }

// A row's maximum before it has seen a token: below all scores.
constexpr float kNoScore = -3.0e38f;
// Scores (log2) from here on are rounded before their row's maximum is subtracted.
constexpr float kLargeScore = 0x1p12f;

__device__ __forceinline__ float exp2_f(float x) { return __builtin_amdgcn_exp2f(x); }

// tanh to about two units in the last place.  Below 0.8 the fraction
// x (945 + 105 x^2 + x^4) / (945 + 420 x^2 + 15 x^4), the fifth convergent of
// its continued fraction (error x^11 / 9.8e6); above, (1 - t) / (1 + t) with
// t = exp(-2 |x|), where nothing cancels.
__device__ __forceinline__ float tanh_f(float x) {
  const float y = x * x;
  const float num = x * __builtin_fmaf(y, __builtin_fmaf(y, 1.0f, 105.0f), 945.0f);
  const float den = __builtin_fmaf(y, __builtin_fmaf(y, 15.0f, 420.0f), 945.0f);
  const float t = exp2_f(-2.8853900817779268f * __builtin_fabsf(x));
  const bool small = __builtin_fabsf(x) < 0.8f;
  const float a = small ? num : __builtin_copysignf(1.0f - t, x);
  return a * __builtin_amdgcn_rcpf(small ? den : 1.0f + t);
}

// ------------------------------------------------------------------ attention
// One thread's share of an output row: N channels from ch.
template <int N>
__device__ __forceinline__ void store_out(const BlockAttendLaunch& a, int b, int head, int token,
                                          int ch, const float* x) {
  const int64_t at = b * a.out.sb + head * a.out.sh + token * a.out.st + ch;
  if (a.out_dtype == RQ_F32) {
    RQ_GLOBAL float* o = gptr((float*)a.out.p) + at;
#pragma unroll
    for (int i = 0; i < N / 4; ++i)
      *(RQ_GLOBAL f4_any*)(o + 4 * i) = (f4){x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]};
    return;
  }
  RQ_GLOBAL uint16_t* o = gptr((uint16_t*)a.out.p) + at;
#pragma unroll
  for (int i = 0; i < N / 4; ++i) {
    u2 w;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const float y = x[4 * i + 2 * j], z = x[4 * i + 2 * j + 1];
      w[j] = a.out_dtype == RQ_BF16 ? bf16_rne(y) | ((uint32_t)bf16_rne(z) << 16)
                                    : narrow_t<false>(y) | ((uint32_t)narrow_t<false>(z) << 16);
    }
    *(RQ_GLOBAL u2_any*)(o + 4 * i) = w;
  }
}

// The position of a tree's nodes of depth 0, and a node's depth.
__device__ __forceinline__ int tree_base(const BlockTreeLaunch& a, int unit, int past) {
  return past > 0 ? gptr(a.c.positions)[(size_t)unit * a.c.cap + past - 1] + 1 : 0;
}
__device__ __forceinline__ int node_depth(const BlockTreeLaunch& a, int b, int node) {
  const int d = gptr(a.depth)[(size_t)b * a.n + node];
  return d < 0 ? 0 : (d < a.n ? d : a.n - 1);
}

// Which nodes 32 d..32 d + 31 node i sees, of nnew.
__device__ __forceinline__ uint32_t node_mask(const BlockTreeLaunch& a, int b, int i, int d, int nnew) {
  const int left = nnew - 32 * d;
  if (left <= 0) return 0u;
  const uint32_t w = gptr(a.mask)[((size_t)b * a.n + i) * a.words + d];
  return left < 32 ? w & ((1u << left) - 1u) : w;
}

// Row i of a tree's own keys or values in head h.
__device__ __forceinline__ const RQ_GLOBAL uint16_t* node_row(const BlockRows& x, int b, int h, int i) {
  return gptr(static_cast<const uint16_t*>(x.p)) + b * x.sb + h * x.sh + i * x.st;
}

// A tile of 16 query rows as one wave holds it: lane (r = lane & 15,
// g = lane >> 4) has, of row r, the channels 64 c + 16 g + 8 f + 0..7 in
// operand 2 c + f.
template <int D>
struct QueryTile {
  h8 f[D / 32];
  float qs;       // factor of the scores (log2 units, or scale / cap)
  float slope;    // of this row's head, log2 units (0: none)
  int token;      // of the call's new tokens: this row's
  int head;       // query head inside its group
  int pos;        // its position (where positions matter)
  bool valid;
};

// fp16 queries are used as they are; bf16 rows are scaled by a power of two to
// magnitudes below 1, which fp16 holds exactly down to 2^-14 of the row's
// largest element and to 2^-25 of it below.
template <int D, bool BF16, class Launch>
__device__ __forceinline__ void load_queries(const Launch& a, int b, int h, int row,
                                             int past, int nnew, QueryTile<D>* t) {
  const int g = (threadIdx.x & 63) >> 4;
  t->token = over(row, a.by_G);
  t->head = row - t->token * a.G;
  t->valid = t->token < nnew;
  if (!t->valid) t->token = nnew > 0 ? nnew - 1 : 0;
  const RQ_GLOBAL uint16_t* q = gptr(static_cast<const uint16_t*>(a.q.p)) + b * a.q.sb +
                                (int64_t)(h * a.G + t->head) * a.q.sh + t->token * a.q.st;
  u4 raw[D / 32];
#pragma unroll
  for (int k = 0; k < D / 32; ++k)
    raw[k] = t->valid ? *(const RQ_GLOBAL u4_any*)(q + 64 * (k >> 1) + 16 * g + 8 * (k & 1))
                      : (u4){0u, 0u, 0u, 0u};
  t->qs = a.qscale;
  if constexpr (!BF16) {
#pragma unroll
    for (int k = 0; k < D / 32; ++k) t->f[k] = as_h8(raw[k]);
  } else {
    float most = 0.0f;
#pragma unroll
    for (int k = 0; k < D / 32; ++k)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        most = __builtin_fmaxf(most, __builtin_fabsf(__uint_as_float(raw[k][i] << 16)));
        most = __builtin_fmaxf(most, __builtin_fabsf(__uint_as_float(raw[k][i] & 0xffff0000u)));
      }
    most = half_all<Max>(pair_all<Max>(most));
    const int e = most > 0.0f ? __builtin_amdgcn_frexp_expf(most) : 0;
#pragma unroll
    for (int k = 0; k < D / 32; ++k) {
      h8 f;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        f[2 * i] = (_Float16)__builtin_amdgcn_ldexpf(__uint_as_float(raw[k][i] << 16), -e);
        f[2 * i + 1] = (_Float16)__builtin_amdgcn_ldexpf(__uint_as_float(raw[k][i] & 0xffff0000u), -e);
      }
      t->f[k] = f;
    }
    t->qs = __builtin_amdgcn_ldexpf(a.qscale, e);
  }
  t->slope = a.slopes ? gptr(a.slopes)[h * a.G + t->head] * 1.4426950408889634f : 0.0f;
  t->pos = 0;
  if (a.slopes || a.window) {
    if constexpr (kIsTree<Launch>) {
      t->pos = tree_base(a, b * a.c.H + h, past) + node_depth(a, b, t->token);
    } else {
      const int slot = past + t->token;
      t->pos = gptr(a.c.positions)[(size_t)(b * a.c.H + h) * a.c.cap + (slot < a.c.cap ? slot : 0)];
    }
  }
}

// The key codes of one block: lane (r, g) has, of tokens 16 m + r, the
// channels 64 c + 16 g + 0..15.
template <int D>
struct KeyBlock {
  u4 w[2][D / 64];
  float scale;
};

template <int D>
__device__ __forceinline__ void load_keys(const RQ_GLOBAL uint8_t* k, const RQ_GLOBAL float* scale,
                                          int blk, KeyBlock<D>* t) {
  const int lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
#pragma unroll
  for (int m = 0; m < 2; ++m)
#pragma unroll
    for (int c = 0; c < D / 64; ++c)
      t->w[m][c] = *(const RQ_GLOBAL u4*)(k + (uint32_t)(blk * kBlockTokens + 16 * m + r) * D + 64 * c + 16 * g);
  t->scale = scale[blk];
}

// Products of a block's keys with QT query tiles: lane (r, g) gets, for query
// row r of tile n, tokens 16 m + 4 g + i in s[n][m][i].
template <int FMT, int D, int QT>
__device__ __forceinline__ void key_products(const KeyBlock<D>& t, const QueryTile<D> q[QT],
                                             f4 s[QT][2]) {
#pragma unroll
  for (int m = 0; m < 2; ++m) {
#pragma unroll
    for (int n = 0; n < QT; ++n) s[n][m] = (f4){0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int k = 0; k < D / 32; ++k) {
      const uint32_t x = t.w[m][k >> 1][2 * (k & 1)], y = t.w[m][k >> 1][2 * (k & 1) + 1];
      const u4 op = {key_pair<FMT>(x, false), key_pair<FMT>(x, true), key_pair<FMT>(y, false),
                     key_pair<FMT>(y, true)};
#pragma unroll
      for (int n = 0; n < QT; ++n)
        s[n][m] = __builtin_amdgcn_mfma_f32_16x16x32_f16(as_h8(op), q[n].f[k], s[n][m], 0, 0, 0);
    }
  }
}

// The same for the 16-bit keys of the tail or of a tree's nodes (key(row, channel)
// loads eight of a row 0..31), on the matrix cores' own 16-bit type (the query rows
// are read again: as bf16 they need no scaling).  Rows behind the last hold
// anything; their products are masked.
template <int D, bool BF16, class Key>
__device__ __forceinline__ void tail_products(const BlockAttendLaunch& a, int b, int h, Key key,
                                              const QueryTile<D>& q, f4 s[2]) {
  const int lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
  const RQ_GLOBAL uint16_t* qp = gptr(static_cast<const uint16_t*>(a.q.p)) + b * a.q.sb +
                                 (int64_t)(h * a.G + q.head) * a.q.sh + q.token * a.q.st;
#pragma unroll
  for (int m = 0; m < 2; ++m) s[m] = (f4){0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
  for (int k = 0; k < D / 32; ++k) {
    const int ch = 64 * (k >> 1) + 16 * g + 8 * (k & 1);
    u4 qr = {0u, 0u, 0u, 0u};
    if constexpr (BF16)
      if (q.valid) qr = *(const RQ_GLOBAL u4_any*)(qp + ch);
#pragma unroll
    for (int m = 0; m < 2; ++m) {
      const u4 kr = key(16 * m + r, ch);
      if constexpr (BF16)
        s[m] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_b8(kr), as_b8(qr), s[m], 0, 0, 0);
      else
        s[m] = __builtin_amdgcn_mfma_f32_16x16x32_f16(as_h8(kr), q.f[k], s[m], 0, 0, 0);
    }
  }
}

// Scores in log2 units from products: scale, cap, distance bias, mask.
// slot0: the slot of the block's first token.  end: the last slot that the row
// sees.  masked: some token of the block may be hidden from some row.
template <int D>
__device__ __forceinline__ void block_scores(const BlockAttendLaunch& a, const QueryTile<D>& q,
                                             const RQ_GLOBAL int32_t* positions, float factor,
                                             int slot0, int end, bool masked, f4 s[2]) {
  const int g = (threadIdx.x & 63) >> 4;
#pragma unroll
  for (int m = 0; m < 2; ++m) s[m] *= factor;
  if (a.cap != 0.0f) {
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
      for (int i = 0; i < 4; ++i) s[m][i] = a.cap * tanh_f(s[m][i]);
  }
  if (a.slopes || (masked && a.window)) {
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int away = q.pos - positions[slot0 + 16 * m + 4 * g + i];
        s[m][i] = __builtin_fmaf(-q.slope, (float)away, s[m][i]);
        if (a.window && away >= a.window) s[m][i] = -__builtin_inff();
      }
  }
  if (masked) {
    const int last = end - slot0;
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (16 * m + 4 * g + i > last) s[m][i] = -__builtin_inff();
  }
}

// The same of a tree's nodes 32 d..32 d + 31; base: tree_base.
template <int D>
__device__ __forceinline__ void node_scores(const BlockTreeLaunch& a, const QueryTile<D>& q, int b,
                                            int d, int nnew, int base, f4 s[2]) {
  const int g = (threadIdx.x & 63) >> 4;
  const uint32_t seen = q.valid ? node_mask(a, b, q.token, d, nnew) : 0u;
#pragma unroll
  for (int m = 0; m < 2; ++m) s[m] *= a.qscale;
  if (a.cap != 0.0f) {
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
      for (int i = 0; i < 4; ++i) s[m][i] = a.cap * tanh_f(s[m][i]);
  }
  if (a.slopes || a.window) {
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int node = 32 * d + 16 * m + 4 * g + i;
        const int away = q.pos - base - node_depth(a, b, node < nnew ? node : nnew - 1);
        s[m][i] = __builtin_fmaf(-q.slope, (float)away, s[m][i]);
        if (a.window && away >= a.window) s[m][i] = -__builtin_inff();
      }
  }
#pragma unroll
  for (int m = 0; m < 2; ++m)
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (!((seen >> (16 * m + 4 * g + i)) & 1u)) s[m][i] = -__builtin_inff();
}

}  // namespace rq
