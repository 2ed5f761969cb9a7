// Attention over the block-scaled 8-bit cache for many query rows a unit
// (prompts and their chunks): matrix products of tiles.
//
// A workgroup of four waves owns 128 rows of a unit (token-major, the heads of
// a group together), 32 a wave, and walks its tokens in tiles of 64; two are on
// a CU.  Codes are converted to fp16 once a workgroup on their way into LDS (two
// buffers, one barrier a tile), keys as [token][channel], values as
// [channel][token].  On v_mfma_f32_32x32x16_f16 S^T = K Q^T leaves a lane with
// 16 tokens of one row, the operand that O^T = V^T P^T wants of it (the values'
// tokens are stored in that order), so probabilities never move between lanes.
//
// A block's value scale goes into the exponent: P' = 2^(x - m + log2(by)),
// by = value scale * unit, and the row's sum takes the block's sum of P' / by.
// P' is an fp16 pair hi + lo (22 bits), whatever the output's type: as fp16 alone
// a call of many rows would answer otherwise than one of few, by 2^-12 of the
// result before its rounding, and take a fifth less time.
//
// Two prompts of 4096 tokens (8 kv-heads of 4 heads, 128 channels, e4m3): 412 us,
// 667 TFLOP/s, bf16 as fp16; capped 480.  Neither unit bounds it alone: a wave's
// tile is, capped, some 500 vector instructions (96 of them exponentials and
// reciprocals) and 1536 cycles of the matrix unit, with two waves a SIMD; the
// units are 60 and 37 % busy.  Workgroups of 256 rows (half the conversions) took
// 2 % longer; the conversion between the products of the tile before does not fit
// the registers.
#include "rq_block.h"

namespace rq {

namespace {

typedef float f16v __attribute__((ext_vector_type(16)));

constexpr int kWaves = 4, kRows = 32 * kWaves, kTile = 64, kThreads = 64 * kWaves;
constexpr int kPasses = 512 / kThreads;     // a tile's conversion is 512 shares

// 16-byte pieces of an LDS row are permuted by a key of the row, so that lanes
// that read the same piece of consecutive rows, or write pieces of every
// fourth, meet different banks.
template <int D>
__device__ __forceinline__ int key_at(int token, int piece) {
  return token * D * 2 + ((piece ^ (token & (D / 8 - 1))) << 4);
}
__device__ __forceinline__ int value_at(int ch, int piece) {
  return ch * kTile * 2 + ((piece ^ ((ch >> 2) & 7) ^ ((ch & 2) << 1)) << 4);
}

// A share of a tile: D / 8 key codes of a token, and 4 channels of 4 tokens of
// the values (with D = 64 the first half of the shares).
struct TileLoad {
  u4 k[kPasses];
  uint32_t v[kPasses][4];
};

template <int D>
__device__ __forceinline__ void load_tile(const RQ_GLOBAL uint8_t* kc, const RQ_GLOBAL uint8_t* vc,
                                          int slot0, int slots, TileLoad* t) {
#pragma unroll
  for (int p = 0; p < kPasses; ++p) {
    const int id = threadIdx.x + p * kThreads;
    const int tok = slot0 + id / 8;
    if (tok < slots) {
      if constexpr (D == 128) {
        t->k[p] = *(const RQ_GLOBAL u4*)(kc + (uint32_t)tok * D + 16 * (id % 8));
      } else {
        const u2 w = *(const RQ_GLOBAL u2*)(kc + (uint32_t)tok * D + 8 * (id % 8));
        t->k[p].x = w.x;
        t->k[p].y = w.y;
      }
    }
    const int quad = id / (D / 4), ch = 4 * (id % (D / 4)), first = slot0 + 4 * quad;
    if (quad < kTile / 4 && first < slots)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        t->v[p][i] = *(const RQ_GLOBAL uint32_t*)(vc + (uint32_t)(first + i) * D + ch);
  }
}

// WHOLE: no slot of the tile lies behind the last (without the comparisons 512
// tokens over 8192 take 2 % less, capped prompts 1 % more).
template <int FMT, int D, bool WHOLE>
__device__ __forceinline__ void store_tile(const TileLoad& t, int slot0, int slots, uint8_t* sk,
                                           uint8_t* sv) {
#pragma unroll
  for (int p = 0; p < kPasses; ++p) {
    const int id = threadIdx.x + p * kThreads, tok = id / 8;
    if (WHOLE || slot0 + tok < slots) {
#pragma unroll
      for (int i = 0; i < D / 64; ++i) {
        const u4 w = {key_pair<FMT>(t.k[p][2 * i], false), key_pair<FMT>(t.k[p][2 * i], true),
                      key_pair<FMT>(t.k[p][2 * i + 1], false), key_pair<FMT>(t.k[p][2 * i + 1], true)};
        *(u4*)(sk + key_at<D>(tok, D / 64 * (id % 8) + i)) = w;
      }
    }
    const int quad = id / (D / 4), ch = 4 * (id % (D / 4));
    if (quad < kTile / 4) {
      uint32_t a[4] = {0u, 0u, 0u, 0u}, b[4] = {0u, 0u, 0u, 0u};
      if (WHOLE || slot0 + 4 * quad < slots) {
        value_pairs<FMT>(t.v[p][0], t.v[p][1], a);
        value_pairs<FMT>(t.v[p][2], t.v[p][3], b);
      }
#pragma unroll
      for (int e = 0; e < 4; ++e)
        *(u2*)(sv + value_at(ch + e, 2 * (quad / 4) + (quad & 1)) + 8 * ((quad >> 1) & 1)) = (u2){a[e], b[e]};
    }
  }
}

// The tail's rows as the block of 32 tokens at `at` of the tile, divided by a
// power of two that brings the largest of the side below 1 (returned as the
// block's scales; fp16 holds the others to 2^-25 of it).  Rows from n_tail on
// count as zero.  The whole workgroup calls it.
template <int FMT, int D, bool BF16>
__device__ __forceinline__ void store_tail(const RQ_GLOBAL uint16_t* kt, int n_tail, int at, uint8_t* sk,
                                           uint8_t* sv, float* red, float* ks, float* vs) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const RQ_GLOBAL uint16_t* vt = kt + kBlockTokens * D;
  // shares of 8 keys of one token, and 2 channels of 4 tokens of the values
  constexpr int kPieces = D / 8;
  u4 k[kPasses];
  uint32_t v[kPasses][4];
  float km = 0.0f, vm = 0.0f;
#pragma unroll
  for (int p = 0; p < kPasses; ++p) {
    const int id = threadIdx.x + p * kThreads, tok = id / kPieces, quad = id / (D / 2);
    k[p] = (u4){0u, 0u, 0u, 0u};
    if (tok < n_tail) k[p] = *(const RQ_GLOBAL u4*)(kt + tok * D + 8 * (id % kPieces));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[p][i] = 0u;
      if (quad < 8 && 4 * quad + i < n_tail)
        v[p][i] = *(const RQ_GLOBAL uint32_t*)(vt + (4 * quad + i) * D + 2 * (id % (D / 2)));
      km = __builtin_fmaxf(km, __builtin_fmaxf(__builtin_fabsf(widen_t<BF16>(k[p][i] & 0xffffu)),
                                               __builtin_fabsf(widen_t<BF16>(k[p][i] >> 16))));
      vm = __builtin_fmaxf(vm, __builtin_fmaxf(__builtin_fabsf(widen_t<BF16>(v[p][i] & 0xffffu)),
                                               __builtin_fabsf(widen_t<BF16>(v[p][i] >> 16))));
    }
  }
  km = wave_all<Max>(km);
  vm = wave_all<Max>(vm);
  if (lane == 0) {
    red[wave] = km;
    red[8 + wave] = vm;
  }
  __syncthreads();
  for (int i = 0; i < kWaves; ++i) {
    km = __builtin_fmaxf(km, red[i]);
    vm = __builtin_fmaxf(vm, red[8 + i]);
  }
  const int ke = km > 0.0f ? __builtin_amdgcn_frexp_expf(km) : 0;
  const int ve = vm > 0.0f ? __builtin_amdgcn_frexp_expf(vm) : 0;
  auto pair = [](uint32_t x, int e) {
    const h2 y = {(_Float16)__builtin_amdgcn_ldexpf(widen_t<BF16>(x & 0xffffu), -e),
                  (_Float16)__builtin_amdgcn_ldexpf(widen_t<BF16>(x >> 16), -e)};
    return as_u32(y);
  };
#pragma unroll
  for (int p = 0; p < kPasses; ++p)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      k[p][i] = pair(k[p][i], ke);
      v[p][i] = pair(v[p][i], ve);
    }
  *ks = __builtin_amdgcn_ldexpf(1.0f, ke);
  *vs = vm > 0.0f ? __builtin_amdgcn_ldexpf(kValueUnit<FMT>, ve) : 0.0f;
#pragma unroll
  for (int p = 0; p < kPasses; ++p) {
    const int id = threadIdx.x + p * kThreads, tok = id / kPieces, quad = id / (D / 2);
    const int ch = 2 * (id % (D / 2));
    if (tok < kBlockTokens) *(u4*)(sk + key_at<D>(at + tok, id % kPieces)) = k[p];
    if (quad < 8) {
      const int q = at / 4 + quad;
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const uint32_t sel = e ? 0x07060302u : 0x05040100u;
        *(u2*)(sv + value_at(ch + e, 2 * (q / 4) + (q & 1)) + 8 * ((q >> 1) & 1)) =
            (u2){__builtin_amdgcn_perm(v[p][1], v[p][0], sel), __builtin_amdgcn_perm(v[p][3], v[p][2], sel)};
      }
    }
  }
}

template <int FMT, int D, bool BF16>
__global__ void __launch_bounds__(kThreads, 2) block_prompt_kernel(BlockAttendLaunch a) {
  __shared__ __align__(16) uint8_t sh_k[2][kTile * D * 2];
  __shared__ __align__(16) uint8_t sh_v[2][kTile * D * 2];
  __shared__ int32_t sh_pos[2][kTile];
  __shared__ float red[16];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 31, hl = lane >> 5;
  // Two workgroups share a SIMD, a wave each.  The wave in the odd slot (the low
  // bit of hardware register 4) goes first, so that one's products meet the
  // other's exponentials: 509 tokens over up to 8192, with weights, 411 -> 381 us,
  // 4096 uncapped ones 436 -> 431, fp16 440 -> 432; capped 488 -> 490, 64 channels
  // alike.
  if (__builtin_amdgcn_s_getreg(4 | (3 << 11)) & 1) __builtin_amdgcn_s_setprio(1);
  // workgroups go round the XCDs: where the units are a multiple of eight, a
  // unit's tiles share an L2; the tiles that see most tokens go first
  const int units = a.c.B * a.c.H, tiles = (a.n * a.G + kRows - 1) / kRows, each = tiles * a.splits;
  int unit, w;
  if (units % 8 == 0) {
    const uint32_t eight = blockIdx.x / 8, u = eight / (uint32_t)each;
    unit = (int)u * 8 + blockIdx.x % 8;
    w = eight - u * each;
  } else {
    unit = blockIdx.x / (uint32_t)each;
    w = blockIdx.x - unit * each;
  }
  const int t = over(w, a.by_splits), rt = tiles - 1 - t, split = w - t * a.splits;
  const int b = over(unit, a.c.by_H), h = unit - b * a.c.H;
  int past, nnew;
  block_lengths(a.past, a.new_len, b, a.n, a.max_tokens, &past, &nnew);
  const int first = over(rt * kRows, a.by_G);
  if (first >= nnew) return;
  int last = over(rt * kRows + kRows - 1, a.by_G);
  last = last < nnew ? last : nnew - 1;
  const int total = past + nnew, full = total / kBlockTokens;
  int lo, hi;
  seen_blocks(past, first, last, a.window, &lo, &hi);
  {
    // splits begin at whole tiles
    const int nt = (hi - lo + 1) / 2, t0 = part_from(nt, split, a.splits, a.by_splits), t1 = part_from(nt, split + 1, a.splits, a.by_splits);
    hi = lo + 2 * t1 < hi ? lo + 2 * t1 : hi;
    lo += 2 * t0;
  }

  const RQ_GLOBAL uint8_t* kc = gptr(a.c.codes) + (size_t)unit * 2 * a.c.cap * D;
  const RQ_GLOBAL uint8_t* vc = kc + (size_t)a.c.cap * D;
  const int coded = (hi < full ? hi : full) * kBlockTokens;     // slots of the split's coded blocks
  TileLoad next;
  if (lo < hi) load_tile<D>(kc, vc, lo * kBlockTokens, coded, &next);

  // this lane's row, as BlockAttendLaunch has it: 16 k + 8 hl + 0..7 in f[k]
  const int row = rt * kRows + wave * 32 + col;
  int token = over(row, a.by_G);
  const int head = row - token * a.G;
  const bool valid = token < nnew;
  if (!valid) token = nnew - 1;
  const int wave_first = over(rt * kRows + wave * 32, a.by_G);      // tokens of the wave's rows
  int wave_last = over(rt * kRows + wave * 32 + 31, a.by_G);
  wave_last = wave_last < nnew ? wave_last : nnew - 1;
  const bool idle = wave_first >= nnew;
  h8 q[D / 16];
  float qs = __builtin_fabsf(a.qscale), slope = 0.0f;
  int qpos = 0;
  {
    const RQ_GLOBAL uint16_t* p = gptr(static_cast<const uint16_t*>(a.q.p)) + b * a.q.sb +
                                  (int64_t)(h * a.G + head) * a.q.sh + token * a.q.st;
    u4 raw[D / 16];
#pragma unroll
    for (int k = 0; k < D / 16; ++k)
      raw[k] = valid ? *(const RQ_GLOBAL u4_any*)(p + 16 * k + 8 * hl) : (u4){0u, 0u, 0u, 0u};
    // (a negative scale turns the queries, so that scores grow with products)
    const uint32_t turn = a.qscale < 0.0f ? 0x80008000u : 0u;
#pragma unroll
    for (int k = 0; k < D / 16; ++k) raw[k] ^= turn;
    if constexpr (BF16) {
      float most = 0.0f;
#pragma unroll
      for (int k = 0; k < D / 16; ++k)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          most = __builtin_fmaxf(most, __builtin_fabsf(widen_t<true>(raw[k][i] & 0xffffu)));
          most = __builtin_fmaxf(most, __builtin_fabsf(widen_t<true>(raw[k][i] >> 16)));
        }
      most = half_all<Max>(most);
      const int e = most > 0.0f ? __builtin_amdgcn_frexp_expf(most) : 0;
#pragma unroll
      for (int k = 0; k < D / 16; ++k)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          q[k][2 * i] = (_Float16)__builtin_amdgcn_ldexpf(widen_t<true>(raw[k][i] & 0xffffu), -e);
          q[k][2 * i + 1] = (_Float16)__builtin_amdgcn_ldexpf(widen_t<true>(raw[k][i] >> 16), -e);
        }
      qs = __builtin_amdgcn_ldexpf(qs, e);
    } else {
#pragma unroll
      for (int k = 0; k < D / 16; ++k) q[k] = as_h8(raw[k]);
    }
    if (a.queries && split == 0 && valid) {       // for the weights' launch
      const size_t at = (size_t)unit * a.row_tiles * 16 + row;
#pragma unroll
      for (int k = 0; k < D / 16; ++k)
        *(RQ_GLOBAL h8*)(gptr(a.queries) + at * D + 16 * k + 8 * hl) = q[k];
      if (hl == 0) gptr(a.factors)[at] = qs;
    }
    if (a.slopes) slope = gptr(a.slopes)[h * a.G + head] * 1.4426950408889634f;
    if (a.slopes || a.window)
      qpos = gptr(a.c.positions)[(size_t)unit * a.c.cap + past + token];
  }

  // (scales by scalar loads: a vector load's wait would be one for the next
  // tile's codes in flight)
  const RQ_CONSTANT float* kscale = cptr(a.c.scales) + (size_t)unit * 2 * (a.c.cap / kBlockTokens);
  const RQ_CONSTANT float* vscale = kscale + a.c.cap / kBlockTokens;
  const RQ_GLOBAL int32_t* pos = gptr(a.c.positions) + (size_t)unit * a.c.cap;
  const RQ_GLOBAL uint16_t* tail = gptr(a.c.tail) + (size_t)unit * 2 * kBlockTokens * D;

  f16v o[D / 32];
#pragma unroll
  for (int c = 0; c < D / 32; ++c)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[c][i] = 0.0f;
  float m = kNoScore, l = 0.0f, unit2 = 0.0f;
  const bool far = a.slopes || a.window;

  float tks[2], tvs[2];               // scales of a tile's blocks
  auto put = [&](int blk, int buf) {
    if ((blk + 2) * kBlockTokens <= coded)
      store_tile<FMT, D, true>(next, blk * kBlockTokens, coded, sh_k[buf], sh_v[buf]);
    else
      store_tile<FMT, D, false>(next, blk * kBlockTokens, coded, sh_k[buf], sh_v[buf]);
    if (far && threadIdx.x < kTile) {
      const int slot = blk * kBlockTokens + threadIdx.x;
      sh_pos[buf][threadIdx.x] = slot < total ? pos[slot] : 0;
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      tks[i] = blk + i < full ? kscale[blk + i] : 0.0f;
      tvs[i] = blk + i < full ? vscale[blk + i] : 0.0f;
    }
    if (full < hi && (blk == full || blk + 1 == full)) {
      // (the zeros that store_tile left for the tail's values come first)
      __syncthreads();
      float k, v;
      store_tail<FMT, D, BF16>(tail, total - full * kBlockTokens, (full - blk) * kBlockTokens, sh_k[buf],
                               sh_v[buf], red, &k, &v);
      if (blk == full) {
        tks[0] = k;
        tvs[0] = v;
      } else {
        tks[1] = k;
        tvs[1] = v;
      }
    }
  };

  auto work = [&](int blk, int buf) {
    const int slot0 = blk * kBlockTokens;
    if (idle || slot0 > past + wave_last) return;
    f16v s[2];
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int i = 0; i < 16; ++i) s[t][i] = 0.0f;
    // (the two blocks' sums in turn: neither waits for its last product)
#pragma unroll
    for (int k = 0; k < D / 16; ++k)
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const h8 f = *(const h8*)(sh_k[buf] + key_at<D>(32 * t + col, 2 * k + hl));
        s[t] = __builtin_amdgcn_mfma_f32_32x32x16_f16(f, q[k], s[t], 0, 0, 0);
      }
    const bool masked = a.window || slot0 + kTile - 1 > past + wave_first;
    // scores are s f + off; a mask needs them formed (f may be 0)
    float f[2] = {tks[0] * qs, tks[1] * qs}, off = 0.0f;
    if (a.cap != 0.0f && !a.fine) {
      // cap tanh(x) = cap - 2 cap / (1 + e^(2x)): off by 2^-22 cap
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const float e2 = f[t] * 2.8853900817779268f;
#pragma unroll
        for (int i = 0; i < 16; ++i) s[t][i] = __builtin_amdgcn_rcpf(-1.0f - exp2_f(s[t][i] * e2));
        f[t] = 2.0f * a.cap;
      }
      off = a.cap;
    }
    if (far || masked || a.fine) {
#pragma unroll
      for (int t = 0; t < 2; ++t) {
#pragma unroll
        for (int i = 0; i < 16; ++i) s[t][i] = __builtin_fmaf(s[t][i], f[t], off);
        if (a.fine) {
#pragma unroll
          for (int i = 0; i < 16; ++i) s[t][i] = a.cap * tanh_f(s[t][i]);
        }
        f[t] = 1.0f;
        if (far) {
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const int away = qpos - sh_pos[buf][32 * t + 8 * (i >> 2) + 4 * hl + (i & 3)];
            s[t][i] = __builtin_fmaf(-slope, (float)away, s[t][i]);
            if (a.window && away >= a.window) s[t][i] = -__builtin_inff();
          }
        }
        if (masked) {
          const int end = past + token - slot0 - 32 * t - 4 * hl;
#pragma unroll
          for (int i = 0; i < 16; ++i)
            if (8 * (i >> 2) + (i & 3) > end) s[t][i] = -__builtin_inff();
        }
      }
      off = 0.0f;
    }
    // the running maximum (moved when a score exceeds it by 8) and unit
    float top = kNoScore;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      float x = s[t][0];
#pragma unroll
      for (int i = 1; i < 16; ++i) x = __builtin_fmaxf(x, s[t][i]);
      top = __builtin_fmaxf(top, __builtin_fmaf(x, f[t], off));
    }
    const float sv = __builtin_fmaxf(tvs[0], tvs[1]);
    // (the same in every lane; scales of zero have no unit to follow)
    const bool grow = sv > 0.0f && (unit2 == 0.0f || sv * unit2 > 128.0f);
    if (grow || __any(top > m + 8.0f)) {
      top = half_all<Max>(top);
      const float mn = __builtin_fmaxf(m, top);
      float by = exp2_f(m - mn);
      m = mn;
      l *= by;
      if (grow) {
        int e = __builtin_amdgcn_frexp_expf(sv);
        e = e < -100 ? -100 : e;
        const float u = __builtin_amdgcn_ldexpf(128.0f, -e);
        by *= unit2 == 0.0f ? 1.0f : u * __builtin_amdgcn_rcpf(unit2);     // (powers of two)
        unit2 = u;
      }
#pragma unroll
      for (int c = 0; c < D / 32; ++c) o[c] *= by;
    }
    // (Scores this large differ from their maximum by more than an exponent
    // holds through its rounding alone, and swallow log2(by): the difference is
    // taken of rounded ones, and first.)
    float reference = m - off;
    if (__any(__builtin_fabsf(m) > kLargeScore && m > kNoScore)) {
#pragma unroll
      for (int t = 0; t < 2; ++t) {
#pragma unroll
        for (int i = 0; i < 16; ++i) s[t][i] = __builtin_fmaf(s[t][i], f[t], off) - m;
        f[t] = 1.0f;
      }
      reference = 0.0f;
    }
    // Probabilities of the second block are formed between the first one's
    // products.
    float by[2], c[2], sum[2] = {0.0f, 0.0f};
    uint32_t hi2[2][8], lo2[2][8];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      // (codes under a scale of zero are zero: any factor serves)
      by[t] = tvs[t] > 0.0f ? __builtin_fmaxf(tvs[t] * unit2, 0x1p-80f) : 1.0f;
      c[t] = reference - __builtin_amdgcn_logf(by[t]);
    }
    auto form = [&](int t, int i) {
      const float x = exp2_f(__builtin_fmaf(s[t][2 * i], f[t], -c[t]));
      const float y = exp2_f(__builtin_fmaf(s[t][2 * i + 1], f[t], -c[t]));
      const h2 p = __builtin_bit_cast(h2, __builtin_amdgcn_cvt_pkrtz(x, y));
      hi2[t][i] = as_u32(p);
      float xl, yl;      // what the halves leave of x and y, exactly
      asm("v_fma_mix_f32 %0, %1, -1.0, %2 op_sel_hi:[1,0,0]" : "=v"(xl) : "v"(p), "v"(x));
      asm("v_fma_mix_f32 %0, %1, -1.0, %2 op_sel:[1,0,0] op_sel_hi:[1,0,0]" : "=v"(yl) : "v"(p), "v"(y));
      lo2[t][i] = as_u32((h2){(_Float16)xl, (_Float16)yl});
      // (of the fp32 numbers: where by is small, fp16 loses P' but the sum
      // must not)
      sum[t] += x;
      sum[t] += y;
    };
    auto value = [&](int t, int j) {
      return *(const h8*)(sh_v[buf] + value_at(32 * (j % (D / 32)) + col, 2 * (2 * t + j / (D / 32)) + hl));
    };
    auto add = [&](int t, int j, h8 vf) {
      const int g = j / (D / 32), c2 = j % (D / 32);
      const h8 ph = as_h8((u4){hi2[t][4 * g], hi2[t][4 * g + 1], hi2[t][4 * g + 2], hi2[t][4 * g + 3]});
      o[c2] = __builtin_amdgcn_mfma_f32_32x32x16_f16(vf, ph, o[c2], 0, 0, 0);
      const h8 pl = as_h8((u4){lo2[t][4 * g], lo2[t][4 * g + 1], lo2[t][4 * g + 2], lo2[t][4 * g + 3]});
      o[c2] = __builtin_amdgcn_mfma_f32_32x32x16_f16(vf, pl, o[c2], 0, 0, 0);
    };
    constexpr int kSteps = D / 16;
#pragma unroll
    for (int i = 0; i < 8; ++i) form(0, i);
    h8 v0 = value(0, 0), v1 = value(0, 1);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int j = 0; j < 2 * kSteps; ++j) {
      const h8 v2 = j + 2 < 2 * kSteps ? value((j + 2) / kSteps, (j + 2) % kSteps) : v0;
      add(j / kSteps, j % kSteps, v0);
      if (j < kSteps)
#pragma unroll
        for (int i = 0; i < 8 / kSteps; ++i) form(1, 8 / kSteps * j + i);
      v0 = v1;
      v1 = v2;
      __builtin_amdgcn_sched_barrier(0);
    }
#pragma unroll
    for (int t = 0; t < 2; ++t) l = __builtin_fmaf(sum[t], __builtin_amdgcn_rcpf(by[t]), l);
  };

  // a wave may be a tile behind the others, never more: one barrier a tile
  for (int blk = lo, buf = 0; blk < hi; blk += 2, buf ^= 1) {
    put(blk, buf);
    __syncthreads();
    if (blk + 2 < hi) load_tile<D>(kc, vc, (blk + 2) * kBlockTokens, coded, &next);
    work(blk, buf);
  }

  l = half_all<Sum>(l);
  const float to_value = unit2 == 0.0f ? 0.0f : 1.0f / (unit2 * kValueUnit<FMT>);
  if (a.splits > 1) {
    if (row >= a.row_tiles * 16) return;
    const size_t at = ((size_t)unit * a.row_tiles + (row >> 4)) * a.splits + split;
    RQ_GLOBAL float* p = gptr(a.part) + (at * 16 + (row & 15)) * D + 4 * hl;
#pragma unroll
    for (int c = 0; c < D / 32; ++c)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *(RQ_GLOBAL f4*)(p + 32 * c + 8 * i) =
            (f4){o[c][4 * i], o[c][4 * i + 1], o[c][4 * i + 2], o[c][4 * i + 3]} * to_value;
    if (hl == 0) {
      gptr(a.part_ml)[(at * 16 + (row & 15)) * 2] = m;
      gptr(a.part_ml)[(at * 16 + (row & 15)) * 2 + 1] = l;
    }
    return;
  }
  if (!valid) return;
  const float inv = l > 0.0f ? 1.0f / l : 0.0f, by = inv * to_value;
#pragma unroll
  for (int c = 0; c < D / 32; ++c)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float x[4] = {o[c][4 * i] * by, o[c][4 * i + 1] * by, o[c][4 * i + 2] * by, o[c][4 * i + 3] * by};
      store_out<4>(a, b, h * a.G + head, token, 32 * c + 8 * i + 4 * hl, x);
    }
  if (a.stats && hl == 0) {
    gptr(a.stats)[((size_t)unit * a.row_tiles * 16 + row) * 2] = m;
    gptr(a.stats)[((size_t)unit * a.row_tiles * 16 + row) * 2 + 1] = inv;
  }
}

template <int FMT, int D, bool BF16>
hipError_t launch(const BlockAttendLaunch& a, hipStream_t s) {
  const dim3 grid((unsigned)((a.n * a.G + kRows - 1) / kRows * a.splits) * a.c.B * a.c.H);
  hipLaunchKernelGGL((block_prompt_kernel<FMT, D, BF16>), grid, dim3(kThreads), 0, s, a);
  return hipGetLastError();
}

template <int FMT, int D>
hipError_t launch(const BlockAttendLaunch& a, hipStream_t s) {
  return a.c.is_bf16 ? launch<FMT, D, true>(a, s) : launch<FMT, D, false>(a, s);
}

}  // namespace

hipError_t launch_block_prompt(const BlockAttendLaunch& a, hipStream_t s) {
  if (a.c.fmt == RQ_INT8) return a.c.D == 64 ? launch<RQ_INT8, 64>(a, s) : launch<RQ_INT8, 128>(a, s);
  return a.c.D == 64 ? launch<RQ_E4M3, 64>(a, s) : launch<RQ_E4M3, 128>(a, s);
}

}  // namespace rq
