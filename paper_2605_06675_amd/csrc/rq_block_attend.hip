// Attention over the block-scaled 8-bit cache, for up to 32 query rows a unit:
// the cache is streamed once, for one or two tiles of 16 rows.
//
//   out = softmax(f(scale q . k^)) v^,  f(x) = cap tanh(x / cap) - slope distance
//
// One pass with a running maximum and sum.  The products run on
// v_mfma_f32_16x16x32_f16 with the tokens as rows and the queries as columns:
// S^T = K Q^T leaves a lane with 8 tokens of one query, which is the operand
// that O^T = V^T P^T wants of it, so the probabilities never move between
// lanes.  Every code is exact in fp16; a block's key scale multiplies the
// fp32 scores, its value scale the probabilities.  These are split into an
// fp16 pair hi + lo (22 bits), in units that keep p * scale below 2^15.
//
// Long contexts are bound by memory: 32 units of 32768 tokens (268 MB) 47 us, 5.7
// TB/s where a plain read reaches 7.  Short ones by a chain of latencies (1001
// tokens 7.8 us): lengths, codes, the four waves' sums, parts, ticket, merge.
//
// A tree of up to 16 rows takes the same way, its own nodes as 16-bit blocks behind the
// cached ones (8 kv-heads of 4 heads: 3 nodes over 1001 tokens 9.8 us, 4 of 16
// sequences over 8192, 270 MB, 46.9 to 49.6, and over one of 131072 48.1).
#include <algorithm>
#include <type_traits>

#include "rq_block.h"

namespace rq {

namespace {

template <int D>
struct ValueBlock {
  u2 w[8];        // D = 64: one word each
  float scale;
};

// Lane (r, g) has, of its 8 tokens 16 (j / 4) + 4 g + j % 4, the channels
// D / 16 r + 0..D/16-1.
template <int D>
__device__ __forceinline__ void load_values(const RQ_GLOBAL uint8_t* v, const RQ_GLOBAL float* scale,
                                            int blk, ValueBlock<D>* t) {
  const int lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const int tok = 16 * (j >> 2) + 4 * g + (j & 3);
    const RQ_GLOBAL uint8_t* p = v + (uint32_t)(blk * kBlockTokens + tok) * D + (D / 16) * r;
    if constexpr (D == 128)
      t->w[j] = __builtin_nontemporal_load((const RQ_GLOBAL u2*)p);
    else
      t->w[j].x = __builtin_nontemporal_load((const RQ_GLOBAL uint32_t*)p);
  }
  t->scale = scale[blk];
}

// The running state of one wave: lane (r, g) holds, of query row r, the
// channels D / 16 (4 g + i) + e in o[e][i], in units of kValueUnit / unit.
template <int D>
struct Running {
  f4 o[D / 16];
  float m, l;      // maximum so far (moved lazily: p <= 2^8), this lane's sum
  float unit;      // a power of two: value scale * unit <= 2^7 (0: no block yet)
};

template <int D>
__device__ __forceinline__ void rescale(Running<D>* st, float by) {
#pragma unroll
  for (int e = 0; e < D / 16; ++e) st->o[e] *= by;
}

// Probabilities of a block's scores, and the sums' rescaling where a score
// exceeds the reference by more than 8 (log2).
template <int D>
__device__ __forceinline__ void probabilities(Running<D>* st, f4 s[2]) {
  float top = kNoScore;
#pragma unroll
  for (int m = 0; m < 2; ++m)
#pragma unroll
    for (int i = 0; i < 4; ++i) top = __builtin_fmaxf(top, s[m][i]);
  if (__any(top > st->m + 8.0f)) {
    top = half_all<Max>(pair_all<Max>(top));
    const float mn = __builtin_fmaxf(st->m, top);
    const float by = exp2_f(st->m - mn);
    st->m = mn;
    st->l *= by;
    rescale<D>(st, by);
  }
  float sum = 0.0f;
#pragma unroll
  for (int m = 0; m < 2; ++m)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      s[m][i] = exp2_f(s[m][i] - st->m);
      sum += s[m][i];
    }
  st->l += sum;
}

// The probabilities of QT tiles times a block's value scale, in the tiles'
// common unit, as fp16 pairs hi + lo.  The unit follows the largest scale; a
// scale of zero has none to follow, and its products are zero.
template <int D, int QT>
__device__ __forceinline__ void split_products(const f4 s[QT][2], float scale, Running<D> st[QT],
                                               u4 hi[QT], u4 lo[QT]) {
  if (scale > 0.0f && (scale * st[0].unit > 128.0f || st[0].unit == 0.0f)) {   // (the same in every lane)
    int e = __builtin_amdgcn_frexp_expf(scale);
    e = e < -100 ? -100 : e;
    const float unit = __builtin_amdgcn_ldexpf(128.0f, -e);
#pragma unroll
    for (int n = 0; n < QT; ++n) {
      rescale<D>(&st[n], st[n].unit == 0.0f ? 1.0f : unit / st[n].unit);
      st[n].unit = unit;
    }
  }
  const float by = scale * st[0].unit;
#pragma unroll
  for (int n = 0; n < QT; ++n)
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const float a = s[n][m][2 * i] * by, b = s[n][m][2 * i + 1] * by;
        // (toward zero by its own instruction: a conversion left to the compiler
        // may be fused with the product above, where hi would not be that of a)
        const h2 h = __builtin_bit_cast(h2, __builtin_amdgcn_cvt_pkrtz(a, b));
        hi[n][2 * m + i] = as_u32(h);
        lo[n][2 * m + i] = as_u32((h2){(_Float16)(a - (float)h.x), (_Float16)(b - (float)h.y)});
      }
}

// Adds one operand of values (channels e of every D / 16) to QT tiles.
template <int D, int QT>
__device__ __forceinline__ void add_operand(u4 f, int e, const u4 hi[QT], const u4 lo[QT],
                                            Running<D> st[QT]) {
#pragma unroll
  for (int n = 0; n < QT; ++n) {
    const f4 o = __builtin_amdgcn_mfma_f32_16x16x32_f16(as_h8(f), as_h8(hi[n]), st[n].o[e], 0, 0, 0);
    st[n].o[e] = __builtin_amdgcn_mfma_f32_16x16x32_f16(as_h8(f), as_h8(lo[n]), o, 0, 0, 0);
  }
}

template <int FMT, int D, int QT>
__device__ __forceinline__ void add_values(const ValueBlock<D>& v, const f4 s[QT][2],
                                           Running<D> st[QT]) {
  u4 hi[QT], lo[QT];
  split_products<D, QT>(s, v.scale, st, hi, lo);
#pragma unroll
  for (int c = 0; c < D / 64; ++c) {
    uint32_t op[4][4];        // [token pair][channel]
#pragma unroll
    for (int j = 0; j < 4; ++j) value_pairs<FMT>(v.w[2 * j][c], v.w[2 * j + 1][c], op[j]);
#pragma unroll
    for (int e = 0; e < 4; ++e)
      add_operand<D, QT>((u4){op[0][e], op[1][e], op[2][e], op[3][e]}, 4 * c + e, hi, lo, st);
  }
}

// The values of this lane of the tail or of a tree's nodes (value(row, channel) loads
// two of a row), as load_values has a block's; rows from n_tail on count as zero.
template <int D>
struct TailValues {
  uint32_t w[D / 32][8];      // [two channels][token]
};

template <int D, class Value>
__device__ __forceinline__ void load_tail(Value value, int n_tail, TailValues<D>* t) {
  const int lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
#pragma unroll
  for (int c = 0; c < D / 32; ++c)
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int tok = 16 * (j >> 2) + 4 * g + (j & 3);
      t->w[c][j] = tok < n_tail ? value(tok, (D / 16) * r + 2 * c) : 0u;
    }
}

// The tail's values, divided by a power of two that brings the largest below 1
// (fp16 holds the others to 2^-25 of it), as a block of that scale.
template <int FMT, int D, bool BF16, int QT>
__device__ __forceinline__ void add_tail(const TailValues<D>& t, const f4 s[QT][2], Running<D> st[QT]) {
  const auto& w = t.w;
  float most = 0.0f;
#pragma unroll
  for (int c = 0; c < D / 32; ++c)
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      most = __builtin_fmaxf(most, __builtin_fmaxf(__builtin_fabsf(widen_t<BF16>(w[c][j] & 0xffffu)),
                                                   __builtin_fabsf(widen_t<BF16>(w[c][j] >> 16))));
    }
  most = wave_all<Max>(most);
  if (most == 0.0f) return;
  const int e = __builtin_amdgcn_frexp_expf(most);
  u4 hi[QT], lo[QT];
  split_products<D, QT>(s, __builtin_amdgcn_ldexpf(kValueUnit<FMT>, e), st, hi, lo);
#pragma unroll
  for (int c = 0; c < D / 32; ++c) {
    u4 f[2];
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const h2 p = {(_Float16)__builtin_amdgcn_ldexpf(widen_t<BF16>((w[c][2 * j] >> (16 * i)) & 0xffffu), -e),
                      (_Float16)__builtin_amdgcn_ldexpf(widen_t<BF16>((w[c][2 * j + 1] >> (16 * i)) & 0xffffu), -e)};
        f[i][j] = as_u32(p);
      }
    add_operand<D, QT>(f[0], 2 * c, hi, lo, st);
    add_operand<D, QT>(f[1], 2 * c + 1, hi, lo, st);
  }
}

// Partial results of one row tile: [split][16][D] sums and [split][16][2]
// maxima (log2) and sums of probabilities.  Stored and loaded with the sc1 bit
// (agent scope): coherent across the XCDs' L2 caches without a flush.
struct Parts {
  __amdgpu_buffer_rsrc_t o, ml;
  __device__ __forceinline__ Parts(const BlockAttendLaunch& a, size_t tile) {
    const int D = a.c.D;
    o = __builtin_amdgcn_make_buffer_rsrc(a.part + tile * a.splits * 16 * D, 0,
                                          a.splits * 16 * D * (int)sizeof(float), 0x00027000);
    ml = __builtin_amdgcn_make_buffer_rsrc(a.part_ml + tile * a.splits * 32, 0,
                                           a.splits * 32 * (int)sizeof(float), 0x00027000);
  }
  template <int D>
  __device__ __forceinline__ void store_o(int split, int row, int ch, f4 x) const {
    __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u4, x), o, ((split * 16 + row) * D + ch) * 4, 0, 16);
  }
  __device__ __forceinline__ void store_ml(int split, int row, f2 x) const {
    __builtin_amdgcn_raw_buffer_store_b64(__builtin_bit_cast(u2, x), ml, (split * 16 + row) * 8, 0, 16);
  }
  template <int D>
  __device__ __forceinline__ f4 load_o(int split, int row, int ch) const {
    return __builtin_bit_cast(f4, __builtin_amdgcn_raw_buffer_load_b128(o, ((split * 16 + row) * D + ch) * 4, 0, 16));
  }
  __device__ __forceinline__ f2 load_ml(int split, int row) const {
    return __builtin_bit_cast(f2, __builtin_amdgcn_raw_buffer_load_b64(ml, (split * 16 + row) * 8, 0, 16));
  }
};

// A tile's splits (at most kTicketSplits) added and written by one workgroup.  D / 4 lanes
// form a group, four channels a lane; a row has `share` groups (a power of two),
// each with every share-th split, so that all loads go out at once.
template <int D>
__device__ __forceinline__ void merge_tile(const BlockAttendLaunch& a, const Parts& parts, int b, int h,
                                           int rt, int rows, f4* lds) {
  constexpr int kCols = D / 4, kGroups = 256 / kCols, kEach = kTicketSplits / kCols;
  const int group = threadIdx.x / kCols, col = threadIdx.x % kCols;
  int share = kGroups;
  while (share > 1 && share * rows > kGroups) share >>= 1;
  for (int row0 = 0; row0 < rows; row0 += kGroups / share) {
    const int row = row0 + group / share, first = group % share;
    const bool on = row < rows;
    // this lane has the maxima and sums of splits col, col + kCols, ..
    f2 ml[kEach];
    float m = kNoScore, l = 0.0f;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      ml[i] = (f2){kNoScore, 0.0f};
      if (on && col + i * kCols < a.splits) ml[i] = parts.load_ml(col + i * kCols, row);
    }
#pragma unroll
    for (int i = 0; i < kEach; ++i) m = __builtin_fmaxf(m, ml[i].x);
    m = row_all<Max>(m);
    if constexpr (kCols == 32) m = pair_all<Max>(m);
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      ml[i].x = exp2_f(ml[i].x - m);
      l = __builtin_fmaf(ml[i].y, ml[i].x, l);
    }
    l = row_all<Sum>(l);
    if constexpr (kCols == 32) l = pair_all<Sum>(l);
    f4 x = {0.0f, 0.0f, 0.0f, 0.0f};
    // eight loads at a time; those behind the last split return zeros
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const int n = a.splits - i * kCols < kCols ? a.splits - i * kCols : kCols;
      for (int s0 = first; s0 < n; s0 += 8 * share) {
        f4 o[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) o[j] = parts.load_o<D>(s0 + j * share + i * kCols, row, col * 4);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int s = s0 + j * share;            // (from kCols on: not of this i)
          const float w = __shfl(ml[i].x, s & (kCols - 1), kCols);
          x += o[j] * (s < kCols ? w : 0.0f);
        }
      }
    }
    if (share > 1) {
      lds[threadIdx.x] = x;
      __syncthreads();
      if (first == 0)
        for (int i = 1; i < share; ++i) x += lds[threadIdx.x + i * kCols];
      __syncthreads();
    }
    if (on && first == 0) {
      x *= l > 0.0f ? 1.0f / l : 0.0f;
      const int grow = rt * 16 + row, token = over(grow, a.by_G);
      store_out<4>(a, b, h * a.G + grow - token * a.G, token, col * 4, (const float*)&x);
    }
  }
}

// QT tiles of 16 rows hold all rows of a unit.  A tree (Launch) has its own rows'
// blocks of 32 nodes behind the cached ones.
template <int FMT, int D, bool BF16, int QT, class Launch>
__global__ void __launch_bounds__(256, 2) block_attend_kernel(Launch a) {
  constexpr bool kTree = kIsTree<Launch>;
  constexpr int kStride = D + 4;           // floats of a row in LDS
  __shared__ float sh_o[4][16 * kStride];
  __shared__ float sh_ml[4][16][2];
  __shared__ uint32_t ticket;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r = lane & 15, g = lane >> 4;
  const int split = blockIdx.x, unit = blockIdx.y;
  const int b = over(unit, a.c.by_H), h = unit - b * a.c.H;
  int past, nnew;
  launch_lengths(a, b, &past, &nnew);
  if (nnew == 0) return;
  const int total = kTree ? past : past + nnew, full = total / kBlockTokens;
  int lo_all, hi_all;                      // block `full` is the tail
  seen_blocks(past, 0, nnew - 1, a.window, &lo_all, &hi_all);
  const int cached = (past + kBlockTokens - 1) / kBlockTokens;
  if constexpr (kTree) hi_all = cached + (nnew + kBlockTokens - 1) / kBlockTokens;   // blocks from `cached` on are nodes
  const int lo = lo_all + part_from(hi_all - lo_all, split, a.splits, a.by_splits);
  const int hi = lo_all + part_from(hi_all - lo_all, split + 1, a.splits, a.by_splits);

  QueryTile<D> q[QT];
  Running<D> st[QT];
#pragma unroll
  for (int n = 0; n < QT; ++n) {
    load_queries<D, BF16>(a, b, h, 16 * n + r, past, nnew, &q[n]);
#pragma unroll
    for (int e = 0; e < D / 16; ++e) st[n].o[e] = (f4){0.0f, 0.0f, 0.0f, 0.0f};
    st[n].m = kNoScore;
    st[n].l = 0.0f;
    st[n].unit = 0.0f;
  }

  const RQ_GLOBAL uint8_t* kc = gptr(a.c.codes) + (size_t)unit * 2 * a.c.cap * D;
  const RQ_GLOBAL uint8_t* vc = kc + (size_t)a.c.cap * D;
  const RQ_GLOBAL float* ks = gptr(a.c.scales) + (size_t)unit * 2 * (a.c.cap / kBlockTokens);
  const RQ_GLOBAL float* vs = ks + a.c.cap / kBlockTokens;
  const RQ_GLOBAL int32_t* pos = gptr(a.c.positions) + (size_t)unit * a.c.cap;
  // blocks below all_seen lie wholly before every row
  const int all_seen = a.window ? 0 : (kTree ? past : past + 1) / kBlockTokens;
  // scores kept for the weights: this lane's row, 4 tokens of each half block
  const int rows = a.n * a.G;
  RQ_GLOBAL float* kept = gptr(a.scores) + ((size_t)unit * ((a.max_tokens + kBlockTokens - 1) / kBlockTokens) * rows + r) * kBlockTokens + 4 * g;
  auto keep = [&](const f4 s[2], int n, int blk) {
    if (!kTree && a.scores && 16 * n + r < rows)
#pragma unroll
      for (int m = 0; m < 2; ++m)
        *(RQ_GLOBAL f4*)(kept + ((size_t)blk * rows + 16 * n) * kBlockTokens + 16 * m) = s[m];
  };

  const int end = hi < full ? hi : full;
  auto step = [&](const KeyBlock<D>& k, const ValueBlock<D>& v, int blk) {
    f4 s[QT][2];
    key_products<FMT, D, QT>(k, q, s);
#pragma unroll
    for (int n = 0; n < QT; ++n) {
      block_scores<D>(a, q[n], pos, k.scale * q[n].qs, blk * kBlockTokens, kTree ? past - 1 : past + q[n].token,
                      blk >= all_seen, s[n]);
      keep(s[n], n, blk);
      probabilities<D>(&st[n], s[n]);
    }
    add_values<FMT, D, QT>(v, s, st);
  };
  int blk = lo + wave;
  if (blk < end) {
    // the next block's codes are in flight while one is worked on (the last
    // load repeats the last block)
    KeyBlock<D> k0, k1;
    ValueBlock<D> v0, v1;
    load_keys<D>(kc, ks, blk, &k0);
    load_values<D>(vc, vs, blk, &v0);
    for (;;) {
      const int b1 = blk + 4 < end ? blk + 4 : blk;
      load_keys<D>(kc, ks, b1, &k1);
      load_values<D>(vc, vs, b1, &v1);
      step(k0, v0, blk);
      if (b1 == blk) break;
      blk = b1;
      const int b2 = blk + 4 < end ? blk + 4 : blk;
      load_keys<D>(kc, ks, b2, &k0);
      load_values<D>(vc, vs, b2, &v0);
      step(k1, v1, blk);
      if (b2 == blk) break;
      blk = b2;
    }
  }
  if (lo <= full && full < hi && (!kTree || full < cached) && (full - lo) % 4 == wave) {
    const RQ_GLOBAL uint16_t* kt = gptr(a.c.tail) + (size_t)unit * 2 * kBlockTokens * D;
    const RQ_GLOBAL uint16_t* vt = kt + kBlockTokens * D;
    TailValues<D> tv;          // (on their way while the keys are)
    load_tail<D>([&](int row, int ch) { return *(const RQ_GLOBAL uint32_t*)(vt + row * D + ch); },
                 total % kBlockTokens, &tv);
    f4 s[QT][2];
#pragma unroll
    for (int n = 0; n < QT; ++n) {
      tail_products<D, BF16>(a, b, h, [&](int row, int ch) { return *(const RQ_GLOBAL u4*)(kt + row * D + ch); }, q[n], s[n]);
      block_scores<D>(a, q[n], pos, a.qscale, full * kBlockTokens, kTree ? past - 1 : past + q[n].token, true, s[n]);
      keep(s[n], n, full);
      probabilities<D>(&st[n], s[n]);
    }
    add_tail<FMT, D, BF16, QT>(tv, s, st);
  }
  if constexpr (kTree) {
    int base = 0;
    if (hi > cached && (a.slopes || a.window)) base = tree_base(a, unit, past);
    for (int blk = lo < cached ? cached : lo; blk < hi; ++blk) {
      if ((blk - lo) % 4 != wave) continue;
      const int d = blk - cached, left = nnew - d * kBlockTokens, n_rows = left < kBlockTokens ? left : kBlockTokens;
      const RQ_GLOBAL uint16_t* kn = node_row(a.k, b, h, d * kBlockTokens);
      const RQ_GLOBAL uint16_t* vn = node_row(a.v, b, h, d * kBlockTokens);
      TailValues<D> tv;
      load_tail<D>([&](int row, int ch) { return (uint32_t)*(const RQ_GLOBAL u1_any*)(vn + row * a.v.st + ch); }, n_rows, &tv);
      f4 s[QT][2];
#pragma unroll
      for (int n = 0; n < QT; ++n) {
        tail_products<D, BF16>(a, b, h, [&](int row, int ch) {
          return (u4)*(const RQ_GLOBAL u4_any*)(kn + (row < n_rows ? row : n_rows - 1) * a.k.st + ch);
        }, q[n], s[n]);
        node_scores<D>(a, q[n], b, d, nnew, base, s[n]);
        probabilities<D>(&st[n], s[n]);
      }
      add_tail<FMT, D, BF16, QT>(tv, s, st);
    }
  }

#pragma unroll
  for (int n = 0; n < QT; ++n) {
    if (16 * n >= nnew * a.G) break;
    // the four waves' sums
    const float lsum = half_all<Sum>(pair_all<Sum>(st[n].l));
    const float to_value = st[n].unit == 0.0f ? 0.0f : 1.0f / (st[n].unit * kValueUnit<FMT>);
    if (n > 0) __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int e = 0; e < D / 16; e += 4)
        *(f4*)&sh_o[wave][r * kStride + (D / 16) * (4 * g + i) + e] =
            (f4){st[n].o[e][i], st[n].o[e + 1][i], st[n].o[e + 2][i], st[n].o[e + 3][i]} * to_value;
    if (g == 0) {
      sh_ml[wave][r][0] = st[n].m;
      sh_ml[wave][r][1] = lsum;
    }
    __syncthreads();
    const int row = threadIdx.x >> 4, ch = (threadIdx.x & 15) * (D / 16);
    float m = sh_ml[0][row][0];
    for (int w = 1; w < 4; ++w) m = __builtin_fmaxf(m, sh_ml[w][row][0]);
    float l = 0.0f, x[D / 16];
#pragma unroll
    for (int e = 0; e < D / 16; ++e) x[e] = 0.0f;
    for (int w = 0; w < 4; ++w) {
      const float by = exp2_f(sh_ml[w][row][0] - m);
      l = __builtin_fmaf(sh_ml[w][row][1], by, l);
#pragma unroll
      for (int e = 0; e < D / 16; ++e)
        x[e] = __builtin_fmaf(sh_o[w][row * kStride + ch + e], by, x[e]);
    }
    const int grow = 16 * n + row, token = over(grow, a.by_G);
    if (token >= nnew) continue;
    if (a.splits > 1) {
      const Parts parts(a, (size_t)unit * QT + n);
#pragma unroll
      for (int e = 0; e < D / 16; e += 4)
        parts.store_o<D>(split, row, ch + e, (f4){x[e], x[e + 1], x[e + 2], x[e + 3]});
      if (ch == 0) parts.store_ml(split, row, (f2){m, l});
      continue;
    }
    const float inv = l > 0.0f ? 1.0f / l : 0.0f;
#pragma unroll
    for (int e = 0; e < D / 16; ++e) x[e] *= inv;
    store_out<D / 16>(a, b, h * a.G + grow - token * a.G, token, ch, x);
    if (a.stats && ch == 0) {
      gptr(a.stats)[((size_t)unit * QT * 16 + grow) * 2] = m;
      gptr(a.stats)[((size_t)unit * QT * 16 + grow) * 2 + 1] = inv;
    }
  }
  // the unit's last workgroup adds its parts
  if (!a.tickets) return;
  RQ_GLOBAL uint32_t* counter = gptr(a.c.counters) + unit;
  __builtin_amdgcn_s_waitcnt(0);                     // this wave's parts are out
  __syncthreads();
  if (threadIdx.x == 0)
    ticket = __hip_atomic_fetch_add(counter, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  __syncthreads();
  if (ticket != (uint32_t)a.splits - 1) return;
  if (threadIdx.x == 0)
    __hip_atomic_store(counter, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
#pragma unroll
  for (int n = 0; n < QT; ++n) {
    const int seen = nnew * a.G - 16 * n;            // rows with a query
    merge_tile<D>(a, Parts(a, (size_t)unit * QT + n), b, h, n, seen < 16 ? seen : 16,
                  reinterpret_cast<f4*>(sh_o));
  }
}

// Adds the splits' partial results of one row: 256 threads hold four channels
// each of 1024 / D splits at a time.  (Eight units of 96 splits: 5.0 us; one
// thread a channel group, a split after the other: 50 us.)
template <int D>
__device__ __forceinline__ void merge_row(const BlockAttendLaunch& a, int grow, int unit, int b,
                                          int h, int nnew) {
  constexpr int kCols = D / 4, kGroups = 256 / kCols;
  __shared__ f4 sum[kGroups][kCols];
  const int token = over(grow, a.by_G), rt = grow >> 4, row = grow & 15;
  if (token >= nnew) return;
  const int lane = threadIdx.x & 63, col = threadIdx.x % kCols, group = threadIdx.x / kCols;
  const size_t base = ((size_t)unit * a.row_tiles + rt) * a.splits;
  const RQ_GLOBAL float* ml = gptr(a.part_ml) + (base * 16 + row) * 2;
  const RQ_GLOBAL float* o = gptr(a.part) + (base * 16 + row) * D + col * 4;
  float m = kNoScore;
  for (int s = lane; s < a.splits; s += 64) m = __builtin_fmaxf(m, ml[s * 32]);
  m = wave_all<Max>(m);
  float l = 0.0f;
  for (int s = lane; s < a.splits; s += 64)
    l = __builtin_fmaf(ml[s * 32 + 1], exp2_f(ml[s * 32] - m), l);
  l = wave_all<Sum>(l);
  f4 x = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 4
  for (int s = group; s < a.splits; s += kGroups) {
    const float by = exp2_f(ml[s * 32] - m);
    x += *(const RQ_GLOBAL f4*)(o + (size_t)s * 16 * D) * by;
  }
  sum[group][col] = x;
  __syncthreads();
  const float inv = l > 0.0f ? 1.0f / l : 0.0f;
  if (group == 0) {
    for (int i = 1; i < kGroups; ++i) x += sum[i][col];
    x *= inv;
    store_out<4>(a, b, h * a.G + grow - token * a.G, token, col * 4, (const float*)&x);
  }
  if (a.stats && threadIdx.x == 0) {
    gptr(a.stats)[((size_t)unit * a.row_tiles * 16 + grow) * 2] = m;
    gptr(a.stats)[((size_t)unit * a.row_tiles * 16 + grow) * 2 + 1] = inv;
  }
}

// Few splits of many rows: 1024 / D rows a workgroup, each thread four channels
// of one.  Up to eight splits are all loaded before any is used: a launch of few rows is
// a chain of latencies (with the attention's, five splits of 256 rows 11.1 us, maxima
// and parts one after the other 11.8; six of 1260 rows 17.2, 18.5).  RAGGED: a sequence
// may have fewer rows than the call, and its lengths are waited for first, so that the
// parts of rows without a query are not read: two splits of 32 units and 1024 rows,
// 31 % of them used, 5.4 us, all read 6.9; no padding 7.9 and 7.6.
template <int D, bool RAGGED>
__global__ void __launch_bounds__(256) block_merge_rows_kernel(BlockAttendLaunch a) {
  constexpr int kCols = D / 4;
  const int unit = blockIdx.y, b = over(unit, a.c.by_H), h = unit - b * a.c.H;
  const int grow = blockIdx.x * (256 / kCols) + threadIdx.x / kCols, col = threadIdx.x % kCols;
  const int token = over(grow, a.by_G), row = grow & 15;
  const size_t base = ((size_t)unit * a.row_tiles + (grow >> 4)) * a.splits;
  const RQ_GLOBAL f2* ml = (const RQ_GLOBAL f2*)(gptr(a.part_ml) + (base * 16 + row) * 2);
  const RQ_GLOBAL float* o = gptr(a.part) + (base * 16 + row) * D + col * 4;
  if constexpr (RAGGED) {
    if (token >= new_tokens(a.new_len, b, a.n, a.max_tokens)) return;
  }
  float m = kNoScore, l = 0.0f;
  f4 x = {0.0f, 0.0f, 0.0f, 0.0f};
  auto at_once = [&](auto most) {
    f2 p[most.value];
    f4 y[most.value];
#pragma unroll
    for (int s = 0; s < most.value; ++s) {
      const int from = s < a.splits ? s : 0;
      p[s] = ml[from * 16];
      y[s] = *(const RQ_GLOBAL f4*)(o + (size_t)from * 16 * D);
    }
    asm volatile("" ::: "memory");         // (all are asked for before any is used)
#pragma unroll
    for (int s = 0; s < most.value; ++s) m = __builtin_fmaxf(m, s < a.splits ? p[s].x : kNoScore);
#pragma unroll
    for (int s = 0; s < most.value; ++s) {
      if (s < a.splits) {
        const float by = exp2_f(p[s].x - m);
        l = __builtin_fmaf(p[s].y, by, l);
        x += y[s] * by;
      }
    }
  };
  if (a.splits <= 2) {
    at_once(std::integral_constant<int, 2>{});
  } else if (a.splits <= 4) {
    at_once(std::integral_constant<int, 4>{});
  } else if (a.splits <= 8) {
    at_once(std::integral_constant<int, 8>{});
  } else {
#pragma unroll 4
    for (int s = 0; s < a.splits; ++s) m = __builtin_fmaxf(m, ml[s * 16].x);
#pragma unroll 4
    for (int s = 0; s < a.splits; ++s) {
      const f2 p = ml[s * 16];
      const float by = exp2_f(p.x - m);
      l = __builtin_fmaf(p.y, by, l);
      x += *(const RQ_GLOBAL f4*)(o + (size_t)s * 16 * D) * by;
    }
  }
  if (!RAGGED && token >= new_tokens(nullptr, b, a.n, a.max_tokens)) return;
  const float inv = l > 0.0f ? 1.0f / l : 0.0f;
  x *= inv;
  store_out<4>(a, b, h * a.G + grow - token * a.G, token, col * 4, (const float*)&x);
  if (a.stats && col == 0) {
    gptr(a.stats)[((size_t)unit * a.row_tiles * 16 + grow) * 2] = m;
    gptr(a.stats)[((size_t)unit * a.row_tiles * 16 + grow) * 2 + 1] = inv;
  }
}

template <int D>
__global__ void __launch_bounds__(256) block_merge_kernel(BlockAttendLaunch a) {
  const int unit = blockIdx.y, b = over(unit, a.c.by_H);
  int past, nnew;
  block_lengths(a.past, a.new_len, b, a.n, a.max_tokens, &past, &nnew);
  merge_row<D>(a, blockIdx.x, unit, b, unit - b * a.c.H, nnew);
}

// The same, and in the workgroups behind those of the rows the weights of 1024
// tokens each: the scores that the first kernel kept against the rows' maxima
// and sums (every workgroup merges those by itself).
template <int D>
__global__ void __launch_bounds__(256) block_merge_weigh_kernel(BlockAttendLaunch a) {
  __shared__ float sh_m[32], sh_inv[32];
  const int unit = blockIdx.y, b = over(unit, a.c.by_H);
  int past, nnew;
  block_lengths(a.past, a.new_len, b, a.n, a.max_tokens, &past, &nnew);
  const int all = a.n * a.G, merges = a.splits > 1 ? all : 0;
  if ((int)blockIdx.x < merges) {
    merge_row<D>(a, blockIdx.x, unit, b, unit - b * a.c.H, nnew);
    return;
  }
  const int rows = nnew * a.G;
  int lo, hi;
  seen_blocks(past, 0, nnew - 1, a.window, &lo, &hi);
  const int first = (lo / 32 + blockIdx.x - merges) * 32;    // blocks first..first + 31
  if (nnew == 0 || first >= hi) return;
  const int lane = threadIdx.x & 15;
  for (int row = threadIdx.x >> 4; row < rows; row += 16) {
    if (a.splits > 1) {
      const RQ_GLOBAL float* ml = gptr(a.part_ml) + (((size_t)unit * a.row_tiles + (row >> 4)) * a.splits * 16 + (row & 15)) * 2;
      float m = kNoScore, l = 0.0f;
      for (int s = lane; s < a.splits; s += 16) m = __builtin_fmaxf(m, ml[s * 32]);
      m = row_all<Max>(m);
      for (int s = lane; s < a.splits; s += 16)
        l = __builtin_fmaf(ml[s * 32 + 1], exp2_f(ml[s * 32] - m), l);
      l = row_all<Sum>(l);
      if (lane == 0) {
        sh_m[row] = m;
        sh_inv[row] = l > 0.0f ? 1.0f / l : 0.0f;
      }
    } else if (lane == 0) {
      sh_m[row] = gptr(a.stats)[((size_t)unit * a.row_tiles * 16 + row) * 2];
      sh_inv[row] = gptr(a.stats)[((size_t)unit * a.row_tiles * 16 + row) * 2 + 1];
    }
  }
  __syncthreads();
  const int blk = first + (threadIdx.x >> 3), slot = blk * kBlockTokens + 4 * (threadIdx.x & 7);
  if (blk < lo || blk >= hi) return;
  const size_t blocks = (a.max_tokens + kBlockTokens - 1) / kBlockTokens;
  const RQ_GLOBAL float* x = gptr(a.scores) + (unit * blocks + blk) * all * kBlockTokens + 4 * (threadIdx.x & 7);
  f4 sum = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 4
  for (int i = 0; i < rows; ++i) {
    const f4 s = *(const RQ_GLOBAL f4*)(x + i * kBlockTokens);
#pragma unroll
    for (int j = 0; j < 4; ++j) sum[j] = __builtin_fmaf(exp2_f(s[j] - sh_m[i]), sh_inv[i], sum[j]);
  }
  RQ_GLOBAL float* w = gptr(a.c.weights) + (size_t)unit * a.c.cap + slot;
#pragma unroll
  for (int j = 0; j < 4; ++j)
    if (slot + j < past + nnew) w[j] += sum[j];
}

template <int FMT, int D, bool BF16>
void launch(const BlockAttendLaunch& a, hipStream_t s) {
  const dim3 grid(a.splits, a.c.B * a.c.H);
  if (a.row_tiles == 1)
    hipLaunchKernelGGL((block_attend_kernel<FMT, D, BF16, 1, BlockAttendLaunch>), grid, dim3(256), 0, s, a);
  else
    hipLaunchKernelGGL((block_attend_kernel<FMT, D, BF16, 2, BlockAttendLaunch>), grid, dim3(256), 0, s, a);
}

template <int FMT, int D, bool BF16>
void launch(const BlockTreeLaunch& a, hipStream_t s) {
  hipLaunchKernelGGL((block_attend_kernel<FMT, D, BF16, 1, BlockTreeLaunch>), dim3(a.splits, a.c.B * a.c.H), dim3(256), 0,
                     s, a);
}

template <int FMT, int D>
hipError_t launch(const BlockTreeLaunch& a, hipStream_t s) {
  if (a.c.is_bf16)
    launch<FMT, D, true>(a, s);
  else
    launch<FMT, D, false>(a, s);
  const hipError_t e = hipGetLastError();
  return e != hipSuccess || a.tickets ? e : launch_block_merge(a, s);
}

template <int FMT, int D>
hipError_t launch(const BlockAttendLaunch& a, hipStream_t s) {
  if (a.c.is_bf16)
    launch<FMT, D, true>(a, s);
  else
    launch<FMT, D, false>(a, s);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int rows = a.n * a.G;
  if (a.scores) {
    // 1024 tokens a workgroup (one more where a window begins inside one)
    int64_t tokens = a.max_tokens;
    if (a.window) tokens = std::min(tokens, (int64_t)a.window + a.n);
    const int parts = (int)((tokens + 1023) / 1024) + (a.window ? 1 : 0);
    hipLaunchKernelGGL((block_merge_weigh_kernel<D>), dim3((a.splits > 1 ? rows : 0) + parts, a.c.B * a.c.H),
                       dim3(256), 0, s, a);
    return hipGetLastError();
  }
  return a.tickets ? hipSuccess : launch_block_merge(a, s);
}

}  // namespace

template <int D>
static hipError_t merge(const BlockAttendLaunch& a, hipStream_t s) {
  const int rows = a.n * a.G, units = a.c.B * a.c.H, per = 1024 / D;
  const bool by_rows = a.splits <= 8 || (int64_t)rows * units >= 4096;
  const dim3 grid((rows + per - 1) / per, units);
  if (by_rows && a.new_len)
    hipLaunchKernelGGL((block_merge_rows_kernel<D, true>), grid, dim3(256), 0, s, a);
  else if (by_rows)
    hipLaunchKernelGGL((block_merge_rows_kernel<D, false>), grid, dim3(256), 0, s, a);
  else
    hipLaunchKernelGGL((block_merge_kernel<D>), dim3(rows, units), dim3(256), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_block_merge(const BlockAttendLaunch& a, hipStream_t s) {
  if (a.splits == 1) return hipSuccess;
  return a.c.D == 64 ? merge<64>(a, s) : merge<128>(a, s);
}

hipError_t launch_tree_attend(const BlockTreeLaunch& a, hipStream_t s) {
  if (a.c.fmt == RQ_INT8) return a.c.D == 64 ? launch<RQ_INT8, 64>(a, s) : launch<RQ_INT8, 128>(a, s);
  return a.c.D == 64 ? launch<RQ_E4M3, 64>(a, s) : launch<RQ_E4M3, 128>(a, s);
}

hipError_t launch_block_attend(const BlockAttendLaunch& a, hipStream_t s) {
  if (a.c.fmt == RQ_INT8) return a.c.D == 64 ? launch<RQ_INT8, 64>(a, s) : launch<RQ_INT8, 128>(a, s);
  return a.c.D == 64 ? launch<RQ_E4M3, 64>(a, s) : launch<RQ_E4M3, 128>(a, s);
}

}  // namespace rq
