// Attention of a tree's nodes over the block-scaled 8-bit cache and each other, for
// more than 16 query rows a unit.
//
//   out = softmax(f(scale q . k) - slope distance) v
//
// A workgroup owns 32 or 64 rows of a unit (token-major, the heads of a group
// together) and a part of its tokens; its four or eight waves take turns at the blocks
// of 32 tokens, each with all rows, one running maximum and sum, and the next block's
// codes in flight.  On v_mfma_f32_32x32x16_f16 S^T = K Q^T leaves a lane with 16 tokens
// of one row, the operand that O^T = V^T P^T wants of it.  Every code is converted to
// fp16 once for the rows, in the registers of the wave that uses it: nothing is shared
// but the queries, which are read from LDS, so no barrier separates the waves.  The
// cached tokens are before every node: only the tail and the nodes' own blocks are
// masked.
//
// A block's value scale goes into the exponent, and P' is an fp16 pair hi + lo (22
// bits), as in the other attention kernels.
//
// 16 sequences of 8 kv-heads, 28 rows and up to 8192 tokens (204 MB) take 43 to 51 us,
// 4 to 4.7 TB/s: memory, and lengths that differ.  256 rows, 64 units of 8192 tokens
// (69 GFLOP, 104 with P's low halves) 103 to 113 us from card to card, 0.65 PFLOP/s (1.0,
// where a large library product reaches 1.2): the products, at the clock that they leave (2.0 GHz).
// Without the low halves' 82.5, without the scores' 82.7, but with all loads from the
// cache 104.5, without exponentials 100.6, queries in registers 98.  Reads of the queries
// further ahead, raised priorities and three stages of codes changed nothing.  1001
// tokens and 32 rows 11.1 us, two launches of latencies: lengths, queries, codes, the
// waves' sums, parts.
#include "rq_block.h"

namespace rq {

namespace {

typedef float f16v __attribute__((ext_vector_type(16)));

// The codes of a block as a wave holds them: lane (col = lane & 31, hl = lane >> 5)
// has of token col the channels 32 j + 16 hl + 0..15 of the keys, and of the values'
// tokens 8 j + 4 hl + i the channels D / 32 col + 0..D/32-1.
template <int D>
struct Codes {
  u4 k[D / 32];
  uint32_t v[16];
  float kscale, vscale;
  int pos;           // token col's position, where positions matter
};

// (Both scales by vector loads, with the keys: a scalar load's wait would be one for
// the queries' LDS reads too, one with the values a wait for these where the value
// scale is first asked for.)
template <int D>
__device__ __forceinline__ void load_keys(const RQ_GLOBAL uint8_t* kc, const RQ_GLOBAL float* ks, const RQ_GLOBAL float* vs,
                                          int blk, Codes<D>* t) {
  const int lane = threadIdx.x & 63, col = lane & 31, hl = lane >> 5;
  const RQ_GLOBAL uint8_t* k = kc + (uint32_t)(blk * kBlockTokens + col) * D + 16 * hl;
#pragma unroll
  for (int j = 0; j < D / 32; ++j) t->k[j] = *(const RQ_GLOBAL u4*)(k + 32 * j);
  t->kscale = ks[blk];
  t->vscale = vs[blk];
}
template <int D>
__device__ __forceinline__ void load_values(const RQ_GLOBAL uint8_t* vc, int blk, Codes<D>* t) {
  const int lane = threadIdx.x & 63, col = lane & 31, hl = lane >> 5;
  const RQ_GLOBAL uint8_t* v = vc + (uint32_t)(blk * kBlockTokens + 4 * hl) * D + D / 32 * col;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const RQ_GLOBAL uint8_t* p = v + (8 * (i >> 2) + (i & 3)) * D;
    if constexpr (D == 128)
      t->v[i] = *(const RQ_GLOBAL uint32_t*)p;
    else
      t->v[i] = *(const RQ_GLOBAL uint16_t*)p;
  }
}

typedef unsigned short us2 __attribute__((ext_vector_type(2)));

// Two bf16 numbers over 2^e, as fp16.
__device__ __forceinline__ uint32_t halves(uint32_t x, uint32_t y, int e) {
  return as_u32((h2){(_Float16)__builtin_amdgcn_ldexpf(widen_t<true>(x), -e), (_Float16)__builtin_amdgcn_ldexpf(widen_t<true>(y), -e)});
}

// RT tiles of 32 rows.  The lane's row of tile n, its sums in units of kValueUnit /
// unit: channel D / 32 (8 (i / 4) + 4 hl + i % 4) + e in o[n][e][i].
template <int D, int RT>
struct Rows {
  f16v o[RT][D / 32];
  float m[RT], l[RT], qs[RT];
  float unit;
};

// PLAIN: no cap, no window, no slopes.
// Registers of a lane: 32 rows 120 to 190; 64 rows 172 to 189 of 64 channels, and all
// 256 of 128 channels (up to 3 more in scratch memory) or with options (4 to 12).
template <int FMT, int D, bool BF16, int RT, int kWaves, bool PLAIN>
__global__ void __launch_bounds__(64 * kWaves, 2) tree_rows_kernel(BlockTreeLaunch a) {
  constexpr int kThreads = 64 * kWaves, kRows = 32 * RT, kStride = D + 4, kE = D / 32, kK = D / 16, kBufs = kWaves / 2;
  __shared__ __align__(16) float sh_o[kBufs][kRows * kStride];    // first the queries: [tile][operand][lane]
  __shared__ float sh_qs[RT][32];
  __shared__ float sh_m[kWaves][kRows], sh_l[kWaves][kRows];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 31, hl = lane >> 5;
  // where the units are a multiple of eight, a unit's workgroups share an XCD's L2
  const int units = a.c.B * a.c.H, groups = (a.n * a.G + kRows - 1) / kRows, each = groups * a.splits;
  int unit, w;
  if (units % 8 == 0) {
    const uint32_t eight = blockIdx.x / 8, u = eight / (uint32_t)each;
    unit = (int)u * 8 + blockIdx.x % 8;
    w = eight - u * each;
  } else {
    unit = blockIdx.x / (uint32_t)each;
    w = blockIdx.x - unit * each;
  }
  const int group = over(w, a.by_splits), split = w - group * a.splits;
  const int b = over(unit, a.c.by_H), h = unit - b * a.c.H;
  int past, nnew;
  launch_lengths(a, b, &past, &nnew);
  const int row0 = group * kRows;
  if (row0 >= nnew * a.G) return;
  const int full = past / kBlockTokens, cached = (past + kBlockTokens - 1) / kBlockTokens;
  int lo, hi, hi_seen;
  seen_blocks(past, 0, 0, a.window, &lo, &hi_seen);
  {
    const int all = cached - lo + (nnew + kBlockTokens - 1) / kBlockTokens, first = lo;
    lo = first + part_from(all, split, a.splits, a.by_splits);
    hi = first + part_from(all, split + 1, a.splits, a.by_splits);
  }

  const RQ_GLOBAL uint8_t* kc = gptr(a.c.codes) + (size_t)unit * 2 * a.c.cap * D;
  const RQ_GLOBAL uint8_t* vc = kc + (size_t)a.c.cap * D;
  // (the compiler does not know the zero, and so not that all lanes load alike)
  int zero = 0;
  asm volatile("" : "+v"(zero));
  const RQ_GLOBAL float* ks = gptr(a.c.scales) + (size_t)unit * 2 * (a.c.cap / kBlockTokens) + zero;
  const RQ_GLOBAL float* vs = ks + a.c.cap / kBlockTokens;
  const RQ_GLOBAL int32_t* pos = gptr(a.c.positions) + (size_t)unit * a.c.cap;
  const int end = hi < full ? hi : full;
  const bool far = !PLAIN && (a.slopes || a.window);
  Codes<D> c;
  auto next_keys = [&](int blk) {
    load_keys<D>(kc, ks, vs, blk, &c);
    if (far) c.pos = pos[blk * kBlockTokens + col];
  };
  // the lane's rows
  Rows<D, RT> st;
  int token[RT], qpos[RT];
  float slope[RT];
  const int base = PLAIN ? 0 : tree_base(a, unit, past);
  u4 raw[kK];
  bool used = false;
#pragma unroll
  for (int n = 0; n < RT; ++n) {
    const int row = row0 + 32 * n + col;
    token[n] = over(row, a.by_G);
    const int head = row - token[n] * a.G;
    const bool valid = token[n] < nnew;
    token[n] = valid ? token[n] : nnew - 1;
    slope[n] = 0.0f;
    qpos[n] = 0;
    if constexpr (!PLAIN) {
      if (a.slopes) slope[n] = gptr(a.slopes)[h * a.G + head] * 1.4426950408889634f;
      if (a.slopes || a.window) qpos[n] = base + node_depth(a, b, token[n]);
    }
    if (wave == n) {
      const RQ_GLOBAL uint16_t* p = gptr(static_cast<const uint16_t*>(a.q.p)) + b * a.q.sb +
                                    (int64_t)(h * a.G + head) * a.q.sh + token[n] * a.q.st + 16 * hl;
#pragma unroll
      for (int k = 0; k < kK; ++k) raw[k] = *(const RQ_GLOBAL u4_any*)(p + 32 * (k >> 1) + 8 * (k & 1));
      used = valid;
    }
  }
  // (behind the queries, which are wanted first)
  if (lo + wave < end) {
    next_keys(lo + wave);
    load_values<D>(vc, lo + wave, &c);
  }
  if (wave < RT) {
    // fp16 queries as they are; bf16 rows over a power of two above their largest
    // (a negative scale turns the queries, so that scores grow with products)
    const uint32_t turn = a.qscale < 0.0f ? 0x80008000u : 0u;
    float qs = __builtin_fabsf(a.qscale);
#pragma unroll
    for (int k = 0; k < kK; ++k)
#pragma unroll
      for (int i = 0; i < 4; ++i) raw[k][i] = used ? raw[k][i] ^ turn : 0u;
    if constexpr (BF16) {
      us2 most = {0, 0};
#pragma unroll
      for (int k = 0; k < kK; ++k)
#pragma unroll
        for (int i = 0; i < 4; ++i) most = __builtin_elementwise_max(most, __builtin_bit_cast(us2, raw[k][i] & 0x7fff7fffu));
      const float largest = half_all<Max>(widen_t<true>(most.x > most.y ? most.x : most.y));
      const int e = largest > 0.0f ? __builtin_amdgcn_frexp_expf(largest) : 0;
#pragma unroll
      for (int k = 0; k < kK; ++k)
#pragma unroll
        for (int i = 0; i < 4; ++i) raw[k][i] = halves(raw[k][i] & 0xffffu, raw[k][i] >> 16, e);
      qs = __builtin_amdgcn_ldexpf(qs, e);
    }
#pragma unroll
    for (int k = 0; k < kK; ++k) *(u4*)((uint8_t*)sh_o + ((wave * kK + k) * 64 + lane) * 16) = raw[k];
    if (hl == 0) sh_qs[wave][col] = qs;
  }
  __syncthreads();
  __builtin_amdgcn_sched_barrier(0);
#pragma unroll
  for (int n = 0; n < RT; ++n) {
#pragma unroll
    for (int e = 0; e < kE; ++e)
#pragma unroll
      for (int i = 0; i < 16; ++i) st.o[n][e][i] = 0.0f;
    st.m[n] = kNoScore;
    st.l[n] = 0.0f;
    st.qs[n] = sh_qs[n][col];
  }
  st.unit = 0.0f;

  // products of a block's keys with all rows: key(k) is operand k
  auto products = [&](auto key, f16v s[RT]) {
#pragma unroll
    for (int n = 0; n < RT; ++n)
#pragma unroll
      for (int i = 0; i < 16; ++i) s[n][i] = 0.0f;
    uint32_t from = lane * 16;
    asm volatile("" : "+v"(from));         // (read here, not kept in registers from before the loop)
#pragma unroll
    for (int k = 0; k < kK; ++k) {
      const h8 f = key(k);
#pragma unroll
      for (int n = 0; n < RT; ++n)
        s[n] = __builtin_amdgcn_mfma_f32_32x32x16_f16(f, *(const h8*)((const uint8_t*)sh_o + from + (n * kK + k) * 1024), s[n], 0, 0, 0);
    }
  };
  // Scores, probabilities and their sums of a block of key scale kscale and value
  // scale vscale.  value(j, x): of the lane's tokens 2 j and 2 j + 1 the pairs of
  // each channel e.  seen[n]: the tokens that the lane's row sees; at:
  // token col's position; then: called when the keys and their scale are used up.
  auto attend = [&](f16v s[RT], float kscale, float vscale, bool masked, const uint32_t seen[RT], int at, auto then, auto value) {
    float f[RT], off = 0.0f;
#pragma unroll
    for (int n = 0; n < RT; ++n) f[n] = kscale * st.qs[n];
    then();
    if constexpr (!PLAIN) {
      if (a.cap != 0.0f && !a.fine) {
        // cap tanh(x) = cap - 2 cap / (1 + e^(2x)): off by 2^-22 cap
#pragma unroll
        for (int n = 0; n < RT; ++n) {
          const float e2 = f[n] * 2.8853900817779268f;
#pragma unroll
          for (int i = 0; i < 16; ++i) s[n][i] = __builtin_amdgcn_rcpf(-1.0f - exp2_f(s[n][i] * e2));
          f[n] = 2.0f * a.cap;
        }
        off = a.cap;
      }
      if (far || a.fine) {
#pragma unroll
        for (int n = 0; n < RT; ++n) {
#pragma unroll
          for (int i = 0; i < 16; ++i) s[n][i] = __builtin_fmaf(s[n][i], f[n], off);
          if (a.fine) {
#pragma unroll
            for (int i = 0; i < 16; ++i) s[n][i] = a.cap * tanh_f(s[n][i]);
          }
          f[n] = 1.0f;
        }
        off = 0.0f;
      }
      if (far) {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int p = __shfl(at, 8 * (i >> 2) + 4 * hl + (i & 3));
#pragma unroll
          for (int n = 0; n < RT; ++n) {
            const int away = qpos[n] - p;
            s[n][i] = __builtin_fmaf(-slope[n], (float)away, s[n][i]);
            if (a.window && away >= a.window) s[n][i] = -__builtin_inff();
          }
        }
      }
    }
    if (masked) {
      // (formed first: a factor of zero would make NaN of an infinity)
#pragma unroll
      for (int n = 0; n < RT; ++n) {
        const uint32_t bits = seen[n] >> (4 * hl);
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const float x = __builtin_fmaf(s[n][i], f[n], off);
          s[n][i] = (bits >> (8 * (i >> 2) + (i & 3))) & 1u ? x : -__builtin_inff();
        }
        f[n] = 1.0f;
      }
      off = 0.0f;
    }
    // the running maximum (moved when a score exceeds it by 8) and unit
    float top[RT];
    bool move = false;
#pragma unroll
    for (int n = 0; n < RT; ++n) {
      float x = s[n][0];
#pragma unroll
      for (int i = 1; i < 16; ++i) x = __builtin_fmaxf(x, s[n][i]);
      top[n] = __builtin_fmaxf(kNoScore, __builtin_fmaf(x, f[n], off));
      move |= top[n] > st.m[n] + 8.0f;
    }
    // (the same in every lane; a scale of zero has no unit to follow)
    const bool grow = vscale > 0.0f && (st.unit == 0.0f || vscale * st.unit > 128.0f);
    if (grow || __any(move)) {
      float ratio = 1.0f;
      if (grow) {
        int e = __builtin_amdgcn_frexp_expf(vscale);
        e = e < -100 ? -100 : e;
        const float u = __builtin_amdgcn_ldexpf(128.0f, -e);
        ratio = st.unit == 0.0f ? 1.0f : u * __builtin_amdgcn_rcpf(st.unit);     // (powers of two)
        st.unit = u;
      }
#pragma unroll
      for (int n = 0; n < RT; ++n) {
        const float mn = __builtin_fmaxf(st.m[n], half_all<Max>(top[n]));
        const float by = exp2_f(st.m[n] - mn);
        st.m[n] = mn;
        st.l[n] *= by;
#pragma unroll
        for (int e = 0; e < kE; ++e) st.o[n][e] *= by * ratio;
      }
    }
    const float by = vscale > 0.0f ? __builtin_fmaxf(vscale * st.unit, 0x1p-80f) : 1.0f;
    const float lg = __builtin_amdgcn_logf(by), inv = __builtin_amdgcn_rcpf(by);
    uint32_t ph[RT][8], pl[RT][8];
    // (scores this large are rounded before their difference is taken)
    float ref[RT];
    bool large = false;
#pragma unroll
    for (int n = 0; n < RT; ++n) {
      ref[n] = st.m[n] - off;
      large |= __builtin_fabsf(st.m[n]) > kLargeScore && st.m[n] > kNoScore;
    }
    if (__any(large)) {
#pragma unroll
      for (int n = 0; n < RT; ++n) {
#pragma unroll
        for (int i = 0; i < 16; ++i) s[n][i] = __builtin_fmaf(s[n][i], f[n], off) - st.m[n];
        f[n] = 1.0f;
        ref[n] = 0.0f;
      }
    }
#pragma unroll
    for (int n = 0; n < RT; ++n) {
      const float c = ref[n] - lg;
      float sum = 0.0f;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float x = exp2_f(__builtin_fmaf(s[n][2 * i], f[n], -c));
        const float y = exp2_f(__builtin_fmaf(s[n][2 * i + 1], f[n], -c));
        const h2 p = __builtin_bit_cast(h2, __builtin_amdgcn_cvt_pkrtz(x, y));
        ph[n][i] = as_u32(p);
        float xl, yl;      // what the halves leave of x and y, exactly
        asm("v_fma_mix_f32 %0, %1, -1.0, %2 op_sel_hi:[1,0,0]" : "=v"(xl) : "v"(p), "v"(x));
        asm("v_fma_mix_f32 %0, %1, -1.0, %2 op_sel:[1,0,0] op_sel_hi:[1,0,0]" : "=v"(yl) : "v"(p), "v"(y));
        pl[n][i] = as_u32((h2){(_Float16)xl, (_Float16)yl});
        sum += x;
        sum += y;
      }
      st.l[n] = __builtin_fmaf(sum, inv, st.l[n]);
    }
#pragma unroll
    for (int g = 0; g < 2; ++g) {
      uint32_t op[4][4];
#pragma unroll
      for (int j = 0; j < 4; ++j) value(4 * g + j, op[j]);
#pragma unroll
      for (int e = 0; e < kE; ++e) {
        const h8 v = as_h8((u4){op[0][e], op[1][e], op[2][e], op[3][e]});
#pragma unroll
        for (int n = 0; n < RT; ++n)
          st.o[n][e] = __builtin_amdgcn_mfma_f32_32x32x16_f16(
              v, as_h8((u4){ph[n][4 * g], ph[n][4 * g + 1], ph[n][4 * g + 2], ph[n][4 * g + 3]}), st.o[n][e], 0, 0, 0);
#pragma unroll
        for (int n = 0; n < RT; ++n)
          st.o[n][e] = __builtin_amdgcn_mfma_f32_32x32x16_f16(
              v, as_h8((u4){pl[n][4 * g], pl[n][4 * g + 1], pl[n][4 * g + 2], pl[n][4 * g + 3]}), st.o[n][e], 0, 0, 0);
      }
    }
  };

  int blk = lo + wave;
  while (blk < end) {
    // The next block's keys are loaded where this one's are used up, its values where
    // these are (at the end, the last block's again).
    const int next = blk + kWaves < end ? blk + kWaves : blk;
    f16v s[RT];
    products([&](int k) {
      const uint32_t x = c.k[k >> 1][2 * (k & 1)], y = c.k[k >> 1][2 * (k & 1) + 1];
      return as_h8((u4){key_pair<FMT>(x, false), key_pair<FMT>(x, true), key_pair<FMT>(y, false), key_pair<FMT>(y, true)});
    }, s);
    const uint32_t all[RT] = {};
    attend(s, c.kscale, __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(c.vscale))), false, all,
           c.pos, [&] { next_keys(next); },
           [&](int j, uint32_t op[4]) { value_pairs<FMT>(c.v[2 * j], c.v[2 * j + 1], op); });
    load_values<D>(vc, next, &c);
    if (next == blk) break;
    blk = next;
  }

  // Blocks of 16-bit rows: the tail, then the nodes.  fp16 numbers are operands as
  // they are; both sides of bf16 ones are divided by a power of two that brings the
  // side's largest below 1 (fp16 holds the others to 2^-25 of it).  Rows behind the
  // last repeat it, their values are 0.
  for (blk = lo < full ? full : lo; blk < hi; ++blk) {
    if ((blk - lo) % kWaves != wave) continue;
    const bool tail = blk < cached;
    const int first = tail ? 0 : (blk - cached) * kBlockTokens;      // node
    const int left = tail ? past - full * kBlockTokens : nnew - first;
    const int n_rows = left < kBlockTokens ? left : kBlockTokens;
    const RQ_GLOBAL uint16_t* kt = gptr(a.c.tail) + (size_t)unit * 2 * kBlockTokens * D;
    const RQ_GLOBAL uint16_t* vt = kt + kBlockTokens * D;
    const int64_t kst = tail ? D : a.k.st, vst = tail ? D : a.v.st;
    kt = tail ? kt : node_row(a.k, b, h, first);
    vt = tail ? vt : node_row(a.v, b, h, first);
    const RQ_GLOBAL uint16_t* kp = kt + (col < n_rows ? col : n_rows - 1) * kst + 16 * hl;
    // channels kE col + 2 e, + 1 of the lane's token i
    auto load_two = [&](int i, int e) {
      const int t = 8 * (i >> 2) + 4 * hl + (i & 3);
      const uint32_t x = *(const RQ_GLOBAL u1_any*)(vt + (t < n_rows ? t : n_rows - 1) * vst + kE * col + 2 * e);
      return t < n_rows ? x : 0u;
    };
    u4 kr[kK];
#pragma unroll
    for (int k = 0; k < kK; ++k) kr[k] = *(const RQ_GLOBAL u4_any*)(kp + 32 * (k >> 1) + 8 * (k & 1));
    // (with two tiles the values are loaded again where they are used: their
    // registers would not fit beside the probabilities')
    uint32_t vr[RT == 1 ? 16 : 1][kE / 2];
    if constexpr (RT == 1)
#pragma unroll
      for (int i = 0; i < 16; ++i)
#pragma unroll
        for (int e = 0; e < kE / 2; ++e) vr[i][e] = load_two(i, e);
    auto two = [&](int i, int e) {
      if constexpr (RT == 1)
        return vr[i][e];
      else
        return load_two(i, e);
    };
    uint32_t seen[RT];
#pragma unroll
    for (int n = 0; n < RT; ++n)
      seen[n] = tail ? (1u << n_rows) - 1u : node_mask(a, b, token[n], blk - cached, nnew);
    int at = 0;
    if (far) {
      const int t = col < n_rows ? col : n_rows - 1;
      at = tail ? pos[full * kBlockTokens + t] : base + node_depth(a, b, first + t);
    }
    int ke = 0, ve = 0;
    float kscale = 1.0f, vscale = kValueUnit<FMT>;
    if constexpr (BF16) {
      us2 km = {0, 0}, vm = {0, 0};        // (magnitudes compare as whole numbers)
#pragma unroll
      for (int k = 0; k < kK; ++k)
#pragma unroll
        for (int i = 0; i < 4; ++i) km = __builtin_elementwise_max(km, __builtin_bit_cast(us2, kr[k][i] & 0x7fff7fffu));
#pragma unroll
      for (int i = 0; i < 16; ++i)
#pragma unroll
        for (int e = 0; e < kE / 2; ++e) vm = __builtin_elementwise_max(vm, __builtin_bit_cast(us2, two(i, e) & 0x7fff7fffu));
      const float kmost = wave_all<Max>(widen_t<true>(km.x > km.y ? km.x : km.y));
      const float vmost = wave_all<Max>(widen_t<true>(vm.x > vm.y ? vm.x : vm.y));
      ke = kmost > 0.0f ? __builtin_amdgcn_frexp_expf(kmost) : 0;
      ve = vmost > 0.0f ? __builtin_amdgcn_frexp_expf(vmost) : 0;
      kscale = __builtin_amdgcn_ldexpf(1.0f, ke);
      vscale = vmost > 0.0f ? __builtin_amdgcn_ldexpf(kValueUnit<FMT>, ve) : 0.0f;
    }
    f16v s[RT];
    products([&](int k) {
      if constexpr (BF16) {
        u4 f;
#pragma unroll
        for (int i = 0; i < 4; ++i) f[i] = halves(kr[k][i] & 0xffffu, kr[k][i] >> 16, ke);
        return as_h8(f);
      } else {
        return as_h8(kr[k]);
      }
    }, s);
    attend(s, kscale, vscale, true, seen, at, [] {}, [&](int j, uint32_t op[4]) {
#pragma unroll
      for (int e = 0; e < kE / 2; ++e) {
        const uint32_t x = two(2 * j, e), y = two(2 * j + 1, e);
        if constexpr (BF16) {
          op[2 * e] = halves(x & 0xffffu, y & 0xffffu, ve);
          op[2 * e + 1] = halves(x >> 16, y >> 16, ve);
        } else {
          op[2 * e] = __builtin_amdgcn_perm(y, x, 0x05040100u);
          op[2 * e + 1] = __builtin_amdgcn_perm(y, x, 0x07060302u);
        }
      }
    });
  }

  // the waves' sums: half of the waves store theirs, the others add
#pragma unroll
  for (int n = 0; n < RT; ++n) {
    const float l = half_all<Sum>(st.l[n]);
    if (hl == 0) {
      sh_m[wave][32 * n + col] = st.m[n];
      sh_l[wave][32 * n + col] = l;
    }
  }
  __syncthreads();                         // (and nobody reads the queries any more)
  const float to_value = st.unit == 0.0f ? 0.0f : 1.0f / (st.unit * kValueUnit<FMT>);
  float factor[RT];
#pragma unroll
  for (int n = 0; n < RT; ++n) {
    float m = sh_m[0][32 * n + col];
#pragma unroll
    for (int i = 1; i < kWaves; ++i) m = __builtin_fmaxf(m, sh_m[i][32 * n + col]);
    factor[n] = exp2_f(st.m[n] - m) * to_value;
  }
  float* mine = sh_o[wave % kBufs] + col * kStride + kE * 4 * hl;
  auto each_piece = [&](auto f) {
#pragma unroll
    for (int n = 0; n < RT; ++n)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        float x[kE];
#pragma unroll
        for (int e = 0; e < kE; ++e) x[e] = st.o[n][e][i] * factor[n];
        f(mine + 32 * n * kStride + kE * (8 * (i >> 2) + (i & 3)), x);
      }
  };
  typedef float piece __attribute__((ext_vector_type(kE)));
  auto in_one = [](const float* x) {
    piece y;
#pragma unroll
    for (int e = 0; e < kE; ++e) y[e] = x[e];
    return y;
  };
  if (wave < kBufs) each_piece([&](float* p, const float* x) { *(piece*)p = in_one(x); });
  __syncthreads();
  if (wave >= kBufs) {
    each_piece([&](float* p, const float* x) { *(piece*)p += in_one(x); });
  } else if (wave < RT && hl == 0) {       // (nobody else reads these until all are added)
    const int r = 32 * wave + col;
    float m = sh_m[0][r], l = 0.0f;
#pragma unroll
    for (int j = 1; j < kWaves; ++j) m = __builtin_fmaxf(m, sh_m[j][r]);
#pragma unroll
    for (int j = 0; j < kWaves; ++j) l = __builtin_fmaf(sh_l[j][r], exp2_f(sh_m[j][r] - m), l);
    sh_m[0][r] = m;
    sh_l[0][r] = l;
  }
  __syncthreads();
  for (int i = threadIdx.x; i < kRows * (D / 4); i += kThreads) {
    const int r = i / (D / 4), ch = 4 * (i % (D / 4)), row = row0 + r;
    const int tok = over(row, a.by_G);
    if (tok >= nnew) continue;
    const float m = sh_m[0][r], l = sh_l[0][r];
    f4 x = *(const f4*)&sh_o[0][r * kStride + ch];
#pragma unroll
    for (int j = 1; j < kBufs; ++j) x += *(const f4*)&sh_o[j][r * kStride + ch];
    if (a.splits > 1) {
      const size_t at = (((size_t)unit * a.row_tiles + (row >> 4)) * a.splits + split) * 16 + (row & 15);
      *(RQ_GLOBAL f4*)(gptr(a.part) + at * D + ch) = x;
      if (ch == 0) *(RQ_GLOBAL f2*)(gptr(a.part_ml) + at * 2) = (f2){m, l};
    } else {
      x *= l > 0.0f ? 1.0f / l : 0.0f;
      store_out<4>(a, b, h * a.G + row - tok * a.G, tok, ch, (const float*)&x);
    }
  }
}

template <int FMT, int D, bool BF16, int RT, int kWaves>
hipError_t launch(const BlockTreeLaunch& a, hipStream_t s) {
  const dim3 grid((unsigned)((a.n * a.G + 32 * RT - 1) / (32 * RT) * a.splits) * a.c.B * a.c.H), block(64 * kWaves);
  if (a.plain)
    hipLaunchKernelGGL((tree_rows_kernel<FMT, D, BF16, RT, kWaves, true>), grid, block, 0, s, a);
  else if constexpr (D == 64 || RT == 1)
    hipLaunchKernelGGL((tree_rows_kernel<FMT, D, BF16, RT, kWaves, false>), grid, block, 0, s, a);
  else
    return hipErrorInvalidValue;           // (no plan asks for it)
  return hipGetLastError();
}

template <int FMT, int D, bool BF16>
hipError_t launch(const BlockTreeLaunch& a, hipStream_t s) {
  if (a.group_rows == 32) return a.waves == 4 ? launch<FMT, D, BF16, 1, 4>(a, s) : launch<FMT, D, BF16, 1, 8>(a, s);
  return a.waves == 4 ? launch<FMT, D, BF16, 2, 4>(a, s) : launch<FMT, D, BF16, 2, 8>(a, s);
}

template <int FMT, int D>
hipError_t launch(const BlockTreeLaunch& a, hipStream_t s) {
  const hipError_t e = a.c.is_bf16 ? launch<FMT, D, true>(a, s) : launch<FMT, D, false>(a, s);
  return e != hipSuccess ? e : launch_block_merge(a, s);
}

}  // namespace

hipError_t launch_tree_rows(const BlockTreeLaunch& a, hipStream_t s) {
  if (a.c.fmt == RQ_INT8) return a.c.D == 64 ? launch<RQ_INT8, 64>(a, s) : launch<RQ_INT8, 128>(a, s);
  return a.c.D == 64 ? launch<RQ_E4M3, 64>(a, s) : launch<RQ_E4M3, 128>(a, s);
}

}  // namespace rq
