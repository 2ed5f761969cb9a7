// Eviction from the block-scaled 8-bit cache by accumulated attention weight:
// of a unit's L tokens the first n_sink, the last n_recent and the heaviest of
// the rest stay (ties: the lowest slot), in order, and are quantized again in
// blocks of the new cache.
//
// Selection: the last weight that stays, by radix; then one ordered pass writes
// the kept slots.  The copy reads 2 D bytes a kept token and side and writes as many.
#include "rq_block.h"

namespace rq {

namespace {

constexpr int kSelThreads = 1024, kSelWaves = kSelThreads / 64;
constexpr int kBins = 2048;
// A wave's lanes would add to one counter one after the other where the
// weights share their leading digits: each counter is held four times, a lane's
// by its number (128 units of 8192 tokens with sixteen copies 2.6 us more, to
// clear and to add up).
constexpr int kCopies = 4;

constexpr int kFew = 256;     // keys that are ranked one against the other

struct SelectShared {
  __align__(16) uint32_t hist[kBins * kCopies];
  __align__(16) uint32_t few[kFew];
  uint32_t sum[kSelWaves], tie[kSelWaves];
  uint32_t pick[3], n_few;
};

// Where the search stands: the last key that stays is among the `span` keys
// from `lo` on, the need-th largest of the `in` of them that occur.
struct Found {
  uint32_t lo, span, need, in;
};

template <int CTRL, int ROWS = 0xf>
__device__ __forceinline__ uint32_t lane_move(uint32_t x) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, ROWS, 0xf, false);
}

// Sums over the lanes up to this one (moves within rows of 16 lanes, then of
// the rows' last lanes).
__device__ __forceinline__ uint32_t wave_scan(uint32_t x) {
  x += lane_move<0x111>(x);
  x += lane_move<0x112>(x);
  x += lane_move<0x114>(x);
  x += lane_move<0x118>(x);
  x += lane_move<0x142, 0xa>(x);
  return x + lane_move<0x143, 0xc>(x);
}
__device__ __forceinline__ uint32_t last_lane(uint32_t x) { return __builtin_amdgcn_readlane(x, 63); }

// Of one number a wave: the sum over the waves before `end`.
__device__ __forceinline__ uint32_t sum_before(const uint32_t x[kSelWaves], int end) {
  static_assert(kSelWaves == 16, "a row of lanes");
  const int i = threadIdx.x & 15;
  uint32_t v = x[i];
  v = i < end ? v : 0u;
  v += lane_move<0x128>(v);
  v += lane_move<0x124>(v);
  v += lane_move<0x122>(v);
  v += lane_move<0x121>(v);
  return __builtin_amdgcn_readfirstlane(v);
}
__device__ __forceinline__ int wave_index() { return __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6); }

// A weight's place in the order, as an unsigned number above 0; the tokens that
// stay in any case are above all others.
__device__ __forceinline__ uint32_t rank_key(float w, int slot, int L, int sink, int recent) {
  if (slot >= L) return 0u;
  if (slot < sink || slot >= L - recent) return 0xffffffffu;
  const uint32_t u = __float_as_uint(w + 0.0f);     // -0 becomes 0
  const uint32_t key = (int32_t)u < 0 ? ~u : u | 0x80000000u;
  return key < 1u ? 1u : (key > 0xfffffffeu ? 0xfffffffeu : key);
}

// Weights of N x 4 tokens a lane.  A wave's tokens follow each other from `base`
// on: group i of a lane is base + 256 i + 4 lane.  (w is 16-byte aligned, and
// its rows hold a multiple of 32.)
template <int N>
__device__ __forceinline__ void load_weights(const RQ_GLOBAL float* w, int base, int end, f4 x[N]) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int t = base + 256 * i + 4 * lane;
    x[i] = t < end ? *(const RQ_GLOBAL f4*)(w + t) : (f4){0.0f, 0.0f, 0.0f, 0.0f};
  }
}

template <int N>
__device__ __forceinline__ void rank_keys(const BlockEvictLaunch& a, const f4 x[N], int base, int L,
                                          uint32_t key[4 * N]) {
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j)
      key[4 * i + j] = rank_key(x[i][j], base + 256 * i + 4 * ((int)threadIdx.x & 63) + j, L, a.n_sink, a.n_recent);
}

// The first digit: weights from 2^-24 to 2^8 in 32 steps an octave (2^18 keys),
// all others in steps of 2^22 keys.  Two digits of 11 bits then end the search.
constexpr uint32_t kFineFrom = 0xb3800000u, kFineTo = 0xc3800000u;
constexpr uint32_t kFineAt = kFineFrom >> 22, kHighAt = kFineAt + ((kFineTo - kFineFrom) >> 18);
static_assert(kHighAt + ((0xffffffffu - kFineTo) >> 22) < kBins, "first digits");

__device__ __forceinline__ uint32_t first_digit(uint32_t key) {
  if (key < kFineFrom) return key >> 22;
  return key < kFineTo ? kFineAt + ((key - kFineFrom) >> 18) : kHighAt + ((key - kFineTo) >> 22);
}

// The keys of a first digit (without 0 and those that stay in any case).
__device__ __forceinline__ void first_range(uint32_t d, uint32_t* lo, uint32_t* span) {
  const bool fine = d >= kFineAt && d < kHighAt;
  *lo = d < kFineAt ? d << 22 : (fine ? kFineFrom + ((d - kFineAt) << 18) : kFineTo + ((d - kHighAt) << 22));
  *span = 1u << (fine ? 18 : 22);
  if (d == 0) {
    *lo += 1;
    *span -= 1;
  }
  if (*span > 0xffffffffu - *lo) *span = 0xffffffffu - *lo;
}

// Later digits: the distance from f.lo, its 11 leading bits.
__device__ __forceinline__ int digit_shift(const Found& f) {
  const int bits = 32 - __builtin_clz((f.span - 1) | 1u);
  return bits > 11 ? bits - 11 : 0;
}

template <int N>
__device__ __forceinline__ void count_digits(SelectShared& sh, const uint32_t key[4 * N], int level,
                                             const Found& f) {
  const int shift = level == 0 ? 0 : digit_shift(f), copy = threadIdx.x & (kCopies - 1);
#pragma unroll
  for (int i = 0; i < 4 * N; ++i) {
    const uint32_t from = key[i] - f.lo;
    if (from < f.span)
      atomicAdd(&sh.hist[(level == 0 ? first_digit(key[i]) : from >> shift) * kCopies + copy], 1u);
  }
}

__device__ __forceinline__ void clear_digits(SelectShared& sh) {
#pragma unroll
  for (int i = 0; i < kBins * kCopies; i += 4 * kSelThreads) *(u4*)&sh.hist[i + 4 * threadIdx.x] = (u4){0u, 0u, 0u, 0u};
  if (threadIdx.x < kFew) sh.few[threadIdx.x] = 0;
  if (threadIdx.x == 0) sh.n_few = 0;
  __syncthreads();
}

// This thread's two counters: those of digits top_digit() and the one below.
__device__ __forceinline__ int top_digit() { return kBins - 1 - 2 * (int)threadIdx.x; }
__device__ __forceinline__ void read_digits(const SelectShared& sh, uint32_t* c1, uint32_t* c2) {
  static_assert(kCopies == 4, "one load a digit");
  const u4 x = *(const u4*)&sh.hist[top_digit() * kCopies], y = *(const u4*)&sh.hist[(top_digit() - 1) * kCopies];
  *c1 = (x.x + x.y) + (x.z + x.w);
  *c2 = (y.x + y.y) + (y.z + y.w);
}

// Narrows f to the digit d with (keys above d) < need <= (keys from d on);
// returns d.
__device__ __forceinline__ uint32_t pick_digit(SelectShared& sh, uint32_t c1, uint32_t c2, int level,
                                               Found* f) {
  const int lane = threadIdx.x & 63, wave = wave_index();
  const uint32_t mine = c1 + c2, x = wave_scan(mine);
  if (lane == 63) sh.sum[wave] = x;
  __syncthreads();
  const uint32_t above = x - mine + sum_before(sh.sum, wave);
  if (above < f->need && f->need <= above + mine) {
    const bool first = f->need <= above + c1;
    sh.pick[0] = top_digit() - (first ? 0 : 1);
    sh.pick[1] = first ? above : above + c1;
    sh.pick[2] = first ? c1 : c2;
  }
  __syncthreads();
  const uint32_t d = __builtin_amdgcn_readfirstlane(sh.pick[0]);
  f->need -= __builtin_amdgcn_readfirstlane(sh.pick[1]);
  f->in = __builtin_amdgcn_readfirstlane(sh.pick[2]);
  if (level == 0) {
    first_range(d, &f->lo, &f->span);
  } else {
    const int shift = digit_shift(*f);
    f->lo += d << shift;
    f->span -= d << shift;
    if (f->span > 1u << shift) f->span = 1u << shift;
  }
  __syncthreads();
  return d;
}

// Where every key of f stays there is no need to look closer: f becomes the
// key below them all, of which none does.
__device__ __forceinline__ bool settle(Found* f) {
  if (f->need != f->in) return false;
  f->lo -= 1;
  f->span = 1;
  f->need = 0;
  return true;
}

// Few keys left: each is ranked among them.
template <int N>
__device__ __forceinline__ void rank_few(SelectShared& sh, const uint32_t key[4 * N], Found* f) {
#pragma unroll
  for (int i = 0; i < 4 * N; ++i)
    if (key[i] - f->lo < f->span) sh.few[atomicAdd(&sh.n_few, 1u)] = key[i];
  __syncthreads();
  // four threads a key, each with every fourth four of the list (0: no key)
  static_assert(4 * kFew == kSelThreads, "four threads a key");
  if (wave_index() * 16u < f->in) {
    const uint32_t mine = sh.few[threadIdx.x >> 2];
    uint32_t rank = 0;                      // keys above; equal ones 16 bits higher
    for (uint32_t i = 0; i < f->in; i += 16) {
      const u4 x = *(const u4*)&sh.few[i + 4 * (threadIdx.x & 3)];
#pragma unroll
      for (int j = 0; j < 4; ++j) rank += x[j] > mine ? 1u : (x[j] == mine ? 0x10000u : 0u);
    }
    rank += lane_move<0xb1>(rank);          // (the other pair's, then of the other two)
    rank += lane_move<0x4e>(rank);
    const uint32_t above = rank & 0xffffu, equal = rank >> 16;
    if (mine && above < f->need && f->need <= above + equal) {      // (equal keys write the same)
      sh.pick[0] = mine;
      sh.pick[1] = above;
      sh.pick[2] = equal;
    }
  }
  __syncthreads();
  f->lo = __builtin_amdgcn_readfirstlane(sh.pick[0]);
  f->span = 1;
  f->need -= __builtin_amdgcn_readfirstlane(sh.pick[1]);
  f->in = __builtin_amdgcn_readfirstlane(sh.pick[2]);
  __syncthreads();
  settle(f);
}

// Writes the slots that stay: keys above f.lo, and of those equal to it the
// first f.need.  *kept, *ties: such keys before this workgroup's tokens; then
// before the next one's.
template <int N>
__device__ __forceinline__ void write_slots(SelectShared& sh, const uint32_t key[4 * N], int base,
                                            const Found& f, RQ_GLOBAL int32_t* out, uint32_t* kept,
                                            uint32_t* ties) {
  const int lane = threadIdx.x & 63, wave = wave_index();
  // keys above, and equal ones 16 bits higher: of this lane's four of a group,
  // then of all lanes up to it
  uint32_t mine[N], upto[N], all = 0;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    mine[i] = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) mine[i] += key[4 * i + j] > f.lo;
    if (f.need > 0)
#pragma unroll
      for (int j = 0; j < 4; ++j) mine[i] += key[4 * i + j] == f.lo ? 0x10000u : 0u;
    upto[i] = wave_scan(mine[i]);
    all += last_lane(upto[i]);
  }
  if (lane == 0) {
    sh.sum[wave] = all & 0xffffu;
    sh.tie[wave] = all >> 16;
  }
  __syncthreads();
  uint32_t g = *kept + sum_before(sh.sum, wave), e = *ties + sum_before(sh.tie, wave);
  *kept += sum_before(sh.sum, kSelWaves);
  *ties += sum_before(sh.tie, kSelWaves);
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const uint32_t ahead = upto[i] - mine[i], group = last_lane(upto[i]);
    uint32_t gl = g + (ahead & 0xffffu), el = e + (ahead >> 16);
    g += group & 0xffffu;
    e += group >> 16;
    if (f.need == 0) {                    // no ties
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (key[4 * i + j] > f.lo) out[gl++] = base + 256 * i + 4 * lane + j;
      continue;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const bool gt = key[4 * i + j] > f.lo, eq = key[4 * i + j] == f.lo;
      if (gt || (eq && el < f.need))
        out[gl + (el < f.need ? el : f.need)] = base + 256 * i + 4 * lane + j;
      gl += gt;
      el += eq;
    }
  }
  __syncthreads();
}

__device__ __forceinline__ int kept_length(const BlockEvictLaunch& a, int b, int* k) {
  int L = gptr(a.lengths)[b];
  L = L < 0 ? 0 : (L > a.src.cap ? a.src.cap : L);
  L = __builtin_amdgcn_readfirstlane(L);
  *k = L < a.keep ? L : a.keep;
  return L;
}

// The search's start: all keys but 0 and those that stay in any case.
__device__ __forceinline__ Found all_keys(const BlockEvictLaunch& a) {
  return {1u, 0xfffffffeu, (uint32_t)(a.keep - a.n_sink - a.n_recent), 0u};
}

// A unit by one workgroup, its keys in registers, N x 4 a thread.  (128 units of
// 8192 tokens: 7.8 us a workgroup, of which 1.6 wait for the weights, 2 count
// and find the first digit, 1.6 rank what is left, 1.5 write; with digits of
// the number itself, three rounds, 13.)
template <int N>
__global__ void __launch_bounds__(kSelThreads) block_select_kernel(BlockEvictLaunch a) {
  __shared__ SelectShared sh;
  const int unit = blockIdx.x, b = over(unit, a.src.by_H), tid = threadIdx.x;
  const int base = (tid >> 6) * N * 256;
  f4 x[N];                // (on their way while the length is)
  load_weights<N>(gptr(a.src.weights) + (size_t)unit * a.src.cap, base, a.src.cap, x);
  int k;
  const int L = kept_length(a, b, &k);
  if (tid == 0 && unit == b * a.src.H) gptr(a.new_lengths)[b] = k;
  RQ_GLOBAL int32_t* out = gptr(a.slots) + (size_t)unit * a.keep;
  if (L <= a.keep) {
    for (int t = tid; t < L; t += kSelThreads) out[t] = t;
    return;
  }
  uint32_t key[4 * N];
  Found f = all_keys(a);
  if (f.need == 0) {
    rank_keys<N>(a, x, base, L, key);
    f.lo = 0xfffffffeu;
  }
  for (int level = 0; f.need > 0 && level < 3; ++level) {
    clear_digits(sh);
    if (level == 0) rank_keys<N>(a, x, base, L, key);
    count_digits<N>(sh, key, level, f);
    __syncthreads();
    uint32_t c1, c2;
    read_digits(sh, &c1, &c2);
    pick_digit(sh, c1, c2, level, &f);
    if (f.span == 1 || settle(&f)) break;
    if (f.in <= kFew) {
      rank_few<N>(sh, key, &f);
      break;
    }
  }
  uint32_t kept = 0, ties = 0;
  write_slots<N>(sh, key, base, f, out, &kept, &ties);
}

// Longer units: a workgroup for every part of a.part tokens, and a launch for
// each digit.  Launch `level` finds the digit before from the parts' counters
// of the launch before, and counts its own; once the digits settle the choice
// (or at level 3) it writes the slots instead, and later launches have nothing
// to do.  A part's place in the output, the keys above the k-th in the parts
// before, is added up on the way.  (Eight units of 131072 tokens in sixteen
// parts: 23 us from the first launch to the fourth.)
__global__ void __launch_bounds__(kSelThreads) block_select_part_kernel(BlockEvictLaunch a, int level) {
  constexpr int N = 2, kTile = 4 * N * kSelThreads;
  __shared__ SelectShared sh;
  const int part = blockIdx.x, unit = blockIdx.y, b = over(unit, a.src.by_H), tid = threadIdx.x;
  const int first = part * a.part, base = (tid >> 6) * N * 256;
  const RQ_GLOBAL float* w = gptr(a.src.weights) + (size_t)unit * a.src.cap;
  f4 x[N];                // (on their way while the counters are)
  load_weights<N>(w, first + base, a.src.cap, x);
  int k;
  const int L = kept_length(a, b, &k);
  const int last = first + a.part < L ? first + a.part : L;
  RQ_GLOBAL int32_t* out = gptr(a.slots) + (size_t)unit * a.keep;
  if (L <= a.keep) {
    if (level == 0) {
      for (int t = first + tid; t < last; t += kSelThreads) out[t] = t;
      if (part == 0 && tid == 0 && unit == b * a.src.H) gptr(a.new_lengths)[b] = k;
    }
    return;
  }
  const size_t side = (size_t)a.src.B * a.src.H * a.parts * kBins;     // one level's counters
  RQ_GLOBAL uint32_t* count = gptr(a.counts) + (size_t)unit * a.parts * kBins;
  RQ_GLOBAL uint32_t* state = gptr(a.state) + (size_t)unit * kSelectState;
  RQ_GLOBAL uint32_t* before = gptr(a.before) + (size_t)unit * a.parts;
  Found f = all_keys(a);
  uint32_t kept = 0, ties = 0;
  bool write = level == 3;
  if (level > 0) {
    if (level > 1) {
      f.lo = state[3 * (level - 2)];
      f.span = state[3 * (level - 2) + 1];
      f.need = state[3 * (level - 2) + 2];
      if (f.need == 0) {                    // settled: the launch before wrote
        if (level == 2 && part == 0 && tid == 0) state[3 * (level - 1) + 2] = 0;
        return;
      }
      kept = before[part];
    } else {
      // the first and last tokens stay in any case
      const int from = L - a.n_recent;
      kept = (first < a.n_sink ? first : a.n_sink) + (first > from ? first - from : 0);
    }
    // (counters lie in falling order of their digits, a thread's two together)
    const int in_use = (L + a.part - 1) / a.part;
    const RQ_GLOBAL u2* c = (const RQ_GLOBAL u2*)(count + side * (level - 1)) + tid;
    u2 all = {0u, 0u}, ahead = {0u, 0u};
    for (int i0 = 0; i0 < in_use; i0 += 16) {
      u2 x[16];
#pragma unroll
      for (int i = 0; i < 16; ++i)
        x[i] = i0 + i < in_use ? c[(size_t)(i0 + i) * (kBins / 2)] : (u2){0u, 0u};
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        all += x[i];
        if (i0 + i < part) ahead += x[i];
      }
    }
    uint32_t g = 0, e = 0;
    if (f.need == 0) {                      // (level 1: nothing to choose)
      f.lo = 0xfffffffeu;
      write = true;
    } else {
      const uint32_t d = pick_digit(sh, all.x, all.y, level - 1, &f);
      const uint32_t hi = top_digit();
      g = (hi > d ? ahead.x : 0u) + (hi - 1 > d ? ahead.y : 0u);
      e = (hi == d ? ahead.x : 0u) + (hi - 1 == d ? ahead.y : 0u);
    }
    if (!write && settle(&f)) {
      write = true;
      g += e;                               // (none is a tie any more)
      e = 0;
    }
    g = last_lane(wave_scan(g));
    e = last_lane(wave_scan(e));
    if ((tid & 63) == 0) {
      sh.sum[wave_index()] = g;
      sh.tie[wave_index()] = e;
    }
    __syncthreads();
    kept += sum_before(sh.sum, kSelWaves);
    ties += sum_before(sh.tie, kSelWaves);
    __syncthreads();
    if (tid == 0) {
      if (part == 0) {
        state[3 * (level - 1)] = f.lo;
        state[3 * (level - 1) + 1] = f.span;
        state[3 * (level - 1) + 2] = f.need;
      }
      before[part] = kept;
    }
  } else if (part == 0 && tid == 0 && unit == b * a.src.H) {
    gptr(a.new_lengths)[b] = k;
  }
  if (first >= L) return;
  if (!write) clear_digits(sh);
  for (int at = first; at < last; at += kTile) {
    uint32_t key[4 * N];
    rank_keys<N>(a, x, at + base, L, key);
    if (at + kTile < last) load_weights<N>(w, at + kTile + base, L, x);
    if (write)
      write_slots<N>(sh, key, at + base, f, out, &kept, &ties);
    else
      count_digits<N>(sh, key, level, f);
  }
  if (write) return;
  __syncthreads();
  u2 c;
  uint32_t c1, c2;
  read_digits(sh, &c1, &c2);
  c.x = c1;
  c.y = c2;
  ((RQ_GLOBAL u2*)(count + side * level + (size_t)part * kBins))[tid] = c;
}

// One wave a (unit, K or V, block of the new cache).  128 units to 2048 tokens
// (137 MB): 26 us, the rate of a copy.
template <int FMT, int D, bool BF16>
__global__ void __launch_bounds__(256) block_gather_kernel(BlockEvictLaunch a) {
  constexpr int kChunks = D / 8, kRows = 64 / kChunks, kLoads = kBlockTokens / kRows;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int unit = blockIdx.y >> 1, kind = blockIdx.y & 1, b = over(unit, a.src.by_H);
  int L = gptr(a.lengths)[b];
  L = L < 0 ? 0 : (L > a.src.cap ? a.src.cap : L);
  const int k = L < a.keep ? L : a.keep;
  const int blk = blockIdx.x * 4 + wave;
  if (blk * kBlockTokens >= k) return;
  const int n_coded = L / kBlockTokens * kBlockTokens;
  const RQ_GLOBAL int32_t* slots = gptr(a.slots) + (size_t)unit * a.keep + blk * kBlockTokens;
  const int rows = k - blk * kBlockTokens < kBlockTokens ? k - blk * kBlockTokens : kBlockTokens;
  const size_t side = (size_t)unit * 2 + kind;
  const RQ_GLOBAL uint8_t* codes = gptr(a.src.codes) + side * a.src.cap * D;
  const RQ_GLOBAL float* scales = gptr(a.src.scales) + side * (a.src.cap / kBlockTokens);
  const RQ_GLOBAL uint16_t* tail = gptr(a.src.tail) + side * kBlockTokens * D;
  const int row0 = lane / kChunks, ch = (lane % kChunks) * 8;
  if (rows == kBlockTokens && slots[kBlockTokens - 1] < n_coded) {
    // 32 coded rows: the codes are held, their values formed twice
    u2 raw[kLoads];
    float by[kLoads];
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int slot = slots[row0 + kRows * i];
      raw[i] = __builtin_nontemporal_load((const RQ_GLOBAL u2*)(codes + (size_t)slot * D + ch));
      by[i] = scales[slot / kBlockTokens];
    }
    float most = 0.0f;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      // (the largest product is the largest code's: rounding is monotonic)
      float top = 0.0f;
#pragma unroll
      for (int e = 0; e < 8; ++e)
        top = __builtin_fmaxf(top, __builtin_fabsf(block_value<FMT>(raw[i][e >> 2], e & 3)));
      most = __builtin_fmaxf(most, top * by[i]);
      asm volatile("" : "+v"(raw[i]));      // not the same values for both uses
    }
    most = wave_all<Max>(most);
    float inv;
    const float scale = block_scale<FMT>(most, &inv);
    RQ_GLOBAL uint8_t* out = gptr(a.dst.codes) + (side * a.dst.cap + (size_t)blk * kBlockTokens) * D;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      float x[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = block_value<FMT>(raw[i][e >> 2], e & 3) * by[i];
      u2 w;
#pragma unroll
      for (int p = 0; p < 2; ++p)
        w[p] = block_codes<FMT>(x[4 * p], x[4 * p + 1], x[4 * p + 2], x[4 * p + 3], inv);
      *(RQ_GLOBAL u2*)(out + (row0 + kRows * i) * D + ch) = w;
    }
    if (lane == 0) gptr(a.dst.scales)[side * (a.dst.cap / kBlockTokens) + blk] = scale;
  } else {
    // a block that takes rows of the source's tail, or the unfinished one
    // (one or two a unit): row by row, read twice
    auto values = [&](int row, float x[8]) {
      const int slot = slots[row];
      if (slot < n_coded) {
        const u2 w = *(const RQ_GLOBAL u2*)(codes + (size_t)slot * D + ch);
        const float by = scales[slot / kBlockTokens];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = block_value<FMT>(w[e >> 2], e & 3) * by;
      } else {
        const u4 w = *(const RQ_GLOBAL u4*)(tail + (slot - n_coded) * D + ch);
#pragma unroll
        for (int e = 0; e < 8; ++e)
          x[e] = widen_t<BF16>(e & 1 ? w[e >> 1] >> 16 : w[e >> 1] & 0xffffu);
      }
    };
    const bool whole = rows == kBlockTokens;
    float most = 0.0f, inv = 0.0f;
    if (whole) {
#pragma unroll 1
      for (int row = row0; row < rows; row += kRows) {
        float x[8];
        values(row, x);
#pragma unroll
        for (int e = 0; e < 8; ++e) most = __builtin_fmaxf(most, __builtin_fabsf(x[e]));
      }
      most = wave_all<Max>(most);
      const float scale = block_scale<FMT>(most, &inv);
      if (lane == 0) gptr(a.dst.scales)[side * (a.dst.cap / kBlockTokens) + blk] = scale;
    }
    RQ_GLOBAL uint8_t* out = gptr(a.dst.codes) + (side * a.dst.cap + (size_t)blk * kBlockTokens) * D;
    RQ_GLOBAL uint16_t* rest = gptr(a.dst.tail) + side * kBlockTokens * D;
#pragma unroll 1
    for (int row = row0; row < rows; row += kRows) {
      float x[8];
      values(row, x);
      if (whole) {
        u2 w;
#pragma unroll
        for (int p = 0; p < 2; ++p)
          w[p] = block_codes<FMT>(x[4 * p], x[4 * p + 1], x[4 * p + 2], x[4 * p + 3], inv);
        *(RQ_GLOBAL u2*)(out + row * D + ch) = w;
      } else {
        u4 w;
#pragma unroll
        for (int e = 0; e < 4; ++e)
          w[e] = narrow_t<BF16>(x[2 * e]) | ((uint32_t)narrow_t<BF16>(x[2 * e + 1]) << 16);
        *(RQ_GLOBAL u4*)(rest + row * D + ch) = w;
      }
    }
  }
  if (kind == 0 && lane < rows) {
    const int to = blk * kBlockTokens + lane, slot = slots[lane];
    gptr(a.dst.positions)[(size_t)unit * a.dst.cap + to] =
        gptr(a.src.positions)[(size_t)unit * a.src.cap + slot];
    if (a.dst.weights)
      gptr(a.dst.weights)[(size_t)unit * a.dst.cap + to] =
          gptr(a.src.weights)[(size_t)unit * a.src.cap + slot];
  }
}

template <int FMT, int D>
hipError_t launch_gather(const BlockEvictLaunch& a, hipStream_t s) {
  const dim3 grid((a.keep + 4 * kBlockTokens - 1) / (4 * kBlockTokens), 2 * a.src.B * a.src.H);
  if (a.src.is_bf16)
    hipLaunchKernelGGL((block_gather_kernel<FMT, D, true>), grid, dim3(256), 0, s, a);
  else
    hipLaunchKernelGGL((block_gather_kernel<FMT, D, false>), grid, dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_block_evict(const BlockEvictLaunch& a, hipStream_t s) {
  const int units = a.src.B * a.src.H;
  if (a.parts == 1) {
    static_assert(kSelectShort == 32 * kSelThreads, "keys of a unit in one workgroup");
    if (a.src.cap <= 4 * kSelThreads)
      hipLaunchKernelGGL((block_select_kernel<1>), dim3(units), dim3(kSelThreads), 0, s, a);
    else if (a.src.cap <= 8 * kSelThreads)
      hipLaunchKernelGGL((block_select_kernel<2>), dim3(units), dim3(kSelThreads), 0, s, a);
    else if (a.src.cap <= 16 * kSelThreads)
      hipLaunchKernelGGL((block_select_kernel<4>), dim3(units), dim3(kSelThreads), 0, s, a);
    else
      hipLaunchKernelGGL((block_select_kernel<8>), dim3(units), dim3(kSelThreads), 0, s, a);
  } else {
    for (int level = 0; level < 4; ++level)
      hipLaunchKernelGGL(block_select_part_kernel, dim3(a.parts, units), dim3(kSelThreads), 0, s, a, level);
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  if (a.src.fmt == RQ_INT8)
    return a.src.D == 64 ? launch_gather<RQ_INT8, 64>(a, s) : launch_gather<RQ_INT8, 128>(a, s);
  return a.src.D == 64 ? launch_gather<RQ_E4M3, 64>(a, s) : launch_gather<RQ_E4M3, 128>(a, s);
}

}  // namespace rq
