// Eviction from the block-scaled 8-bit cache by accumulated attention weight:
// of a unit's L tokens the first n_sink, the last n_recent and the heaviest of
// the rest stay (ties: the lowest slot), in order, and are quantized again in
// blocks of the new cache.
//
// Selection: the k-th largest weight by radix, digits of 11, 11 and 10 bits;
// then one ordered pass writes the kept slots.  The copy reads 2 D bytes a kept token
// and side and writes as many.
#include "rq_block.h"

namespace rq {

namespace {

constexpr int kSelThreads = 1024, kSelWaves = kSelThreads / 64;
constexpr int kBins = 2048;
// A wave's lanes would add to one counter one after the other where the
// weights share their leading digits: each counter is held four times, a lane's
// by its number (128 units of 8192 tokens 15.7 us; sixteen times, with more to
// clear and to add up, 18.3).
constexpr int kCopies = 4;

struct SelectShared {
  uint32_t hist[kBins * kCopies];
  uint32_t sum[kSelWaves], tie[kSelWaves];
  uint32_t pick[3];
};

// Where the search stands: the leading digits of the k-th largest key, and how
// many of the keys with these digits stay.
struct Found {
  uint32_t prefix, need;
  uint32_t all;             // all of them do
};

// A weight's place in the order, as an unsigned number above 0; the tokens that
// stay in any case are above all others.
__device__ __forceinline__ uint32_t rank_key(float w, int slot, int L, int sink, int recent) {
  if (slot >= L) return 0u;
  if (slot < sink || slot >= L - recent) return 0xffffffffu;
  const uint32_t u = __float_as_uint(w + 0.0f);     // -0 becomes 0
  const uint32_t key = (int32_t)u < 0 ? ~u : u | 0x80000000u;
  return key < 1u ? 1u : (key > 0xfffffffeu ? 0xfffffffeu : key);
}

// Keys of N x 4 tokens a lane.  A wave's tokens follow each other from `base`
// on: group i of a lane is base + 256 i + 4 lane.  (w is 16-byte aligned, and
// its rows hold a multiple of 32.)
template <int N>
__device__ __forceinline__ void load_ranks(const BlockEvictLaunch& a, const RQ_GLOBAL float* w,
                                           int base, int L, uint32_t key[4 * N]) {
  const int lane = threadIdx.x & 63;
  f4 x[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int t = base + 256 * i + 4 * lane;
    x[i] = t < L ? *(const RQ_GLOBAL f4*)(w + t) : (f4){0.0f, 0.0f, 0.0f, 0.0f};
  }
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j)
      key[4 * i + j] = rank_key(x[i][j], base + 256 * i + 4 * lane + j, L, a.n_sink, a.n_recent);
}

// Digits of 11, 11 and 10 bits.
__device__ __forceinline__ int digit_shift(int level) { return level == 0 ? 21 : (level == 1 ? 10 : 0); }

template <int N>
__device__ __forceinline__ void count_digits(SelectShared& sh, const uint32_t key[4 * N], int level,
                                             uint32_t prefix) {
  const int shift = digit_shift(level), copy = threadIdx.x & (kCopies - 1);
  const uint32_t mask = level == 2 ? 1023u : 2047u;
#pragma unroll
  for (int i = 0; i < 4 * N; ++i) {
    const bool in = level == 0 || (level == 1 ? key[i] >> 21 : key[i] >> 10) == prefix;
    if (in && key[i]) atomicAdd(&sh.hist[((key[i] >> shift) & mask) * kCopies + copy], 1u);
  }
}

__device__ __forceinline__ void clear_digits(SelectShared& sh) {
  for (int i = threadIdx.x; i < kBins * kCopies; i += kSelThreads) sh.hist[i] = 0;
  __syncthreads();
}

// This thread's two counters: those of digits top_digit() and the one below.
__device__ __forceinline__ int top_digit() { return kBins - 1 - 2 * (int)threadIdx.x; }
__device__ __forceinline__ void read_digits(const SelectShared& sh, uint32_t* c1, uint32_t* c2) {
  *c1 = *c2 = 0;
#pragma unroll
  for (int i = 0; i < kCopies; ++i) {
    const int at = (i + threadIdx.x) & (kCopies - 1);
    *c1 += sh.hist[top_digit() * kCopies + at];
    *c2 += sh.hist[(top_digit() - 1) * kCopies + at];
  }
}

// Extends f by the digit d with (keys above d) < need <= (keys from d on);
// returns d.
__device__ __forceinline__ uint32_t pick_digit(SelectShared& sh, uint32_t c1, uint32_t c2, int level,
                                               Found* f) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const uint32_t mine = c1 + c2;
  uint32_t x = mine;
  for (int d = 1; d < 64; d <<= 1) {
    const uint32_t y = __shfl_up(x, d, 64);
    if (lane >= d) x += y;
  }
  if (lane == 63) sh.sum[wave] = x;
  __syncthreads();
  uint32_t above = x - mine;
  for (int i = 0; i < wave; ++i) above += sh.sum[i];
  if (above < f->need && f->need <= above + mine) {
    const bool first = f->need <= above + c1;
    sh.pick[0] = top_digit() - (first ? 0 : 1);
    sh.pick[1] = first ? above : above + c1;
    sh.pick[2] = f->need - sh.pick[1] == (first ? c1 : c2);
  }
  __syncthreads();
  const uint32_t d = sh.pick[0];
  f->prefix = level == 0 ? d : (f->prefix << (level == 1 ? 11 : 10)) | d;
  f->need -= sh.pick[1];
  f->all = sh.pick[2];
  __syncthreads();
  return d;
}

// Where every key from f's digits on stays there is no need to look closer: f
// becomes a bound below them all.
__device__ __forceinline__ bool settle(int level, Found* f) {
  if (!f->all) return false;
  const uint32_t from = f->prefix << digit_shift(level);
  f->prefix = from > 0 ? from - 1 : 0;
  f->need = 0;
  return true;
}

__device__ __forceinline__ uint32_t wave_sum(uint32_t x) {
  for (int d = 32; d >= 1; d >>= 1) x += __shfl_xor(x, d, 64);
  return x;
}

// Writes the slots that stay: keys above f.prefix, and of those equal to it the
// first f.need.  *kept, *ties: such keys before this workgroup's tokens; then
// before the next one's.
template <int N>
__device__ __forceinline__ void write_slots(SelectShared& sh, const uint32_t key[4 * N], int base,
                                            const Found& f, RQ_GLOBAL int32_t* out, uint32_t* kept,
                                            uint32_t* ties) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  uint32_t g = 0, e = 0;
#pragma unroll
  for (int i = 0; i < 4 * N; ++i) {
    g += key[i] > f.prefix;
    e += key[i] == f.prefix;
  }
  g = wave_sum(g);
  e = wave_sum(e);
  if (lane == 0) {
    sh.sum[wave] = g;
    sh.tie[wave] = e;
  }
  __syncthreads();
  g = *kept;
  e = *ties;
  for (int i = 0; i < kSelWaves; ++i) {
    if (i < wave) {
      g += sh.sum[i];
      e += sh.tie[i];
    }
    *kept += sh.sum[i];
    *ties += sh.tie[i];
  }
  const uint64_t below = (1ull << lane) - 1;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    uint32_t gl = g, el = e;               // before this lane's first token
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint64_t mg = __ballot(key[4 * i + j] > f.prefix);
      const uint64_t me = __ballot(key[4 * i + j] == f.prefix);
      gl += __popcll(mg & below);
      el += __popcll(me & below);
      g += __popcll(mg);
      e += __popcll(me);
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const bool gt = key[4 * i + j] > f.prefix, eq = key[4 * i + j] == f.prefix;
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

// A unit by one workgroup, its keys in registers, N x 4 a thread.
template <int N>
__global__ void __launch_bounds__(kSelThreads) block_select_kernel(BlockEvictLaunch a) {
  __shared__ SelectShared sh;
  const int unit = blockIdx.x, b = unit / a.src.H, tid = threadIdx.x;
  int k;
  const int L = kept_length(a, b, &k);
  if (tid == 0 && unit % a.src.H == 0) gptr(a.new_lengths)[b] = k;
  RQ_GLOBAL int32_t* out = gptr(a.slots) + (size_t)unit * a.keep;
  if (L <= a.keep) {
    for (int t = tid; t < L; t += kSelThreads) out[t] = t;
    return;
  }
  uint32_t key[4 * N];
  const int base = (tid >> 6) * N * 256;
  load_ranks<N>(a, gptr(a.src.weights) + (size_t)unit * a.src.cap, base, L, key);
  Found f = {0, (uint32_t)k, 0};
  for (int level = 0; level < 3; ++level) {
    clear_digits(sh);
    count_digits<N>(sh, key, level, f.prefix);
    __syncthreads();
    uint32_t c1, c2;
    read_digits(sh, &c1, &c2);
    pick_digit(sh, c1, c2, level, &f);
    if (level < 2 && settle(level, &f)) break;
  }
  uint32_t kept = 0, ties = 0;
  write_slots<N>(sh, key, base, f, out, &kept, &ties);
}

// Longer units: a workgroup for every part of a.part tokens, and a launch for
// each digit.  Launch `level` finds the digit before from the parts' counters
// of the launch before, and counts its own; once the digits settle the choice
// (or at level 3) it writes the slots instead, and later launches have nothing
// to do.  A part's place in the output, the keys above the k-th in the parts
// before, is added up on the way.
__global__ void __launch_bounds__(kSelThreads) block_select_part_kernel(BlockEvictLaunch a, int level) {
  constexpr int N = 2, kTile = 4 * N * kSelThreads;
  __shared__ SelectShared sh;
  const int part = blockIdx.x, unit = blockIdx.y, b = unit / a.src.H, tid = threadIdx.x;
  int k;
  const int L = kept_length(a, b, &k);
  const int first = part * a.part, last = first + a.part < L ? first + a.part : L;
  RQ_GLOBAL int32_t* out = gptr(a.slots) + (size_t)unit * a.keep;
  if (L <= a.keep) {
    if (level == 0) {
      for (int t = first + tid; t < last; t += kSelThreads) out[t] = t;
      if (part == 0 && tid == 0 && unit % a.src.H == 0) gptr(a.new_lengths)[b] = k;
    }
    return;
  }
  const size_t side = (size_t)a.src.B * a.src.H * a.parts * kBins;     // one level's counters
  RQ_GLOBAL uint32_t* count = gptr(a.counts) + (size_t)unit * a.parts * kBins;
  RQ_GLOBAL uint32_t* state = gptr(a.state) + (size_t)unit * 8;
  RQ_GLOBAL uint32_t* before = gptr(a.before) + (size_t)unit * a.parts;
  Found f = {0, (uint32_t)k, 0};
  uint32_t kept = 0, ties = 0;
  const int in_use = (L + a.part - 1) / a.part;
  bool write = level == 3;
  if (level > 0) {
    if (level > 1) {
      f.prefix = state[2 * (level - 2)];
      f.need = state[2 * (level - 2) + 1];
      if (f.need == 0) {                    // settled: the launch before wrote
        if (level == 2 && part == 0 && tid == 0) state[2 * (level - 1) + 1] = 0;
        return;
      }
      kept = before[part];
    }
    // (counters lie in falling order of their digits, a thread's two together)
    const RQ_GLOBAL u2* c = (const RQ_GLOBAL u2*)(count + side * (level - 1)) + tid;
    u2 all = {0u, 0u}, ahead = {0u, 0u};
#pragma unroll 8
    for (int i = 0; i < in_use; ++i) {
      const u2 x = c[(size_t)i * (kBins / 2)];
      all += x;
      if (i < part) ahead += x;
    }
    const uint32_t d = pick_digit(sh, all.x, all.y, level - 1, &f);
    const uint32_t hi = top_digit();
    uint32_t g = (hi > d ? ahead.x : 0u) + (hi - 1 > d ? ahead.y : 0u);
    uint32_t e = (hi == d ? ahead.x : 0u) + (hi - 1 == d ? ahead.y : 0u);
    if (!write && settle(level - 1, &f)) {
      write = true;
      g += e;                               // (none is a tie any more)
      e = 0;
    }
    g = wave_sum(g);
    e = wave_sum(e);
    if ((tid & 63) == 0) {
      sh.sum[tid >> 6] = g;
      sh.tie[tid >> 6] = e;
    }
    __syncthreads();
    for (int i = 0; i < kSelWaves; ++i) {
      kept += sh.sum[i];
      ties += sh.tie[i];
    }
    __syncthreads();
    if (tid == 0) {
      if (part == 0) {
        state[2 * (level - 1)] = f.prefix;
        state[2 * (level - 1) + 1] = f.need;
      }
      before[part] = kept;
    }
  } else if (part == 0 && tid == 0 && unit % a.src.H == 0) {
    gptr(a.new_lengths)[b] = k;
  }
  if (first >= L) return;
  const RQ_GLOBAL float* w = gptr(a.src.weights) + (size_t)unit * a.src.cap;
  if (!write) clear_digits(sh);
  for (int at = first; at < last; at += kTile) {
    uint32_t key[4 * N];
    const int base = at + (tid >> 6) * N * 256;
    load_ranks<N>(a, w, base, L, key);
    if (write)
      write_slots<N>(sh, key, base, f, out, &kept, &ties);
    else
      count_digits<N>(sh, key, level, f.prefix);
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

// One wave a (unit, K or V, block of the new cache).
template <int FMT, int D, bool BF16>
__global__ void __launch_bounds__(256) block_gather_kernel(BlockEvictLaunch a) {
  constexpr int kChunks = D / 8, kRows = 64 / kChunks, kLoads = kBlockTokens / kRows;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int unit = blockIdx.y >> 1, kind = blockIdx.y & 1, b = unit / a.src.H;
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
    for (int d = 32; d >= 1; d >>= 1) most = __builtin_fmaxf(most, __shfl_xor(most, d, 64));
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
      for (int d = 32; d >= 1; d >>= 1) most = __builtin_fmaxf(most, __shfl_xor(most, d, 64));
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
