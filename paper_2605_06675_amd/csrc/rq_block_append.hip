// Append to the block-scaled 8-bit cache: quantize every block that becomes
// full, keep the rows of the unfinished one in the 16-bit tail.
//
// s = fp32(max|x| * fp32(1 / M)) over the 32 tokens x D channels of a block, M = 127
// (int8) or 448 (e4m3); code = round_half_even(x * fp32(1 / s)).
//
// Memory bound: 2 bytes read and one written an element.  One wave a block, all
// its rows in flight; codes go out non-temporally.  4 x 8192 tokens of 8 heads
// (203 MB): 32.5 us, 6.2 TB/s.  A token of each of 16 sequences: 2.4 us.
#include "rq_block.h"

namespace rq {

namespace {

// A block's rows as a wave holds them: a lane has 8 channels of every row it loads,
// 64 lanes cover 512 / D rows a load.
template <int D>
constexpr int kRowsOf = 512 / D;
template <int D>
constexpr int kLoadsOf = kBlockTokens / kRowsOf<D>;

// The largest magnitude of eight numbers and `most`; their codes.
template <bool BF16>
__device__ __forceinline__ float largest_of(u4 x, float most) {
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    most = __builtin_fmaxf(most, __builtin_fabsf(widen_t<BF16>(x[w] & 0xffffu)));
    most = __builtin_fmaxf(most, __builtin_fabsf(widen_t<BF16>(x[w] >> 16)));
  }
  return most;
}
template <int FMT, bool BF16>
__device__ __forceinline__ void store_codes(u4 x, float inv, RQ_GLOBAL uint8_t* out) {
  u2 w;
#pragma unroll
  for (int p = 0; p < 2; ++p)
    w[p] = block_codes<FMT>(widen_t<BF16>(x[2 * p] & 0xffffu), widen_t<BF16>(x[2 * p] >> 16),
                            widen_t<BF16>(x[2 * p + 1] & 0xffffu), widen_t<BF16>(x[2 * p + 1] >> 16), inv);
  __builtin_nontemporal_store(w, (RQ_GLOBAL u2*)out);
}

// One wave a (unit, K or V, block).
template <int FMT, int D, bool BF16>
__global__ void __launch_bounds__(256) block_append_kernel(BlockAppendLaunch a) {
  constexpr int kChunks = D / 8, kRows = kRowsOf<D>, kLoads = kLoadsOf<D>;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int waves = (a.n + kBlockTokens - 1) / kBlockTokens;   // most blocks a call fills
  const int j = blockIdx.x * 4 + wave;
  if (j >= waves) return;
  const int unit = blockIdx.y >> 1, kind = blockIdx.y & 1;
  const int b = over(unit, a.c.by_H), h = unit - b * a.c.H;
  int past, nnew;
  block_lengths(a.past, nullptr, b, 0, a.c.cap, &past, &nnew);
  nnew = a.new_len ? __builtin_amdgcn_readfirstlane(gptr(a.new_len)[b]) : a.n;
  nnew = nnew < 0 ? 0 : (nnew > a.n ? a.n : nnew);
  nnew = nnew > a.c.cap - past ? a.c.cap - past : nnew;
  const int total = past + nnew, full = total / kBlockTokens;
  const int blk = past / kBlockTokens + j;
  const BlockRows& src = kind ? a.v : a.k;
  const RQ_GLOBAL uint16_t* in = gptr(static_cast<const uint16_t*>(src.p)) + b * src.sb + h * src.sh;
  RQ_GLOBAL uint16_t* tail = gptr(a.c.tail) + (size_t)(unit * 2 + kind) * kBlockTokens * D;
  const int row0 = lane / kChunks, ch = (lane % kChunks) * 8;

  if (blk < full) {
    u4 x[kLoads];
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int row = row0 + kRows * i, slot = blk * kBlockTokens + row;
      x[i] = slot < past ? *(const RQ_GLOBAL u4*)(tail + row * D + ch)
                         : __builtin_nontemporal_load((const RQ_GLOBAL u4_any*)(in + (int64_t)(slot - past) * src.st + ch));
    }
    float most = 0.0f;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) most = largest_of<BF16>(x[i], most);
    most = wave_all<Max>(most);
    float inv;
    const float scale = block_scale<FMT>(most, &inv);
    RQ_GLOBAL uint8_t* out = gptr(a.c.codes) + ((size_t)(unit * 2 + kind) * a.c.cap + (size_t)blk * kBlockTokens) * D;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) store_codes<FMT, BF16>(x[i], inv, out + (row0 + kRows * i) * D + ch);
    if (lane == 0) gptr(a.c.scales)[(size_t)(unit * 2 + kind) * (a.c.cap / kBlockTokens) + blk] = scale;
  }
  if (j == 0) {
    // the unfinished block's new rows, after the rows that they may replace
    // have been read (by this wave, above)
    const int first = past > full * kBlockTokens ? past : full * kBlockTokens;
    for (int slot = first + row0; slot < total; slot += kRows)
      *(RQ_GLOBAL u4*)(tail + (slot % kBlockTokens) * D + ch) =
          *(const RQ_GLOBAL u4_any*)(in + (int64_t)(slot - past) * src.st + ch);
  }
  if (kind == 0) {
    RQ_GLOBAL int32_t* pos = gptr(a.c.positions) + (size_t)unit * a.c.cap;
    const int t = j * kBlockTokens + lane;
    if (lane < kBlockTokens && t < nnew) {
      pos[past + t] = (past > 0 ? pos[past - 1] : -1) + 1 + t;
      if (a.c.weights) gptr(a.c.weights)[(size_t)unit * a.c.cap + past + t] = 0.0f;
    }
  }
}

// The rows of an accepted path.  A workgroup takes a sequence in one layer, all heads and
// both sides, so that the lengths are read by the workgroup that writes them.  First
// its waves code the blocks that become full, one (kv-head, side) after the other; then
// its threads copy the unfinished block's rows, 16 bytes each.
//
// A chain of latencies (lengths and path, rows, stores), and of so many small
// workgroups the launch of their waves: one wave a (kv-head, side) took 16 us where eight
// for all took 12.1 (32 layers of 16 sequences, 8 kv-heads, some four rows of each).
// Workgroups next to each other are a sequence's layers: all XCDs then share a sequence
// that takes many rows or fills blocks, where a sequence to an XCD takes 12.3 us this
// way takes 8.0, 1.4 TB/s (80 layers of 16 even sequences and 8 rows 8.5, 2.5 TB/s).
constexpr int kAcceptWaves = 8, kAcceptThreads = 64 * kAcceptWaves;

template <int FMT, int D, bool BF16>
__global__ void __launch_bounds__(kAcceptThreads) block_accept_kernel(BlockAcceptLaunch a) {
  constexpr int kChunks = D / 8, kRows = kRowsOf<D>, kLoads = kLoadsOf<D>;
  __shared__ int node[RQ_MAX_NODES];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int layer = blockIdx.x, b = blockIdx.y, at = layer * a.c.B + b;
  int past = gptr(a.lengths)[at], count = gptr(a.count)[b];
  for (int t = threadIdx.x; t < a.n_path; t += kAcceptThreads) {
    const int i = gptr(a.path)[(size_t)b * a.n_path + t];
    node[t] = i < 0 ? 0 : (i < a.n ? i : a.n - 1);
  }
  past = __builtin_amdgcn_readfirstlane(past < 0 ? 0 : (past < a.c.cap ? past : a.c.cap));
  count = __builtin_amdgcn_readfirstlane(count < 0 ? 0 : (count < a.n_path ? count : a.n_path));
  const int fit = count < a.c.cap - past ? count : a.c.cap - past;
  const int total = past + fit, full = total / kBlockTokens;
  __syncthreads();                       // (every wave has read the lengths)
  if (threadIdx.x == 0) {
    gptr(a.new_lengths)[at] = total;
    if (a.past) gptr(a.past)[at] = past;
    if (a.fitting) gptr(a.fitting)[at] = fit;
    if (a.dropped) gptr(a.dropped)[at] = count - fit;
  }
  if (fit == 0) return;
  const int pairs = 2 * a.c.H, chunk = threadIdx.x % kChunks;
  auto rows_of = [&](int pair) {         // the call's rows of a (head, side), at this thread's chunk
    const BlockRows& src = pair & 1 ? a.v : a.k;
    return gptr(static_cast<const uint16_t*>(src.p)) + layer * (pair & 1 ? a.v_layer : a.k_layer) + b * src.sb +
           (pair >> 1) * src.sh + chunk * 8;
  };
  auto tail_of = [&](int pair) {
    return gptr(a.c.tail) + ((size_t)at * pairs + pair) * kBlockTokens * D + chunk * 8;
  };

  if (full > past / kBlockTokens) {
    const int row0 = lane / kChunks;
    for (int pair = wave; pair < pairs; pair += kAcceptWaves) {
      const size_t us = (size_t)at * pairs + pair;
      const RQ_GLOBAL uint16_t* in = rows_of(pair);
      const RQ_GLOBAL uint16_t* tail = tail_of(pair);
      const int64_t st = pair & 1 ? a.v.st : a.k.st;
      for (int blk = past / kBlockTokens; blk < full; ++blk) {
        u4 x[kLoads];
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
          const int row = row0 + kRows * i, t = blk * kBlockTokens + row - past;
          const RQ_GLOBAL uint16_t* from = t >= 0 ? in + node[t >= 0 ? t : 0] * st : tail + row * D;
          x[i] = *(const RQ_GLOBAL u4_any*)from;
        }
        float most = 0.0f;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) most = largest_of<BF16>(x[i], most);
        float inv;
        const float scale = block_scale<FMT>(wave_all<Max>(most), &inv);
        RQ_GLOBAL uint8_t* out = gptr(a.c.codes) + (us * a.c.cap + (size_t)blk * kBlockTokens) * D + chunk * 8;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) store_codes<FMT, BF16>(x[i], inv, out + (row0 + kRows * i) * D);
        if (lane == 0) gptr(a.c.scales)[us * (a.c.cap / kBlockTokens) + blk] = scale;
      }
    }
    __syncthreads();                     // the rows that the next ones may replace are read
  }

  const int first = full * kBlockTokens > past ? full * kBlockTokens - past : 0;
  const int rows = (fit - first) * pairs;               // pair by pair
  constexpr int kStep = kAcceptThreads / kChunks;       // rows at a time
  for (int r0 = threadIdx.x / kChunks; r0 < rows; r0 += 4 * kStep) {
    u4 x[4];
    RQ_GLOBAL u4* to[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int r = r0 + i * kStep < rows ? r0 + i * kStep : r0;
      const int pair = (uint32_t)r / (uint32_t)(fit - first), t = first + r - pair * (fit - first);
      x[i] = *(const RQ_GLOBAL u4_any*)(rows_of(pair) + node[t] * (pair & 1 ? a.v.st : a.k.st));
      to[i] = (RQ_GLOBAL u4*)(tail_of(pair) + ((past + t) % kBlockTokens) * D);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (i == 0 || r0 + i * kStep < rows) *to[i] = x[i];
  }
  for (int i = threadIdx.x; i < a.c.H * fit; i += kAcceptThreads) {
    const int h = (uint32_t)i / (uint32_t)fit, t = i - h * fit;
    RQ_GLOBAL int32_t* pos = gptr(a.c.positions) + ((size_t)at * a.c.H + h) * a.c.cap + past;
    pos[t] = (past > 0 ? pos[-1] + 1 : 0) + t;
    if (a.c.weights) gptr(a.c.weights)[((size_t)at * a.c.H + h) * a.c.cap + past + t] = 0.0f;
  }
}

// A thread a sequence: the rule by which the kernel above drops tokens.
__global__ void __launch_bounds__(256) block_advance_kernel(BlockAdvanceLaunch a) {
  const int b = blockIdx.x * 256 + threadIdx.x;
  if (b >= a.B) return;
  int past = gptr(a.lengths)[b], nnew = a.new_len ? gptr(a.new_len)[b] : a.n;
  past = past < 0 ? 0 : (past > a.cap ? a.cap : past);
  nnew = nnew < 0 ? 0 : (nnew > a.n ? a.n : nnew);
  const int fit = nnew > a.cap - past ? a.cap - past : nnew;
  gptr(a.lengths)[b] = past + fit;
  if (a.past) gptr(a.past)[b] = past;
  if (a.fitting) gptr(a.fitting)[b] = fit;
  if (a.dropped) gptr(a.dropped)[b] = nnew - fit;
}

template <int FMT, int D>
hipError_t launch(const BlockAppendLaunch& a, hipStream_t s) {
  const dim3 grid((a.n + 4 * kBlockTokens - 1) / (4 * kBlockTokens), 2 * a.c.B * a.c.H);
  if (a.c.is_bf16)
    hipLaunchKernelGGL((block_append_kernel<FMT, D, true>), grid, dim3(256), 0, s, a);
  else
    hipLaunchKernelGGL((block_append_kernel<FMT, D, false>), grid, dim3(256), 0, s, a);
  return hipGetLastError();
}

template <int FMT, int D>
hipError_t launch(const BlockAcceptLaunch& a, hipStream_t s) {
  const dim3 grid(a.layers, a.c.B), block(kAcceptThreads);
  if (a.c.is_bf16)
    hipLaunchKernelGGL((block_accept_kernel<FMT, D, true>), grid, block, 0, s, a);
  else
    hipLaunchKernelGGL((block_accept_kernel<FMT, D, false>), grid, block, 0, s, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_block_accept(const BlockAcceptLaunch& a, hipStream_t s) {
  if (a.c.fmt == RQ_INT8) return a.c.D == 64 ? launch<RQ_INT8, 64>(a, s) : launch<RQ_INT8, 128>(a, s);
  return a.c.D == 64 ? launch<RQ_E4M3, 64>(a, s) : launch<RQ_E4M3, 128>(a, s);
}

hipError_t launch_block_advance(const BlockAdvanceLaunch& a, hipStream_t s) {
  hipLaunchKernelGGL(block_advance_kernel, dim3((a.B + 255) / 256), dim3(256), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_block_append(const BlockAppendLaunch& a, hipStream_t s) {
  if (a.c.fmt == RQ_INT8) return a.c.D == 64 ? launch<RQ_INT8, 64>(a, s) : launch<RQ_INT8, 128>(a, s);
  return a.c.D == 64 ? launch<RQ_E4M3, 64>(a, s) : launch<RQ_E4M3, 128>(a, s);
}

}  // namespace rq
