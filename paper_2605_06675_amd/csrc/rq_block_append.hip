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

// One wave a (unit, K or V, block).  A lane holds 8 channels of every row it
// loads: 64 lanes cover 512 / D rows a load.
template <int FMT, int D, bool BF16>
__global__ void __launch_bounds__(256) block_append_kernel(BlockAppendLaunch a) {
  constexpr int kChunks = D / 8, kRows = 64 / kChunks, kLoads = kBlockTokens / kRows;
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
    for (int i = 0; i < kLoads; ++i)
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        most = __builtin_fmaxf(most, __builtin_fabsf(widen_t<BF16>(x[i][w] & 0xffffu)));
        most = __builtin_fmaxf(most, __builtin_fabsf(widen_t<BF16>(x[i][w] >> 16)));
      }
    most = wave_all<Max>(most);
    float inv;
    const float scale = block_scale<FMT>(most, &inv);
    RQ_GLOBAL uint8_t* out = gptr(a.c.codes) + ((size_t)(unit * 2 + kind) * a.c.cap + (size_t)blk * kBlockTokens) * D;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      u2 w;
#pragma unroll
      for (int p = 0; p < 2; ++p)
        w[p] = block_codes<FMT>(widen_t<BF16>(x[i][2 * p] & 0xffffu), widen_t<BF16>(x[i][2 * p] >> 16),
                                widen_t<BF16>(x[i][2 * p + 1] & 0xffffu), widen_t<BF16>(x[i][2 * p + 1] >> 16), inv);
      __builtin_nontemporal_store(w, (RQ_GLOBAL u2*)(out + (row0 + kRows * i) * D + ch));
    }
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

}  // namespace

hipError_t launch_block_advance(const BlockAdvanceLaunch& a, hipStream_t s) {
  hipLaunchKernelGGL(block_advance_kernel, dim3((a.B + 255) / 256), dim3(256), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_block_append(const BlockAppendLaunch& a, hipStream_t s) {
  if (a.c.fmt == RQ_INT8) return a.c.D == 64 ? launch<RQ_INT8, 64>(a, s) : launch<RQ_INT8, 128>(a, s);
  return a.c.D == 64 ? launch<RQ_E4M3, 64>(a, s) : launch<RQ_E4M3, 128>(a, s);
}

}  // namespace rq
