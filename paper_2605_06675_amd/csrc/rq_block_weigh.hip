// Accumulated attention weight of every cached token: after an attention call
// has left each row's maximum and sum, the scores are computed again and each
// token's probabilities added over the call's rows.  One wave owns 32 tokens
// and adds its rows in order, so the result does not depend on scheduling.
#include "rq_block.h"

namespace rq {

namespace {

template <int FMT, int D, bool BF16>
__global__ void __launch_bounds__(256) block_weigh_kernel(BlockAttendLaunch a) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r = lane & 15, g = lane >> 4;
  const int unit = blockIdx.y, b = unit / a.c.H, h = unit - b * a.c.H;
  int past, nnew;
  block_lengths(a.past, a.new_len, b, a.n, a.max_tokens, &past, &nnew);
  const int total = past + nnew, full = total / kBlockTokens;
  const int blk = blockIdx.x * 4 + wave, slot0 = blk * kBlockTokens;
  if (slot0 >= total) return;
  KeyBlock<D> k;
  const RQ_GLOBAL uint16_t* kt = gptr(a.c.tail) + (size_t)unit * 2 * kBlockTokens * D;
  if (blk < full)
    load_keys<D>(gptr(a.c.codes) + (size_t)unit * 2 * a.c.cap * D,
                 gptr(a.c.scales) + (size_t)unit * 2 * (a.c.cap / kBlockTokens), blk, &k);
  const RQ_GLOBAL int32_t* pos = gptr(a.c.positions) + (size_t)unit * a.c.cap;
  const RQ_GLOBAL float* stats = gptr(a.stats) + (size_t)unit * a.row_tiles * 32;
  // the first token that sees the block, and the tiles from its row on
  const int sees = slot0 - past > 0 ? slot0 - past : 0;
  const int tiles = (nnew * a.G + 15) / 16;
  f4 sum[2] = {{0.0f, 0.0f, 0.0f, 0.0f}, {0.0f, 0.0f, 0.0f, 0.0f}};
  for (int rt = sees * a.G / 16; rt < tiles; ++rt) {
    const int row = rt * 16 + r;
    QueryTile<D> q;
    load_queries<D, BF16>(a, b, h, row, past, nnew, &q);
    f4 s[2];
    float factor = a.qscale;
    if (blk < full) {
      key_products<FMT, D>(k, q, s);
      factor = k.scale * q.qs;
    } else {
      tail_products<D, BF16>(a, b, h, kt, q, s);
    }
    block_scores<D>(a, q, pos, factor, slot0, past, true, s);
    if (q.valid) {
      const float m = stats[row * 2], inv = stats[row * 2 + 1];
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          sum[t][i] = __builtin_fmaf(exp2_f(s[t][i] - m), inv, sum[t][i]);
    }
  }
#pragma unroll
  for (int t = 0; t < 2; ++t)
#pragma unroll
    for (int i = 0; i < 4; ++i)
      for (int d = 1; d < 16; d <<= 1) sum[t][i] += __shfl_xor(sum[t][i], d, 64);
  // lane (r, g) with r < 8 writes token 16 (r / 4) + 4 g + r % 4
  float add = 0.0f;
#pragma unroll
  for (int t = 0; t < 2; ++t)
#pragma unroll
    for (int i = 0; i < 4; ++i) add = r == 4 * t + i ? sum[t][i] : add;
  const int slot = slot0 + 16 * (r >> 2) + 4 * g + (r & 3);
  if (r < 8 && slot < total) gptr(a.c.weights)[(size_t)unit * a.c.cap + slot] += add;
}

template <int FMT, int D>
hipError_t launch(const BlockAttendLaunch& a, hipStream_t s) {
  const dim3 grid((a.max_tokens + 4 * kBlockTokens - 1) / (4 * kBlockTokens), a.c.B * a.c.H);
  if (a.c.is_bf16)
    hipLaunchKernelGGL((block_weigh_kernel<FMT, D, true>), grid, dim3(256), 0, s, a);
  else
    hipLaunchKernelGGL((block_weigh_kernel<FMT, D, false>), grid, dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_block_weigh(const BlockAttendLaunch& a, hipStream_t s) {
  if (a.c.fmt == RQ_INT8) return a.c.D == 64 ? launch<RQ_INT8, 64>(a, s) : launch<RQ_INT8, 128>(a, s);
  return a.c.D == 64 ? launch<RQ_E4M3, 64>(a, s) : launch<RQ_E4M3, 128>(a, s);
}

}  // namespace rq
