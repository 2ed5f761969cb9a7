// Eviction from the block-scaled 8-bit cache by accumulated attention weight:
// of a unit's L tokens the first n_sink, the last n_recent and the heaviest of
// the rest stay (ties: the lowest slot), in order, and are quantized again in
// blocks of the new cache.
//
// Selection: the k-th largest weight by radix, 11 + 11 + 10 bits; then one
// ordered pass writes the kept slots.  The copy reads 2 D bytes a kept token
// and side and writes as many.
#include "rq_block.h"

namespace rq {

namespace {

constexpr int kSelThreads = 1024;

// A weight's place in the order, as an unsigned number; the tokens that stay
// in any case are above all others.
__device__ __forceinline__ uint32_t rank_key(float w, int slot, int L, int sink, int recent) {
  const uint32_t u = __float_as_uint(w + 0.0f);     // -0 becomes 0
  const uint32_t key = (int32_t)u < 0 ? ~u : u | 0x80000000u;
  return slot < sink || slot >= L - recent ? 0xffffffffu : (key == 0xffffffffu ? 0xfffffffeu : key);
}

__global__ void __launch_bounds__(kSelThreads) block_select_kernel(BlockEvictLaunch a) {
  __shared__ uint32_t hist[2048];
  __shared__ uint32_t wsum[kSelThreads / 64], wtie[kSelThreads / 64];
  __shared__ uint32_t pick[2];            // chosen digit, tokens above it
  const int unit = blockIdx.x, b = unit / a.src.H, tid = threadIdx.x;
  int L = gptr(a.lengths)[b];
  L = L < 0 ? 0 : (L > a.src.cap ? a.src.cap : L);
  const int k = L < a.keep ? L : a.keep;
  if (tid == 0 && unit % a.src.H == 0) gptr(a.new_lengths)[b] = k;
  RQ_GLOBAL int32_t* out = gptr(a.slots) + (size_t)unit * a.keep;
  if (L <= a.keep) {
    for (int t = tid; t < L; t += kSelThreads) out[t] = t;
    return;
  }
  const RQ_GLOBAL float* w = gptr(a.src.weights) + (size_t)unit * a.src.cap;
  uint32_t prefix = 0, need = (uint32_t)k;     // the k-th largest key's digits so far
  for (int pass = 0; pass < 3; ++pass) {
    const int shift = pass == 0 ? 21 : (pass == 1 ? 10 : 0), bins = pass == 2 ? 1024 : 2048;
    for (int i = tid; i < 2048; i += kSelThreads) hist[i] = 0;
    __syncthreads();
    for (int t = tid; t < L; t += kSelThreads) {
      const uint32_t key = rank_key(w[t], t, L, a.n_sink, a.n_recent);
      const bool in = pass == 0 || (pass == 1 ? key >> 21 == prefix : key >> 10 == prefix);
      if (in) atomicAdd(&hist[(key >> shift) & (bins - 1)], 1u);
    }
    __syncthreads();
    // the digit d with (tokens above d) < need <= (tokens above d) + hist[d]:
    // each thread sums two bins, highest first
    const int hi = 2047 - 2 * tid;
    const uint32_t c1 = hist[hi], c2 = hist[hi - 1], mine = c1 + c2;
    uint32_t x = mine;
    for (int d = 1; d < 64; d <<= 1) {
      const uint32_t y = __shfl_up(x, d, 64);
      if ((tid & 63) >= d) x += y;
    }
    if ((tid & 63) == 63) wsum[tid >> 6] = x;
    __syncthreads();
    uint32_t above = x - mine;
    for (int i = 0; i < (tid >> 6); ++i) above += wsum[i];
    if (above < need && need <= above + mine) {
      const bool first = need <= above + c1;
      pick[0] = first ? hi : hi - 1;
      pick[1] = first ? above : above + c1;
    }
    __syncthreads();
    prefix = pass == 0 ? pick[0] : (prefix << (pass == 1 ? 11 : 10)) | pick[0];
    need -= pick[1];
    __syncthreads();
  }
  // keys above `prefix` stay, and the first `need` equal to it
  uint32_t kept = 0, ties = 0;
  for (int base = 0; base < L; base += kSelThreads) {
    const int t = base + tid;
    const uint32_t key = t < L ? rank_key(w[t], t, L, a.n_sink, a.n_recent) : 0u;
    const bool gt = t < L && key > prefix, eq = t < L && key == prefix;
    const uint64_t mg = __ballot(gt), me = __ballot(eq);
    const uint64_t below = (1ull << (tid & 63)) - 1;
    if ((tid & 63) == 0) {
      wsum[tid >> 6] = __popcll(mg);
      wtie[tid >> 6] = __popcll(me);
    }
    __syncthreads();
    uint32_t g = kept + __popcll(mg & below), e = ties + __popcll(me & below);
    for (int i = 0; i < kSelThreads / 64; ++i) {
      if (i < (tid >> 6)) {
        g += wsum[i];
        e += wtie[i];
      }
      kept += wsum[i];
      ties += wtie[i];
    }
    const uint32_t at = g + (e < need ? e : need);
    if (gt || (eq && e < need)) out[at] = t;
    __syncthreads();
  }
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
  const int coded = L / kBlockTokens * kBlockTokens;
  const RQ_GLOBAL int32_t* slots = gptr(a.slots) + (size_t)unit * a.keep + blk * kBlockTokens;
  const int rows = k - blk * kBlockTokens < kBlockTokens ? k - blk * kBlockTokens : kBlockTokens;
  const size_t side = (size_t)unit * 2 + kind;
  const RQ_GLOBAL uint8_t* codes = gptr(a.src.codes) + side * a.src.cap * D;
  const RQ_GLOBAL float* scales = gptr(a.src.scales) + side * (a.src.cap / kBlockTokens);
  const RQ_GLOBAL uint16_t* tail = gptr(a.src.tail) + side * kBlockTokens * D;
  const int row0 = lane / kChunks, ch = (lane % kChunks) * 8;
  float x[kLoads][8];
  float most = 0.0f;
#pragma unroll
  for (int i = 0; i < kLoads; ++i) {
    const int row = row0 + kRows * i;
    const int slot = row < rows ? slots[row] : 0;
    if (row >= rows) {
#pragma unroll
      for (int e = 0; e < 8; ++e) x[i][e] = 0.0f;
    } else if (slot < coded) {
      const u2 w = *(const RQ_GLOBAL u2*)(codes + (size_t)slot * D + ch);
      const float s = scales[slot / kBlockTokens];
#pragma unroll
      for (int e = 0; e < 8; ++e) x[i][e] = block_value<FMT>(w[e >> 2], e & 3) * s;
    } else {
      const u4 w = *(const RQ_GLOBAL u4*)(tail + (slot - coded) * D + ch);
#pragma unroll
      for (int e = 0; e < 8; ++e)
        x[i][e] = widen_t<BF16>(e & 1 ? w[e >> 1] >> 16 : w[e >> 1] & 0xffffu);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) most = __builtin_fmaxf(most, __builtin_fabsf(x[i][e]));
  }
  if (rows == kBlockTokens) {
    for (int d = 32; d >= 1; d >>= 1) most = __builtin_fmaxf(most, __shfl_xor(most, d, 64));
    float inv;
    const float scale = block_scale<FMT>(most, &inv);
    RQ_GLOBAL uint8_t* out = gptr(a.dst.codes) + (side * a.dst.cap + (size_t)blk * kBlockTokens) * D;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      u2 w;
#pragma unroll
      for (int p = 0; p < 2; ++p)
        w[p] = block_codes<FMT>(x[i][4 * p], x[i][4 * p + 1], x[i][4 * p + 2], x[i][4 * p + 3], inv);
      *(RQ_GLOBAL u2*)(out + (row0 + kRows * i) * D + ch) = w;
    }
    if (lane == 0) gptr(a.dst.scales)[side * (a.dst.cap / kBlockTokens) + blk] = scale;
  } else {
    RQ_GLOBAL uint16_t* out = gptr(a.dst.tail) + side * kBlockTokens * D;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int row = row0 + kRows * i;
      u4 w;
#pragma unroll
      for (int e = 0; e < 4; ++e)
        w[e] = narrow_t<BF16>(x[i][2 * e]) | ((uint32_t)narrow_t<BF16>(x[i][2 * e + 1]) << 16);
      if (row < rows) *(RQ_GLOBAL u4*)(out + row * D + ch) = w;
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
  hipLaunchKernelGGL(block_select_kernel, dim3(a.src.B * a.src.H), dim3(kSelThreads), 0, s, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  if (a.src.fmt == RQ_INT8)
    return a.src.D == 64 ? launch_gather<RQ_INT8, 64>(a, s) : launch_gather<RQ_INT8, 128>(a, s);
  return a.src.D == 64 ? launch_gather<RQ_E4M3, 64>(a, s) : launch_gather<RQ_E4M3, 128>(a, s);
}

}  // namespace rq
