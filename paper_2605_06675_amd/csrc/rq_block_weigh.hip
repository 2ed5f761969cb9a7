// Accumulated attention weight of every cached token, for calls of many query
// rows: after an attention launch has left each row's maximum and sum, the
// scores are computed again and each token's probabilities added over the rows.
//
// A wave holds the keys of 64 tokens as fp16 operands and walks the rows in
// tiles of 64 (their fp16 copies that the attention launch left), which the
// workgroup's four waves share through LDS (two buffers, one barrier a tile).
// With the tokens as the products' rows every lane adds up 32 tokens' weights
// over its query rows; the lanes' sums meet at the end.  Where the tokens'
// workgroups are few, several share the rows, and a small launch adds their sums
// in order: the result does not depend on scheduling.
//
// 32 units of up to 8192 tokens, 2036 rows: 116 us.  A wave's 32 rows are 512
// cycles of products and 600 of exponentials and sums, two waves a SIMD; a
// workgroup takes 70 us, 4 of them to begin, and the last round is half empty.
#include "rq_block.h"

namespace rq {

namespace {

typedef float f16v __attribute__((ext_vector_type(16)));

constexpr int kWaveTokens = 64, kTokens = 4 * kWaveTokens, kTileRows = 64;

template <int D>
__device__ __forceinline__ int query_at(int row, int piece) {
  return row * D * 2 + ((piece ^ (row & (D / 8 - 1))) << 4);
}

// Keys of 32 tokens: lane (r = lane & 31, hl = lane >> 5) gets, of token r, the
// channels 16 k + 8 hl + 0..7 in f[k]; returns the block's scale.
template <int FMT, int D>
__device__ __forceinline__ float coded_keys(const RQ_GLOBAL uint8_t* kc, const RQ_CONSTANT float* scales,
                                            int blk, h8 f[D / 16]) {
  const int lane = threadIdx.x & 63;
  const RQ_GLOBAL uint8_t* p = kc + (uint32_t)(blk * kBlockTokens + (lane & 31)) * D + 8 * (lane >> 5);
#pragma unroll
  for (int k = 0; k < D / 16; ++k) {
    const u2 w = *(const RQ_GLOBAL u2*)(p + 16 * k);
    f[k] = as_h8((u4){key_pair<FMT>(w.x, false), key_pair<FMT>(w.x, true), key_pair<FMT>(w.y, false),
                      key_pair<FMT>(w.y, true)});
  }
  return scales[blk];
}

// Largest magnitude of packed bf16 numbers.
__device__ __forceinline__ float bf16_top(u4 x) {
  float m = 0.0f;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    m = __builtin_fmaxf(m, __builtin_fmaxf(__builtin_fabsf(widen_t<true>(x[i] & 0xffffu)),
                                           __builtin_fabsf(widen_t<true>(x[i] >> 16))));
  return m;
}
// bf16 numbers times 2^-e as fp16.
__device__ __forceinline__ h8 bf16_scaled(u4 x, int e) {
  h8 f;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    f[2 * i] = (_Float16)__builtin_amdgcn_ldexpf(widen_t<true>(x[i] & 0xffffu), -e);
    f[2 * i + 1] = (_Float16)__builtin_amdgcn_ldexpf(widen_t<true>(x[i] >> 16), -e);
  }
  return f;
}

// The same of the tail's first n_tail rows (bf16 keys over a power of two, which
// is returned).
template <int D, bool BF16>
__device__ __forceinline__ float tail_keys(const RQ_GLOBAL uint16_t* kt, int n_tail, h8 f[D / 16]) {
  const int lane = threadIdx.x & 63, row = lane & 31;
  u4 raw[D / 16];
  float most = 0.0f;
#pragma unroll
  for (int k = 0; k < D / 16; ++k) {
    raw[k] = row < n_tail ? *(const RQ_GLOBAL u4*)(kt + row * D + 16 * k + 8 * (lane >> 5))
                          : (u4){0u, 0u, 0u, 0u};
    most = __builtin_fmaxf(most, bf16_top(raw[k]));
  }
  if constexpr (!BF16) {
#pragma unroll
    for (int k = 0; k < D / 16; ++k) f[k] = as_h8(raw[k]);
    return 1.0f;
  }
  most = wave_all<Max>(most);
  const int e = most > 0.0f ? __builtin_amdgcn_frexp_expf(most) : 0;
#pragma unroll
  for (int k = 0; k < D / 16; ++k) f[k] = bf16_scaled(raw[k], e);
  return __builtin_amdgcn_ldexpf(1.0f, e);
}

// One step of the sums at the kernel's end, with the lane that a move names: it
// differs in bit d, and in lower bits that later steps add up all the same.
template <int d, int MOVE>
__device__ __forceinline__ void halve(float x[32], int col) {
  const bool upper = col & d;
#pragma unroll
  for (int i = 0; i < d; ++i)
    x[i] = (upper ? x[i + d] : x[i]) + moved<MOVE>(upper ? x[i] : x[i + d]);
}

// What a score needs of its row.
struct RowInfo {
  float qs, m, inv, slope;
  int token, pos;
};

template <int FMT, int D, bool BF16>
__global__ void __launch_bounds__(256, 2) block_weigh_kernel(BlockAttendLaunch a) {
  constexpr int kShare = kTileRows * D / 256;       // channels of a row that a thread loads
  constexpr int kLanes = D / kShare;                // threads of a row: 4
  __shared__ __align__(16) uint8_t sh_q[2][kTileRows * D * 2];
  __shared__ RowInfo sh_row[2][kTileRows];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 31, hl = lane >> 5;
  const int unit = blockIdx.y, b = over(unit, a.c.by_H), h = unit - b * a.c.H;
  int past, nnew;
  block_lengths(a.past, a.new_len, b, a.n, a.max_tokens, &past, &nnew);
  const int total = past + nnew, full = total / kBlockTokens;
  const int part = blockIdx.x % a.row_parts, wg_slot = blockIdx.x / a.row_parts * kTokens;
  if (wg_slot >= total) return;
  const int slot0 = wg_slot + wave * kWaveTokens, blk = slot0 / kBlockTokens;

  h8 key[2][D / 16];
  float ks[2];
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    ks[t] = 0.0f;
    if (blk + t < full)
      ks[t] = coded_keys<FMT, D>(gptr(a.c.codes) + (size_t)unit * 2 * a.c.cap * D,
                                 cptr(a.c.scales) + (size_t)unit * 2 * (a.c.cap / kBlockTokens), blk + t, key[t]);
    else if (blk + t == full)
      ks[t] = tail_keys<D, BF16>(gptr(a.c.tail) + (size_t)unit * 2 * kBlockTokens * D, total - full * kBlockTokens, key[t]);
    else
#pragma unroll
      for (int k = 0; k < D / 16; ++k) key[t][k] = as_h8((u4){0u, 0u, 0u, 0u});
  }
  const bool far = a.slopes || a.window;
  int pos[2][16];
  if (far) {
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int slot = slot0 + 32 * t + 8 * (i >> 2) + 4 * hl + (i & 3);
        pos[t][i] = slot < total ? gptr(a.c.positions)[(size_t)unit * a.c.cap + slot] : 0;
      }
  }

  // tiles of rows that see some of the workgroup's tokens
  const int rows = nnew * a.G;
  int from = wg_slot - past, to = nnew;              // tokens of the call
  from = from > 0 ? from : 0;
  if (a.window) {
    const int64_t seen = (int64_t)wg_slot + kTokens - 1 + a.window - past;
    to = seen < to ? (int)seen : to;
  }
  int tile0 = from * a.G / kTileRows, tile1 = (to * a.G + kTileRows - 1) / kTileRows;
  {
    // this workgroup's part of all tiles
    const int all = (a.n * a.G + kTileRows - 1) / kTileRows;
    const int p0 = part_from(all, part, a.row_parts, a.by_parts);
    const int p1 = part_from(all, part + 1, a.row_parts, a.by_parts);
    tile0 = tile0 > p0 ? tile0 : p0;
    tile1 = tile1 < p1 ? tile1 : p1;
  }

  // this thread's share of a tile
  const int row_in = threadIdx.x / kLanes, ch = (threadIdx.x % kLanes) * kShare;
  const RQ_GLOBAL uint16_t* queries = gptr(a.queries) + ((size_t)unit * a.row_tiles * 16 + row_in) * D + ch;
  const RQ_GLOBAL float* stats = gptr(a.stats) + ((size_t)unit * a.row_tiles * 16 + row_in) * 2;
  const RQ_GLOBAL float* factors = gptr(a.factors) + (size_t)unit * a.row_tiles * 16 + row_in;
  u4 raw[kShare / 8];
  RowInfo info;
  auto fetch = [&](int tile) {
    const int row = tile * kTileRows + row_in;
#pragma unroll
    for (int i = 0; i < kShare / 8; ++i) raw[i] = (u4){0u, 0u, 0u, 0u};
    // (a row behind the last adds exp2(-3e38) * 0)
    info.m = -kNoScore;
    info.qs = info.inv = info.slope = 0.0f;
    info.token = info.pos = 0;
    if (row >= rows) return;
#pragma unroll
    for (int i = 0; i < kShare / 8; ++i)
      raw[i] = *(const RQ_GLOBAL u4*)(queries + (size_t)tile * kTileRows * D + 8 * i);
    if (ch == 0) {
      info.qs = factors[tile * kTileRows];
      info.m = stats[tile * kTileRows * 2];
      info.inv = stats[tile * kTileRows * 2 + 1];
      info.token = over(row, a.by_G);
      if (a.slopes) info.slope = gptr(a.slopes)[h * a.G + row - info.token * a.G] * 1.4426950408889634f;
      if (far) info.pos = gptr(a.c.positions)[(size_t)unit * a.c.cap + past + info.token];
    }
  };
  auto put = [&](int buf) {
#pragma unroll
    for (int i = 0; i < kShare / 8; ++i)
      *(u4*)(sh_q[buf] + query_at<D>(row_in, ch / 8 + i)) = raw[i];
    if (ch == 0) sh_row[buf][row_in] = info;
  };

  f16v sum[2];
#pragma unroll
  for (int t = 0; t < 2; ++t)
#pragma unroll
    for (int i = 0; i < 16; ++i) sum[t][i] = 0.0f;
  auto work = [&](int tile, int buf, int half) {          // 32 rows of a tile
    const int row0 = tile * kTileRows + 32 * half;
    if (past + over(row0 + 31, a.by_G) < slot0) return;
    const RowInfo r = sh_row[buf][32 * half + col];
    f16v s[2];
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int i = 0; i < 16; ++i) s[t][i] = 0.0f;
#pragma unroll
    for (int k = 0; k < D / 16; ++k) {
      const h8 q = *(const h8*)(sh_q[buf] + query_at<D>(32 * half + col, 2 * k + hl));
#pragma unroll
      for (int t = 0; t < 2; ++t)
        s[t] = __builtin_amdgcn_mfma_f32_32x32x16_f16(key[t][k], q, s[t], 0, 0, 0);
    }
    const bool masked = a.window || slot0 + kWaveTokens - 1 > past + over(row0, a.by_G);
    const bool large = __any(__builtin_fabsf(r.m) > kLargeScore && r.m < -kNoScore);
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      float f = ks[t] * r.qs, off = 0.0f;      // scores are s f + off
      if (a.cap != 0.0f && !a.fine) {
        // cap tanh(x) = cap - 2 cap / (1 + e^(2x)), off by 2^-22 cap
        const float e2 = f * 2.8853900817779268f;
#pragma unroll
        for (int i = 0; i < 16; ++i) s[t][i] = __builtin_amdgcn_rcpf(-1.0f - exp2_f(s[t][i] * e2));
        f = 2.0f * a.cap;
        off = a.cap;
      }
      if (far || masked || a.fine || large) {
#pragma unroll
        for (int i = 0; i < 16; ++i) s[t][i] = __builtin_fmaf(s[t][i], f, off);
        if (a.fine) {
#pragma unroll
          for (int i = 0; i < 16; ++i) s[t][i] = a.cap * tanh_f(s[t][i]);
        }
        f = 1.0f;
        off = 0.0f;
        if (far) {
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const int away = r.pos - pos[t][i];
            s[t][i] = __builtin_fmaf(-r.slope, (float)away, s[t][i]);
            if (a.window && away >= a.window) s[t][i] = -__builtin_inff();
          }
        }
        if (masked) {
          const int end = past + r.token - slot0 - 32 * t - 4 * hl;
#pragma unroll
          for (int i = 0; i < 16; ++i)
            if (8 * (i >> 2) + (i & 3) > end) s[t][i] = -__builtin_inff();
        }
      }
      const float c = off - r.m;
#pragma unroll
      for (int i = 0; i < 16; ++i)
        sum[t][i] = __builtin_fmaf(exp2_f(__builtin_fmaf(s[t][i], f, c)), r.inv, sum[t][i]);
    }
  };

  if (from < to && tile0 < tile1) {
    fetch(tile0);
    for (int tile = tile0, buf = 0; tile < tile1; ++tile, buf ^= 1) {
      put(buf);
      __syncthreads();
      if (tile + 1 < tile1) fetch(tile + 1);
#pragma unroll 1
      for (int half = 0; half < 2; ++half) work(tile, buf, half);
    }
  }

  // The 32 numbers of each lane are added over the 32 rows' lanes, halved in every
  // step: a lane keeps the half that its own bit names and hands on the other.
  // Lane (col, hl) ends with number col.
  float x[32];
#pragma unroll
  for (int i = 0; i < 32; ++i) x[i] = sum[i >> 4][i & 15];
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const u2 p = __builtin_bit_cast(u2, __builtin_amdgcn_permlane16_swap(
        __float_as_uint(x[i]), __float_as_uint(x[i + 16]), false, false));
    x[i] = __uint_as_float(p.x) + __uint_as_float(p.y);
  }
  halve<8, 0x128>(x, col);
  halve<4, 0x141>(x, col);
  halve<2, 0x4e>(x, col);
  halve<1, 0xb1>(x, col);
  const int slot = slot0 + (col & 16) * 2 + 8 * ((col & 15) >> 2) + 4 * hl + (col & 3);
  if (slot < total) {
    if (a.row_parts > 1)
      gptr(a.sums)[((size_t)part * gridDim.y + unit) * a.max_tokens + slot] = x[0];
    else
      gptr(a.c.weights)[(size_t)unit * a.c.cap + slot] += x[0];
  }
}

__global__ void __launch_bounds__(256) block_add_kernel(BlockAttendLaunch a) {
  const int unit = blockIdx.y, slot = blockIdx.x * 256 + threadIdx.x;
  int past, nnew;
  block_lengths(a.past, a.new_len, over(unit, a.c.by_H), a.n, a.max_tokens, &past, &nnew);
  if (slot >= past + nnew) return;
  float sum = 0.0f;
#pragma unroll 4
  for (int p = 0; p < a.row_parts; ++p)
    sum += gptr(a.sums)[((size_t)p * gridDim.y + unit) * a.max_tokens + slot];
  gptr(a.c.weights)[(size_t)unit * a.c.cap + slot] += sum;
}

template <int FMT, int D>
hipError_t launch(const BlockAttendLaunch& a, hipStream_t s) {
  const dim3 grid((a.max_tokens + kTokens - 1) / kTokens * a.row_parts, a.c.B * a.c.H);
  if (a.c.is_bf16)
    hipLaunchKernelGGL((block_weigh_kernel<FMT, D, true>), grid, dim3(256), 0, s, a);
  else
    hipLaunchKernelGGL((block_weigh_kernel<FMT, D, false>), grid, dim3(256), 0, s, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.row_parts == 1) return e;
  hipLaunchKernelGGL(block_add_kernel, dim3((a.max_tokens + 255) / 256, a.c.B * a.c.H), dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_block_weigh(const BlockAttendLaunch& a, hipStream_t s) {
  if (a.c.fmt == RQ_INT8) return a.c.D == 64 ? launch<RQ_INT8, 64>(a, s) : launch<RQ_INT8, 128>(a, s);
  return a.c.D == 64 ? launch<RQ_E4M3, 64>(a, s) : launch<RQ_E4M3, 128>(a, s);
}

}  // namespace rq
