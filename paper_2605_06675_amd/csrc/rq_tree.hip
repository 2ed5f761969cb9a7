// Trees of drafted tokens: which nodes each one sees, and which of them the
// target's probabilities accept.
#include "rq_block.h"
#include "rq_tree.h"

namespace rq {

namespace {

// Nodes of sequence b, whatever the device array holds.
__device__ __forceinline__ int node_count(const int32_t* new_len, int b, int n) {
  int m = new_len ? gptr(new_len)[b] : n;
  m = m < 0 ? 0 : (m > n ? n : m);
  return __builtin_amdgcn_readfirstlane(m);
}

__device__ __forceinline__ int parent_of(const int32_t* parents, int b, int n, int i) {
  const int p = gptr(parents)[(size_t)b * n + i];
  return p < -1 ? -1 : (p < i ? p : i - 1);
}

// --------------------------------------------------------------------- layout
// sees(i) = {i} + sees(parent of i).
//
// In two levels of 32 nodes, a word each: a node first follows its parents inside
// its own word (at most 31 steps), which gives that word's bits and the ancestor
// where the chain leaves it; a row then goes from word to word by those (at most
// 31 steps more).  Bound by latency: some 60 dependent LDS reads at worst, where
// a chain of 1024 nodes followed parent by parent takes 1023.
constexpr int kMaskThreads = 256;

__global__ void __launch_bounds__(kMaskThreads) tree_mask_kernel(TreeMaskLaunch a) {
  __shared__ int32_t parent[RQ_MAX_NODES];
  __shared__ uint32_t bits[RQ_MAX_NODES];
  __shared__ int32_t leave[RQ_MAX_NODES];     // the chain's first node before the word, or -1
  const int b = blockIdx.y, m = node_count(a.new_len, b, a.n);
  const int first = blockIdx.x * kMaskThreads, end = min(first + kMaskThreads, m);
  if (first >= m) return;
  for (int i = threadIdx.x; i < end; i += kMaskThreads) parent[i] = parent_of(a.parents, b, a.n, i);
  __syncthreads();
  for (int i = threadIdx.x; i < end; i += kMaskThreads) {
    uint32_t w = 0;
    int j = i;
    do {
      w |= 1u << (j & 31);
      j = parent[j];
    } while (j >= (i & ~31));
    bits[i] = w;
    leave[i] = j;
  }
  __syncthreads();
  const int i = first + threadIdx.x;
  if (i >= end) return;
  RQ_GLOBAL uint32_t* row = gptr(a.mask) + ((size_t)b * a.n + i) * a.words;
  int j = i, count = 0;
  for (int w = a.words - 1; w >= 0; --w) {
    uint32_t x = 0;
    if (j >= w * 32) {         // (never further than this word)
      x = bits[j];
      j = leave[j];
      count += __popc(x);
    }
    row[w] = x;
  }
  if (a.depth) gptr(a.depth)[(size_t)b * a.n + i] = count - 1;
}

// --------------------------------------------------------------- verification
// Walk: from the root, the children of the last accepted node in order,
//   accept child c where u_c q(x) s < r(x);   r <- max(0, r / s - q), s <- sum r
// (q = 1 and r(x) <- 0, s <- max(0, s - r(x)) without the draft's rows).  A test needs one
// entry of each row, which all nodes load at once; without the draft's rows the
// mass before each test is a sum over the earlier siblings, so all tests are
// decided before the walk.  With them a rejection that leaves a sibling to test
// needs the residual's sum over a whole row.
//
// Every workgroup of a sequence walks by itself, to the same end, and adds its part
// of the residual that the last token is drawn from; the second kernel finds the
// part, and in it the token.  All in fp64: the results are decisions, which fp32
// sums would make otherwise next to a border.
constexpr int kThreads = 1024, kEach = kVerifyStep / kThreads;
constexpr int kNone = 1 << 30;

template <int DTYPE>
struct Prob {
  typedef uint16_t type;
  static constexpr bool kBf16 = DTYPE == RQ_BF16;
};
template <>
struct Prob<RQ_F32> {
  typedef float type;
};

template <int DTYPE>
__device__ __forceinline__ float prob(const RQ_GLOBAL typename Prob<DTYPE>::type* p) {
  if constexpr (DTYPE == RQ_F32)
    return *p;
  else
    return widen_t<DTYPE == RQ_BF16>(*p);
}

// Entries v..v + 15 of a row; zeros behind its end.
template <int DTYPE>
__device__ __forceinline__ void load_probs(const RQ_GLOBAL typename Prob<DTYPE>::type* row, int v, int vocab, float x[kEach]) {
  if (v + kEach <= vocab) {
    if constexpr (DTYPE == RQ_F32) {
#pragma unroll
      for (int i = 0; i < kEach / 4; ++i) {
        const f4 y = *(const RQ_GLOBAL f4_any*)(row + v + 4 * i);
#pragma unroll
        for (int j = 0; j < 4; ++j) x[4 * i + j] = y[j];
      }
    } else {
#pragma unroll
      for (int i = 0; i < kEach / 8; ++i) {
        const u4 y = *(const RQ_GLOBAL u4_any*)(row + v + 8 * i);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          x[8 * i + 2 * j] = widen_t<DTYPE == RQ_BF16>(y[j] & 0xffffu);
          x[8 * i + 2 * j + 1] = widen_t<DTYPE == RQ_BF16>(y[j] >> 16);
        }
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < kEach; ++i) x[i] = v + i < vocab ? prob<DTYPE>(row + v + i) : 0.0f;
  }
}

// A node's residual: its rows, and what its children's rejections did to it.
template <int DTYPE, bool DRAFT>
struct Residual {
  typedef typename Prob<DTYPE>::type type;
  const RQ_GLOBAL type *target, *draft;
  int rejected;             // with the draft's rows: how many
  const double* inverse;    // 1 / s before each of them (LDS)
  const int* gone;          // without: the tokens taken out of [.., ..) (LDS),
  int n_gone;               // how many

  __device__ __forceinline__ Residual(const TreeVerifyLaunch& a, int b, int node) {
    target = gptr(static_cast<const type*>(a.target)) + b * a.t_sb + node * a.t_sn;
    draft = DRAFT ? gptr(static_cast<const type*>(a.draft)) + b * a.d_sb + node * a.d_sn : target;
    rejected = n_gone = 0;
  }

  __device__ __forceinline__ void load(int v, int vocab, double r[kEach]) const {
    float p[kEach], q[kEach];
    load_probs<DTYPE>(target, v, vocab, p);
    if (DRAFT && rejected) load_probs<DTYPE>(draft, v, vocab, q);
#pragma unroll
    for (int i = 0; i < kEach; ++i) r[i] = p[i];
    if constexpr (DRAFT) {
      for (int j = 0; j < rejected; ++j) {
        const double by = inverse[j];
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
          const double x = r[i] * by - (double)q[i];
          r[i] = x > 0.0 ? x : 0.0;
        }
      }
    } else {
      for (int j = 0; j < n_gone; ++j) {
        const int at = gone[j] - v;
#pragma unroll
        for (int i = 0; i < kEach; ++i)
          if (at == i) r[i] = 0.0;
      }
    }
  }
};

__device__ __forceinline__ double wave_sum(double x) {
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) x += __shfl_xor(x, d);
  return x;
}

// The sum over the workgroup, in every thread.
__device__ __forceinline__ double block_sum(double x, double* lds) {
  x = wave_sum(x);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = x;
  __syncthreads();
  double sum = 0.0;
#pragma unroll
  for (int w = 0; w < kThreads / 64; ++w) sum += lds[w];
  return sum;
}

template <int DTYPE, bool DRAFT>
__device__ __forceinline__ double residual_sum(const Residual<DTYPE, DRAFT>& res, int lo, int hi, int vocab, double* lds) {
  double sum = 0.0;
  for (int v = lo + (int)threadIdx.x * kEach; v < hi; v += kVerifyStep) {
    double r[kEach];
    res.load(v, vocab, r);
#pragma unroll
    for (int i = 0; i < kEach; ++i) sum += r[i];
  }
  return block_sum(sum, lds);
}

// What walk and selection hold of the nodes.
struct Nodes {
  int parent[RQ_MAX_NODES], token[RQ_MAX_NODES];
};

// The tokens of node's children in [lo, hi), into gone.
__device__ __forceinline__ int gone_tokens(const Nodes& s, int m, int node, int lo, int hi, int* gone, int* count) {
  if (threadIdx.x == 0) *count = 0;
  __syncthreads();
  for (int i = threadIdx.x; i < m; i += kThreads)
    if (s.parent[i] == node && s.token[i] >= lo && s.token[i] < hi) gone[atomicAdd(count, 1)] = s.token[i];
  __syncthreads();
  return *count;
}

template <int DTYPE, bool DRAFT>
__global__ void __launch_bounds__(kThreads) tree_walk_kernel(TreeVerifyLaunch a) {
  __shared__ Nodes s;
  __shared__ float p[RQ_MAX_NODES], q[RQ_MAX_NODES];   // of a node's token, in its parent's rows
  __shared__ float u[RQ_MAX_NODES];
  __shared__ int child[RQ_MAX_NODES];     // the first child (without a draft: the first accepted one)
  __shared__ int sibling[RQ_MAX_NODES];   // the next one
  __shared__ double inverse[RQ_MAX_NODES];
  __shared__ double red[kThreads / 64];
  __shared__ int n_gone;
  const int b = blockIdx.y, part = blockIdx.x, t = threadIdx.x;
  const int m = node_count(a.new_len, b, a.n);
  RQ_GLOBAL int32_t* path = gptr(a.path) + (size_t)b * a.n_path;
  if (m == 0) {
    if (part == 0) {
      if (t < a.n_path) path[t] = -1;
      if (t == 0) {
        gptr(a.count)[b] = 0;
        gptr(a.found)[b * 4] = -1;
      }
    }
    return;
  }
  const int me = t;                       // (at most as many nodes as threads)
  if (me < m) {
    const size_t at = (size_t)b * a.n + me;
    const int up = me == 0 ? -1 : parent_of(a.parents, b, a.n, me);
    int x = gptr(a.tokens)[at];
    x = x < 0 ? 0 : (x < a.vocab ? x : a.vocab - 1);
    s.parent[me] = up;
    s.token[me] = x;
    u[me] = gptr(a.uniforms)[at];
    child[me] = sibling[me] = kNone;
    const Residual<DTYPE, DRAFT> row(a, b, up < 0 ? 0 : up);
    p[me] = prob<DTYPE>(row.target + x);
    if (DRAFT) q[me] = prob<DTYPE>(row.draft + x);
  }
  __syncthreads();
  const int up = me < m ? s.parent[me] : -1;
  if constexpr (DRAFT) {
    if (up >= 0) {
      int before = -1;
      for (int j = 0; j < me; ++j) before = s.parent[j] == up ? j : before;
      if (before < 0)
        child[up] = me;
      else
        sibling[before] = me;
    }
  } else {
    if (up >= 0) {
      // a token that an earlier sibling has is gone by its turn
      const int x = s.token[me];
      bool twice = false;
      for (int j = 0; j < me; ++j) twice |= s.parent[j] == up && s.token[j] == x;
      q[me] = twice ? 0.0f : p[me];
    }
    __syncthreads();
    if (up >= 0) {
      double mass = 1.0;
      for (int j = 0; j < me; ++j) {
        mass -= s.parent[j] == up ? (double)q[j] : 0.0;
        mass = mass > 0.0 ? mass : 0.0;
      }
      if ((double)u[me] * mass < (double)q[me]) atomicMin(&child[up], me);
    }
  }
  __syncthreads();

  // the walk, alike in every thread
  int cur = 0, count = 1, rejected = 0, full = 0;
  if (part == 0 && t == 0) path[0] = 0;
  for (;;) {
    if (count == a.n_path) {
      full = 1;
      break;
    }
    int c = child[cur];
    if constexpr (DRAFT) {
      double mass = 1.0;
      rejected = 0;
      while (c != kNone) {
        double r = p[c];
        for (int j = 0; j < rejected; ++j) {
          r = r * inverse[j] - (double)q[c];
          r = r > 0.0 ? r : 0.0;
        }
        if ((double)u[c] * (double)q[c] * mass < r) break;
        if (t == 0) inverse[rejected] = rejected == 0 ? 1.0 : (mass > 0.0 ? 1.0 / mass : 0.0);
        ++rejected;
        c = sibling[c];
        __syncthreads();
        if (c == kNone || mass == 0.0) {      // (no mass: none of the others is accepted)
          c = kNone;
          break;
        }
        Residual<DTYPE, DRAFT> res(a, b, cur);
        res.rejected = rejected;
        res.inverse = inverse;
        mass = residual_sum(res, 0, a.vocab, a.vocab, red);
      }
    }
    if (c == kNone) break;
    rejected = 0;
    cur = c;
    if (part == 0 && t == 0) path[count] = c;
    ++count;
  }

  Residual<DTYPE, DRAFT> res(a, b, cur);
  const int lo = part * a.part, hi = min(lo + a.part, a.vocab);
  res.rejected = rejected;
  res.inverse = inverse;
  if (!DRAFT && !full) {
    res.n_gone = gone_tokens(s, m, cur, lo, hi, sibling, &n_gone);
    res.gone = sibling;
  }
  const double sum = residual_sum(res, lo, hi, a.vocab, red);
  if (t == 0) gptr(a.sums)[(size_t)b * a.parts + part] = sum;
  if (part != 0) return;
  for (int i = count + t; i < a.n_path; i += kThreads) path[i] = -1;
  for (int i = t; i < rejected; i += kThreads) gptr(a.inverse)[(size_t)b * a.n + i] = inverse[i];
  if (t == 0) {
    gptr(a.count)[b] = count;
    RQ_GLOBAL int32_t* found = gptr(a.found) + b * 4;
    found[0] = cur;
    found[1] = rejected;
    found[2] = full;
  }
}

// The token: the first whose running sum exceeds u times the whole.
template <int DTYPE, bool DRAFT>
__global__ void __launch_bounds__(kThreads) tree_select_kernel(TreeVerifyLaunch a) {
  __shared__ Nodes s;
  __shared__ int gone[RQ_MAX_NODES];
  __shared__ double inverse[RQ_MAX_NODES];
  __shared__ double sums[kVerifyParts], red[kThreads / 64];
  __shared__ int n_gone, at_first, at_last;
  const int b = blockIdx.x, t = threadIdx.x;
  const int m = node_count(a.new_len, b, a.n);
  if (m == 0) {
    if (t == 0) gptr(a.next)[b] = -1;
    return;
  }
  const RQ_GLOBAL int32_t* found = gptr(a.found) + b * 4;
  const int cur = found[0], full = found[2];
  Residual<DTYPE, DRAFT> res(a, b, cur);
  res.rejected = found[1];
  res.inverse = inverse;
  res.gone = gone;
  for (int i = t; i < res.rejected; i += kThreads) inverse[i] = gptr(a.inverse)[(size_t)b * a.n + i];
  if (!DRAFT && t < m) {
    s.parent[t] = t == 0 ? -1 : parent_of(a.parents, b, a.n, t);
    const int x = gptr(a.tokens)[(size_t)b * a.n + t];
    s.token[t] = x < 0 ? 0 : (x < a.vocab ? x : a.vocab - 1);
  }
  if (t < a.parts) sums[t] = gptr(a.sums)[(size_t)b * a.parts + t];
  if (t == 0) {
    at_first = kNone;
    at_last = -1;
  }
  __syncthreads();
  double whole = 0.0;
  for (int i = 0; i < a.parts; ++i) whole += sums[i];
  bool taken = !DRAFT && !full;           // the children's tokens are
  if (!(whole > 0.0)) {
    // no mass left: the target's row
    res.rejected = 0;
    taken = false;
    whole = 0.0;
    for (int i = 0; i < a.parts; ++i) {
      const int lo = i * a.part;
      const double sum = residual_sum(res, lo, min(lo + a.part, a.vocab), a.vocab, red);
      if (t == 0) sums[i] = sum;
      whole += sum;
    }
    __syncthreads();
    if (!(whole > 0.0)) {
      if (t == 0) gptr(a.next)[b] = 0;
      return;
    }
  }
  const double bar = (double)gptr(a.uniforms)[(size_t)b * a.n] * whole;
  int part = -1, last = 0;
  double before = 0.0, run = 0.0;
  for (int i = 0; i < a.parts; ++i) {
    if (sums[i] > 0.0) last = i;
    if (part < 0 && run + sums[i] > bar) {
      part = i;
      before = run;
    }
    run += sums[i];
  }
  if (part < 0) {
    part = last;
    before = -1.0;                        // (none exceeds: the last of r > 0)
  }
  const int lo = part * a.part, hi = min(lo + a.part, a.vocab);
  if (taken) res.n_gone = gone_tokens(s, m, cur, lo, hi, gone, &n_gone);
  for (int v0 = lo; v0 < hi; v0 += kVerifyStep) {
    const int v = v0 + t * kEach;
    double r[kEach], mine = 0.0;
    if (v < hi) {
      res.load(v, a.vocab, r);
    } else {
#pragma unroll
      for (int i = 0; i < kEach; ++i) r[i] = 0.0;
    }
#pragma unroll
    for (int i = 0; i < kEach; ++i) mine += r[i];
    // the sum before this thread's entries
    double upto = mine;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const double x = __shfl_up(upto, d);
      if ((t & 63) >= d) upto += x;
    }
    __syncthreads();
    if ((t & 63) == 63) red[t >> 6] = upto;
    __syncthreads();
    double base = before, all = 0.0;
    for (int w = 0; w < kThreads / 64; ++w) {
      if (w < (t >> 6)) base += red[w];
      all += red[w];
    }
    double x = base + (upto - mine);
    int first = kNone, end = -1;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      x += r[i];
      if (r[i] > 0.0) {
        end = v + i;
        if (first == kNone && before >= 0.0 && x > bar) first = v + i;
      }
    }
    if (first != kNone) atomicMin(&at_first, first);
    if (end >= 0) atomicMax(&at_last, end);
    __syncthreads();
    if (at_first != kNone) break;
    if (before >= 0.0) before += all;
  }
  if (t == 0) gptr(a.next)[b] = at_first != kNone ? at_first : (at_last >= 0 ? at_last : 0);
}

template <int DTYPE, bool DRAFT>
hipError_t launch(const TreeVerifyLaunch& a, hipStream_t s) {
  hipLaunchKernelGGL((tree_walk_kernel<DTYPE, DRAFT>), dim3(a.parts, a.B), dim3(kThreads), 0, s, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((tree_select_kernel<DTYPE, DRAFT>), dim3(a.B), dim3(kThreads), 0, s, a);
  return hipGetLastError();
}

template <int DTYPE>
hipError_t launch(const TreeVerifyLaunch& a, hipStream_t s) {
  return a.draft ? launch<DTYPE, true>(a, s) : launch<DTYPE, false>(a, s);
}

}  // namespace

hipError_t launch_tree_mask(const TreeMaskLaunch& a, hipStream_t s) {
  hipLaunchKernelGGL(tree_mask_kernel, dim3((a.n + kMaskThreads - 1) / kMaskThreads, a.B), dim3(kMaskThreads), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_tree_verify(const TreeVerifyLaunch& a, hipStream_t s) {
  if (a.dtype == RQ_F32) return launch<RQ_F32>(a, s);
  return a.dtype == RQ_F16 ? launch<RQ_F16>(a, s) : launch<RQ_BF16>(a, s);
}

}  // namespace rq
