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
// its own word, twice as far a step (5 at most), which gives that word's bits and the
// ancestor where the chain leaves it; a row then goes from word to word by those (at
// most 31 steps more).  Bound by latency.
constexpr int kMaskThreads = 256;

__global__ void __launch_bounds__(kMaskThreads) tree_mask_kernel(TreeMaskLaunch a) {
  __shared__ int32_t parent[RQ_MAX_NODES];
  __shared__ uint32_t bits[RQ_MAX_NODES];
  __shared__ int32_t leave[RQ_MAX_NODES];     // the chain's first node before the word, or -1
  const int b = blockIdx.y, m = node_count(a.new_len, b, a.n);
  const int first = blockIdx.x * kMaskThreads, end = min(first + kMaskThreads, m);
  if (first >= m) return;
  for (int i = threadIdx.x; i < end; i += kMaskThreads) parent[i] = parent_of(a.parents, b, a.n, i);
  // most words of a row of many are zero: the workgroup's rows first, then its chains
  RQ_GLOBAL uint32_t* rows = gptr(a.mask) + ((size_t)b * a.n + first) * a.words;
  if (a.words > 2) {
    const int all = (end - first) * a.words;
    for (int i = 4 * threadIdx.x; i < all; i += 4 * kMaskThreads) {
      if (i + 4 <= all)
        *(RQ_GLOBAL u4_any*)(rows + i) = (u4){0u, 0u, 0u, 0u};
      else
        for (int k = i; k < all; ++k) rows[k] = 0u;
    }
  }
  __syncthreads();
  for (int i0 = 0; i0 < end; i0 += kMaskThreads) {       // (a word's nodes are lanes of one wave)
    const int i = i0 + threadIdx.x, lane = threadIdx.x & 63;
    uint32_t w = 1u << (i & 31);
    int j = i < end ? parent[i] : -1;
    while (__any(j >= (i & ~31))) {
      const bool inside = j >= (i & ~31);
      const uint32_t more = __shfl(w, inside ? j & 63 : lane);
      const int next = __shfl(j, inside ? j & 63 : lane);
      if (inside) {
        w |= more;
        j = next;
      }
    }
    if (i < end) {
      bits[i] = w;
      leave[i] = j;
    }
  }
  __syncthreads();
  const int i = first + threadIdx.x;
  if (i >= end) return;
  RQ_GLOBAL uint32_t* row = rows + threadIdx.x * a.words;
  int count = 0;
  if (a.words <= 2)
    for (int w = 0; w < a.words; ++w) row[w] = 0u;
  for (int j = i; j >= 0; j = leave[j]) {
    row[j >> 5] = bits[j];
    count += __popc(bits[j]);
  }
  if (a.depth) gptr(a.depth)[(size_t)b * a.n + i] = count - 1;
}

// --------------------------------------------------------------- verification
// Walk: from the root, the children of the last accepted node in order,
//   accept child c where u_c q(x) s < r(x);   r <- max(0, r / s - q), s <- sum r
// (q = 1 and r(x) <- 0, s <- max(0, s - r(x)) without the draft's rows).  A test needs
// one entry of each row, which all nodes load at once; without the draft's rows the
// mass before each test is a sum over the earlier siblings, so all tests are decided
// before the walk.  With them a rejection that leaves a sibling to test needs the
// residual's sum over a whole row, and so does the last token.
//
// A sequence's workgroups, a part of the rows each, all walk by themselves, to the same
// end.  For a sum each adds its part, puts it where the others see it and waits for
// theirs; what does not come in time (a workgroup that does not run) it adds itself, in
// the same order.  So no wait is without an end, and the results are the same either
// way.  The one whose part holds the last token finds it.  The last to finish clears
// what was put down.
//
// All sums are fp64 in one order: the results are decisions, which fp32 sums would make
// otherwise next to a border.  Bound by latency: launch, nodes, entries, a row's part,
// the parts' exchange.
constexpr int kThreads = 1024, kEach = kVerifyStep / kThreads;
constexpr int kNone = 1 << 30;
constexpr int kPolls = 4096;      // some milliseconds

template <int DTYPE>
struct Prob {
  typedef uint16_t type;
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

// Entries v..v + 7 of a row; zeros behind its end.
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
      const u4 y = *(const RQ_GLOBAL u4_any*)(row + v);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        x[2 * j] = widen_t<DTYPE == RQ_BF16>(y[j] & 0xffffu);
        x[2 * j + 1] = widen_t<DTYPE == RQ_BF16>(y[j] >> 16);
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
  const int* gone;          // without: the tokens taken out (LDS),
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
        if (at >= 0 && at < kEach) {
#pragma unroll
          for (int i = 0; i < kEach; ++i)
            if (at == i) r[i] = 0.0;
        }
      }
    }
  }
};

// Register moves of doubles (see row_all and its like): CTRL of a lane's row; rows
// outside ROWS, and lanes without a source, get 0.
template <int CTRL, int ROWS>
__device__ __forceinline__ double moved_d(double x) {
  const u2 w = __builtin_bit_cast(u2, x);
  return __builtin_bit_cast(double, (u2){(uint32_t)__builtin_amdgcn_update_dpp(0, (int)w.x, CTRL, ROWS, 0xf, true),
                                         (uint32_t)__builtin_amdgcn_update_dpp(0, (int)w.y, CTRL, ROWS, 0xf, true)});
}
// Sums up to each lane, it included.
__device__ __forceinline__ double wave_scan(double x) {
  x += moved_d<0x111, 0xf>(x);          // 1, 2, 4 and 8 lanes before, in a row of 16,
  x += moved_d<0x112, 0xf>(x);
  x += moved_d<0x114, 0xf>(x);
  x += moved_d<0x118, 0xf>(x);
  x += moved_d<0x142, 0xa>(x);          // the last of rows 0 and 2 to the next ones,
  return x + moved_d<0x143, 0xc>(x);    // the first half's last to the second half
}

template <int DTYPE, bool DRAFT>
__global__ void __launch_bounds__(kThreads) tree_verify_kernel(TreeVerifyLaunch a) {
  __shared__ __align__(16) int parent[RQ_MAX_NODES], token[RQ_MAX_NODES];
  __shared__ __align__(16) float p[RQ_MAX_NODES], q[RQ_MAX_NODES];   // of a node's token, in its parent's rows
  __shared__ float u[RQ_MAX_NODES];
  __shared__ int child[RQ_MAX_NODES];     // the first child (without a draft: the first accepted one)
  __shared__ int sibling[RQ_MAX_NODES];   // the next one
  __shared__ double inverse[RQ_MAX_NODES];
  __shared__ double waves[kThreads / 64], sums[kVerifyParts];
  __shared__ int here[kVerifyParts];
  __shared__ int n_gone, at_first, at_last;
  const int b = blockIdx.y, part = blockIdx.x, t = threadIdx.x;
  int up = -1;
  if (t < a.n) {                          // (at most as many nodes as threads)
    const size_t at = (size_t)b * a.n + t;
    int x = gptr(a.tokens)[at];
    up = t == 0 ? -1 : parent_of(a.parents, b, a.n, t);
    x = x < 0 ? 0 : (x < a.vocab ? x : a.vocab - 1);
    parent[t] = up;
    token[t] = x;
    u[t] = gptr(a.uniforms)[at];
    child[t] = kNone;
    sibling[t] = -1;
  }
  const int m = node_count(a.new_len, b, a.n);
  RQ_GLOBAL int32_t* path = gptr(a.path) + (size_t)b * a.n_path;
  if (m == 0) {
    if (part == 0) {
      if (t < a.n_path) path[t] = -1;
      if (t == 0) {
        gptr(a.count)[b] = 0;
        gptr(a.next)[b] = -1;
      }
    }
    return;
  }
  if (t >= m) up = -1;
  if (up >= 0) {
    const Residual<DTYPE, DRAFT> row(a, b, up);
    p[t] = prob<DTYPE>(row.target + token[t]);
    if (DRAFT) q[t] = prob<DTYPE>(row.draft + token[t]);
  }
  __syncthreads();
  // Each node's earlier siblings, found by 2^spread threads: every 2^spread-th node
  // before it is one's, eight at a time (LDS reads are slow one by one).
  const int spread = a.spread, node = t >> spread, slice = t & ((1 << spread) - 1);
  const int mother = node < m ? parent[node] : -1;
  auto earlier = [&](auto f) {
    if (mother >= 0)
      for (int j0 = slice; j0 < node; j0 += 8 << spread) {
        int j[8], of[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          j[i] = j0 + (i << spread);
          of[i] = parent[j[i] < node ? j[i] : 0];       // (the root has none)
        }
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (of[i] == mother) f(j[i]);
      }
  };
  if constexpr (DRAFT) {
    earlier([&](int j) { atomicMax(&sibling[node], j); });         // (the one before, at first)
    __syncthreads();
    const int before = t < m ? sibling[t] : -1;
    __syncthreads();
    if (t < m) sibling[t] = kNone;
    __syncthreads();
    if (up >= 0) {
      if (before < 0)
        child[up] = t;
      else
        sibling[before] = t;
    }
  } else {
    // a token that an earlier sibling has is gone by its turn
    bool twice = false;
    const int x = node < m ? token[node] : 0;
    earlier([&](int j) { twice |= token[j] == x; });
    const uint64_t group = (2ull << ((1 << spread) - 1)) - 1;      // 2^spread lanes
    twice = (__ballot(twice) >> (t & 63 & ~((1 << spread) - 1))) & group;
    if (mother >= 0 && slice == 0) q[node] = twice ? 0.0f : p[node];
    __syncthreads();
    double taken = 0.0;
    earlier([&](int j) { taken += (double)q[j]; });
    for (int d = 1; d < 1 << spread; d <<= 1) taken += __shfl_xor(taken, d);
    const double mass = taken < 1.0 ? 1.0 - taken : 0.0;
    if (mother >= 0 && slice == 0 && (double)u[node] * mass < (double)q[node]) atomicMin(&child[mother], node);
  }
  __syncthreads();

  // the workgroup's sum of a part, in every thread
  auto part_sum = [&](const Residual<DTYPE, DRAFT>& res, int i) {
    const int lo = i * a.part, hi = min(lo + a.part, a.vocab);
    double sum = 0.0;
    for (int v = lo + t * kEach; v < hi; v += kVerifyStep) {
      double r[kEach];
      res.load(v, a.vocab, r);
#pragma unroll
      for (int k = 0; k < kEach; ++k) sum += r[k];
    }
    sum = wave_scan(sum);
    __syncthreads();
    if ((t & 63) == 63) waves[t >> 6] = sum;
    __syncthreads();
    sum = 0.0;
#pragma unroll
    for (int w = 0; w < kThreads / 64; ++w) sum += waves[w];
    return sum;
  };
  // All parts' sums, in `sums`, and the whole.  (A sum is not negative: with its sign
  // set it is no zero, which stands for one that is not there.)
  int asked = 0;
  RQ_GLOBAL uint64_t* slots = gptr(a.slots) + (size_t)b * kVerifySums * a.parts;
  auto all_sums = [&](const Residual<DTYPE, DRAFT>& res) {
    double mine = part_sum(res, part);
    mine = mine > 0.0 ? mine : 0.0;       // (no NaN either)
    const bool shared = asked < kVerifySums;
    RQ_GLOBAL uint64_t* slot = slots + (size_t)asked * a.parts;
    ++asked;
    if (shared && t == 0 && a.parts > 1)
      __hip_atomic_store(slot + part, __builtin_bit_cast(uint64_t, mine) | 1ull << 63, __ATOMIC_RELAXED,
                         __HIP_MEMORY_SCOPE_AGENT);
    if (t < a.parts) {
      uint64_t x = 0;
      if (shared && t != part)
        for (int i = 0; i < kPolls && x == 0; ++i)
          x = __hip_atomic_load(slot + t, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      sums[t] = t == part ? mine : __builtin_bit_cast(double, x & ~(1ull << 63));
      here[t] = t == part || x != 0;
    }
    __syncthreads();
    double whole = 0.0;
    for (int i = 0; i < a.parts; ++i) {
      if (!here[i]) {                     // (the same in every thread)
        double sum = part_sum(res, i);
        sum = sum > 0.0 ? sum : 0.0;
        if (t == 0) sums[i] = sum;
        whole += sum;
      } else {
        whole += sums[i];
      }
    }
    __syncthreads();
    return whole;
  };

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
        mass = all_sums(res);
      }
    }
    if (c == kNone) break;
    rejected = 0;
    cur = c;
    if (part == 0 && t == 0) path[count] = c;
    ++count;
  }
  if (part == 0) {
    for (int i = count + t; i < a.n_path; i += kThreads) path[i] = -1;
    if (t == 0) gptr(a.count)[b] = count;
  }

  // the last token: the first whose running sum exceeds u times the whole
  if (t == 0) {
    n_gone = 0;
    at_first = kNone;
    at_last = -1;
  }
  __syncthreads();
  Residual<DTYPE, DRAFT> res(a, b, cur);
  res.rejected = rejected;
  res.inverse = inverse;
  if (!DRAFT && !full) {
    if (t < m && up == cur) sibling[atomicAdd(&n_gone, 1)] = token[t];     // (the children's tokens)
    __syncthreads();
    res.n_gone = n_gone;
    res.gone = sibling;
  }
  double whole = all_sums(res);
  if (!(whole > 0.0)) {                   // no mass left: the target's row
    res.rejected = res.n_gone = 0;
    whole = all_sums(res);
  }
  if (a.parts > 1 && t == 0) {
    // the last of the sequence's workgroups to come here clears the slots
    __builtin_amdgcn_s_waitcnt(0);        // this one's sums are out
    RQ_GLOBAL uint32_t* done = gptr(a.done) + b;
    if (__hip_atomic_fetch_add(done, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (uint32_t)a.parts - 1) {
      const int used = (asked < kVerifySums ? asked : kVerifySums) * a.parts;
      for (int i = 0; i < used; ++i) __hip_atomic_store(slots + i, 0ull, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      __hip_atomic_store(done, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
  }
  const double bar = (double)u[0] * whole;
  int holds = -1, last = 0;
  double before = 0.0, run = 0.0;
  for (int i = 0; i < a.parts; ++i) {
    if (sums[i] > 0.0) last = i;
    if (holds < 0 && run + sums[i] > bar) {
      holds = i;
      before = run;
    }
    run += sums[i];
  }
  const bool beyond = holds < 0;          // (none exceeds: the last of r > 0)
  if (beyond) holds = last;
  if (part != holds) return;
  if (!(whole > 0.0)) {
    if (t == 0) gptr(a.next)[b] = 0;
    return;
  }
  const int lo = part * a.part, hi = min(lo + a.part, a.vocab);
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
    const double upto = wave_scan(mine);
    __syncthreads();
    if ((t & 63) == 63) waves[t >> 6] = upto;
    __syncthreads();
    double x = before + (upto - mine), all = 0.0;     // the sum before this thread's entries
#pragma unroll
    for (int w = 0; w < kThreads / 64; ++w) {
      x += w < (t >> 6) ? waves[w] : 0.0;
      all += waves[w];
    }
    int first = kNone, end = -1;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      x += r[i];
      if (r[i] > 0.0) {
        end = v + i;
        if (first == kNone && !beyond && x > bar) first = v + i;
      }
    }
    if (first != kNone) atomicMin(&at_first, first);
    if (end >= 0) atomicMax(&at_last, end);
    __syncthreads();
    if (at_first != kNone) break;
    before += all;
  }
  if (t == 0) gptr(a.next)[b] = at_first != kNone ? at_first : (at_last >= 0 ? at_last : 0);
}

template <int DTYPE, bool DRAFT>
hipError_t launch(const TreeVerifyLaunch& a, hipStream_t s) {
  hipLaunchKernelGGL((tree_verify_kernel<DTYPE, DRAFT>), dim3(a.parts, a.B), dim3(kThreads), 0, s, a);
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
