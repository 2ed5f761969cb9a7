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
// most 31 steps more).  Bound by the launch and latency: 16 trees of 64 nodes 2.4 us,
// eight of 1000 3.8, a chain of 1024 8.0 (followed node by node in its words 12.8).
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
// the parts' exchange.  So what LDS is read for one by one counts: which first children
// are accepted is decided by their threads, a walk then reads one word a node; a lane
// has a part's sum, and scans find the whole and the part of the last token.  us so / one
// by one: 32 chains of 6 nodes 8.7 / 11.1, four trees of 31 over 100003 tokens 10.9 /
// 15.8, 16 of 64 without a draft's rows over 131072 9.9 / 14.0.
constexpr int kThreads = 1024, kEach = kVerifyStep / kThreads;
constexpr int kNone = 1 << 30;
constexpr int kPolls = 128;       // 15 us of polling; a part that is computed instead takes about one

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

  // Rejections j and on.
  __device__ __forceinline__ void reject(int j, const float q[kEach], double r[kEach]) const {
    for (; j < rejected; ++j) {
      const double by = inverse[j];
#pragma unroll
      for (int i = 0; i < kEach; ++i) {
        const double x = r[i] * by - (double)q[i];
        r[i] = x > 0.0 ? x : 0.0;
      }
    }
  }

  // Entries v..v + 7, and the draft's where it has a part in them.
  __device__ __forceinline__ void load(int v, int vocab, float q[kEach], double r[kEach]) const {
    float p[kEach];
    load_probs<DTYPE>(target, v, vocab, p);
    if (DRAFT && rejected) load_probs<DTYPE>(draft, v, vocab, q);
#pragma unroll
    for (int i = 0; i < kEach; ++i) r[i] = p[i];
    if constexpr (DRAFT) {
      reject(0, q, r);
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
  __shared__ int child[RQ_MAX_NODES];     // the first child, ~ of it where it is rejected (without a draft: the first accepted one)
  __shared__ int sibling[RQ_MAX_NODES];   // the next one
  __shared__ double inverse[RQ_MAX_NODES];
  __shared__ double waves[2][kThreads / 64], sums[64];
  __shared__ uint64_t there;
  __shared__ int n_gone, at_first, at_last;
  static_assert(kVerifyParts <= 64, "a lane a part");
  const int b = blockIdx.y, part = blockIdx.x, t = threadIdx.x;
  int up = -1;
  if (t < a.n) {                          // (at most as many nodes as threads)
    const size_t at = (size_t)b * a.n + t;
    int x = gptr(a.tokens)[at];
    up = t == 0 ? -1 : parent_of(a.parents, b, a.n, t);
    x = x < 0 ? 0 : (x < a.vocab ? x : a.vocab - 1);
    parent[t] = up;
    token[t] = x;
    const float number = gptr(a.uniforms)[at];
    u[t] = number > 0.0f ? __builtin_fminf(number, 1.0f) : 0.0f;     // (NaN as 0)
    child[t] = sibling[t] = kNone;
  }
  if (t == 0) {
    n_gone = 0;
    at_first = kNone;
    at_last = -1;
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
  auto earlier = [&](const auto* values, auto f) {
    if (mother >= 0)
      for (int j0 = slice; j0 < node; j0 += 8 << spread) {
        int of[8];
        auto x = *values;
        decltype(x) value[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int j = j0 + (i << spread);
          of[i] = parent[j < node ? j : 0];             // (the root has none)
          value[i] = values[j < node ? j : 0];
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) f(of[i] == mother, j0 + (i << spread), value[i]);
      }
  };
  if constexpr (DRAFT) {
    int before = -1;
    earlier(parent, [&](bool is, int j, int) { before = is ? j : before; });
    for (int d = 1; d < 1 << spread; d <<= 1) before = max(before, __shfl_xor(before, d));
    if (mother >= 0 && slice == 0) {
      if (before < 0)
        child[mother] = (double)u[node] * (double)q[node] < (double)p[node] ? node : ~node;
      else
        sibling[before] = node;
    }
  } else {
    // a token that an earlier sibling has is gone by its turn
    bool twice = false;
    const int x = node < m ? token[node] : 0;
    earlier(token, [&](bool is, int, int y) { twice |= is && y == x; });
    const uint64_t group = (2ull << ((1 << spread) - 1)) - 1;      // 2^spread lanes
    twice = (__ballot(twice) >> (t & 63 & ~((1 << spread) - 1))) & group;
    if (mother >= 0 && slice == 0) q[node] = twice ? 0.0f : p[node];
    __syncthreads();
    double taken = 0.0;
    earlier(q, [&](bool is, int, float y) { taken += is ? (double)y : 0.0; });
    for (int d = 1; d < 1 << spread; d <<= 1) taken += __shfl_xor(taken, d);
    const double mass = taken < 1.0 ? 1.0 - taken : 0.0;
    if (mother >= 0 && slice == 0 && (double)u[node] * mass < (double)q[node]) atomicMin(&child[mother], node);
  }
  __syncthreads();

  // A part of one step stays in registers, for the node's next rejection and the last
  // token: after `applied` rejections, or -1.
  const int lo = part * a.part, hi = min(lo + a.part, a.vocab);
  const bool held = a.part <= kVerifyStep;
  double r[kEach];
  float q_held[kEach];
  int applied = -1, turn = 0;

  // the workgroup's sum of a part, in every thread
  auto part_sum = [&](const Residual<DTYPE, DRAFT>& res, int i) {
    double sum = 0.0;
    if (held && i == part) {
      if (applied >= 0) {
        res.reject(applied, q_held, r);
      } else if (lo + t * kEach < hi) {
        res.load(lo + t * kEach, a.vocab, q_held, r);
      } else {
#pragma unroll
        for (int k = 0; k < kEach; ++k) r[k] = q_held[k] = 0.0f;
      }
      applied = res.rejected;
#pragma unroll
      for (int k = 0; k < kEach; ++k) sum += r[k];
    } else {
      const int end = min(i * a.part + a.part, a.vocab);
      for (int v = i * a.part + t * kEach; v < end; v += kVerifyStep) {
        double x[kEach];
        float y[kEach];
        res.load(v, a.vocab, y, x);
#pragma unroll
        for (int k = 0; k < kEach; ++k) sum += x[k];
      }
    }
    sum = wave_scan(sum);
    double* each = waves[turn];           // (by turns: those of the last sum may be read still)
    turn ^= 1;
    if ((t & 63) == 63) each[t >> 6] = sum;
    __syncthreads();
    sum = 0.0;
#pragma unroll
    for (int w = 0; w < kThreads / 64; ++w) sum += each[w];
    return sum > 0.0 ? sum : 0.0;         // (no NaN)
  };
  // All parts' sums, in `sums`, those up to a lane's part, in `upto`, and the whole.  (A
  // sum is not negative: with its sign set it is no zero, which stands for one that is
  // not there.)
  int asked = 0;
  double upto = 0.0;
  RQ_GLOBAL uint64_t* slots = gptr(a.slots) + (size_t)b * kVerifySums * a.parts;
  auto all_sums = [&](const Residual<DTYPE, DRAFT>& res) {
    const double mine = part_sum(res, part);
    const bool shared = asked < kVerifySums;
    RQ_GLOBAL uint64_t* slot = slots + (size_t)asked * a.parts;
    ++asked;
    if (shared && t == 0 && a.parts > 1)
      __hip_atomic_store(slot + part, __builtin_bit_cast(uint64_t, mine) | 1ull << 63, __ATOMIC_RELAXED,
                         __HIP_MEMORY_SCOPE_AGENT);
    if (t < 64) {
      uint64_t x = t < a.parts && t != part ? 0 : 1ull << 63;
      if (shared && x == 0)
        for (int i = 0; i < kPolls && x == 0; ++i)
          x = __hip_atomic_load(slot + t, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      sums[t] = t == part ? mine : __builtin_bit_cast(double, x & ~(1ull << 63));
      const uint64_t all = __ballot(x != 0);
      if (t == 0) there = all;
    }
    __syncthreads();
    const uint64_t missing = ~there;      // (the same in every thread)
    if (missing) {
      for (int i = 0; i < a.parts; ++i)
        if ((missing >> i) & 1) {
          const double sum = part_sum(res, i);
          if (t == 0) sums[i] = sum;
        }
      __syncthreads();
    }
    upto = wave_scan(sums[t & 63]);
    return __shfl(upto, 63);
  };

  // the walk, alike in every thread
  int cur = 0, count = 1, rejected = 0;
  bool full = false;
  if (part == 0 && t == 0) path[0] = 0;
  for (;;) {
    full = count == a.n_path;
    if (full) break;
    int c = child[cur];
    if (DRAFT && c < 0) {
      Residual<DTYPE, DRAFT> res(a, b, cur);
      res.inverse = inverse;
      double mass = 1.0;
      c = ~c;
      for (;;) {                          // c is rejected
        if (t == 0) inverse[rejected] = rejected == 0 ? 1.0 : (mass > 0.0 ? 1.0 / mass : 0.0);
        res.rejected = ++rejected;
        c = sibling[c];
        if (c == kNone) break;
        if (mass == 0.0) {                // (none of the others is accepted)
          c = kNone;
          break;
        }
        const double by = (double)u[c] * (double)q[c];
        double left = p[c];
        __syncthreads();
        mass = all_sums(res);
        for (int j = 0; j < rejected; ++j) {
          left = left * inverse[j] - (double)q[c];
          left = left > 0.0 ? left : 0.0;
        }
        if (by * mass < left) break;
      }
    }
    if (c == kNone) break;
    rejected = 0;
    applied = -1;
    cur = c;
    if (part == 0 && t == 0) path[count] = c;
    ++count;
  }
  if (part == 0) {
    for (int i = count + t; i < a.n_path; i += kThreads) path[i] = -1;
    if (t == 0) gptr(a.count)[b] = count;
  }

  // the last token: the first whose running sum exceeds u times the whole
  Residual<DTYPE, DRAFT> res(a, b, cur);
  res.rejected = rejected;
  res.inverse = inverse;
  if (!DRAFT && !full && t < m && up == cur) sibling[atomicAdd(&n_gone, 1)] = token[t];     // (the children's tokens)
  __syncthreads();
  if (!DRAFT) {
    res.n_gone = n_gone;
    res.gone = sibling;
  }
  double whole = all_sums(res);
  if (!(whole > 0.0)) {                   // no mass left: the target's row
    res.rejected = res.n_gone = 0;
    applied = -1;
    whole = all_sums(res);
  }
  // the last of the sequence's workgroups to come here clears the slots, at its end
  uint32_t ticket = 0;
  if (a.parts > 1 && t == 0) {
    __builtin_amdgcn_s_waitcnt(0);        // this one's sums are out
    ticket = __hip_atomic_fetch_add(gptr(a.done) + b, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
  auto finish = [&] {
    if (a.parts > 1 && t < 64 && __builtin_amdgcn_readfirstlane(ticket) == (uint32_t)a.parts - 1) {
      const int used = (asked < kVerifySums ? asked : kVerifySums) * a.parts;
      for (int i = t; i < used; i += 64) __hip_atomic_store(slots + i, 0ull, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      if (t == 0) __hip_atomic_store(gptr(a.done) + b, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
  };
  const double bar = (double)u[0] * whole;
  const uint64_t parts = ~0ull >> (64 - a.parts);
  const uint64_t exceed = __ballot(upto > bar) & parts, some = __ballot(sums[t & 63] > 0.0) & parts;
  const bool beyond = exceed == 0;        // (none exceeds: the last of r > 0)
  const int holds = beyond ? (some ? 63 - __builtin_clzll(some) : 0) : __builtin_ctzll(exceed);
  if (part != holds) {
    finish();
    return;
  }
  double before = holds > 0 ? __shfl(upto, holds - 1) : 0.0;
  for (int v0 = lo; v0 < hi; v0 += kVerifyStep) {
    const int v = v0 + t * kEach;
    double mine = 0.0;
    if (!held) {
      if (v < hi) {
        res.load(v, a.vocab, q_held, r);
      } else {
#pragma unroll
        for (int i = 0; i < kEach; ++i) r[i] = 0.0;
      }
    }
#pragma unroll
    for (int i = 0; i < kEach; ++i) mine += r[i];
    const double scan = wave_scan(mine);
    double* each = waves[turn];
    turn ^= 1;
    if ((t & 63) == 63) each[t >> 6] = scan;
    __syncthreads();
    double x = before + (scan - mine), all = 0.0;     // the sum before this thread's entries
#pragma unroll
    for (int w = 0; w < kThreads / 64; ++w) {
      x += w < (t >> 6) ? each[w] : 0.0;
      all += each[w];
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
    // (a wave's first and last, where it has any)
    const uint64_t firsts = __ballot(first != kNone), ends = __ballot(end >= 0);
    if (firsts && (t & 63) == __builtin_ctzll(firsts)) atomicMin(&at_first, first);
    if (ends && (t & 63) == 63 - __builtin_clzll(ends)) atomicMax(&at_last, end);
    __syncthreads();
    if (at_first != kNone) break;
    before += all;
  }
  if (t == 0) gptr(a.next)[b] = at_first != kNone ? at_first : (at_last >= 0 ? at_last : 0);
  finish();
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
