// Which drafted tokens stay, and the token that follows.
//
// What happens at a node depends on the node's own rows and the given numbers alone, not on how the walk got there: so a workgroup has a node, and a walk over what they found (a node onward, or
// a token) is a second launch.  A node that the walk cannot come to ends at once: each of its ancestors is asked what a first child needs, two numbers.  At a node whose first child is taken nothing more is read.  A child that is
// not taken costs a pass over both rows, in which wave w has the w-th part: the sums of these parts are what the token is looked for in, if no other child is taken.  Children that were chosen, not drawn, cost
// one pass together.
//
// Measured (kernels alone, under the profiler): 64 trees of up to 26 nodes, rows of 131 072 in 32 bits, 61 us and 5 for the walk: the nodes with most refusals, some 10 us a pass (a compute unit's memory and 64-bit instructions
// about alike), while others are done; what is read, about 100 MB, would take the whole card 20.  16 trees of up to 40 nodes, chosen children, rows of 100 003 in bfloat16, 20 us; a chain of 8, rows of 32 003, 13 us: dependent
// loads and one pass.
#pragma once
#include "draft_attend.hpp"

namespace spg {

constexpr int kVerifyThreads = 1024, kVerifyWaves = kVerifyThreads / kWave;

struct VerifyArgs {
  TreeView trees;
  const void *target, *draft;              // draft: null where children were chosen, not drawn
  int64_t target_stride, draft_stride;     // elements
  int vocab;
  const int32_t* ids;
  const float* u;
  int2* onward;                            // tokens: the child that is taken or -1, and then the token that follows
  int32_t *path, *kept, *next;
};

// An entry of a row: what is negative or NaN counts as 0 (a maximum of NaN and 0 is 0).  In the loops that is taken in 64 bits, where it is one instruction; in 32 bits a second one first
// quiets NaN (64 trees over 131 072 tokens 62.5 -> 60.8 us).
template <typename T> __device__ __forceinline__ float proper(T v) { return fmaxf((float)v, 0.0f); }
__device__ __forceinline__ double proper64(float v) { return fmax((double)v, 0.0); }

template <typename T>
struct Loaded {            // 16 bytes of a row, which may begin at any element
  static constexpr int kCount = 16 / sizeof(T);
  T v[kCount];
};
template <typename T>
__device__ __forceinline__ Loaded<T> load_some(const T* row, int64_t at, int vocab) {
  Loaded<T> r;
  if (at + Loaded<T>::kCount <= vocab) {
    __builtin_memcpy(&r, row + at, 16);
  } else {
#pragma unroll
    for (int i = 0; i < Loaded<T>::kCount; ++i) r.v[i] = at + i < vocab ? row[at + i] : T(0);
  }
  return r;
}

// Sums of 64 bits over the lanes up to each, by moves within the registers.
template <int CTRL, int ROWS, bool BOUND>
__device__ __forceinline__ double from_lanes(double v) {
  const uint64_t u = __builtin_bit_cast(uint64_t, v);
  const unsigned lo = __builtin_amdgcn_update_dpp(0, (int)u, CTRL, ROWS, 0xf, BOUND), hi = __builtin_amdgcn_update_dpp(0, (int)(u >> 32), CTRL, ROWS, 0xf, BOUND);
  return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
__device__ __forceinline__ double row_scan(double v) {      // over the 16 lanes of a row
  v += from_lanes<0x111, 0xf, true>(v);
  v += from_lanes<0x112, 0xf, true>(v);
  v += from_lanes<0x114, 0xf, true>(v);
  return v + from_lanes<0x118, 0xf, true>(v);
}
__device__ __forceinline__ double wave_scan(double v) {
  v = row_scan(v);
  v += from_lanes<0x142, 0xa, false>(v);      // the last lane of rows 0 and 2 to rows 1 and 3, then of row 1 to rows 2 and 3
  return v + from_lanes<0x143, 0xc, false>(v);
}
__device__ __forceinline__ double lane_of(double v, int lane) {
  const uint64_t u = __builtin_bit_cast(uint64_t, v);
  return __builtin_bit_cast(double, (uint64_t)(unsigned)__builtin_amdgcn_readlane((int)(u >> 32), lane) << 32 | (unsigned)__builtin_amdgcn_readlane((int)u, lane));
}
__device__ __forceinline__ double wave_sum(double v) { return lane_of(wave_scan(v), kWave - 1); }

// Is child `i` taken at its parent's rows as they are?
template <typename T, bool DRAFT>
__device__ __forceinline__ bool first_taken(const VerifyArgs& a, int64_t parent, int64_t i) {
  const int x = a.ids[i];
  if (x < 0 || x >= a.vocab) return false;
  const double p = proper(static_cast<const T*>(a.target)[parent * a.target_stride + x]);
  const double q = DRAFT ? (double)proper(static_cast<const T*>(a.draft)[parent * a.draft_stride + x]) : 1.0;
  return (double)a.u[i] * q < p;
}

// The sum of f(token, entry of p, entry of q) over a part of the rows, by one wave.  Tokens of children are left out: where a batch of tokens may hold one (a bit of `marks` for every
// batch, of 64 in turn) each is compared.  The loads of two batches are on their way while two others are
// used (of four and four, of six and six: 68 | 69 and 90 us for 64 trees over 131 072 tokens).  Entries come as they are.
constexpr int kInFlight = 2;
template <typename T, bool DRAFT, typename F>
__device__ __forceinline__ void walk_tokens(const T* p, const T* q, int vocab, int from, int to, unsigned long long marks, const int* children, int count, F each) {
  constexpr int kCount = Loaded<T>::kCount, kBatch = kWave * kCount;
  auto batch = [&](int b, const Loaded<T>& r, const Loaded<T>& s) {
    const int v0 = b + lane_id() * kCount;
    if (marks >> (b / kBatch % 64) & 1) {
      unsigned out = 0;
      for (int j = 0; j < count; ++j) {
        const int at = children[j] - v0;
        out |= at >= 0 && at < kCount ? 1u << at : 0u;
      }
#pragma unroll
      for (int i = 0; i < kCount; ++i) each(v0 + i, out >> i & 1 ? 0.0f : (float)r.v[i], DRAFT && !(out >> i & 1) ? (float)s.v[i] : 0.0f);
    } else {
#pragma unroll
      for (int i = 0; i < kCount; ++i) each(v0 + i, (float)r.v[i], DRAFT ? (float)s.v[i] : 0.0f);
    }
  };
  Loaded<T> r[2][kInFlight], s[2][kInFlight];
  auto fetch = [&](int n, int b) {
#pragma unroll
    for (int i = 0; i < kInFlight; ++i) {
      __builtin_memcpy(&r[n][i], p + b + i * kBatch + lane_id() * kCount, 16);
      if constexpr (DRAFT) __builtin_memcpy(&s[n][i], q + b + i * kBatch + lane_id() * kCount, 16);
    }
  };
  auto use = [&](int n, int b) {
#pragma unroll
    for (int i = 0; i < kInFlight; ++i) batch(b + i * kBatch, r[n][i], s[n][i]);
  };
  constexpr int kStep = kInFlight * kBatch;
  int b = from;
  if (b + kStep <= to) {
    fetch(0, b);
    for (; b + 3 * kStep <= to; b += 2 * kStep) {
      fetch(1, b + kStep);
      use(0, b);
      fetch(0, b + 2 * kStep);
      use(1, b + kStep);
    }
    if (b + 2 * kStep <= to) {
      fetch(1, b + kStep);
      use(0, b);
      use(1, b + kStep);
      b += 2 * kStep;
    } else {
      use(0, b);
      b += kStep;
    }
  }
  for (; b < to; b += kBatch) {
    const Loaded<T> r = load_some(p, b + lane_id() * kCount, vocab);
    Loaded<T> s = {};
    if constexpr (DRAFT) s = load_some(q, b + lane_id() * kCount, vocab);
    batch(b, r, s);
  }
}

// The children of a node, in order, and the entries of the rows at their tokens.
struct Children {
  int count, node[kMostNodes], token[kMostNodes];
  float p[kMostNodes], q[kMostNodes], u[kMostNodes];
};

// Both rows after some children were refused, as far as they are not at children's tokens: r = a max(P - b Q, 0), for max(max(x, 0) - c, 0) is max(x - c, 0) where c is not
// negative, and q = c Q.  So a pass takes the same few operations however many children were refused.  What r and q are at children's tokens every wave holds in registers.
template <typename T, bool DRAFT>
__global__ void __launch_bounds__(kVerifyThreads) k_verify_nodes(VerifyArgs a) {
  constexpr int kGroups = kMostNodes / kWave, kBatch = kWave * Loaded<T>::kCount;
  __shared__ Children kids;
  __shared__ int found[kGroups];
  __shared__ double parts[2][kVerifyWaves], weights[kMostNodes];
  const int64_t token = blockIdx.x;
  const int wave = uniform(threadIdx.x / kWave), lane = lane_id();
  const int4 place = load_uniform(a.trees.place + token);
  const Tree tree{place.x, place.y};
  const int node = (int)(token - tree.first);
  if (node < 0 || node >= tree.n) return;
  const T* p = static_cast<const T*>(a.target) + token * a.target_stride;
  const T* q = DRAFT ? static_cast<const T*>(a.draft) + token * a.draft_stride : nullptr;
  {
    // Can the walk come here?  It begins at node 0; a first child on the way has to be taken, and before another one the first may not be.
    bool barred = false, mine = false;
    int i = threadIdx.x, rank = 0, x = 0;
    float px = 0.0f, qx = 0.0f, ux = 0.0f;
    if (i < kMostNodes) {
      if (i < tree.n && i / 64 < a.trees.words && a.trees.up[token * a.trees.words + i / 64] >> (i % 64) & 1) {
        const TreeNode at = a.trees.node[tree.first + i];
        if (at.parent < 0 || at.parent >= tree.n || at.eldest >= tree.n) barred = i != 0;
        else barred = first_taken<T, DRAFT>(a, tree.first + at.parent, tree.first + at.eldest) != (at.eldest == i);
      }
    } else if (i < 2 * kMostNodes) {
      i -= kMostNodes;
      if (i < tree.n && a.trees.node[tree.first + i].parent == node) {
        x = a.ids[tree.first + i];
        mine = x >= 0 && x < a.vocab;
        if (mine) {
          ux = a.u[tree.first + i];
          px = proper(p[x]);
          if constexpr (DRAFT) qx = proper(q[x]);
        }
      }
      const unsigned long long all = __ballot(mine);
      rank = __popcll(all & ((1ull << lane) - 1));
      if (lane == 0) found[i / kWave] = __popcll(all);
    }
    if (__syncthreads_or(barred)) return;
    if (mine) {
      for (int g = 0; g < i / kWave; ++g) rank += found[g];
      kids.node[rank] = i; kids.token[rank] = x;
      kids.p[rank] = px; kids.q[rank] = qx; kids.u[rank] = ux;
    }
    if (threadIdx.x == 0) {
      int n = 0;
      for (int g = 0; g < kGroups; ++g) n += found[g];
      kids.count = n;
    }
    __syncthreads();
  }
  const int count = uniform(kids.count), groups = ceil_div_d(count, kWave);
  // r and q at the children's tokens (0 for one whose token an earlier one has), as they are and as they were at first
  double r[kGroups] = {}, q_now[kGroups] = {}, q_all[kGroups] = {};
  int x[kGroups];
  bool again[kGroups];
  unsigned long long marks = 0;
#pragma unroll
  for (int g = 0; g < kGroups; ++g) {
    const int j = g * kWave + lane;
    x[g] = -1;
    again[g] = false;
    if (g < groups && j < count) {
      x[g] = kids.token[j];
      for (int i = 0; i < j; ++i) again[g] |= kids.token[i] == x[g];
      r[g] = again[g] ? 0.0 : kids.p[j];
      q_now[g] = q_all[g] = again[g] ? 0.0 : kids.q[j];
      marks |= 1ull << (x[g] / kBatch % 64);
    }
  }
#pragma unroll
  for (int d = 1; d < kWave; d *= 2) marks |= __shfl_xor(marks, d);
  const unsigned marks_lo = uniform((int)marks), marks_hi = uniform((int)(marks >> 32));
  marks = (unsigned long long)marks_hi << 32 | marks_lo;

  const int part = ceil_div_d(ceil_div_d(a.vocab, kVerifyWaves), kBatch) * kBatch;
  const int from = min(wave * part, a.vocab), to = min(from + part, a.vocab);
  double ra = 1.0, rb = 0.0, qc = 1.0;
  // parts: of every wave's part of the rows, without the children's tokens, the sums of max(P - by Q, 0), and of Q from the first pass over it
  bool have = false;
  double by = 0.0, all_q = 0.0;
  auto pass = [&](double times, bool first) {
    double sum = 0.0, other = 0.0;
    by = times;
    if (DRAFT && first)
      walk_tokens<T, DRAFT>(p, q, a.vocab, from, to, marks, kids.token, count, [&](int, float r0, float q0) {
        const double qv = proper64(q0);
        sum += fmax(__builtin_fma(-by, qv, (double)r0), 0.0);
        other += qv;
      });
    else if (DRAFT && by != 0.0)
      walk_tokens<T, DRAFT>(p, q, a.vocab, from, to, marks, kids.token, count,
                            [&](int, float r0, float q0) { sum += fmax(__builtin_fma(-by, proper64(q0), (double)r0), 0.0); });
    else                                 // (the draft's row of a node without children may hold anything)
      walk_tokens<T, false>(p, q, a.vocab, from, to, marks, kids.token, count, [&](int, float r0, float) { sum += proper64(r0); });
    sum = wave_sum(sum);
    if (first) other = wave_sum(other);
    __syncthreads();                     // (whoever read the parts before is done)
    if (lane == 0) {
      parts[0][wave] = sum;
      if (first) parts[1][wave] = other;
    }
    __syncthreads();
    have = true;
  };
  static_assert(kVerifyWaves == 16, "a row of lanes");
  auto total = [&](int which) { return lane_of(row_scan(parts[which][lane % kVerifyWaves]), kVerifyWaves - 1); };
  // the sum over children of f(group, lane's child)
  auto over = [&](auto f) {
    double v = 0.0;
    if (groups == 0) return v;
#pragma unroll
    for (int g = 0; g < kGroups; ++g)
      if (g < groups && x[g] >= 0) v += f(g);
    return wave_sum(v);
  };
  double w[kGroups] = {};                // what r was at the children's tokens before it was divided by its sum
  double unit = 1.0;                     // ... and a then
  bool undivided = false;                // parts, w and unit are of r before that
  for (int k = 0; k < count; ++k) {
    double rk = 0.0, qk = 0.0;
#pragma unroll
    for (int g = 0; g < kGroups; ++g)
      if (g == k / kWave) { rk = __shfl(r[g], k % kWave); qk = __shfl(q_now[g], k % kWave); }
    const int xk = kids.token[k];
    // (a token that an earlier child has: its r and q are at that child)
    bool repeated = false;
    for (int i = 0; i < k && !repeated; ++i)
      if (kids.token[i] == xk) {
        repeated = true;
#pragma unroll
        for (int g = 0; g < kGroups; ++g)
          if (g == i / kWave) { rk = __shfl(r[g], i % kWave); qk = __shfl(q_now[g], i % kWave); }
      }
    if ((double)kids.u[k] * (DRAFT ? qk : 1.0) < rk) {
      if (threadIdx.x == 0) a.onward[token] = make_int2(kids.node[k], -1);
      return;
    }
    if constexpr (DRAFT) {
      const double times = rb + qc / ra;
      pass(times, !have);
#pragma unroll
      for (int g = 0; g < kGroups; ++g) {
        w[g] = fmax(r[g] - q_now[g], 0.0);
        if (x[g] == xk) q_all[g] = 0.0;
      }
      const double left = ra * total(0) + over([&](int g) { return w[g]; });
      const double rest = total(1) + over([&](int g) { return q_all[g]; });
      undivided = left > 0.0;
      unit = ra;
      if (undivided) {
        ra /= left;
        rb = times;
      }
      qc = rest > 0.0 ? 1.0 / rest : 0.0;
#pragma unroll
      for (int g = 0; g < kGroups; ++g) {
        if (undivided) r[g] = w[g] / left;
        q_now[g] = q_all[g] * qc;
      }
    } else {
      if (!have) pass(0.0, false);
      const double left = ra * total(0) + over([&](int g) { return x[g] == xk ? 0.0 : r[g]; });
      if (left > 0.0) {
        ra /= left;
#pragma unroll
        for (int g = 0; g < kGroups; ++g) r[g] = x[g] == xk ? 0.0 : r[g] / left;
      }
    }
  }
  // The token that follows: from r, in the units of the parts where those are at hand.
  if (!DRAFT || !undivided) unit = ra;
  if (!have || (DRAFT && !undivided)) pass(rb, false);
#pragma unroll
  for (int g = 0; g < kGroups; ++g) {
    if (!(DRAFT && undivided)) w[g] = r[g];
    if (wave == 0 && g < groups && x[g] >= 0) weights[g * kWave + lane] = w[g];
  }
  // ... with the children's tokens in the parts that they lie in
  auto with_children = [&](int b, int e) { return over([&](int g) { return x[g] >= b && x[g] < e ? w[g] : 0.0; }); };
  {
    const double mine = parts[0][wave] * unit + with_children(from, to);
    __syncthreads();
    if (lane == 0) parts[0][wave] = mine;
    __syncthreads();
  }
  const double goal = (double)a.u[tree.first] * total(0);
  auto weights_of = [&](int b, int e, auto f) {
    if (DRAFT && by != 0.0)
      walk_tokens<T, DRAFT>(p, q, a.vocab, b, e, marks, kids.token, count, [&](int v, float r0, float q0) { f(v, unit * fmax(__builtin_fma(-by, proper64(q0), (double)r0), 0.0)); });
    else walk_tokens<T, false>(p, q, a.vocab, b, e, marks, kids.token, count, [&](int v, float r0, float) { f(v, unit * proper64(r0)); });
  };
  // The part in which the running sum passes the goal, the share of it, and the token: where rounding lets none pass, the last that is above 0.
  int begin = 0, size = part;
  double sum = 0.0;
  for (int level = 0; level < 2; ++level) {
    const double mine16 = parts[0][lane % kVerifyWaves], upto16 = row_scan(mine16);
    const unsigned some = (unsigned)__ballot(mine16 > 0.0) & 0xffffu, passed = (unsigned)__ballot(sum + upto16 > goal) & some;
    if (!some) {                         // (nothing above 0)
      if (threadIdx.x == 0) a.onward[token] = make_int2(-1, -1);
      return;
    }
    const int pick = passed ? __builtin_ctz(passed) : 31 - __builtin_clz(some);
    sum += lane_of(upto16, pick) - lane_of(mine16, pick);
    begin += pick * size;
    if (level == 1) break;
    const int limit = min(begin + size, a.vocab);
    size = ceil_div_d(ceil_div_d(size, kVerifyWaves), kBatch) * kBatch;
    double mine = 0.0;
    const int b = min(begin + wave * size, limit), e = min(b + size, limit);
    weights_of(b, e, [&](int, double v) { mine += v; });
    mine = wave_sum(mine) + with_children(b, e);
    __syncthreads();
    if (lane == 0) parts[0][wave] = mine;
    __syncthreads();
  }
  if (wave) return;
  const int end = min(begin + size, a.vocab);
  int best = -1;
  for (int b = begin; b < end; b += kBatch) {
    constexpr int kCount = Loaded<T>::kCount;
    double each[kCount] = {}, mine = 0.0;
    const int v0 = b + lane * kCount;
    weights_of(b, min(b + kBatch, end), [&](int v, double x) {
#pragma unroll
      for (int i = 0; i < kCount; ++i) each[i] = v == v0 + i ? x : each[i];
    });
    if (marks >> (b / kBatch % 64) & 1)
      for (int j = 0; j < count; ++j)
#pragma unroll
        for (int i = 0; i < kCount; ++i) each[i] += kids.token[j] == v0 + i ? weights[j] : 0.0;
#pragma unroll
    for (int i = 0; i < kCount; ++i) mine += each[i];
    const double upto = wave_scan(mine);
    double at = sum + (upto - mine);
    int first = -1, above = -1;          // the lane's first token that passes the goal, its last above 0
#pragma unroll
    for (int i = 0; i < kCount; ++i) {
      at += each[i];
      if (each[i] > 0.0) {
        above = v0 + i;
        if (at > goal && first < 0) first = above;
      }
    }
    const unsigned long long some = __ballot(above >= 0), passed = __ballot(first >= 0);
    if (passed) { best = __builtin_amdgcn_readlane(first, __builtin_ctzll(passed)); break; }
    if (some) best = __builtin_amdgcn_readlane(above, 63 - __builtin_clzll(some));
    sum += lane_of(upto, kWave - 1);
  }
  if (lane == 0) a.onward[token] = make_int2(-1, best);
}

// The walk: a wave has a tree, and what was found at its nodes in LDS.
__global__ void __launch_bounds__(256) k_verify_walk(VerifyArgs a) {
  __shared__ int2 onward[4][kMostNodes];
  __shared__ int way[4][kMostNodes];
  const int wave = threadIdx.x / kWave, lane = lane_id();
  const int64_t s = (int64_t)blockIdx.x * 4 + wave;
  const bool here = s < a.trees.rows;
  const Tree tree = here ? tree_of(a.trees, (int)s) : Tree{0, 0};
  for (int i = lane; i < tree.n; i += kWave) {
    onward[wave][i] = a.onward[tree.first + i];
    way[wave][i] = -1;
  }
  __syncthreads();
  if (lane == 0 && here) {
    int node = tree.n > 0 ? 0 : -1, count = 0, next = -1;
    while (node >= 0 && count < tree.n) {
      way[wave][count++] = node;
      const int2 o = onward[wave][node];
      next = o.y;
      node = o.x > node && o.x < tree.n ? o.x : -1;
    }
    a.kept[s] = count;
    a.next[s] = next;
  }
  __syncthreads();
  for (int i = lane; i < tree.n; i += kWave) a.path[tree.first + i] = way[wave][i];
}

}  // namespace spg
