// Which drafted tokens stay, and the token that follows.
//
// What happens at a node depends on the node's own rows and the given numbers alone, not on how the walk got there: so a workgroup has a node, and a walk over what they found (a node onward, or
// a token) is a second launch.  A node that the walk cannot come to ends at once: each of its ancestors is asked what a first child needs, two numbers.  At a node whose first child is taken nothing more is read.  A child that is
// not taken costs a pass over both rows, in which wave w has the w-th part: the sums of these parts are what the token is looked for in, if no other child is taken.
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

// A row of probabilities.  What is negative or NaN counts as 0.
template <typename T> __device__ __forceinline__ float proper(T v) { return fmaxf((float)v, 0.0f); }

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

// What the rows have become after some children were not taken: r = max(r - q, 0) * r_by (r itself where r_by is 0), q = q * q_by, 0 at the token.
struct Refused {
  int count;
  int token[kMostNodes];
  double r_by[kMostNodes], q_by[kMostNodes];
};

struct Weights { double r, q; };
// r and q of token v after the first `count` refusals.  near: v may be one of their tokens.
template <bool DRAFT>
__device__ __forceinline__ Weights weights(const Refused& f, int count, int v, float r0, float q0, bool near) {
  Weights w{(double)r0, DRAFT ? (double)q0 : 0.0};
  for (int i = 0; i < count; ++i) {
    const bool is = near && f.token[i] == v;
    if constexpr (DRAFT) {
      const double by = f.r_by[i];
      w.r = by != 0.0 ? fmax(w.r - w.q, 0.0) * by : w.r;
      w.q = is ? 0.0 : w.q * f.q_by[i];
    } else {
      const double by = f.r_by[i];
      w.r = by != 0.0 ? (is ? 0.0 : w.r * by) : w.r;
    }
  }
  return w;
}
// What r becomes when x is refused, not divided by its sum.
template <bool DRAFT>
__device__ __forceinline__ double left_of(const Weights& w, bool is_x) {
  return DRAFT ? fmax(w.r - w.q, 0.0) : is_x ? 0.0 : w.r;
}

__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
  for (int d = 1; d < kWave; d *= 2) v += __shfl_xor(v, d);
  return v;
}

// Is child `i` taken at its parent's rows as they are?
template <typename T, bool DRAFT>
__device__ __forceinline__ bool first_taken(const VerifyArgs& a, int64_t parent, int64_t i) {
  const int x = a.ids[i];
  if (x < 0 || x >= a.vocab) return false;
  const double p = proper(static_cast<const T*>(a.target)[parent * a.target_stride + x]);
  const double q = DRAFT ? (double)proper(static_cast<const T*>(a.draft)[parent * a.draft_stride + x]) : 1.0;
  return (double)a.u[i] * q < p;
}

// f(v, r0, q0, near) for tokens from .. to - 1 of the rows, by one wave.  near: one of the first `count` refused tokens, or x, may be among the lane's.
template <typename T, bool DRAFT, typename F>
__device__ __forceinline__ void walk_tokens(const T* p, const T* q, int vocab, int from, int to, const Refused& f, int count, int x, F each) {
  constexpr int kCount = Loaded<T>::kCount, kBatch = kWave * kCount;
  for (int b = from; b < to; b += kBatch) {
    const int v0 = b + lane_id() * kCount;
    const Loaded<T> r = load_some(p, v0, vocab);
    Loaded<T> s = {};
    if constexpr (DRAFT) s = load_some(q, v0, vocab);
    bool near = x >= b && x < b + kBatch;
    for (int i = 0; i < count; ++i) near |= f.token[i] >= b && f.token[i] < b + kBatch;
#pragma unroll
    for (int i = 0; i < kCount; ++i)
      if (v0 + i < to) each(v0 + i, proper(r.v[i]), DRAFT ? proper(s.v[i]) : 0.0f, near);
  }
}

template <typename T, bool DRAFT>
__global__ void __launch_bounds__(kVerifyThreads) k_verify_nodes(VerifyArgs a) {
  __shared__ Refused refused;
  __shared__ double parts[2][kVerifyWaves];
  __shared__ int found;
  const int64_t token = blockIdx.x;
  const int wave = uniform(threadIdx.x / kWave), lane = lane_id();
  const int s = uniform(find_seq(a.trees.rows, token, [&](int i) { return tree_begin(a.trees, i); }));
  const Tree tree = tree_of(a.trees, s);
  const int node = (int)(token - tree.first);
  if (node < 0 || node >= tree.n) return;
  // Can the walk come here?  It begins at node 0; a first child on the way has to be taken, and before another one the first may not be.
  {
    bool barred = false;
    const int i = threadIdx.x;
    if (i < tree.n && i / 64 < a.trees.words && a.trees.up[token * a.trees.words + i / 64] >> (i % 64) & 1) {
      const int parent = a.trees.node[tree.first + i].x;
      if (parent < 0) barred = i != 0;
      else {
        const int first = a.trees.node[tree.first + parent].y;
        barred = first_taken<T, DRAFT>(a, tree.first + parent, tree.first + first) != (first == i);
      }
    }
    if (__syncthreads_or(barred)) return;
  }
  const T* p = static_cast<const T*>(a.target) + token * a.target_stride;
  const T* q = DRAFT ? static_cast<const T*>(a.draft) + token * a.draft_stride : nullptr;
  constexpr int kBatch = kWave * Loaded<T>::kCount;
  const int part = ceil_div_d(ceil_div_d(a.vocab, kVerifyWaves), kBatch) * kBatch;
  const int from = min(wave * part, a.vocab), to = min(from + part, a.vocab);
  if (threadIdx.x == 0) refused.count = 0;
  // sums over the row of what f gives for a token, part by part
  auto sums = [&](int count, int x, auto f) {
    double r = 0.0, other = 0.0;
    walk_tokens<T, DRAFT>(p, q, a.vocab, from, to, refused, count, x, [&](int v, float r0, float q0, bool near) { f(v, r0, q0, near, r, other); });
    r = wave_sum(r);
    other = wave_sum(other);
    __syncthreads();                     // (whoever read the parts before is done)
    if (lane == 0) { parts[0][wave] = r; parts[1][wave] = other; }
    __syncthreads();
    r = other = 0.0;
    for (int w = 0; w < kVerifyWaves; ++w) { r += parts[0][w]; other += parts[1][w]; }
    return Weights{r, other};
  };
  int last = -1, count = 0;              // the last refused token, where the sums of the parts are of what r is after it
  double total = 0.0;
  for (int child = a.trees.node[token].y; child >= 0; child = a.trees.node[tree.first + child].z) {
    const int x = a.ids[tree.first + child];
    if (x < 0 || x >= a.vocab) continue;
    __syncthreads();
    const Weights w = weights<DRAFT>(refused, count, x, proper(p[x]), DRAFT ? proper(q[x]) : 0.0f, true);
    if ((double)a.u[tree.first + child] * (DRAFT ? w.q : 1.0) < w.r) {
      if (threadIdx.x == 0) a.onward[token] = make_int2(child, -1);
      return;
    }
    const Weights sum = sums(count, x, [&](int v, float r0, float q0, bool near, double& r, double& other) {
      const Weights w = weights<DRAFT>(refused, count, v, r0, q0, near);
      const bool is = near && v == x;
      r += left_of<DRAFT>(w, is);
      if constexpr (DRAFT) other += is ? 0.0 : w.q;
    });
    if (threadIdx.x == 0) {
      refused.token[count] = x;
      refused.r_by[count] = sum.r > 0.0 ? 1.0 / sum.r : 0.0;
      refused.q_by[count] = sum.q > 0.0 ? 1.0 / sum.q : 0.0;
    }
    last = sum.r > 0.0 ? x : -1;
    total = sum.r;
    ++count;
  }
  __syncthreads();
  // The token that follows: from r as it is.  Where the last refusal left something, its sums are at hand: r is what was left, not yet divided.
  const int before = last >= 0 ? count - 1 : count;
  auto weight = [&](int v, float r0, float q0, bool near) {
    const Weights w = weights<DRAFT>(refused, before, v, r0, q0, near);
    return last >= 0 ? left_of<DRAFT>(w, near && v == last) : w.r;
  };
  if (last < 0) total = sums(before, -1, [&](int v, float r0, float q0, bool near, double& r, double&) { r += weight(v, r0, q0, near); }).r;
  const double goal = (double)a.u[tree.first] * total;
  // The part in which the running sum passes the goal, the share of it, and the token: where rounding lets none pass, the last that is above 0.
  int begin = 0, size = part;
  double sum = 0.0;
  for (int level = 0; level < 2; ++level) {
    int pick = -1;
    double at = sum;
    for (int w = 0; w < kVerifyWaves; ++w) {
      const double mine = parts[0][w];
      if (mine > 0.0 && (pick < 0 || at <= goal)) { pick = w; sum = at; }
      at += mine;
      if (at > goal && pick >= 0) break;
    }
    if (pick < 0) {                      // (nothing above 0)
      if (threadIdx.x == 0) a.onward[token] = make_int2(-1, -1);
      return;
    }
    begin += pick * size;
    if (level == 1) break;
    const int limit = min(begin + size, a.vocab);
    size = ceil_div_d(ceil_div_d(size, kVerifyWaves), kBatch) * kBatch;
    double mine = 0.0;
    const int b = min(begin + wave * size, limit), e = min(b + size, limit);
    walk_tokens<T, DRAFT>(p, q, a.vocab, b, e, refused, before, last, [&](int v, float r0, float q0, bool near) { mine += weight(v, r0, q0, near); });
    mine = wave_sum(mine);
    __syncthreads();
    if (lane == 0) parts[0][wave] = mine;
    __syncthreads();
  }
  if (wave) return;
  const int end = min(begin + size, a.vocab);
  int best = -1;
  for (int b = begin; b < end; b += kBatch) {
    constexpr int kCount = Loaded<T>::kCount;
    double w[kCount] = {}, mine = 0.0;
    walk_tokens<T, DRAFT>(p, q, a.vocab, b, min(b + kBatch, end), refused, before, last, [&](int v, float r0, float q0, bool near) {
      const double x = weight(v, r0, q0, near);
#pragma unroll
      for (int i = 0; i < kCount; ++i) w[i] = v == b + lane * kCount + i ? x : w[i];
      mine += x;
    });
    double upto = mine;                  // of the lanes up to this one
#pragma unroll
    for (int d = 1; d < kWave; d *= 2) {
      const double o = __shfl_up(upto, d);
      upto += lane >= d ? o : 0.0;
    }
    const double whole = __shfl(upto, kWave - 1);
    double at = sum + (upto - mine);
    int first = a.vocab, above = -1;     // the lane's first token that passes the goal, its last above 0
#pragma unroll
    for (int i = 0; i < kCount; ++i) {
      at += w[i];
      if (w[i] > 0.0) {
        above = b + lane * kCount + i;
        if (at > goal && first == a.vocab) first = above;
      }
    }
#pragma unroll
    for (int d = 1; d < kWave; d *= 2) {
      first = min(first, __shfl_xor(first, d));
      above = max(above, __shfl_xor(above, d));
    }
    best = first < a.vocab ? first : max(best, above);
    if (first < a.vocab) break;
    sum += whole;
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
