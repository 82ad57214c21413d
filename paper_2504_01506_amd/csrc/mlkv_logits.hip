// Log probabilities of given tokens with entropy and top alternatives, and
// their gradient in the logits.
//
// A row is cut into chunks, a block each, that hold their logits in registers:
// every logit is read once. A thread sums e = exp(x - m) and e (x - m) against
// the largest logit m of its own, and the joins (lanes, waves, chunks) rescale
// to the largest of all, the running softmax. A second kernel joins a row's
// chunks; where there are rows enough for the device, a block takes a row's
// chunks in turn instead, and rows of few logits are a wave each. Bound by
// HBM: 9 operations a logit, one of them an exponential (of the rate of four),
// against 2 or 4 bytes. 4096 rows of 128,000 bf16 logits with five alternatives
// take 189 us, 5.5 TB/s; 8192 of 32,000 fp32 182 (5.8).
//
// Alternatives: a chunk leaves the largest logit of each group of 16 vectors.
// A row's k largest logits are in the k groups whose largest are (equal ones
// in the order of their indices, which is that of the groups), so only those
// groups are read again, 1 of 250 for k = 4 and 128,000 logits. (Candidates
// picked by each block from its own logits: 4096 x 128,000 271 us against 190.)
#include "mlkv_ops.h"

#include <algorithm>

namespace mlkv {
namespace {

constexpr int kChunkThreads = 256;
constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLn2 = 0.69314718055994530942f;
constexpr float kInf = __builtin_inff();

// Sums of a part of a row: m its largest logit, s = sum 2^z, t = sum z 2^z
// with z = (x - m) log2(e).
struct Part {
  float m, s, t, pad;
};

// The part's sums against a larger maximum (or its own).
__device__ __forceinline__ Part part_scale(const Part& p, float m) {
  Part r;
  const float d = p.m == -kInf ? 0.0f : (p.m - m) * kLog2e;  // (-inf alone: nothing to rescale)
  const float f = __builtin_amdgcn_exp2f(d);
  r.m = m;
  r.s = f * p.s;
  // (2^d is 0 long before d leaves the range in which d 2^d is 0)
  r.t = f * __builtin_fmaf(fmaxf(d, -1e4f), p.s, p.t);
  r.pad = 0.0f;
  return r;
}
__device__ __forceinline__ Part part_join(const Part& a, const Part& b) {
  const float m = fmaxf(a.m, b.m);
  Part x = part_scale(a, m);
  const Part y = part_scale(b, m);
  x.s += y.s;
  x.t += y.t;
  return x;
}
// ... of a wave's lanes, in every lane; a block's from its waves'.
__device__ __forceinline__ Part wave_join(const Part& p) {
  Part r = part_scale(p, wave_max(p.m));
  r.s = group_sum(r.s, 64);
  r.t = group_sum(r.t, 64);
  return r;
}
template <int kWaves>
__device__ __forceinline__ Part waves_join(const Part* p) {
  float m = p[0].m;
#pragma unroll
  for (int w = 1; w < kWaves; ++w) m = fmaxf(m, p[w].m);
  Part r = part_scale(p[0], m);
#pragma unroll
  for (int w = 1; w < kWaves; ++w) {
    const Part x = part_scale(p[w], m);
    r.s += x.s;
    r.t += x.t;
  }
  return r;
}

// Order of logits as unsigned numbers; -0 counts as +0. Every logit's is over 0.
__device__ __forceinline__ uint32_t value_key(float x) {
  const uint32_t b = __float_as_uint(x + 0.0f);
  return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float key_value(uint32_t k) {
  return __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k);
}
// value, then lowest index first; 0 for a NaN, as for what is not there
__device__ __forceinline__ uint64_t full_key(float x, uint32_t i) {
  return x == x ? (uint64_t)value_key(x) << 32 | (uint32_t)~i : 0;
}
__device__ __forceinline__ uint32_t key_index(uint64_t k) { return ~(uint32_t)k; }

struct LogpArgs {
  const void* logits;
  const int64_t* tokens;  // or NULL
  float* logp;            // or NULL, as are all outputs
  float* entropy;
  float* stats;
  int64_t* top_ids;
  float* top_logp;
  Part* parts;            // [n][chunks]
  uint32_t* groups;       // [n][chunks][kGroups * L] value keys of the groups' largest logits
  int64_t stride, n;
  int vocab, top, chunks;
  int chunk_groups;       // kGroups * L
};

constexpr int kGroupVecs = 16;                          // vectors of a group: lanes that a DPP row joins
constexpr int kGroups = kChunkThreads / kGroupVecs;     // groups of a chunk, for each vector of a thread

// What a row's sums give.
struct RowStats {
  float m, logs, ent;
  bool none;  // nothing but -inf
};

__device__ __forceinline__ RowStats row_stats(const Part& p) {
  RowStats r;
  r.none = p.m == -kInf && p.s == 0.0f;
  if (r.none) {
    r.m = -kInf;
    r.logs = r.ent = 0.0f;
  } else if (!(p.s < kInf)) {  // a NaN or +inf
    r.m = r.logs = r.ent = __builtin_nanf("");
  } else {
    r.m = p.m;
    r.logs = logf(p.s);
    r.ent = r.logs - p.t * kLn2 / p.s;  // (t <= 0: nothing cancels)
  }
  return r;
}

__device__ __forceinline__ float log_prob(float x, const RowStats& r) { return r.none ? -kInf : (x - r.m) - r.logs; }

// The row's token and its logit, loaded by the thread that writes them, well before.
struct Given {
  int64_t token;
  float logit;
};
template <class T>
__device__ __forceinline__ Given given(const LogpArgs& a, int64_t row, const T* x) {
  Given g = {-1, 0.0f};
  if (a.logp != nullptr) g.token = a.tokens[row];
  if (g.token >= 0 && g.token < a.vocab) g.logit = (float)x[g.token];
  return g;
}

__device__ __forceinline__ void write_row(const LogpArgs& a, int64_t row, const RowStats& r, const Given& g) {
  if (a.stats != nullptr) {
    a.stats[2 * row] = r.m;
    a.stats[2 * row + 1] = r.logs;
  }
  if (a.entropy != nullptr) a.entropy[row] = r.ent;
  if (a.logp != nullptr) {
    a.logp[row] = g.token >= a.vocab ? __builtin_nanf("") : g.token < 0 ? 0.0f : log_prob(g.logit, r);
  }
}

__device__ __forceinline__ void write_top(const LogpArgs& a, int64_t row, int rank, uint64_t key, const RowStats& r) {
  if (a.top_ids != nullptr) a.top_ids[row * a.top + rank] = r.m != r.m ? -1 : (int64_t)key_index(key);
  if (a.top_logp != nullptr) a.top_logp[row * a.top + rank] = log_prob(key_value((uint32_t)(key >> 32)), r);
}

// Vectors of V elements of a row that lie on 16-byte boundaries, and the few
// elements before and behind them.
template <class T>
struct Cut {
  static constexpr int V = 16 / sizeof(T);
  int head, vecs, tail;
  __device__ __forceinline__ Cut(const T* row, int n) {
    const int at = (int)((reinterpret_cast<uintptr_t>(row) / sizeof(T)) % V);
    head = min(at ? V - at : 0, n);
    vecs = (n - head) / V;
    tail = n - head - vecs * V;
  }
};

// ---- the k largest keys of a team (a wave or a block) ----
// The k-th largest of the threads' largest values, cut to 16 bits, is a bound
// that the k largest reach; the keys over it, hardly more than k, are ranked by
// counting. Many equal values can leave
// more than kCands of them: then the bound is the k-th largest of the threads'
// own largest keys, which no more than k threads reach, and where even those
// hold too many (large ones in few threads), the largest key below the last is
// sought k times.
template <int kTeam>
struct Select {
  static constexpr int kCands = kTeam == 64 ? 512 : 1024;
  uint32_t seen[kTeam];
  uint64_t list[kTeam];
  uint64_t cand[kCands];
  uint64_t out[MLKV_LOGITS_MAX_TOP];  // largest first
  uint64_t bound;
  int listed, cands;
};

template <int kTeam>
__device__ __forceinline__ void team_sync() {
  if constexpr (kTeam > 64) {
    __syncthreads();
  } else {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
  }
}

// How many of p[0 .. n) are larger than f.
__device__ __forceinline__ int count_over(const uint64_t* p, int n, uint64_t f) {
  int over = 0, i = 0;
  for (; i + 8 <= n; i += 8)
#pragma unroll
    for (int e = 0; e < 8; ++e) over += p[i + e] > f;
  for (; i < n; ++i) over += p[i] > f;
  return over;
}

// each(f) calls f with every key of the thread: no two equal in the team, but
// for 0, which does not count. q: the largest one's value. Returns how many of
// the k there are, the same in all threads; s.out is ready for all.
template <int kTeam, class Each>
__device__ __forceinline__ int select_top(Select<kTeam>& s, int tid, uint32_t q, int k, const Each& each) {
  constexpr int kCands = Select<kTeam>::kCands;
  const int lane = tid & 63;
  s.seen[tid] = q;
  if (tid == 0) s.listed = s.cands = 0;
  team_sync<kTeam>();
  uint32_t seen[kTeam / 64], most = 0, low = 0;
#pragma unroll
  for (int w = 0; w < kTeam / 64; ++w) {
    seen[w] = s.seen[w * 64 + lane];
    most = max(most, seen[w]);
  }
  // (few keys: the largest of every four threads will do, a quarter of the work)
  if (kTeam == 64 || k <= 16) {
#pragma unroll 1
    for (int bit = 31; bit >= 16; --bit) {
      const uint32_t t = low | 1u << bit;
      if (__popcll(__ballot(most >= t)) >= k) low = t;
    }
  } else {
#pragma unroll 1
    for (int bit = 31; bit >= 16; --bit) {
      const uint32_t t = low | 1u << bit;
      int reach = 0;
#pragma unroll
      for (int w = 0; w < kTeam / 64; ++w) reach += __popcll(__ballot(seen[w] >= t));
      if (reach >= k) low = t;
    }
  }
  const auto collect = [&](uint64_t least) {
    each([&](uint64_t f) {
      if (f < least) return;
      const int at = atomicAdd(&s.cands, 1);
      if (at < kCands) s.cand[at] = f;
    });
  };
  // (a key is at least its value's, and 1 where it counts)
  if (q >= low && q != 0) collect((uint64_t)low << 32 | 1);
  team_sync<kTeam>();
  int nc = s.cands;
  if (nc > kCands) {
    uint64_t best = 0;
    each([&](uint64_t f) { best = max(best, f); });
    team_sync<kTeam>();
    if (best != 0) s.list[atomicAdd(&s.listed, 1)] = best;
    if (tid == 0) {
      s.cands = 0;
      s.bound = 1;  // (fewer than k threads have keys: all of those count)
    }
    team_sync<kTeam>();
    const int nl = s.listed;
    if (best != 0 && count_over(s.list, nl, best) == k - 1) s.bound = best;
    team_sync<kTeam>();
    if (best >= s.bound) collect(s.bound);
    team_sync<kTeam>();
    nc = s.cands;
  }
  if (nc <= kCands) {
    for (int i = tid; i < nc; i += kTeam) {
      const uint64_t f = s.cand[i];
      const int over = count_over(s.cand, nc, f);
      if (over < k) s.out[over] = f;
    }
    team_sync<kTeam>();
    return min(nc, k);
  }
  uint64_t last = ~0ull;
  for (int r = 0; r < k; ++r) {
    uint64_t m = 0;
    each([&](uint64_t f) {
      if (f < last) m = max(m, f);
    });
#pragma unroll
    for (int o = 1; o < 64; o *= 2) m = max(m, (uint64_t)__shfl_xor((unsigned long long)m, o));
    if constexpr (kTeam > 64) {
      if (lane == 0) s.list[tid >> 6] = m;
      __syncthreads();
      m = max(max(s.list[0], s.list[1]), max(s.list[2], s.list[3]));
      __syncthreads();
    }
    if (tid == 0) s.out[r] = m;
    last = m;
  }
  team_sync<kTeam>();
  return k;  // (there are more than kCands)
}

// ... of the keys key(i), i < n, thread i % kTeam's.
template <int kTeam, class Key>
__device__ __forceinline__ int select_of(Select<kTeam>& s, int tid, int n, int k, const Key& key) {
  constexpr int kHeld = 4;  // keys of a thread that are made once; the others for each look at them, as many at a time
  const auto some = [&](int from, uint64_t (&f)[kHeld]) {
#pragma unroll
    for (int j = 0; j < kHeld; ++j) f[j] = from + j * kTeam < n ? key(from + j * kTeam) : 0;
  };
  uint64_t held[kHeld], more[kHeld], best = 0;
  some(tid, held);
#pragma unroll
  for (int j = 0; j < kHeld; ++j) best = max(best, held[j]);
#pragma unroll 1
  for (int i = tid + kHeld * kTeam; i < n; i += kHeld * kTeam) {
    some(i, more);
#pragma unroll
    for (int j = 0; j < kHeld; ++j) best = max(best, more[j]);
  }
  return select_top<kTeam>(s, tid, (uint32_t)(best >> 32), k, [&](const auto& f) {
#pragma unroll
    for (int j = 0; j < kHeld; ++j) f(held[j]);
#pragma unroll 1
    for (int i = tid + kHeld * kTeam; i < n; i += kHeld * kTeam) {
      some(i, more);
#pragma unroll
      for (int j = 0; j < kHeld; ++j) f(more[j]);
    }
  });
}
static_assert(kChunkThreads == 256, "select_top's slow way joins four waves");

// The k largest logits of a row from its groups' largest (in LDS or global memory).
template <class T>
__device__ __forceinline__ int select_logits(Select<kChunkThreads>& s, int tid, const T* x, const Cut<T>& cut,
                                             const uint32_t* groups, int k, uint32_t* chosen) {
  constexpr int V = 16 / sizeof(T);
  const int ng = (cut.vecs + kGroupVecs - 1) / kGroupVecs;
  const int nsel = select_of<kChunkThreads>(s, tid, ng, k, [&](int i) { return (uint64_t)groups[i] << 32 | (uint32_t)~i; });
  if (tid < nsel) chosen[tid] = key_index(s.out[tid]);
  __syncthreads();
  // their vectors, and the logits before and behind all vectors, one a thread
  constexpr int kMost = MLKV_LOGITS_MAX_TOP * kGroupVecs / kChunkThreads;
  Raw p[kMost];
  int at[kMost];
#pragma unroll
  for (int j = 0; j < kMost; ++j) {
    const int i = tid + j * kChunkThreads;
    const int v = i < nsel * kGroupVecs ? (int)chosen[i / kGroupVecs] * kGroupVecs + i % kGroupVecs : cut.vecs;
    at[j] = v < cut.vecs ? cut.head + v * V : -1;
    if (v < cut.vecs) p[j] = load_raw(x + at[j]);
  }
  int extra = -1;
  if (tid < cut.head) extra = tid;
  if (tid >= V && tid < V + cut.tail) extra = cut.head + cut.vecs * V + tid - V;
  const uint64_t ex = extra >= 0 ? full_key((float)x[extra], (uint32_t)extra) : 0;
  uint32_t q = (uint32_t)(ex >> 32);
#pragma unroll
  for (int j = 0; j < kMost; ++j)
    if (at[j] >= 0) {
      float m = -kInf;
#pragma unroll
      for (int e = 0; e < V; ++e) m = fmaxf(m, element<T>(p[j], e));
      q = max(q, value_key(m));
    }
  return select_top<kChunkThreads>(s, tid, q, k, [&](const auto& f) {
    f(ex);
#pragma unroll
    for (int j = 0; j < kMost; ++j)
      if (at[j] >= 0) {
#pragma unroll
        for (int e = 0; e < V; ++e) f(full_key(element<T>(p[j], e), (uint32_t)(at[j] + e)));
      }
  });
}

// A thread's sums of L vectors and one more logit. vm: the vectors' largest.
template <class T, int L>
__device__ __forceinline__ Part thread_part(const Raw (&p)[L], float ex, float (&vm)[L]) {
  constexpr int V = 16 / sizeof(T);
  Part mine;
  float m = ex;
#pragma unroll
  for (int j = 0; j < L; ++j) {
    vm[j] = -kInf;
#pragma unroll
    for (int e = 0; e < V; ++e) vm[j] = fmaxf(vm[j], element<T>(p[j], e));
    m = fmaxf(m, vm[j]);
  }
  if (m != m) m = -kInf;  // (a lone NaN)
  const float base = m == -kInf ? 0.0f : m;
  mine.m = m;
  mine.pad = 0.0f;
  // z = x log2(e) - m log2(e) in one operation; what the product's rounding
  // shifts every z by (at most 2^-24 |m|) comes off the sums, to first order.
  // Where that is not small, or a logit is -inf and t no number, the sums are
  // taken again by steps.
  const float c = base * kLog2e;
  const float shift = __builtin_fmaf(base, kLog2e, -c);
  mine.s = mine.t = 0.0f;
#pragma unroll
  for (int j = 0; j < L; ++j)
#pragma unroll
    for (int e = 0; e < V; ++e) {
      const float z = __builtin_fmaf(element<T>(p[j], e), kLog2e, -c), q = __builtin_amdgcn_exp2f(z);
      mine.s += q;
      mine.t = __builtin_fmaf(q, z, mine.t);
    }
  mine.s = __builtin_fmaf(mine.s, -shift * kLn2, mine.s);
  mine.t = __builtin_fmaf(mine.t, -shift * kLn2, mine.t) - shift * mine.s;
  if (!(fabsf(mine.t) < kInf) || !(fabsf(shift) <= 0x1p-12f)) {
    mine.s = mine.t = 0.0f;
#pragma unroll
    for (int j = 0; j < L; ++j)
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const float z = (element<T>(p[j], e) - base) * kLog2e, q = __builtin_amdgcn_exp2f(z);
        mine.s += q;
        mine.t = __builtin_fmaf(q, fmaxf(z, -150.0f), mine.t);
      }
  }
  const float z = (ex - base) * kLog2e, q = __builtin_amdgcn_exp2f(z);
  mine.s += q;
  mine.t = __builtin_fmaf(q, fmaxf(z, -150.0f), mine.t);
  return mine;
}

// The value keys of the groups of a chunk, from its vectors' largest logits:
// lane j of a group writes that of the group of vector j.
template <int L>
__device__ __forceinline__ void group_maxima(const float (&vm)[L], uint32_t* to, int tid) {
  const int lane = tid & (kGroupVecs - 1);
  uint32_t mine = 0;
#pragma unroll
  for (int j = 0; j < L; ++j) {
    uint32_t g = value_key(vm[j]);
    g = max(g, dpp_bits<0xB1>(g));
    g = max(g, dpp_bits<0x4E>(g));
    g = max(g, dpp_bits<0x141>(g));
    g = max(g, dpp_bits<0x140>(g));
    if (lane == j) mine = g;
  }
  if (lane < L) to[lane * kGroups + tid / kGroupVecs] = mine;
}

// The thread's vectors, -inf where the row has none.
template <class T, int L>
__device__ __forceinline__ void load_vecs(Raw (&p)[L], const T* body, int first, int step, int vecs) {
  constexpr int V = 16 / sizeof(T);
  constexpr uint32_t kNone = sizeof(T) == 4 ? 0xFF800000u : std::is_same<T, bf16>::value ? 0xFF80FF80u : 0xFC00FC00u;
#pragma unroll
  for (int j = 0; j < L; ++j) {
    const int v = first + j * step;
    p[j] = Raw{kNone, kNone, kNone, kNone};
    if (v < vecs) p[j] = load_raw(body + (int64_t)v * V);
  }
}

// One chunk of a row: L vectors a thread. kTop: the alternatives are not
// wanted, left to the join, or taken from this chunk, the row's only one.
enum Top : int { kNoTop, kLeaveTop, kTakeTop };
template <class T, int L, int kTop>
__global__ __launch_bounds__(kChunkThreads) void k_logp_chunk(LogpArgs a) {
  constexpr int V = 16 / sizeof(T), kWaves = kChunkThreads / 64;
  __shared__ Part wave_part[kWaves];
  __shared__ uint32_t group_max[kTop == kTakeTop ? kGroups * L : 1];
  const int tid = threadIdx.x, lane = tid & 63;
  const int64_t row = blockIdx.x / (uint32_t)a.chunks;
  const int chunk = (int)(blockIdx.x % (uint32_t)a.chunks);
  const T* x = static_cast<const T*>(a.logits) + row * a.stride;
  const Cut<T> cut(x, a.vocab);
  Given token;
  if (tid == 0 && a.chunks == 1) token = given(a, row, x);
  Raw p[L];
  load_vecs<T, L>(p, x + cut.head, chunk * L * kChunkThreads + tid, kChunkThreads, cut.vecs);
  // the first chunk takes the logits before the vectors, the last those behind, one a thread
  float ex = -kInf;
  if (chunk == 0 && tid < cut.head) ex = (float)x[tid];
  if (chunk == a.chunks - 1 && tid >= V && tid < V + cut.tail) ex = (float)x[cut.head + cut.vecs * V + tid - V];
  float vm[L];
  const Part joined = wave_join(thread_part<T, L>(p, ex, vm));
  if (lane == 0) wave_part[tid >> 6] = joined;
  if constexpr (kTop != kNoTop) {
    group_maxima<L>(vm, kTop == kTakeTop ? group_max : a.groups + (row * a.chunks + chunk) * (kGroups * L), tid);
  }
  __syncthreads();
  const Part all = waves_join<kWaves>(wave_part);
  if (a.chunks > 1) {
    if (tid == 0) a.parts[row * a.chunks + chunk] = all;
    return;
  }
  const RowStats r = row_stats(all);
  if (tid == 0) write_row(a, row, r, token);
  if constexpr (kTop == kTakeTop) {
    __shared__ Select<kChunkThreads> sel;
    __shared__ uint32_t chosen[MLKV_LOGITS_MAX_TOP];
    const int found = select_logits<T>(sel, tid, x, cut, group_max, a.top, chosen);
    // (fewer keys than alternatives only where NaNs took their places)
    if (tid < a.top) write_top(a, row, tid, tid < found ? sel.out[tid] : 0, r);
  }
}

// Joins a row's chunks: a block a row. Bound by latency, one choice among the
// groups and one among their logits: 8 us for one row of 128,000, of which the
// chunks take 3.
template <class T>
__global__ __launch_bounds__(kChunkThreads) void k_logp_join(LogpArgs a) {
  constexpr int kWaves = kChunkThreads / 64;
  __shared__ Part wave_part[kWaves];
  __shared__ Select<kChunkThreads> sel;
  __shared__ uint32_t chosen[MLKV_LOGITS_MAX_TOP];
  const int tid = threadIdx.x;
  const int64_t row = blockIdx.x;
  const T* x = static_cast<const T*>(a.logits) + row * a.stride;
  const Part* parts = a.parts + row * a.chunks;
  Given token;
  if (tid == 0) token = given(a, row, x);
  Part mine;
  mine.m = -kInf;
  mine.s = mine.t = mine.pad = 0.0f;
  if (tid < a.chunks) mine = parts[tid];
  int found = 0;
  if (a.top > 0) {
    const Cut<T> cut(x, a.vocab);
    found = select_logits<T>(sel, tid, x, cut, a.groups + row * a.chunks * a.chunk_groups, a.top, chosen);
  }
  for (int c = tid + kChunkThreads; c < a.chunks; c += kChunkThreads) mine = part_join(mine, parts[c]);
  mine = wave_join(mine);
  if ((tid & 63) == 0) wave_part[tid >> 6] = mine;
  __syncthreads();
  const RowStats r = row_stats(waves_join<kWaves>(wave_part));
  if (tid == 0) write_row(a, row, r, token);
  if (tid < a.top) write_top(a, row, tid, tid < found ? sel.out[tid] : 0, r);
}

// A row a block, chunk by chunk: no join, and while a block seeks its
// alternatives the others on its unit read (4096 x 128,000 bf16 with five: 189 us).
constexpr int kRowVecs = 8, kRowGroups = 4096;  // vectors a thread and chunk; groups of a row at most
template <class T, bool kTop>
__global__ __launch_bounds__(kChunkThreads) void k_logp_long(LogpArgs a) {
  constexpr int V = 16 / sizeof(T), kWaves = kChunkThreads / 64, L = kRowVecs;
  __shared__ Part wave_part[kWaves];
  extern __shared__ uint32_t row_groups[];  // [chunks][kGroups * L]
  const int tid = threadIdx.x, lane = tid & 63;
  const int64_t row = blockIdx.x;
  const T* x = static_cast<const T*>(a.logits) + row * a.stride;
  const Cut<T> cut(x, a.vocab);
  Given token;
  if (tid == 0) token = given(a, row, x);
  float ex = -kInf;
  if (tid < cut.head) ex = (float)x[tid];
  if (tid >= V && tid < V + cut.tail) ex = (float)x[cut.head + cut.vecs * V + tid - V];
  Part mine;
  for (int chunk = 0; chunk < a.chunks; ++chunk) {
    Raw p[L];
    load_vecs<T, L>(p, x + cut.head, chunk * L * kChunkThreads + tid, kChunkThreads, cut.vecs);
    float vm[L];
    const Part part = thread_part<T, L>(p, chunk == 0 ? ex : -kInf, vm);
    mine = chunk == 0 ? part : part_join(mine, part);
    if constexpr (kTop) group_maxima<L>(vm, row_groups + chunk * (kGroups * L), tid);
  }
  mine = wave_join(mine);
  if (lane == 0) wave_part[tid >> 6] = mine;
  __syncthreads();
  const RowStats r = row_stats(waves_join<kWaves>(wave_part));
  if (tid == 0) write_row(a, row, r, token);
  if constexpr (kTop) {
    __shared__ Select<kChunkThreads> sel;
    __shared__ uint32_t chosen[MLKV_LOGITS_MAX_TOP];
    const int found = select_logits<T>(sel, tid, x, cut, row_groups, a.top, chosen);
    if (tid < a.top) write_top(a, row, tid, tid < found ? sel.out[tid] : 0, r);
  }
}

// Rows of at most 64 * L vectors: a wave each, four a block (16,384 x 1000 bf16
// 22 us, 43 with a block a row; 100,000 x 100 78, bound by the latency of a wave's
// dependent steps, 234 with a block).
template <class T, int L, bool kTop>
__global__ __launch_bounds__(kChunkThreads) void k_logp_rows(LogpArgs a) {
  constexpr int V = 16 / sizeof(T), kWaves = kChunkThreads / 64;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t row = (int64_t)blockIdx.x * kWaves + wave;
  if (row >= a.n) return;
  const T* x = static_cast<const T*>(a.logits) + row * a.stride;
  const Cut<T> cut(x, a.vocab);
  Raw p[L];
  load_vecs<T, L>(p, x + cut.head, lane, 64, cut.vecs);
  float ex = -kInf;
  if (lane < cut.head) ex = (float)x[lane];
  if (lane >= V && lane < V + cut.tail) ex = (float)x[cut.head + cut.vecs * V + lane - V];
  float vm[L];
  Given token;
  if (lane == 0) token = given(a, row, x);
  const RowStats r = row_stats(wave_join(thread_part<T, L>(p, ex, vm)));
  if (lane == 0) write_row(a, row, r, token);
  if constexpr (kTop) {
    __shared__ Select<64> sel[kWaves];
    Select<64>& s = sel[wave];
    // the lane's logits are its vectors' and perhaps one before or behind them
    const bool has = lane < cut.head || (lane >= V && lane < V + cut.tail);
    const uint32_t at = lane < cut.head ? lane : cut.head + cut.vecs * V + lane - V;
    float best = has ? ex : -kInf;
    bool any = has && ex == ex;
#pragma unroll
    for (int j = 0; j < L; ++j) {
      best = fmaxf(best, vm[j]);
      any |= lane + j * 64 < cut.vecs;
    }
    const int found = select_top<64>(s, lane, any ? value_key(best) : 0, a.top, [&](const auto& f) {
      if (has) f(full_key(ex, at));
#pragma unroll
      for (int j = 0; j < L; ++j)
        if (lane + j * 64 < cut.vecs) {
#pragma unroll
          for (int e = 0; e < V; ++e)
            f(full_key(element<T>(p[j], e), (uint32_t)(cut.head + (lane + j * 64) * V + e)));
        }
    });
    if (lane < a.top) write_top(a, row, lane, lane < found ? s.out[lane] : 0, r);
  }
}

// ---- gradient ----
struct GradArgs {
  const void* logits;
  const int64_t* tokens;
  const float* stats;
  const float* entropy;
  const float* g_logp;     // or NULL
  const float* g_entropy;  // or NULL
  void* out;
  int64_t stride, out_stride, n;
  int vocab, chunks;
};

constexpr int kGradVecs = 4;  // vectors of a thread

// One logit's gradient: g its row's a, b and stats.
struct RowGrad {
  float m, logs, ent, a, b;
  int token;  // or -1
  bool none;  // zeros
};
template <bool kEntropy>
__device__ __forceinline__ float grad_of(float x, int i, const RowGrad& g) {
  const float lp = (x - g.m) - g.logs;
  const float p = expf(lp);
  float d = -g.a * p;
  // (p is 0 from lp = -104 on, whatever lp is then)
  if constexpr (kEntropy) d = __builtin_fmaf(-g.b * p, (lp < -200.0f ? -200.0f : lp) + g.ent, d);
  if (i == g.token) d += g.a;
  return g.none ? 0.0f : d;
}

// kTeam threads take a chunk of a row: a block, or a wave where that is all of
// it. Bound by HBM: 8192 x 32,000 bf16 takes 214 us, 4.9 TB/s; 100,000 rows of 100 a
// wave each 40.
template <class T, bool kEntropy, int kTeam>
__global__ __launch_bounds__(kChunkThreads) void k_logp_grad(GradArgs a) {
  constexpr int V = 16 / sizeof(T);
  const int tid = threadIdx.x % kTeam;
  const int64_t row = kTeam == 64 ? (int64_t)blockIdx.x * (kChunkThreads / 64) + threadIdx.x / 64
                                  : blockIdx.x / (uint32_t)a.chunks;
  const int chunk = kTeam == 64 ? 0 : (int)(blockIdx.x % (uint32_t)a.chunks);
  if (row >= a.n) return;
  const T* x = static_cast<const T*>(a.logits) + row * a.stride;
  T* out = static_cast<T*>(a.out) + row * a.out_stride;
  const Cut<T> cut(x, a.vocab);
  const int first = chunk * kGradVecs * kTeam + tid;
  Raw p[kGradVecs] = {};
#pragma unroll
  for (int j = 0; j < kGradVecs; ++j) {
    const int v = first + j * kTeam;
    if (v < cut.vecs) p[j] = load_raw(x + cut.head + (int64_t)v * V);
  }
  int extra = -1;
  if (chunk == 0 && tid < cut.head) extra = tid;
  if (chunk == a.chunks - 1 && tid >= V && tid < V + cut.tail) extra = cut.head + cut.vecs * V + tid - V;
  float ex = 0.0f;
  if (extra >= 0) ex = (float)x[extra];

  RowGrad g;
  g.m = a.stats[2 * row];
  g.logs = a.stats[2 * row + 1];
  g.none = g.m == -kInf;
  g.a = g.b = g.ent = 0.0f;
  g.token = -1;
  if constexpr (kEntropy) {
    g.b = a.g_entropy[row];
    g.ent = a.entropy[row];
  }
  if (a.g_logp != nullptr) {
    const int64_t t = a.tokens[row];
    if (t >= 0) {
      g.a = t < a.vocab ? a.g_logp[row] : __builtin_nanf("");
      g.token = t < a.vocab ? (int)t : -1;
      if (t >= a.vocab) g.none = false;
    } else if (g.b == 0.0f) {
      g.none = true;  // (the logits behind a batch's last position may be anything)
    }
  }
#pragma unroll
  for (int j = 0; j < kGradVecs; ++j) {
    const int v = first + j * kTeam;
    if (v < cut.vecs) {
      const int i = cut.head + v * V;
      LoosePack<T, V> o;
#pragma unroll
      for (int e = 0; e < V; ++e) o.v[e] = (T)grad_of<kEntropy>(element<T>(p[j], e), i + e, g);
      *reinterpret_cast<LoosePack<T, V>*>(out + i) = o;
    }
  }
  if (extra >= 0) out[extra] = (T)grad_of<kEntropy>(ex, extra, g);
}

// How rows are cut: a wave a row of few logits; a block a row, chunk by chunk,
// where the rows fill the device; else chunks on blocks of their own and a
// join. A row that fits one chunk is one, with the fewest vectors a thread; a
// longer one has the largest chunks unless these are too few to fill the device.
constexpr int64_t kFillBlocks = 512, kFillRows = 1024;
constexpr int kWaveVecs = 128;  // vectors of a row that a wave takes
enum Cutting : int { kWaveRow, kBlockRow, kChunks };
struct ChunkPlan {
  int L, chunks;
  Cutting how;
};
ChunkPlan chunk_plan(int64_t n, int64_t vocab, int size) {
  const int64_t vecs = vocab / (16 / size);
  ChunkPlan c;
  c.L = 1;
  c.chunks = 1;
  c.how = vecs <= kWaveVecs ? kWaveRow : kChunks;
  const int64_t across = c.how == kWaveRow ? 64 : kChunkThreads;
  while (c.L < 8 && vecs > c.L * across) c.L *= 2;
  const auto chunks = [&] { return std::max<int64_t>(1, (vecs + c.L * across - 1) / (c.L * across)); };
  if (chunks() > 1) {
    if (n >= kFillRows && chunks() * kGroups * kRowVecs <= kRowGroups) c.how = kBlockRow;
    else
      while (c.L > 1 && n * chunks() < kFillBlocks) c.L /= 2;
  }
  c.chunks = (int)chunks();
  return c;
}
static_assert(kRowVecs == 8, "chunk_plan's largest chunks are those of k_logp_long");

// Rows of one launch: at most 2^23 blocks (a grid has fewer than 2^32 threads).
constexpr int64_t kGridBlocks = 1 << 23;

template <class T, int L>
hipError_t launch_chunks(const LogpArgs& a, Cutting how, hipStream_t st) {
  const dim3 block(kChunkThreads), rows((unsigned)a.n);
  if (how == kWaveRow) {
    if constexpr (L <= 2) {
      const dim3 grid((unsigned)((a.n + 3) / 4));
      if (a.top > 0) hipLaunchKernelGGL((k_logp_rows<T, L, true>), grid, block, 0, st, a);
      else hipLaunchKernelGGL((k_logp_rows<T, L, false>), grid, block, 0, st, a);
    }
  } else if (how == kBlockRow) {
    if constexpr (L == kRowVecs) {
      const size_t lds = sizeof(uint32_t) * a.chunks * a.chunk_groups;
      if (a.top > 0) hipLaunchKernelGGL((k_logp_long<T, true>), rows, block, lds, st, a);
      else hipLaunchKernelGGL((k_logp_long<T, false>), rows, block, 0, st, a);
    }
  } else {
    const dim3 grid((unsigned)(a.n * a.chunks));
    if (a.top == 0) hipLaunchKernelGGL((k_logp_chunk<T, L, kNoTop>), grid, block, 0, st, a);
    else if (a.chunks > 1) hipLaunchKernelGGL((k_logp_chunk<T, L, kLeaveTop>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((k_logp_chunk<T, L, kTakeTop>), grid, block, 0, st, a);
    if (a.chunks > 1) hipLaunchKernelGGL((k_logp_join<T>), rows, block, 0, st, a);
  }
  return hipGetLastError();
}

template <class T>
hipError_t launch_logp(LogpArgs a, const ChunkPlan& c, hipStream_t st) {
  const int64_t slice = std::max<int64_t>(1, kGridBlocks / a.chunks), n = a.n;
  for (int64_t at = 0; at < n; at += slice) {
    a.n = std::min(slice, n - at);
    const hipError_t e = c.L == 1 ? launch_chunks<T, 1>(a, c.how, st) : c.L == 2 ? launch_chunks<T, 2>(a, c.how, st)
                       : c.L == 4 ? launch_chunks<T, 4>(a, c.how, st) : launch_chunks<T, 8>(a, c.how, st);
    if (e != hipSuccess) return e;
    a.logits = static_cast<const T*>(a.logits) + a.n * a.stride;
    if (a.tokens != nullptr) a.tokens += a.n;
    if (a.logp != nullptr) a.logp += a.n;
    if (a.entropy != nullptr) a.entropy += a.n;
    if (a.stats != nullptr) a.stats += 2 * a.n;
    if (a.top_ids != nullptr) a.top_ids += a.n * a.top;
    if (a.top_logp != nullptr) a.top_logp += a.n * a.top;
    if (a.parts != nullptr) {
      a.parts += a.n * a.chunks;
      a.groups += a.n * a.chunks * a.chunk_groups;
    }
  }
  return hipSuccess;
}

template <class T>
hipError_t launch_logp_grad(GradArgs a, bool wave, hipStream_t st) {
  const int64_t slice = std::max<int64_t>(1, kGridBlocks / a.chunks), n = a.n;
  for (int64_t at = 0; at < n; at += slice) {
    a.n = std::min(slice, n - at);
    const dim3 grid((unsigned)(wave ? (a.n + 3) / 4 : a.n * a.chunks)), block(kChunkThreads);
    if (wave) {
      if (a.g_entropy != nullptr) hipLaunchKernelGGL((k_logp_grad<T, true, 64>), grid, block, 0, st, a);
      else hipLaunchKernelGGL((k_logp_grad<T, false, 64>), grid, block, 0, st, a);
    } else {
      if (a.g_entropy != nullptr) hipLaunchKernelGGL((k_logp_grad<T, true, kChunkThreads>), grid, block, 0, st, a);
      else hipLaunchKernelGGL((k_logp_grad<T, false, kChunkThreads>), grid, block, 0, st, a);
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    a.logits = static_cast<const T*>(a.logits) + a.n * a.stride;
    a.out = static_cast<T*>(a.out) + a.n * a.out_stride;
    a.stats += 2 * a.n;
    if (a.tokens != nullptr) a.tokens += a.n;
    if (a.entropy != nullptr) a.entropy += a.n;
    if (a.g_logp != nullptr) a.g_logp += a.n;
    if (a.g_entropy != nullptr) a.g_entropy += a.n;
  }
  return hipSuccess;
}

int check_logits(const void* logits, int64_t stride, int64_t n, int64_t vocab, int dtype) {
  if (n < 0 || n > 0x7FFFFFFFll) return op_error(MLKV_EINVAL, "n must be in [0, 2^31 - 1]");
  if (vocab < 1 || vocab > MLKV_LOGITS_MAX_VOCAB) return op_error(MLKV_EINVAL, "vocab must be in [1, 2^24]");
  const int size = dtype_size(dtype);
  if (size == 0) return op_error(MLKV_EINVAL, "unknown dtype");
  if (n > 0 && logits == nullptr) return op_error(MLKV_EINVAL, "logits is NULL");
  if (!stride_ok(stride, n, vocab, true)) return op_error(MLKV_EINVAL, "stride must be 0 or >= vocab");
  if (!all_aligned(size, {logits}))
    return op_error(MLKV_EINVAL, "a pointer is not aligned to its element type");
  return MLKV_OK;
}

}  // namespace
}  // namespace mlkv

using namespace mlkv;

extern "C" {

int64_t mlkv_log_probs_workspace(int64_t n, int64_t vocab, int32_t top, int dtype) {
  const int rc = check_logits(nullptr, vocab, 0, vocab, dtype);
  if (rc) return rc;
  if (n < 0 || n > 0x7FFFFFFFll) return op_error(MLKV_EINVAL, "n must be in [0, 2^31 - 1]");
  if (top < 0 || top > MLKV_LOGITS_MAX_TOP || top > vocab)
    return op_error(MLKV_EINVAL, "top must be in [0, min(vocab, 64)]");
  const ChunkPlan c = chunk_plan(n, vocab, dtype_size(dtype));
  if (c.how != kChunks || c.chunks == 1) return 0;
  return n * c.chunks * (int64_t)(sizeof(Part) + (top > 0 ? sizeof(uint32_t) * kGroups * c.L : 0));
}

int mlkv_log_probs(const void* d_logits, int64_t stride, const int64_t* d_tokens, int64_t n, int64_t vocab,
                   int32_t top, int dtype, float* d_logp, float* d_entropy, float* d_stats, int64_t* d_top_ids,
                   float* d_top_logp, void* d_work, int64_t work_bytes, void* hip_stream) {
  const int rc = check_logits(d_logits, stride, n, vocab, dtype);
  if (rc) return rc;
  const int64_t bytes = mlkv_log_probs_workspace(n, vocab, top, dtype);
  if (bytes < 0) return (int)bytes;
  if (d_logp != nullptr && d_tokens == nullptr && n > 0) return op_error(MLKV_EINVAL, "tokens is NULL");
  if (top == 0 && (d_top_ids != nullptr || d_top_logp != nullptr))
    return op_error(MLKV_EINVAL, "top_ids and top_logp must be NULL with top = 0");
  if (!all_aligned(8, {d_tokens, d_top_ids}) ||
      !all_aligned(4, {d_logp, d_entropy, d_stats, d_top_logp}))
    return op_error(MLKV_EINVAL, "a pointer is not aligned to its element type");
  if (bytes > 0) {
    if (d_work == nullptr || work_bytes < bytes)
      return op_error(MLKV_EINVAL, "work is smaller than mlkv_log_probs_workspace");
    if (!all_aligned(16, {d_work})) return op_error(MLKV_EINVAL, "work must be at a multiple of 16 bytes");
  }
  if (n == 0) return MLKV_OK;
  const ChunkPlan c = chunk_plan(n, vocab, dtype_size(dtype));
  LogpArgs a{};
  a.logits = d_logits;
  a.tokens = d_tokens;
  a.logp = d_logp;
  a.entropy = d_entropy;
  a.stats = d_stats;
  a.top_ids = d_top_ids;
  a.top_logp = d_top_logp;
  if (bytes > 0) {
    a.parts = static_cast<Part*>(d_work);
    a.groups = reinterpret_cast<uint32_t*>(static_cast<char*>(d_work) + sizeof(Part) * (size_t)(n * c.chunks));
  }
  a.stride = stride;
  a.n = n;
  a.vocab = (int)vocab;
  a.top = d_top_ids != nullptr || d_top_logp != nullptr ? top : 0;
  a.chunks = c.chunks;
  a.chunk_groups = kGroups * c.L;
  const hipError_t e = dispatch_type(dtype, [&](auto t) {
    return launch_logp<decltype(t)>(a, c, static_cast<hipStream_t>(hip_stream));
  });
  return e == hipSuccess ? MLKV_OK : op_launch_error(e, "mlkv_log_probs launch");
}

int mlkv_log_probs_grad(const void* d_logits, int64_t stride, const int64_t* d_tokens, const float* d_stats,
                        const float* d_entropy, const float* d_logp_grad, const float* d_entropy_grad, int64_t n,
                        int64_t vocab, int dtype, void* d_logits_grad, int64_t grad_stride, void* hip_stream) {
  const int rc = check_logits(d_logits, stride, n, vocab, dtype);
  if (rc) return rc;
  const int size = dtype_size(dtype);
  if (n > 0) {
    if (d_stats == nullptr) return op_error(MLKV_EINVAL, "stats is NULL");
    if (d_logits_grad == nullptr) return op_error(MLKV_EINVAL, "logits_grad is NULL");
    if (d_logp_grad != nullptr && d_tokens == nullptr) return op_error(MLKV_EINVAL, "tokens is NULL");
    if (d_entropy_grad != nullptr && d_entropy == nullptr) return op_error(MLKV_EINVAL, "entropy is NULL");
  }
  if (!stride_ok(grad_stride, n, vocab, false)) return op_error(MLKV_EINVAL, "grad_stride must be >= vocab");
  if (!all_aligned(size, {d_logits_grad}) || !all_aligned(8, {d_tokens}) ||
      !all_aligned(4, {d_stats, d_entropy, d_logp_grad, d_entropy_grad}))
    return op_error(MLKV_EINVAL, "a pointer is not aligned to its element type");
  if (n > 1 && d_logits_grad == d_logits && stride != grad_stride)
    return op_error(MLKV_EINVAL, "logits_grad may be logits only with the same stride");
  const RowSpan out = row_span(d_logits_grad, grad_stride, n, vocab, size);
  const auto meets = [&](const void* p, int64_t bytes) { return rows_meet({p, 0, 1, n * bytes}, out); };
  if (!out_ok(row_span(d_logits, stride, n, vocab, size), out) || meets(d_tokens, 8) || meets(d_stats, 8) ||
      meets(d_entropy, 4) || meets(d_logp_grad, 4) || meets(d_entropy_grad, 4))
    return op_error(MLKV_EINVAL, "logits_grad overlaps an input");
  if (n == 0) return MLKV_OK;
  GradArgs a{};
  a.logits = d_logits;
  a.tokens = d_tokens;
  a.stats = d_stats;
  a.entropy = d_entropy;
  a.g_logp = d_logp_grad;
  a.g_entropy = d_entropy_grad;
  a.out = d_logits_grad;
  a.stride = stride;
  a.out_stride = grad_stride;
  a.vocab = (int)vocab;
  a.n = n;
  const int64_t per = (int64_t)kGradVecs * kChunkThreads, vecs = vocab / (16 / size);
  const bool wave = vecs <= kGradVecs * 64;
  a.chunks = (int)std::max<int64_t>(1, (vecs + per - 1) / per);
  const hipError_t e = dispatch_type(dtype, [&](auto t) {
    return launch_logp_grad<decltype(t)>(a, wave, static_cast<hipStream_t>(hip_stream));
  });
  return e == hipSuccess ? MLKV_OK : op_launch_error(e, "mlkv_log_probs_grad launch");
}

}  // extern "C"
