// Log probabilities of given tokens with entropy and top alternatives, and
// their gradient in the logits.
//
// A row is cut into chunks, a block each, that hold their logits in registers:
// every logit is read once. A thread sums e = exp(x - m) and e (x - m) against
// the largest logit m of its own, and the joins (lanes, waves, chunks) rescale
// to the larger of two maxima, the running softmax. A second kernel joins a
// row's chunks, if there are several. Bound by HBM: about 12 operations a
// logit, one of them an exponential, against 2 or 4 bytes.
//
// Alternatives are ordered by one 64-bit key of value and index, so that equal
// logits have an order and no two keys are equal. The k-th largest of the
// threads' own largest keys is a bound that the row's k largest reach, and at
// most k threads reach it: only their few logits are ranked.
#include "mlkv_ops.h"

#include <algorithm>

namespace mlkv {
namespace {

constexpr int kChunkThreads = 256;
constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kInf = __builtin_inff();

// Sums of a part of a row: m its largest logit, s = sum 2^z, t = sum z 2^z
// with z = (x - m) log2(e).
struct Part {
  float m, s, t, pad;
};

__device__ __forceinline__ Part part_join(const Part& a, const Part& b) {
  Part r;
  r.m = fmaxf(a.m, b.m);
  // a part of -inf alone has nothing to rescale
  const float da = a.m == -kInf ? 0.0f : (a.m - r.m) * kLog2e;
  const float db = b.m == -kInf ? 0.0f : (b.m - r.m) * kLog2e;
  const float fa = __builtin_amdgcn_exp2f(da), fb = __builtin_amdgcn_exp2f(db);
  r.s = fa * a.s + fb * b.s;
  // (2^z is 0 long before z leaves the range in which z 2^z is 0)
  r.t = fa * __builtin_fmaf(fmaxf(da, -1e4f), a.s, a.t) + fb * __builtin_fmaf(fmaxf(db, -1e4f), b.s, b.t);
  r.pad = 0.0f;
  return r;
}

__device__ __forceinline__ Part wave_join(Part p) {
#pragma unroll
  for (int o = 1; o < 64; o *= 2) {
    Part q;
    q.m = __shfl_xor(p.m, o);
    q.s = __shfl_xor(p.s, o);
    q.t = __shfl_xor(p.t, o);
    q.pad = 0.0f;
    // the lower lane's part first on both sides: equal bits in every lane
    p = (threadIdx.x & o) ? part_join(q, p) : part_join(p, q);
  }
  return p;
}

// Order of logits as unsigned numbers; -0 counts as +0. Every logit's is over 0.
__device__ __forceinline__ uint32_t value_key(float x) {
  const uint32_t b = __float_as_uint(x + 0.0f);
  return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float key_value(uint32_t k) {
  return __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k);
}
// value, then lowest index first
__device__ __forceinline__ uint64_t full_key(float x, uint32_t i) {
  return (uint64_t)value_key(x) << 32 | (uint32_t)~i;
}

struct LogpArgs {
  const void* logits;
  const int64_t* tokens;  // or NULL
  float* logp;            // or NULL, as are all outputs
  float* entropy;
  float* stats;
  int64_t* top_ids;
  float* top_logp;
  Part* parts;            // [n][chunks]
  uint64_t* keys;         // [n][chunks][top], largest first; 0 where a chunk has fewer
  int64_t stride, n;
  int vocab, top, chunks;
};

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
    const double s = (double)p.s, l = log(s);
    r.m = p.m;
    r.logs = (float)l;
    r.ent = (float)(l - (double)p.t * 0.693147180559945309417 / s);
  }
  return r;
}

__device__ __forceinline__ float log_prob(float x, const RowStats& r) { return r.none ? -kInf : (x - r.m) - r.logs; }

template <class T>
__device__ __forceinline__ void write_row(const LogpArgs& a, int64_t row, const RowStats& r) {
  if (a.stats != nullptr) {
    a.stats[2 * row] = r.m;
    a.stats[2 * row + 1] = r.logs;
  }
  if (a.entropy != nullptr) a.entropy[row] = r.ent;
  if (a.logp != nullptr) {
    const int64_t t = a.tokens[row];
    float lp = 0.0f;
    if (t >= a.vocab) lp = __builtin_nanf("");
    else if (t >= 0) lp = log_prob((float)static_cast<const T*>(a.logits)[row * a.stride + t], r);
    a.logp[row] = lp;
  }
}

__device__ __forceinline__ void write_top(const LogpArgs& a, int64_t row, int rank, uint64_t key, const RowStats& r) {
  if (a.top_ids != nullptr) a.top_ids[row * a.top + rank] = r.m != r.m ? -1 : (int64_t)(uint32_t)~(uint32_t)key;
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

// One chunk of a row: L vectors a thread.
template <class T, int L, bool kTop>
__global__ __launch_bounds__(kChunkThreads) void k_logp_chunk(LogpArgs a) {
  constexpr int V = 16 / sizeof(T), kWaves = kChunkThreads / 64;
  __shared__ Part wave_part[kWaves];
  __shared__ uint32_t quad_key[64];
  __shared__ uint64_t list[kChunkThreads];
  __shared__ uint64_t bound;
  __shared__ int listed, cands;
  extern __shared__ uint64_t cand[];  // [top * (L * V + 1)]
  const int tid = threadIdx.x, lane = tid & 63;
  const int64_t row = blockIdx.x / (uint32_t)a.chunks;
  const int chunk = (int)(blockIdx.x % (uint32_t)a.chunks);
  const T* x = static_cast<const T*>(a.logits) + row * a.stride;
  const Cut<T> cut(x, a.vocab);
  const T* body = x + cut.head;
  const int first = chunk * L * kChunkThreads + tid;  // the thread's vectors: first + j * kChunkThreads
  Pack<T, V> p[L];
#pragma unroll
  for (int j = 0; j < L; ++j) {
    const int v = first + j * kChunkThreads;
    if (v < cut.vecs) {
      p[j] = *reinterpret_cast<const Pack<T, V>*>(body + (int64_t)v * V);
    } else {
#pragma unroll
      for (int e = 0; e < V; ++e) p[j].v[e] = (T)-kInf;
    }
  }
  // the first chunk takes the elements before the vectors, the last those behind, one a thread
  int extra = -1;
  float ex = -kInf;
  if (chunk == 0 && tid < cut.head) extra = tid;
  if (chunk == a.chunks - 1 && tid >= V && tid < V + cut.tail) extra = cut.head + cut.vecs * V + tid - V;
  if (extra >= 0) ex = (float)x[extra];

  if constexpr (kTop) {
    if (tid == 0) listed = cands = 0;
  }
  float vm[L], m = ex;
#pragma unroll
  for (int j = 0; j < L; ++j) {
    vm[j] = -kInf;
#pragma unroll
    for (int e = 0; e < V; ++e) vm[j] = fmaxf(vm[j], (float)p[j].v[e]);
    m = fmaxf(m, vm[j]);
  }
  if (m != m) m = -kInf;  // (a lone NaN)
  const float base = m == -kInf ? 0.0f : m;
  Part mine;
  mine.m = m;
  mine.pad = 0.0f;
  {
    const float z = (ex - base) * kLog2e, q = __builtin_amdgcn_exp2f(z);
    mine.s = q;
    mine.t = q * fmaxf(z, -150.0f);
  }
#pragma unroll
  for (int j = 0; j < L; ++j)
#pragma unroll
    for (int e = 0; e < V; ++e) {
      const float z = ((float)p[j].v[e] - base) * kLog2e, q = __builtin_amdgcn_exp2f(z);
      mine.s += q;
      mine.t = __builtin_fmaf(q, fmaxf(z, -150.0f), mine.t);  // (z may be -inf)
    }
  const Part joined = wave_join(mine);
  if (lane == 0) wave_part[tid >> 6] = joined;

  const bool owns = first < cut.vecs || extra >= 0;
  if constexpr (kTop) {
    // a value that at least `top` threads reach, from the largest of every four threads
    uint32_t k = owns ? value_key(m) : 0;
    k = max(k, (uint32_t)__shfl_xor((int)k, 1));
    k = max(k, (uint32_t)__shfl_xor((int)k, 2));
    if ((lane & 3) == 0) quad_key[tid >> 2] = k;
  }
  __syncthreads();
  Part all = wave_part[0];
#pragma unroll
  for (int w = 1; w < kWaves; ++w) all = part_join(all, wave_part[w]);

  uint64_t best = 0;
  int nc = 0;
  if constexpr (kTop) {
    const uint32_t q = quad_key[lane];
    uint32_t low = 0;
#pragma unroll 1
    for (int bit = 31; bit >= 16; --bit) {
      const uint32_t t = low | 1u << bit;
      if (__popcll(__ballot(q >= t)) >= a.top) low = t;
    }
    // the first of a thread's largest logits, for the threads that reach it
    const bool reach = owns && value_key(m) >= low;
    if (__any(reach)) {
      uint32_t at = 0xFFFFFFFFu;
      if (extra >= 0 && ex == m) at = (uint32_t)extra;
#pragma unroll
      for (int j = L - 1; j >= 0; --j) {
        const int v = first + j * kChunkThreads;
        if (reach && v < cut.vecs && vm[j] == m) {
#pragma unroll
          for (int e = V - 1; e >= 0; --e)
            if ((float)p[j].v[e] == m && !(extra >= 0 && extra < cut.head && ex == m))
              at = (uint32_t)(cut.head + v * V + e);
        }
      }
      if (reach && at != 0xFFFFFFFFu) {
        best = full_key(m, at);
        list[atomicAdd(&listed, 1)] = best;
      }
    }
    __syncthreads();
    // the top-th largest of them: no more than `top` threads hold keys as large
    const int nl = listed;
    if (best != 0) {
      int over = 0;
      for (int i = 0; i < nl; ++i) over += list[i] > best;
      if (over == a.top - 1) bound = best;
    }
    if (nl < a.top && tid == 0) bound = 0;  // fewer threads have logits: all of those count
    __syncthreads();
    const uint64_t least = bound;
    if (best != 0 && best >= least) {
      const float lv = least ? key_value((uint32_t)(least >> 32)) : -kInf;
      if (extra >= 0 && ex >= lv) {
        const uint64_t f = full_key(ex, (uint32_t)extra);
        if (f >= least) cand[atomicAdd(&cands, 1)] = f;
      }
#pragma unroll
      for (int j = 0; j < L; ++j) {
        const int v = first + j * kChunkThreads;
        if (v < cut.vecs && vm[j] >= lv) {
#pragma unroll
          for (int e = 0; e < V; ++e) {
            const uint64_t f = full_key((float)p[j].v[e], (uint32_t)(cut.head + v * V + e));
            if (f >= least && !((float)p[j].v[e] != (float)p[j].v[e])) cand[atomicAdd(&cands, 1)] = f;
          }
        }
      }
    }
    __syncthreads();
    nc = cands;
  }
  if (a.chunks == 1) {
    const RowStats r = row_stats(all);
    if (tid == 0) write_row<T>(a, row, r);
    if constexpr (kTop) {
      for (int i = tid; i < nc; i += kChunkThreads) {
        const uint64_t f = cand[i];
        int over = 0;
        for (int o = 0; o < nc; ++o) over += cand[o] > f;
        if (over < a.top) write_top(a, row, over, f, r);
      }
      // (fewer keys than alternatives only where NaNs took their places)
      for (int i = nc + tid; i < a.top; i += kChunkThreads) write_top(a, row, i, 0, r);
    }
  } else {
    if (tid == 0) a.parts[row * a.chunks + chunk] = all;
    if constexpr (kTop) {
      uint64_t* to = a.keys + (row * a.chunks + chunk) * a.top;
      for (int i = tid; i < nc; i += kChunkThreads) {
        const uint64_t f = cand[i];
        int over = 0;
        for (int o = 0; o < nc; ++o) over += cand[o] > f;
        if (over < a.top) to[over] = f;
      }
      for (int i = nc + tid; i < a.top; i += kChunkThreads) to[i] = 0;
    }
  }
}

// Joins a row's chunks: a block a row. The bound on the alternatives: of the
// chunks' keys number d the r-th largest, with r (d + 1) >= top keys as large.
constexpr int kJoinThreads = 256;
inline size_t join_lds(int chunks, int top) {
  return sizeof(uint64_t) * ((size_t)chunks + (size_t)top * (std::min(chunks, top) + 1));
}
template <class T>
__global__ __launch_bounds__(kJoinThreads) void k_logp_join(LogpArgs a) {
  constexpr int kWaves = kJoinThreads / 64;
  __shared__ Part wave_part[kWaves];
  __shared__ uint64_t bound;
  __shared__ int cands;
  extern __shared__ uint64_t lds[];
  uint64_t* head = lds;              // [chunks]
  uint64_t* cand = lds + a.chunks;   // [top * (min(chunks, top) + 1)]
  const int tid = threadIdx.x;
  const int64_t row = blockIdx.x;
  Part mine;
  mine.m = -kInf;
  mine.s = mine.t = mine.pad = 0.0f;
  for (int c = tid; c < a.chunks; c += kJoinThreads) mine = part_join(mine, a.parts[row * a.chunks + c]);
  mine = wave_join(mine);
  if ((tid & 63) == 0) wave_part[tid >> 6] = mine;
  const uint64_t* keys = a.keys + row * a.chunks * a.top;
  const int depth = a.top ? (a.top + a.chunks - 1) / a.chunks - 1 : 0;
  const int need = a.top ? (a.top + depth) / (depth + 1) : 0;  // <= chunks
  if (a.top) {
    for (int c = tid; c < a.chunks; c += kJoinThreads) head[c] = keys[(int64_t)c * a.top + depth];
    if (tid == 0) {
      cands = 0;
      bound = 0;  // (stays where fewer chunks have a key there: all keys count then)
    }
  }
  __syncthreads();
  Part all = wave_part[0];
#pragma unroll
  for (int w = 1; w < kWaves; ++w) all = part_join(all, wave_part[w]);
  const RowStats r = row_stats(all);
  if (tid == 0) write_row<T>(a, row, r);
  if (a.top == 0) return;
  for (int c = tid; c < a.chunks; c += kJoinThreads) {
    const uint64_t k = head[c];
    if (k == 0) continue;
    int over = 0;
    for (int o = 0; o < a.chunks; ++o) over += head[o] > k;
    if (over == need - 1) bound = k;
  }
  __syncthreads();
  const uint64_t least = bound;
  // `need` chunks have up to `top` keys as large as the bound, the others up to
  // `depth`: fewer than top * (need + 1) in all. More (no bound, because NaNs
  // left chunks without keys) only where the ids are -1 anyway.
  const int total = a.chunks * a.top, most = a.top * (min(a.chunks, a.top) + 1);
  for (int i = tid; i < total; i += kJoinThreads) {
    const uint64_t k = keys[i];
    if (k != 0 && k >= least) {
      const int at = atomicAdd(&cands, 1);
      if (at < most) cand[at] = k;
    }
  }
  __syncthreads();
  const int nc = min(cands, most);
  for (int i = tid; i < nc; i += kJoinThreads) {
    const uint64_t f = cand[i];
    int over = 0;
    for (int o = 0; o < nc; ++o) over += cand[o] > f;
    if (over < a.top) write_top(a, row, over, f, r);
  }
  for (int i = nc + tid; i < a.top; i += kJoinThreads) write_top(a, row, i, 0, r);
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
  int64_t stride, out_stride;
  int vocab, chunks;
};

constexpr int kGradVecs = 4;  // vectors of a thread

// One logit's gradient: g its row's a, b and stats.
struct RowGrad {
  float m, logs, ent, a, b;
  int token;  // or -1
  bool none;
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

template <class T, bool kEntropy>
__global__ __launch_bounds__(kChunkThreads) void k_logp_grad(GradArgs a) {
  constexpr int V = 16 / sizeof(T);
  const int64_t row = blockIdx.x / (uint32_t)a.chunks;
  const int chunk = (int)(blockIdx.x % (uint32_t)a.chunks);
  const int tid = threadIdx.x;
  const T* x = static_cast<const T*>(a.logits) + row * a.stride;
  T* out = static_cast<T*>(a.out) + row * a.out_stride;
  const Cut<T> cut(x, a.vocab);
  const int first = chunk * kGradVecs * kChunkThreads + tid;
  Pack<T, V> p[kGradVecs];
#pragma unroll
  for (int j = 0; j < kGradVecs; ++j) {
    const int v = first + j * kChunkThreads;
    if (v < cut.vecs) p[j] = *reinterpret_cast<const Pack<T, V>*>(x + cut.head + (int64_t)v * V);
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
  g.a = 0.0f;
  g.token = -1;
  if (a.g_logp != nullptr) {
    const int64_t t = a.tokens[row];
    if (t >= 0) {
      g.a = t < a.vocab ? a.g_logp[row] : __builtin_nanf("");
      g.token = t < a.vocab ? (int)t : -1;
      if (t >= a.vocab) g.none = false;
    }
  }
  g.b = g.ent = 0.0f;
  if constexpr (kEntropy) {
    g.b = a.g_entropy[row];
    g.ent = a.entropy[row];
  }
#pragma unroll
  for (int j = 0; j < kGradVecs; ++j) {
    const int v = first + j * kChunkThreads;
    if (v < cut.vecs) {
      const int i = cut.head + v * V;
      LoosePack<T, V> o;
#pragma unroll
      for (int e = 0; e < V; ++e) o.v[e] = (T)grad_of<kEntropy>((float)p[j].v[e], i + e, g);
      *reinterpret_cast<LoosePack<T, V>*>(out + i) = o;
    }
  }
  if (extra >= 0) out[extra] = (T)grad_of<kEntropy>(ex, extra, g);
}

// How rows are cut: vectors a thread and chunks a row. A row that fits one
// chunk is one, with the fewest vectors a thread; a longer one has the largest
// chunks unless these are too few to fill the device.
constexpr int64_t kFillBlocks = 512;
struct ChunkPlan {
  int L, chunks;
};
ChunkPlan chunk_plan(int64_t n, int64_t vocab, int size) {
  const int64_t vecs = vocab / (16 / size);
  ChunkPlan c;
  c.L = 1;
  while (c.L < 8 && vecs > (int64_t)c.L * kChunkThreads) c.L *= 2;
  const auto chunks = [&] {
    const int64_t per = (int64_t)c.L * kChunkThreads;
    return std::max<int64_t>(1, (vecs + per - 1) / per);
  };
  if (chunks() > 1)
    while (c.L > 1 && n * chunks() < kFillBlocks) c.L /= 2;
  c.chunks = (int)chunks();
  return c;
}

// Rows of one launch: at most 2^23 blocks (a grid has fewer than 2^32 threads).
constexpr int64_t kGridBlocks = 1 << 23;

template <class T, int L>
hipError_t launch_chunks(const LogpArgs& a, int64_t rows, hipStream_t st) {
  const dim3 grid((unsigned)(rows * a.chunks)), block(kChunkThreads);
  if (a.top > 0) {
    constexpr int V = 16 / sizeof(T);
    hipLaunchKernelGGL((k_logp_chunk<T, L, true>), grid, block, sizeof(uint64_t) * a.top * (L * V + 1), st, a);
  } else {
    hipLaunchKernelGGL((k_logp_chunk<T, L, false>), grid, block, 0, st, a);
  }
  return hipGetLastError();
}

template <class T>
hipError_t launch_logp(LogpArgs a, int L, hipStream_t st) {
  const int64_t slice = std::max<int64_t>(1, kGridBlocks / a.chunks), n = a.n;
  for (int64_t at = 0; at < n; at += slice) {
    const int64_t rows = std::min(slice, n - at);
    hipError_t e = L == 1 ? launch_chunks<T, 1>(a, rows, st) : L == 2 ? launch_chunks<T, 2>(a, rows, st)
                 : L == 4 ? launch_chunks<T, 4>(a, rows, st) : launch_chunks<T, 8>(a, rows, st);
    if (e == hipSuccess && a.chunks > 1) {
      hipLaunchKernelGGL((k_logp_join<T>), dim3((unsigned)rows), dim3(kJoinThreads),
                         a.top ? join_lds(a.chunks, a.top) : 0, st, a);
      e = hipGetLastError();
    }
    if (e != hipSuccess) return e;
    a.logits = static_cast<const T*>(a.logits) + rows * a.stride;
    if (a.tokens != nullptr) a.tokens += rows;
    if (a.logp != nullptr) a.logp += rows;
    if (a.entropy != nullptr) a.entropy += rows;
    if (a.stats != nullptr) a.stats += 2 * rows;
    if (a.top_ids != nullptr) a.top_ids += rows * a.top;
    if (a.top_logp != nullptr) a.top_logp += rows * a.top;
    a.parts += rows * a.chunks;
    a.keys += rows * a.chunks * a.top;
  }
  return hipSuccess;
}

template <class T>
hipError_t launch_logp_grad(GradArgs a, int64_t n, hipStream_t st) {
  const int64_t slice = std::max<int64_t>(1, kGridBlocks / a.chunks);
  for (int64_t at = 0; at < n; at += slice) {
    const int64_t rows = std::min(slice, n - at);
    const dim3 grid((unsigned)(rows * a.chunks)), block(kChunkThreads);
    if (a.g_entropy != nullptr) hipLaunchKernelGGL((k_logp_grad<T, true>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((k_logp_grad<T, false>), grid, block, 0, st, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    a.logits = static_cast<const T*>(a.logits) + rows * a.stride;
    a.out = static_cast<T*>(a.out) + rows * a.out_stride;
    a.stats += 2 * rows;
    if (a.tokens != nullptr) a.tokens += rows;
    if (a.entropy != nullptr) a.entropy += rows;
    if (a.g_logp != nullptr) a.g_logp += rows;
    if (a.g_entropy != nullptr) a.g_entropy += rows;
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
  if (!all_aligned(size, size, {logits}, {}))
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
  if (c.chunks == 1) return 0;
  return n * c.chunks * (int64_t)(sizeof(Part) + sizeof(uint64_t) * top);
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
  if (!all_aligned(8, 1, {d_tokens, d_top_ids}, {}) ||
      !all_aligned(4, 1, {d_logp, d_entropy, d_stats, d_top_logp}, {}))
    return op_error(MLKV_EINVAL, "a pointer is not aligned to its element type");
  if (bytes > 0) {
    if (d_work == nullptr || work_bytes < bytes)
      return op_error(MLKV_EINVAL, "work is smaller than mlkv_log_probs_workspace");
    if (!all_aligned(16, 1, {d_work}, {})) return op_error(MLKV_EINVAL, "work must be at a multiple of 16 bytes");
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
  a.parts = static_cast<Part*>(d_work);
  a.keys = reinterpret_cast<uint64_t*>(static_cast<char*>(d_work) + sizeof(Part) * (size_t)(n * c.chunks));
  a.stride = stride;
  a.n = n;
  a.vocab = (int)vocab;
  a.top = d_top_ids != nullptr || d_top_logp != nullptr ? top : 0;
  a.chunks = c.chunks;
  const hipError_t e = dispatch_type(dtype, [&](auto t) {
    return launch_logp<decltype(t)>(a, c.L, static_cast<hipStream_t>(hip_stream));
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
  if (!all_aligned(size, size, {d_logits_grad}, {}) || !all_aligned(8, 1, {d_tokens}, {}) ||
      !all_aligned(4, 1, {d_stats, d_entropy, d_logp_grad, d_entropy_grad}, {}))
    return op_error(MLKV_EINVAL, "a pointer is not aligned to its element type");
  if (n > 1 && d_logits_grad == d_logits && stride != grad_stride)
    return op_error(MLKV_EINVAL, "logits_grad may be logits only with the same stride");
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
  const int64_t per = (int64_t)kGradVecs * kChunkThreads, vecs = vocab / (16 / size);
  a.chunks = (int)std::max<int64_t>(1, (vecs + per - 1) / per);
  const hipError_t e = dispatch_type(dtype, [&](auto t) {
    return launch_logp_grad<decltype(t)>(a, n, static_cast<hipStream_t>(hip_stream));
  });
  return e == hipSuccess ? MLKV_OK : op_launch_error(e, "mlkv_log_probs_grad launch");
}

}  // extern "C"
