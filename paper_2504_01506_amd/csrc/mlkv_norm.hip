// Layer norm and its gradient.
//
// A row belongs to a group of G lanes that holds it whole in registers, I
// vectors of 16 bytes a lane at any alignment, so each element is read once
// and both passes of the variance (mean, then squares about it) run on
// registers. Rows of up to 1024 elements have a group within a wave, several
// groups a block; longer ones have a block of waves each that exchange their
// sums through LDS. Both kernels are bound by HBM: 8 and 16 operations an
// element against 4 to 12 bytes. 16,384 x 4096 bf16 takes 52 us (5.2 TB/s) and
// its gradient 100 (4.0), a million fp32 rows of 128 the gradient 290 (5.3); of
// 10, 30. Rows of few bytes in all are bound by the launches.
//
// A row's loads are whole vectors in every lane, so that the next row's are in
// flight while a row is worked on: the vector that would reach past the row's
// end is moved back to end there and takes part with its last elements only,
// and a lane without any reads that vector too. (Element by element behind
// branches, the gradient of 16,384 x 4096 bf16 took 212 us.)
#include "mlkv_ops.h"

#include <algorithm>
#include <cmath>

namespace mlkv {
namespace {

constexpr int kNormThreads = 256;      // of a block of groups within waves
// Threads of a block that holds one row: up to kNormMidThreads the row after
// the present one is loaded ahead; more threads have too few registers for it.
constexpr int kNormMidThreads = 512, kNormMaxThreads = 1024;

struct NormArgs {
  const void* x;
  const void* grad;    // gradient only
  const void* weight;  // or NULL
  const void* bias;    // or NULL
  void* out;           // or NULL (gradient)
  void* sums;          // gradient: [blocks][2][dim] floats (doubles for rows shorter than a vector), or NULL
  int64_t x_stride, grad_stride, out_stride;
  int64_t n;
  int dim;
  int G;               // lanes of a row
  float eps;
  bool wide_weight;    // weight and bias are fp32, not of x's type
};

// A row's sums over the block's waves (rows that a whole block holds).
template <int N>
__device__ __forceinline__ void block_sums(float (&v)[N], float* lds) {
  const int waves = blockDim.x >> 6, wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
#pragma unroll
  for (int k = 0; k < N; ++k) {
    v[k] = group_sum(v[k], 64);
    if (lane == 0) lds[wave * N + k] = v[k];
  }
  __syncthreads();
  const int from = lane & 15;  // (at most 16 waves)
#pragma unroll
  for (int k = 0; k < N; ++k) v[k] = from < waves ? lds[from * N + k] : 0.0f;
#pragma unroll
  for (int k = 0; k < N; ++k) v[k] = group_sum(v[k], 16);
}

template <bool kBlock, int N>
__device__ __forceinline__ void row_sums(float (&v)[N], int G, float* lds) {
  if constexpr (kBlock) {
    block_sums(v, lds);
  } else {
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] = group_sum(v[k], G);
  }
}

// The columns of lane l: vector i begins at column at[i], and its elements
// from skip[i] on are the lane's own (all where kFull: a row is G * I vectors).
// Rows shorter than a vector (kShort) are loaded by elements, a lane a row.
template <class T, int I, bool kFull>
struct Columns {
  static constexpr int V = 16 / sizeof(T);
  int at[I], skip[I];
  __device__ __forceinline__ Columns(int l, int G, int dim) {
#pragma unroll
    for (int i = 0; i < I; ++i) {
      const int c = (i * G + l) * V;
      at[i] = kFull ? c : max(min(c, dim - V), 0);
      skip[i] = kFull ? 0 : min(c - at[i], V);
    }
  }
  __device__ __forceinline__ bool own(int i, int j) const { return kFull || j >= skip[i]; }
};

template <class T, int I, bool kFull, bool kShort>
__device__ __forceinline__ void load_row(Raw (&p)[I], const T* row, const Columns<T, I, kFull>& cols, int dim) {
  if constexpr (kShort) {
    constexpr int V = 16 / sizeof(T);
    union {
      Raw r;
      T v[V];
    } u;
    u.r = Raw{0, 0, 0, 0};
#pragma unroll
    for (int j = 0; j < V - 1; ++j)
      if (j < dim) u.v[j] = row[j];
    p[0] = u.r;
  } else {
#pragma unroll
    for (int i = 0; i < I; ++i) p[i] = load_raw(row + cols.at[i]);
  }
}

template <class T, int V, bool kShort>
__device__ __forceinline__ void store_row(T* row, int c, int dim, const LoosePack<T, V>& o) {
  if constexpr (kShort) {
#pragma unroll
    for (int j = 0; j < V - 1; ++j)
      if (j < dim) row[j] = o.v[j];
  } else {
    *reinterpret_cast<LoosePack<T, V>*>(row + c) = o;
  }
}

// One thread's columns of weight or bias.
template <class T, int I, bool kFull, bool kShort>
__device__ __forceinline__ void load_params(float (&w)[I * (16 / sizeof(T))], const void* p, bool wide, float none,
                                            const Columns<T, I, kFull>& cols, int dim) {
  constexpr int V = 16 / sizeof(T);
  const auto take = [&](auto of) {
    using P = decltype(of);
    constexpr int kPer = 16 / sizeof(P);
#pragma unroll
    for (int i = 0; i < I; ++i) {
      const P* at = static_cast<const P*>(p) + cols.at[i];
      if constexpr (kShort) {
#pragma unroll
        for (int j = 0; j < V; ++j) w[j] = j < dim ? (float)at[j] : none;
      } else {
#pragma unroll
        for (int j = 0; j < V; j += kPer) {
          const Raw r = load_raw(at + j);
#pragma unroll
          for (int e = 0; e < kPer; ++e) w[i * V + j + e] = element<P>(r, e);
        }
      }
    }
  };
  if (p == nullptr) {
#pragma unroll
    for (int e = 0; e < I * V; ++e) w[e] = none;
  } else if (wide) {
    take(float{});
  } else {
    take(T{});
  }
}

// kMost: threads of a block at most, 0 for rows within waves
template <class T, int I, int kMost, bool kFull, bool kShort>
__global__ __launch_bounds__(kMost ? kMost : kNormThreads) void k_layer_norm(NormArgs a) {
  __shared__ float lds1[kNormMaxThreads / 64];
  __shared__ float lds2[2 * kNormMaxThreads / 64];
  constexpr int V = 16 / sizeof(T);
  constexpr bool kBlock = kMost != 0, kAhead = kMost != kNormMaxThreads;
  const int G = a.G, l = kBlock ? threadIdx.x : threadIdx.x & (G - 1), dim = a.dim;
  const int per = kBlock ? 1 : kNormThreads / G;
  const float inv = 1.0f / (float)dim;
  const Columns<T, I, kFull> cols(l, G, dim);
  // (kShort: a lane has a row of its own, elements from dim on are not)
  const auto own = [&](int i, int j) { return kShort ? j < dim : cols.own(i, j); };
  float w[I * V], b[I * V];
  load_params<T, I, kFull, kShort>(w, a.weight, a.wide_weight, 1.0f, cols, dim);
  load_params<T, I, kFull, kShort>(b, a.bias, a.wide_weight, 0.0f, cols, dim);
  int64_t r = (int64_t)blockIdx.x * per + (kBlock ? 0 : threadIdx.x / G);
  const int64_t step = (int64_t)gridDim.x * per;
  Raw next[I] = {};
  const auto load = [&](int64_t row) {
    if (row < a.n) load_row<T, I, kFull, kShort>(next, static_cast<const T*>(a.x) + row * a.x_stride, cols, dim);
  };
  if constexpr (kAhead) load(r);
  for (int64_t base = (int64_t)blockIdx.x * per; base < a.n; base += step, r += step) {
    if constexpr (!kAhead) load(r);
    float x[I * V];
    float s[1] = {0.0f};
#pragma unroll
    for (int i = 0; i < I; ++i)
#pragma unroll
      for (int j = 0; j < V; ++j) {
        x[i * V + j] = element<T>(next[i], j);
        s[0] += own(i, j) ? x[i * V + j] : 0.0f;
      }
    if constexpr (kAhead) load(r + step);
    row_sums<kBlock>(s, G, lds1);
    const float mean = s[0] * inv;
    float q[2] = {0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < I; ++i)
#pragma unroll
      for (int j = 0; j < V; ++j) {
        x[i * V + j] -= mean;
        const float d = own(i, j) ? x[i * V + j] : 0.0f;
        q[0] += d;
        q[1] = __builtin_fmaf(d, d, q[1]);
      }
    row_sums<kBlock>(q, G, lds2);
    // what the rounding of `mean` left over, out of the variance and the differences
    const float off = q[0] * inv;
    const float var = __builtin_fmaf(-off, off, q[1] * inv);
    const float rstd = 1.0f / __builtin_sqrtf((var > 0.0f || var != var ? var : 0.0f) + a.eps);
    if (r < a.n) {
      T* out = static_cast<T*>(a.out) + r * a.out_stride;
#pragma unroll
      for (int i = 0; i < I; ++i) {
        LoosePack<T, V> o;
#pragma unroll
        for (int j = 0; j < V; ++j)
          o.v[j] = rounded<T>(__builtin_fmaf((x[i * V + j] - off) * rstd, w[i * V + j], b[i * V + j]));
        // (elements that are another lane's too get the same value from both, to the last bit)
        if (kFull || kShort || cols.skip[i] < V) store_row<T, V, kShort>(out, cols.at[i], dim, o);
      }
    }
  }
}

// The gradient. After the mean one exchange gives the four sums that the rest
// needs: of d = x - mean, d^2, g and g d. Each thread keeps the sums over rows
// of its own columns in registers; a block joins them at its end, in fp64, and
// leaves its sums in fp32 (rounded once) for k_norm_join.
// Rows shorter than a vector are worked on, summed and left in fp64 throughout:
// of a handful of sums one can come out near zero, and the gradient of a row of
// one element is zero, of two all but zero (9 x 2 fp32 was off by 4e-3 of it, as
// 32 bits are). 1M x 3 fp16 23 us, 25 in fp32; 10M x 7 fp16 311 and 296, 10M x 2 fp32
// 46 and 52.
// (Sums in fp64 at any width: 200,000 x 500 fp16 156 us, 127 in fp32.)
// (whole 16-bit rows a block: four waves a SIMD, 128 registers; forced also
// where that spills, 60,000 x 1021 fp16 took 245 us against 84)
template <class T, int I, int kMost, bool kFull, bool kShort>
__global__ __launch_bounds__(kMost ? kMost : kNormThreads, sizeof(T) == 2 && kMost && kFull ? 4 : 1) void k_layer_norm_grad(NormArgs a) {
  __shared__ float lds1[kNormMaxThreads / 64];
  __shared__ __align__(16) float lds2[4 * kNormMaxThreads / 64];
  extern __shared__ __align__(16) float join[];  // of Sum: [groups of the block, or its waves][G * I * V] (not kBlock)
  constexpr int V = 16 / sizeof(T);
  constexpr bool kBlock = kMost != 0, kAhead = kMost != kNormMaxThreads;
  const int G = a.G, l = kBlock ? threadIdx.x : threadIdx.x & (G - 1), dim = a.dim;
  const int per = kBlock ? 1 : kNormThreads / G;
  const float inv = 1.0f / (float)dim;
  const Columns<T, I, kFull> cols(l, G, dim);
  const auto own = [&](int i, int j) { return cols.own(i, j); };
  using Sum = std::conditional_t<kShort, double, float>;
  float w[I * V];
  Sum dw[I * V], db[I * V];
  load_params<T, I, kFull, kShort>(w, a.weight, a.wide_weight, 1.0f, cols, dim);
#pragma unroll
  for (int e = 0; e < I * V; ++e) dw[e] = db[e] = 0;
  const int sub = kBlock ? 0 : threadIdx.x / G;
  int64_t r = (int64_t)blockIdx.x * per + sub;
  const int64_t step = (int64_t)gridDim.x * per;
  Raw nx[I] = {}, ng[I] = {};
  const auto load = [&](int64_t row) {
    if (row < a.n) {
      load_row<T, I, kFull, kShort>(nx, static_cast<const T*>(a.x) + row * a.x_stride, cols, dim);
      load_row<T, I, kFull, kShort>(ng, static_cast<const T*>(a.grad) + row * a.grad_stride, cols, dim);
    }
  };
  if constexpr (kAhead) load(r);
  for (int64_t base = (int64_t)blockIdx.x * per; base < a.n; base += step, r += step) {
    if constexpr (!kAhead) load(r);
    if constexpr (kShort) {
      // (places from dim on are 0 in x and grad)
      double x[V - 1], g[V - 1], s = 0.0, q = 0.0, g_sum = 0.0, gd = 0.0;
#pragma unroll
      for (int j = 0; j < V - 1; ++j) {
        x[j] = element<T>(nx[0], j);
        g[j] = element<T>(ng[0], j);
        s += x[j];
      }
      load(r + step);
      // (s / dim to the last bit: a row of equal elements is its mean)
      const double over = 1.0 / dim, near = s * over, mean = __builtin_fma(__builtin_fma(-near, (double)dim, s), over, near);
#pragma unroll
      for (int j = 0; j < V - 1; ++j) {
        x[j] = j < dim ? x[j] - mean : 0.0;
        q = __builtin_fma(x[j], x[j], q);
        g_sum += g[j] * w[j];
        gd = __builtin_fma(g[j] * w[j], x[j], gd);
      }
      // 1 / sqrt: the unit's estimate and two of Newton's steps (10M x 2 fp32 46 us; divided by a root 64)
      const double v = __builtin_fma(q, over, (double)a.eps);
      double rstd = __builtin_amdgcn_rsq(v);
#pragma unroll
      for (int e = 0; e < 2; ++e) rstd = __builtin_fma(0.5 * rstd, __builtin_fma(-v * rstd, rstd, 1.0), rstd);
      const double g_mean = g_sum * over, gh_mean = gd * over * rstd;
      if (r < a.n) {
        LoosePack<T, V> o;
#pragma unroll
        for (int j = 0; j < V - 1; ++j) {
          const double h = x[j] * rstd;
          o.v[j] = (T)(float)(rstd * (g[j] * w[j] - g_mean - h * gh_mean));
          dw[j] = __builtin_fma(g[j], h, dw[j]);
          db[j] += g[j];
        }
        if (a.out != nullptr) store_row<T, V, true>(static_cast<T*>(a.out) + r * a.out_stride, 0, dim, o);
      }
      continue;
    }
    float x[I * V];
    Raw gr[I];
    float s[1] = {0.0f};
#pragma unroll
    for (int i = 0; i < I; ++i) {
      gr[i] = ng[i];
#pragma unroll
      for (int j = 0; j < V; ++j) {
        x[i * V + j] = element<T>(nx[i], j);
        s[0] += own(i, j) ? x[i * V + j] : 0.0f;
      }
    }
    if constexpr (kAhead) load(r + step);
    row_sums<kBlock>(s, G, lds1);
    const float mean = s[0] * inv;
    float q[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < I; ++i)
#pragma unroll
      for (int j = 0; j < V; ++j) {
        x[i * V + j] -= mean;
        const float d = own(i, j) ? x[i * V + j] : 0.0f;
        const float gw = own(i, j) ? element<T>(gr[i], j) * w[i * V + j] : 0.0f;
        q[0] += d;
        q[1] = __builtin_fmaf(d, d, q[1]);
        q[2] += gw;
        q[3] = __builtin_fmaf(gw, d, q[3]);
      }
    row_sums<kBlock>(q, G, lds2);
    const float off = q[0] * inv;
    const float var = __builtin_fmaf(-off, off, q[1] * inv);
    const float rstd = 1.0f / __builtin_sqrtf((var > 0.0f || var != var ? var : 0.0f) + a.eps);
    const float g_mean = q[2] * inv;
    const float gh_mean = __builtin_fmaf(-off, q[2], q[3]) * inv * rstd;
    if (r < a.n) {
#pragma unroll
      for (int i = 0; i < I; ++i) {
        LoosePack<T, V> o;
#pragma unroll
        for (int j = 0; j < V; ++j) {
          const float h = (x[i * V + j] - off) * rstd, dy = element<T>(gr[i], j);
          o.v[j] = rounded<T>(rstd * (__builtin_fmaf(dy, w[i * V + j], -g_mean) - h * gh_mean));
          dw[i * V + j] = __builtin_fmaf(dy, h, dw[i * V + j]);
          db[i * V + j] += dy;
        }
        if (a.out != nullptr && (kFull || cols.skip[i] < V))
          store_row<T, V, false>(static_cast<T*>(a.out) + r * a.out_stride, cols.at[i], dim, o);
      }
    }
  }
  if (a.sums == nullptr) return;
  Sum* mine = static_cast<Sum*>(a.sums) + (int64_t)blockIdx.x * 2 * dim;
  if constexpr (kBlock) {
#pragma unroll
    for (int i = 0; i < I; ++i)
#pragma unroll
      for (int j = 0; j < V; ++j)
        if (own(i, j)) {
          mine[cols.at[i] + j] = dw[i * V + j];
          mine[dim + cols.at[i] + j] = db[i * V + j];
        }
  } else {
    // by nominal column: vector i of lane l begins at (i G + l) V, its own elements end it
    const int width = G * I * V, parts = kShort ? kNormThreads / 64 : per;
#pragma unroll
    for (int which = 0; which < 2; ++which) {
      __syncthreads();
      if constexpr (kShort) {
        // (a lane a row: 64 for a few columns, joined by exchanges)
#pragma unroll
        for (int e = 0; e < V; ++e) {
          double t = which ? db[e] : dw[e];
          for (int o = 1; o < 64; o *= 2) t += __shfl_xor(t, o);
          if ((threadIdx.x & 63) == 0) reinterpret_cast<double*>(join)[threadIdx.x / 64 * V + e] = t;
        }
      } else {
#pragma unroll
        for (int i = 0; i < I; ++i) {
          const Sum* t = (which ? db : dw) + i * V;
#pragma unroll
          for (int e = 0; e < V; e += 4)
            *reinterpret_cast<float4*>(join + sub * width + (i * G + l) * V + e) =
                make_float4(t[e], t[e + 1], t[e + 2], t[e + 3]);
        }
      }
      __syncthreads();
      for (int c = threadIdx.x; c < dim; c += kNormThreads) {
        // column c's place: in the last vector of the row the elements are at its end
        const int first = c / V * V, at = kFull || kShort || first + V <= dim ? c : c + V - (dim - first);
        const auto* sums = reinterpret_cast<const Sum*>(join);
        double t = 0.0;
        for (int k = 0; k < parts; k += 4) {  // (a power of two from 4 on)
          const Sum* at4 = sums + k * width + at;
          t += ((double)at4[0] + (double)at4[width]) + ((double)at4[2 * width] + (double)at4[3 * width]);
        }
        mine[which * dim + c] = (Sum)t;
      }
    }
  }
}

// The blocks' sums to weight_grad and bias_grad, fp64 from here on: 16 columns
// (of both arrays) a block, a column's sums taken by 64 threads in turn: bound by
// the latency of their loads, 4 us for 625 blocks' sums of 1021 columns.
constexpr int kJoinCols = 16, kJoinSlices = 64;
template <class T, class Sum>
__global__ __launch_bounds__(kJoinCols * kJoinSlices) void k_norm_join(const Sum* sums, int blocks, int dim, void* dw,
                                                                       void* db, bool wide) {
  __shared__ double part[kJoinSlices][kJoinCols];
  const int col = threadIdx.x % kJoinCols, slice = threadIdx.x / kJoinCols;
  const int c = blockIdx.x * kJoinCols + col;
  double t = 0.0;
  if (c < 2 * dim) {
#pragma unroll 8
    for (int b = slice; b < blocks; b += kJoinSlices) t += (double)sums[(int64_t)b * 2 * dim + c];
  }
  part[slice][col] = t;
  __syncthreads();
  if (slice >= 4) return;
  t = 0.0;
  for (int k = slice; k < kJoinSlices; k += 4) t += part[k][col];
  t += __shfl_xor(t, kJoinCols);
  t += __shfl_xor(t, 2 * kJoinCols);
  void* to = c < dim ? dw : db;
  if (slice != 0 || c >= 2 * dim || to == nullptr) return;
  const int at = c < dim ? c : c - dim;
  if (wide) static_cast<float*>(to)[at] = (float)t;
  else static_cast<T*>(to)[at] = (T)(float)t;
}

// How a row lies on lanes: one vector a lane where that leaves the row within
// a wave, else 16 elements (one vector also for blocks of up to 512: the gradient
// of 16,384 x 4096 bf16 104 us against 99, rows of 8192 slower still).
struct NormPlan {
  int I, G;
  bool block;  // a block a row
  bool full;   // the lanes' vectors are the row, no more
};

// Blocks that the device holds at a time, and no call has more: a block takes
// its rows in turn, and its columns of weight and bias once. (Each block of a
// gradient also leaves 2 * dim sums.)
constexpr int kUnits = 256;
int blocks_max(const NormPlan& p, bool grad) {
  // waves a unit by the kernels' registers
  const int threads = p.block ? p.G : kNormThreads;
  const int waves = p.I == 1 ? (grad ? 20 : 32)
                    : threads > kNormMidThreads || (grad && p.I == 2 && p.full && p.block) ? 16 : grad ? 12 : 20;
  return kUnits * std::max(1, waves / (threads / 64));
}

// The rows in equal shares: the blocks of as many rounds as the most blocks
// need. A gradient's blocks take at least kGradRows rows where that leaves a
// block for each unit: a block's sums are written and read, 16 bytes a column
// against 6 or 12 a row and column (2000 x 5120 bf16 34 us with 8, 45 with 2, 39
// with 4, 34 with 16).
constexpr int kGradRows = 8;
int norm_blocks(const NormPlan& p, int64_t n, bool grad) {
  const int64_t per = p.block ? 1 : kNormThreads / p.G, groups = (n + per - 1) / per;
  int64_t most = blocks_max(p, grad);
  if (grad) most = std::min(most, std::max<int64_t>(kUnits, n / kGradRows));
  const int64_t rounds = (groups + most - 1) / most;
  return (int)((groups + rounds - 1) / rounds);
}

NormPlan norm_plan(int dim, int size) {
  NormPlan p;
  const int V = 16 / size, nvec = (dim + V - 1) / V;
  for (int i : {1, 16 / V}) {
    p.I = i;
    p.G = 1;
    while (p.G * i < nvec) p.G *= 2;
    p.block = p.G > 64;
    if (!p.block) break;
  }
  if (p.block) p.G = (nvec + p.I * 64 - 1) / (p.I * 64) * 64;
  p.full = dim == p.G * p.I * V;
  return p;
}

template <class T, bool kGrad>
hipError_t launch_norm(const NormPlan& p, const NormArgs& a, int blocks, hipStream_t st) {
  constexpr int V = 16 / sizeof(T), kMany = sizeof(T);  // vectors of 16 elements
  const size_t lds = kGrad && !p.block && a.sums != nullptr ? sizeof(float) * kNormThreads * p.I * V : 0;
  const dim3 grid(blocks), block(p.block ? p.G : kNormThreads);
  const auto go = [&](auto i, auto most, auto full, auto shrt) {
    constexpr int I = decltype(i)::value, kMost = decltype(most)::value;
    constexpr bool kFull = decltype(full)::value, kShort = decltype(shrt)::value;
    if constexpr (kGrad) hipLaunchKernelGGL((k_layer_norm_grad<T, I, kMost, kFull, kShort>), grid, block, lds, st, a);
    else hipLaunchKernelGGL((k_layer_norm<T, I, kMost, kFull, kShort>), grid, block, lds, st, a);
  };
  using std::integral_constant;
  using Yes = std::true_type;
  using No = std::false_type;
  const auto sized = [&](auto full) {
    if (p.I == 1) go(integral_constant<int, 1>{}, integral_constant<int, 0>{}, full, No{});
    else if (!p.block) go(integral_constant<int, kMany>{}, integral_constant<int, 0>{}, full, No{});
    else if (p.G <= kNormMidThreads)
      go(integral_constant<int, kMany>{}, integral_constant<int, kNormMidThreads>{}, full, No{});
    else go(integral_constant<int, kMany>{}, integral_constant<int, kNormMaxThreads>{}, full, No{});
  };
  if (a.dim < V) go(integral_constant<int, 1>{}, integral_constant<int, 0>{}, No{}, Yes{});
  else if (p.full) sized(Yes{});
  else sized(No{});
  return hipGetLastError();
}

int check_norm(const void* x, int64_t x_stride, int64_t n, int32_t dim, float eps, int dtype, int weight_dtype) {
  if (n < 0 || n > 0x7FFFFFFFll) return op_error(MLKV_EINVAL, "n must be in [0, 2^31 - 1]");
  if (dim < 1 || dim > MLKV_NORM_MAX_DIM) return op_error(MLKV_EINVAL, "dim must be in [1, 16384]");
  if (!(eps >= 0.0f) || std::isinf(eps)) return op_error(MLKV_EINVAL, "eps must be finite and >= 0");
  if (dtype_size(dtype) == 0) return op_error(MLKV_EINVAL, "unknown dtype");
  if (weight_dtype != MLKV_F32 && weight_dtype != dtype)
    return op_error(MLKV_EINVAL, "weight_dtype must be MLKV_F32 or dtype");
  if (n > 0 && x == nullptr) return op_error(MLKV_EINVAL, "x is NULL");
  if (!stride_ok(x_stride, n, dim, true)) return op_error(MLKV_EINVAL, "x_stride must be 0 or >= dim");
  return MLKV_OK;
}

}  // namespace
}  // namespace mlkv

using namespace mlkv;

extern "C" {

int mlkv_layer_norm(const void* d_x, int64_t x_stride, const void* d_weight, const void* d_bias, int64_t n,
                    int32_t dim, float eps, int dtype, int weight_dtype, void* d_out, int64_t out_stride,
                    void* hip_stream) {
  const int rc = check_norm(d_x, x_stride, n, dim, eps, dtype, weight_dtype);
  if (rc) return rc;
  if (n == 0) return MLKV_OK;
  if (d_out == nullptr) return op_error(MLKV_EINVAL, "out is NULL");
  if (!stride_ok(out_stride, n, dim, false)) return op_error(MLKV_EINVAL, "out_stride must be >= dim");
  const int size = dtype_size(dtype), wsize = dtype_size(weight_dtype);
  if (!all_aligned(size, {d_x, d_out}) || !all_aligned(wsize, {d_weight, d_bias}))
    return op_error(MLKV_EINVAL, "a pointer is not aligned to its element type");
  if (d_out == d_x && n > 1 && x_stride != out_stride)
    return op_error(MLKV_EINVAL, "out may be x only with the same stride");
  const RowSpan x = row_span(d_x, x_stride, n, dim, size), out = row_span(d_out, out_stride, n, dim, size);
  const int64_t params = (int64_t)dim * wsize;
  if (!out_ok(x, out) || rows_meet({d_weight, 0, 1, params}, out) || rows_meet({d_bias, 0, 1, params}, out))
    return op_error(MLKV_EINVAL, "out overlaps x, weight or bias");
  const NormPlan p = norm_plan(dim, size);
  NormArgs a{};
  a.x = d_x;
  a.weight = d_weight;
  a.bias = d_bias;
  a.out = d_out;
  a.x_stride = x_stride;
  a.out_stride = out_stride;
  a.n = n;
  a.dim = dim;
  a.G = p.G;
  a.eps = eps;
  a.wide_weight = weight_dtype == MLKV_F32;
  const int blocks = norm_blocks(p, n, false);
  const hipError_t e = dispatch_type(dtype, [&](auto t) {
    return launch_norm<decltype(t), false>(p, a, blocks, static_cast<hipStream_t>(hip_stream));
  });
  return e == hipSuccess ? MLKV_OK : op_launch_error(e, "mlkv_layer_norm launch");
}

int64_t mlkv_layer_norm_grad_workspace(int64_t n, int32_t dim) {
  if (n < 0 || n > 0x7FFFFFFFll) return op_error(MLKV_EINVAL, "n must be in [0, 2^31 - 1]");
  if (dim < 1 || dim > MLKV_NORM_MAX_DIM) return op_error(MLKV_EINVAL, "dim must be in [1, 16384]");
  if (n == 0) return 0;
  // (the type is not known here: the most blocks of any)
  int64_t blocks = 0;
  for (int size : {2, 4}) blocks = std::max<int64_t>(blocks, norm_blocks(norm_plan(dim, size), n, true));
  return (int64_t)(dim < 16 / 2 ? sizeof(double) : sizeof(float)) * 2 * dim * blocks;
}

int mlkv_layer_norm_grad(const void* d_x, int64_t x_stride, const void* d_weight, const void* d_grad,
                         int64_t grad_stride, int64_t n, int32_t dim, float eps, int dtype, int weight_dtype,
                         void* d_x_grad, int64_t x_grad_stride, void* d_weight_grad, void* d_bias_grad, void* d_work,
                         int64_t work_bytes, void* hip_stream) {
  const int rc = check_norm(d_x, x_stride, n, dim, eps, dtype, weight_dtype);
  if (rc) return rc;
  const int size = dtype_size(dtype), wsize = dtype_size(weight_dtype);
  const bool sums = d_weight_grad != nullptr || d_bias_grad != nullptr;
  if (n > 0 && d_grad == nullptr) return op_error(MLKV_EINVAL, "grad is NULL");
  if (!stride_ok(grad_stride, n, dim, true)) return op_error(MLKV_EINVAL, "grad_stride must be 0 or >= dim");
  if (d_x_grad != nullptr && !stride_ok(x_grad_stride, n, dim, false))
    return op_error(MLKV_EINVAL, "x_grad_stride must be >= dim");
  if (!all_aligned(size, {d_x, d_grad, d_x_grad}) ||
      !all_aligned(wsize, {d_weight, d_weight_grad, d_bias_grad}))
    return op_error(MLKV_EINVAL, "a pointer is not aligned to its element type");
  if (n > 1 && d_x_grad != nullptr &&
      ((d_x_grad == d_x && x_grad_stride != x_stride) || (d_x_grad == d_grad && x_grad_stride != grad_stride)))
    return op_error(MLKV_EINVAL, "x_grad may be x or grad only with the same stride");
  const RowSpan x = row_span(d_x, x_stride, n, dim, size), grad = row_span(d_grad, grad_stride, n, dim, size),
                x_grad = row_span(d_x_grad, x_grad_stride, n, dim, size);
  if (!out_ok(x, x_grad) || !out_ok(grad, x_grad) || rows_meet({d_weight, 0, 1, (int64_t)dim * wsize}, x_grad))
    return op_error(MLKV_EINVAL, "x_grad overlaps x, grad or weight");
  if (sums && n > 0) {
    if (d_work == nullptr || work_bytes < mlkv_layer_norm_grad_workspace(n, dim))
      return op_error(MLKV_EINVAL, "work is smaller than mlkv_layer_norm_grad_workspace");
    if (!all_aligned(16, {d_work})) return op_error(MLKV_EINVAL, "work must be at a multiple of 16 bytes");
  }
  if (!sums && (n == 0 || d_x_grad == nullptr)) return MLKV_OK;
  const hipStream_t st = static_cast<hipStream_t>(hip_stream);
  int blocks = 0;
  if (n > 0) {
    const NormPlan p = norm_plan(dim, size);
    NormArgs a{};
    a.x = d_x;
    a.grad = d_grad;
    a.weight = d_weight;
    a.out = d_x_grad;
    a.sums = sums ? d_work : nullptr;
    a.x_stride = x_stride;
    a.grad_stride = grad_stride;
    a.out_stride = x_grad_stride;
    a.n = n;
    a.dim = dim;
    a.G = p.G;
    a.eps = eps;
    a.wide_weight = weight_dtype == MLKV_F32;
    blocks = norm_blocks(p, n, true);
    const hipError_t e =
        dispatch_type(dtype, [&](auto t) { return launch_norm<decltype(t), true>(p, a, blocks, st); });
    if (e != hipSuccess) return op_launch_error(e, "mlkv_layer_norm_grad launch");
  }
  if (!sums) return MLKV_OK;
  const hipError_t e = dispatch_type(dtype, [&](auto t) {
    const auto join = [&](auto of) {
      using Sum = decltype(of);
      hipLaunchKernelGGL((k_norm_join<decltype(t), Sum>), dim3((2 * dim + kJoinCols - 1) / kJoinCols),
                         dim3(kJoinCols * kJoinSlices), 0, st, static_cast<const Sum*>(d_work), blocks, dim,
                         d_weight_grad, d_bias_grad, weight_dtype == MLKV_F32);
    };
    if (dim < 16 / size) join(double{});
    else join(float{});
    return hipGetLastError();
  });
  return e == hipSuccess ? MLKV_OK : op_launch_error(e, "mlkv_layer_norm_grad launch");
}

}  // extern "C"
