// Layer norm and its gradient.
//
// A row belongs to a group of G lanes that holds it whole in registers, I
// vectors of V elements a lane, so each element is read once and both passes
// of the variance (mean, then squares about it) run on registers. Rows of up
// to 1024 elements have a group within a wave, several groups a block; longer
// ones have a block of waves each that exchange their sums through LDS. Both
// kernels are bound by HBM: 8 and 16 operations an element against 4 to 12 bytes.
#include "mlkv_ops.h"

#include <algorithm>
#include <cmath>

namespace mlkv {
namespace {

constexpr int kNormThreads = 256;      // of a block of groups within waves
constexpr int kNormMaxThreads = 1024;  // of a block that holds one row

// Most blocks of a gradient call that sums over rows: each leaves 2 * dim floats of sums.
constexpr int kGradBlocksNarrow = 2048;
constexpr int kGradBlocksWide = 512;
inline int grad_blocks_max(int32_t dim) { return dim <= 1024 ? kGradBlocksNarrow : kGradBlocksWide; }

struct NormArgs {
  const void* x;
  const void* grad;    // gradient only
  const void* weight;  // or NULL
  const void* bias;    // or NULL
  void* out;           // or NULL (gradient)
  float* sums;         // gradient: [blocks][2][dim], or NULL
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
  const int waves = blockDim.x >> 6, wave = threadIdx.x >> 6;
#pragma unroll
  for (int k = 0; k < N; ++k) {
    v[k] = group_sum(v[k], 64);
    if ((threadIdx.x & 63) == 0) lds[wave * N + k] = v[k];
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < N; ++k) v[k] = 0.0f;
  for (int w = 0; w < waves; ++w)
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] += lds[w * N + k];
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

template <class T, int V, int I>
struct Row {
  Pack<T, V> p[I];
  // Loads the lane's vectors; zeros where it has none.
  __device__ __forceinline__ void load(const T* row, int l, int G, int nvec, bool live) {
#pragma unroll
    for (int i = 0; i < I; ++i) {
      const int v = i * G + l;
      if (live && v < nvec) {
        p[i] = *reinterpret_cast<const Pack<T, V>*>(row + (int64_t)v * V);
      } else {
#pragma unroll
        for (int j = 0; j < V; ++j) p[i].v[j] = (T)0.0f;
      }
    }
  }
};

template <class T>
__device__ __forceinline__ float param(const void* p, bool wide, int c) {
  return wide ? static_cast<const float*>(p)[c] : (float)static_cast<const T*>(p)[c];
}

// One thread's columns of weight or bias.
template <class T, int V, int I>
__device__ __forceinline__ void load_params(float (&w)[I * V], const void* p, bool wide, float none, int l, int G,
                                            int nvec) {
#pragma unroll
  for (int i = 0; i < I; ++i)
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const int v = i * G + l;
      w[i * V + j] = p != nullptr && v < nvec ? param<T>(p, wide, v * V + j) : none;
    }
}

template <class T, int V, int I, bool kBlock>
__global__ __launch_bounds__(kBlock ? kNormMaxThreads : kNormThreads) void k_layer_norm(NormArgs a) {
  __shared__ float lds1[kNormMaxThreads / 64];
  __shared__ float lds2[2 * kNormMaxThreads / 64];
  const int G = a.G, l = kBlock ? threadIdx.x : threadIdx.x & (G - 1);
  const int per = kBlock ? 1 : kNormThreads / G;
  const int nvec = a.dim / V;
  const float inv = 1.0f / (float)a.dim;
  float w[I * V], b[I * V];
  load_params<T, V, I>(w, a.weight, a.wide_weight, 1.0f, l, G, nvec);
  load_params<T, V, I>(b, a.bias, a.wide_weight, 0.0f, l, G, nvec);
  const int sub = kBlock ? 0 : threadIdx.x / G;
  Row<T, V, I> next;
  int64_t r = (int64_t)blockIdx.x * per + sub;
  const int64_t step = (int64_t)gridDim.x * per;
  next.load(static_cast<const T*>(a.x) + r * a.x_stride, l, G, nvec, r < a.n);
  for (int64_t base = (int64_t)blockIdx.x * per; base < a.n; base += step, r += step) {
    const Row<T, V, I> cur = next;
    next.load(static_cast<const T*>(a.x) + (r + step) * a.x_stride, l, G, nvec, r + step < a.n);
    float s[1] = {0.0f};
#pragma unroll
    for (int i = 0; i < I; ++i)
#pragma unroll
      for (int j = 0; j < V; ++j) s[0] += (float)cur.p[i].v[j];
    row_sums<kBlock>(s, G, lds1);
    const float mean = s[0] * inv;
    float q[2] = {0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < I; ++i)
      if (i * G + l < nvec) {
#pragma unroll
        for (int j = 0; j < V; ++j) {
          const float d = (float)cur.p[i].v[j] - mean;
          q[0] += d;
          q[1] = __builtin_fmaf(d, d, q[1]);
        }
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
        const int v = i * G + l;
        if (v < nvec) {
          Pack<T, V> o;
#pragma unroll
          for (int j = 0; j < V; ++j) {
            const float h = (((float)cur.p[i].v[j] - mean) - off) * rstd;
            o.v[j] = (T)__builtin_fmaf(h, w[i * V + j], b[i * V + j]);
          }
          *reinterpret_cast<Pack<T, V>*>(out + (int64_t)v * V) = o;
        }
      }
    }
  }
}

// The gradient. After the mean one exchange gives the four sums that the rest
// needs: of d = x - mean, d^2, g and g d. Each thread keeps the sums over rows
// of its own columns in registers; a block joins them at its end.
template <class T, int V, int I, bool kBlock>
__global__ __launch_bounds__(kBlock ? kNormMaxThreads : kNormThreads) void k_layer_norm_grad(NormArgs a) {
  __shared__ float lds1[kNormMaxThreads / 64];
  __shared__ float lds2[4 * kNormMaxThreads / 64];
  extern __shared__ float join[];  // [groups of the block][G * I * V] (not kBlock)
  const int G = a.G, l = kBlock ? threadIdx.x : threadIdx.x & (G - 1);
  const int per = kBlock ? 1 : kNormThreads / G;
  const int nvec = a.dim / V;
  const float inv = 1.0f / (float)a.dim;
  float w[I * V], dw[I * V], db[I * V];
  load_params<T, V, I>(w, a.weight, a.wide_weight, 1.0f, l, G, nvec);
#pragma unroll
  for (int e = 0; e < I * V; ++e) dw[e] = db[e] = 0.0f;
  const int sub = kBlock ? 0 : threadIdx.x / G;
  Row<T, V, I> nx, ng;
  int64_t r = (int64_t)blockIdx.x * per + sub;
  const int64_t step = (int64_t)gridDim.x * per;
  nx.load(static_cast<const T*>(a.x) + r * a.x_stride, l, G, nvec, r < a.n);
  ng.load(static_cast<const T*>(a.grad) + r * a.grad_stride, l, G, nvec, r < a.n);
  for (int64_t base = (int64_t)blockIdx.x * per; base < a.n; base += step, r += step) {
    const Row<T, V, I> x = nx, g = ng;
    const bool more = r + step < a.n;
    nx.load(static_cast<const T*>(a.x) + (r + step) * a.x_stride, l, G, nvec, more);
    ng.load(static_cast<const T*>(a.grad) + (r + step) * a.grad_stride, l, G, nvec, more);
    float s[1] = {0.0f};
#pragma unroll
    for (int i = 0; i < I; ++i)
#pragma unroll
      for (int j = 0; j < V; ++j) s[0] += (float)x.p[i].v[j];
    row_sums<kBlock>(s, G, lds1);
    const float mean = s[0] * inv;
    float q[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < I; ++i)
      if (i * G + l < nvec) {
#pragma unroll
        for (int j = 0; j < V; ++j) {
          const float d = (float)x.p[i].v[j] - mean, gw = (float)g.p[i].v[j] * w[i * V + j];
          q[0] += d;
          q[1] = __builtin_fmaf(d, d, q[1]);
          q[2] += gw;
          q[3] = __builtin_fmaf(gw, d, q[3]);
        }
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
        const int v = i * G + l;
        if (v < nvec) {
          Pack<T, V> o;
#pragma unroll
          for (int j = 0; j < V; ++j) {
            const float h = (((float)x.p[i].v[j] - mean) - off) * rstd, dy = (float)g.p[i].v[j];
            o.v[j] = (T)(rstd * (__builtin_fmaf(dy, w[i * V + j], -g_mean) - h * gh_mean));
            dw[i * V + j] = __builtin_fmaf(dy, h, dw[i * V + j]);
            db[i * V + j] += dy;
          }
          if (a.out != nullptr)
            *reinterpret_cast<Pack<T, V>*>(static_cast<T*>(a.out) + r * a.out_stride + (int64_t)v * V) = o;
        }
      }
    }
  }
  if (a.sums == nullptr) return;
  float* mine = a.sums + (int64_t)blockIdx.x * 2 * a.dim;
  if constexpr (kBlock) {
#pragma unroll
    for (int i = 0; i < I; ++i)
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const int c = (i * G + l) * V + j;
        if (c < a.dim) {
          mine[c] = dw[i * V + j];
          mine[a.dim + c] = db[i * V + j];
        }
      }
  } else {
    const int width = G * I * V;
#pragma unroll
    for (int which = 0; which < 2; ++which) {
      __syncthreads();
#pragma unroll
      for (int i = 0; i < I; ++i)
#pragma unroll
        for (int j = 0; j < V; ++j) join[sub * width + (i * G + l) * V + j] = which ? db[i * V + j] : dw[i * V + j];
      __syncthreads();
      for (int c = threadIdx.x; c < a.dim; c += kNormThreads) {
        float t = 0.0f;
        for (int k = 0; k < per; ++k) t += join[k * width + c];
        mine[which * a.dim + c] = t;
      }
    }
  }
}

// The blocks' sums to weight_grad and bias_grad: 64 columns a block, its waves
// take every 16th block's sums, fp64 from here on.
constexpr int kJoinSlices = 16;
template <class T>
__global__ __launch_bounds__(64 * kJoinSlices) void k_norm_join(const float* sums, int blocks, int dim, void* dw,
                                                                void* db, bool wide) {
  __shared__ double part[kJoinSlices][64];
  const int lane = threadIdx.x & 63, slice = threadIdx.x >> 6;
  const int c = blockIdx.x * 64 + lane;  // over both arrays
  double t = 0.0;
  if (c < 2 * dim) {
#pragma unroll 4
    for (int b = slice; b < blocks; b += kJoinSlices) t += (double)sums[(int64_t)b * 2 * dim + c];
  }
  part[slice][lane] = t;
  __syncthreads();
  if (slice != 0 || c >= 2 * dim) return;
  for (int k = 1; k < kJoinSlices; ++k) t += part[k][lane];
  void* to = c < dim ? dw : db;
  if (to == nullptr) return;
  const int at = c < dim ? c : c - dim;
  if (wide) static_cast<float*>(to)[at] = (float)t;
  else static_cast<T*>(to)[at] = (T)(float)t;
}

// How a row lies on lanes. Vectors are as wide as widths, strides and
// addresses allow, at most 16 bytes; a lane takes the smaller number of them
// that leaves the row within a wave, else 16 elements.
struct NormPlan {
  int V, I, G;
  bool block;
};

NormPlan norm_plan(int dim, int size, std::initializer_list<const void*> ptrs, std::initializer_list<int64_t> strides) {
  NormPlan p;
  p.V = 16 / size;
  while (p.V > 1 && (dim % p.V != 0 || !all_aligned((size_t)p.V * size, size, ptrs, strides))) p.V = p.V > 2 ? 2 : 1;
  const int few = p.V == 8 ? 1 : p.V == 4 ? 1 : p.V == 2 ? 2 : 4, many = 16 / p.V;
  const int nvec = dim / p.V;
  p.block = false;
  for (int i : {few, many}) {
    p.I = i;
    p.G = 1;
    while (p.G * i < nvec) p.G *= 2;
    if (p.G <= 64) return p;
  }
  p.block = true;
  p.G = (nvec + p.I * 64 - 1) / (p.I * 64) * 64;
  return p;
}

template <class T, bool kGrad, int V, int I>
hipError_t launch_norm(const NormPlan& p, const NormArgs& a, int blocks, hipStream_t st) {
  const size_t lds = kGrad && !p.block && a.sums != nullptr ? sizeof(float) * kNormThreads * I * V : 0;
  if constexpr (kGrad) {
    if (p.block) hipLaunchKernelGGL((k_layer_norm_grad<T, V, I, true>), dim3(blocks), dim3(p.G), lds, st, a);
    else hipLaunchKernelGGL((k_layer_norm_grad<T, V, I, false>), dim3(blocks), dim3(kNormThreads), lds, st, a);
  } else {
    if (p.block) hipLaunchKernelGGL((k_layer_norm<T, V, I, true>), dim3(blocks), dim3(p.G), 0, st, a);
    else hipLaunchKernelGGL((k_layer_norm<T, V, I, false>), dim3(blocks), dim3(kNormThreads), 0, st, a);
  }
  return hipGetLastError();
}

template <class T, bool kGrad>
hipError_t dispatch_norm(const NormPlan& p, const NormArgs& a, int blocks, hipStream_t st) {
  constexpr int kFull = 16 / sizeof(T);
  const bool many = p.I * p.V == 16;
  if (p.V == kFull) {
    return many ? launch_norm<T, kGrad, kFull, 16 / kFull>(p, a, blocks, st)
                : launch_norm<T, kGrad, kFull, 1>(p, a, blocks, st);
  }
  if (p.V == 2) {
    return many ? launch_norm<T, kGrad, 2, 8>(p, a, blocks, st) : launch_norm<T, kGrad, 2, 2>(p, a, blocks, st);
  }
  return many ? launch_norm<T, kGrad, 1, 16>(p, a, blocks, st) : launch_norm<T, kGrad, 1, 4>(p, a, blocks, st);
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
  if (!all_aligned(size, size, {d_x, d_out}, {}) || !all_aligned(wsize, wsize, {d_weight, d_bias}, {}))
    return op_error(MLKV_EINVAL, "a pointer is not aligned to its element type");
  if (d_out == d_x && n > 1 && x_stride != out_stride)
    return op_error(MLKV_EINVAL, "out may be x only with the same stride");
  const NormPlan p = norm_plan(dim, size, {d_x, d_out}, {x_stride, out_stride});
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
  const int64_t per = p.block ? 1 : kNormThreads / p.G;
  const int blocks = (int)std::min<int64_t>((n + per - 1) / per, 2048);
  const hipError_t e = dispatch_type(dtype, [&](auto t) {
    return dispatch_norm<decltype(t), false>(p, a, blocks, static_cast<hipStream_t>(hip_stream));
  });
  return e == hipSuccess ? MLKV_OK : op_launch_error(e, "mlkv_layer_norm launch");
}

int64_t mlkv_layer_norm_grad_workspace(int64_t n, int32_t dim) {
  if (n < 0 || n > 0x7FFFFFFFll) return op_error(MLKV_EINVAL, "n must be in [0, 2^31 - 1]");
  if (dim < 1 || dim > MLKV_NORM_MAX_DIM) return op_error(MLKV_EINVAL, "dim must be in [1, 16384]");
  return (int64_t)sizeof(float) * 2 * dim * std::min<int64_t>(n, grad_blocks_max(dim));
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
  if (!all_aligned(size, size, {d_x, d_grad, d_x_grad}, {}) ||
      !all_aligned(wsize, wsize, {d_weight, d_weight_grad, d_bias_grad}, {}))
    return op_error(MLKV_EINVAL, "a pointer is not aligned to its element type");
  if (n > 1 && d_x_grad != nullptr &&
      ((d_x_grad == d_x && x_grad_stride != x_stride) || (d_x_grad == d_grad && x_grad_stride != grad_stride)))
    return op_error(MLKV_EINVAL, "x_grad may be x or grad only with the same stride");
  if (sums && n > 0) {
    if (d_work == nullptr || work_bytes < mlkv_layer_norm_grad_workspace(n, dim))
      return op_error(MLKV_EINVAL, "work is smaller than mlkv_layer_norm_grad_workspace");
    if (!all_aligned(16, 1, {d_work}, {})) return op_error(MLKV_EINVAL, "work must be at a multiple of 16 bytes");
  }
  if (!sums && (n == 0 || d_x_grad == nullptr)) return MLKV_OK;
  const hipStream_t st = static_cast<hipStream_t>(hip_stream);
  int blocks = 0;
  if (n > 0) {
    const NormPlan p = norm_plan(dim, size, {d_x, d_grad, d_x_grad},
                                 {x_stride, grad_stride, d_x_grad != nullptr ? x_grad_stride : 0});
    NormArgs a{};
    a.x = d_x;
    a.grad = d_grad;
    a.weight = d_weight;
    a.out = d_x_grad;
    a.sums = sums ? static_cast<float*>(d_work) : nullptr;
    a.x_stride = x_stride;
    a.grad_stride = grad_stride;
    a.out_stride = x_grad_stride;
    a.n = n;
    a.dim = dim;
    a.G = p.G;
    a.eps = eps;
    a.wide_weight = weight_dtype == MLKV_F32;
    const int64_t per = p.block ? 1 : kNormThreads / p.G;
    blocks = (int)std::min<int64_t>((n + per - 1) / per, grad_blocks_max(dim));
    const hipError_t e =
        dispatch_type(dtype, [&](auto t) { return dispatch_norm<decltype(t), true>(p, a, blocks, st); });
    if (e != hipSuccess) return op_launch_error(e, "mlkv_layer_norm_grad launch");
  }
  if (!sums) return MLKV_OK;
  const hipError_t e = dispatch_type(dtype, [&](auto t) {
    hipLaunchKernelGGL((k_norm_join<decltype(t)>), dim3((2 * dim + 63) / 64), dim3(64 * kJoinSlices), 0, st,
                       static_cast<const float*>(d_work), blocks, dim, d_weight_grad, d_bias_grad,
                       weight_dtype == MLKV_F32);
    return hipGetLastError();
  });
  return e == hipSuccess ? MLKV_OK : op_launch_error(e, "mlkv_layer_norm_grad launch");
}

}  // extern "C"
