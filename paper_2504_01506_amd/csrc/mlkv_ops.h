// What the dense operators (mlkv_norm.hip, mlkv_logits.hip, mlkv_orth.hip)
// share: element types, vectors of them, sums over lanes, host-side checks.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <initializer_list>
#include <numeric>
#include <type_traits>

#include "mlkv.h"

namespace mlkv {

// Set the calling thread's error text (mlkv_last_error) and return the code.
int op_error(int code, const char* msg) noexcept;
int op_launch_error(hipError_t e, const char* what) noexcept;

using bf16 = __bf16;
using f16 = _Float16;

inline int dtype_size(int dtype) {
  return dtype == MLKV_F32 ? 4 : dtype == MLKV_BF16 || dtype == MLKV_F16 ? 2 : 0;
}

// Calls f(T{}) with T the C++ type of dtype, which has been checked.
template <class F>
auto dispatch_type(int dtype, F f) {
  if (dtype == MLKV_F32) return f(float{});
  if (dtype == MLKV_BF16) return f(bf16{});
  return f(f16{});
}

// Whether all of `ptrs` are multiples of `bytes`.
inline bool all_aligned(size_t bytes, std::initializer_list<const void*> ptrs) {
  uintptr_t x = 0;
  for (const void* p : ptrs) x |= reinterpret_cast<uintptr_t>(p);
  return x % bytes == 0;
}

// Whether `rows` rows of `width` elements `stride` apart are something an
// input (same: stride 0 allowed) or an output can be: no rows that overlap,
// and offsets in bytes within 63 bits.
inline bool stride_ok(int64_t stride, int64_t rows, int64_t width, bool same) {
  if (rows <= 1) return true;
  if (same && stride == 0) return true;
  return stride >= width && stride <= (int64_t(1) << 60) / rows;
}

// `rows` rows of `width` bytes, `stride` bytes apart.
struct RowSpan {
  const void* p;
  int64_t stride, rows, width;
};

// ... of elements of `size` bytes, as stride_ok has passed them (one row's stride may be anything).
inline RowSpan row_span(const void* p, int64_t stride, int64_t rows, int64_t width, int size) {
  return {p, rows > 1 ? stride * size : 0, rows, width * size};
}

// Whether a byte of a's rows is one of b's; b's rows do not overlap each other.
// Exact, so that rows side by side in one buffer are told apart: at once where
// the strides are equal or leave the rows apart in every common period, else
// row by row of a (up to the first that meets b's).
inline bool rows_meet(RowSpan a, RowSpan b) {
  using Wide = __int128;  // (addresses and their differences)
  if (a.p == nullptr || b.p == nullptr || a.rows <= 0 || b.rows <= 0) return false;
  if (a.stride == 0 || a.rows == 1) a.rows = 1, a.stride = 0;
  if (b.rows == 1) b.stride = 0;
  const Wide at = (Wide)reinterpret_cast<uintptr_t>(b.p) - (Wide)reinterpret_cast<uintptr_t>(a.p);  // b from a
  if (at >= (Wide)(a.rows - 1) * a.stride + a.width || -at >= (Wide)(b.rows - 1) * b.stride + b.width) return false;
  const auto floor_div = [](Wide x, Wide y) { return x / y - (x % y < 0); };
  if (a.stride != 0 && b.stride != 0) {
    const int64_t period = std::gcd(a.stride, b.stride);
    const Wide in = at - floor_div(at, period) * period;
    if (in >= a.width && in + b.width <= period) return false;
    if (a.stride == b.stride && a.width <= a.stride) {
      // row i of a and row i - m of b: at - m stride apart
      for (Wide m = floor_div(at, a.stride); m <= floor_div(at, a.stride) + 1; ++m) {
        const Wide apart = at - m * a.stride;
        if (m < a.rows && -m < b.rows && apart < a.width && -apart < b.width) return true;
      }
      return false;
    }
  }
  // (the rows of a from the first that reaches b's on, to the last)
  const Wide reach = (Wide)(b.rows - 1) * b.stride + b.width;
  int64_t i = 0, end = a.rows;
  if (a.stride != 0) {
    i = (int64_t)std::max<Wide>(floor_div(at - a.width, a.stride) + 1, 0);
    end = (int64_t)std::min<Wide>(floor_div(at + reach - 1, a.stride) + 1, a.rows);
  }
  for (; i < end; ++i) {
    const Wide from = (Wide)i * a.stride - at;  // row i of a from b's first
    if (b.stride == 0) {
      if (from < b.width && -from < a.width) return true;
      continue;
    }
    const Wide first = std::max<Wide>(floor_div(from - b.width, b.stride) + 1, 0);
    const Wide last = std::min<Wide>(floor_div(from + a.width - 1, b.stride), b.rows - 1);
    if (first <= last) return true;
  }
  return false;
}

// Whether output rows may lie there: they are the input's own, in place, or share no byte with them.
inline bool out_ok(const RowSpan& in, const RowSpan& out) {
  return (in.p == out.p && in.stride == out.stride) || !rows_meet(in, out);
}

// V elements of T as one load or store at any address that T may have: 16
// bytes are one instruction, which the memory pipeline takes at any alignment.
template <class T, int V>
struct __attribute__((packed, aligned(sizeof(T)))) LoosePack {
  T v[V];
};

// 16 bytes in flight: whole registers, so that what is loaded is not unpacked,
// and waited for, before it is used.
using Raw = uint32_t __attribute__((ext_vector_type(4)));
struct __attribute__((packed, aligned(2))) LooseRaw {
  Raw v;
};
__device__ __forceinline__ Raw load_raw(const void* p) { return static_cast<const LooseRaw*>(p)->v; }

// Element j of 16 bytes of T.
template <class T>
__device__ __forceinline__ float element(const Raw& r, int j) {
  if constexpr (sizeof(T) == 4) {
    return __uint_as_float(r[j]);
  } else if constexpr (std::is_same<T, bf16>::value) {
    return __uint_as_float(j & 1 ? r[j >> 1] & 0xFFFF0000u : r[j >> 1] << 16);
  } else {
    const uint16_t h = (uint16_t)(j & 1 ? r[j >> 1] >> 16 : r[j >> 1]);
    return (float)__builtin_bit_cast(f16, h);
  }
}

// v as a T, rounded from fp32 wherever it stands. fp16: an operation before it
// that the compiler takes together with the rounding (v_fma_mixlo_f16 does not
// round to fp32 between, which in 235 of 4.2 million results shows) would make
// an element's last bit depend on its place in a vector.
template <class T>
__device__ __forceinline__ T rounded(float v) {
  if constexpr (std::is_same<T, f16>::value) asm("" : "+v"(v));
  return (T)v;
}

// The sum of v over groups of G lanes (a power of two, at most 64), in every
// lane of the group. All lanes of the wave must be active. Within 16 lanes by
// data-parallel moves (xor 1, xor 2, then mirrors, which meet equal values),
// then by exchanging rows of 16 and halves of the wave.
template <int kCtrl>
__device__ __forceinline__ uint32_t dpp_bits(uint32_t v) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, kCtrl, 0xF, 0xF, false);
}
template <int kCtrl>
__device__ __forceinline__ float dpp_move(float v) {
  return __uint_as_float(dpp_bits<kCtrl>(__float_as_uint(v)));
}
__device__ __forceinline__ float group_sum(float v, int G) {
  if (G > 1) v += dpp_move<0xB1>(v);    // quad_perm 1 0 3 2
  if (G > 2) v += dpp_move<0x4E>(v);    // quad_perm 2 3 0 1
  if (G > 4) v += dpp_move<0x141>(v);   // row_half_mirror
  if (G > 8) v += dpp_move<0x140>(v);   // row_mirror
  if (G > 16) {
    const auto x = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(x[0]) + __uint_as_float(x[1]);
  }
  if (G > 32) {
    const auto x = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(x[0]) + __uint_as_float(x[1]);
  }
  return v;
}

// The largest v of a wave, in every lane (a NaN counts only beside NaNs).
__device__ __forceinline__ float wave_max(float v) {
  v = fmaxf(v, dpp_move<0xB1>(v));
  v = fmaxf(v, dpp_move<0x4E>(v));
  v = fmaxf(v, dpp_move<0x141>(v));
  v = fmaxf(v, dpp_move<0x140>(v));
  auto x = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = fmaxf(__uint_as_float(x[0]), __uint_as_float(x[1]));
  x = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(x[0]), __uint_as_float(x[1]));
}

}  // namespace mlkv
