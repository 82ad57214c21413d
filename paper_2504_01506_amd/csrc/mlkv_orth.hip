// Updates made orthogonal by Newton-Schulz steps.
//
// Three products a step, all of the form C[i][j] = sum_k P[i][k] Q[j][k] with
// both operands' k running in memory, as the matrix units want it: X X^T, then
// A A (A is symmetric), then B X from X^T, which is kept beside X. The first
// two results are symmetric: only tiles on and below the diagonal are computed,
// and written twice.
//
// Numbers are held as fp16 pairs hi + lo, 22 bits: norms bound every entry
// (|X| <= 1.21, |A| <= 1.45, |B| <= 2.81, the quintic's largest values), so one
// power of two a matrix, 2^15 for X and A, 2^14 for B, keeps hi below 65504
// and lo in its range. A product takes hi hi + hi lo + lo hi; what is left out
// is 2^-22 of it, below the rounding of the fp32 sums. Bound by the matrix
// units: three fp16 products instead of one fp32 product, at 7 times the rate. Five
// steps of 4096 x 4096 take 4.1 ms, 1.0 PFLOP/s of fp16 products, of which a large
// library product reaches 1.08 to 1.33, by card.
//
// Updates in bf16 and fp16 take the same pairs: what a step rounds off lies in
// the directions of small singular values too, and each later step stretches it
// there by up to 3.4445. With operands of 11 bits a result is off by 0.7e-3 of its norm
// (noise, 5 steps) to 2.4e-2 (low rank, 8 steps), bf16's own rounding being
// 1.7e-3; with pairs by about as much as the steps in fp32.
//
// Products of a few hundred to 1024 rows have fewer tiles than the device has
// units; they are bound by what one unit loads, 60 to 80 KB a us, and by launches,
// three a step: 1024 x 4096 425 us (X X^T 33 a step on 136 tiles, A A 13, B X 43),
// 1024 x 1024 192, 512 x 512 136.
#include "mlkv_ops.h"
#include "mlkv_tiles.h"

#include <algorithm>
#include <atomic>
#include <cmath>

namespace mlkv {
namespace {

constexpr float kA = 3.4445f, kB = -4.7750f, kC = 2.0315f;
constexpr int kThreads = 256;
constexpr int kNormBlocks = 512; // sums of squares a matrix, at most
constexpr int kPlanes = 2;       // hi and lo

using half4 = _Float16 __attribute__((ext_vector_type(4)));
using half8 = _Float16 __attribute__((ext_vector_type(8)));
using float16v = float __attribute__((ext_vector_type(16)));

struct Shape {
  int m, n;    // as iterated on: m <= n
  int mp, np;  // padded, zeros in the padding
  bool turned; // rows > cols
};

struct User {
  const void* g;
  void* out;
  int64_t g_batch, g_row, o_batch, o_row;
};

// Lets a kernel take more LDS than 64 KB on the current device, once a device.
template <auto kKernel>
hipError_t allow_lds(int bytes) {
  static std::atomic<uint64_t> done{0};
  int dev = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return e;
  const uint64_t bit = dev < 64 ? 1ull << dev : 0;
  if (done.load(std::memory_order_relaxed) & bit) return hipSuccess;
  e = hipFuncSetAttribute(reinterpret_cast<const void*>(kKernel), hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (e == hipSuccess) done.fetch_or(bit, std::memory_order_relaxed);
  return e;
}

// ---- norm and first X ----
// A wave a row in turn. Bound by memory: 4096 x 4096 fp32 14 to 17 us.
template <class T>
__global__ __launch_bounds__(kThreads) void k_orth_norm(User u, int64_t rows, int64_t cols, double* sums) {
  constexpr int V = 16 / sizeof(T), kUnroll = 4;
  __shared__ double part[kThreads / 64];
  const T* g = static_cast<const T*>(u.g) + blockIdx.y * u.g_batch;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int vecs = (int)(cols / V);
  double t = 0.0;
  const auto add = [&](float x) { t = __builtin_fma((double)x, (double)x, t); };
  for (int64_t r = blockIdx.x * 4 + wave; r < rows; r += gridDim.x * 4) {
    const T* row = g + r * u.g_row;
    for (int v = lane; v < vecs; v += 64 * kUnroll) {
      Raw p[kUnroll];
#pragma unroll
      for (int k = 0; k < kUnroll; ++k) {
        p[k] = Raw{0, 0, 0, 0};
        if (v + 64 * k < vecs) p[k] = load_raw(row + (int64_t)(v + 64 * k) * V);
      }
#pragma unroll
      for (int k = 0; k < kUnroll; ++k)
#pragma unroll
        for (int e = 0; e < V; ++e) add(element<T>(p[k], e));
    }
    const int rest = vecs * V + lane;
    if (rest < cols) add((float)row[rest]);
  }
  for (int o = 32; o; o >>= 1) t += __shfl_xor(t, o);
  if (lane == 0) part[wave] = t;
  __syncthreads();
  if (threadIdx.x == 0) sums[(int64_t)blockIdx.y * gridDim.x + blockIdx.x] = part[0] + part[1] + part[2] + part[3];
}

__device__ __forceinline__ void split(float v, _Float16& hi, _Float16& lo) {
  hi = (_Float16)v;
  lo = (_Float16)(v - (float)hi);
}

// Planes of one matrix: hi at p, lo `plane` elements behind it.
struct Planes {
  _Float16* p;
  int64_t plane, batch;
  int ld;
};

// X and X^T from G, 64 x 64 elements a block, 8 a thread at a time, the
// transposed ones through LDS. Bound by memory: 2 or 4 bytes read and 8 written
// an element (4096 x 4096 fp32 31 us, 6.5 TB/s).
template <class T>
__global__ __launch_bounds__(kThreads) void k_orth_begin(User u, const double* sums, int nsums, float eps, Planes straight,
                                                         Planes turned, int rows, int cols) {
  constexpr int V = 16 / sizeof(T);
  __shared__ float tile[64][65];
  __shared__ double part[kThreads / 64];
  const T* g = static_cast<const T*>(u.g) + blockIdx.z * u.g_batch;
  const int r0 = blockIdx.y * 64, c0 = blockIdx.x * 64;
  const int y = threadIdx.x >> 3, c = (threadIdx.x & 7) * 8;  // (rows y and y + 32 of the tile)
  Raw raw[2][8 / V];
  bool whole[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int r = r0 + y + h * 32;
    whole[h] = r < rows && c0 + c + 8 <= cols;
#pragma unroll
    for (int k = 0; k < 8 / V; ++k) {
      raw[h][k] = Raw{0, 0, 0, 0};
      if (whole[h]) raw[h][k] = load_raw(g + r * u.g_row + c0 + c + k * V);
    }
  }
  double t = 0.0;
  for (int k = threadIdx.x; k < nsums; k += kThreads) t += sums[(int64_t)blockIdx.z * nsums + k];
  for (int o = 32; o; o >>= 1) t += __shfl_xor(t, o);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = t;
  __syncthreads();
  t = part[0] + part[1] + part[2] + part[3];
  const double inv = 32768.0 / (sqrt(t) + (double)eps);
  const auto store = [](const float (&v)[8], const Planes& to, _Float16* at) {
    half8 hi, lo;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      _Float16 h, l;
      split(v[e], h, l);
      hi[e] = h;
      lo[e] = l;
    }
    *reinterpret_cast<half8*>(at) = hi;
    *reinterpret_cast<half8*>(at + to.plane) = lo;
  };
  // (sides are padded to whole tiles, with zeros)
  _Float16* a = straight.p + blockIdx.z * straight.batch + (int64_t)r0 * straight.ld + c0;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int in = y + h * 32, r = r0 + in;
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      float x = element<T>(raw[h][e / V], e % V);
      if (!whole[h] && r < rows && c0 + c + e < cols) x = (float)g[r * u.g_row + c0 + c + e];
      v[e] = (float)((double)x * inv);
      tile[in][c + e] = v[e];
    }
    store(v, straight, a + (int64_t)in * straight.ld + c);
  }
  __syncthreads();
  _Float16* b = turned.p + blockIdx.z * turned.batch + (int64_t)c0 * turned.ld + r0;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int in = y + h * 32;
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = tile[c + e][in];
    store(v, turned, b + (int64_t)in * turned.ld + c);
  }
}

// ---- products ----
enum Step : int { kSquareX, kSquareA, kApplyB, kApplyLast };

struct ProdArgs {
  Planes P, Q;   // operands
  Planes add;    // what the epilogue adds a multiple of, read as [j][i]: A (symmetric) or X^T
  Planes out;    // written as [j][i] (A, B: symmetric; X^T)
  Planes out2;   // kApplyB: X, written as [i][j]
  User u;        // kApplyLast
  Shape s;
  int k;         // padded length of the sum
  int ti, tj;    // tiles of i and of j
};

using lds_ptr = __attribute__((address_space(3))) void*;
using global_ptr = const __attribute__((address_space(1))) void*;

// Where row r's 16-byte piece c lies in a stage with rows of kDepth halves. LDS
// has 64 banks, 256 bytes side by side, which hold 4 (2) such rows: their pieces
// are exchanged alike, those of the next 4 (2) otherwise, so that pieces c of 16
// rows in a row fall into 16 different groups of banks. Exchanged by the row
// within 128 bytes only, half of LDS's cycles were conflicts; so, one in ten
// (4096 x 4096 fp32 4.22 ms then, 4.14 now; 2048 x 2048 bf16 437 us, 418).
template <int kDepth>
__device__ __forceinline__ int piece(int r, int c) {
  return kDepth == 32 ? r * 32 + ((c ^ (r >> 2)) & 3) * 8 : r * 64 + ((c ^ (r >> 1)) & 7) * 8;
}

// Waits until at most kLater of the wave's loads are in flight and its reads of
// LDS are done, then for the block's other waves.
template <int kLater>
__device__ __forceinline__ void stage_barrier() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(kLater) : "memory");
}

// A square tile of C, kSide a side, and its waves: kI x kJ that share it in
// equal parts, or (kK > 1) kK that each have all of it for every kK-th piece of
// 16 of k and join their sums at the end. Blocks of 32 x 32; kBytes of LDS for
// stages of kDepth. A small tile in parts reads four pieces of LDS for three
// products and waits for each in turn; by pieces of k it reads eight for twelve.
template <int kSide, int kI, int kJ, int kK, int kDepth_, int kBytes>
struct Tile {
  static_assert(kK == 1 || (kI == 1 && kJ == 1 && kK == 4 && kSide == 64), "four waves, a block of the sum each");
  static constexpr int side = kSide, depth = kDepth_, lds = kBytes, waves_k = kK, waves = kI * kJ * kK;
  static constexpr int blocks_i = kSide / kI / 32, blocks_j = kSide / kJ / 32;  // of a wave
  static constexpr int across = kK > 1 ? 2 : kJ;                               // waves along j of the result
  static constexpr int out_i = kK > 1 ? 1 : blocks_i, out_j = kK > 1 ? 1 : blocks_j;
};

// kStages stages in LDS: while one is multiplied, the others are on their way
// from memory.
template <class T, class Tile_, int kStep>
__global__ __launch_bounds__(64 * Tile_::waves) void k_orth_product(ProdArgs a) {
  constexpr int kTile = Tile_::side, kDepth = Tile_::depth, kWaves = Tile_::waves;
  constexpr int kBi = Tile_::blocks_i, kBj = Tile_::blocks_j, kOi = Tile_::out_i, kOj = Tile_::out_j;
  constexpr int kStage = 2 * kPlanes * kTile * kDepth;  // halves
  constexpr int kStages = Tile_::lds / (int)(kStage * sizeof(_Float16));
  constexpr int kRows = 512 / kDepth;                   // rows of a load: a kilobyte
  constexpr int kLoads = 2 * kPlanes * kTile / kRows / kWaves;  // of a wave and stage
  static_assert(kStages >= 2 && 2 * kPlanes * kTile / kRows % kWaves == 0, "stages and loads");
  extern __shared__ __align__(16) _Float16 lds[];
  constexpr bool kSym = kStep == kSquareX || kStep == kSquareA;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  // neighbouring tiles on one XCD (blocks go round the 8 in turn), for its L2
  const int total = gridDim.x, q8 = total / 8, r8 = total % 8, xcd = blockIdx.x % 8;
  const int id = xcd * q8 + min(xcd, r8) + blockIdx.x / 8;
  int bi, bj;
  if constexpr (kSym) {
    bi = (int)((__builtin_sqrtf(8.0f * (float)id + 1.0f) - 1.0f) * 0.5f);
    while ((bi + 1) * (bi + 2) / 2 <= id) ++bi;
    while (bi * (bi + 1) / 2 > id) --bi;
    bj = id - bi * (bi + 1) / 2;
  } else {
    // columns of 8 tiles
    const int band = id / (8 * a.tj), in = id - band * 8 * a.tj;
    const int high = min(8, a.ti - band * 8);
    bj = in / high;
    bi = band * 8 + in - bj * high;
  }
  const int rows_i = a.s.mp, rows_j = kSym ? a.s.mp : a.s.np;

  // A load takes kRows rows of a plane, a lane a piece. Rows that a tile has
  // beyond the matrix are read as its last.
  constexpr int kLanes = 64 / kRows;  // of a row
  const _Float16* from[kLoads];
#pragma unroll
  for (int q = 0; q < kLoads; ++q) {
    const int seg = q * kWaves + wave, plane = seg / (kTile / kRows), rows = seg % (kTile / kRows) * kRows;
    const bool is_p = plane < kPlanes;
    const Planes& o = is_p ? a.P : a.Q;
    const int in = rows + lane / kLanes, r = min((is_p ? bi : bj) * kTile + in, (is_p ? rows_i : rows_j) - 1);
    from[q] = o.p + blockIdx.z * o.batch + (plane % kPlanes) * o.plane + (int64_t)r * o.ld +
              (piece<kDepth>(in, lane % kLanes) - in * kDepth);
  }
  const auto fill = [&](int t) {
#pragma unroll
    for (int q = 0; q < kLoads; ++q) {
      const int seg = q * kWaves + wave, plane = seg / (kTile / kRows), rows = seg % (kTile / kRows) * kRows;
      _Float16* to = lds + (t % kStages) * kStage + plane * kTile * kDepth + rows * kDepth;
      __builtin_amdgcn_global_load_lds((global_ptr)(from[q] + t * kDepth), (lds_ptr)to, 16, 0, 0);
    }
  };

  float16v acc[kBi][kBj];
#pragma unroll
  for (int x = 0; x < kBi; ++x)
#pragma unroll
    for (int y = 0; y < kBj; ++y)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[x][y][e] = 0.0f;

  const int wi = Tile_::waves_k > 1 ? 0 : wave / Tile_::across * (kBi * 32);
  const int wj = Tile_::waves_k > 1 ? 0 : wave % Tile_::across * (kBj * 32);
  const int stages = a.k / kDepth;
#pragma unroll
  for (int t = 0; t < kStages - 1; ++t)
    if (t < stages) fill(t);
  // stage t is there, and all waves are done reading stage t - 1, whose place is filled next
  const auto next_stage = [&](int t) {
    if (t + kStages - 2 < stages) stage_barrier<(kStages - 2) * kLoads>();
    else stage_barrier<0>();
    if (t + kStages - 1 < stages) fill(t + kStages - 1);
  };
  struct Pieces {
    half8 p[kBi][kPlanes], q[kBj][kPlanes];
  };
  const auto read = [&](Pieces& s, int t, int h) {
    const _Float16* st = lds + (t % kStages) * kStage;
    const int c = (Tile_::waves_k > 1 ? h * Tile_::waves_k + wave : h) * 2 + lane / 32;
#pragma unroll
    for (int e = 0; e < kPlanes; ++e) {
#pragma unroll
      for (int x = 0; x < kBi; ++x)
        s.p[x][e] = *reinterpret_cast<const half8*>(st + e * kTile * kDepth +
                                                    piece<kDepth>(wi + x * 32 + (lane & 31), c));
#pragma unroll
      for (int y = 0; y < kBj; ++y)
        s.q[y][e] = *reinterpret_cast<const half8*>(st + (kPlanes + e) * kTile * kDepth +
                                                    piece<kDepth>(wj + y * 32 + (lane & 31), c));
    }
  };
  const auto multiply = [&](const Pieces& s) {
#pragma unroll
    for (int x = 0; x < kBi; ++x)
#pragma unroll
      for (int y = 0; y < kBj; ++y)
        acc[x][y] = __builtin_amdgcn_mfma_f32_32x32x16_f16(s.p[x][0], s.q[y][0], acc[x][y], 0, 0, 0);
#pragma unroll
    for (int x = 0; x < kBi; ++x)
#pragma unroll
      for (int y = 0; y < kBj; ++y)
        acc[x][y] = __builtin_amdgcn_mfma_f32_32x32x16_f16(s.p[x][0], s.q[y][1], acc[x][y], 0, 0, 0);
#pragma unroll
    for (int x = 0; x < kBi; ++x)
#pragma unroll
      for (int y = 0; y < kBj; ++y)
        acc[x][y] = __builtin_amdgcn_mfma_f32_32x32x16_f16(s.p[x][1], s.q[y][0], acc[x][y], 0, 0, 0);
  };
  if constexpr (Tile_::waves_k > 1) {
    // a wave has one piece of a stage: it reads the next while it multiplies this one
    static_assert(kDepth / 16 == Tile_::waves_k, "a piece a wave and stage");
    Pieces s[2];
    next_stage(0);
    read(s[0], 0, 0);
    int t = 1;
    for (; t + 1 < stages; t += 2) {
      next_stage(t);
      read(s[1], t, 0);
      multiply(s[0]);
      next_stage(t + 1);
      read(s[0], t + 1, 0);
      multiply(s[1]);
    }
    if (t < stages) {
      next_stage(t);
      read(s[1], t, 0);
      multiply(s[0]);
      multiply(s[1]);
    } else {
      multiply(s[0]);
    }
  } else {
    for (int t = 0; t < stages; ++t) {
      next_stage(t);
#pragma unroll
      for (int h = 0; h < kDepth / 16; ++h) {
        Pieces s;
        read(s, t, h);
        multiply(s);
      }
    }
  }

  // A wave's sums to write: its own, or the block of its number, of all waves.
  float16v sum[kOi][kOj];
  const int oi = Tile_::waves_k > 1 ? wave / 2 * 32 : wi, oj = Tile_::waves_k > 1 ? wave % 2 * 32 : wj;
  if constexpr (Tile_::waves_k == 1) {
#pragma unroll
    for (int x = 0; x < kOi; ++x)
#pragma unroll
      for (int y = 0; y < kOj; ++y) sum[x][y] = acc[x][y];
  } else {
    float4* part = reinterpret_cast<float4*>(lds);  // [waves][4 blocks][4][64 lanes]
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 4; ++k)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float16v& v = acc[k >> 1][k & 1];
        part[((wave * 4 + k) * 4 + e) * 64 + lane] = make_float4(v[e * 4], v[e * 4 + 1], v[e * 4 + 2], v[e * 4 + 3]);
      }
    __syncthreads();
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      float4 t = part[(wave * 4 + e) * 64 + lane];
#pragma unroll
      for (int w = 1; w < 4; ++w) {
        const float4 v = part[((w * 4 + wave) * 4 + e) * 64 + lane];
        t.x += v.x;
        t.y += v.y;
        t.z += v.z;
        t.w += v.w;
      }
      sum[0][0][e * 4] = t.x;
      sum[0][0][e * 4 + 1] = t.y;
      sum[0][0][e * 4 + 2] = t.z;
      sum[0][0][e * 4 + 3] = t.w;
    }
  }

  // Epilogue. A lane holds column j = lane % 32 of each block, rows i in fours.
  // Blocks go to and from memory through LDS, a wave's own 5 KB, as rows of 64
  // bytes in 16-byte pieces: written straight from these registers a row is
  // four pieces of 16 bytes, or its other side 2 bytes a lane (4096 x 4096 B X 384
  // us, 411 straight).
  constexpr int kRow = 40;  // halves of a row there: 16 bytes more than it holds, against bank conflicts
  // These 5 KB lie behind the parts of the sum, where there are such: in the
  // parts' place a wave would write them before another has read its own. (A
  // barrier between did not hold that: the compiler takes reads of LDS whose values
  // only one branch needs into that branch, also past a barrier before it.)
  constexpr int kParts = Tile_::waves_k > 1 ? kWaves * 4 * 4 * 64 * (int)(sizeof(float4) / sizeof(_Float16)) : 0;
  static_assert((kParts + kWaves * 2 * 32 * kRow) * (int)sizeof(_Float16) <= Tile_::lds, "LDS of the epilogue");
  if constexpr (Tile_::waves_k == 1) __syncthreads();
  _Float16* mine = lds + kParts + wave * (2 * 32 * kRow);
  // the block's rows of a plane from LDS, or to it; `from` and `to` point at the block's corner
  const auto store_block = [&](const _Float16* from, _Float16* to, int ld) {
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int r = (lane + 64 * k) >> 2, c = lane & 3;
      *reinterpret_cast<half8*>(to + (int64_t)r * ld + c * 8) = *reinterpret_cast<const half8*>(from + r * kRow + c * 8);
    }
  };
  const auto load_block = [&](const _Float16* from, int ld, _Float16* to) {
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int r = (lane + 64 * k) >> 2, c = lane & 3;
      *reinterpret_cast<half8*>(to + r * kRow + c * 8) = *reinterpret_cast<const half8*>(from + (int64_t)r * ld + c * 8);
    }
  };
  const auto wave_sync = [] {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
  };
#pragma unroll
  for (int x = 0; x < kOi; ++x)
#pragma unroll
    for (int y = 0; y < kOj; ++y) {
      const int i0 = bi * kTile + oi + x * 32, j0 = bj * kTile + oj + y * 32;
      if (i0 >= rows_i || j0 >= rows_j) continue;  // (sides are padded to whole blocks)
      const int il = (lane >> 5) * 4, jl = lane & 31;
      if constexpr (kStep != kSquareX) {
        const _Float16* add = a.add.p + blockIdx.z * a.add.batch + (int64_t)j0 * a.add.ld + i0;
        load_block(add, a.add.ld, mine);
        load_block(add + a.add.plane, a.add.ld, mine + 32 * kRow);
        wave_sync();
      }
      half4 hi[4], lo[4];
#pragma unroll
      for (int f = 0; f < 4; ++f) {
        float v[4];
        if constexpr (kStep == kSquareX) {
#pragma unroll
          for (int e = 0; e < 4; ++e) v[e] = sum[x][y][f * 4 + e] * 0x1p-15f;
        } else {
          const half4 h = *reinterpret_cast<const half4*>(mine + jl * kRow + f * 8 + il);
          const half4 l = *reinterpret_cast<const half4*>(mine + 32 * kRow + jl * kRow + f * 8 + il);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float old = (float)h[e] + (float)l[e];
            v[e] = kStep == kSquareA ? __builtin_fmaf(kC * 0x1p-16f, sum[x][y][f * 4 + e], kB * 0.5f * old)
                                     : __builtin_fmaf(0x1p-14f, sum[x][y][f * 4 + e], kA * old);
          }
        }
        if constexpr (kStep == kApplyLast) {
          const int i = i0 + f * 8 + il, j = j0 + jl;
          T* to = static_cast<T*>(a.u.out) + blockIdx.z * a.u.o_batch;
          if (j < a.s.n) {
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (i + e < a.s.m)
                to[a.s.turned ? j * a.u.o_row + i + e : (i + e) * a.u.o_row + j] = (T)(v[e] * 0x1p-15f);
          }
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            _Float16 h, l;
            split(v[e], h, l);
            hi[f][e] = h;
            lo[f][e] = l;
          }
        }
      }
      wave_sync();
      if constexpr (kStep != kApplyLast) {
#pragma unroll
        for (int f = 0; f < 4; ++f) {
          *reinterpret_cast<half4*>(mine + jl * kRow + f * 8 + il) = hi[f];
          *reinterpret_cast<half4*>(mine + 32 * kRow + jl * kRow + f * 8 + il) = lo[f];
        }
        wave_sync();
        _Float16* out = a.out.p + blockIdx.z * a.out.batch + (int64_t)j0 * a.out.ld + i0;
        store_block(mine, out, a.out.ld);
        store_block(mine + 32 * kRow, out + a.out.plane, a.out.ld);
        wave_sync();
        if (kStep == kApplyB || (kSym && bi != bj)) {
          const Planes& o = kSym ? a.out : a.out2;
#pragma unroll
          for (int f = 0; f < 4; ++f)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              mine[(f * 8 + il + e) * kRow + jl] = hi[f][e];
              mine[(32 + f * 8 + il + e) * kRow + jl] = lo[f][e];
            }
          wave_sync();
          _Float16* to = o.p + blockIdx.z * o.batch + (int64_t)i0 * o.ld + j0;
          store_block(mine, to, o.ld);
          store_block(mine + 32 * kRow, to + o.plane, o.ld);
          wave_sync();
        }
      }
    }
}

// ---- matrices of few rows: panels in LDS ----
// Matrices of at most 64 rows (as iterated on) are cut into panels of 256
// columns. A block holds one in LDS, X and X^T as pairs, A, and B in the place
// of X X^T's second half sums: all 160 KB of a unit. Eight waves: X X^T a block
// of 32 x 32 and half the sum each, A A the blocks, B X 32 columns each. A
// matrix of one panel takes all steps in one launch; of several, a launch a
// step, in which every block joins all panels' X X^T and works out A and B for
// itself. Bound by the latency of the chain, three products and four exchanges
// through LDS a step: 16 matrices of 64 x 250 39 us, 5 steps of 5.9 and the first
// load; 64 x 4096 in 16 panels 83. (Both row blocks of B X
// at a time, each piece of X^T read once: no faster.)
constexpr int kPanelRows = 64, kPanelCols = 256, kPanelThreads = 512;
constexpr int kPanelX = kPanelRows * kPanelCols, kPanelA = kPanelRows * kPanelRows;  // halves of a plane
constexpr size_t kPanelLds = sizeof(_Float16) * (4 * kPanelX + 4 * kPanelA);

// Element k of row r of a plane with rows of kRow halves, pieces of 16 bytes
// exchanged by the row as in a stage.
template <int kRow>
__device__ __forceinline__ int spot(int r, int k) {
  const int by = kRow == 64 ? (r >> 1) & 7 : r & 15;
  return r * kRow + (((k >> 3) ^ by) << 3) + (k & 7);
}

// What a step's launch leaves to the next (matrices of several panels).
struct PanelWork {
  _Float16* xt;        // [batch][panels][2][256][64]: X^T, as it lies in LDS
  float4* sums;        // [batch][2 turns][panels][2 halves][4 blocks][4][64 lanes]: X X^T
  const double* norm;  // [batch][nsums]
  int nsums;
};

// kWhole: a matrix's only panel, all steps. kFirst: X and its X X^T. kNext: one step.
enum PanelStep : int { kWhole, kFirst, kNext };
template <class T, int kStep>
__global__ __launch_bounds__(kPanelThreads) void k_orth_panel(User u, PanelWork w, int rows, int cols, bool turned,
                                                             int steps, float eps, int turn, bool last) {
  constexpr int kSums = 4 * 4 * 64;  // float4s of the sums of half a panel
  extern __shared__ __align__(16) _Float16 panel_lds[];
  _Float16* X = panel_lds;                // [2][64][256]
  _Float16* XT = X + 2 * kPanelX;         // [2][256][64]
  _Float16* A = XT + 2 * kPanelX;         // [2][64][64]
  _Float16* B = A + 2 * kPanelA;          // [2][64][64]
  float4* half = reinterpret_cast<float4*>(B);  // [4 blocks][4][64 lanes]: the sums' second halves, before B
  double* part = reinterpret_cast<double*>(A);  // [8], before A
  int lane = threadIdx.x & 63;
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int m = turned ? cols : rows, n_all = turned ? rows : cols;
  const int panel = blockIdx.x, panels = gridDim.x, from = panel * kPanelCols, n = min(n_all - from, kPanelCols);
  _Float16* keep = kStep == kWhole ? nullptr : w.xt + ((int64_t)blockIdx.y * panels + panel) * 2 * kPanelX;
  float4* sums = kStep == kWhole ? nullptr : w.sums + (int64_t)blockIdx.y * 2 * panels * 2 * kSums;
  if constexpr (kStep == kNext) {
#pragma unroll
    for (int e = 0; e < 2 * kPanelX / 8 / kPanelThreads; ++e)
      reinterpret_cast<Raw*>(XT)[e * kPanelThreads + tid] = reinterpret_cast<const Raw*>(keep)[e * kPanelThreads + tid];
  } else {
    const T* g = static_cast<const T*>(u.g) + blockIdx.y * u.g_batch + (turned ? from * u.g_row : from);
    const int g_rows = turned ? n : rows, g_cols = turned ? cols : n;

    // G's rows along the threads: 64 x 256, or 256 x 64 where it is turned
    constexpr int kEach = kPanelX / kPanelThreads;
    const int wide = turned ? 6 : 8;  // log2 of that
    float v[kEach];
    double t = 0.0;
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
      const int at = e * kPanelThreads + tid, r = at >> wide, c = at & ((1 << wide) - 1);
      v[e] = r < g_rows && c < g_cols ? (float)g[r * u.g_row + c] : 0.0f;
    }
    if constexpr (kStep == kWhole) {
#pragma unroll
      for (int e = 0; e < kEach; ++e) t = __builtin_fma((double)v[e], (double)v[e], t);
    } else {
      for (int k = tid; k < w.nsums; k += kPanelThreads) t += w.norm[(int64_t)blockIdx.y * w.nsums + k];
    }
    for (int o = 32; o; o >>= 1) t += __shfl_xor(t, o);
    if (lane == 0) part[wave] = t;
    __syncthreads();
    t = 0.0;
    for (int k = 0; k < kPanelThreads / 64; ++k) t += part[k];
    const double inv = 32768.0 / (sqrt(t) + (double)eps);
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
      const int at = e * kPanelThreads + tid, r = at >> wide, c = at & ((1 << wide) - 1);
      const int i = turned ? c : r, j = turned ? r : c;
      _Float16 hi, lo;
      split((float)((double)v[e] * inv), hi, lo);
      X[spot<kPanelCols>(i, j)] = hi;
      X[kPanelX + spot<kPanelCols>(i, j)] = lo;
      XT[spot<kPanelRows>(j, i)] = hi;
      XT[kPanelX + spot<kPanelRows>(j, i)] = lo;
    }
  }
  __syncthreads();

  const int bi = (wave >> 1) & 1, bj = wave & 1, second = wave >> 2;  // of X X^T and A A
  // sums over pieces of 16 of k, from k0 on, of the block of rows p0 and q0 of planes of rows of kRow
  const auto multiply = [&](auto width, const _Float16* P, int p0, const _Float16* Q, int q0, int plane_p,
                            int plane_q, int k0, int count) {
    constexpr int kRow = decltype(width)::value;
    float16v a, b, c;  // (three chains of dependent products)
#pragma unroll
    for (int e = 0; e < 16; ++e) a[e] = b[e] = c[e] = 0.0f;
    const int row = lane & 31, deep = (lane >> 5) * 8;
    // two pieces at a time; one too many is of zeros
    for (int t = 0; t < count; t += 2) {
      half8 ph[2], pl[2], qh[2], ql[2];
#pragma unroll
      for (int d = 0; d < 2; ++d) {
        const int k = k0 + (t + d) * 16;
        const int sp = spot<kRow>(p0 + row, k + deep), sq = spot<kRow>(q0 + row, k + deep);
        ph[d] = *reinterpret_cast<const half8*>(P + sp);
        pl[d] = *reinterpret_cast<const half8*>(P + plane_p + sp);
        qh[d] = *reinterpret_cast<const half8*>(Q + sq);
        ql[d] = *reinterpret_cast<const half8*>(Q + plane_q + sq);
      }
#pragma unroll
      for (int d = 0; d < 2; ++d) {
        a = __builtin_amdgcn_mfma_f32_32x32x16_f16(ph[d], qh[d], a, 0, 0, 0);
        b = __builtin_amdgcn_mfma_f32_32x32x16_f16(ph[d], ql[d], b, 0, 0, 0);
        c = __builtin_amdgcn_mfma_f32_32x32x16_f16(pl[d], qh[d], c, 0, 0, 0);
      }
    }
#pragma unroll
    for (int e = 0; e < 16; ++e) a[e] += b[e] + c[e];
    return a;
  };
  // calls f(i, j, e): elements e .. e + 3 of a block at (i0, j0) are those at (i .. i + 3, j)
  const auto fours = [&](int i0, int j0, const auto& f) {
#pragma unroll
    for (int e = 0; e < 16; e += 4) f(i0 + e * 2 + (lane >> 5) * 4, j0 + (lane & 31), e);
  };
  const auto halves = [](const float16v& x, int e, half4& hi, half4& lo) {
#pragma unroll
    for (int d = 0; d < 4; ++d) {
      _Float16 h, l;
      split(x[e + d], h, l);
      hi[d] = h;
      lo[d] = l;
    }
  };
  // (A and B are symmetric: written as [j][i])
  const auto put = [&](_Float16* to, const float16v& x) {
    fours(bi * 32, bj * 32, [&](int i, int j, int e) {
      half4 hi, lo;
      halves(x, e, hi, lo);
      *reinterpret_cast<half4*>(to + spot<kPanelRows>(j, i)) = hi;
      *reinterpret_cast<half4*>(to + kPanelA + spot<kPanelRows>(j, i)) = lo;
    });
  };
  using OfX = std::integral_constant<int, kPanelCols>;
  using OfA = std::integral_constant<int, kPanelRows>;
  // pieces of the sum over n: an even number for each half, those behind n of zeros
  const int each = ((n + 15) / 16 + 3) / 4 * 2;
  const auto square = [&] {
    return multiply(OfX{}, X, bi * 32, X, bj * 32, kPanelX, kPanelX, second ? each * 16 : 0, each);
  };
  // the panel for the next launch: its X X^T, by halves, and X^T
  const auto leave = [&](int to) {
    const float16v s = square();
    float4* at = sums + ((int64_t)(to * panels + panel) * 2 + second) * kSums + (wave & 3) * 4 * 64 + lane;
#pragma unroll
    for (int e = 0; e < 4; ++e) at[e * 64] = make_float4(s[e * 4], s[e * 4 + 1], s[e * 4 + 2], s[e * 4 + 3]);
#pragma unroll
    for (int e = 0; e < 2 * kPanelX / 8 / kPanelThreads; ++e)
      reinterpret_cast<Raw*>(keep)[e * kPanelThreads + tid] = reinterpret_cast<const Raw*>(XT)[e * kPanelThreads + tid];
  };
  if constexpr (kStep == kFirst) {
    leave(0);
    return;
  }
  for (int step = 0; step < steps; ++step) {
    asm volatile("" : "+v"(lane));  // (places in LDS are worked out again: kept over the steps they take all registers)
    float16v s;
    if constexpr (kStep == kWhole) {
      s = square();
    } else {
#pragma unroll
      for (int e = 0; e < 16; ++e) s[e] = 0.0f;
      const float4* at = sums + ((int64_t)turn * panels * 2 + second) * kSums + (wave & 3) * 4 * 64 + lane;
#pragma unroll 2
      for (int k = 0; k < panels; ++k)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float4 x = at[(int64_t)k * 2 * kSums + e * 64];
          s[e * 4] += x.x;
          s[e * 4 + 1] += x.y;
          s[e * 4 + 2] += x.z;
          s[e * 4 + 3] += x.w;
        }
    }
    if (second) {
#pragma unroll
      for (int e = 0; e < 16; e += 4)
        half[((wave & 3) * 4 + e / 4) * 64 + lane] = make_float4(s[e], s[e + 1], s[e + 2], s[e + 3]);
    }
    __syncthreads();
    if (!second) {
#pragma unroll
      for (int e = 0; e < 16; e += 4) {
        const float4 h = half[(wave * 4 + e / 4) * 64 + lane];
        s[e] = (s[e] + h.x) * 0x1p-15f;
        s[e + 1] = (s[e + 1] + h.y) * 0x1p-15f;
        s[e + 2] = (s[e + 2] + h.z) * 0x1p-15f;
        s[e + 3] = (s[e + 3] + h.w) * 0x1p-15f;
      }
      put(A, s);
    }
    __syncthreads();
    if (!second) {
      const float16v q = multiply(OfA{}, A, bi * 32, A, bj * 32, kPanelA, kPanelA, 0, 4);
#pragma unroll
      for (int e = 0; e < 16; ++e) s[e] = __builtin_fmaf(kC * 0x1p-16f, q[e], kB * 0.5f * s[e]);
      put(B, s);
    }
    __syncthreads();
    // the wave's 32 columns; no other wave reads their rows of X^T, and none X
    const int j0 = wave * 32;
    if (kStep == kNext || j0 < n) {  // (columns behind n: zeros, which a panel keeps)
      float16v y[2];  // both are computed before either is written
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        y[x] = multiply(OfA{}, B, x * 32, XT, j0, kPanelA, kPanelX, 0, 4);
        fours(x * 32, j0, [&](int i, int j, int e) {
          const half4 hi = *reinterpret_cast<const half4*>(XT + spot<kPanelRows>(j, i));
          const half4 lo = *reinterpret_cast<const half4*>(XT + kPanelX + spot<kPanelRows>(j, i));
#pragma unroll
          for (int d = 0; d < 4; ++d)
            y[x][e + d] = __builtin_fmaf(0x1p-14f, y[x][e + d], kA * ((float)hi[d] + (float)lo[d]));
        });
      }
      const bool ends = kStep == kWhole ? step + 1 == steps : last;
      T* out = static_cast<T*>(u.out) + blockIdx.y * u.o_batch + (turned ? from * u.o_row : from);
#pragma unroll
      for (int x = 0; x < 2; ++x)
        fours(x * 32, j0, [&](int i, int j, int e) {
          if (!ends) {
            half4 hi, lo;
            halves(y[x], e, hi, lo);
            *reinterpret_cast<half4*>(XT + spot<kPanelRows>(j, i)) = hi;
            *reinterpret_cast<half4*>(XT + kPanelX + spot<kPanelRows>(j, i)) = lo;
#pragma unroll
            for (int d = 0; d < 4; ++d) {
              X[spot<kPanelCols>(i + d, j)] = hi[d];
              X[kPanelX + spot<kPanelCols>(i + d, j)] = lo[d];
            }
          } else if (j < n) {
#pragma unroll
            for (int d = 0; d < 4; ++d)
              if (i + d < m)
                out[turned ? j * u.o_row + i + d : (i + d) * u.o_row + j] = (T)(y[x][e + d] * 0x1p-15f);
          }
        });
    }
    __syncthreads();
    if constexpr (kStep == kNext) {
      if (!last) leave(turn ^ 1);
      return;
    }
  }
}

struct Layout {
  Shape s;
  int64_t xs, as;  // elements of a plane of X and of A
  int64_t sums, bytes;  // offset of the sums of squares; all
  int nsums;            // of a matrix
  int panels;           // of a matrix of few rows, or 0
};

Layout layout(int64_t batch, int64_t rows, int64_t cols) {
  Layout l{};
  l.s.turned = rows > cols;
  l.s.m = (int)std::min(rows, cols);
  l.s.n = (int)std::max(rows, cols);
  const auto up = [](int64_t v, int64_t t) { return (v + t - 1) / t * t; };
  l.nsums = (int)std::min<int64_t>((rows + 3) / 4, kNormBlocks);
  // (as many bytes for a matrix as for its transpose)
  const int64_t sums = batch * std::min<int64_t>((l.s.n + 3) / 4, kNormBlocks) * (int64_t)sizeof(double);
  l.panels = l.s.m <= kPanelRows ? (l.s.n + kPanelCols - 1) / kPanelCols : 0;
  if (l.panels > 0) {
    l.sums = batch * l.panels * (int64_t)(sizeof(_Float16) * 2 * kPanelX + sizeof(float4) * 4096);
    l.bytes = l.panels == 1 ? 0 : l.sums + sums;
    return l;
  }
  l.s.mp = (int)up(l.s.m, kOrthPad);
  l.s.np = (int)up(l.s.n, kOrthPad);
  l.xs = (int64_t)l.s.mp * l.s.np;
  l.as = (int64_t)l.s.mp * l.s.mp;
  // X, two of X^T, A and B, two planes each
  l.sums = up(batch * (l.xs * 6 + l.as * 4) * (int64_t)sizeof(_Float16), 256);
  l.bytes = l.sums + sums;
  return l;
}

using Tile64K = Tile<64, 1, 1, 4, 64, 131072>;
using Tile64 = Tile<64, 2, 2, 1, 32, 65536>;
using Tile128 = Tile<128, 2, 2, 1, 32, 65536>;
using Tile192 = Tile<192, 2, 2, 1, 32, 98304>;
using Tile256 = Tile<256, 2, 4, 1, 32, 131072>;

template <class T, class Tile_, int kStep>
hipError_t product_of(ProdArgs a, int64_t batch, hipStream_t st) {
  constexpr bool kSym = kStep == kSquareX || kStep == kSquareA;
  a.ti = (a.s.mp + Tile_::side - 1) / Tile_::side;
  a.tj = kSym ? a.ti : (a.s.np + Tile_::side - 1) / Tile_::side;
  const unsigned tiles = kSym ? (unsigned)(a.ti * (a.ti + 1) / 2) : (unsigned)(a.ti * a.tj);
  const hipError_t e = allow_lds<k_orth_product<T, Tile_, kStep>>(Tile_::lds);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((k_orth_product<T, Tile_, kStep>), dim3(tiles, 1, (unsigned)batch),
                     dim3(64 * Tile_::waves), Tile_::lds, st, a);
  return hipGetLastError();
}

template <class T, int kStep>
hipError_t product(const ProdArgs& a, int64_t batch, hipStream_t st) {
  switch (orth_tile(a.s.mp, a.s.np, batch, kStep == kSquareX || kStep == kSquareA, a.k)) {
    case OrthTile::k64K: return product_of<T, Tile64K, kStep>(a, batch, st);
    case OrthTile::k64: return product_of<T, Tile64, kStep>(a, batch, st);
    case OrthTile::k128: return product_of<T, Tile128, kStep>(a, batch, st);
    case OrthTile::k192: return product_of<T, Tile192, kStep>(a, batch, st);
    case OrthTile::k256: break;
  }
  return product_of<T, Tile256, kStep>(a, batch, st);
}

template <class T>
hipError_t iterate(const Layout& l, const User& u, int64_t batch, int steps, hipStream_t st, Planes X, Planes XT0,
                   Planes XT1, Planes A, Planes B) {
  Planes now = XT0, next = XT1;
  for (int k = 0; k < steps; ++k) {
    const bool last = k + 1 == steps;
    ProdArgs a{};
    a.s = l.s;
    a.u = u;
    a.P = a.Q = X;
    a.out = A;
    a.k = l.s.np;
    hipError_t e = product<float, kSquareX>(a, batch, st);
    if (e != hipSuccess) return e;
    a.P = a.Q = a.add = A;
    a.out = B;
    a.k = l.s.mp;
    if ((e = product<float, kSquareA>(a, batch, st)) != hipSuccess) return e;
    a.P = B;
    a.Q = a.add = now;
    a.out = next;
    a.out2 = X;
    e = last ? product<T, kApplyLast>(a, batch, st) : product<float, kApplyB>(a, batch, st);
    if (e != hipSuccess) return e;
    std::swap(now, next);
  }
  return hipSuccess;
}

template <class T, int kStep>
hipError_t panel_step(const Layout& l, const User& u, const PanelWork& w, int64_t batch, int64_t rows, int64_t cols,
                      int steps, float eps, int turn, bool last, hipStream_t st) {
  const hipError_t e = allow_lds<k_orth_panel<T, kStep>>((int)kPanelLds);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((k_orth_panel<T, kStep>), dim3((unsigned)l.panels, (unsigned)batch), dim3(kPanelThreads), kPanelLds,
                     st, u, w, (int)rows, (int)cols, l.s.turned, steps, eps, turn, last);
  return hipGetLastError();
}

template <class T>
hipError_t panel_steps(const Layout& l, const User& u, int64_t batch, int64_t rows, int64_t cols, int steps, float eps,
                       char* work, hipStream_t st) {
  PanelWork w{};
  if (l.panels == 1) return panel_step<T, kWhole>(l, u, w, batch, rows, cols, steps, eps, 0, true, st);
  double* norm = reinterpret_cast<double*>(work + l.sums);
  w.sums = reinterpret_cast<float4*>(work);
  w.xt = reinterpret_cast<_Float16*>(work + batch * l.panels * (int64_t)sizeof(float4) * 4096);
  w.norm = norm;
  w.nsums = l.nsums;
  hipLaunchKernelGGL((k_orth_norm<T>), dim3(l.nsums, (unsigned)batch), dim3(kThreads), 0, st, u, rows, cols, norm);
  hipError_t e = hipGetLastError();
  if (e == hipSuccess) e = panel_step<T, kFirst>(l, u, w, batch, rows, cols, 1, eps, 0, false, st);
  for (int k = 0; k < steps && e == hipSuccess; ++k)
    e = panel_step<T, kNext>(l, u, w, batch, rows, cols, 1, eps, k & 1, k + 1 == steps, st);
  return e;
}

template <class T>
hipError_t orthogonalize(const Layout& l, const User& u, int64_t batch, int64_t rows, int64_t cols, int steps,
                         float eps, char* work, hipStream_t st) {
  if (l.panels > 0) return panel_steps<T>(l, u, batch, rows, cols, steps, eps, work, st);
  _Float16* at = reinterpret_cast<_Float16*>(work);
  const auto planes = [&](int64_t elems, int ld) {
    Planes p;
    p.p = at;
    p.plane = elems;
    p.batch = 2 * elems;
    p.ld = ld;
    at += batch * 2 * elems;
    return p;
  };
  const Planes X = planes(l.xs, l.s.np), XT0 = planes(l.xs, l.s.mp), XT1 = planes(l.xs, l.s.mp),
               A = planes(l.as, l.s.mp), B = planes(l.as, l.s.mp);
  double* sums = reinterpret_cast<double*>(work + l.sums);
  hipLaunchKernelGGL((k_orth_norm<T>), dim3(l.nsums, (unsigned)batch), dim3(kThreads), 0, st, u, rows, cols, sums);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((k_orth_begin<T>), dim3((unsigned)(cols + 63) / 64, (unsigned)(rows + 63) / 64, (unsigned)batch),
                     dim3(kThreads), 0, st, u, sums, l.nsums, eps, l.s.turned ? XT0 : X, l.s.turned ? X : XT0,
                     (int)rows, (int)cols);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  return iterate<T>(l, u, batch, steps, st, X, XT0, XT1, A, B);
}

// A stack of matrices: `n` things `step` bytes apart, each `rows` rows of
// `width` bytes, `stride` apart; the longer way is the outer one.
struct Stack {
  int64_t step, n;
  RowSpan one;
  int64_t span() const { return (one.rows - 1) * one.stride + one.width; }
};
Stack stack_of(const void* p, int64_t batch_stride, int64_t row_stride, int64_t batch, int64_t rows, int64_t cols,
               int size) {
  if (batch <= 1 || batch_stride == 0) batch = 1, batch_stride = 0;
  if (rows <= 1 || row_stride == 0) rows = 1, row_stride = 0;
  batch_stride *= size;
  row_stride *= size;
  const int64_t width = cols * size;
  if (batch > 1 && (rows == 1 || row_stride <= batch_stride))
    return {batch_stride, batch, {p, row_stride, rows, width}};
  return {row_stride, rows, {p, batch_stride, batch, width}};
}

// Whether a byte of G's is one of out's, whose rows do not overlap: at once
// where both lie apart as a whole or each thing of the outer way does, else
// thing by thing.
bool stacks_meet(const Stack& g, const Stack& out) {
  if (!rows_meet({g.one.p, g.step, g.n, g.span()}, {out.one.p, out.step, out.n, out.span()})) return false;
  for (int64_t i = 0; i < g.n; ++i) {
    RowSpan a = g.one;
    a.p = static_cast<const char*>(a.p) + i * g.step;
    const int64_t from = (int64_t)(reinterpret_cast<uintptr_t>(a.p) - reinterpret_cast<uintptr_t>(out.one.p));
    const int64_t step = std::max<int64_t>(out.step, 1);
    const int64_t first = std::max<int64_t>((from - out.span()) / step, 0);
    const int64_t last = std::min((from + g.span()) / step, out.n - 1);
    for (int64_t j = first; j <= last; ++j) {
      RowSpan b = out.one;
      b.p = static_cast<const char*>(b.p) + j * out.step;
      if (rows_meet(a, b)) return true;
    }
  }
  return false;
}

int check_sizes(int64_t batch, int64_t rows, int64_t cols) {
  if (batch < 0 || batch > 65535) return op_error(MLKV_EINVAL, "batch must be in [0, 65535]");
  if (rows < 1 || rows > MLKV_ORTH_MAX_DIM || cols < 1 || cols > MLKV_ORTH_MAX_DIM)
    return op_error(MLKV_EINVAL, "rows and cols must be in [1, 32768]");
  return MLKV_OK;
}

}  // namespace
}  // namespace mlkv

using namespace mlkv;

extern "C" {

int64_t mlkv_orthogonalize_workspace(int64_t batch, int64_t rows, int64_t cols) {
  const int rc = check_sizes(batch, rows, cols);
  return rc ? rc : layout(batch, rows, cols).bytes;
}

int mlkv_orthogonalize(const void* d_g, int64_t batch_stride, int64_t row_stride, int64_t batch, int64_t rows,
                       int64_t cols, int32_t steps, float eps, int dtype, void* d_out, int64_t out_batch_stride,
                       int64_t out_row_stride, void* d_work, int64_t work_bytes, void* hip_stream) {
  const int rc = check_sizes(batch, rows, cols);
  if (rc) return rc;
  const int size = dtype_size(dtype);
  if (size == 0) return op_error(MLKV_EINVAL, "unknown dtype");
  if (steps < 1 || steps > 64) return op_error(MLKV_EINVAL, "steps must be in [1, 64]");
  if (!(eps > 0.0f) || std::isinf(eps)) return op_error(MLKV_EINVAL, "eps must be finite and > 0");
  if (batch == 0) return MLKV_OK;
  if (d_g == nullptr || d_out == nullptr) return op_error(MLKV_EINVAL, "g or out is NULL");
  if (!all_aligned(size, {d_g, d_out}))
    return op_error(MLKV_EINVAL, "a pointer is not aligned to its element type");
  if (!stride_ok(row_stride, rows, cols, true) || !stride_ok(out_row_stride, rows, cols, false))
    return op_error(MLKV_EINVAL, "row strides must be >= cols (or 0 in g)");
  // out's matrices one behind another, or their rows in turn (a matrix a head, heads side by side in a row)
  const int64_t span = (rows - 1) * (rows > 1 ? out_row_stride : 0) + cols;
  if (batch > 1 && (batch_stride < 0 || batch_stride > (int64_t(1) << 44) ||
                    !(stride_ok(out_batch_stride, batch, span, false) ||
                      (stride_ok(out_batch_stride, batch, cols, false) &&
                       out_row_stride >= (batch - 1) * out_batch_stride + cols))))
    return op_error(MLKV_EINVAL, "batch strides must not make matrices overlap");
  if (d_out == d_g && ((rows > 1 && row_stride != out_row_stride) || (batch > 1 && batch_stride != out_batch_stride)))
    return op_error(MLKV_EINVAL, "out may be g only with the same strides");
  if (d_out != d_g && stacks_meet(stack_of(d_g, batch_stride, row_stride, batch, rows, cols, size),
                                  stack_of(d_out, out_batch_stride, out_row_stride, batch, rows, cols, size)))
    return op_error(MLKV_EINVAL, "out overlaps g");
  const Layout l = layout(batch, rows, cols);
  if (l.bytes > 0 && (d_work == nullptr || work_bytes < l.bytes))
    return op_error(MLKV_EINVAL, "work is smaller than mlkv_orthogonalize_workspace");
  if (l.bytes > 0 && !all_aligned(256, {d_work}))
    return op_error(MLKV_EINVAL, "work must be at a multiple of 256 bytes");
  User u;
  u.g = d_g;
  u.out = d_out;
  u.g_batch = batch_stride;
  u.g_row = row_stride;
  u.o_batch = out_batch_stride;
  u.o_row = out_row_stride;
  const hipError_t e = dispatch_type(dtype, [&](auto t) {
    return orthogonalize<decltype(t)>(l, u, batch, rows, cols, steps, eps, static_cast<char*>(d_work),
                                      static_cast<hipStream_t>(hip_stream));
  });
  return e == hipSuccess ? MLKV_OK : op_launch_error(e, "mlkv_orthogonalize launch");
}

}  // extern "C"
