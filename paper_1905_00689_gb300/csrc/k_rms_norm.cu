// Root-mean-square norm with the residual's addition, its 8-bit output with
// scales, and its gradients (include/lstm_approx_ops.h).
//
// Forward, per row:   s = x + residual; rstd = (mean s^2 + eps)^-1/2; y = s rstd w
// Backward, per row:  ds = rstd (w dy - s rstd^2 mean(w dy s)) + dsum
//            columns: dw = sum over rows of dy s rstd
//
// Bound by memory: a row is read once, kept in registers as fp32 while its
// sum is formed, and written once.  `blockDim.x` threads share a row, each
// holds VPT times 8 neighbouring columns, and rows of at most 32 threads share
// a block (no block-wide sum then).
//
// Measured (device time, of the 6784 GB/s that a copy reaches): forward with
// residual, sum and output, 8192 x 4096 bf16 42 us (94%), 4000 x 7168 fp32 71 us
// (95%), 5001 x 1531 fp32 24 us (77%: unaligned rows in single values); with 8-bit output 8192 x 4096 46.5 us
// (74%: the conversions).  With the sum's low parts kept for the backward
// pass, 8192 x 4096 bf16 52 us (95%).  Backward, 8192 x 4096 bf16 49 us (81%), 20000 x
// 512 19 us (63%), 5001 x 1531 fp32 27 us (67%), 3000 x 7001 fp32 75 us (66%): every
// row's sum is a barrier (two warps to a row of 512 16-bit values already), behind which
// only the next row's loads are under way, and the column sums take 2 to 3 us more.
// One token: 2.9 us, the launch and one pass of latencies.
//
// Rows of more than 8192 columns are slower: backward their blocks of 1024 threads have 64
// registers to a thread and spill 0.4 to 0.8 KB of it up to 16384 columns, 1.2 to 2 KB above
// (3000 x 10000 fp32 163 us, 44%; 3000 x 12288 bf16 146 us, 30%; 1500 x 16392 bf16 202
// us, 14%); forward up to 0.1 KB above 16384 (3000 x 12288 bf16 81 us with low parts, 67%; in 32 bits 95,
// 91%).
//
// A warp moves its 256 columns in accesses of kUnit values: of 8 where every
// address is a multiple of 16 bytes, 8 neighbouring columns to a thread; else of
// 2 16-bit values at even addresses or of single values, a thread's columns 64
// or 32 apart, so that the lanes' lie next to one another.  For the forward
// pass's sum, and for groups of 8-bit outputs, these change hands through shared
// memory: the sum has the same bits in all three.  (With 8 neighbouring columns
// fetched one by one, 5001 x 1531 in 32 bits took 48 us forward; with all four
// tensors changing hands 25 forward and 32 backward.)
#include <cuda_fp8.h>

#include <algorithm>
#include <initializer_list>

#include "ops_common.cuh"
#include "ptx.cuh"

namespace lstm_approx_impl {
namespace {

using namespace lstm_approx_dev;

constexpr int kMaxD = 32768;
constexpr float kE4m3Max = 448.0f;
constexpr float kMinScale = 1.17549435e-38f;  // 2^-126

// Column of the thread's first of 8 neighbours in group j, and of its warp's first.
__device__ __forceinline__ int column(int j) { return (j * (int)blockDim.x + (int)threadIdx.x) * 8; }
__device__ __forceinline__ int warp_column(int j) { return (j * (int)blockDim.x + (int)(threadIdx.x & ~31u)) * 8; }

// Column of a thread's e-th value in group j.
template <int kUnit>
__device__ __forceinline__ int column_of(int j, int e) {
  return kUnit == 8 ? column(j) + e : warp_column(j) + (e / kUnit * 32 + (int)(threadIdx.x & 31)) * kUnit + e % kUnit;
}

// One warp's 256 columns on their way from lane to lane.  Every second 32 words have the halves of their 8 words
// exchanged: no two lanes meet in a bank, neither by single words nor when a lane takes 8 words (as 2 x 16 bytes).
struct Swap {
  float4 v[64];

  __device__ __forceinline__ static int place(int word) { return word ^ (word >> 3 & 4); }
  __device__ __forceinline__ float& word(int w) { return reinterpret_cast<float*>(v)[place(w)]; }
  __device__ __forceinline__ float2& pair(int w) { return *reinterpret_cast<float2*>(&word(w)); }
  __device__ __forceinline__ float4& four(int w) { return *reinterpret_cast<float4*>(&word(w)); }
};
__device__ __forceinline__ Swap& swap_of_warp() {
  __shared__ Swap swaps[32];
  return swaps[(threadIdx.y * blockDim.x + threadIdx.x) >> 5];
}

// A thread's 8 values in the order of kUnit become those of 8 neighbouring columns; called by whole warps.
template <int kUnit>
__device__ __forceinline__ void to_neighbours(float (&v)[8]) {
  if constexpr (kUnit != 8) {
    const int lane = threadIdx.x & 31;
    Swap& swap = swap_of_warp();
    __syncwarp();
#pragma unroll
    for (int e = 0; e < 8; e += kUnit) {
      const int at = (e / kUnit * 32 + lane) * kUnit;
      if constexpr (kUnit == 2) swap.pair(at) = make_float2(v[e], v[e + 1]);
      else swap.word(at) = v[e];
    }
    __syncwarp();
    const float4 lo = swap.four(8 * lane), hi = swap.four(8 * lane + 4);
    v[0] = lo.x, v[1] = lo.y, v[2] = lo.z, v[3] = lo.w, v[4] = hi.x, v[5] = hi.y, v[6] = hi.z, v[7] = hi.w;
  }
}

// A thread's part of group j as it lies in memory (zero past D), and as fp32.
template <typename T, int kUnit>
struct Raw8 {
  uint32_t w[8 * sizeof(T) / 4];

  __device__ __forceinline__ void load(const T* row, int j, int D) {
    const int lane = threadIdx.x & 31;
    if constexpr (kUnit == 8) {
      const int col = column(j);
#pragma unroll
      for (int q = 0; q < (int)sizeof(T) / 2; ++q) {
        uint4 v = make_uint4(0u, 0u, 0u, 0u);
        if (col < D) v = reinterpret_cast<const uint4*>(row + col)[q];
        w[4 * q] = v.x, w[4 * q + 1] = v.y, w[4 * q + 2] = v.z, w[4 * q + 3] = v.w;
      }
    } else if constexpr (kUnit * sizeof(T) == 4) {
#pragma unroll
      for (int q = 0; q < 8 / kUnit; ++q) {
        const int col = warp_column(j) + (q * 32 + lane) * kUnit;
        w[q] = col < D ? *reinterpret_cast<const uint32_t*>(row + col) : 0u;
      }
    } else {
#pragma unroll
      for (int q = 0; q < 8; ++q) {
        const int col = warp_column(j) + q * 32 + lane;
        const uint32_t v = col < D ? *reinterpret_cast<const uint16_t*>(row + col) : 0u;
        w[q / 2] = q & 1 ? w[q / 2] | v << 16 : v;
      }
    }
  }
  __device__ __forceinline__ float2 pair(int p) const {
    if constexpr (sizeof(T) == 4) return make_float2(__uint_as_float(w[2 * p]), __uint_as_float(w[2 * p + 1]));
    else return Pair<T>::get(*reinterpret_cast<const typename Pair<T>::Raw*>(&w[p]));
  }
  __device__ __forceinline__ void get(float (&v)[8]) const {
#pragma unroll
    for (int p = 0; p < 4; ++p) {
      const float2 f = pair(p);
      v[2 * p] = f.x;
      v[2 * p + 1] = f.y;
    }
  }
};
// Stores a thread's part of group j.
template <typename T, int kUnit>
__device__ __forceinline__ void put8(T* row, int j, int D, const float (&v)[8]) {
  if constexpr (kUnit == 8) {
    const int col = column(j);
    if (col < D) store8(row + col, v);
  } else {
#pragma unroll
    for (int e = 0; e < 8; e += kUnit) {
      const int col = column_of<kUnit>(j, e);
      if (col >= D) continue;
      if constexpr (kUnit == 2) *reinterpret_cast<typename Pair<T>::Raw*>(row + col) = Pair<T>::put(v[e], v[e + 1]);
      else row[col] = from_f32<T>(v[e]);
    }
  }
}
template <int kUnit>
__device__ __forceinline__ void weights8(const float* w, int j, int D, bool aligned, float (&v)[8]) {
  if (kUnit == 8 && aligned && column(j) < D) {
    load8(w + column(j), v);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = column_of<kUnit>(j, e) < D ? w[column_of<kUnit>(j, e)] : 0.0f;
  }
}

// What a 16-bit type T takes off a 32-bit sum: the distance of their bit patterns (both as fp32, magnitudes), at most half
// a unit of T in its last place.  So 16 + 16 bits give the sum back (a tie's half unit of bf16, and what rounds to a
// subnormal of fp16, up to the bound), and whatever the low part holds, the result is within its bound of the high part.
template <typename T>
constexpr int kMostLow = std::is_same_v<T, __half> ? 1 << 12 : (1 << 15) - 1;
template <typename T>
__device__ __forceinline__ float low_part(float s) {  // an integer, as the bits of a float
  const unsigned high = __float_as_uint(to_f32(from_f32<T>(s))) & 0x7fffffffu;
  const int d = (int)(__float_as_uint(s) & 0x7fffffffu) - (int)high;
  return __int_as_float(high < 0x7f800000u ? min(max(d, -kMostLow<T>), kMostLow<T>) : 0);
}
template <typename T>
__device__ __forceinline__ float with_low_part(float high, float low) {
  const unsigned bits = __float_as_uint(high), m = bits & 0x7fffffffu;
  const int d = min(max(__float_as_int(low), -kMostLow<T>), kMostLow<T>);
  return m < 0x7f800000u ? __uint_as_float((bits & 0x80000000u) | (unsigned)max((int)m + d, 0)) : high;
}

struct NormArgs {
  const void* x;
  long long x_pitch;
  const void* residual;
  long long residual_pitch;
  const float* weight;
  float eps;
  long long rows;
  int D;
  void* out;
  float* scales;
  int group, n_groups;  // columns per scale (0: no scales), scales per row
  void* sum_out;
  int16_t* sum_low;
  float* rstd;
  bool weight_vec;  // weight is 16-byte aligned
};

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// Sum over the threads of a row, the same bits in all of them.  `part`: one
// slot per warp of the row; every use of a `part` array has its own.  kMany:
// rows share a block (threadIdx.y) and each meet in a barrier of their own (with
// which a block takes all 16 of its barriers, and fewer blocks fit on an SM).
template <bool kMany>
__device__ __forceinline__ float row_sum(float v, float* part) {
  v = warp_sum(v);
  const int warps = blockDim.x >> 5;
  if (warps > 1) {
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = v;
    if (!kMany || blockDim.y == 1) __syncthreads();
    else asm volatile("bar.sync %0, %1;" ::"r"(threadIdx.y + 1), "r"(blockDim.x) : "memory");
    v = warp_sum((threadIdx.x & 31) < warps ? part[threadIdx.x & 31] : 0.0f);
  }
  return v;
}

// Largest bit pattern over the threads of a row: of |y| taken as an unsigned
// number, which orders finite values, infinity and NaN in this order.
__device__ __forceinline__ unsigned row_max(unsigned v, unsigned* part) {
  v = __reduce_max_sync(0xffffffffu, v);
  const int warps = blockDim.x >> 5;
  if (warps > 1) {
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = v;
    __syncthreads();
    v = __reduce_max_sync(0xffffffffu, (threadIdx.x & 31) < warps ? part[threadIdx.x & 31] : 0u);
  }
  return v;
}

__device__ __forceinline__ float scale_of(unsigned amax_bits) {
  if (amax_bits == 0u) return 1.0f;
  const float s = __uint_as_float(amax_bits) * (1.0f / kE4m3Max);
  return s < kMinScale ? kMinScale : s;  // NaN stays
}

__device__ __forceinline__ uint2 to_e4m3(const float (&y)[8], float scale) {
  const float inv = rcp_approx(scale);  // (a scale is at least 2^-126)
  unsigned w[2];
#pragma unroll
  for (int q = 0; q < 2; ++q) {
    const unsigned lo = __nv_cvt_float2_to_fp8x2(make_float2(y[4 * q] * inv, y[4 * q + 1] * inv), __NV_SATFINITE, __NV_E4M3);
    const unsigned hi =
        __nv_cvt_float2_to_fp8x2(make_float2(y[4 * q + 2] * inv, y[4 * q + 3] * inv), __NV_SATFINITE, __NV_E4M3);
    w[q] = lo | hi << 16;
  }
  return make_uint2(w[0], w[1]);
}

template <typename T, int VPT, int kMost, int kUnit, bool kQuant>
__global__ void __launch_bounds__(kMost, kMost == 512 && kUnit == 8 ? 3 : 1) rms_norm_kernel(const NormArgs a) {
  begin_op();
  __shared__ float part[32];
  __shared__ unsigned part_max[32];
  const long long row = (long long)blockIdx.x * blockDim.y + threadIdx.y;
  if (row >= a.rows) return;  // a whole warp (rows share a block only where a row is one warp)
  const T* x = static_cast<const T*>(a.x) + row * a.x_pitch;
  Raw8<T, kUnit> raw[VPT];
  float s[VPT][8];
#pragma unroll
  for (int j = 0; j < VPT; ++j) raw[j].load(x, j, a.D);
  if (a.residual) {
    const T* res = static_cast<const T*>(a.residual) + row * a.residual_pitch;
    Raw8<T, kUnit> more[VPT];
#pragma unroll
    for (int j = 0; j < VPT; ++j) more[j].load(res, j, a.D);
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
      float v[8];
      raw[j].get(s[j]);
      more[j].get(v);
#pragma unroll
      for (int e = 0; e < 8; ++e) s[j][e] += v[e];
    }
  } else {
#pragma unroll
    for (int j = 0; j < VPT; ++j) raw[j].get(s[j]);
  }
  float sum = 0.0f;
#pragma unroll
  for (int j = 0; j < VPT; ++j) {
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = s[j][e];
    to_neighbours<kUnit>(v);
#pragma unroll
    for (int e = 0; e < 8; ++e) sum = fmaf(v[e], v[e], sum);
  }
  if (a.sum_out) {
    T* so = static_cast<T*>(a.sum_out) + row * a.D;
#pragma unroll
    for (int j = 0; j < VPT; ++j) put8<T, kUnit>(so, j, a.D, s[j]);
  }
  if constexpr (sizeof(T) == 2 && !kQuant) {
    if (a.sum_low) {
#pragma unroll
      for (int j = 0; j < VPT; ++j) {
        float low[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) low[e] = low_part<T>(s[j][e]);
        put8<int16_t, kUnit>(a.sum_low + row * a.D, j, a.D, low);
      }
    }
  }
  sum = row_sum<false>(sum, part);
  const float rstd = rsqrtf(sum / (float)a.D + a.eps);
  if (a.rstd && threadIdx.x == 0) a.rstd[row] = rstd;
#pragma unroll
  for (int j = 0; j < VPT; ++j) {
    float w[8];
    weights8<kUnit>(a.weight, j, a.D, a.weight_vec, w);
#pragma unroll
    for (int e = 0; e < 8; ++e) s[j][e] = s[j][e] * rstd * w[e];
    if (kQuant) to_neighbours<kUnit>(s[j]);
  }
  if constexpr (!kQuant) {
    T* out = static_cast<T*>(a.out) + row * a.D;
#pragma unroll
    for (int j = 0; j < VPT; ++j) put8<T, kUnit>(out, j, a.D, s[j]);
  } else {
    // the largest |y| of each group: a group of 32 to 256 columns is 4 to 32
    // neighbouring lanes (blockDim.x is a multiple of 32), a longer one the row
    unsigned m[VPT];
    const bool whole = a.group >= a.D;
    unsigned all = 0u;
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
      m[j] = 0u;
#pragma unroll
      for (int e = 0; e < 8; ++e)  // (a column past D: zero times an rstd that may not be finite)
        if (column(j) + e < a.D) m[j] = max(m[j], __float_as_uint(s[j][e]) & 0x7fffffffu);
      all = max(all, m[j]);
    }
    if (whole) {
      all = row_max(all, part_max);
#pragma unroll
      for (int j = 0; j < VPT; ++j) m[j] = all;
    } else {
#pragma unroll
      for (int j = 0; j < VPT; ++j) {
        for (int o = 1; o < a.group / 8; o <<= 1) m[j] = max(m[j], __shfl_xor_sync(0xffffffffu, m[j], o));
      }
    }
    uint8_t* out = static_cast<uint8_t*>(a.out) + row * a.D;
    float* scales = a.scales + row * a.n_groups;
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
      const int col = column(j);
      if (col < a.D) {
        const float scale = scale_of(m[j]);
        const uint2 q = to_e4m3(s[j], scale);
        if (kUnit == 8) {
          *reinterpret_cast<uint2*>(out + col) = q;
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (col + e < a.D) out[col + e] = (uint8_t)((e < 4 ? q.x >> (8 * e) : q.y >> (8 * (e - 4))) & 255u);
        }
        if (whole ? col == 0 : col % a.group == 0) scales[whole ? 0 : col / a.group] = scale;
      }
    }
  }
}

constexpr int kMaxRows = 8;  // of a block

struct NormBackwardArgs {
  const void* dy;
  long long dy_pitch;
  const void* s;
  long long s_pitch;
  const int16_t* s_low;
  const float* weight;
  const float* rstd;
  const void* dsum;
  long long dsum_pitch;
  long long rows;
  int D;
  void* dx;
  float* partial;  // [gridDim.x][pitch_of_partial(D)]: each block's sum of dy s rstd over its rows; or null
  bool weight_vec;
};
__host__ __device__ constexpr int pitch_of_partial(int D) { return (D + 7) / 8 * 8; }

// A block's rows go on by all blocks' rows; the next one's values are on their way while this one's sum is formed,
// except of the widest rows, of which one alone keeps an SM's loads busy.
// kLow: s comes with the low parts of sum_out.
template <typename T, int VPT, int kMost, int kUnit, bool kLow>
__global__ void __launch_bounds__(kMost, 1) rms_norm_backward_kernel(const NormBackwardArgs a) {
  begin_op();
  constexpr bool kAhead = VPT * sizeof(T) < 8;  // else a thread's registers do not hold the next row's values too
  __shared__ float part[2][kMaxRows][32];
  extern __shared__ __align__(16) float merged[];  // [rows of the block][pitch] where there are several
  float w[VPT][8], dw[VPT][8];
#pragma unroll
  for (int j = 0; j < VPT; ++j) {
    weights8<kUnit>(a.weight, j, a.D, a.weight_vec, w[j]);
#pragma unroll
    for (int e = 0; e < 8; ++e) dw[j][e] = 0.0f;
  }
  const long long step = (long long)gridDim.x * blockDim.y;
  long long row = (long long)blockIdx.x * blockDim.y + threadIdx.y;
  Raw8<T, kUnit> raw_g[VPT], raw_s[VPT], raw_d[VPT];
  Raw8<int16_t, kUnit> raw_low[kLow ? VPT : 1];
  float rstd = 0.0f;
  auto load = [&](long long row) {
    const T* dy = static_cast<const T*>(a.dy) + row * a.dy_pitch;
    const T* s = static_cast<const T*>(a.s) + row * a.s_pitch;
#pragma unroll
    for (int j = 0; j < VPT; ++j) raw_g[j].load(dy, j, a.D), raw_s[j].load(s, j, a.D);
    if constexpr (kLow) {
#pragma unroll
      for (int j = 0; j < VPT; ++j) raw_low[j].load(a.s_low + row * a.D, j, a.D);
    }
    if (a.dsum) {
      const T* ds = static_cast<const T*>(a.dsum) + row * a.dsum_pitch;
#pragma unroll
      for (int j = 0; j < VPT; ++j) raw_d[j].load(ds, j, a.D);
    }
    rstd = a.rstd[row];
  };
  if (kAhead && row < a.rows) load(row);
  int turn = 0;
  for (; row < a.rows; row += step) {
    float g[VPT][8], v[VPT][8], r[VPT][8];
    float sum = 0.0f;
    if (!kAhead) load(row);
    const float scale = rstd;
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
      raw_g[j].get(g[j]);
      raw_s[j].get(v[j]);
      if constexpr (kLow) {
        float low[8];
        raw_low[j].get(low);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[j][e] = with_low_part<T>(v[j][e], low[e]);
      }
      if (a.dsum) raw_d[j].get(r[j]);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        if (!a.dsum) r[j][e] = 0.0f;
        v[j][e] *= scale;
        dw[j][e] = fmaf(g[j][e], v[j][e], dw[j][e]);
        g[j][e] *= w[j][e];
        sum = fmaf(g[j][e], v[j][e], sum);
      }
    }
    if (kAhead && row + step < a.rows) load(row + step);
    sum = row_sum<true>(sum, part[turn][threadIdx.y]);
    turn ^= 1;  // the next row's sums may be written while slow threads still read this row's
    const float mean = sum / (float)a.D;
    T* dx = static_cast<T*>(a.dx) + row * a.D;
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
#pragma unroll
      for (int e = 0; e < 8; ++e) r[j][e] = fmaf(scale, g[j][e] - v[j][e] * mean, r[j][e]);
      put8<T, kUnit>(dx, j, a.D, r[j]);
    }
  }
  if (a.partial) {
    const int pitch = pitch_of_partial(a.D);
    float* p = a.partial + (long long)blockIdx.x * pitch;
    float* to = blockDim.y == 1 ? p : merged + threadIdx.y * pitch;
#pragma unroll
    for (int j = 0; j < VPT; ++j) put8<float, kUnit>(to, j, pitch, dw[j]);
    if (blockDim.y > 1) {  // the block's rows, in their order
      __syncthreads();
      for (int col = threadIdx.y * blockDim.x + threadIdx.x; col < a.D; col += blockDim.x * blockDim.y) {
        float v = 0.0f;
        for (int y = 0; y < (int)blockDim.y; ++y) v += merged[y * pitch + col];
        p[col] = v;
      }
    }
  }
}

// Column sums of partial [n][pitch_of_partial(D)], in a fixed order: kColumns columns to a block, 1024 / kColumns rows at a
// time.  8 columns up to 2048 of them, so that the few blocks have few loads one behind the other, else 32 (backward pass
// of 20000 x 512 bf16 19.1 us with 8, 20.0 with 32; of 3000 x 8192 bf16 41.9 and 38.0).
template <int kColumns>
__global__ void __launch_bounds__(1024) column_sum_kernel(const float* partial, int n, int D, float* out) {
  begin_op();
  constexpr int kRows = 1024 / kColumns;
  __shared__ float acc[kRows][kColumns + 1];
  const int col = blockIdx.x * kColumns + threadIdx.x;
  float v = 0.0f;
  if (col < D)
#pragma unroll 8
    for (int k = threadIdx.y; k < n; k += kRows) v += partial[(long long)k * pitch_of_partial(D) + col];
  acc[threadIdx.y][threadIdx.x] = v;
  __syncthreads();
  const int t = threadIdx.y * kColumns + threadIdx.x, c = t >> 5, lane = t & 31;  // a warp to a column
  if (c >= kColumns) return;
  v = 0.0f;
#pragma unroll
  for (int k = 0; k < kRows; k += 32) v += acc[k + lane][c];
  v = warp_sum(v);
  if (lane == 0 && blockIdx.x * kColumns + c < D) out[blockIdx.x * kColumns + c] = v;
}

// Threads of a row and the groups of 8 columns of each.
struct RowShape {
  int threads, vpt, rows_per_block;
};
// 16-bit values in 16-byte accesses: two groups to a thread above 256 columns and four above 4096 (at 8192 x 4096, 512
// threads with one group took 50 us, 256 with two 44); else two only where one would take more than 512 threads.
RowShape row_shape(int D, bool wide) {
  const int n = (D + 7) / 8;
  RowShape r;
  r.vpt = n > 2048 ? 4 : (n > 512 ? (wide && n <= 1024 ? 4 : 2) : (wide && n > 32 ? 2 : 1));
  r.threads = ((n + r.vpt - 1) / r.vpt + 31) / 32 * 32;
  r.rows_per_block = r.threads == 32 ? 4 : 1;
  return r;
}

// The same backward, where a thread holds three tensors' columns and those of the next row: two groups above 256 of them
// (16-byte accesses: from 128 on), in 32 bits above 768 (with two groups of 32-bit values 3000 x 5001 took 54 us, with one 47).  Blocks of up to 256 threads, of as many rows as fit, and as many blocks as are on
// the GPU at once.
RowShape backward_shape(int D, size_t es, bool wide) {
  RowShape r;
  const int n = (D + 7) / 8;
  r.vpt = n > 2048 ? 4 : (n > (es == 4 ? 768 : 256) || (wide && n >= 128) ? 2 : 1);
  r.threads = ((n + r.vpt - 1) / r.vpt + 31) / 32 * 32;
  r.rows_per_block = std::max(1, 256 / r.threads);
  return r;
}
int backward_blocks(long long rows, const RowShape& r) {
  const int per_sm = std::max(1, (r.vpt == 1 ? 768 : 512) / (r.threads * r.rows_per_block));
  return (int)std::min<long long>((rows + r.rows_per_block - 1) / r.rows_per_block, per_sm * 152);
}

// Values of an access (see the top): every pointer a multiple of it and every pitch.
struct Access {
  const void* p;
  long long pitch;
};
int unit_of(int D, size_t es, std::initializer_list<Access> all) {
  auto fits = [&](size_t bytes) {
    for (const Access& a : all)
      if (a.p && (!op_aligned(a.p, bytes) || a.pitch * es % bytes != 0)) return false;
    return D * es % bytes == 0;
  };
  return D % 8 == 0 && fits(16) ? 8 : (es == 2 && fits(4) ? 2 : 1);
}

// f(groups of 8 columns to a thread, most threads of the kernel) for a row's shape.
template <typename F>
cudaError_t with_shape(const RowShape& r, F f) {
  using std::integral_constant;
  if (r.vpt == 1) return f(integral_constant<int, 1>(), integral_constant<int, 512>());
  if (r.vpt == 2 && r.threads <= 512) return f(integral_constant<int, 2>(), integral_constant<int, 512>());
  if (r.vpt == 2) return f(integral_constant<int, 2>(), integral_constant<int, 1024>());
  if (r.threads <= 256) return f(integral_constant<int, 4>(), integral_constant<int, 256>());
  return f(integral_constant<int, 4>(), integral_constant<int, 1024>());
}

// The same for the backward kernel's shapes.
template <typename F>
cudaError_t with_backward_shape(const RowShape& r, F f) {
  using std::integral_constant;
  if (r.vpt == 1) return f(integral_constant<int, 1>(), integral_constant<int, 768>());
  if (r.vpt == 2 && r.threads <= 512) return f(integral_constant<int, 2>(), integral_constant<int, 512>());
  if (r.vpt == 2) return f(integral_constant<int, 2>(), integral_constant<int, 1024>());
  return f(integral_constant<int, 4>(), integral_constant<int, 1024>());
}

}  // namespace
}  // namespace lstm_approx_impl

using namespace lstm_approx_impl;

extern "C" int lstm_approx_rms_norm(int dtype, int group, const void* x, long long x_pitch, const void* residual,
                                    long long residual_pitch, const float* weight, float eps, long long rows, int D,
                                    void* out, float* scales, void* sum_out, short* sum_low, float* rstd,
                                    void* cuda_stream, char* msg, int msg_len) {
  if (msg && msg_len > 0) msg[0] = '\0';
  if (!op_float_dtype(dtype)) return op_report(msg, msg_len, LSTM_APPROX_EINVAL, "dtype %d", dtype);
  if (rows < 0 || rows > 0x7fffffffll || D < 1 || D > kMaxD)
    return op_report(msg, msg_len, LSTM_APPROX_EINVAL, "need 0 <= rows < 2^31 and 1 <= D <= %d", kMaxD);
  if (group < 0 || (group > 0 && group < D && group != 32 && group != 64 && group != 128 && group != 256))
    return op_report(msg, msg_len, LSTM_APPROX_EINVAL, "group must be 0, 32, 64, 128, 256 or >= D, not %d", group);
  if (!(eps >= 0.0f)) return op_report(msg, msg_len, LSTM_APPROX_EINVAL, "eps must not be negative");
  if (sum_low && (dtype == LSTM_APPROX_OP_FP32 || group > 0))
    return op_report(msg, msg_len, LSTM_APPROX_EINVAL, "sum_low is for 16-bit types, and not for 8-bit output");
  if (rows > 0 && (!x || !weight || !out || (group > 0) != (scales != nullptr)))
    return op_report(msg, msg_len, LSTM_APPROX_EINVAL,
                     "x, weight and out must not be NULL; scales are given for 8-bit output only");
  const size_t es = op_dtype_bytes(dtype);
  if (x_pitch < 0 || residual_pitch < 0 || !op_aligned(x, es) || !op_aligned(residual, es) || !op_aligned(sum_out, es) ||
      !op_aligned(weight, 4) || !op_aligned(scales, 4) || !op_aligned(sum_low, 2) || !op_aligned(rstd, 4) ||
      (group == 0 && !op_aligned(out, es)))
    return op_report(msg, msg_len, LSTM_APPROX_EINVAL, "a negative pitch, or a pointer not aligned to its type");
  if (int rc = op_check_device(msg, msg_len)) return rc;
  if (rows == 0) return LSTM_APPROX_OK;
  NormArgs a{x, x_pitch, residual, residual_pitch, weight, eps, rows, D, out, scales, group, 0, sum_out, sum_low, rstd,
             false};
  a.n_groups = group > 0 ? (group >= D ? 1 : (D + group - 1) / group) : 0;
  int unit = unit_of(D, es, {{x, x_pitch}, {residual, residual_pitch}, {sum_out, D}, {sum_low, D},
                        {group > 0 ? nullptr : out, D}});
  if (unit == 8 && group > 0 && !op_aligned(out, 8)) unit = 1;
  a.weight_vec = op_aligned(weight, 16);
  const RowShape r = row_shape(D, unit == 8 && es == 2);
  const dim3 grid((unsigned)((rows + r.rows_per_block - 1) / r.rows_per_block)), block(r.threads, r.rows_per_block);
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  const cudaError_t e = op_for_type(dtype, [&](auto* t) {
    using T = std::remove_pointer_t<decltype(t)>;
    return with_shape(r, [&](auto vpt, auto most) {
      constexpr int V = decltype(vpt)::value, M = decltype(most)::value;
      if constexpr (sizeof(T) == 2)
        if (unit == 2)
          return op_launch(group > 0 ? rms_norm_kernel<T, V, M, 2, true> : rms_norm_kernel<T, V, M, 2, false>, grid, block,
                           0, s, a);
      if (unit == 8)
        return op_launch(group > 0 ? rms_norm_kernel<T, V, M, 8, true> : rms_norm_kernel<T, V, M, 8, false>, grid, block, 0,
                         s, a);
      return op_launch(group > 0 ? rms_norm_kernel<T, V, M, 1, true> : rms_norm_kernel<T, V, M, 1, false>, grid, block, 0, s,
                       a);
    });
  });
  return op_launched(e, "norm launch", msg, msg_len);
}

extern "C" size_t lstm_approx_rms_norm_workspace_bytes(long long rows, int D) {
  if (rows < 0 || rows > 0x7fffffffll || D < 1 || D > kMaxD) return 0;
  size_t parts = 0;  // of any of the shapes
  for (const RowShape& r : {backward_shape(D, 4, false), backward_shape(D, 2, false), backward_shape(D, 2, true)})
    parts = std::max(parts, (size_t)backward_blocks(rows, r));
  return parts * pitch_of_partial(D) * sizeof(float) + 16;
}

extern "C" int lstm_approx_rms_norm_backward(int dtype, const void* dy, long long dy_pitch, const void* s,
                                             long long s_pitch, const short* s_low, const float* weight, const float* rstd,
                                             const void* dsum, long long dsum_pitch, long long rows, int D, void* dx,
                                             float* dweight, void* workspace, size_t workspace_bytes,
                                             void* cuda_stream, char* msg, int msg_len) {
  if (msg && msg_len > 0) msg[0] = '\0';
  if (!op_float_dtype(dtype)) return op_report(msg, msg_len, LSTM_APPROX_EINVAL, "dtype %d", dtype);
  if (s_low && dtype == LSTM_APPROX_OP_FP32)
    return op_report(msg, msg_len, LSTM_APPROX_EINVAL, "s_low is for 16-bit types");
  if (rows < 0 || rows > 0x7fffffffll || D < 1 || D > kMaxD)
    return op_report(msg, msg_len, LSTM_APPROX_EINVAL, "need 0 <= rows < 2^31 and 1 <= D <= %d", kMaxD);
  if (rows > 0 && (!dy || !s || !weight || !rstd || !dx))
    return op_report(msg, msg_len, LSTM_APPROX_EINVAL, "dy, s, weight, rstd and dx must not be NULL");
  const size_t es = op_dtype_bytes(dtype);
  if (dy_pitch < 0 || s_pitch < 0 || dsum_pitch < 0 || !op_aligned(dy, es) || !op_aligned(s, es) ||
      !op_aligned(s_low, 2) || !op_aligned(dsum, es) || !op_aligned(dx, es) || !op_aligned(weight, 4) || !op_aligned(rstd, 4) ||
      !op_aligned(dweight, 4))
    return op_report(msg, msg_len, LSTM_APPROX_EINVAL, "a negative pitch, or a pointer not aligned to its type");
  const size_t need = lstm_approx_rms_norm_workspace_bytes(rows, D);
  if (dweight && (!workspace || !op_aligned(workspace, 16) || workspace_bytes < need))
    return op_report(msg, msg_len, LSTM_APPROX_EINVAL, "dweight needs a 16-byte aligned workspace of %zu bytes", need);
  if (int rc = op_check_device(msg, msg_len)) return rc;
  const int unit = unit_of(D, es, {{dy, dy_pitch}, {s, s_pitch}, {s_low, D}, {dsum, dsum_pitch}, {dx, D}});
  const RowShape r = backward_shape(D, es, unit == 8 && es == 2);
  const int blocks = backward_blocks(rows, r);
  const size_t smem = r.rows_per_block > 1 ? (size_t)r.rows_per_block * pitch_of_partial(D) * sizeof(float) : 0;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  if (rows > 0) {
    NormBackwardArgs a{dy, dy_pitch, s, s_pitch, s_low, weight, rstd, dsum, dsum_pitch, rows, D, dx,
                       dweight ? static_cast<float*>(workspace) : nullptr, op_aligned(weight, 16)};
    const cudaError_t e = op_for_type(dtype, [&](auto* t) {
      using T = std::remove_pointer_t<decltype(t)>;
      return with_backward_shape(r, [&](auto vpt, auto most) {
        constexpr int V = decltype(vpt)::value, M = decltype(most)::value;
        const dim3 block(r.threads, r.rows_per_block);
        auto run = [&](auto low) {
          constexpr bool kLow = decltype(low)::value;
          auto kern = unit == 8 ? rms_norm_backward_kernel<T, V, M, 8, kLow> : rms_norm_backward_kernel<T, V, M, 1, kLow>;
          if constexpr (sizeof(T) == 2)
            if (unit == 2) kern = rms_norm_backward_kernel<T, V, M, 2, kLow>;
          return op_launch(kern, dim3(blocks), block, smem, st, a);
        };
        if constexpr (sizeof(T) == 2)
          if (s_low) return run(std::true_type());
        return run(std::false_type());
      });
    });
    if (int rc = op_launched(e, "norm backward launch", msg, msg_len)) return rc;
  }
  if (!dweight) return LSTM_APPROX_OK;
  const int columns = D <= 2048 ? 8 : 32;
  const cudaError_t e = op_launch(columns == 8 ? column_sum_kernel<8> : column_sum_kernel<32>, dim3((D + columns - 1) / columns),
                                  dim3(columns, 1024 / columns), 0, st, static_cast<const float*>(workspace), blocks, D, dweight);
  return op_launched(e, "weight gradient launch", msg, msg_len);
}
