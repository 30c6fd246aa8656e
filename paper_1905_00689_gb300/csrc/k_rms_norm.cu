// Root-mean-square norm with the residual's addition, its 8-bit output with
// scales, and its gradients (include/lstm_approx_ops.h).
//
// Forward, per row:   s = x + residual; rstd = (mean s^2 + eps)^-1/2; y = s rstd w
// Backward, per row:  ds = rstd (w dy - s rstd^2 mean(w dy s)) + dsum
//            columns: dw = sum over rows of dy s rstd
//
// Bound by memory: a row is read once, kept in registers as fp32 while its
// sum is formed, and written once.  A thread holds VPT groups of 8
// neighbouring columns (16-byte accesses where the addresses allow them),
// `blockDim.x` threads share a row, and rows of at most 32 threads share a
// block (no block-wide sum then).
#include <cuda_fp8.h>

#include <algorithm>

#include "ops_common.cuh"

namespace lstm_approx_impl {
namespace {

constexpr int kMaxD = 32768;
constexpr float kE4m3Max = 448.0f;
constexpr float kMinScale = 1.17549435e-38f;  // 2^-126

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
  float* rstd;
};

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// Sum over the threads of a row, the same bits in all of them.  `part`: one
// slot per warp; every use of a `part` array has its own.
__device__ __forceinline__ float row_sum(float v, float* part) {
  v = warp_sum(v);
  const int warps = blockDim.x >> 5;
  if (warps > 1) {
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = v;
    __syncthreads();
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
  const float s = __uint_as_float(amax_bits) / kE4m3Max;
  return s < kMinScale ? kMinScale : s;  // NaN stays
}

__device__ __forceinline__ uint2 to_e4m3(const float (&y)[8], float scale) {
  const float inv = 1.0f / scale;
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

template <typename T, int VPT, bool kVec, bool kQuant>
__global__ void __launch_bounds__(1024) rms_norm_kernel(const NormArgs a) {
  __shared__ float part[32];
  __shared__ unsigned part_max[32];
  const long long row = (long long)blockIdx.x * blockDim.y + threadIdx.y;
  if (row >= a.rows) return;  // a whole warp (rows share a block only where a row is one warp)
  const T* x = static_cast<const T*>(a.x) + row * a.x_pitch;
  const T* res = a.residual ? static_cast<const T*>(a.residual) + row * a.residual_pitch : nullptr;
  float s[VPT][8];
  float sum = 0.0f;
#pragma unroll
  for (int j = 0; j < VPT; ++j) {
    const int col = 8 * (threadIdx.x + j * blockDim.x);
#pragma unroll
    for (int e = 0; e < 8; ++e) s[j][e] = 0.0f;
    if (col < a.D) load8<T, kVec>(x + col, a.D - col, s[j]);
  }
  if (res) {
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
      const int col = 8 * (threadIdx.x + j * blockDim.x);
      if (col < a.D) {
        float v[8];
        load8<T, kVec>(res + col, a.D - col, v);
#pragma unroll
        for (int e = 0; e < 8; ++e) s[j][e] += v[e];
      }
    }
  }
#pragma unroll
  for (int j = 0; j < VPT; ++j) {
#pragma unroll
    for (int e = 0; e < 8; ++e) sum = fmaf(s[j][e], s[j][e], sum);
  }
  if (a.sum_out) {
    T* so = static_cast<T*>(a.sum_out) + row * a.D;
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
      const int col = 8 * (threadIdx.x + j * blockDim.x);
      if (col < a.D) store8<T, kVec>(so + col, a.D - col, s[j]);
    }
  }
  sum = row_sum(sum, part);
  const float rstd = rsqrtf(sum / (float)a.D + a.eps);
  if (a.rstd && threadIdx.x == 0) a.rstd[row] = rstd;
#pragma unroll
  for (int j = 0; j < VPT; ++j) {
    const int col = 8 * (threadIdx.x + j * blockDim.x);
    if (col < a.D) {
      float w[8];
      load8<float, kVec>(a.weight + col, a.D - col, w);
#pragma unroll
      for (int e = 0; e < 8; ++e) s[j][e] = s[j][e] * rstd * w[e];
    }
  }
  if constexpr (!kQuant) {
    T* out = static_cast<T*>(a.out) + row * a.D;
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
      const int col = 8 * (threadIdx.x + j * blockDim.x);
      if (col < a.D) store8<T, kVec>(out + col, a.D - col, s[j]);
    }
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
      for (int e = 0; e < 8; ++e) m[j] = max(m[j], __float_as_uint(s[j][e]) & 0x7fffffffu);
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
      const int col = 8 * (threadIdx.x + j * blockDim.x);
      if (col < a.D) {
        const float scale = scale_of(m[j]);
        const uint2 q = to_e4m3(s[j], scale);
        if constexpr (kVec) {
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

struct NormBackwardArgs {
  const void* dy;
  long long dy_pitch;
  const void* s;
  long long s_pitch;
  const float* weight;
  const float* rstd;
  const void* dsum;
  long long dsum_pitch;
  long long rows;
  int D;
  void* dx;
  float* partial;  // [gridDim.x * blockDim.y][D]: sums of dy s rstd over the rows of each block row; or null
};

template <typename T, int VPT, bool kVec>
__global__ void __launch_bounds__(1024) rms_norm_backward_kernel(const NormBackwardArgs a) {
  __shared__ float part[2][32];
  float w[VPT][8], dw[VPT][8];
#pragma unroll
  for (int j = 0; j < VPT; ++j) {
    const int col = 8 * (threadIdx.x + j * blockDim.x);
#pragma unroll
    for (int e = 0; e < 8; ++e) w[j][e] = dw[j][e] = 0.0f;
    if (col < a.D) load8<float, kVec>(a.weight + col, a.D - col, w[j]);
  }
  const long long step = (long long)gridDim.x * blockDim.y;
  int turn = 0;
  for (long long row = (long long)blockIdx.x * blockDim.y + threadIdx.y; row < a.rows; row += step) {
    const T* dy = static_cast<const T*>(a.dy) + row * a.dy_pitch;
    const T* s = static_cast<const T*>(a.s) + row * a.s_pitch;
    const T* ds = a.dsum ? static_cast<const T*>(a.dsum) + row * a.dsum_pitch : nullptr;
    const float rstd = a.rstd[row];
    float g[VPT][8], v[VPT][8];
    float sum = 0.0f;
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
      const int col = 8 * (threadIdx.x + j * blockDim.x);
#pragma unroll
      for (int e = 0; e < 8; ++e) g[j][e] = v[j][e] = 0.0f;
      if (col < a.D) {
        load8<T, kVec>(dy + col, a.D - col, g[j]);
        load8<T, kVec>(s + col, a.D - col, v[j]);
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        v[j][e] *= rstd;
        dw[j][e] = fmaf(g[j][e], v[j][e], dw[j][e]);
        g[j][e] *= w[j][e];
        sum = fmaf(g[j][e], v[j][e], sum);
      }
    }
    sum = row_sum(sum, part[turn]);
    turn ^= 1;  // the next row's sums may be written while slow threads still read this row's
    const float mean = sum / (float)a.D;
    T* dx = static_cast<T*>(a.dx) + row * a.D;
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
      const int col = 8 * (threadIdx.x + j * blockDim.x);
      if (col < a.D) {
        float r[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) r[e] = 0.0f;
        if (ds) load8<T, kVec>(ds + col, a.D - col, r);
#pragma unroll
        for (int e = 0; e < 8; ++e) r[e] = fmaf(rstd, g[j][e] - v[j][e] * mean, r[e]);
        store8<T, kVec>(dx + col, a.D - col, r);
      }
    }
  }
  if (a.partial) {
    float* p = a.partial + ((long long)blockIdx.x * blockDim.y + threadIdx.y) * a.D;
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
      const int col = 8 * (threadIdx.x + j * blockDim.x);
      if (col < a.D) store8<float, kVec>(p + col, a.D - col, dw[j]);
    }
  }
}

// Column sums of partial [n][D], in a fixed order.
__global__ void __launch_bounds__(1024) column_sum_kernel(const float* partial, int n, int D, float* out) {
  __shared__ float acc[32][33];
  const int col = blockIdx.x * 32 + threadIdx.x;
  float v = 0.0f;
  if (col < D)
    for (int k = threadIdx.y; k < n; k += 32) v += partial[(long long)k * D + col];
  acc[threadIdx.y][threadIdx.x] = v;
  __syncthreads();
  v = warp_sum(acc[threadIdx.x][threadIdx.y]);
  const int c = blockIdx.x * 32 + threadIdx.y;
  if (threadIdx.x == 0 && c < D) out[c] = v;
}

// Threads of a row and the groups of 8 columns of each.
struct RowShape {
  int threads, vpt, rows_per_block;
};
RowShape row_shape(int D) {
  const int n = (D + 7) / 8;
  RowShape r;
  r.vpt = n > 2048 ? 4 : (n > 512 ? 2 : 1);
  r.threads = ((n + r.vpt - 1) / r.vpt + 31) / 32 * 32;
  r.rows_per_block = r.threads == 32 ? 4 : 1;
  return r;
}

int backward_blocks(long long rows, const RowShape& r) {
  const int per = std::max(1, 1024 / (r.threads * r.rows_per_block));
  const long long need = (rows + r.rows_per_block - 1) / r.rows_per_block;
  return (int)std::min<long long>(need, 152ll * per);
}

}  // namespace
}  // namespace lstm_approx_impl

using namespace lstm_approx_impl;

extern "C" int lstm_approx_rms_norm(int dtype, int group, const void* x, long long x_pitch, const void* residual,
                                    long long residual_pitch, const float* weight, float eps, long long rows, int D,
                                    void* out, float* scales, void* sum_out, float* rstd, void* cuda_stream, char* msg,
                                    int msg_len) {
  if (msg && msg_len > 0) msg[0] = '\0';
  if (!op_float_dtype(dtype)) return op_report(msg, msg_len, LSTM_APPROX_EINVAL, "dtype %d", dtype);
  if (rows < 0 || rows > 0x7fffffffll || D < 1 || D > kMaxD)
    return op_report(msg, msg_len, LSTM_APPROX_EINVAL, "need 0 <= rows < 2^31 and 1 <= D <= %d", kMaxD);
  if (group < 0 || (group > 0 && group < D && group != 32 && group != 64 && group != 128 && group != 256))
    return op_report(msg, msg_len, LSTM_APPROX_EINVAL, "group must be 0, 32, 64, 128, 256 or >= D, not %d", group);
  if (!(eps >= 0.0f)) return op_report(msg, msg_len, LSTM_APPROX_EINVAL, "eps must not be negative");
  if (rows > 0 && (!x || !weight || !out || (group > 0) != (scales != nullptr)))
    return op_report(msg, msg_len, LSTM_APPROX_EINVAL,
                     "x, weight and out must not be NULL; scales are given for 8-bit output only");
  const size_t es = op_dtype_bytes(dtype);
  if (x_pitch < 0 || residual_pitch < 0 || !op_aligned(x, es) || !op_aligned(residual, es) || !op_aligned(sum_out, es) ||
      !op_aligned(weight, 4) || !op_aligned(scales, 4) || !op_aligned(rstd, 4) || (group == 0 && !op_aligned(out, es)))
    return op_report(msg, msg_len, LSTM_APPROX_EINVAL, "a negative pitch, or a pointer not aligned to its type");
  if (int rc = op_check_device(msg, msg_len)) return rc;
  if (rows == 0) return LSTM_APPROX_OK;
  NormArgs a{x, x_pitch, residual, residual_pitch, weight, eps, rows, D, out, scales, group, 0, sum_out, rstd};
  a.n_groups = group > 0 ? (group >= D ? 1 : (D + group - 1) / group) : 0;
  const bool vec = D % 8 == 0 && op_aligned(x, 16) && op_aligned(residual, 16) && op_aligned(weight, 16) &&
                   op_aligned(sum_out, 16) && op_aligned(out, group > 0 ? 8 : 16) && x_pitch * es % 16 == 0 &&
                   (!residual || residual_pitch * es % 16 == 0);
  const RowShape r = row_shape(D);
  const dim3 grid((unsigned)((rows + r.rows_per_block - 1) / r.rows_per_block)), block(r.threads, r.rows_per_block);
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  const cudaError_t e = op_for_type(dtype, [&](auto* t) {
    using T = std::remove_pointer_t<decltype(t)>;
    auto at = [&](auto vpt) {
      constexpr int V = decltype(vpt)::value;
      auto k = vec ? (group > 0 ? rms_norm_kernel<T, V, true, true> : rms_norm_kernel<T, V, true, false>)
                   : (group > 0 ? rms_norm_kernel<T, V, false, true> : rms_norm_kernel<T, V, false, false>);
      return op_launch(k, grid, block, 0, s, a);
    };
    if (r.vpt == 1) return at(std::integral_constant<int, 1>());
    if (r.vpt == 2) return at(std::integral_constant<int, 2>());
    return at(std::integral_constant<int, 4>());
  });
  return op_launched(e, "norm launch", msg, msg_len);
}

extern "C" size_t lstm_approx_rms_norm_workspace_bytes(long long rows, int D) {
  if (rows < 0 || rows > 0x7fffffffll || D < 1 || D > kMaxD) return 0;
  const RowShape r = row_shape(D);
  return ((size_t)backward_blocks(rows, r) * r.rows_per_block * D * sizeof(float) + 15) / 16 * 16 + 16;
}

extern "C" int lstm_approx_rms_norm_backward(int dtype, const void* dy, long long dy_pitch, const void* s,
                                             long long s_pitch, const float* weight, const float* rstd,
                                             const void* dsum, long long dsum_pitch, long long rows, int D, void* dx,
                                             float* dweight, void* workspace, size_t workspace_bytes,
                                             void* cuda_stream, char* msg, int msg_len) {
  if (msg && msg_len > 0) msg[0] = '\0';
  if (!op_float_dtype(dtype)) return op_report(msg, msg_len, LSTM_APPROX_EINVAL, "dtype %d", dtype);
  if (rows < 0 || rows > 0x7fffffffll || D < 1 || D > kMaxD)
    return op_report(msg, msg_len, LSTM_APPROX_EINVAL, "need 0 <= rows < 2^31 and 1 <= D <= %d", kMaxD);
  if (rows > 0 && (!dy || !s || !weight || !rstd || !dx))
    return op_report(msg, msg_len, LSTM_APPROX_EINVAL, "dy, s, weight, rstd and dx must not be NULL");
  const size_t es = op_dtype_bytes(dtype);
  if (dy_pitch < 0 || s_pitch < 0 || dsum_pitch < 0 || !op_aligned(dy, es) || !op_aligned(s, es) ||
      !op_aligned(dsum, es) || !op_aligned(dx, es) || !op_aligned(weight, 4) || !op_aligned(rstd, 4) ||
      !op_aligned(dweight, 4))
    return op_report(msg, msg_len, LSTM_APPROX_EINVAL, "a negative pitch, or a pointer not aligned to its type");
  const size_t need = lstm_approx_rms_norm_workspace_bytes(rows, D);
  if (dweight && (!workspace || !op_aligned(workspace, 16) || workspace_bytes < need))
    return op_report(msg, msg_len, LSTM_APPROX_EINVAL, "dweight needs a 16-byte aligned workspace of %zu bytes", need);
  if (int rc = op_check_device(msg, msg_len)) return rc;
  const RowShape r = row_shape(D);
  const int blocks = backward_blocks(rows, r);
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  if (rows > 0) {
    NormBackwardArgs a{dy, dy_pitch, s, s_pitch, weight, rstd, dsum, dsum_pitch, rows, D, dx,
                       dweight ? static_cast<float*>(workspace) : nullptr};
    const bool vec = D % 8 == 0 && op_aligned(dy, 16) && op_aligned(s, 16) && op_aligned(dsum, 16) &&
                     op_aligned(dx, 16) && op_aligned(weight, 16) && dy_pitch * es % 16 == 0 &&
                     s_pitch * es % 16 == 0 && (!dsum || dsum_pitch * es % 16 == 0);
    const cudaError_t e = op_for_type(dtype, [&](auto* t) {
      using T = std::remove_pointer_t<decltype(t)>;
      auto at = [&](auto vpt) {
        constexpr int V = decltype(vpt)::value;
        return op_launch(vec ? rms_norm_backward_kernel<T, V, true> : rms_norm_backward_kernel<T, V, false>,
                         dim3(blocks), dim3(r.threads, r.rows_per_block), 0, st, a);
      };
      if (r.vpt == 1) return at(std::integral_constant<int, 1>());
      if (r.vpt == 2) return at(std::integral_constant<int, 2>());
      return at(std::integral_constant<int, 4>());
    });
    if (int rc = op_launched(e, "norm backward launch", msg, msg_len)) return rc;
  }
  if (!dweight) return LSTM_APPROX_OK;
  const cudaError_t e = op_launch(column_sum_kernel, dim3((D + 31) / 32), dim3(32, 32), 0, st,
                                  static_cast<const float*>(workspace), blocks * r.rows_per_block, D, dweight);
  return op_launched(e, "weight gradient launch", msg, msg_len);
}
