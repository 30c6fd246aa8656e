// Matrix-vector products with 4-bit weights, a scale and a zero point per
// group of columns, and the quantiser that makes such weights
// (include/lstm_approx_ops.h):
//
//   y[m][n] = sum_g scale[n][g] sum_{k in g} (q[n][k] - zero[n][g]) x[m][k]
//
// Bound by memory: the 4-bit matrix is read once for up to kTokens rows of x.
#include <cuda_fp8.h>

#include <algorithm>

#include "ops_common.cuh"

namespace lstm_approx_impl {
namespace {

constexpr int kTokens = 4;

__device__ __forceinline__ float e4m3_to_f32(uint8_t v) {
  return __half2float(__half(__nv_cvt_fp8_to_halfraw(v, __NV_E4M3)));
}

struct W4Args {
  int x_dtype;
  const void* x;
  long long x_pitch;
  const float* x_scale;
  int x_group, x_groups;
  const uint8_t* q;
  long long q_pitch;
  const void* scale;
  int scale_dtype;
  const uint8_t* zero;
  const float* bias;
  int M, N, K, group, groups;
  void* y;
  int y_dtype;
};

__device__ __forceinline__ float load_any(const void* p, long long at, int dtype) {
  if (dtype == LSTM_APPROX_OP_FP32) return static_cast<const float*>(p)[at];
  if (dtype == LSTM_APPROX_OP_BF16) return __bfloat162float(static_cast<const __nv_bfloat16*>(p)[at]);
  if (dtype == LSTM_APPROX_OP_FP16) return __half2float(static_cast<const __half*>(p)[at]);
  return e4m3_to_f32(static_cast<const uint8_t*>(p)[at]);
}
__device__ __forceinline__ void store_any(void* p, long long at, int dtype, float v) {
  if (dtype == LSTM_APPROX_OP_FP32) static_cast<float*>(p)[at] = v;
  else if (dtype == LSTM_APPROX_OP_BF16) static_cast<__nv_bfloat16*>(p)[at] = __float2bfloat16_rn(v);
  else static_cast<__half*>(p)[at] = __float2half_rn(v);
}

// A warp per row of the matrix; a lane takes 8 neighbouring columns at a time.
__global__ void __launch_bounds__(256) w4_matvec_kernel(const W4Args a) {
  const int lane = threadIdx.x & 31;
  const int n = blockIdx.x * 8 + (threadIdx.x >> 5);
  if (n >= a.N) return;
  for (int m0 = blockIdx.y * kTokens; m0 < a.M; m0 += gridDim.y * kTokens) {
    float acc[kTokens] = {};
    for (int k0 = lane * 8; k0 < a.K; k0 += 256) {
      const unsigned w = *reinterpret_cast<const unsigned*>(a.q + (long long)n * a.q_pitch + k0 / 2);
      const long long g = (long long)n * a.groups + k0 / a.group;
      const float scale = load_any(a.scale, g, a.scale_dtype);
      const float zero = a.zero ? (float)(a.zero[g] & 15) : 8.0f;
#pragma unroll
      for (int j = 0; j < kTokens; ++j) {
        const int m = m0 + j;
        if (m < a.M) {
          float part = 0.0f;
          for (int e = 0; e < 8 && k0 + e < a.K; ++e)
            part = fmaf((float)(w >> (4 * e) & 15u) - zero, load_any(a.x, m * a.x_pitch + k0 + e, a.x_dtype), part);
          if (a.x_scale) part *= a.x_scale[(long long)m * a.x_groups + k0 / a.x_group];
          acc[j] = fmaf(part, scale, acc[j]);
        }
      }
    }
#pragma unroll
    for (int j = 0; j < kTokens; ++j) {
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) acc[j] += __shfl_xor_sync(0xffffffffu, acc[j], o);
      if (lane == 0 && m0 + j < a.M)
        store_any(a.y, (long long)(m0 + j) * a.N + n, a.y_dtype, acc[j] + (a.bias ? a.bias[n] : 0.0f));
    }
  }
}

struct W4QuantizeArgs {
  int dtype;
  const void* w;
  long long w_pitch;
  int N, K, group, groups;
  uint8_t* q;
  long long q_pitch;
  void* scale;
  int scale_dtype;
  uint8_t* zero;
};

__device__ __forceinline__ float round_to(float v, int dtype) {
  if (dtype == LSTM_APPROX_OP_BF16) return __bfloat162float(__float2bfloat16_rn(v));
  if (dtype == LSTM_APPROX_OP_FP16) return __half2float(__float2half_rn(v));
  return v;
}

// A warp per group of columns of one row; lane l packs columns 4 l .. 4 l + 3
// of the group (two bytes).  The last group's warp also clears the row's rest.
__global__ void __launch_bounds__(256) w4_quantize_kernel(const W4QuantizeArgs a) {
  const long long item = (long long)blockIdx.x * 8 + (threadIdx.x >> 5);
  if (item >= (long long)a.N * a.groups) return;
  const int lane = threadIdx.x & 31;
  const int n = (int)(item / a.groups), g = (int)(item % a.groups);
  const int k0 = g * a.group + 4 * lane, end = min(a.K, (g + 1) * a.group);
  float v[4];
  float lo = 0.0f, hi = 0.0f;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    v[e] = 4 * lane < a.group && k0 + e < end ? load_any(a.w, n * a.w_pitch + k0 + e, a.dtype) : 0.0f;
    lo = fminf(lo, v[e]);
    hi = fmaxf(hi, v[e]);
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    lo = fminf(lo, __shfl_xor_sync(0xffffffffu, lo, o));
    hi = fmaxf(hi, __shfl_xor_sync(0xffffffffu, hi, o));
  }
  float scale = round_to((hi - lo) / 15.0f, a.scale_dtype);
  if (scale == 0.0f) scale = 1.0f;
  const float zero = fminf(fmaxf(rintf(-lo / scale), 0.0f), 15.0f);
  unsigned w = 0;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const float q = fminf(fmaxf(rintf(v[e] / scale) + zero, 0.0f), 15.0f);
    if (k0 + e < end) w |= (unsigned)q << (4 * e);
  }
  uint8_t* row = a.q + (long long)n * a.q_pitch;
  if (4 * lane < a.group) {
    if (k0 < end || g == a.groups - 1) {  // bytes k0 / 2 and the next, inside the pitch
#pragma unroll
      for (int e = 0; e < 2; ++e)
        if (k0 / 2 + e < a.q_pitch) row[k0 / 2 + e] = (uint8_t)(w >> (8 * e));
    }
  }
  if (g == a.groups - 1)
    for (long long p = (long long)(g + 1) * a.group / 2 + lane; p < a.q_pitch; p += 32) row[p] = 0;
  if (lane == 0) {
    if (a.scale_dtype == LSTM_APPROX_OP_FP32) static_cast<float*>(a.scale)[item] = scale;
    else store_any(a.scale, item, a.scale_dtype, scale);
    a.zero[item] = (uint8_t)zero;
  }
}

int check_matrix(int N, int K, int group, const void* q, long long q_pitch, const void* scale, int scale_dtype,
                 char* msg, int msg_len) {
  if (N < 0 || K < 1 || K > 0x7fffff00)
    return op_report(msg, msg_len, LSTM_APPROX_EINVAL, "need N >= 0 and K >= 1");
  if (group != 32 && group != 64 && group != 128)
    return op_report(msg, msg_len, LSTM_APPROX_EINVAL, "group must be 32, 64 or 128, not %d", group);
  if (!op_float_dtype(scale_dtype)) return op_report(msg, msg_len, LSTM_APPROX_EINVAL, "scale_dtype %d", scale_dtype);
  if (N > 0 && (!q || !scale)) return op_report(msg, msg_len, LSTM_APPROX_EINVAL, "q and scale must not be NULL");
  if (!op_aligned(q, 16) || q_pitch % 16 != 0 || q_pitch < ((long long)K + 1) / 2)
    return op_report(msg, msg_len, LSTM_APPROX_EINVAL,
                     "q must be 16-byte aligned, its pitch a multiple of 16 and at least ceil(K / 2) bytes");
  if (!op_aligned(scale, op_dtype_bytes(scale_dtype)))
    return op_report(msg, msg_len, LSTM_APPROX_EINVAL, "scale is not aligned to its type");
  return LSTM_APPROX_OK;
}

}  // namespace
}  // namespace lstm_approx_impl

using namespace lstm_approx_impl;

extern "C" int lstm_approx_w4_quantize(int dtype, const void* w, long long w_pitch, int N, int K, int group,
                                       unsigned char* q, long long q_pitch, void* scale, int scale_dtype,
                                       unsigned char* zero, void* cuda_stream, char* msg, int msg_len) {
  if (msg && msg_len > 0) msg[0] = '\0';
  if (!op_float_dtype(dtype)) return op_report(msg, msg_len, LSTM_APPROX_EINVAL, "dtype %d", dtype);
  if (int rc = check_matrix(N, K, group, q, q_pitch, scale, scale_dtype, msg, msg_len)) return rc;
  if (N > 0 && (!w || !zero)) return op_report(msg, msg_len, LSTM_APPROX_EINVAL, "w and zero must not be NULL");
  if (w_pitch < 0 || !op_aligned(w, op_dtype_bytes(dtype)))
    return op_report(msg, msg_len, LSTM_APPROX_EINVAL, "a negative pitch, or w is not aligned to its type");
  const int groups = (K + group - 1) / group;
  if ((long long)N * groups > 8ll * 0x7fffffff) return op_report(msg, msg_len, LSTM_APPROX_EINVAL, "N K is too large");
  if (int rc = op_check_device(msg, msg_len)) return rc;
  if (N == 0) return LSTM_APPROX_OK;
  W4QuantizeArgs a{dtype, w, w_pitch, N, K, group, groups, q, q_pitch, scale, scale_dtype, zero};
  const long long items = (long long)N * groups;
  return op_launched(op_launch(w4_quantize_kernel, dim3((unsigned)((items + 7) / 8)), dim3(256), 0,
                               static_cast<cudaStream_t>(cuda_stream), a),
                     "quantiser launch", msg, msg_len);
}

extern "C" int lstm_approx_w4_matvec(int x_dtype, const void* x, long long x_pitch, const float* x_scale, int x_group,
                                     const unsigned char* q, long long q_pitch, const void* scale, int scale_dtype,
                                     const unsigned char* zero, const float* bias, int M, int N, int K, int group,
                                     void* y, int y_dtype, void* cuda_stream, char* msg, int msg_len) {
  if (msg && msg_len > 0) msg[0] = '\0';
  const bool x8 = x_dtype == LSTM_APPROX_OP_E4M3;
  if ((!op_float_dtype(x_dtype) && !x8) || !op_float_dtype(y_dtype))
    return op_report(msg, msg_len, LSTM_APPROX_EINVAL, "x_dtype %d, y_dtype %d", x_dtype, y_dtype);
  if (int rc = check_matrix(N, K, group, q, q_pitch, scale, scale_dtype, msg, msg_len)) return rc;
  if (M < 0) return op_report(msg, msg_len, LSTM_APPROX_EINVAL, "M must not be negative");
  if (M > 0 && N > 0 && (!x || !y || x8 != (x_scale != nullptr)))
    return op_report(msg, msg_len, LSTM_APPROX_EINVAL, "x and y must not be NULL; x_scale is given for 8-bit x only");
  if (x8 && x_group != 128 && x_group < K)
    return op_report(msg, msg_len, LSTM_APPROX_EINVAL, "x_group must be 128 or >= K, not %d", x_group);
  if (x_pitch < 0 || !op_aligned(x, op_dtype_bytes(x_dtype)) || !op_aligned(x_scale, 4) || !op_aligned(bias, 4) ||
      !op_aligned(y, op_dtype_bytes(y_dtype)))
    return op_report(msg, msg_len, LSTM_APPROX_EINVAL, "a negative pitch, or a pointer not aligned to its type");
  if (int rc = op_check_device(msg, msg_len)) return rc;
  if (M == 0 || N == 0) return LSTM_APPROX_OK;
  W4Args a{x_dtype, x, x_pitch, x_scale, x_group, x_group >= K || !x8 ? 1 : (K + 127) / 128, q, q_pitch, scale,
           scale_dtype, zero, bias, M, N, K, group, (K + group - 1) / group, y, y_dtype};
  const dim3 grid((N + 7) / 8, std::min((M + kTokens - 1) / kTokens, 65535));
  return op_launched(op_launch(w4_matvec_kernel, grid, dim3(256), 0, static_cast<cudaStream_t>(cuda_stream), a),
                     "matrix-vector launch", msg, msg_len);
}
