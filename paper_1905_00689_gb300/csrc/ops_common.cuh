// What the operators of include/lstm_approx_ops.h share: element types,
// argument reports, the device check.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <cstdarg>
#include <cstdint>
#include <cstdio>

#include "../../include/lstm_approx_ops.h"
#include "internal.h"
#include "ptx.cuh"

namespace lstm_approx_impl {

// Every kernel is launched before the one ahead of it in the stream has ended
// (op_launch) and begins with this: it waits for that end and lets the next
// kernel be set up.  Two kinds of kernel fetch inputs before it, which is sound
// where another kernel of the same call goes ahead: that one has waited for
// everything older, and does not write them.  (Small kernels back to back:
// 4.2 us each launched one after the other's end, so 1.7 to 2.6.)
__device__ __forceinline__ void begin_op() {
  lstm_approx_dev::griddep_wait();
  lstm_approx_dev::griddep_launch_dependents();
}

// ---- element types ----------------------------------------------------------

template <typename T>
__device__ __forceinline__ float to_f32(T v);
template <>
__device__ __forceinline__ float to_f32<float>(float v) { return v; }
template <>
__device__ __forceinline__ float to_f32<__nv_bfloat16>(__nv_bfloat16 v) { return __bfloat162float(v); }
template <>
__device__ __forceinline__ float to_f32<__half>(__half v) { return __half2float(v); }

template <typename T>
__device__ __forceinline__ T from_f32(float v);
template <>
__device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <>
__device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <>
__device__ __forceinline__ __half from_f32<__half>(float v) { return __float2half_rn(v); }

// Integers, carried as the bits of a float.
template <>
__device__ __forceinline__ float to_f32<int16_t>(int16_t v) { return __int_as_float(v); }
template <>
__device__ __forceinline__ int16_t from_f32<int16_t>(float v) { return (int16_t)__float_as_int(v); }

// Two neighbouring elements in one access.
template <typename T>
struct Pair;
template <>
struct Pair<float> {
  using Raw = float2;
  static __device__ __forceinline__ float2 get(Raw v) { return v; }
  static __device__ __forceinline__ Raw put(float a, float b) { return make_float2(a, b); }
};
template <>
struct Pair<__nv_bfloat16> {
  using Raw = __nv_bfloat162;
  static __device__ __forceinline__ float2 get(Raw v) { return __bfloat1622float2(v); }
  static __device__ __forceinline__ Raw put(float a, float b) { return __floats2bfloat162_rn(a, b); }
};
template <>
struct Pair<__half> {
  using Raw = __half2;
  static __device__ __forceinline__ float2 get(Raw v) { return __half22float2(v); }
  static __device__ __forceinline__ Raw put(float a, float b) { return __floats2half2_rn(a, b); }
};
template <>
struct Pair<int16_t> {
  using Raw = short2;
  static __device__ __forceinline__ float2 get(Raw v) { return make_float2(to_f32(v.x), to_f32(v.y)); }
  static __device__ __forceinline__ Raw put(float a, float b) { return make_short2(from_f32<int16_t>(a), from_f32<int16_t>(b)); }
};

// Eight neighbouring elements in 16-byte accesses (the address is 16-byte aligned).
template <typename T>
__device__ __forceinline__ void load8(const T* p, float (&v)[8]) {
  constexpr int kParts = (int)sizeof(T) / 2;  // 16-byte parts
  constexpr int kPer = 8 / kParts;
#pragma unroll
  for (int q = 0; q < kParts; ++q) {
    const uint4 w = reinterpret_cast<const uint4*>(p)[q];
    const typename Pair<T>::Raw* h = reinterpret_cast<const typename Pair<T>::Raw*>(&w);
#pragma unroll
    for (int j = 0; j < kPer / 2; ++j) {
      const float2 f = Pair<T>::get(h[j]);
      v[q * kPer + 2 * j] = f.x;
      v[q * kPer + 2 * j + 1] = f.y;
    }
  }
}
template <typename T>
__device__ __forceinline__ void store8(T* p, const float (&v)[8]) {
  constexpr int kParts = (int)sizeof(T) / 2;
  constexpr int kPer = 8 / kParts;
#pragma unroll
  for (int q = 0; q < kParts; ++q) {
    uint4 w;
    typename Pair<T>::Raw* h = reinterpret_cast<typename Pair<T>::Raw*>(&w);
#pragma unroll
    for (int j = 0; j < kPer / 2; ++j) h[j] = Pair<T>::put(v[q * kPer + 2 * j], v[q * kPer + 2 * j + 1]);
    reinterpret_cast<uint4*>(p)[q] = w;
  }
}

// ---- host -------------------------------------------------------------------

inline int op_report(char* msg, int msg_len, int code, const char* fmt, ...) {
  if (msg && msg_len > 0) {
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(msg, (size_t)msg_len, fmt, ap);
    va_end(ap);
  }
  return code;
}

inline bool op_float_dtype(int dtype) {
  return dtype == LSTM_APPROX_OP_FP32 || dtype == LSTM_APPROX_OP_BF16 || dtype == LSTM_APPROX_OP_FP16;
}
inline size_t op_dtype_bytes(int dtype) {
  return dtype == LSTM_APPROX_OP_FP32 ? 4 : (dtype == LSTM_APPROX_OP_E4M3 ? 1 : 2);
}
inline bool op_aligned(const void* p, size_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }

// OK on an sm_103 device (asked once per thread and device).
inline int op_check_device(char* msg, int msg_len) {
  static thread_local DeviceSet good;
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return op_report(msg, msg_len, LSTM_APPROX_ECUDA, "no CUDA device");
  if (good.has(dev)) return LSTM_APPROX_OK;
  int major = 0, minor = 0;
  if (cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, dev) != cudaSuccess ||
      cudaDeviceGetAttribute(&minor, cudaDevAttrComputeCapabilityMinor, dev) != cudaSuccess || major != 10 ||
      minor != 3)
    return op_report(msg, msg_len, LSTM_APPROX_ECUDA, "needs an sm_103 device");
  good.add(dev);
  return LSTM_APPROX_OK;
}

inline int op_launched(cudaError_t e, const char* what, char* msg, int msg_len) {
  if (e == cudaSuccess) return LSTM_APPROX_OK;
  return op_report(msg, msg_len, LSTM_APPROX_ECUDA, "%s: %s", what, cudaGetErrorString(e));
}

// A kernel launch whose own error is returned (an earlier call's is left alone).
//
// A programmatic dependent of what the stream holds before it: it may be set up
// while that still runs, and every kernel launched here begins with begin_op(),
// which waits for it (and all that it waited for) to be complete and visible.
// Back to back, small kernels then take 1.7 to 2.6 us each instead of 4.2.
template <typename... KArgs, typename... Args>
cudaError_t op_launch(void (*kern)(KArgs...), dim3 grid, dim3 block, size_t smem, cudaStream_t s, const Args&... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = block;
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kern, KArgs(args)...);
}

// The sizes of the gated delta rule's calls.
constexpr int kDeltaMostDk = 128;
inline int delta_check_sizes(int T, int B, int H, int Hk, int Dk, int Dv, char* msg, int msg_len) {
  if (T < 0 || B < 0) return op_report(msg, msg_len, LSTM_APPROX_EINVAL, "negative sizes");
  if (H < 1 || Hk < 1 || H % Hk) return op_report(msg, msg_len, LSTM_APPROX_EINVAL, "H (%d) must be a multiple of Hk (%d)", H, Hk);
  if (Dk < 1 || Dk > kDeltaMostDk || Dv < 1)
    return op_report(msg, msg_len, LSTM_APPROX_EINVAL, "need 1 <= Dk <= %d and 1 <= Dv, not %d and %d", kDeltaMostDk, Dk, Dv);
  return LSTM_APPROX_OK;
}

// Calls f with a null pointer of the element type of `dtype` (FP32, BF16, FP16).
template <typename F>
cudaError_t op_for_type(int dtype, F f) {
  if (dtype == LSTM_APPROX_OP_FP32) return f(static_cast<float*>(nullptr));
  if (dtype == LSTM_APPROX_OP_BF16) return f(static_cast<__nv_bfloat16*>(nullptr));
  return f(static_cast<__half*>(nullptr));
}

}  // namespace lstm_approx_impl
