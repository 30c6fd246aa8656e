// One AdamW update of many tensors at once (include/lstm_approx_ops.h).
//
//   g' = s g;  m = b1 m + (1 - b1) g';  v = b2 v + (1 - b2) g'^2
//   p = p (1 - lr wd) - lr / (1 - b1^t) m / (sqrt(v / (1 - b2^t)) + eps)
//
// Bound by memory: every value is read once and written once.  A warp takes
// 256 neighbouring values of a tensor, which is also what shares a scale of
// the 8-bit averages: their largest is one warp-wide maximum.  A block of 8
// warps takes 2048 values; which tensor they belong to it finds in the table
// that comes with the kernel's arguments (nothing is copied to the device
// before the launch, and a captured graph holds its own copy).
//
// The averages in 8 bits: m, and u = sqrt(v) (half the range of exponents), as
// e4m3 times a scale.  A moving average that moves by 0.1% a step never leaves
// its 8-bit value where it is rounded to the nearest, so both are rounded to one
// of their two neighbours with the chances that keep the mean: 16 bits from a
// hash of seed, step and position for each.  A u above zero never becomes zero
// (m / (0 + eps) would be a step of any size): it is at least the type's smallest.
#include <cuda_fp8.h>

#include <cmath>

#include "ops_common.cuh"

namespace lstm_approx_impl {
namespace {

constexpr int kThreads = 256;
constexpr int kTile = kThreads * 8;
constexpr int kBlock = 256;  // values to a scale
static_assert(kBlock == 32 * 8, "a warp's values share a scale");
constexpr float kMost = 448.0f, kLeast = 1.953125e-3f, kMinScale = 1.17549435e-38f;  // of e4m3: largest, 2^-9; 2^-126

struct AdamWTensor {
  void *p, *m, *v, *copy;
  const void* g;
  float *m_scale, *v_scale;
  long long n;
  unsigned long long first;  // of its values among those of all tensors
  unsigned tile;             // its first tile
  unsigned char p_type, g_type, copy_type, wide;  // wide: 16 bytes (8-bit averages: 8) at a time
};

struct AdamWShared {
  const int* step_at;
  const float *lr_at, *grad_scale;
  const unsigned char* skip;
  float lr, log_b1, log_b2, b1, b1_rest, b2, b2_rest, eps, decay;
  int step;
  unsigned seed;
};

// (The kernel's arguments may take 32764 bytes; few tensors get a small table, which is cheaper to launch.)
template <int kTensors>
struct AdamWArgs {
  AdamWShared all;
  int count;
  AdamWTensor t[kTensors];
};
constexpr int kFew = 24, kMany = 380;
static_assert(sizeof(AdamWArgs<kMany>) <= 32764, "kernel arguments");

__device__ __forceinline__ unsigned mix(unsigned h) {
  h ^= h >> 16;
  h *= 0x9E3779B1u;
  h ^= h >> 13;
  h *= 0xB7E15163u;
  return h ^ h >> 16;
}

// Where a thread's e-th value lies in its warp's 256: 8 neighbours, or 32 apart.
__device__ __forceinline__ int place(bool wide, int e) {
  const int lane = threadIdx.x & 31;
  return wide ? lane * 8 + e : e * 32 + lane;
}

// A thread's values of the 256 that begin at p; `left` of them lie in the tensor.
template <typename T>
__device__ __forceinline__ void get8(const T* p, bool wide, int left, float (&x)[8]) {
  if (wide && left >= place(true, 8)) {
    load8(p + place(true, 0), x);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = place(wide, e) < left ? to_f32(p[place(wide, e)]) : 0.0f;
  }
}
template <typename T>
__device__ __forceinline__ void put8(T* p, bool wide, int left, const float (&x)[8]) {
  if (wide && left >= place(true, 8)) {
    store8(p + place(true, 0), x);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (place(wide, e) < left) p[place(wide, e)] = from_f32<T>(x[e]);
  }
}
__device__ __forceinline__ void get8(int type, const void* p, long long at, bool wide, int left, float (&x)[8]) {
  if (type == LSTM_APPROX_OP_FP32) get8(static_cast<const float*>(p) + at, wide, left, x);
  else if (type == LSTM_APPROX_OP_BF16) get8(static_cast<const __nv_bfloat16*>(p) + at, wide, left, x);
  else get8(static_cast<const __half*>(p) + at, wide, left, x);
}
__device__ __forceinline__ void put8(int type, void* p, long long at, bool wide, int left, const float (&x)[8]) {
  if (type == LSTM_APPROX_OP_FP32) put8(static_cast<float*>(p) + at, wide, left, x);
  else if (type == LSTM_APPROX_OP_BF16) put8(static_cast<__nv_bfloat16*>(p) + at, wide, left, x);
  else put8(static_cast<__half*>(p) + at, wide, left, x);
}

// The same for 8-bit floats, as they lie in memory.
__device__ __forceinline__ uint2 get8(const uint8_t* p, bool wide, int left) {
  if (wide && left >= place(true, 8)) return *reinterpret_cast<const uint2*>(p + place(true, 0));
  unsigned w[2] = {0u, 0u};
#pragma unroll
  for (int e = 0; e < 8; ++e)
    if (place(wide, e) < left) w[e / 4] |= (unsigned)p[place(wide, e)] << (8 * (e % 4));
  return make_uint2(w[0], w[1]);
}
__device__ __forceinline__ void put8(uint8_t* p, bool wide, int left, uint2 x) {
  if (wide && left >= place(true, 8)) {
    *reinterpret_cast<uint2*>(p + place(true, 0)) = x;
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (place(wide, e) < left) p[place(wide, e)] = (uint8_t)((e < 4 ? x.x : x.y) >> (8 * (e % 4)));
  }
}
__device__ __forceinline__ void from_e4m3(uint2 q, float (&x)[8]) {
#pragma unroll
  for (int e = 0; e < 8; e += 2) {
    const unsigned pair = (e < 4 ? q.x : q.y) >> (8 * (e % 4));
    const __half2 h = __half2(__nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(pair & 0xffffu), __NV_E4M3));
    const float2 f = __half22float2(h);
    x[e] = f.x;
    x[e + 1] = f.y;
  }
}
__device__ __forceinline__ uint2 to_e4m3(const float (&x)[8]) {  // (of values that the type holds)
  unsigned w[2] = {0u, 0u};
#pragma unroll
  for (int e = 0; e < 8; e += 2)
    w[e / 4] |= (unsigned)__nv_cvt_float2_to_fp8x2(make_float2(x[e], x[e + 1]), __NV_SATFINITE, __NV_E4M3) << (8 * (e % 4));
  return make_uint2(w[0], w[1]);
}

// x in [0, 448] to one of its neighbours in e4m3, the upper one if 16 random bits fall below its share of the distance.
// Below 2^-6 the type's values lie 2^-9 apart, as they do from 2^-6 to 2^-5: there x is taken 2^-6 higher.
__device__ __forceinline__ float to_neighbour(float x, unsigned bits16) {
  const float up = x < 0.015625f ? 0.015625f : 0.0f;
  const unsigned b = __float_as_uint(x + up) + (bits16 << 4) + 8u;
  return __uint_as_float(b & ~0xfffffu) - up;
}

// The scale of a warp's 256 values (a NaN among them makes it one).
__device__ __forceinline__ float scale_of(const float (&x)[8]) {
  unsigned most = 0u;
#pragma unroll
  for (int e = 0; e < 8; ++e) most = max(most, __float_as_uint(x[e]) & 0x7fffffffu);
  const float s = __fdiv_rn(__uint_as_float(__reduce_max_sync(0xffffffffu, most)), kMost);
  return s < kMinScale ? kMinScale : s;
}

struct Rates {
  float keep, step, root, eps;  // 1 - lr wd, lr / (1 - b1^t), (1 - b2^t)^-1/2
};

template <int kBits, int kTensors>
__global__ void __launch_bounds__(kThreads) adamw_kernel(const __grid_constant__ AdamWArgs<kTensors> a) {
  __shared__ Rates rates_of_block;
  begin_op();
  const AdamWShared& all = a.all;
  if (all.skip && *all.skip) return;
  int lo = 0, hi = a.count - 1;  // the last tensor whose first tile is not behind this one
  while (lo < hi) {
    const int mid = (lo + hi + 1) / 2;
    if (a.t[mid].tile <= blockIdx.x) lo = mid;
    else hi = mid - 1;
  }
  const AdamWTensor& t = a.t[lo];
  const long long at = (long long)(blockIdx.x - t.tile) * kTile + (threadIdx.x >> 5) * kBlock;
  const long long rest = t.n - at;
  const int left = rest > kBlock ? kBlock : rest > 0 ? (int)rest : 0;
  const bool wide = t.wide;

  float p[8], g[8], m[8], v[8];
  uint2 m8, v8;
  float m_scale = 0.0f, v_scale = 0.0f;
  get8(t.p_type, t.p, at, wide, left, p);
  get8(t.g_type, t.g, at, wide, left, g);
  if constexpr (kBits == 8) {
    m8 = get8(static_cast<const uint8_t*>(t.m) + at, wide, left);
    v8 = get8(static_cast<const uint8_t*>(t.v) + at, wide, left);
    if (left > 0) m_scale = t.m_scale[at / kBlock], v_scale = t.v_scale[at / kBlock];
  } else {
    get8(static_cast<const float*>(t.m) + at, wide, left, m);
    get8(static_cast<const float*>(t.v) + at, wide, left, v);
  }
  const float clip = all.grad_scale ? *all.grad_scale : 1.0f;
  const int step = all.step_at ? *all.step_at : all.step;
  if (threadIdx.x == 0) {  // 1 - b^t = -(e^(t log b) - 1), without the cancellation of small t
    const float lr = all.lr_at ? *all.lr_at : all.lr, n = (float)step;
    rates_of_block = {1.0f - lr * all.decay, __fdiv_rn(lr, -expm1f(n * all.log_b1)),
                      __frsqrt_rn(-expm1f(n * all.log_b2)), all.eps};
  }
  __syncthreads();
  if (left == 0) return;
  const Rates r = rates_of_block;

  if constexpr (kBits == 8) {
    from_e4m3(m8, m);
    from_e4m3(v8, v);
  }
  float u[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float gs = g[e] * clip;
    if constexpr (kBits == 8) {
      m[e] *= m_scale;
      v[e] *= v_scale;
      v[e] *= v[e];
    }
    m[e] = fmaf(m[e], all.b1, gs * all.b1_rest);
    v[e] = fmaf(v[e], all.b2, gs * gs * all.b2_rest);
    asm("sqrt.approx.f32 %0, %1;" : "=f"(u[e]) : "f"(v[e]));
    p[e] = fmaf(p[e], r.keep, -r.step * __fdividef(m[e], fmaf(u[e], r.root, r.eps)));
  }
  put8(t.p_type, t.p, at, wide, left, p);
  if (t.copy) put8(t.copy_type, t.copy, at, wide, left, p);
  if constexpr (kBits == 8) {
    const float ms = scale_of(m), us = scale_of(u), m_inv = __frcp_rn(ms), u_inv = __frcp_rn(us);
    const unsigned key = mix(mix(all.seed + 1u) ^ (unsigned)step);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const unsigned long long where = t.first + (unsigned long long)(at + place(wide, e));
      const unsigned chance = mix((unsigned)where + (key ^ (unsigned)(where >> 32)));
      const float x = fabsf(m[e]) * m_inv, y = u[e] * u_inv;
      m[e] = copysignf(to_neighbour(x > kMost ? kMost : x, chance & 0xffffu), m[e]);
      const float z = to_neighbour(y > kMost ? kMost : y, chance >> 16);
      u[e] = u[e] > 0.0f && z < kLeast ? kLeast : z;
    }
    put8(static_cast<uint8_t*>(t.m) + at, wide, left, to_e4m3(m));
    put8(static_cast<uint8_t*>(t.v) + at, wide, left, to_e4m3(u));
    if ((threadIdx.x & 31) == 0) t.m_scale[at / kBlock] = ms, t.v_scale[at / kBlock] = us;
  } else {
    put8(static_cast<float*>(t.m) + at, wide, left, m);
    put8(static_cast<float*>(t.v) + at, wide, left, v);
  }
}

template <int kTensors>
cudaError_t launch(int bits, const AdamWArgs<kTensors>& a, unsigned tiles, cudaStream_t s) {
  return op_launch(bits == 8 ? adamw_kernel<8, kTensors> : adamw_kernel<32, kTensors>, dim3(tiles), dim3(kThreads), 0, s, a);
}

}  // namespace
}  // namespace lstm_approx_impl

using namespace lstm_approx_impl;

extern "C" int lstm_approx_adamw_step(int count, const lstm_approx_adamw_tensor* tensors, int bits, int step,
                                      const int32_t* step_at, double lr, const float* lr_at, double beta1, double beta2,
                                      double eps, double weight_decay, const float* grad_scale,
                                      const unsigned char* skip, unsigned seed, void* cuda_stream, char* msg, int msg_len) {
  if (msg && msg_len > 0) msg[0] = '\0';
  if (count < 0 || (count > 0 && !tensors)) return op_report(msg, msg_len, LSTM_APPROX_EINVAL, "count %d, or no tensors", count);
  if (bits != 8 && bits != 32) return op_report(msg, msg_len, LSTM_APPROX_EINVAL, "averages have 8 or 32 bits, not %d", bits);
  if (!step_at && step < 1) return op_report(msg, msg_len, LSTM_APPROX_EINVAL, "the first step is 1");
  if (!(beta1 >= 0.0 && beta1 < 1.0 && beta2 >= 0.0 && beta2 < 1.0))
    return op_report(msg, msg_len, LSTM_APPROX_EINVAL, "betas must lie in [0, 1)");
  if (!(eps >= 0.0) || !std::isfinite(eps) || !std::isfinite(weight_decay) || (!lr_at && !std::isfinite(lr)))
    return op_report(msg, msg_len, LSTM_APPROX_EINVAL, "lr and weight_decay must be finite, eps finite and not negative");
  if (!op_aligned(step_at, 4) || !op_aligned(lr_at, 4) || !op_aligned(grad_scale, 4))
    return op_report(msg, msg_len, LSTM_APPROX_EINVAL, "a pointer not aligned to its type");
  for (int i = 0; i < count; ++i) {
    const lstm_approx_adamw_tensor& t = tensors[i];
    if (t.n < 0 || t.n > (1ll << 40)) return op_report(msg, msg_len, LSTM_APPROX_EINVAL, "tensor %d: %lld values", i, t.n);
    if (!op_float_dtype(t.p_dtype) || !op_float_dtype(t.g_dtype) || (t.copy && !op_float_dtype(t.copy_dtype)))
      return op_report(msg, msg_len, LSTM_APPROX_EINVAL, "tensor %d: a type that is not fp32, bf16 or fp16", i);
    if (t.n == 0 || !t.g) continue;
    if (!t.p || !t.m || !t.v || (bits == 8 && (!t.m_scale || !t.v_scale)))
      return op_report(msg, msg_len, LSTM_APPROX_EINVAL, "tensor %d: p, m, v (and the scales of 8-bit averages) must not be NULL", i);
    if (!op_aligned(t.p, op_dtype_bytes(t.p_dtype)) || !op_aligned(t.g, op_dtype_bytes(t.g_dtype)) ||
        (bits == 32 && (!op_aligned(t.m, 4) || !op_aligned(t.v, 4))) || !op_aligned(t.m_scale, 4) || !op_aligned(t.v_scale, 4) ||
        (t.copy && !op_aligned(t.copy, op_dtype_bytes(t.copy_dtype))))
      return op_report(msg, msg_len, LSTM_APPROX_EINVAL, "tensor %d: a pointer not aligned to its type", i);
  }
  if (int rc = op_check_device(msg, msg_len)) return rc;

  AdamWShared all{step_at, lr_at, grad_scale, skip, (float)lr, (float)std::log(beta1), (float)std::log(beta2), (float)beta1,
                  (float)(1.0 - beta1), (float)beta2, (float)(1.0 - beta2), (float)eps, (float)weight_decay, step, seed};
  static thread_local AdamWArgs<kMany> args;  // (32 KB: not on the stack)
  unsigned long long first = 0;
  for (int i = 0; i < count;) {
    args.count = 0;
    long long tiles = 0;
    for (; i < count && args.count < kMany; ++i) {
      const lstm_approx_adamw_tensor& t = tensors[i];
      const long long mine = (t.n + kTile - 1) / kTile;
      const unsigned long long from = first;
      if (t.n == 0 || !t.g) {
        first += (unsigned long long)t.n;
        continue;
      }
      if (tiles + mine > 0x7fffffffll) {
        if (args.count > 0) break;
        return op_report(msg, msg_len, LSTM_APPROX_EINVAL, "tensor %d: %lld values are too many", i, t.n);
      }
      first += (unsigned long long)t.n;
      const size_t state = bits == 8 ? 8 : 16;
      const bool wide = op_aligned(t.p, 16) && op_aligned(t.g, 16) && op_aligned(t.m, state) && op_aligned(t.v, state) &&
                        (!t.copy || op_aligned(t.copy, 16));
      args.t[args.count++] = {t.p, t.m, t.v, t.copy, t.g, t.m_scale, t.v_scale, t.n, from, (unsigned)tiles,
                              (unsigned char)t.p_dtype, (unsigned char)t.g_dtype, (unsigned char)t.copy_dtype, wide};
      tiles += mine;
    }
    if (args.count == 0) continue;
    args.all = all;
    cudaError_t e;
    if (args.count <= kFew) {
      AdamWArgs<kFew> few;
      few.all = all;
      few.count = args.count;
      for (int k = 0; k < args.count; ++k) few.t[k] = args.t[k];
      e = launch(bits, few, (unsigned)tiles, static_cast<cudaStream_t>(cuda_stream));
    } else {
      e = launch(bits, args, (unsigned)tiles, static_cast<cudaStream_t>(cuda_stream));
    }
    if (int rc = op_launched(e, "adamw launch", msg, msg_len)) return rc;
  }
  return LSTM_APPROX_OK;
}
