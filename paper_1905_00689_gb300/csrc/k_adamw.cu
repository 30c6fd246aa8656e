// One AdamW update of many tensors at once (include/lstm_approx_ops.h).
//
//   g' = s g;  m = b1 m + (1 - b1) g';  v = b2 v + (1 - b2) g'^2
//   p = p (1 - lr wd) - lr / (1 - b1^t) m / (sqrt(v / (1 - b2^t)) + eps)
//
// Bound by memory: every value is read once and written once.  A warp takes
// 256 neighbouring values of a tensor, which is also what shares a scale of
// the 8-bit averages: their largest is one warp-wide maximum.  A block of 8
// warps takes 2048 values at a time; which tensor they belong to it finds in the
// table that comes with the kernel's arguments (nothing is copied to the device
// before the launch, and a captured graph holds its own copy).
//
// The averages in 8 bits: m, and u = sqrt(v) (half the range of exponents), as
// e4m3 times a scale.  A moving average that moves by 0.1% a step never leaves
// its 8-bit value where it is rounded to the nearest, so both are rounded to one
// of their two neighbours with the chances that keep the mean: 16 bits from a
// hash of seed, step and position for each.  A u above zero never becomes zero
// (m / (0 + eps) would be a step of any size): it is at least the type's smallest.
//
// Measured, of the 6790 GB/s of a copy: 302 M parameters in 32 bits, gradients and
// copies in 16: 1217 us (102%); the same with 8-bit averages 888 us (80%: the rounding
// is 82 instructions a value, 69% of the issue slots); 13 M in 16 bits with 8-bit
// averages at odd addresses 63 us (31%: values one by one).
//
// With 32-bit averages the root and the reciprocal are the hardware's, each off by one
// unit of its last place, of a step that is a thousandth of p: 1217 us, 1229 with the
// rounded ones.  m and v see neither.
#include <cuda_fp8.h>

#include <cmath>
#include <initializer_list>
#include <type_traits>

#include "ops_common.cuh"
#include "ptx.cuh"

namespace lstm_approx_impl {
namespace {

using namespace lstm_approx_dev;

constexpr int kThreads = 256;
constexpr int kTile = kThreads * 8;
constexpr int kBlock = 256;  // values to a scale
static_assert(kBlock == 32 * 8, "a warp's values share a scale");
constexpr float kMost = 448.0f, kMinScale = 1.17549435e-38f;  // of e4m3; 2^-126
constexpr float kLeastY = 5.42101086e-20f;                     // 2^-64

struct AdamWTensor {
  void *p, *m, *v, *copy;
  const void* g;
  float *m_scale, *v_scale;
  long long n;
  unsigned long long first;  // of its values among those of all tensors
  unsigned tile;             // its first tile
  unsigned char p_type, g_type, copy_type;
};

struct AdamWShared {
  const int* step_at;
  const float *lr_at, *grad_scale;
  const unsigned char* skip;
  float lr, log_b1, log_b2, b1, b1_rest, b2, b2_rest, eps, decay, one;
  int step;
  unsigned seed;
  int rounds;  // tiles to a block
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
__device__ __forceinline__ int place(bool near, int e) {
  const int lane = threadIdx.x & 31;
  return near ? lane * 8 + e : e * 32 + lane;
}

// A thread's values of the 256 that begin at p, of a type known when the kernel runs.  kNear: p is a multiple of 16 bytes (of 8 for
// 8-bit floats) and all of them lie in the tensor; else `left` do, and they are moved one by one.  (Whole pieces of 16 bytes shifted
// into place between lanes took 80 us where this takes 62: 13 M parameters in 16 bits with 8-bit averages, at odd addresses.)
template <bool kNear, typename T>
__device__ __forceinline__ void get8(const T* p, int left, float (&x)[8]) {
  if constexpr (kNear) {
    load8(p + place(true, 0), x);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = place(false, e) < left ? to_f32(p[place(false, e)]) : 0.0f;
  }
}
template <bool kNear, typename T>
__device__ __forceinline__ void put8(T* p, int left, const float (&x)[8]) {
  if constexpr (kNear) {
    store8(p + place(true, 0), x);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (place(false, e) < left) p[place(false, e)] = from_f32<T>(x[e]);
  }
}
template <bool kNear>
__device__ __forceinline__ void get8(int type, const void* p, long long at, int left, float (&x)[8]) {
  if (type == LSTM_APPROX_OP_FP32) get8<kNear>(static_cast<const float*>(p) + at, left, x);
  else if (type == LSTM_APPROX_OP_BF16) get8<kNear>(static_cast<const __nv_bfloat16*>(p) + at, left, x);
  else get8<kNear>(static_cast<const __half*>(p) + at, left, x);
}
template <bool kNear>
__device__ __forceinline__ void put8(int type, void* p, long long at, int left, const float (&x)[8]) {
  if (type == LSTM_APPROX_OP_FP32) put8<kNear>(static_cast<float*>(p) + at, left, x);
  else if (type == LSTM_APPROX_OP_BF16) put8<kNear>(static_cast<__nv_bfloat16*>(p) + at, left, x);
  else put8<kNear>(static_cast<__half*>(p) + at, left, x);
}

// The same for 8-bit floats, four to a word.
template <bool kNear>
__device__ __forceinline__ uint2 get8(const uint8_t* p, int left) {
  if constexpr (kNear) {
    return *reinterpret_cast<const uint2*>(p + place(true, 0));
  } else {
    unsigned b[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) b[e] = place(false, e) < left ? p[place(false, e)] : 0u;
    return make_uint2(b[0] | b[1] << 8 | b[2] << 16 | b[3] << 24, b[4] | b[5] << 8 | b[6] << 16 | b[7] << 24);
  }
}
template <bool kNear>
__device__ __forceinline__ void put8(uint8_t* p, int left, uint2 x) {
  if constexpr (kNear) {
    *reinterpret_cast<uint2*>(p + place(true, 0)) = x;
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (place(false, e) < left) p[place(false, e)] = (uint8_t)((e < 4 ? x.x : x.y) >> (8 * (e % 4)));
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

// x in [0, 448] as an e4m3 code in the upper byte, rounded to one of x's neighbours: the upper one if 16 random bits (bits 8 to 23
// of `chance`) fall below x's share of the distance.  A code is a 32-bit float's exponent and upper 3 bits of fraction, less 960 (64
// more, in 8 bits).  Below 2^-6 the type's values lie 2^-9 apart, as they do from 2^-6 to 2^-5: there x is taken 2^-6, 8 codes,
// higher.  positive: not to zero.
__device__ __forceinline__ unsigned code_of(float x, unsigned chance, bool positive) {
  const bool small = x < 0.015625f;
  if (small) x += 0.015625f;
  unsigned c = __float_as_uint(x) * 16u + ((chance & 0xffff00u) | 0x40000080u);
  if (small) c -= 8u << 24;
  if (small && positive) c = max(c, 1u << 24);
  return c;
}
// The upper bytes of four words.
__device__ __forceinline__ unsigned upper_bytes(unsigned a, unsigned b, unsigned c, unsigned d) {
  return __byte_perm(__byte_perm(a, b, 0x0073), __byte_perm(c, d, 0x0073), 0x5410);
}

__device__ __forceinline__ float max_or_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
// The scale of a warp's 256 values (a NaN among them makes it one).  Times the 32-bit number next to 1 / 448: a division by 448 is
// off by half a unit instead of one, and took 914 us where this takes 891 (302 M parameters).
__device__ __forceinline__ float scale_of(const float (&x)[8]) {
  float most = fabsf(x[0]);
#pragma unroll
  for (int e = 1; e < 8; ++e) most = max_or_nan(most, fabsf(x[e]));
  const float s = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(most) & 0x7fffffffu)) * (1.0f / kMost);
  return s < kMinScale ? kMinScale : s;
}

// sqrt x of two values: Newton's step on y = x^-1/2 with the exact remainder (P. Markstein, "Computation of elementary functions
// on the IBM RISC System/6000 processor", 1990), rounded as sqrtf's from 2^-126 on; below, about x 2^63.  Of infinity, where the
// remainder has no value, x 2^-64, which is less than any other root.  (Without that 877 us, with it 883: 302 M parameters with
// 8-bit averages.)
__device__ __forceinline__ void roots_of(uint64_t x, float x0, float x1, float& u0, float& u1) {
  float y0, y1, r0, r1, l0, l1;
  asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(y0) : "f"(fmaxf(x0, kMinScale)));
  asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(y1) : "f"(fmaxf(x1, kMinScale)));
  const uint64_t y = f32x2(y0, y1), g = mul2(x, y), half = f32x2(0.5f, 0.5f), minus = f32x2(-1.0f, -1.0f);
  f32x2_split(fma2(fma2(mul2(g, minus), g, x), mul2(y, half), g), r0, r1);
  f32x2_split(mul2(x, f32x2(kLeastY, kLeastY)), l0, l1);
  u0 = fmaxf(r0, l0), u1 = fmaxf(r1, l1);  // (NaN in both of NaN)
}

struct Rates {
  float keep, step, root, eps, one;  // 1 - lr wd, lr / (1 - b1^t), (1 - b2^t)^-1/2
};

// What one tile needs beside its tensor.
struct Update {
  float clip, b1, b1_rest, b2, b2_rest;
  unsigned key;  // of the random bits
};

// Loads, to be followed by update() when the rates are there.
// kExact: roots by sqrtf's.
template <int kBits, bool kNear, bool kExact>
struct Tile {
  float p[8], g[8], m[8], v[8];
  uint2 m8, v8;
  float m_scale, v_scale;

  __device__ __forceinline__ void load(const AdamWTensor& t, long long at, int left) {
    get8<kNear>(t.p_type, t.p, at, left, p);
    get8<kNear>(t.g_type, t.g, at, left, g);
    if constexpr (kBits == 8) {
      m8 = get8<kNear>(static_cast<const uint8_t*>(t.m) + at, left);
      v8 = get8<kNear>(static_cast<const uint8_t*>(t.v) + at, left);
      m_scale = t.m_scale[at / kBlock], v_scale = t.v_scale[at / kBlock];
    } else {
      get8<kNear>(static_cast<const float*>(t.m) + at, left, m);
      get8<kNear>(static_cast<const float*>(t.v) + at, left, v);
    }
  }

  // (Two values to an instruction; each operation rounded by itself, so that which neighbour an 8-bit average becomes follows from
  // the formula alone.)
  __device__ __forceinline__ void update(const AdamWTensor& t, long long at, int left, const Update& w, const Rates& r) {
    float u[8];
    if constexpr (kBits == 8) {
      from_e4m3(m8, m);
      from_e4m3(v8, v);
    }
    const uint64_t clip = f32x2(w.clip, w.clip), b1 = f32x2(w.b1, w.b1), b1_rest = f32x2(w.b1_rest, w.b1_rest);
    const uint64_t b2 = f32x2(w.b2, w.b2), b2_rest = f32x2(w.b2_rest, w.b2_rest), keep = f32x2(r.keep, r.keep);
    const uint64_t back = f32x2(-r.step, -r.step), root = f32x2(r.root, r.root), eps = f32x2(r.eps, r.eps), one = f32x2(r.one, r.one);
#pragma unroll
    for (int e = 0; e < 8; e += 2) {
      const uint64_t gs = mul2(f32x2(g[e], g[e + 1]), clip);
      uint64_t mm = f32x2(m[e], m[e + 1]), vv = f32x2(v[e], v[e + 1]);
      if constexpr (kBits == 8) {
        mm = mul2(mm, f32x2(m_scale, m_scale));
        vv = mul2(vv, f32x2(v_scale, v_scale));
        vv = mul2(vv, vv);
      }
      // (times one, which the compiler does not know: it would make one operation of a product and a sum)
      mm = fma2(mul2(mm, b1), one, mul2(gs, b1_rest));
      vv = fma2(mul2(vv, b2), one, mul2(mul2(gs, gs), b2_rest));
      f32x2_split(mm, m[e], m[e + 1]);
      f32x2_split(vv, v[e], v[e + 1]);
      if constexpr (kExact) {
        u[e] = __fsqrt_rn(v[e]), u[e + 1] = __fsqrt_rn(v[e + 1]);
      } else if constexpr (kBits == 8) {
        roots_of(vv, v[e], v[e + 1], u[e], u[e + 1]);
      } else {
        asm("sqrt.approx.f32 %0, %1;" : "=f"(u[e]) : "f"(v[e]));
        asm("sqrt.approx.f32 %0, %1;" : "=f"(u[e + 1]) : "f"(v[e + 1]));
      }
      float d0, d1;
      f32x2_split(fma2(f32x2(u[e], u[e + 1]), root, eps), d0, d1);
      const uint64_t ratio = mul2(mm, f32x2(rcp_approx(d0), rcp_approx(d1)));
      f32x2_split(fma2(f32x2(p[e], p[e + 1]), keep, mul2(back, ratio)), p[e], p[e + 1]);
    }
    put8<kNear>(t.p_type, t.p, at, left, p);
    if (t.copy) put8<kNear>(t.copy_type, t.copy, at, left, p);
    if constexpr (kBits == 8) {
      const float ms = scale_of(m), us = scale_of(u), m_inv = __frcp_rn(ms), u_inv = __frcp_rn(us);
      const unsigned long long first = t.first + (unsigned long long)at;
      const unsigned low = (unsigned)first, high = (unsigned)(first >> 32);
      unsigned mc[8], uc[8], mq[2], uq[2];
      auto round_all = [&](auto wraps) {
        const unsigned key0 = w.key ^ high, key1 = w.key ^ (high + 1u);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const unsigned where = low + place(kNear, e);
          const unsigned chance = mix(where + (decltype(wraps)::value && where < low ? key1 : key0));
          mc[e] = code_of(fminf(fabsf(m[e]) * m_inv, kMost), chance << 8, false);
          uc[e] = code_of(fminf(u[e] * u_inv, kMost), chance >> 8, u[e] > 0.0f);
        }
      };
      if (low > 0u - kBlock) round_all(std::true_type());  // positions pass a multiple of 2^32 among these
      else round_all(std::false_type());
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const unsigned sign = upper_bytes(__float_as_uint(m[4 * x]), __float_as_uint(m[4 * x + 1]), __float_as_uint(m[4 * x + 2]),
                                          __float_as_uint(m[4 * x + 3]));
        mq[x] = upper_bytes(mc[4 * x], mc[4 * x + 1], mc[4 * x + 2], mc[4 * x + 3]) | (sign & 0x80808080u);
        uq[x] = upper_bytes(uc[4 * x], uc[4 * x + 1], uc[4 * x + 2], uc[4 * x + 3]);
      }
      put8<kNear>(static_cast<uint8_t*>(t.m) + at, left, make_uint2(mq[0], mq[1]));
      put8<kNear>(static_cast<uint8_t*>(t.v) + at, left, make_uint2(uq[0], uq[1]));
      if ((threadIdx.x & 31) == 0) t.m_scale[at / kBlock] = ms, t.v_scale[at / kBlock] = us;
    } else {
      put8<kNear>(static_cast<float*>(t.m) + at, left, m);
      put8<kNear>(static_cast<float*>(t.v) + at, left, v);
    }
  }
};

template <int kBits, int kTensors, bool kWide, bool kExact = false>
__global__ void __launch_bounds__(kThreads, kBits == 8 ? 5 : 4) adamw_kernel(const __grid_constant__ AdamWArgs<kTensors> a) {
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
  const long long tile = (long long)(blockIdx.x - t.tile) * all.rounds;
  const int step = all.step_at ? *all.step_at : all.step;
  const Update w{all.grad_scale ? *all.grad_scale : 1.0f, all.b1, all.b1_rest, all.b2, all.b2_rest, mix(mix(all.seed + 1u) ^ (unsigned)step)};
  Rates rates{};
  auto run = [&](auto near, long long at, int left, bool first) {
    Tile<kBits, decltype(near)::value, kExact> tile;
    tile.load(t, at, left);
    if (first) {  // 1 - b^t = -(e^(t log b) - 1), without the cancellation of small t; while the loads are under way
      const float lr = all.lr_at ? *all.lr_at : all.lr, n = (float)step;
      rates = {1.0f - lr * all.decay, __fdiv_rn(lr, -expm1f(n * all.log_b1)), __frsqrt_rn(-expm1f(n * all.log_b2)), all.eps, all.one};
    }
    tile.update(t, at, left, w, rates);
  };
#pragma unroll 1
  for (int round = 0; round < all.rounds; ++round) {
    const long long at = (tile + round) * kTile + (threadIdx.x >> 5) * kBlock, rest = t.n - at;
    if (rest <= 0) return;
    if (kWide && rest >= kBlock) run(std::true_type(), at, kBlock, round == 0);
    else run(std::false_type(), at, rest < kBlock ? (int)rest : kBlock, round == 0);
  }
}

// Roots below 2^-63 by roots_of are too small, which beside an eps of 1e-9 nobody sees (1e-19, 1000 times that for a beta2 of
// 0.999999); with a smaller eps, or none, 8-bit averages take sqrtf's (973 us where roots_of takes 883).
template <int kTensors>
cudaError_t launch(int bits, bool wide, const AdamWArgs<kTensors>& a, unsigned tiles, cudaStream_t s) {
  auto kern = bits == 8 && a.all.eps < 1e-9f ? (wide ? adamw_kernel<8, kTensors, true, true> : adamw_kernel<8, kTensors, false, true>)
              : bits == 8 ? (wide ? adamw_kernel<8, kTensors, true> : adamw_kernel<8, kTensors, false>)
                        : (wide ? adamw_kernel<32, kTensors, true> : adamw_kernel<32, kTensors, false>);
  return op_launch(kern, dim3(tiles), dim3(kThreads), 0, s, a);
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
  // (the reciprocal of what is below or above counts as that of zero or as zero: 0 / eps would not be 0)
  const float least = 1.17549435e-38f, most = 8.50705917e37f;
  if (eps != 0.0 && !((float)eps >= least && (float)eps <= most))
    return op_report(msg, msg_len, LSTM_APPROX_EINVAL, "eps must be 0 or between 2^-126 and 2^126");
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
                  (float)(1.0 - beta1), (float)beta2, (float)(1.0 - beta2), (float)eps, (float)weight_decay, 1.0f, step, seed, 1};
  static thread_local AdamWArgs<kMany> args;  // (32 KB: not on the stack)
  // What a block does once (its tensor, the rates) is a quarter of its instructions with one tile: four tiles to a block where
  // there are enough of them for that (302 M parameters with 8-bit averages 1020 us with one, 890 with four).
  long long all_tiles = 0;
  for (int i = 0; i < count; ++i) all_tiles += (tensors[i].n + kTile - 1) / kTile;
  all.rounds = all_tiles >= 152 * 32 ? 4 : 1;
  const long long tile_values = (long long)kTile * all.rounds;
  for (const bool wide : {true, false}) {  // those at multiples of 16 bytes (8, 8-bit averages), then the others
    unsigned long long first = 0;
    for (int i = 0; i < count;) {
      args.count = 0;
      long long tiles = 0;
      for (; i < count && args.count < kMany; ++i) {
        const lstm_approx_adamw_tensor& t = tensors[i];
        const long long mine = (t.n + tile_values - 1) / tile_values;
        const size_t state = bits == 8 ? 8 : 16;
        const bool is_wide = op_aligned(t.p, 16) && op_aligned(t.g, 16) && op_aligned(t.m, state) && op_aligned(t.v, state) &&
                             (!t.copy || op_aligned(t.copy, 16));
        if (t.n > 0 && t.g && is_wide == wide) {
          if (tiles + mine > 0x7fffffffll) break;  // (one tensor's are fewer)
          args.t[args.count++] = {t.p, t.m, t.v, t.copy, t.g, t.m_scale, t.v_scale, t.n, first, (unsigned)tiles,
                                  (unsigned char)t.p_dtype, (unsigned char)t.g_dtype, (unsigned char)t.copy_dtype};
          tiles += mine;
        }
        first += (unsigned long long)t.n;
      }
      if (args.count == 0) continue;
      args.all = all;
      cudaError_t e;
      if (args.count <= kFew) {
        AdamWArgs<kFew> few;
        few.all = all;
        few.count = args.count;
        for (int k = 0; k < args.count; ++k) few.t[k] = args.t[k];
        e = launch(bits, wide, few, (unsigned)tiles, static_cast<cudaStream_t>(cuda_stream));
      } else {
        e = launch(bits, wide, args, (unsigned)tiles, static_cast<cudaStream_t>(cuda_stream));
      }
      if (int rc = op_launched(e, "adamw launch", msg, msg_len)) return rc;
    }
  }
  return LSTM_APPROX_OK;
}
