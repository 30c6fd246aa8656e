// Matrix-vector products with 4-bit weights, a scale and a zero point per
// group of columns, and the quantiser that makes such weights
// (include/lstm_approx_ops.h):
//
//   y[m][n] = sum_g scale[n][g] sum_{k in g} (q[n][k] - zero[n][g]) x[m][k]
//
// Bound by memory: the 4-bit matrix, which is read once for up to 32 columns
// (below) at a time.  The products are warp MMAs of 16 rows of W by 16 k by 8
// columns of x^T, their operands in registers: tcgen05 takes both operands from
// shared memory or tensor memory, to which 4-bit weights would first have to be
// expanded, four bytes written for each byte read.
//
//   W   A block of 16 rows by 128 k (1 KB, 64 bytes to a row) comes into shared
//       memory by asynchronous copies, kDepth blocks in flight to a warp.  Four
//       lanes share a row; a lane's 32-bit word holds 8 k as 4 pairs of 16-bit
//       integers after one AND-OR each, (0, 4) (1, 5) (2, 6) (3, 7): or-ed into
//       the mantissa of 128 (bf16) or 1024 (fp16), from which 128 + zero or 1024
//       + zero is subtracted: q - zero, exactly.  Which k a lane holds in which
//       MMA does not matter as long as x is laid out alike, and so that one MMA
//       sums over one group only.
//   x   Once per block of threads, into shared memory in the order in which the
//       lanes read it (16 bytes each, no conflicts): bf16 or fp16 as they are,
//       8-bit values as fp16, and 32-bit values as three columns of bf16 (the
//       upper 8 bits of the mantissa, the next, the last; their sum is exactly x).
//   sum Each group's sum, in fp32 (8 exact products to an addition), times its
//       scale, is added to the row's; the warps of a block share its rows' K and
//       add up through shared memory, always in the same order.
#include <cuda_fp8.h>

#include <algorithm>

#include "ops_common.cuh"
#include "ptx.cuh"

namespace lstm_approx_impl {
namespace {

using namespace lstm_approx_dev;

constexpr int kBlockK = 128;  // k of a block
constexpr int kDepth = 4;     // blocks in flight or in use to a warp
constexpr int kMaxWarps = 16;

__device__ __forceinline__ float e4m3_to_f32(uint8_t v) {
  return __half2float(__half(__nv_cvt_fp8_to_halfraw(v, __NV_E4M3)));
}

struct W4Args {
  int x_dtype;
  const void* x;
  long long x_pitch;
  const float* x_scale;
  int x_groups;  // scales of a row of x
  const uint8_t* q;
  long long q_pitch;
  const void* scale;
  int scale_dtype;
  const uint8_t* zero;
  const float* bias;
  int M, N, K, groups;
  void* y;
  int y_dtype;
  bool x_vec;  // 8 values of x lie in aligned accesses
  int tokens;  // rows of x at a time
  int tiles;   // of kMt * 16 rows
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

// The four pairs of a word's nibbles as 16-bit numbers less `bias` (a pair of 128 + zero or 1024 + zero).
template <bool kBf16>
__device__ __forceinline__ uint32_t nibbles(uint32_t w, int shift, uint32_t bias) {
  uint32_t v;  // (w >> shift & 0x000f000f) | magic
  asm("lop3.b32 %0, %1, 0x000f000f, %2, 0xea;" : "=r"(v) : "r"(w >> shift), "r"(kBf16 ? 0x43004300u : 0x64006400u));
  if constexpr (kBf16) {
    const __nv_bfloat162 d = __hsub2(*reinterpret_cast<const __nv_bfloat162*>(&v), *reinterpret_cast<const __nv_bfloat162*>(&bias));
    return *reinterpret_cast<const uint32_t*>(&d);
  } else {
    const __half2 d = __hsub2(*reinterpret_cast<const __half2*>(&v), *reinterpret_cast<const __half2*>(&bias));
    return *reinterpret_cast<const uint32_t*>(&d);
  }
}

// Place of k's chunk of 8 (sub-block of 32, word of 8 in it) among a block's: slot of the lane, lane of the four.
// kSubs = group / 32: all chunks of a slot lie in one group.
template <int kSubs>
__device__ __forceinline__ void place(int sub, int word, int& slot, int& t) {
  if constexpr (kSubs == 4) {
    slot = word;
    t = sub;
  } else if constexpr (kSubs == 2) {
    slot = (sub & 2) | (word & 1);
    t = (word & 2) | (sub & 1);
  } else {
    slot = sub;
    t = word;
  }
}

// 8 values of x from k on (zero from K on), as fp32 bits or 16-bit values.
template <int kX>
__device__ __forceinline__ void load_chunk(const W4Args& a, long long row, int k, bool vec, uint32_t (&v)[8]) {
  if (vec && k + 8 <= a.K) {
    if constexpr (kX == LSTM_APPROX_OP_FP32) {
      const uint4* p = reinterpret_cast<const uint4*>(static_cast<const float*>(a.x) + row * a.x_pitch + k);
      const uint4 lo = p[0], hi = p[1];
      v[0] = lo.x, v[1] = lo.y, v[2] = lo.z, v[3] = lo.w, v[4] = hi.x, v[5] = hi.y, v[6] = hi.z, v[7] = hi.w;
    } else if constexpr (kX == LSTM_APPROX_OP_E4M3) {
      const uint2 w = *reinterpret_cast<const uint2*>(static_cast<const uint8_t*>(a.x) + row * a.x_pitch + k);
#pragma unroll
      for (int e = 0; e < 8; ++e)
        v[e] = __half_raw(__nv_cvt_fp8_to_halfraw((uint8_t)((e < 4 ? w.x : w.y) >> (8 * (e & 3))), __NV_E4M3)).x;
    } else {
      const uint4 w = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(a.x) + row * a.x_pitch + k);
      const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = u[e / 2] >> (16 * (e & 1)) & 0xffffu;
    }
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      v[e] = 0u;
      if (k + e < a.K) {
        const long long at = row * a.x_pitch + k + e;
        if constexpr (kX == LSTM_APPROX_OP_FP32) v[e] = static_cast<const uint32_t*>(a.x)[at];
        else if constexpr (kX == LSTM_APPROX_OP_E4M3)
          v[e] = __half_raw(__nv_cvt_fp8_to_halfraw(static_cast<const uint8_t*>(a.x)[at], __NV_E4M3)).x;
        else v[e] = static_cast<const uint16_t*>(a.x)[at];
      }
    }
  }
}
__device__ __forceinline__ uint4 in_order(const uint32_t (&v)[8]) {  // 16-bit values as pairs (0, 4) (1, 5) (2, 6) (3, 7)
  return make_uint4(v[0] | v[4] << 16, v[1] | v[5] << 16, v[2] | v[6] << 16, v[3] | v[7] << 16);
}

// Columns of x^T to a row of x: its three parts in 32 bits.
template <int kX>
constexpr int kParts = kX == LSTM_APPROX_OP_FP32 ? 3 : 1;

// kX: type of x.  A tile is kMt * 16 rows of W; kNt * 8 columns of x^T.  kSubs = group / 32.
template <int kX, int kMt, int kNt, int kSubs>
__global__ void __launch_bounds__(kMaxWarps * 32) w4_matvec_kernel(const W4Args a) {
  constexpr bool kBf16 = kX == LSTM_APPROX_OP_BF16 || kX == LSTM_APPROX_OP_FP32;
  constexpr bool kScaled = kX == LSTM_APPROX_OP_E4M3;
  constexpr int kP = kParts<kX>;
  constexpr int kRed = kNt * 8 + 1;         // pitch of the sums
  constexpr int kSets = 4 / kSubs;          // groups of a block
  extern __shared__ __align__(128) unsigned char memory[];
  const int warps = blockDim.x >> 5, warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int blocks = (a.K + kBlockK - 1) / kBlockK, mine = (blocks + warps - 1) / warps;  // of K, to a warp
  const int m0 = blockIdx.y * a.tokens, tokens = min(a.tokens, a.M - m0), cols = tokens * kP;
  // ring [warps][kDepth][kMt][16][64 bytes], sums [2][warps][kMt * 16][kRed], x [blocks][4][cols][4] x 16 bytes, scales
  // of x [blocks][kNt * 8]
  unsigned char* ring = memory + warp * kDepth * kMt * 1024;
  float* sums = reinterpret_cast<float*>(memory + warps * kDepth * kMt * 1024);
  uint4* xs = reinterpret_cast<uint4*>(sums + 2 * warps * kMt * 16 * kRed);
  float* x_scales = reinterpret_cast<float*>(xs + blocks * 16 * cols);

  // position (tile, j): block warp + warps * j of that tile; the copies run kDepth - 1 positions ahead
  int to_tile = blockIdx.x, to_j = 0, to_stage = 0;
  auto fetch = [&]() {
    const int block = warp + warps * to_j;
    if (to_tile < a.tiles && block < blocks) {
#pragma unroll
      for (int q = 0; q < 2 * kMt; ++q) {  // 8 rows of 64 bytes at a time
        const int row = q * 8 + g, n = min(to_tile * kMt * 16 + row, a.N - 1);
        const bool in = block * kBlockK + t * 32 < a.K;
        const uint8_t* from = a.q + (long long)n * a.q_pitch + (in ? block * 64 + t * 16 : 0);
        // sub-block t of row r at place t ^ (r / 2 % 4): no two lanes of a read below meet in a bank
        const uint32_t at = smem_u32(ring + to_stage * kMt * 1024 + row * 64 + ((t ^ (row >> 1 & 3)) << 4));
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(at), "l"(from), "r"(in ? 16 : 0) : "memory");
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
    to_stage = to_stage + 1 == kDepth ? 0 : to_stage + 1;
    if (++to_j == mine) to_j = 0, to_tile += gridDim.x;
  };
  // scales and zero points: a lane takes one group's of the next kSubs positions, for rows g and g + 8 of each 16
  struct Set {
    float s[2 * kMt];
    unsigned z[2 * kMt];
  };
  auto load_set = [&](int tile, int j) {
    Set v;
    const int block = warp + warps * (j + t / kSets), group = block * kSets + t % kSets;
    const bool in = tile < a.tiles && j + t / kSets < mine && group < a.groups;
#pragma unroll
    for (int q = 0; q < 2 * kMt; ++q) {
      const long long at = (long long)min(tile * kMt * 16 + q * 8 + g, a.N - 1) * a.groups + group;
      v.s[q] = in ? load_any(a.scale, at, a.scale_dtype) : 0.0f;
      v.z[q] = in && a.zero ? a.zero[at] & 15u : 8u;
    }
    return v;
  };
#pragma unroll
  for (int d = 0; d < kDepth - 1; ++d) fetch();
  Set now, next = load_set(blockIdx.x, 0);

  for (int c = threadIdx.x; c < tokens * blocks * 16; c += blockDim.x) {
    const int token = c / (blocks * 16), chunk = c % (blocks * 16), k = chunk * 8;
    uint32_t v[8];
    load_chunk<kX>(a, m0 + token, k, a.x_vec, v);
    int slot, lane_t;
    place<kSubs>(chunk >> 2 & 3, chunk & 3, slot, lane_t);
    uint4* to = xs + (((chunk >> 4) * 4 + slot) * cols + token * kP) * 4 + lane_t;
    if constexpr (kP == 3) {
      // three times the upper 16 bits of what is left; not finite: all in the first
#pragma unroll
      for (int part = 0; part < 3; ++part) {
        uint32_t u[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          u[e] = v[e] >> 16;
          const bool finite = (v[e] & 0x7f800000u) != 0x7f800000u;
          if (!finite && (v[e] & 0x007f0000u) == 0u && (v[e] & 0x007fffffu) != 0u) u[e] |= 0x40u;  // a NaN stays one
          v[e] = finite ? __float_as_uint(__uint_as_float(v[e]) - __uint_as_float(v[e] & 0xffff0000u)) : 0u;
        }
        to[part * 4] = in_order(u);
      }
    } else {
      to[0] = in_order(v);
    }
  }
  if constexpr (kScaled) {
    for (int c = threadIdx.x; c < blocks * kNt * 8; c += blockDim.x) {
      const int token = c % (kNt * 8), block = c / (kNt * 8);
      x_scales[c] = token < tokens ? a.x_scale[(long long)(m0 + token) * a.x_groups + (a.x_groups > 1 ? block : 0)] : 0.0f;
    }
  }
  __syncthreads();

  float acc[kMt][kNt][4] = {};
  int stage = 0, j = 0, turn = 0;
  for (int tile = blockIdx.x; tile < a.tiles;) {
    if (j % kSubs == 0) {
      now = next;
      next = j + kSubs < mine ? load_set(tile, j + kSubs) : load_set(tile + gridDim.x, 0);
    }
    asm volatile("cp.async.wait_group %0;" ::"n"(kDepth - 2) : "memory");
    __syncwarp();
    fetch();
    const int block = warp + warps * j;
    if (block < blocks) {
      const unsigned char* here = ring + stage * kMt * 1024;
      float xsc[kNt][2];
      if constexpr (kScaled) {
#pragma unroll
        for (int n = 0; n < kNt; ++n) {
          const float2 v = *reinterpret_cast<const float2*>(x_scales + block * kNt * 8 + n * 8 + 2 * t);
          xsc[n][0] = v.x;
          xsc[n][1] = v.y;
        }
      }
#pragma unroll
      for (int set = 0; set < kSets; ++set) {  // groups of the block
        const int from = (lane & ~3) | ((j % kSubs) * kSets + set);
        float s[2 * kMt];
        uint32_t z[2 * kMt];
#pragma unroll
        for (int q = 0; q < 2 * kMt; ++q) {
          s[q] = __shfl_sync(0xffffffffu, now.s[q], from);
          z[q] = (kBf16 ? 0x43004300u : 0x64006400u) + __shfl_sync(0xffffffffu, now.z[q], from) * 0x00010001u;
        }
        uint4 b[kSubs][kNt];
#pragma unroll
        for (int i = 0; i < kSubs; ++i) {
#pragma unroll
          for (int n = 0; n < kNt; ++n) {
            b[i][n] = make_uint4(0u, 0u, 0u, 0u);
            if (n * 8 + g < cols) b[i][n] = xs[((block * 4 + set * kSubs + i) * cols + n * 8 + g) * 4 + t];
          }
        }
#pragma unroll
        for (int m = 0; m < kMt; ++m) {
          // the lane's kSubs words of rows g and g + 8
          uint32_t w[2][kSubs];
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const int row = m * 16 + h * 8 + g, swz = row >> 1 & 3;
            const unsigned char* p = here + row * 64;
            if constexpr (kSubs == 4) {
              const uint4 v = *reinterpret_cast<const uint4*>(p + ((t ^ swz) << 4));
              w[h][0] = v.x, w[h][1] = v.y, w[h][2] = v.z, w[h][3] = v.w;
            } else if constexpr (kSubs == 2) {
              const uint2 v = *reinterpret_cast<const uint2*>(p + (((2 * set + (t & 1)) ^ swz) << 4) + (t >> 1) * 8);
              w[h][0] = v.x, w[h][1] = v.y;
            } else {
              w[h][0] = *reinterpret_cast<const uint32_t*>(p + ((set ^ swz) << 4) + t * 4);
            }
          }
          float part[kNt][4] = {};
#pragma unroll
          for (int i = 0; i < kSubs; ++i) {
#pragma unroll
            for (int half = 0; half < 2; ++half) {
              const uint32_t a0 = nibbles<kBf16>(w[0][i], 8 * half, z[2 * m]);
              const uint32_t a1 = nibbles<kBf16>(w[1][i], 8 * half, z[2 * m + 1]);
              const uint32_t a2 = nibbles<kBf16>(w[0][i], 8 * half + 4, z[2 * m]);
              const uint32_t a3 = nibbles<kBf16>(w[1][i], 8 * half + 4, z[2 * m + 1]);
#pragma unroll
              for (int n = 0; n < kNt; ++n) {
                const uint32_t b0 = half ? b[i][n].z : b[i][n].x, b1 = half ? b[i][n].w : b[i][n].y;
                if constexpr (kBf16) mma_16816_bf16<true>(part[n], a0, a1, a2, a3, b0, b1);
                else mma_16816_f16<true>(part[n], a0, a1, a2, a3, b0, b1);
              }
            }
          }
#pragma unroll
          for (int n = 0; n < kNt; ++n) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const float v = kScaled ? part[n][e] * xsc[n][e & 1] : part[n][e];
              acc[m][n][e] = fmaf(v, s[2 * m + (e >> 1)], acc[m][n][e]);
            }
          }
        }
      }
    }
    stage = stage + 1 == kDepth ? 0 : stage + 1;
    if (++j < mine) continue;
    // the tile's sums: the warps' parts, in their order
    float* to = sums + (turn * warps + warp) * kMt * 16 * kRed;
#pragma unroll
    for (int m = 0; m < kMt; ++m) {
#pragma unroll
      for (int n = 0; n < kNt; ++n) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          to[(m * 16 + (e >> 1) * 8 + g) * kRed + n * 8 + 2 * t + (e & 1)] = acc[m][n][e];
          acc[m][n][e] = 0.0f;
        }
      }
    }
    __syncthreads();
    const float* from = sums + turn * warps * kMt * 16 * kRed;
    for (int o = threadIdx.x; o < kMt * 16 * tokens; o += blockDim.x) {
      const int row = o % (kMt * 16), token = o / (kMt * 16), n = tile * kMt * 16 + row;
      if (n >= a.N) continue;
      float v = 0.0f;
      for (int w = 0; w < warps; ++w) {
        const float* p = from + (w * kMt * 16 + row) * kRed + token * kP;
        if constexpr (kP == 3) v += p[0] + (p[1] + p[2]);
        else v += p[0];
      }
      if (a.bias) v += a.bias[n];
      store_any(a.y, (long long)(m0 + token) * a.N + n, a.y_dtype, v);
    }
    turn ^= 1;  // the next tile's parts go beside these
    j = 0;
    tile += gridDim.x;
  }
  asm volatile("cp.async.wait_group 0;" ::: "memory");
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

// What a launch of the kernel takes: rows of x at a time, warps of a block, shared memory.
struct W4Plan {
  int tokens, warps;
  size_t smem;
};
constexpr size_t kMostShared = 227 * 1024;
constexpr int kMaxK = 32768;  // one row of x in 32 bits then fits beside four warps' blocks

inline W4Plan plan_matvec(int M, int K, int parts, int mt, int nt, bool scaled) {
  const int blocks = (K + kBlockK - 1) / kBlockK;
  const size_t per_warp = kDepth * mt * 1024 + 2 * mt * 16 * (nt * 8 + 1) * sizeof(float);
  W4Plan p{std::min(M, nt * 8 / parts), 0, 0};
  // as many rows of x as leave room for four warps, then as many warps as fit: 8 of them share a tile's K where
  // several blocks of threads fit on an SM, up to 16 where one does
  for (;; --p.tokens) {
    const size_t x = (size_t)blocks * (256 * p.tokens * parts + (scaled ? 32 * nt : 0));
    const int most = x > 40 * 1024 ? kMaxWarps : 8;
    const int fit = x < kMostShared ? (int)((kMostShared - x) / per_warp) : 0;
    if (fit >= 4 || p.tokens == 1) {
      p.warps = std::max(1, std::min({most, fit, blocks}));
      p.smem = p.warps * per_warp + x;
      return p;
    }
  }
}

template <int kX, int kMt, int kNt, int kSubs>
cudaError_t launch_matvec(W4Args a, cudaStream_t s) {
  static thread_local DeviceSet ready;  // of the one kernel that this instance launches
  auto kern = w4_matvec_kernel<kX, kMt, kNt, kSubs>;
  const cudaError_t e = once_per_device(
      &ready, [&] { return cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kMostShared); });
  if (e != cudaSuccess) return e;
  const W4Plan p = plan_matvec(a.M, a.K, kParts<kX>, kMt, kNt, kX == LSTM_APPROX_OP_E4M3);
  if (p.smem > kMostShared) return cudaErrorInvalidValue;
  a.tokens = p.tokens;
  a.tiles = (a.N + kMt * 16 - 1) / (kMt * 16);
  const int per_sm = (int)std::max<size_t>(1, std::min<size_t>(228 * 1024 / (p.smem + 1024), 32 / p.warps));
  const dim3 grid(std::min(a.tiles, 152 * per_sm), (a.M + p.tokens - 1) / p.tokens);
  return op_launch(kern, grid, dim3(p.warps * 32), p.smem, s, a);
}

int check_matrix(int N, int K, int group, const void* q, long long q_pitch, const void* scale, int scale_dtype,
                 char* msg, int msg_len) {
  if (N < 0 || K < 1 || K > kMaxK)
    return op_report(msg, msg_len, LSTM_APPROX_EINVAL, "need N >= 0 and 1 <= K <= %d", kMaxK);
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
  if (M < 0 || M > 65535) return op_report(msg, msg_len, LSTM_APPROX_EINVAL, "need 0 <= M <= 65535");
  if (M > 0 && N > 0 && (!x || !y || x8 != (x_scale != nullptr)))
    return op_report(msg, msg_len, LSTM_APPROX_EINVAL, "x and y must not be NULL; x_scale is given for 8-bit x only");
  if (x8 && x_group != 128 && x_group < K)
    return op_report(msg, msg_len, LSTM_APPROX_EINVAL, "x_group must be 128 or >= K, not %d", x_group);
  if (x_pitch < 0 || !op_aligned(x, op_dtype_bytes(x_dtype)) || !op_aligned(x_scale, 4) || !op_aligned(bias, 4) ||
      !op_aligned(y, op_dtype_bytes(y_dtype)))
    return op_report(msg, msg_len, LSTM_APPROX_EINVAL, "a negative pitch, or a pointer not aligned to its type");
  if (int rc = op_check_device(msg, msg_len)) return rc;
  if (M == 0 || N == 0) return LSTM_APPROX_OK;
  const size_t xs = op_dtype_bytes(x_dtype);
  W4Args a{x_dtype, x, x_pitch, x_scale, x_group >= K || !x8 ? 1 : (K + 127) / 128, q, q_pitch, scale, scale_dtype, zero,
           bias, M, N, K, (K + group - 1) / group, y, y_dtype,
           op_aligned(x, std::min<size_t>(16, 8 * xs)) && x_pitch * xs % std::min<size_t>(16, 8 * xs) == 0, 0, 0};
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  auto of_type = [&](auto type) {
    constexpr int kX = decltype(type)::value;
    const int cols = std::min(M, 32) * kParts<kX>;
    auto of_group = [&](auto subs) {
      constexpr int kSubs = decltype(subs)::value;
      if (cols <= 8) return launch_matvec<kX, 1, 1, kSubs>(a, s);
      if (cols <= 16) return launch_matvec<kX, 2, 2, kSubs>(a, s);
      return launch_matvec<kX, 2, 4, kSubs>(a, s);
    };
    if (group == 128) return of_group(std::integral_constant<int, 4>());
    if (group == 64) return of_group(std::integral_constant<int, 2>());
    return of_group(std::integral_constant<int, 1>());
  };
  const cudaError_t e = x_dtype == LSTM_APPROX_OP_FP32   ? of_type(std::integral_constant<int, LSTM_APPROX_OP_FP32>())
                        : x_dtype == LSTM_APPROX_OP_BF16 ? of_type(std::integral_constant<int, LSTM_APPROX_OP_BF16>())
                        : x_dtype == LSTM_APPROX_OP_FP16 ? of_type(std::integral_constant<int, LSTM_APPROX_OP_FP16>())
                                                         : of_type(std::integral_constant<int, LSTM_APPROX_OP_E4M3>());
  return op_launched(e, "matrix-vector launch", msg, msg_len);
}
