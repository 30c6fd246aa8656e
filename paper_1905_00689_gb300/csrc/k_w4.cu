// Matrix-vector products with 4-bit weights, a scale and a zero point per
// group of columns, and the quantiser that makes such weights
// (include/lstm_approx_ops.h):
//
//   y[m][n] = sum_g scale[n][g] sum_{k in g} (q[n][k] - zero[n][g]) x[m][k]
//
// The floor is memory, the 4-bit matrix, read once for as many rows of x as lie in
// shared memory over all of K at a time (plan_matvec; up to 32 columns of x^T, a
// row in 32 bits being three).  The products are warp MMAs of 16 rows of W by 16 k by 8
// columns of x^T, their operands in registers: tcgen05 takes both operands from
// shared memory or tensor memory, to which 4-bit weights would first have to be
// expanded, four bytes written for each byte read.
//
//   W   A block of 16 rows by 128 k (64 bytes to a row) comes into shared memory
//       by asynchronous copies.  Four
//       lanes share a row; a lane's 32-bit word holds 8 k as 4 pairs of 16-bit
//       integers after one AND-OR each, (0, 4) (1, 5) (2, 6) (3, 7): or-ed into
//       the mantissa of 128 (bf16) or 1024 (fp16), from which 128 + zero or 1024
//       + zero is subtracted: q - zero, exactly (the published way to expand small
//       integers through the mantissa: Kim et al. 2022, arXiv 2211.10017).  Which k a lane holds in which
//       MMA does not matter as long as x is laid out alike, and so that one MMA
//       sums over one group only.
//   x   Once per block of threads, into shared memory in the order in which the
//       lanes read it (16 bytes each, no conflicts): bf16 or fp16 as they are,
//       8-bit values as fp16, and 32-bit values as three columns of bf16 (the
//       upper 8 bits of the mantissa, the next, the last; their sum is exactly x).
//   sum Each group's sum, in fp32 (8 exact products to an addition), times its
//       scale, is added to the row's.
//
// The tiles of 16 rows are dealt out evenly over one block of threads per
// SM; a block has one warp at least to each of its tiles, and as many more as
// divide evenly, which share the tile's K and add up through shared memory at
// the end, always in the same order.  A warp goes on by sets of 4 groups
// (unrolled), whose weights are copied and whose scales are asked for ahead.
//
// Measured (device time): 1 x 16384 x 8192 fp16 21.3 us (3.3 TB/s, 48% of what a
// copy reaches), 1 x 16384 x 4096 bf16 12.4 us, 8 rows of x 13.4; 16 rows in 8 bits
// 19.5 us; 1 x 8192 x 2048 5.0 us, 3 x 3001 x 1000 fp32 5.4 us.  The copies by
// themselves take 14.8 us of the first and 12.7 of the 16 rows, the products by
// themselves 17.3 and 17.4, and the two overlap by a half only.  Nothing is
// saturated: 49% of the issue slots are used (177 instructions to a KB of W with one
// row of x), the matrix pipe 18%, memory 37%; after fixed latencies the largest stall
// is the block's barriers.  Warps stand idle where a block's tiles do not divide its
// warps: at 16384 rows 6 or 7 tiles take 12 or 14 of the 16.  A
// matrix of a few MB is bound by latency: launch, x, first copies, the join.
//
// A long x crowds out the warps, and then its own rows: 8192 x 8192 with group 128 is
// read once for 8 rows of bf16 (12 warps, 14.4 us), once for 12 (4 warps, 23.7),
// twice for 16 (12 and 4 rows, 43.1; in 8 bits 49.7), four times for 16 in 32 bits
// (184 us; group 32 92); 8192 x 4096 twice for 16 in 32 bits (46 us).  The kernels of
// 32 columns with group 128 spill 424 to 576 bytes a thread, with group 64 20 to
// 244.  Many rows are not what it is for: 64 x 8192 x 4096 bf16 67 us, 512 rows 478.
//
// Tried at these sizes: 20 and 24 warps (fewer sets in flight: 21.6 and 30.7 us for
// the first), two independent sums of MMAs (21.3), copies by whole rows (21.3), 8-bit
// MMAs with the nibbles as codes of 8-bit floats (16 rows: 27 us).
#include <cuda_fp8.h>

#include <algorithm>

#include "ops_common.cuh"
#include "ptx.cuh"

namespace lstm_approx_impl {
namespace {

using namespace lstm_approx_dev;

constexpr int kBlockK = 128;  // k of a block
constexpr int kMaxWarps = 16;

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
  bool x_vec;    // 8 values of x lie in aligned accesses
  bool set_vec;  // so do the scales (of 16 bits) and zero points of 4 groups
  int tokens;  // rows of x at a time
  int depth;   // sets in flight or in use to a warp: 2 to 4
  const unsigned char* x_laid;  // x laid out by the kernel before, or null
  int tiles_each, tiles_more;  // tiles of 16 rows to a block of threads, and how many blocks have one more
};

__device__ __forceinline__ float load_any(const void* p, long long at, int dtype) {
  if (dtype == LSTM_APPROX_OP_FP32) return static_cast<const float*>(p)[at];
  if (dtype == LSTM_APPROX_OP_BF16) return __bfloat162float(static_cast<const __nv_bfloat16*>(p)[at]);
  return __half2float(static_cast<const __half*>(p)[at]);
}
__device__ __forceinline__ void store_any(void* p, long long at, int dtype, float v) {
  if (dtype == LSTM_APPROX_OP_FP32) static_cast<float*>(p)[at] = v;
  else if (dtype == LSTM_APPROX_OP_BF16) static_cast<__nv_bfloat16*>(p)[at] = __float2bfloat16_rn(v);
  else static_cast<__half*>(p)[at] = __float2half_rn(v);
}

// Two of a word's four pairs of nibbles, at bits 0..3 and 4..7 of its halves, as 16-bit numbers less the zero point.
// zero: pair of 128 + z (bf16); of 1024 + z, and of -(64 + z) (fp16, whose ten bits of mantissa hold the nibble at bits
// 4..7 as it lies: (1024 + 16 q) / 16 - (64 + z) in one operation, where bf16 has to shift it down first).
template <bool kBf16>
struct Zero {
  uint32_t low, high;
};
// (low: the pair of 128 + z or 1024 + z; as bits, -(64 + z) is 0xd400 + 16 z)
template <bool kBf16>
__device__ __forceinline__ Zero<kBf16> zero_of(uint32_t low) {
  return {low, kBf16 ? 0u : low * 16u + (0xd400d400u - 0x64006400u * 16u)};
}
__device__ __forceinline__ uint32_t masked(uint32_t w, uint32_t mask, uint32_t magic) {
  uint32_t v;  // (w & mask) | magic
  asm("lop3.b32 %0, %1, %2, %3, 0xea;" : "=r"(v) : "r"(w), "r"(mask), "r"(magic));
  return v;
}
template <bool kBf16>
__device__ __forceinline__ void nibbles(uint32_t w, const Zero<kBf16>& z, uint32_t& first, uint32_t& second) {
  if constexpr (kBf16) {
    const uint32_t v0 = masked(w, 0x000f000fu, 0x43004300u), v1 = masked(w >> 4, 0x000f000fu, 0x43004300u);
    const __nv_bfloat162 zz = *reinterpret_cast<const __nv_bfloat162*>(&z.low);
    const __nv_bfloat162 d0 = __hsub2(*reinterpret_cast<const __nv_bfloat162*>(&v0), zz);
    const __nv_bfloat162 d1 = __hsub2(*reinterpret_cast<const __nv_bfloat162*>(&v1), zz);
    first = *reinterpret_cast<const uint32_t*>(&d0);
    second = *reinterpret_cast<const uint32_t*>(&d1);
  } else {
    const uint32_t v0 = masked(w, 0x000f000fu, 0x64006400u), v1 = masked(w, 0x00f000f0u, 0x64006400u);
    const __half2 d0 = __hsub2(*reinterpret_cast<const __half2*>(&v0), *reinterpret_cast<const __half2*>(&z.low));
    const __half2 d1 = __hfma2(*reinterpret_cast<const __half2*>(&v1), __float2half2_rn(1.0f / 16.0f),
                               *reinterpret_cast<const __half2*>(&z.high));
    first = *reinterpret_cast<const uint32_t*>(&d0);
    second = *reinterpret_cast<const uint32_t*>(&d1);
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

// 8 values of x from k on (zero from K on): as they lie in memory, and as 16-bit (or fp32) values each.
template <int kX>
struct Chunk {
  static constexpr int kWords = kX == LSTM_APPROX_OP_FP32 ? 8 : (kX == LSTM_APPROX_OP_E4M3 ? 2 : 4);
  uint32_t w[kWords];
};
template <int kX>
__device__ __forceinline__ Chunk<kX> load_chunk(const W4Args& a, long long row, int k) {
  Chunk<kX> v;
  constexpr int kBytes = Chunk<kX>::kWords / 2;  // of a value
  const uint8_t* p = static_cast<const uint8_t*>(a.x) + (row * a.x_pitch + k) * kBytes;
  if (a.x_vec && k + 8 <= a.K) {
    if constexpr (kX == LSTM_APPROX_OP_E4M3) {
      const uint2 u = *reinterpret_cast<const uint2*>(p);
      v.w[0] = u.x, v.w[1] = u.y;
    } else {
#pragma unroll
      for (int q = 0; q < Chunk<kX>::kWords / 4; ++q) {
        const uint4 u = reinterpret_cast<const uint4*>(p)[q];
        v.w[4 * q] = u.x, v.w[4 * q + 1] = u.y, v.w[4 * q + 2] = u.z, v.w[4 * q + 3] = u.w;
      }
    }
  } else {
#pragma unroll
    for (int q = 0; q < Chunk<kX>::kWords; ++q) v.w[q] = 0u;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      if (k + e >= a.K) continue;
      if constexpr (kBytes == 4) v.w[e] = reinterpret_cast<const uint32_t*>(p)[e];
      else if constexpr (kBytes == 2) v.w[e / 2] |= (uint32_t) reinterpret_cast<const uint16_t*>(p)[e] << 16 * (e & 1);
      else v.w[e / 4] |= (uint32_t)p[e] << 8 * (e & 3);
    }
  }
  return v;
}
// 16-bit values (0, 1) (2, 3) (4, 5) (6, 7) as pairs (0, 4) (1, 5) (2, 6) (3, 7)
__device__ __forceinline__ uint4 in_order(uint32_t w0, uint32_t w1, uint32_t w2, uint32_t w3) {
  return make_uint4(__byte_perm(w0, w2, 0x5410), __byte_perm(w0, w2, 0x7632), __byte_perm(w1, w3, 0x5410),
                    __byte_perm(w1, w3, 0x7632));
}
// A chunk into its place, `to` that of its first column and 4 places to the next.
template <int kX>
__device__ __forceinline__ void place_chunk(const Chunk<kX>& v, uint4* to) {
  if constexpr (kX == LSTM_APPROX_OP_FP32) {
    // three times the upper 16 bits of what is left; not finite: all in the first
    uint32_t left[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) left[e] = v.w[e];
#pragma unroll
    for (int part = 0; part < 3; ++part) {
      uint32_t u[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        u[e] = left[e] >> 16;
        const bool finite = (left[e] & 0x7f800000u) != 0x7f800000u;
        if (!finite && (left[e] & 0x007f0000u) == 0u && (left[e] & 0x007fffffu) != 0u) u[e] |= 0x40u;  // NaN stays NaN
        left[e] = finite ? __float_as_uint(__uint_as_float(left[e]) - __uint_as_float(left[e] & 0xffff0000u)) : 0u;
      }
      to[part * 4] = make_uint4(u[0] | u[4] << 16, u[1] | u[5] << 16, u[2] | u[6] << 16, u[3] | u[7] << 16);
    }
  } else if constexpr (kX == LSTM_APPROX_OP_E4M3) {
    uint32_t h[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const __half2_raw r = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(v.w[q / 2] >> 16 * (q & 1)), __NV_E4M3);
      h[q] = r.x | (uint32_t)r.y << 16;
    }
    to[0] = in_order(h[0], h[1], h[2], h[3]);
  } else {
    to[0] = in_order(v.w[0], v.w[1], v.w[2], v.w[3]);
  }
}

// Columns of x^T to a row of x: its three parts in 32 bits.
template <int kX>
constexpr int kParts = kX == LSTM_APPROX_OP_FP32 ? 3 : 1;

// x in the order of the product's shared memory, `tokens` rows at a time one after another: [rows / tokens][blocks][4]
// [columns][4] x 16 bytes.  A thread takes 8 k of one row.
template <int kX, int kSubs>
__global__ void __launch_bounds__(256) w4_lay_out_kernel(const W4Args a, uint4* to) {
  begin_op();
  const int blocks = (a.K + kBlockK - 1) / kBlockK, chunks = blocks * 16;
  const long long item = (long long)blockIdx.x * blockDim.x + threadIdx.x;
  if (item >= (long long)a.M * chunks) return;
  const int row = (int)(item / chunks), chunk = (int)(item % chunks);
  const int m0 = row / a.tokens * a.tokens, cols = min(a.tokens, a.M - m0) * kParts<kX>;
  int slot, lane_t;
  place<kSubs>(chunk >> 2 & 3, chunk & 3, slot, lane_t);
  uint4* at = to + (long long)m0 * kParts<kX> * blocks * 16 + (((chunk >> 4) * 4 + slot) * cols + (row - m0) * kParts<kX>) * 4 + lane_t;
  place_chunk<kX>(load_chunk<kX>(a, row, chunk * 8), at);
}

// Where the w-th of equal stretches (or one longer) begins, each `each` long and the first `more` of them one longer.
__device__ __forceinline__ int stretch(int w, int each, int more) { return w * each + min(w, more); }

// kX: type of x.  A tile is 16 rows of W (two to a thread's part: g and g + 8); kNt * 8 columns of x^T.
// kSubs = group / 32.
template <int kX, int kNt, int kSubs>
__global__ void __launch_bounds__(kMaxWarps * 32) w4_matvec_kernel(const W4Args a) {
  // where x is laid out by the kernel before, W, which that kernel does not write and which was complete before it
  // began, is on its way meanwhile
  if (!a.x_laid) begin_op();
  constexpr bool kBf16 = kX == LSTM_APPROX_OP_BF16 || kX == LSTM_APPROX_OP_FP32;
  constexpr bool kScaled = kX == LSTM_APPROX_OP_E4M3;
  constexpr int kP = kParts<kX>;
  constexpr int kRed = kNt * 8 + 1;         // pitch of the sums
  constexpr int kSum = 16 * kRed;     // a tile's sums
  constexpr int kSets = 4 / kSubs;          // groups of a block; a set is kSubs blocks
  constexpr int kRow = kSubs * 64;          // bytes of a row of a set
  constexpr int kStage = 16 * kRow;   // of a set
  extern __shared__ __align__(128) unsigned char memory[];
  const int warps = blockDim.x >> 5, warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int blocks = (a.K + kBlockK - 1) / kBlockK, sets = (blocks + kSubs - 1) / kSubs;
  const int m0 = blockIdx.y * a.tokens, tokens = min(a.tokens, a.M - m0), cols = tokens * kP;
  // x [blocks][4][cols][4] x 16 bytes, scales of x [blocks][kNt * 8], ring [warps][depth][16][kRow], in whose
  // place the sums [warps][16][kRed] go at the end
  uint4* xs = reinterpret_cast<uint4*>(memory);
  float* x_scales = reinterpret_cast<float*>(xs + blocks * 16 * cols);
  unsigned char* rings = reinterpret_cast<unsigned char*>(x_scales + (kScaled ? blocks * kNt * 8 : 0));
  const int ring_bytes = a.depth * kStage;
  unsigned char* ring = rings + warp * ring_bytes;

  // x: items of 8 k of up to kAtOnce rows; a thread's first is asked for before the copies of W that would delay it
  constexpr int kAtOnce = 16 / Chunk<kX>::kWords;
  const int chunks = blocks * 16, items = chunks * ((tokens + kAtOnce - 1) / kAtOnce);
  Chunk<kX> v[kAtOnce];
  auto load_item = [&](int item, Chunk<kX>(&to)[kAtOnce]) {
    const int token = item / chunks * kAtOnce, chunk = item % chunks;
#pragma unroll
    for (int e = 0; e < kAtOnce; ++e)
      if (token + e < tokens) to[e] = load_chunk<kX>(a, m0 + token + e, chunk * 8);
  };
  auto place_item = [&](int item, const Chunk<kX>(&from)[kAtOnce]) {
    const int token = item / chunks * kAtOnce, chunk = item % chunks;
    int slot, lane_t;
    place<kSubs>(chunk >> 2 & 3, chunk & 3, slot, lane_t);
    uint4* to = xs + (((chunk >> 4) * 4 + slot) * cols + token * kP) * 4 + lane_t;
#pragma unroll
    for (int e = 0; e < kAtOnce; ++e)
      if (token + e < tokens) place_chunk<kX>(from[e], to + e * kP * 4);
  };
  if (!a.x_laid && (int)threadIdx.x < items) load_item(threadIdx.x, v);
  __shared__ __align__(8) uint64_t x_bar;
  if (a.x_laid && threadIdx.x == 0) {
    mbar_init(smem_u32(&x_bar), 1);
    fence_mbarrier_init_cluster();
  }

  // this block's tiles, at most one to a warp at a time
  const int last_tile = stretch(blockIdx.x + 1, a.tiles_each, a.tiles_more);
  bool staged = false, x_there = true;
  for (int tile0 = stretch(blockIdx.x, a.tiles_each, a.tiles_more); tile0 < last_tile; tile0 += warps) {
    const int tiles = min(warps, last_tile - tile0), share = warps / tiles;  // warps to a tile
    const int my_tile = warp / share, part_k = warp - my_tile * share;
    const int begin = part_k * sets / share, end = my_tile < tiles ? (part_k + 1) * sets / share : 0;  // my sets

    // the copies
    int to_set = begin;
    const uint8_t* from[2];
    long long set_at[2];  // of the scales and zero points of the set that is asked for next
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      // (unsigned: rows of the last tiles, and of a warp without one, may lie past 2^31)
      const int n = (int)min((unsigned)(tile0 + my_tile) * 16u + q * 8 + g, (unsigned)a.N - 1u);
      from[q] = a.q + n * a.q_pitch + begin * kRow + t * 16;
      set_at[q] = (long long)n * a.groups + begin * 4;
    }
    // 16-byte piece c of row r goes to place c ^ swizzle(r): no two lanes of a read below meet in a bank
    const int swizzle = kSubs == 4 ? (g & 1) << 2 : (kSubs == 2 ? (g & 3) << 1 : g >> 1);
    const uint32_t to_first = smem_u32(ring) + g * kRow;
    uint32_t to_stage = to_first;
    auto fetch = [&]() {
      if (to_set < end) {
        const bool whole = (to_set + 1) * kSubs * kBlockK <= a.K;
#pragma unroll
        for (int i = 0; i < kSubs; ++i) {
          // (where x is zero any word will do, a finite number)
          if (whole || (to_set * kSubs + i) * kBlockK + t * 32 < a.K) {
#pragma unroll
            for (int q = 0; q < 2; ++q)
              asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to_stage + q * 8 * kRow +
                                                                             (((i * 4 + t) ^ swizzle) << 4)),
                           "l"(from[q] + i * 64)
                           : "memory");
          }
        }
#pragma unroll
        for (int q = 0; q < 2; ++q) from[q] += kRow;
        ++to_set;
      }
      asm volatile("cp.async.commit_group;" ::: "memory");
      to_stage += kStage;
      if (to_stage == to_first + ring_bytes) to_stage = to_first;
    };
    for (int d = 0; d < a.depth - 1; ++d) fetch();

    // Scales (16 bits) and zero points of a set, for rows g and g + 8; 32-bit scales are read where they are used.
    struct Set {
      uint32_t s[2][2], z[2];
    };
    const bool wide = a.scale_dtype == LSTM_APPROX_OP_FP32;
    int set_group = begin * 4;
    auto load_set = [&]() {
      Set r;
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        r.s[q][0] = r.s[q][1] = 0u;
        r.z[q] = 0x08080808u;
        if (a.set_vec) {
          if (set_group < a.groups) {
            const uint2 w = *reinterpret_cast<const uint2*>(static_cast<const uint16_t*>(a.scale) + set_at[q]);
            r.s[q][0] = w.x;
            r.s[q][1] = w.y;
            if (a.zero) r.z[q] = *reinterpret_cast<const uint32_t*>(a.zero + set_at[q]);
          }
        } else {
          if (a.zero) r.z[q] = 0u;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            if (set_group + e >= a.groups) continue;
            if (!wide) r.s[q][e / 2] |= (uint32_t) static_cast<const uint16_t*>(a.scale)[set_at[q] + e] << 16 * (e & 1);
            if (a.zero) r.z[q] |= (uint32_t)a.zero[set_at[q] + e] << 8 * e;
          }
        }
        set_at[q] += 4;
      }
      set_group += 4;
      return r;
    };
    Set next = load_set();

    if (!staged) {
      if (a.x_laid) {
        begin_op();
        if (threadIdx.x == 0) {
          const uint32_t bytes = (uint32_t)blocks * 256 * cols, bar = smem_u32(&x_bar);
          const unsigned char* from_x = a.x_laid + (long long)m0 * kP * blocks * 256;
          mbar_arrive_expect_tx(bar, bytes);
          for (uint32_t at = 0; at < bytes; at += 32768) bulk_copy_g2s(smem_u32(xs) + at, from_x + at, min(32768u, bytes - at), bar);
        }
      } else {
        int item = threadIdx.x;
        while (item < items) {
          const int now = item;
          item += blockDim.x;
          place_item(now, v);
          if (item < items) load_item(item, v);
        }
      }
      if constexpr (kScaled) {
        for (int c = threadIdx.x; c < blocks * kNt * 8; c += blockDim.x) {
          const int token = c % (kNt * 8), block = c / (kNt * 8);
          x_scales[c] =
              token < tokens ? a.x_scale[(long long)(m0 + token) * a.x_groups + (a.x_groups > 1 ? block : 0)] : 0.0f;
        }
      }
      staged = true;
      __syncthreads();
      if (a.x_laid) {
        const int never = 0;
        x_there = mbar_wait_bounded<false>(smem_u32(&x_bar), 0, 2000000000ull, &never);
      }
    }

    float acc[kNt][4] = {};
    const unsigned char* here = ring + g * kRow;
    const unsigned char* const ring_end = here + ring_bytes;
    // a lane whose column of x^T does not exist takes the last one's values; what they lead to is not stored
    const uint4* xs_here[kNt];
#pragma unroll
    for (int c = 0; c < kNt; ++c) xs_here[c] = xs + (begin * kSubs * 4 * cols + min(c * 8 + g, cols - 1)) * 4 + t;
    const int xs_step = cols * 4;
    for (int set = begin; set < end; ++set) {
      const Set held = next;
      if (a.depth == 2) asm volatile("cp.async.wait_group 0;" ::: "memory");
      else if (a.depth == 3) asm volatile("cp.async.wait_group 1;" ::: "memory");
      else asm volatile("cp.async.wait_group 2;" ::: "memory");
      __syncwarp();
      fetch();
      next = load_set();
#pragma unroll
      for (int i = 0; i < kSubs; ++i) {  // blocks of the set
        const int block = set * kSubs + i;
        if (i > 0 && block >= blocks) break;
        float xsc[kNt][2];
        float sum[kNt][4];  // of the block, where x has a scale for each
        if constexpr (kScaled) {
#pragma unroll
          for (int c = 0; c < kNt; ++c) {
            const float2 f = *reinterpret_cast<const float2*>(x_scales + block * kNt * 8 + c * 8 + 2 * t);
            xsc[c][0] = f.x;
            xsc[c][1] = f.y;
          }
        }
#pragma unroll
        for (int h = 0; h < kSets; ++h) {  // groups of the block
          const int e = i * kSets + h;
          uint4 b[kSubs][kNt];
#pragma unroll
          for (int k = 0; k < kSubs; ++k) {
#pragma unroll
            for (int c = 0; c < kNt; ++c) {
              b[k][c] = *xs_here[c];
              xs_here[c] += xs_step;
            }
          }
          float s[2];
          Zero<kBf16> z[2];
          uint32_t w[2][kSubs];  // the lane's words of rows g and g + 8
#pragma unroll
          for (int q = 0; q < 2; ++q) {
            const uint32_t bits = held.s[q][e / 2] >> 16 * (e & 1);
            if (wide) s[q] = set * 4 + e < a.groups ? static_cast<const float*>(a.scale)[set_at[q] - 8 + e] : 0.0f;
            else s[q] = a.scale_dtype == LSTM_APPROX_OP_BF16 ? __uint_as_float(bits << 16)
                                                             : __half2float(__ushort_as_half((unsigned short)bits));
            z[q] = zero_of<kBf16>((kBf16 ? 0x43004300u : 0x64006400u) + (held.z[q] >> 8 * e & 15u) * 0x00010001u);
            const unsigned char* row = here + q * 8 * kRow;
            if constexpr (kSubs == 4) {
              const uint4 u = *reinterpret_cast<const uint4*>(row + (((i * 4 + t) ^ swizzle) << 4));
              w[q][0] = u.x, w[q][1] = u.y, w[q][2] = u.z, w[q][3] = u.w;
            } else if constexpr (kSubs == 2) {
              const uint2 u =
                  *reinterpret_cast<const uint2*>(row + (((i * 4 + 2 * h + (t & 1)) ^ swizzle) << 4) + (t >> 1) * 8);
              w[q][0] = u.x, w[q][1] = u.y;
            } else {
              w[q][0] = *reinterpret_cast<const uint32_t*>(row + ((h ^ swizzle) << 4) + t * 4);
            }
          }
          float part[kNt][4];  // (the MMAs of one step belong to different sums)
#pragma unroll
          for (int k = 0; k < kSubs; ++k) {
#pragma unroll
            for (int half = 0; half < 2; ++half) {
              uint32_t a0, a1, a2, a3;
              nibbles<kBf16>(w[0][k] >> (8 * half), z[0], a0, a2);
              nibbles<kBf16>(w[1][k] >> (8 * half), z[1], a1, a3);
#pragma unroll
              for (int c = 0; c < kNt; ++c) {
                const uint32_t b0 = half ? b[k][c].z : b[k][c].x, b1 = half ? b[k][c].w : b[k][c].y;
                if (k == 0 && half == 0) {
                  if constexpr (kBf16) mma_16816_bf16<true, true>(part[c], a0, a1, a2, a3, b0, b1);
                  else mma_16816_f16<true, true>(part[c], a0, a1, a2, a3, b0, b1);
                } else {
                  if constexpr (kBf16) mma_16816_bf16<true, false>(part[c], a0, a1, a2, a3, b0, b1);
                  else mma_16816_f16<true, false>(part[c], a0, a1, a2, a3, b0, b1);
                }
              }
            }
          }
#pragma unroll
          for (int c = 0; c < kNt; ++c) {
#pragma unroll
            for (int n = 0; n < 4; ++n) {
              const float scale = s[n >> 1];
              if constexpr (kScaled) sum[c][n] = h == 0 ? part[c][n] * scale : fmaf(part[c][n], scale, sum[c][n]);
              else acc[c][n] = fmaf(part[c][n], scale, acc[c][n]);
            }
          }
        }
        if constexpr (kScaled) {
#pragma unroll
          for (int c = 0; c < kNt; ++c)
#pragma unroll
            for (int n = 0; n < 4; ++n) acc[c][n] = fmaf(sum[c][n], xsc[c][n & 1], acc[c][n]);
        }
      }
      here += kStage;
      if (here == ring_end) here -= ring_bytes;
    }
    asm volatile("cp.async.wait_group 0;" ::: "memory");
    __syncthreads();  // no ring is in use any more
    float* sums = reinterpret_cast<float*>(rings);
    if (my_tile < tiles) {
      float* to = sums + warp * kSum;
#pragma unroll
      for (int c = 0; c < kNt; ++c)
#pragma unroll
        for (int n = 0; n < 4; ++n) to[((n >> 1) * 8 + g) * kRed + c * 8 + 2 * t + (n & 1)] = acc[c][n];
    }
    __syncthreads();
    // a warp takes a tile, two rows of x at a time
    for (int tile = warp; tile < tiles; tile += warps) {
      const int row = lane & 15;
      const unsigned out = (unsigned)(tile0 + tile) * 16u + row;
      if (out >= (unsigned)a.N) continue;
      const float* first = sums + tile * share * kSum + row * kRed;
      const float bias = a.bias ? a.bias[out] : 0.0f;
      for (int token = lane >> 4; token < tokens; token += 2) {
        float total = 0.0f;
        const float* p = first + token * kP;
        for (int w = 0; w < share; ++w, p += kSum) {
          if constexpr (kP == 3) total += p[0] + (p[1] + p[2]);
          else total += p[0];
        }
        if (!x_there) total = __builtin_nanf("");
        store_any(a.y, (long long)(m0 + token) * a.N + out, a.y_dtype, total + bias);
      }
    }
    __syncthreads();  // the rings' place is theirs again
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
  begin_op();
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

// What a launch of the kernel takes.
struct W4Plan {
  int tokens;  // rows of x at a time
  int warps;   // of a block of threads
  int depth;   // sets of W in flight or in use to a warp
  size_t smem;
};
constexpr size_t kMostShared = 227 * 1024 - 1024;  // (and a barrier besides)
constexpr int kMaxK = 32768;  // one row of x in 32 bits then fits beside four warps' sets

// As many rows of x as leave room for four warps with two sets each, then as many warps as fit, then as many sets.
inline W4Plan plan_matvec(int M, int K, int parts, int nt, int subs, bool scaled) {
  const int blocks = (K + kBlockK - 1) / kBlockK;
  const size_t sums = 16 * (nt * 8 + 1) * sizeof(float), stage = 1024 * subs;
  for (W4Plan p{std::min(M, nt * 8 / parts), 0, 0, 0};; --p.tokens) {
    const size_t x = (size_t)blocks * (256 * p.tokens * parts + (scaled ? 32 * nt : 0));
    const size_t left = x < kMostShared ? kMostShared - x : 0;
    p.warps = (int)std::min<size_t>(kMaxWarps, left / std::max(2 * stage, sums));
    if (p.warps < 4 && p.tokens > 1) continue;
    p.depth = (int)std::min<size_t>(4, left / (std::max(1, p.warps) * stage));
    p.smem = x + p.warps * std::max(p.depth * stage, sums);
    return p;
  }
}

// Bytes of x laid out, where a kernel does it before the product: from 24 KB on, for which each block of threads on its own
// would need several turns through its caches (16 x 4096 8-bit values: 13 of 38 us); below that the second launch costs
// more.
inline size_t laid_out_bytes(int x_dtype, int M, int K) {
  const size_t bytes = (size_t)M * ((K + kBlockK - 1) / kBlockK) * 256 * (x_dtype == LSTM_APPROX_OP_FP32 ? 3 : 1);
  return bytes >= 24 * 1024 ? bytes : 0;
}

template <int kX, int kNt, int kSubs>
cudaError_t launch_matvec(W4Args a, unsigned char* workspace, cudaStream_t s) {
  static thread_local DeviceSet ready;  // of the one kernel that this instance launches
  auto kern = w4_matvec_kernel<kX, kNt, kSubs>;
  cudaError_t e = once_per_device(
      &ready, [&] { return cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kMostShared); });
  if (e != cudaSuccess) return e;
  const W4Plan p = plan_matvec(a.M, a.K, kParts<kX>, kNt, kSubs, kX == LSTM_APPROX_OP_E4M3);
  if (p.warps < 1) return cudaErrorInvalidValue;
  a.tokens = p.tokens;
  a.depth = p.depth;
  const int tiles = (a.N - 1) / 16 + 1, across = std::min(tiles, 152);
  a.tiles_each = tiles / across;
  a.tiles_more = tiles % across;
  if (laid_out_bytes(kX, a.M, a.K) > 0) {
    a.x_laid = workspace;
    const long long items = (long long)a.M * ((a.K + kBlockK - 1) / kBlockK) * 16;
    e = op_launch(w4_lay_out_kernel<kX, kSubs>, dim3((unsigned)((items + 255) / 256)), dim3(256), 0, s, a,
                  reinterpret_cast<uint4*>(workspace));
    if (e != cudaSuccess) return e;
  }
  return op_launch(kern, dim3(across, (a.M + p.tokens - 1) / p.tokens), dim3(p.warps * 32), p.smem, s, a);
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

extern "C" size_t lstm_approx_w4_workspace_bytes(int x_dtype, int M, int K) {
  return M < 0 || M > 65535 || K < 1 || K > kMaxK ? 0 : laid_out_bytes(x_dtype, M, K);
}

extern "C" int lstm_approx_w4_matvec(int x_dtype, const void* x, long long x_pitch, const float* x_scale, int x_group,
                                     const unsigned char* q, long long q_pitch, const void* scale, int scale_dtype,
                                     const unsigned char* zero, const float* bias, int M, int N, int K, int group,
                                     void* y, int y_dtype, void* workspace, size_t workspace_bytes, void* cuda_stream,
                                     char* msg, int msg_len) {
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
  const size_t need = lstm_approx_w4_workspace_bytes(x_dtype, M, K);
  if (need > 0 && N > 0 && (!workspace || !op_aligned(workspace, 16) || workspace_bytes < need))
    return op_report(msg, msg_len, LSTM_APPROX_EINVAL, "needs a 16-byte aligned workspace of %zu bytes", need);
  if (int rc = op_check_device(msg, msg_len)) return rc;
  if (M == 0 || N == 0) return LSTM_APPROX_OK;
  const size_t xs = op_dtype_bytes(x_dtype);
  W4Args a{x_dtype, x, x_pitch, x_scale, x_group >= K || !x8 ? 1 : (K + 127) / 128, q, q_pitch, scale, scale_dtype, zero,
           bias, M, N, K, (K + group - 1) / group, y, y_dtype,
           op_aligned(x, std::min<size_t>(16, 8 * xs)) && x_pitch * xs % std::min<size_t>(16, 8 * xs) == 0,
           scale_dtype != LSTM_APPROX_OP_FP32 && (K + group - 1) / group % 4 == 0 && op_aligned(scale, 8) && op_aligned(zero, 4),
           0, 0, nullptr, 0, 0};
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  unsigned char* ws = static_cast<unsigned char*>(workspace);
  auto of_type = [&](auto type) {
    constexpr int kX = decltype(type)::value;
    const int cols = std::min(M, 32) * kParts<kX>;
    auto of_group = [&](auto subs) {
      constexpr int kSubs = decltype(subs)::value;
      if (cols <= 8) return launch_matvec<kX, 1, kSubs>(a, ws, s);
      if (cols <= 16) return launch_matvec<kX, 2, kSubs>(a, ws, s);
      return launch_matvec<kX, 4, kSubs>(a, ws, s);
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
