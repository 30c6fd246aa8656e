// The gated delta rule over a sequence, forward and backward
// (include/lstm_approx_ops.h).
//
// For every stream and value head a state S [Dk][Dv]:
//
//   u_t = beta_t (v_t - e^{g_t} S_{t-1}^T k_t);  S_t = e^{g_t} S_{t-1} + k_t u_t^T;  o_t = scale S_t^T q_t
//
// By chunks of 64 timesteps (i, j: rows of a chunk; S0: the state before it; G: the sum of g up to and with a row):
//
//   D_ij = e^{G_i - G_j} (i >= j);  gam_i = e^{G_i};  dec_j = e^{G_63 - G_j}
//   A_ij = beta_i D_ij k_i . k_j (i > j);  Tm = (I + A)^-1;  M_ij = D_ij q_i . k_j
//   U = Tm diag(beta) (V - diag(gam) K S0);  O = scale (diag(gam) Q S0 + M U);  S = gam_63 S0 + K^T diag(dec) U
//
// and for the gradients (dS that of S, R = Tm^T dU):
//
//   dU = scale M^T dO + diag(dec) K dS;  dV = diag(beta) R
//   dS0 = gam_63 dS + Q^T diag(scale gam) dO - K^T diag(beta gam) R
//   P_ij = scale D_ij dO_i . u_j (i >= j);  E_ij = D_ij R_i . u_j (i > j);  w = diag(gam) R S0^T + E K
//   dQ = P K + diag(scale gam) dO S0^T;  t = P^T Q - E^T diag(beta) K + diag(dec) U dS^T;  dK = t - diag(beta) w
//   dbeta_i = R_i . v_i - k_i . w_i;  dG_i = q_i . dq_i - k_i . (beta_i w_i + t_i)
//   dG_63 += gam_63 <dS, S0> + sum_j dec_j k_j . (dS u_j);  dg_t = sum of dG_i over i >= t
//
// Kernels: one per chunk and head makes Tm and M; one per head and 16 or 32
// columns of S (which do not see one another) runs along the chunks, forward or
// backward; one per chunk makes the gradients of q, k, g and beta.
//
// Products run on the warp MMAs of 32-bit floats cut to 11 bits (m16n8k8): an
// operand that came in 16 bits is exact there, any other is taken in two parts,
// value = high + low, and two or three products are summed in 32 bits, which
// leaves 2^-21 of a factor at most.  A state carries thousands of timesteps, so
// these are not rounded to 16 bits.
//
// At a reset the state before counts as zero, and so does everything before it
// in its chunk: a chunk with resets is taken piece by piece, and rows of other
// pieces are left out, not multiplied by zero.
#include <algorithm>

#include "ops_common.cuh"

namespace lstm_approx_impl {
namespace {

using namespace lstm_approx_dev;

constexpr int C = LSTM_APPROX_DELTA_CHUNK;
static_assert(C == 64, "rows of a chunk");
constexpr int kThreads = 256;
constexpr float kLeastG = -200.0f;

// ---- matrices in shared memory and the products of warps ---------------------

// [64][W] values of T.  Every row's 16-byte pieces (16 bits) or 8-word groups (32 bits) are exchanged by a rule on the row, so
// that eight rows of a column, or a row's neighbours, lie in different banks.
template <typename T, int W>
struct Tile {
  T* p;
  __device__ __forceinline__ static int at(int row, int col) {
    if constexpr (sizeof(T) == 2) return row * W + (col ^ (row & 7) << 3);
    else return row * W + (col ^ ((row ^ row >> 2) & 3) << 3);
  }
  __device__ __forceinline__ float2 pair(int row, int col) const {
    return Pair<T>::get(*reinterpret_cast<const typename Pair<T>::Raw*>(p + at(row, col)));
  }
  __device__ __forceinline__ float one(int row, int col) const { return to_f32(p[at(row, col)]); }
};
// 32-bit values, rows LD apart.
template <int LD>
struct Padded {
  float* p;
  __device__ __forceinline__ float2 pair(int row, int col) const { return *reinterpret_cast<const float2*>(p + row * LD + col); }
  __device__ __forceinline__ float one(int row, int col) const { return p[row * LD + col]; }
  __device__ __forceinline__ float& to(int row, int col) { return p[row * LD + col]; }
};

// The products below are reached by whole warps: a barrier lies before each, and between that and the last of its loads and
// MMAs only branches that a warp's lanes take alike.
//
// Parts of the m16n8k8 MMA's operands: lane = 4 g + t holds rows g, g + 8 of A (columns 2 t, then 2 t + 1: the order of k is
// free as long as both agree) and column g of B.
struct FragA {
  float x[4];  // (g, 2t), (g + 8, 2t), (g, 2t + 1), (g + 8, 2t + 1)
};
struct FragB {
  float x[2];  // (2t, g), (2t + 1, g)
};

__device__ __forceinline__ int lane_g() { return (threadIdx.x & 31) >> 2; }
__device__ __forceinline__ int lane_t() { return threadIdx.x & 3; }

template <typename T>
__device__ __forceinline__ float2 unpack(uint32_t v) {
  return Pair<T>::get(*reinterpret_cast<const typename Pair<T>::Raw*>(&v));
}

// A of 16 rows and 16 columns of k from a tile whose rows are A's.
template <typename T, int W>
__device__ __forceinline__ void load_a(const Tile<T, W>& tile, int m0, int k0, FragA (&f)[2]) {
  if constexpr (sizeof(T) == 2) {
    const int l = threadIdx.x & 31;
    uint32_t r[4];
    ldmatrix4<true>(smem_u32(tile.p + tile.at(m0 + (l & 15), k0 + (l >> 4) * 8)), r);
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const float2 a = unpack<T>(r[2 * s]), b = unpack<T>(r[2 * s + 1]);
      f[s] = {{a.x, b.x, a.y, b.y}};
    }
  } else {
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const float2 a = tile.pair(m0 + lane_g(), k0 + 8 * s + 2 * lane_t()), b = tile.pair(m0 + 8 + lane_g(), k0 + 8 * s + 2 * lane_t());
      f[s] = {{a.x, b.x, a.y, b.y}};
    }
  }
}
template <int LD>
__device__ __forceinline__ void load_a(const Padded<LD>& m, int m0, int k0, FragA (&f)[2]) {
#pragma unroll
  for (int s = 0; s < 2; ++s) {
    const float2 a = m.pair(m0 + lane_g(), k0 + 8 * s + 2 * lane_t()), b = m.pair(m0 + 8 + lane_g(), k0 + 8 * s + 2 * lane_t());
    f[s] = {{a.x, b.x, a.y, b.y}};
  }
}
// The same from a tile whose columns are A's rows.
template <typename Mat>
__device__ __forceinline__ void load_at_words(const Mat& m, int m0, int k0, FragA (&f)[2]) {
#pragma unroll
  for (int s = 0; s < 2; ++s) {
    const int k = k0 + 8 * s + 2 * lane_t(), r = m0 + lane_g();
    f[s] = {{m.one(k, r), m.one(k, r + 8), m.one(k + 1, r), m.one(k + 1, r + 8)}};
  }
}
template <typename T, int W>
__device__ __forceinline__ void load_at(const Tile<T, W>& tile, int m0, int k0, FragA (&f)[2]) {
  if constexpr (sizeof(T) == 2) {
    const int l = threadIdx.x & 31;
    uint32_t r[4];
    ldmatrix4_trans<true>(smem_u32(tile.p + tile.at(k0 + (l & 7) + (l >> 4) * 8, m0 + (l >> 3 & 1) * 8)), r);
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const float2 a = unpack<T>(r[2 * s]), b = unpack<T>(r[2 * s + 1]);
      f[s] = {{a.x, b.x, a.y, b.y}};
    }
  } else {
    load_at_words(tile, m0, k0, f);
  }
}
template <int LD>
__device__ __forceinline__ void load_at(const Padded<LD>& m, int m0, int k0, FragA (&f)[2]) {
  load_at_words(m, m0, k0, f);
}

// B of 16 rows of k and 16 columns (f[column / 8][k / 8]) from a tile whose rows are B's columns.
template <typename T, int W>
__device__ __forceinline__ void load_b16(const Tile<T, W>& tile, int n0, int k0, FragB (&f)[2][2]) {
  if constexpr (sizeof(T) == 2) {
    const int l = threadIdx.x & 31;
    uint32_t r[4];
    ldmatrix4<true>(smem_u32(tile.p + tile.at(n0 + (l & 15), k0 + (l >> 4) * 8)), r);
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const float2 v = unpack<T>(r[q]);
      f[q & 1][q >> 1] = {{v.x, v.y}};
    }
  } else {
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const float2 v = tile.pair(n0 + 8 * (q & 1) + lane_g(), k0 + 8 * (q >> 1) + 2 * lane_t());
      f[q & 1][q >> 1] = {{v.x, v.y}};
    }
  }
}
// From a tile whose rows are B's.
template <typename T, int W>
__device__ __forceinline__ void load_bt16(const Tile<T, W>& tile, int n0, int k0, FragB (&f)[2][2]) {
  if constexpr (sizeof(T) == 2) {
    const int l = threadIdx.x & 31;
    uint32_t r[4];
    ldmatrix4_trans<true>(smem_u32(tile.p + tile.at(k0 + (l & 15), n0 + (l >> 4) * 8)), r);
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const float2 v = unpack<T>(r[q]);
      f[q >> 1][q & 1] = {{v.x, v.y}};
    }
  } else {
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int n = n0 + 8 * (q >> 1) + lane_g(), k = k0 + 8 * (q & 1) + 2 * lane_t();
      f[q >> 1][q & 1] = {{tile.one(k, n), tile.one(k + 1, n)}};
    }
  }
}
// 8 columns and 8 rows of k from 32-bit rows that are B's columns; that are B's rows.
template <int LD>
__device__ __forceinline__ FragB load_b(const Padded<LD>& m, int n0, int k0) {
  const float2 v = m.pair(n0 + lane_g(), k0 + 2 * lane_t());
  return {{v.x, v.y}};
}
template <int LD>
__device__ __forceinline__ FragB load_bt(const Padded<LD>& m, int n0, int k0) {
  return {{m.one(k0 + 2 * lane_t(), n0 + lane_g()), m.one(k0 + 2 * lane_t() + 1, n0 + lane_g())}};
}

// x = high + low: the MMA reads a sign, 8 bits of exponent and 10 of fraction.  high: x to the nearest of those (its further
// bits are not read); low: what is left, of either sign (cut off instead, x would lose 2^-22 of itself on average, and a long
// sequence of that shows: 9e-7 of o, so 4e-7).  Not finite values stay so in one of the two.
__device__ __forceinline__ float high(float x) { return __uint_as_float(__float_as_uint(x) + 0x1000u); }
__device__ __forceinline__ float low(float x) { return x - __uint_as_float((__float_as_uint(x) + 0x1000u) & 0xffffe000u); }

// d + e += a b: the high parts' product to d, the others to e (two chains of sums; d and e may be the same).
// kOneA, kOneB: the operand is exact in 11 bits.
template <bool kOneA, bool kOneB>
__device__ __forceinline__ void mma(float (&d)[4], float (&e)[4], const FragA& a, const FragB& b) {
  float ah[4], bh[2];
#pragma unroll
  for (int i = 0; i < 4; ++i) ah[i] = kOneA ? a.x[i] : high(a.x[i]);
#pragma unroll
  for (int i = 0; i < 2; ++i) bh[i] = kOneB ? b.x[i] : high(b.x[i]);
  if constexpr (!kOneB) mma_1688_tf32<true>(e, ah[0], ah[1], ah[2], ah[3], low(b.x[0]), low(b.x[1]));
  if constexpr (!kOneA) mma_1688_tf32<true>(e, low(a.x[0]), low(a.x[1]), low(a.x[2]), low(a.x[3]), bh[0], bh[1]);
  mma_1688_tf32<true>(d, ah[0], ah[1], ah[2], ah[3], bh[0], bh[1]);
}

// ---- what the kernels share ----------------------------------------------------

struct Gates {  // of a chunk and head
  float gam[C], dec[C], beta[C], g_high[C], g_low[C];
  unsigned long long cuts;  // bit i: a reset at row i
  unsigned long long pad;
};
static_assert(sizeof(Gates) % 16 == 0, "copied in 16-byte pieces");

// Row strides of a tensor [T][B][heads][D].
struct Strides {
  long long t, b, h;
};

struct DeltaArgs {
  const void *q, *k, *v, *d_o;
  const float *g, *beta;
  long long gt, gb, bt, bb;
  Strides qs, ks, vs, os, dos, dqs, dks, dvs;
  float scale;
  const float* h0;
  const int32_t* lengths;
  const unsigned char* reset;
  int T, B, H, share, Dk, Dv, tiles;
  bool wide;   // q and k in 16-byte pieces
  bool pairs;  // v, o, dO and dV two at a time
  void* o;
  float *h_last, *states;
  // workspace: per chunk, stream and head
  float *Tm, *M;
  Gates* gates;
  // backward
  const float* dh_last;
  float *dS, *R, *sum_q, *sum_k;
  void *dq, *dk, *dv;
  float *dg, *dbeta, *dh0;
  long long dgt, dgb, dbt, dbb;
};

__device__ __forceinline__ int length_of(const DeltaArgs& a, int b) {
  return a.lengths ? min(max(a.lengths[b], 0), a.T) : a.T;
}

__device__ __forceinline__ void copy16(void* to, const void* from, int bytes) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(smem_u32(to)), "l"(from), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int kLeft>
__device__ __forceinline__ void copies_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(kLeft) : "memory");
}

// Rows [lo, hi) of a chunk of q or k; zeros elsewhere and past Dk.  p: the chunk's first row.
template <typename T, int W>
__device__ __forceinline__ void fetch_tile(Tile<T, W> to, const T* p, long long t_stride, int lo, int hi, int Dk, bool wide) {
  constexpr int kPer = 16 / (int)sizeof(T);
  for (int i = threadIdx.x; i < C * (W / kPer); i += kThreads) {
    const int row = i / (W / kPer), col = i % (W / kPer) * kPer;
    T* dst = to.p + to.at(row, col);
    const bool in = row >= lo && row < hi;
    if (wide) {
      const bool some = in && col < Dk;
      copy16(dst, some ? p + row * t_stride + col : p, some ? 16 : 0);
    } else {
      T x[kPer];
#pragma unroll
      for (int e = 0; e < kPer; ++e) x[e] = in && col + e < Dk ? p[row * t_stride + col + e] : from_f32<T>(0.0f);
      *reinterpret_cast<uint4*>(dst) = *reinterpret_cast<const uint4*>(x);
    }
  }
}
template <typename P>
__device__ __forceinline__ void fetch_plain(P* to, const P* from, int bytes) {
  for (int i = threadIdx.x; i < bytes / 16; i += kThreads)
    copy16(reinterpret_cast<char*>(to) + i * 16, reinterpret_cast<const char*>(from) + i * 16, 16);
}

// Two neighbouring values of a row (the second only if it lies in the row).
template <typename T>
__device__ __forceinline__ float2 get2(const T* row, int col, int D, bool pairs) {
  if (pairs) return col < D ? Pair<T>::get(*reinterpret_cast<const typename Pair<T>::Raw*>(row + col)) : make_float2(0.0f, 0.0f);
  return make_float2(col < D ? to_f32(row[col]) : 0.0f, col + 1 < D ? to_f32(row[col + 1]) : 0.0f);
}
template <typename T>
__device__ __forceinline__ void put2(T* row, int col, int D, bool pairs, float x, float y) {
  if (pairs) {
    if (col < D) *reinterpret_cast<typename Pair<T>::Raw*>(row + col) = Pair<T>::put(x, y);
  } else {
    if (col < D) row[col] = from_f32<T>(x);
    if (col + 1 < D) row[col + 1] = from_f32<T>(y);
  }
}

// The piece of a chunk that begins at row lo ends before this row.
__device__ __forceinline__ int piece_end(unsigned long long cuts, int lo) {
  const unsigned long long behind = lo >= 63 ? 0ull : cuts >> (lo + 1);
  return behind ? lo + __ffsll((long long)behind) : C;
}
// Whether a reset lies at or before the row.
__device__ __forceinline__ bool cut_before(unsigned long long cuts, int row) { return (cuts << (63 - row)) != 0ull; }

// Whether one lies behind row j and not behind row i >= j.
__device__ __forceinline__ bool cut_between(unsigned long long cuts, int j, int i) {
  return i > j && cuts >> (j + 1) << (64 - (i - j)) != 0ull;
}

// ---- per chunk and head: gates, Tm and M ----------------------------------------

template <typename T, int KD>
__global__ void __launch_bounds__(kThreads) delta_prepare_kernel(const DeltaArgs a) {
  extern __shared__ __align__(128) unsigned char smem[];
  Tile<T, KD> K{reinterpret_cast<T*>(smem)}, Q{K.p + C * KD};
  Padded<C + 4> A{reinterpret_cast<float*>(Q.p + C * KD)}, Ti{A.p + C * (C + 4)};
  Gates& gates = *reinterpret_cast<Gates*>(Ti.p + C * (C + 4));
  begin_op();
  const long long chunk = blockIdx.x;  // (n B + b) H + h
  const int h = (int)(chunk % a.H), b = (int)(chunk / a.H % a.B), n = (int)(chunk / a.H / a.B);
  const int t0 = n * C, rows = min(length_of(a, b) - t0, C);
  if (rows <= 0) return;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const T* k = static_cast<const T*>(a.k) + t0 * a.ks.t + b * a.ks.b + (h / a.share) * a.ks.h;
  const T* q = static_cast<const T*>(a.q) + t0 * a.qs.t + b * a.qs.b + (h / a.share) * a.qs.h;
  fetch_tile(K, k, a.ks.t, 0, rows, a.Dk, a.wide);
  fetch_tile(Q, q, a.qs.t, 0, rows, a.Dk, a.wide);
  copies_commit();
  if (warp == 0) {  // rows lane and lane + 32; the sums in 64 bits: differences of far sums keep their digits
    double G[2];
    unsigned cut[2];
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const int row = lane + 32 * s, t = t0 + row;
      float g = 0.0f, beta = 0.0f;
      bool reset = false;
      if (row < rows) {
        g = a.g[t * a.gt + b * a.gb + h];
        g = g < kLeastG ? kLeastG : g;
        beta = a.beta[t * a.bt + b * a.bb + h];
        reset = a.reset && a.reset[(long long)t * a.B + b];
      }
      gates.beta[row] = beta;
      cut[s] = __ballot_sync(0xffffffffu, reset);
      // from the last reset on; the row of the reset counts as zero (its state before does not pass)
      const unsigned before = cut[s] & (2u << lane) - 1u;
      const int start = before ? 31 - __clz((int)before) : 0;
      double x = reset ? 0.0 : (double)g;
#pragma unroll
      for (int d = 1; d < 32; d *= 2) {
        const double y = __shfl_up_sync(0xffffffffu, x, d);
        if (lane - d >= start) x += y;
      }
      G[s] = x;
    }
    const double first = __shfl_sync(0xffffffffu, G[0], 31);
    if (!(cut[1] & (2u << lane) - 1u)) G[1] += first;
    const double last = __shfl_sync(0xffffffffu, G[1], 31);
    const unsigned long long cuts = cut[0] | (unsigned long long)cut[1] << 32;
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const int row = lane + 32 * s;
      const float high = (float)G[s], rest = (float)(G[s] - (double)high), e = expf(high);
      gates.g_high[row] = high;
      gates.g_low[row] = rest;
      gates.gam[row] = cut_before(cuts, row) ? 0.0f : fmaf(e, rest, e);
      gates.dec[row] = row < 63 && cuts >> (row + 1) ? 0.0f : expf((float)(last - G[s]));
    }
    if (lane == 0) gates.cuts = cuts;
  }
  copies_wait<0>();
  __syncthreads();

  // K K^T and Q K^T where j <= i: ten blocks of 16 x 16 each
  const unsigned long long cuts = gates.cuts;
  float* M = a.M + chunk * C * C;
  for (int task = warp; task < 20; task += 8) {
    const int block = task % 10;
    const int bi = block < 1 ? 0 : block < 3 ? 1 : block < 6 ? 2 : 3, bj = block - bi * (bi + 1) / 2;
    const bool keys = task < 10;
    float d[2][4] = {}, e[2][4] = {};
    constexpr bool kOne = sizeof(T) == 2;
#pragma unroll
    for (int k0 = 0; k0 < KD; k0 += 16) {
      FragA fa[2];
      FragB fb[2][2];
      load_a(keys ? K : Q, bi * 16, k0, fa);
      load_b16(K, bj * 16, k0, fb);
#pragma unroll
      for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int x = 0; x < 2; ++x) mma<kOne, kOne>(d[x], kOne ? d[x] : e[x], fa[s], fb[x][s]);
    }
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int i = bi * 16 + lane_g() + 8 * (r >> 1), j = bj * 16 + x * 8 + 2 * lane_t() + (r & 1);
        const float dist = (gates.g_high[i] - gates.g_high[j]) + (gates.g_low[i] - gates.g_low[j]);
        const bool same = i >= j && !cut_between(cuts, j, i);
        const float v = same ? expf(dist) * (d[x][r] + e[x][r]) : 0.0f;
        if (keys) A.to(i, j) = i > j ? gates.beta[i] * v : 0.0f;
        else M[Tile<float, C>::at(i, j)] = v;
      }
  }
  __syncthreads();

  // (I + A)^-1: the 16 x 16 blocks on the diagonal column by column, then [L 0; X R]^-1 = [L^-1 0; -R^-1 X L^-1 R^-1]
  if (warp < 4 && lane < 16) {
    const int o = warp * 16;
    float x[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      float s = i == lane ? 1.0f : 0.0f;
#pragma unroll
      for (int j = 0; j < i; ++j) s = fmaf(-A.one(o + i, o + j), x[j], s);
      x[i] = i < lane ? 0.0f : s;  // (whatever the rows of another document hold)
      Ti.to(o + i, o + lane) = x[i];
    }
  }
  __syncthreads();
#pragma unroll
  for (int half = 16; half < C; half *= 2) {
    const int per = half * half, count = C / (2 * half) * per;  // outputs of all blocks of this size
    // X L^-1 goes where A's block above the diagonal lies (never read)
    for (int i = threadIdx.x; i < count; i += kThreads) {
      const int o = i / per * 2 * half, r = i % per / half, c = i % half;
      float s = 0.0f;
      for (int j = c; j < half; ++j) s = fmaf(A.one(o + half + r, o + j), Ti.one(o + j, o + c), s);
      A.to(o + r, o + half + c) = s;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < count; i += kThreads) {
      const int o = i / per * 2 * half, r = i % per / half, c = i % half;
      float s = 0.0f;
      for (int j = 0; j <= r; ++j) s = fmaf(Ti.one(o + half + r, o + half + j), A.one(o + j, o + half + c), s);
      Ti.to(o + half + r, o + c) = -s;
    }
    __syncthreads();
  }
  float* Tm = a.Tm + chunk * C * C;
  for (int x = threadIdx.x; x < C * C; x += kThreads) {
    const int i = x / C, j = x % C;
    const bool same = i >= j && !cut_between(cuts, j, i);
    Tm[Tile<float, C>::at(i, j)] = same ? Ti.one(i, j) : 0.0f;
  }
  for (int i = threadIdx.x; i < (int)sizeof(Gates) / 4; i += kThreads)
    reinterpret_cast<unsigned*>(a.gates + chunk)[i] = reinterpret_cast<const unsigned*>(&gates)[i];
}

template <typename T, int KD>
constexpr size_t prepare_smem() {
  return 2 * C * KD * sizeof(T) + 2 * C * (C + 4) * 4 + sizeof(Gates);
}

// ---- along the chunks, forward ---------------------------------------------------

// What a chunk brings along for a run over the chunks.
template <typename T, int KD>
struct Stage {
  Tile<T, KD> K, Q;
  Tile<float, C> Tm, M;
  Gates* gates;
  static constexpr size_t kBytes = 2 * C * KD * sizeof(T) + 2 * C * C * 4 + sizeof(Gates);
  __device__ __forceinline__ explicit Stage(unsigned char* p)
      : K{reinterpret_cast<T*>(p)}, Q{K.p + C * KD}, Tm{reinterpret_cast<float*>(Q.p + C * KD)}, M{Tm.p + C * C},
        gates(reinterpret_cast<Gates*>(M.p + C * C)) {}
  __device__ __forceinline__ void fetch(const DeltaArgs& a, int n, int b, int h, int len) const {
    const int t0 = n * C, rows = min(len - t0, C);
    const long long chunk = ((long long)n * a.B + b) * a.H + h;
    fetch_tile(K, static_cast<const T*>(a.k) + t0 * a.ks.t + b * a.ks.b + (h / a.share) * a.ks.h, a.ks.t, 0, rows, a.Dk, a.wide);
    fetch_tile(Q, static_cast<const T*>(a.q) + t0 * a.qs.t + b * a.qs.b + (h / a.share) * a.qs.h, a.qs.t, 0, rows, a.Dk, a.wide);
    fetch_plain(Tm.p, a.Tm + chunk * C * C, C * C * 4);
    fetch_plain(M.p, a.M + chunk * C * C, C * C * 4);
    fetch_plain(gates, a.gates + chunk, (int)sizeof(Gates));
  }
};

// A block's part of the state: 16 rows of S (a warp's) and kTiles times 8 columns in the MMA's result layout.
template <int KD, int NV>
struct StatePart {
  static constexpr int kGroups = 8 / (KD / 16), kTiles = NV / 8 / kGroups;  // warps that share rows; column tiles to each
  float x[kTiles][4];
  __device__ __forceinline__ static int row0() { return (threadIdx.x >> 5) % (KD / 16) * 16; }
  __device__ __forceinline__ static int col0() { return (threadIdx.x >> 5) / (KD / 16) * (NV / kGroups); }
  template <typename F>
  __device__ __forceinline__ void each(F f) {  // f(row, column, value)
#pragma unroll
    for (int n = 0; n < kTiles; ++n)
#pragma unroll
      for (int r = 0; r < 4; ++r) f(row0() + lane_g() + 8 * (r >> 1), col0() + n * 8 + 2 * lane_t() + (r & 1), x[n][r]);
  }
  __device__ __forceinline__ void load(const float* p, int Dk, int Dv, int v0) {
    each([&](int r, int c, float& v) { v = p && r < Dk && v0 + c < Dv ? p[(long long)r * Dv + v0 + c] : 0.0f; });
  }
  __device__ __forceinline__ void store(float* p, int Dk, int Dv, int v0) {
    each([&](int r, int c, float& v) {
      if (r < Dk && v0 + c < Dv) p[(long long)r * Dv + v0 + c] = v;
    });
  }
};

template <typename T, int KD, int NV>
__global__ void __launch_bounds__(kThreads, 1) delta_forward_kernel(const DeltaArgs a) {
  extern __shared__ __align__(128) unsigned char smem[];
  constexpr int kTiles = NV / 16;  // column tiles of a warp's 16 rows of the chunk: half of the columns
  constexpr bool kOne = sizeof(T) == 2;
  using St = Stage<T, KD>;
  // [column][row]: the state before the chunk, and the next
  const Padded<KD + 8> S{reinterpret_cast<float*>(smem + 2 * St::kBytes)};
  Padded<C + 8> X{S.p + 2 * NV * (KD + 8)}, U{X.p + NV * (C + 8)}, Ud{U.p + NV * (C + 8)};  // [column][timestep]
  begin_op();
  const int v0 = (int)(blockIdx.x % a.tiles) * NV, bh = blockIdx.x / a.tiles, h = bh % a.H, b = bh / a.H;
  const int len = length_of(a, b), chunks = (len + C - 1) / C;
  const int warp = threadIdx.x >> 5, g = lane_g(), t = lane_t();
  const int rb = (warp & 3) * 16, rb2 = (warp < 4 ? warp : 7 - warp) * 16;  // the second balances triangles over the SM's parts
  const int cb = (warp >> 2) * (NV / 2);
  const long long DD = (long long)a.Dk * a.Dv;
  const T* v = static_cast<const T*>(a.v) + b * a.vs.b + h * a.vs.h;
  T* o = static_cast<T*>(a.o) + b * a.os.b + h * a.os.h;

  StatePart<KD, NV> s;
  s.load(a.h0 ? a.h0 + (long long)bh * DD : nullptr, a.Dk, a.Dv, v0);
  s.each([&](int r, int c, float& x) { S.p[c * (KD + 8) + r] = x; });
  float2 vx[kTiles][2];
  auto fetch_v = [&](int n) {
#pragma unroll
    for (int x = 0; x < kTiles; ++x)
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        const int time = n * C + rb + g + 8 * r;
        vx[x][r] = time < len ? get2(v + time * a.vs.t, v0 + cb + x * 8 + 2 * t, a.Dv, a.pairs) : make_float2(0.0f, 0.0f);
      }
  };
  if (chunks > 0) {
    St(smem).fetch(a, 0, b, h, len);
    fetch_v(0);
  }
  copies_commit();

  for (int n = 0; n < chunks; ++n) {
    copies_wait<0>();
    __syncthreads();
    const St now(smem + (n & 1) * St::kBytes);
    const Padded<KD + 8> S0{S.p + (n & 1) * NV * (KD + 8)};
    Padded<KD + 8> S1{S.p + (~n & 1) * NV * (KD + 8)};
    const Gates& gate = *now.gates;
    float2 vn[kTiles][2];
#pragma unroll
    for (int x = 0; x < kTiles; ++x) vn[x][0] = vx[x][0], vn[x][1] = vx[x][1];
    if (n + 1 < chunks) {
      St(smem + (~n & 1) * St::kBytes).fetch(a, n + 1, b, h, len);
      fetch_v(n + 1);
    }
    copies_commit();
    if (a.states) s.store(a.states + (((long long)n * a.B + b) * a.H + h) * DD, a.Dk, a.Dv, v0);
    const unsigned long long cuts = gate.cuts;

    for (int lo = 0; lo < C;) {
      const int hi = piece_end(cuts, lo);
      __syncwarp();
      {  // X = beta (V - gam K S0)
        float d[kTiles][4] = {}, e[kTiles][4] = {};
        if (!cut_before(cuts, lo)) {
#pragma unroll
          for (int k0 = 0; k0 < KD; k0 += 16) {
            FragA fa[2];
            load_a(now.K, rb, k0, fa);
#pragma unroll
            for (int q = 0; q < 2; ++q)
#pragma unroll
              for (int x = 0; x < kTiles; ++x) mma<kOne, false>(d[x], e[x], fa[q], load_b(S0, cb + x * 8, k0 + 8 * q));
          }
        }
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          const int i = rb + g + 8 * r;
          const float gam = gate.gam[i], beta = gate.beta[i];
          const bool in = i >= lo && i < hi;
#pragma unroll
          for (int x = 0; x < kTiles; ++x) {
            const float p = vn[x][r].x - gam * (d[x][2 * r] + e[x][2 * r]), q = vn[x][r].y - gam * (d[x][2 * r + 1] + e[x][2 * r + 1]);
            const int c = cb + x * 8 + 2 * t;
            X.to(c, i) = in ? beta * p : 0.0f;
            X.to(c + 1, i) = in ? beta * q : 0.0f;
          }
        }
      }
      __syncthreads();
      {  // U = Tm X
        float d[kTiles][4] = {}, e[kTiles][4] = {};
        for (int k0 = 0; k0 <= rb2; k0 += 16) {
          FragA fa[2];
          load_a(now.Tm, rb2, k0, fa);
#pragma unroll
          for (int q = 0; q < 2; ++q)
#pragma unroll
            for (int x = 0; x < kTiles; ++x) mma<false, false>(d[x], e[x], fa[q], load_b(X, cb + x * 8, k0 + 8 * q));
        }
#pragma unroll
        for (int x = 0; x < kTiles; ++x)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const int i = rb2 + g + 8 * (r >> 1), c = cb + x * 8 + 2 * t + (r & 1);
            const float u = i >= lo && i < hi ? d[x][r] + e[x][r] : 0.0f;
            U.to(c, i) = u;
            Ud.to(c, i) = gate.dec[i] * u;
          }
      }
      if (hi == C && lo > 0)  // the last piece's keys alone reach the next chunk
        for (int i = threadIdx.x; i < lo * KD; i += kThreads) now.K.p[i] = from_f32<T>(0.0f);
      __syncthreads();
      if (hi == C) {  // S = gam_63 S0 + K^T dec U
        float e[StatePart<KD, NV>::kTiles][4] = {};
        const float keep = gate.gam[C - 1];
        s.each([&](int, int, float& x) { x = cuts ? 0.0f : keep * x; });
#pragma unroll
        for (int k0 = 0; k0 < C; k0 += 16) {
          FragA fa[2];
          load_at(now.K, s.row0(), k0, fa);
#pragma unroll
          for (int q = 0; q < 2; ++q)
#pragma unroll
            for (int x = 0; x < s.kTiles; ++x) mma<kOne, false>(s.x[x], e[x], fa[q], load_b(Ud, s.col0() + x * 8, k0 + 8 * q));
        }
#pragma unroll
        for (int x = 0; x < s.kTiles; ++x)
#pragma unroll
          for (int r = 0; r < 4; ++r) s.x[x][r] += e[x][r];
        s.each([&](int r, int c, float& x) { S1.to(c, r) = x; });
      }
      __syncwarp();
      {  // O = scale (gam Q S0 + M U)
        float d[kTiles][4] = {}, e[kTiles][4] = {};
        if (!cut_before(cuts, lo)) {
#pragma unroll
          for (int k0 = 0; k0 < KD; k0 += 16) {
            FragA fa[2];
            load_a(now.Q, rb2, k0, fa);
#pragma unroll
            for (int q = 0; q < 2; ++q)
#pragma unroll
              for (int x = 0; x < kTiles; ++x) mma<kOne, false>(d[x], e[x], fa[q], load_b(S0, cb + x * 8, k0 + 8 * q));
          }
#pragma unroll
          for (int x = 0; x < kTiles; ++x)
#pragma unroll
            for (int r = 0; r < 4; ++r) d[x][r] = gate.gam[rb2 + g + 8 * (r >> 1)] * (d[x][r] + e[x][r]), e[x][r] = 0.0f;
        }
        for (int k0 = 0; k0 <= rb2; k0 += 16) {
          FragA fa[2];
          load_a(now.M, rb2, k0, fa);
#pragma unroll
          for (int q = 0; q < 2; ++q)
#pragma unroll
            for (int x = 0; x < kTiles; ++x) mma<false, false>(d[x], e[x], fa[q], load_b(U, cb + x * 8, k0 + 8 * q));
        }
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          const int i = rb2 + g + 8 * r, time = n * C + i;
          if (i < lo || i >= hi || time >= len) continue;
#pragma unroll
          for (int x = 0; x < kTiles; ++x)
            put2(o + time * a.os.t, v0 + cb + x * 8 + 2 * t, a.Dv, a.pairs, a.scale * (d[x][2 * r] + e[x][2 * r]),
                 a.scale * (d[x][2 * r + 1] + e[x][2 * r + 1]));
        }
      }
      lo = hi;
      if (lo < C) __syncthreads();
    }
  }
  s.store(a.h_last + (long long)bh * DD, a.Dk, a.Dv, v0);
  for (long long i = (long long)len * NV + threadIdx.x; i < (long long)a.T * NV; i += kThreads) {
    const int c = v0 + (int)(i % NV);
    if (c < a.Dv) o[i / NV * a.os.t + c] = from_f32<T>(0.0f);
  }
}

template <typename T, int KD, int NV>
constexpr size_t forward_smem() {
  return 2 * Stage<T, KD>::kBytes + (2 * NV * (KD + 8) + 3 * NV * (C + 8)) * 4;
}

// ---- along the chunks, backward ------------------------------------------------

// dS before a chunk from dS behind it; keeps the latter and R for the gradients of the rest, and writes dV.
template <typename T, int KD, int NV>
__global__ void __launch_bounds__(kThreads, 1) delta_backward_kernel(const DeltaArgs a) {
  extern __shared__ __align__(128) unsigned char smem[];
  constexpr int kTiles = NV / 16;
  constexpr bool kOne = sizeof(T) == 2;
  using St = Stage<T, KD>;
  const Padded<KD + 8> S{reinterpret_cast<float*>(smem + 2 * St::kBytes)};                      // dS, [column][row]
  Padded<C + 8> X{S.p + 2 * NV * (KD + 8)}, Y{X.p + NV * (C + 8)}, Z{Y.p + NV * (C + 8)};  // [column][timestep]
  begin_op();
  const int v0 = (int)(blockIdx.x % a.tiles) * NV, bh = blockIdx.x / a.tiles, h = bh % a.H, b = bh / a.H;
  const int len = length_of(a, b), chunks = (len + C - 1) / C;
  const int warp = threadIdx.x >> 5, g = lane_g(), t = lane_t();
  const int rb = (warp & 3) * 16, rb2 = (warp < 4 ? warp : 7 - warp) * 16;
  const int cb = (warp >> 2) * (NV / 2);
  const long long DD = (long long)a.Dk * a.Dv;
  const T* d_o = static_cast<const T*>(a.d_o) + b * a.dos.b + h * a.dos.h;
  T* dv = static_cast<T*>(a.dv) + b * a.dvs.b + h * a.dvs.h;

  StatePart<KD, NV> s;
  s.load(a.dh_last ? a.dh_last + (long long)bh * DD : nullptr, a.Dk, a.Dv, v0);
  s.each([&](int r, int c, float& x) { S.p[c * (KD + 8) + r] = x; });
  float2 ox[kTiles][2];
  auto fetch_o = [&](int n) {
#pragma unroll
    for (int x = 0; x < kTiles; ++x)
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        const int time = n * C + rb + g + 8 * r;
        ox[x][r] = time < len ? get2(d_o + time * a.dos.t, v0 + cb + x * 8 + 2 * t, a.Dv, a.pairs) : make_float2(0.0f, 0.0f);
      }
  };
  if (chunks > 0) {
    St(smem + ((chunks - 1) & 1) * St::kBytes).fetch(a, chunks - 1, b, h, len);
    fetch_o(chunks - 1);
  }
  copies_commit();

  for (int n = chunks - 1; n >= 0; --n) {
    const int turn = (chunks - 1 - n) & 1;
    copies_wait<0>();
    __syncthreads();
    const St now(smem + (n & 1) * St::kBytes);
    const Padded<KD + 8> S1{S.p + turn * NV * (KD + 8)};
    Padded<KD + 8> S0{S.p + (turn ^ 1) * NV * (KD + 8)};
    const Gates& gate = *now.gates;
    const long long chunk = ((long long)n * a.B + b) * a.H + h;
    float2 on[kTiles][2];
#pragma unroll
    for (int x = 0; x < kTiles; ++x) on[x][0] = ox[x][0], on[x][1] = ox[x][1];
    if (n > 0) {
      St(smem + (~n & 1) * St::kBytes).fetch(a, n - 1, b, h, len);
      fetch_o(n - 1);
    }
    copies_commit();
    s.store(a.dS + chunk * DD, a.Dk, a.Dv, v0);
    const unsigned long long cuts = gate.cuts;
    float* R = a.R + chunk * C * a.Dv;

    for (int hi = C; hi > 0;) {  // pieces, the last first
      int lo = 0;
      for (int next = piece_end(cuts, lo); next < hi; next = piece_end(cuts, lo)) lo = next;
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        const int i = rb + g + 8 * r;
        const bool in = i >= lo && i < hi;
        const float gam = a.scale * gate.gam[i];
#pragma unroll
        for (int x = 0; x < kTiles; ++x) {
          const int c = cb + x * 8 + 2 * t;
          const float p = in ? on[x][r].x : 0.0f, q = in ? on[x][r].y : 0.0f;
          X.to(c, i) = p, X.to(c + 1, i) = q;
          Y.to(c, i) = gam * p, Y.to(c + 1, i) = gam * q;
        }
      }
      __syncthreads();
      {  // dU = scale M^T dO + dec K dS
        float d[kTiles][4] = {}, e[kTiles][4] = {};
        if (hi == C) {
#pragma unroll
          for (int k0 = 0; k0 < KD; k0 += 16) {
            FragA fa[2];
            load_a(now.K, rb2, k0, fa);
#pragma unroll
            for (int q = 0; q < 2; ++q)
#pragma unroll
              for (int x = 0; x < kTiles; ++x) mma<kOne, false>(d[x], e[x], fa[q], load_b(S1, cb + x * 8, k0 + 8 * q));
          }
        }
        float du[kTiles][4];
#pragma unroll
        for (int x = 0; x < kTiles; ++x)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            du[x][r] = hi == C ? gate.dec[rb2 + g + 8 * (r >> 1)] * (d[x][r] + e[x][r]) : 0.0f;
            d[x][r] = e[x][r] = 0.0f;
          }
        for (int k0 = rb2; k0 < C; k0 += 16) {
          FragA fa[2];
          load_at(now.M, rb2, k0, fa);
#pragma unroll
          for (int q = 0; q < 2; ++q)
#pragma unroll
            for (int x = 0; x < kTiles; ++x) mma<false, kOne>(d[x], e[x], fa[q], load_b(X, cb + x * 8, k0 + 8 * q));
        }
#pragma unroll
        for (int x = 0; x < kTiles; ++x)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const int i = rb2 + g + 8 * (r >> 1);
            Z.to(cb + x * 8 + 2 * t + (r & 1), i) = i >= lo && i < hi ? fmaf(a.scale, d[x][r] + e[x][r], du[x][r]) : 0.0f;
          }
      }
      __syncthreads();
      {  // R = Tm^T dU, dV = beta R; - beta gam R goes where dO was
        float d[kTiles][4] = {}, e[kTiles][4] = {};
        for (int k0 = rb2; k0 < C; k0 += 16) {
          FragA fa[2];
          load_at(now.Tm, rb2, k0, fa);
#pragma unroll
          for (int q = 0; q < 2; ++q)
#pragma unroll
            for (int x = 0; x < kTiles; ++x) mma<false, false>(d[x], e[x], fa[q], load_b(Z, cb + x * 8, k0 + 8 * q));
        }
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          const int i = rb2 + g + 8 * r, time = n * C + i;
          const bool in = i >= lo && i < hi;
          const float beta = gate.beta[i], back = in ? -beta * gate.gam[i] : 0.0f;
#pragma unroll
          for (int x = 0; x < kTiles; ++x) {
            const int c = cb + x * 8 + 2 * t;
            const float p = in ? d[x][2 * r] + e[x][2 * r] : 0.0f, q = in ? d[x][2 * r + 1] + e[x][2 * r + 1] : 0.0f;
            X.to(c, i) = back * p, X.to(c + 1, i) = back * q;
            if (!in) continue;
            if (v0 + c < a.Dv) R[(long long)i * a.Dv + v0 + c] = p;
            if (v0 + c + 1 < a.Dv) R[(long long)i * a.Dv + v0 + c + 1] = q;
            if (time < len) put2(dv + time * a.dvs.t, v0 + c, a.Dv, a.pairs, beta * p, beta * q);
          }
        }
      }
      if (lo == 0 && cuts)  // rows behind the first reset do not reach the state before
        for (int i = threadIdx.x + hi * KD; i < C * KD; i += kThreads) now.K.p[i] = now.Q.p[i] = from_f32<T>(0.0f);
      __syncthreads();
      if (lo == 0) {  // dS = gam_63 dS + Q^T scale gam dO - K^T beta gam R
        float e[StatePart<KD, NV>::kTiles][4] = {};
        const bool fresh = cuts & 1ull;
        const float keep = gate.gam[C - 1];
        s.each([&](int, int, float& x) { x = cuts ? 0.0f : keep * x; });
        if (!fresh) {
#pragma unroll
          for (int k0 = 0; k0 < C; k0 += 16) {
            FragA fa[2];
            load_at(now.Q, s.row0(), k0, fa);
#pragma unroll
            for (int q = 0; q < 2; ++q)
#pragma unroll
              for (int x = 0; x < s.kTiles; ++x) mma<kOne, false>(s.x[x], e[x], fa[q], load_b(Y, s.col0() + x * 8, k0 + 8 * q));
            load_at(now.K, s.row0(), k0, fa);
#pragma unroll
            for (int q = 0; q < 2; ++q)
#pragma unroll
              for (int x = 0; x < s.kTiles; ++x) mma<kOne, false>(s.x[x], e[x], fa[q], load_b(X, s.col0() + x * 8, k0 + 8 * q));
          }
        }
#pragma unroll
        for (int x = 0; x < s.kTiles; ++x)
#pragma unroll
          for (int r = 0; r < 4; ++r) s.x[x][r] += e[x][r];
        s.each([&](int r, int c, float& x) { S0.to(c, r) = x; });
      }
      hi = lo;
      if (hi > 0) __syncthreads();
    }
  }
  s.store(a.dh0 + (long long)bh * DD, a.Dk, a.Dv, v0);
  for (long long i = (long long)len * NV + threadIdx.x; i < (long long)a.T * NV; i += kThreads) {
    const int c = v0 + (int)(i % NV);
    if (c < a.Dv) dv[i / NV * a.dvs.t + c] = from_f32<T>(0.0f);
  }
}

// ---- per chunk and key head: the gradients of q, k, g and beta ---------------------

// Rows of a tile whose pitch is 40 words: 32 columns of S, dS, dO, R and U.
constexpr int kSlice = 32, kPitch = kSlice + 8;

template <typename T, int KD>
struct GradShared {
  Tile<T, KD> K, Q;
  Tile<float, C> Tm;
  Padded<kPitch> S, dS, dO, R, U;
  Padded<C + 8> X, P, E;  // X: [column][timestep]; P, E: [i][j]
  Gates* gates;
  float* sums;  // [5][2][C], [8]
  static constexpr size_t kBytes = 2 * C * KD * sizeof(T) + C * C * 4 + (2 * KD + 3 * C) * kPitch * 4 + (kSlice + 2 * C) * (C + 8) * 4 +
                                   sizeof(Gates) + (10 * C + 8) * 4;
  __device__ __forceinline__ explicit GradShared(unsigned char* p)
      : K{reinterpret_cast<T*>(p)}, Q{K.p + C * KD}, Tm{reinterpret_cast<float*>(Q.p + C * KD)}, S{Tm.p + C * C},
        dS{S.p + KD * kPitch}, dO{dS.p + KD * kPitch}, R{dO.p + C * kPitch}, U{R.p + C * kPitch}, X{U.p + C * kPitch},
        P{X.p + kSlice * (C + 8)}, E{P.p + C * (C + 8)}, gates(reinterpret_cast<Gates*>(E.p + C * (C + 8))),
        sums(reinterpret_cast<float*>(gates + 1)) {}
};

template <typename T, int KD>
__global__ void __launch_bounds__(kThreads, 1) delta_gradients_kernel(const DeltaArgs a) {
  extern __shared__ __align__(128) unsigned char smem[];
  constexpr bool kOne = sizeof(T) == 2;
  constexpr int kHalf = KD / 2, kTiles = kHalf / 8;  // a warp has 16 rows and half of the columns
  GradShared<T, KD> sh(smem);
  Gates& gate = *sh.gates;
  begin_op();
  const int Hk = a.H / a.share;
  const int hk = (int)(blockIdx.x % Hk), b = (int)(blockIdx.x / Hk % a.B), n = (int)(blockIdx.x / Hk / a.B);
  const int len = length_of(a, b), t0 = n * C, rows = min(len - t0, C), all = min(a.T - t0, C);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane_g(), t = lane_t();
  const int rb = (warp & 3) * 16, side = warp >> 2, rb2 = (warp < 4 ? warp : 7 - warp) * 16;
  T* dq = static_cast<T*>(a.dq) + t0 * a.dqs.t + b * a.dqs.b + hk * a.dqs.h;
  T* dk = static_cast<T*>(a.dk) + t0 * a.dks.t + b * a.dks.b + hk * a.dks.h;
  for (int i = threadIdx.x + max(rows, 0) * a.Dk; i < all * a.Dk; i += kThreads) {  // past the stream's length
    dq[i / a.Dk * a.dqs.t + i % a.Dk] = from_f32<T>(0.0f);
    dk[i / a.Dk * a.dks.t + i % a.Dk] = from_f32<T>(0.0f);
  }
  for (int i = threadIdx.x + max(rows, 0) * a.share; i < all * a.share; i += kThreads) {
    const int row = t0 + i / a.share, h = hk * a.share + i % a.share;
    a.dg[row * a.dgt + b * a.dgb + h] = 0.0f;
    a.dbeta[row * a.dbt + b * a.dbb + h] = 0.0f;
  }
  if (rows <= 0) return;
  const T* k = static_cast<const T*>(a.k) + t0 * a.ks.t + b * a.ks.b + hk * a.ks.h;
  const T* q = static_cast<const T*>(a.q) + t0 * a.qs.t + b * a.qs.b + hk * a.qs.h;
  const long long DD = (long long)a.Dk * a.Dv;

  for (int h = hk * a.share; h < (hk + 1) * a.share; ++h) {
    const long long chunk = ((long long)n * a.B + b) * a.H + h;
    const T* v = static_cast<const T*>(a.v) + t0 * a.vs.t + b * a.vs.b + h * a.vs.h;
    const T* d_o = static_cast<const T*>(a.d_o) + t0 * a.dos.t + b * a.dos.b + h * a.dos.h;
    __syncthreads();
    fetch_plain(sh.Tm.p, a.Tm + chunk * C * C, C * C * 4);
    fetch_plain(sh.gates, a.gates + chunk, (int)sizeof(Gates));
    copies_commit();
    copies_wait<0>();
    __syncthreads();
    const unsigned long long cuts = gate.cuts;

    for (int lo = 0; lo < rows;) {
      const int hi = min(piece_end(cuts, lo), rows);
      const bool fresh = cut_before(cuts, lo), last = hi == rows;  // the state before counts as zero; the one behind goes on
      __syncthreads();
      fetch_tile(sh.K, k, a.ks.t, lo, hi, a.Dk, a.wide);
      fetch_tile(sh.Q, q, a.qs.t, lo, hi, a.Dk, a.wide);
      copies_commit();
      float acc_q[kTiles][4] = {}, acc_w[kTiles][4] = {}, acc_t[kTiles][4] = {};  // dO S0^T, R S0^T, U dS^T
      float acc_p[4][4] = {}, acc_e[4][4] = {};                                  // dO U^T, R U^T
      float rv[2] = {}, dots = 0.0f;                                             // R . V, <dS, S0>

      for (int v0 = 0; v0 < a.Dv; v0 += kSlice) {
        __syncthreads();
        const float* S = a.states + chunk * DD;
        const float* dS = a.dS + chunk * DD;
        for (int i = threadIdx.x; i < KD * kSlice; i += kThreads) {
          const int r = i / kSlice, c = i % kSlice;
          const bool in = r < a.Dk && v0 + c < a.Dv;
          const float x = in && !fresh ? S[(long long)r * a.Dv + v0 + c] : 0.0f, y = in && last ? dS[(long long)r * a.Dv + v0 + c] : 0.0f;
          sh.S.to(r, c) = x;
          sh.dS.to(r, c) = y;
          dots = fmaf(x, y, dots);
        }
        for (int i = threadIdx.x; i < C * kSlice; i += kThreads) {
          const int r = i / kSlice, c = i % kSlice;
          const bool in = r >= lo && r < hi && v0 + c < a.Dv;
          sh.dO.to(r, c) = in ? to_f32(d_o[r * a.dos.t + v0 + c]) : 0.0f;
          sh.R.to(r, c) = in ? a.R[(chunk * C + r) * a.Dv + v0 + c] : 0.0f;
        }
        copies_wait<0>();
        __syncthreads();
        {  // X = beta (V - gam K S0), and R . V
          float d[2][4] = {}, e[2][4] = {};
          if (!fresh) {
#pragma unroll
            for (int k0 = 0; k0 < KD; k0 += 16) {
              FragA fa[2];
              load_a(sh.K, rb, k0, fa);
#pragma unroll
              for (int s = 0; s < 2; ++s)
#pragma unroll
                for (int x = 0; x < 2; ++x) mma<kOne, false>(d[x], e[x], fa[s], load_bt(sh.S, side * 16 + x * 8, k0 + 8 * s));
            }
          }
#pragma unroll
          for (int r = 0; r < 2; ++r) {
            const int i = rb + g + 8 * r;
            const bool in = i >= lo && i < hi;
            const float gam = gate.gam[i], beta = gate.beta[i];
#pragma unroll
            for (int x = 0; x < 2; ++x) {
              const int c = side * 16 + x * 8 + 2 * t;
              const float2 w = in ? get2(v + i * a.vs.t, v0 + c, a.Dv, a.pairs) : make_float2(0.0f, 0.0f);
              const float2 y = sh.R.pair(i, c);
              rv[r] = fmaf(y.x, w.x, fmaf(y.y, w.y, rv[r]));
              sh.X.to(c, i) = in ? beta * (w.x - gam * (d[x][2 * r] + e[x][2 * r])) : 0.0f;
              sh.X.to(c + 1, i) = in ? beta * (w.y - gam * (d[x][2 * r + 1] + e[x][2 * r + 1])) : 0.0f;
            }
          }
        }
        __syncthreads();
        {  // U = Tm X
          float d[2][4] = {}, e[2][4] = {};
          for (int k0 = 0; k0 <= rb2; k0 += 16) {
            FragA fa[2];
            load_a(sh.Tm, rb2, k0, fa);
#pragma unroll
            for (int s = 0; s < 2; ++s)
#pragma unroll
              for (int x = 0; x < 2; ++x) mma<false, false>(d[x], e[x], fa[s], load_b(sh.X, side * 16 + x * 8, k0 + 8 * s));
          }
#pragma unroll
          for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              const int i = rb2 + g + 8 * (r >> 1);
              sh.U.to(i, side * 16 + x * 8 + 2 * t + (r & 1)) = i >= lo && i < hi ? d[x][r] + e[x][r] : 0.0f;
            }
        }
        __syncthreads();
#pragma unroll
        for (int k0 = 0; k0 < kSlice; k0 += 16) {
          FragA fo[2], fr[2], fu[2];
          load_a(sh.dO, rb, k0, fo);
          load_a(sh.R, rb, k0, fr);
          load_a(sh.U, rb, k0, fu);
#pragma unroll
          for (int s = 0; s < 2; ++s) {
#pragma unroll
            for (int x = 0; x < 4; ++x) {
              if (side * 32 + x * 8 > rb + 15) continue;
              const FragB fb = load_b(sh.U, side * 32 + x * 8, k0 + 8 * s);
              mma<kOne, false>(acc_p[x], acc_p[x], fo[s], fb);
              mma<false, false>(acc_e[x], acc_e[x], fr[s], fb);
            }
            if (!fresh) {
#pragma unroll
              for (int x = 0; x < kTiles; ++x) {
                const FragB fb = load_b(sh.S, side * kHalf + x * 8, k0 + 8 * s);
                mma<kOne, false>(acc_q[x], acc_q[x], fo[s], fb);
                mma<false, false>(acc_w[x], acc_w[x], fr[s], fb);
              }
            }
            if (last) {
#pragma unroll
              for (int x = 0; x < kTiles; ++x)
                mma<false, false>(acc_t[x], acc_t[x], fu[s], load_b(sh.dS, side * kHalf + x * 8, k0 + 8 * s));
            }
          }
        }
      }

#pragma unroll
      for (int x = 0; x < 4; ++x)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int i = rb + g + 8 * (r >> 1), j = side * 32 + x * 8 + 2 * t + (r & 1);
          const float dist = (gate.g_high[i] - gate.g_high[j]) + (gate.g_low[i] - gate.g_low[j]);
          const float D = i >= j && j >= lo && i < hi ? expf(dist) : 0.0f;
          sh.P.to(i, j) = D != 0.0f ? a.scale * D * acc_p[x][r] : 0.0f;
          sh.E.to(i, j) = D != 0.0f && i > j ? D * acc_e[x][r] : 0.0f;
        }
      __syncthreads();

      float far[2] = {}, dot_q[2] = {}, dot_w[2] = {}, dot_t[2] = {};  // row sums with K or Q
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        const int i = rb + g + 8 * r;
        const float gam = gate.gam[i], dec = gate.dec[i];
#pragma unroll
        for (int x = 0; x < kTiles; ++x) {
          const float2 kx = sh.K.pair(i, side * kHalf + x * 8 + 2 * t);
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            acc_q[x][2 * r + c] = fresh ? 0.0f : a.scale * gam * acc_q[x][2 * r + c];
            acc_w[x][2 * r + c] = fresh ? 0.0f : gam * acc_w[x][2 * r + c];
            acc_t[x][2 * r + c] = last ? dec * acc_t[x][2 * r + c] : 0.0f;
            far[r] = fmaf(c ? kx.y : kx.x, acc_t[x][2 * r + c], far[r]);
          }
        }
      }
      for (int k0 = 0; k0 <= rb; k0 += 16) {  // P K, E K
        FragA fp[2], fe[2];
        load_a(sh.P, rb, k0, fp);
        load_a(sh.E, rb, k0, fe);
#pragma unroll
        for (int x = 0; x < kTiles; x += 2) {
          FragB fb[2][2];
          load_bt16(sh.K, side * kHalf + x * 8, k0, fb);
#pragma unroll
          for (int y = 0; y < 2; ++y)
#pragma unroll
            for (int s = 0; s < 2; ++s) {
              mma<false, kOne>(acc_q[x + y], acc_q[x + y], fp[s], fb[y][s]);
              mma<false, kOne>(acc_w[x + y], acc_w[x + y], fe[s], fb[y][s]);
            }
        }
      }
      for (int k0 = rb; k0 < C; k0 += 16) {  // P^T Q, - E^T beta K
        FragA fp[2], fe[2];
        load_at(sh.P, rb, k0, fp);
        load_at(sh.E, rb, k0, fe);
#pragma unroll
        for (int s = 0; s < 2; ++s) {
          const int i = k0 + 8 * s + 2 * t;
          const float b0 = i >= lo && i < hi ? -gate.beta[i] : 0.0f, b1 = i + 1 >= lo && i + 1 < hi ? -gate.beta[i + 1] : 0.0f;
          fe[s].x[0] *= b0, fe[s].x[1] *= b0, fe[s].x[2] *= b1, fe[s].x[3] *= b1;
        }
#pragma unroll
        for (int x = 0; x < kTiles; x += 2) {
          FragB fq[2][2], fk[2][2];
          load_bt16(sh.Q, side * kHalf + x * 8, k0, fq);
          load_bt16(sh.K, side * kHalf + x * 8, k0, fk);
#pragma unroll
          for (int y = 0; y < 2; ++y)
#pragma unroll
            for (int s = 0; s < 2; ++s) {
              mma<false, kOne>(acc_t[x + y], acc_t[x + y], fp[s], fq[y][s]);
              mma<false, kOne>(acc_t[x + y], acc_t[x + y], fe[s], fk[y][s]);
            }
        }
      }
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        const int i = rb + g + 8 * r;
        const bool in = i >= lo && i < hi;
        const float beta = gate.beta[i];
        float* sum_q = a.sum_q + (((long long)n * a.B + b) * Hk + hk) * C * KD + i * KD;
        float* sum_k = a.sum_k + (((long long)n * a.B + b) * Hk + hk) * C * KD + i * KD;
#pragma unroll
        for (int x = 0; x < kTiles; ++x) {
          const int c = side * kHalf + x * 8 + 2 * t;
          const float2 kx = sh.K.pair(i, c), qx = sh.Q.pair(i, c);
          float gq[2], gk[2];
#pragma unroll
          for (int y = 0; y < 2; ++y) {
            const float aq = acc_q[x][2 * r + y], aw = acc_w[x][2 * r + y], at = acc_t[x][2 * r + y];
            dot_q[r] = fmaf(y ? qx.y : qx.x, aq, dot_q[r]);
            dot_w[r] = fmaf(y ? kx.y : kx.x, aw, dot_w[r]);
            dot_t[r] = fmaf(y ? kx.y : kx.x, at, dot_t[r]);
            gq[y] = aq;
            gk[y] = fmaf(-beta, aw, at);
          }
          if (!in) continue;
          if (a.share > 1) {  // over the value heads of a key head: each thread goes on with what it wrote itself
            const bool first = h == hk * a.share;
#pragma unroll
            for (int y = 0; y < 2; ++y) {
              if (!first) gq[y] += sum_q[c + y], gk[y] += sum_k[c + y];
              sum_q[c + y] = gq[y], sum_k[c + y] = gk[y];
            }
          }
          if (h + 1 == (hk + 1) * a.share) {
            put2(dq + i * a.dqs.t, c, a.Dk, a.wide, gq[0], gq[1]);
            put2(dk + i * a.dks.t, c, a.Dk, a.wide, gk[0], gk[1]);
          }
        }
      }
      // sums over a row's columns: four lanes and two warps; over the block for <dS, S0>
      auto row_sum = [&](int which, float (&x)[2]) {
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          float y = x[r];
          y += __shfl_xor_sync(0xffffffffu, y, 1);
          y += __shfl_xor_sync(0xffffffffu, y, 2);
          if (t == 0) sh.sums[(which * 2 + side) * C + rb + g + 8 * r] = y;
        }
      };
      row_sum(0, rv);
      row_sum(1, far);
      row_sum(2, dot_q);
      row_sum(3, dot_w);
      row_sum(4, dot_t);
#pragma unroll
      for (int d = 16; d > 0; d /= 2) dots += __shfl_xor_sync(0xffffffffu, dots, d);
      if (lane == 0) sh.sums[10 * C + warp] = dots;
      __syncthreads();
      if (warp == 0) {  // dbeta, and dg as sums from the piece's end (rows lane and lane + 32)
        auto sum_of = [&](int which, int row) { return sh.sums[which * 2 * C + row] + sh.sums[(which * 2 + 1) * C + row]; };
        float G[2], far_all = 0.0f;
#pragma unroll
        for (int s = 0; s < 2; ++s) {
          const int row = lane + 32 * s;
          const bool in = row >= lo && row < hi;
          G[s] = in ? sum_of(2, row) - fmaf(gate.beta[row], sum_of(3, row), sum_of(4, row)) : 0.0f;
          far_all += in ? sum_of(1, row) : 0.0f;
          if (in) a.dbeta[(t0 + row) * a.dbt + b * a.dbb + h] = sum_of(0, row) - sum_of(3, row);
        }
#pragma unroll
        for (int d = 16; d > 0; d /= 2) far_all += __shfl_xor_sync(0xffffffffu, far_all, d);
        float all_dots = 0.0f;
#pragma unroll
        for (int w = 0; w < 8; ++w) all_dots += sh.sums[10 * C + w];
        const float end = last ? (cuts ? far_all : fmaf(gate.gam[C - 1], all_dots, far_all)) : 0.0f;
#pragma unroll
        for (int s = 1; s >= 0; --s) {
          if (lane + 32 * s == hi - 1) G[s] += end;
#pragma unroll
          for (int d = 1; d < 32; d *= 2) {
            const float y = __shfl_down_sync(0xffffffffu, G[s], d);
            if (lane + d < 32) G[s] += y;
          }
          if (s == 1) {
            const float behind = __shfl_sync(0xffffffffu, G[1], 0);
            if (lane == 31) G[0] += behind;
          }
        }
#pragma unroll
        for (int s = 0; s < 2; ++s) {
          const int row = lane + 32 * s;
          if (row < lo || row >= hi) continue;
          const float g_in = a.g[(t0 + row) * a.gt + b * a.gb + h];
          const bool none = (cuts >> row & 1ull) || g_in < kLeastG;  // a decay that nothing passes through
          a.dg[(t0 + row) * a.dgt + b * a.dgb + h] = none ? 0.0f : G[s];
        }
      }
      lo = hi;
    }
  }
}

// ---- host ----------------------------------------------------------------------

struct Workspace {
  size_t Tm, M, gates, dS, R, sum_q, sum_k, bytes;
};
Workspace workspace_of(long long T, long long B, long long H, long long Hk, long long Dk, long long Dv, bool backward) {
  const size_t chunks = (size_t)((T + C - 1) / C) * B * H, KD = Dk <= 64 ? 64 : 128;
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t from = at;
    at += (bytes + 255) / 256 * 256;
    return from;
  };
  Workspace w{};
  w.Tm = take(chunks * C * C * 4);
  w.M = take(chunks * C * C * 4);
  w.gates = take(chunks * sizeof(Gates));
  if (backward) {
    w.dS = take(chunks * Dk * Dv * 4);
    w.R = take(chunks * C * Dv * 4);
    if (H > Hk) {
      w.sum_q = take(chunks / H * Hk * C * KD * 4);
      w.sum_k = take(chunks / H * Hk * C * KD * 4);
    }
  }
  w.bytes = at + 256;
  return w;
}

// Columns of S to a block: 16 while that fits the device in one wave, and where two chunks of 32-bit keys fill the
// shared memory.
int columns_of(long long heads, int Dk, int Dv, size_t es) {
  return heads * ((Dv + 15) / 16) <= 152 || (es == 4 && Dk > 64) ? 16 : 32;
}

template <auto kKern>
cudaError_t launch_big(dim3 grid, size_t smem, cudaStream_t s, const DeltaArgs& a) {
  static thread_local DeviceSet ready;  // of this kernel
  const cudaError_t e =
      once_per_device(&ready, [&] { return cudaFuncSetAttribute(kKern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem); });
  return e != cudaSuccess ? e : op_launch(kKern, grid, dim3(kThreads), smem, s, a);
}

template <typename F>
cudaError_t for_shape(int dtype, int Dk, F f) {
  return op_for_type(dtype, [&](auto* t) {
    if (Dk <= 64) return f(t, std::integral_constant<int, 64>());
    return f(t, std::integral_constant<int, 128>());
  });
}

cudaError_t prepare(int dtype, const DeltaArgs& a, cudaStream_t s) {
  const long long blocks = (long long)((a.T + C - 1) / C) * a.B * a.H;
  if (blocks == 0) return cudaSuccess;
  return for_shape(dtype, a.Dk, [&](auto* t, auto kd) {
    using T = std::remove_pointer_t<decltype(t)>;
    constexpr int KD = decltype(kd)::value;
    return launch_big<delta_prepare_kernel<T, KD>>(dim3((unsigned)blocks), prepare_smem<T, KD>(), s, a);
  });
}

bool wide_rows(const void* p, const Strides& s, int D, size_t es) {
  return op_aligned(p, 16) && D * es % 16 == 0 && s.t * es % 16 == 0 && s.b * es % 16 == 0 && s.h * es % 16 == 0;
}
bool pair_rows(const void* p, const Strides& s, int D, size_t es) {
  return op_aligned(p, 2 * es) && D % 2 == 0 && s.t % 2 == 0 && s.b % 2 == 0 && s.h % 2 == 0;
}

// The checks that both directions make.
int check(int dtype, const void* q, const void* k, const void* v, const float* g, const float* beta, int T, int B, int H, int Hk,
          int Dk, int Dv, const long long* strides, int n_strides, char* msg, int msg_len) {
  if (!op_float_dtype(dtype)) return op_report(msg, msg_len, LSTM_APPROX_EINVAL, "dtype %d", dtype);
  if (int rc = delta_check_sizes(T, B, H, Hk, Dk, Dv, msg, msg_len)) return rc;
  const long long tiles = (Dv + 15) / 16;
  if ((long long)B * H > 0x7fffffffll / tiles || (long long)((T + 63ll) / 64) * B > 0x7fffffffll / H)
    return op_report(msg, msg_len, LSTM_APPROX_EINVAL, "B H ceil(Dv / 16) and ceil(T / 64) B H must be below 2^31");
  const size_t es = op_dtype_bytes(dtype);
  if (T > 0 && B > 0 && (!q || !k || !v || !g || !beta))
    return op_report(msg, msg_len, LSTM_APPROX_EINVAL, "q, k, v, g and beta must not be NULL");
  if (!op_aligned(q, es) || !op_aligned(k, es) || !op_aligned(v, es) || !op_aligned(g, 4) || !op_aligned(beta, 4))
    return op_report(msg, msg_len, LSTM_APPROX_EINVAL, "a pointer not aligned to its type");
  for (int i = 0; strides && i < n_strides; ++i)
    if (strides[i] < 0) return op_report(msg, msg_len, LSTM_APPROX_EINVAL, "strides must not be negative");
  return LSTM_APPROX_OK;
}

}  // namespace
}  // namespace lstm_approx_impl

using namespace lstm_approx_impl;

extern "C" size_t lstm_approx_delta_scan_workspace_bytes(int T, int B, int H, int Hk, int Dk, int Dv, int backward) {
  if (check(LSTM_APPROX_OP_FP32, nullptr, nullptr, nullptr, nullptr, nullptr, 0, B, H, Hk, Dk, Dv, nullptr, 0, nullptr, 0) || T < 0 ||
      (long long)((T + 63ll) / 64) * B > 0x7fffffffll / H)
    return 0;
  return workspace_of(T, B, H, Hk, Dk, Dv, backward != 0).bytes;
}

extern "C" int lstm_approx_delta_scan(int dtype, const void* q, const void* k, const void* v, const float* g, const float* beta,
                                      float scale, const float* h0, const int32_t* lengths, const unsigned char* reset, int T,
                                      int B, int H, int Hk, int Dk, int Dv, void* o, const long long* strides, float* h_last,
                                      float* states, void* workspace, size_t workspace_bytes, void* cuda_stream, char* msg,
                                      int msg_len) {
  if (msg && msg_len > 0) msg[0] = '\0';
  if (int rc = check(dtype, q, k, v, g, beta, T, B, H, Hk, Dk, Dv, strides, 16, msg, msg_len)) return rc;
  const size_t es = op_dtype_bytes(dtype);
  if (B > 0 && (!h_last || (T > 0 && !o)))
    return op_report(msg, msg_len, LSTM_APPROX_EINVAL, "o and h_last must not be NULL");
  if (!op_aligned(o, es) || !op_aligned(h0, 4) || !op_aligned(h_last, 4) || !op_aligned(states, 4) || !op_aligned(lengths, 4))
    return op_report(msg, msg_len, LSTM_APPROX_EINVAL, "a pointer not aligned to its type");
  const Workspace w = workspace_of(T, B, H, Hk, Dk, Dv, false);
  if (!workspace || !op_aligned(workspace, 16) || workspace_bytes < w.bytes)
    return op_report(msg, msg_len, LSTM_APPROX_EINVAL, "needs a 16-byte aligned workspace of %zu bytes", w.bytes);
  if (int rc = op_check_device(msg, msg_len)) return rc;
  if (B == 0) return LSTM_APPROX_OK;
  const long long K = (long long)Hk * Dk, V = (long long)H * Dv;
  const long long dense[16] = {B * K, K, Dk, B * K, K, Dk, B * V, V, Dv, B * V, V, Dv, (long long)B * H, H, (long long)B * H, H};
  const long long* p = strides ? strides : dense;
  DeltaArgs a{};
  a.q = q, a.k = k, a.v = v, a.g = g, a.beta = beta, a.o = o;
  a.qs = {p[0], p[1], p[2]}, a.ks = {p[3], p[4], p[5]}, a.vs = {p[6], p[7], p[8]}, a.os = {p[9], p[10], p[11]};
  a.gt = p[12], a.gb = p[13], a.bt = p[14], a.bb = p[15];
  a.scale = scale, a.h0 = h0, a.lengths = lengths, a.reset = reset;
  a.T = T, a.B = B, a.H = H, a.share = H / Hk, a.Dk = Dk, a.Dv = Dv;
  a.wide = wide_rows(q, a.qs, Dk, es) && wide_rows(k, a.ks, Dk, es);
  a.pairs = pair_rows(v, a.vs, Dv, es) && pair_rows(o, a.os, Dv, es);
  a.h_last = h_last, a.states = states;
  char* ws = reinterpret_cast<char*>((reinterpret_cast<uintptr_t>(workspace) + 255) / 256 * 256);
  a.Tm = reinterpret_cast<float*>(ws + w.Tm), a.M = reinterpret_cast<float*>(ws + w.M);
  a.gates = reinterpret_cast<Gates*>(ws + w.gates);
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  if (int rc = op_launched(prepare(dtype, a, s), "delta scan launch", msg, msg_len)) return rc;
  const int NV = columns_of((long long)B * H, Dk, Dv, es);
  a.tiles = (Dv + NV - 1) / NV;
  const dim3 grid((unsigned)(B * H * a.tiles));
  const cudaError_t e = for_shape(dtype, Dk, [&](auto* t, auto kd) {
    using Ty = std::remove_pointer_t<decltype(t)>;
    constexpr int KD = decltype(kd)::value;
    if constexpr (sizeof(Ty) == 2 || KD == 64)
      if (NV == 32) return launch_big<delta_forward_kernel<Ty, KD, 32>>(grid, forward_smem<Ty, KD, 32>(), s, a);
    return launch_big<delta_forward_kernel<Ty, KD, 16>>(grid, forward_smem<Ty, KD, 16>(), s, a);
  });
  return op_launched(e, "delta scan launch", msg, msg_len);
}

extern "C" int lstm_approx_delta_scan_backward(int dtype, const void* d_o, const float* dh_last, const void* q, const void* k,
                                               const void* v, const float* g, const float* beta, float scale,
                                               const float* states, const int32_t* lengths, const unsigned char* reset, int T,
                                               int B, int H, int Hk, int Dk, int Dv, void* dq, void* dk, void* dv, float* dg,
                                               float* dbeta, float* dh0, const long long* strides, void* workspace,
                                               size_t workspace_bytes, void* cuda_stream, char* msg, int msg_len) {
  if (msg && msg_len > 0) msg[0] = '\0';
  if (int rc = check(dtype, q, k, v, g, beta, T, B, H, Hk, Dk, Dv, strides, 29, msg, msg_len)) return rc;
  const size_t es = op_dtype_bytes(dtype);
  if (B > 0 && (!dh0 || (T > 0 && (!d_o || !states || !dq || !dk || !dv || !dg || !dbeta))))
    return op_report(msg, msg_len, LSTM_APPROX_EINVAL, "d_o, states and the gradients must not be NULL");
  if (!op_aligned(d_o, es) || !op_aligned(dq, es) || !op_aligned(dk, es) || !op_aligned(dv, es) || !op_aligned(dh_last, 4) ||
      !op_aligned(states, 4) || !op_aligned(lengths, 4) || !op_aligned(dg, 4) || !op_aligned(dbeta, 4) || !op_aligned(dh0, 4))
    return op_report(msg, msg_len, LSTM_APPROX_EINVAL, "a pointer not aligned to its type");
  const Workspace w = workspace_of(T, B, H, Hk, Dk, Dv, true);
  if (!workspace || !op_aligned(workspace, 16) || workspace_bytes < w.bytes)
    return op_report(msg, msg_len, LSTM_APPROX_EINVAL, "needs a 16-byte aligned workspace of %zu bytes", w.bytes);
  if (int rc = op_check_device(msg, msg_len)) return rc;
  if (B == 0) return LSTM_APPROX_OK;
  const long long K = (long long)Hk * Dk, V = (long long)H * Dv, N = H;
  const long long dense[29] = {B * V, V, Dv, B * K, K, Dk, B * K, K, Dk, B * V, V, Dv, B * K, K, Dk, B * K, K, Dk, B * V, V, Dv,
                               B * N, N, B * N, N, B * N, N, B * N, N};
  const long long* p = strides ? strides : dense;
  DeltaArgs a{};
  a.d_o = d_o, a.q = q, a.k = k, a.v = v, a.g = g, a.beta = beta;
  a.dos = {p[0], p[1], p[2]}, a.qs = {p[3], p[4], p[5]}, a.ks = {p[6], p[7], p[8]}, a.vs = {p[9], p[10], p[11]};
  a.dqs = {p[12], p[13], p[14]}, a.dks = {p[15], p[16], p[17]}, a.dvs = {p[18], p[19], p[20]};
  a.gt = p[21], a.gb = p[22], a.bt = p[23], a.bb = p[24], a.dgt = p[25], a.dgb = p[26], a.dbt = p[27], a.dbb = p[28];
  a.scale = scale, a.lengths = lengths, a.reset = reset;
  a.T = T, a.B = B, a.H = H, a.share = H / Hk, a.Dk = Dk, a.Dv = Dv;
  a.wide = wide_rows(q, a.qs, Dk, es) && wide_rows(k, a.ks, Dk, es) && wide_rows(dq, a.dqs, Dk, es) && wide_rows(dk, a.dks, Dk, es);
  a.pairs = pair_rows(v, a.vs, Dv, es) && pair_rows(d_o, a.dos, Dv, es) && pair_rows(dv, a.dvs, Dv, es);
  a.states = const_cast<float*>(states), a.dh_last = dh_last;
  a.dq = dq, a.dk = dk, a.dv = dv, a.dg = dg, a.dbeta = dbeta, a.dh0 = dh0;
  char* ws = reinterpret_cast<char*>((reinterpret_cast<uintptr_t>(workspace) + 255) / 256 * 256);
  a.Tm = reinterpret_cast<float*>(ws + w.Tm), a.M = reinterpret_cast<float*>(ws + w.M);
  a.gates = reinterpret_cast<Gates*>(ws + w.gates);
  a.dS = reinterpret_cast<float*>(ws + w.dS), a.R = reinterpret_cast<float*>(ws + w.R);
  a.sum_q = reinterpret_cast<float*>(ws + w.sum_q), a.sum_k = reinterpret_cast<float*>(ws + w.sum_k);
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  if (int rc = op_launched(prepare(dtype, a, s), "delta scan launch", msg, msg_len)) return rc;
  const int NV = columns_of((long long)B * H, Dk, Dv, es);
  a.tiles = (Dv + NV - 1) / NV;
  const dim3 grid((unsigned)(B * H * a.tiles));
  cudaError_t e = for_shape(dtype, Dk, [&](auto* t, auto kd) {
    using Ty = std::remove_pointer_t<decltype(t)>;
    constexpr int KD = decltype(kd)::value;
    if constexpr (sizeof(Ty) == 2 || KD == 64)
      if (NV == 32) return launch_big<delta_backward_kernel<Ty, KD, 32>>(grid, forward_smem<Ty, KD, 32>(), s, a);
    return launch_big<delta_backward_kernel<Ty, KD, 16>>(grid, forward_smem<Ty, KD, 16>(), s, a);
  });
  if (int rc = op_launched(e, "delta scan backward launch", msg, msg_len)) return rc;
  if (T == 0) return LSTM_APPROX_OK;
  const dim3 blocks((unsigned)((T + C - 1) / C * B * Hk));
  e = for_shape(dtype, Dk, [&](auto* t, auto kd) {
    using Ty = std::remove_pointer_t<decltype(t)>;
    constexpr int KD = decltype(kd)::value;
    return launch_big<delta_gradients_kernel<Ty, KD>>(blocks, GradShared<Ty, KD>::kBytes, s, a);
  });
  return op_launched(e, "delta gradients launch", msg, msg_len);
}
