// The gated delta rule over a sequence, forward and backward
// (include/lstm_approx_ops.h).
//
// For every stream and value head a state S [Dk][Dv]:
//
//   u_t = beta_t (v_t - e^{g_t} S_{t-1}^T k_t);  S_t = e^{g_t} S_{t-1} + k_t u_t^T;  o_t = scale S_t^T q_t
//
// By chunks of 64 timesteps (i, j: rows of a chunk; S0: the state before it; G: the sum of g up to and with a row; B:
// diag(beta)):
//
//   D_ij = e^{G_i - G_j} (i >= j);  gam_i = e^{G_i};  dec_j = e^{G_63 - G_j}
//   A_ij = D_ij k_i . k_j (i > j);  N = (I + A B)^-1 A;  M_ij = D_ij q_i . k_j
//   X = V - diag(gam) K S0;  Y = X - N B X;  U = B Y
//   O = scale (diag(gam) Q S0 + M U);  S = gam_63 S0 + K^T diag(dec) U
//
// and for the gradients (dS that of S):
//
//   dU = scale M^T dO + diag(dec) K dS;  R = dU - N^T B dU;  dV = B R
//   dS0 = gam_63 dS + Q^T diag(scale gam) dO - K^T diag(gam) dV;  dbeta_i = R_i . Y_i
//   P_ij = scale D_ij dO_i . u_j (i >= j);  E_ij = beta_i D_ij R_i . u_j (i > j)
//   dQ = P K + diag(scale gam) dO S0^T
//   dK = P^T Q + diag(dec) U dS^T - E^T K - E K - diag(gam) dV S0^T
//
// Scaling g_t scales what is there of S_t, of which everything behind is linear:
//
//   dg_t = <dS0, S0> - the sum of q_i . dq_i - v_i . dv_i over rows i < t
//
// Kernels: one per chunk and key head makes N and M, and copies of q and k whose
// rows have 64 or 128 columns; one per value head and 16 or 32 columns of S (which
// do not see one another) runs along the chunks, forward or backward; one per
// chunk and key head makes the gradients of q, k, g and beta.
//
// Products run on warp MMAs of bf16 with 32-bit sums.  An operand of 32 bits is
// taken in three parts of 8 bits each (x = high + middle + low), one in fp16 in
// two, and the products of parts down to 2^-16 of the largest are summed: 2^-24
// of a factor is left out.  So a 16-bit output differs from a 32-bit sum's, rounded,
// where that lies next to a border alone.  A state carries thousands of
// timesteps, so it is never rounded to 16 bits.  An operand is split once, where
// it is made, and lies in shared memory as the MMA wants it.  (Split where it is
// used, in two parts of 11 bits on MMAs of 32-bit floats, these kernels executed
// 4 times the instructions: a chunk of 64 x 128 x 16 took 5.1 us.)
//
// Measured, bf16 and 128 x 128 states: 8191 timesteps of 16 heads 416 us (82 the
// chunks' matrices, 335 along them: 2.6 us a chunk, of which the products are 0.9
// of the tensor pipes; 21 times the time of its bytes at a copy's rate), 4 streams of
// 2048 timesteps and 8 heads forward and backward 724 us (47 + 162, 47 + 197 + 251,
// each alone under a profiler; 36 times).  Bound by what follows one another: three products of 64 x 128 x 16 and
// four barriers to a chunk, T / 64 chunks.
//
// At a reset the state before counts as zero, and so does everything before it
// in its chunk: a chunk with resets is taken piece by piece, and rows of other
// pieces are left out, not multiplied by zero.
#include <atomic>
#include <cstddef>
#include <limits>
#include <type_traits>

#include "ops_common.cuh"

namespace lstm_approx_impl {
namespace {

using namespace lstm_approx_dev;

constexpr int C = LSTM_APPROX_DELTA_CHUNK;
static_assert(C == 64, "rows of a chunk");
constexpr int kThreads = 256;
constexpr float kLeastG = -200.0f;
constexpr float kNaN = std::numeric_limits<float>::quiet_NaN();

using bf16 = __nv_bfloat16;

// Parts of a value of T.
template <typename T>
constexpr int kParts = sizeof(T) == 4 ? 3 : std::is_same_v<T, bf16> ? 1 : 2;

// ---- matrices in shared memory and the products of warps ---------------------

// Where a value of a matrix of W columns lies.  16-byte pieces of a row are exchanged by a rule on the row: the same piece of eight
// neighbouring rows lies in different banks.
template <int W>
__device__ __forceinline__ int place(int row, int col) {
  constexpr int kPieces = W / 8;
  const int turn = kPieces >= 8 ? row & 7 : row / (8 / kPieces) & (kPieces - 1);
  return row * W + (col ^ turn << 3);
}
// The layouts of matrices: all values;
template <int kRows, int W>
struct Whole {
  static constexpr int kSize = kRows * W;
  __device__ __forceinline__ static int at(int row, int col) { return place<W>(row, col); }
};
// those of a square one that is zero above the diagonal, without the upper right quarter, which nobody asks for (two stages of whole
// ones do not fit beside 32 columns of S and 128 wide keys).
template <int W>
struct Lower {
  static constexpr int kHalf = W / 2, kSize = kHalf * kHalf + kHalf * W;
  __device__ __forceinline__ static bool has(int row, int col) { return row >= kHalf || col < kHalf; }
  __device__ __forceinline__ static int at(int row, int col) {
    return row < kHalf ? place<kHalf>(row, col) : kHalf * kHalf + place<W>(row - kHalf, col);
  }
};

// kP parts of each of its values, one matrix behind the other.
template <typename Layout, int kP>
struct MatOf : Layout {
  bf16* p;
  __device__ __forceinline__ explicit MatOf(bf16* p_) : p(p_) {}
  using Layout::at;
  using Layout::kSize;
  static constexpr int kHas = kP, kBytes = kSize * kP * 2;
  // Columns col and col + 1 (col even).
  __device__ __forceinline__ void put(int row, int col, float x, float y) const {
    const int i = at(row, col);
#pragma unroll
    for (int q = 0; q < kP; ++q) {
      const __nv_bfloat162 h = __floats2bfloat162_rn(x, y);
      *reinterpret_cast<__nv_bfloat162*>(p + q * kSize + i) = h;
      if (q + 1 < kP) {
        const float2 f = __bfloat1622float2(h);
        x -= f.x;
        y -= f.y;
      }
    }
  }
  // Four of them (col a multiple of 4).
  __device__ __forceinline__ void put4(int row, int col, float4 x) const {
    const int i = at(row, col);
#pragma unroll
    for (int q = 0; q < kP; ++q) {
      const __nv_bfloat162 h[2] = {__floats2bfloat162_rn(x.x, x.y), __floats2bfloat162_rn(x.z, x.w)};
      *reinterpret_cast<uint2*>(p + q * kSize + i) = *reinterpret_cast<const uint2*>(h);
      if (q + 1 < kP) {
        const float2 f = __bfloat1622float2(h[0]), g = __bfloat1622float2(h[1]);
        x = make_float4(x.x - f.x, x.y - f.y, x.z - g.x, x.w - g.y);
      }
    }
  }
  __device__ __forceinline__ float2 pair(int row, int col) const {
    const int i = at(row, col);
    float2 s = make_float2(0.0f, 0.0f);
#pragma unroll
    for (int q = kP - 1; q >= 0; --q) {
      const float2 f = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(p + q * kSize + i));
      s.x += f.x;
      s.y += f.y;
    }
    return s;
  }
};
template <int kRows, int W, int kP>
using Mat = MatOf<Whole<kRows, W>, kP>;

// The loads and MMAs below are reached by whole warps: a barrier lies before each, and between that and the last of them only
// branches that a warp's lanes take alike.  Lane = 4 g + t of an MMA has rows g and g + 8 and columns 2 t and 2 t + 1 of its
// result.
__device__ __forceinline__ int lane_g() { return (threadIdx.x & 31) >> 2; }
__device__ __forceinline__ int lane_t() { return threadIdx.x & 3; }

// A, 16 rows and 16 columns (k): kP parts of it, from rows that are A's; from rows that are A's columns.
template <int kP, typename M>
__device__ __forceinline__ void load_a(const M& m, int m0, int k0, uint32_t (&a)[kP][4]) {
  static_assert(kP <= M::kHas, "parts");
  const int l = threadIdx.x & 31;
  const uint32_t addr = smem_u32(m.p + m.at(m0 + (l & 15), k0 + (l >> 4) * 8));
#pragma unroll
  for (int q = 0; q < kP; ++q) ldmatrix4<true>(addr + q * m.kSize * 2, a[q]);
}
template <int kP, typename M>
__device__ __forceinline__ void load_at(const M& m, int m0, int k0, uint32_t (&a)[kP][4]) {
  static_assert(kP <= M::kHas, "parts");
  const int l = threadIdx.x & 31;
  const uint32_t addr = smem_u32(m.p + m.at(k0 + (l & 7) + (l >> 4) * 8, m0 + (l >> 3 & 1) * 8));
#pragma unroll
  for (int q = 0; q < kP; ++q) ldmatrix4_trans<true>(addr + q * m.kSize * 2, a[q]);
}
// B, 16 rows (k) and 16 columns, [part][column / 8][k / 8]: from rows that are B's columns; from rows that are B's.
template <int kP, typename M>
__device__ __forceinline__ void load_b(const M& m, int n0, int k0, uint32_t (&b)[kP][2][2]) {
  static_assert(kP <= M::kHas, "parts");
  const int l = threadIdx.x & 31;
  const uint32_t addr = smem_u32(m.p + m.at(n0 + (l & 7) + (l >> 4) * 8, k0 + (l >> 3 & 1) * 8));
#pragma unroll
  for (int q = 0; q < kP; ++q) {
    uint32_t r[4];
    ldmatrix4<true>(addr + q * m.kSize * 2, r);
    b[q][0][0] = r[0], b[q][0][1] = r[1], b[q][1][0] = r[2], b[q][1][1] = r[3];
  }
}
template <int kP, typename M>
__device__ __forceinline__ void load_bt(const M& m, int n0, int k0, uint32_t (&b)[kP][2][2]) {
  static_assert(kP <= M::kHas, "parts");
  const int l = threadIdx.x & 31;
  const uint32_t addr = smem_u32(m.p + m.at(k0 + (l & 15), n0 + (l >> 4) * 8));
#pragma unroll
  for (int q = 0; q < kP; ++q) {
    uint32_t r[4];
    ldmatrix4_trans<true>(addr + q * m.kSize * 2, r);
    b[q][0][0] = r[0], b[q][0][1] = r[1], b[q][1][0] = r[2], b[q][1][1] = r[3];
  }
}
// The same of 32 rows of k and 8 columns: [part][k / 16][k / 8 % 2].
template <int kP, typename M>
__device__ __forceinline__ void load_bt_tall(const M& m, int n0, int k0, uint32_t (&b)[kP][2][2]) {
  static_assert(kP <= M::kHas, "parts");
  const uint32_t addr = smem_u32(m.p + m.at(k0 + (threadIdx.x & 31), n0));
#pragma unroll
  for (int q = 0; q < kP; ++q) {
    uint32_t r[4];
    ldmatrix4_trans<true>(addr + q * m.kSize * 2, r);
    b[q][0][0] = r[0], b[q][0][1] = r[1], b[q][1][0] = r[2], b[q][1][1] = r[3];
  }
}

// d + e (+ f) += a b, column tile x of b: part i of a with part j of b where i + j <= 2, to d, e and f by i + j.
template <int kPA, int kPB>
__device__ __forceinline__ void mma(float (&d)[4], float (&e)[4], float (&f)[4], const uint32_t (&a)[kPA][4], const uint32_t (&b)[kPB][2][2],
                                    int x) {
#pragma unroll
  for (int i = 0; i < kPA; ++i)
#pragma unroll
    for (int s = 2; s >= 0; --s)
      if (s - i >= 0 && s - i < kPB)
        mma_16816_bf16<true, false>(s == 0 ? d : s == 1 ? e : f, a[i][0], a[i][1], a[i][2], a[i][3], b[s - i][x][0], b[s - i][x][1]);
}
template <int kPA, int kPB>
__device__ __forceinline__ void mma(float (&d)[4], float (&e)[4], const uint32_t (&a)[kPA][4], const uint32_t (&b)[kPB][2][2], int x) {
  mma(d, e, e, a, b, x);
}

// ---- what the kernels share ----------------------------------------------------

// A wait for a copy that a working device always completes lasts 2 s at the most; where it runs out the results are NaN.
constexpr int kWaitUs = 2000000;
__device__ const int g_never = 0;

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
  uint64_t wait_ns;
  int withheld;  // a chunk that is not copied (its waits run out), or -1
  bool wide;   // q, k, dq and dk in 16-byte pieces
  bool pairs;  // v, o, dO and dV two at a time
  bool even;   // states two at a time
  bool quads;  // states four at a time
  void* o;
  float *h_last, *states;
  // workspace: per chunk, stream and key head the parts of k and q; per value head those of N and M, and the gates
  unsigned char *keys, *heads;
  // backward
  const float* dh_last;
  float *dS, *R, *dots, *sum_q, *sum_k;
  void *dq, *dk, *dv;
  float *dg, *dbeta, *dh0;
  long long dgt, dgb, dbt, dbb;
};

// The workspace's parts.
template <typename T, int KD>
using KeyMat = Mat<C, KD, kParts<T>>;
using SquareMat = Mat<C, C, 3>;
using LowerMat = MatOf<Lower<C>, 3>;
template <typename T, int KD>
constexpr size_t kKeysBytes = 2 * KeyMat<T, KD>::kBytes;
constexpr size_t kHeadBytes = 2 * LowerMat::kBytes + sizeof(Gates);

// The resets of a chunk, for the loops over its pieces.  They come from memory and not from the stage: what a stage holds after a wait
// that has run out may change at any time, and these loops hold barriers.
__device__ __forceinline__ unsigned long long cuts_of(const DeltaArgs& a, int n, int chunks, int b, int h) {
  if (!a.reset || n < 0 || n >= chunks) return 0ull;
  const unsigned char* head = a.heads + ((size_t)((long long)n * a.B + b) * a.H + h) * kHeadBytes;
  return *reinterpret_cast<const unsigned long long*>(head + LowerMat::kBytes + offsetof(Gates, cuts));
}

__device__ __forceinline__ int length_of(const DeltaArgs& a, int b) {
  return a.lengths ? min(max(a.lengths[b], 0), a.T) : a.T;
}

// Copies that this thread waits for (of `bytes`; zeros for the rest of 16, 4).
__device__ __forceinline__ void copy16(void* to, const void* from, int bytes) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(smem_u32(to)), "l"(from), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copy4(void* to, const void* from, int bytes) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(smem_u32(to)), "l"(from), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int kLeft>
__device__ __forceinline__ void copies_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(kLeft) : "memory");
}
template <int kBytes, int kBy>
__device__ __forceinline__ void fetch(void* to, const void* from) {
#pragma unroll
  for (int i = 0; i < kBytes; i += kBy * 16)
    if (i + kBy * 16 <= kBytes || i + (int)threadIdx.x * 16 < kBytes)
      copy16(static_cast<char*>(to) + i + threadIdx.x * 16, static_cast<const char*>(from) + i + threadIdx.x * 16, 16);
}

// Two neighbouring values of a row (the second only if it lies in the row).
template <typename T>
__device__ __forceinline__ float2 get2(const T* row, int col, int D, bool pairs) {
  if (pairs) return col < D ? Pair<T>::get(*reinterpret_cast<const typename Pair<T>::Raw*>(row + col)) : make_float2(0.0f, 0.0f);
  return make_float2(col < D ? to_f32(row[col]) : 0.0f, col + 1 < D ? to_f32(row[col + 1]) : 0.0f);
}
// The same as they lie in memory, to be converted where they are used: nothing waits for them before.  (Without the empty
// statement the compiler converts them where they are loaded, and a chunk forward took 0.6 us more.)
template <typename T>
struct Raw2 {
  typename Pair<T>::Raw v;
  __device__ __forceinline__ void load(const T* row, int col, int D, bool pairs, bool in) {
    v = Pair<T>::put(0.0f, 0.0f);
    if (pairs) {
      if (in && col < D) v = *reinterpret_cast<const typename Pair<T>::Raw*>(row + col);
    } else {
      if (in && col < D) v.x = row[col];
      if (in && col + 1 < D) v.y = row[col + 1];
    }
  }
  __device__ __forceinline__ float2 get() {
    if constexpr (sizeof(T) == 4) {
      asm volatile("" : "+f"(v.x), "+f"(v.y));
    } else {
      uint32_t& bits = reinterpret_cast<uint32_t&>(v);
      asm volatile("" : "+r"(bits));
    }
    return Pair<T>::get(v);
  }
};
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

// ---- per chunk and key head: copies of q and k, gates, N and M --------------------

template <typename T, int KD>
struct PrepareShared {
  static constexpr size_t kFirst = kKeysBytes<T, KD> > LowerMat::kBytes ? kKeysBytes<T, KD> : LowerMat::kBytes;
  static constexpr int kPitch = C + 4;
  KeyMat<T, KD> K, Q;
  LowerMat N;  // where K and Q were
  Gates* gates;
  LowerMat M;    // behind the gates, as in the workspace
  SquareMat AB;  // A B
  Mat<C / 2, C / 2, 3> BH;
  float* A;  // [C][kPitch]; then N's blocks on the diagonal
  static constexpr uint32_t kTail = sizeof(Gates) + LowerMat::kBytes;
  static constexpr size_t kBytes = kFirst + kTail + SquareMat::kBytes + decltype(BH)::kBytes + C * kPitch * 4;
  __device__ __forceinline__ explicit PrepareShared(unsigned char* p)
      : K{reinterpret_cast<bf16*>(p)}, Q{K.p + K.kSize * kParts<T>}, N{K.p}, gates(reinterpret_cast<Gates*>(p + kFirst)),
        M{reinterpret_cast<bf16*>(gates + 1)}, AB{M.p + M.kSize * 3}, BH{AB.p + AB.kSize * 3},
        A(reinterpret_cast<float*>(BH.p + BH.kSize * 3)) {}
};

// Rows of q or k as the MMAs read them: in parts, zeros past the stream's length and past Dk.
template <typename T, int KD>
__device__ __forceinline__ void fill_keys(const KeyMat<T, KD>& to, const T* p, long long t_stride, int rows, int Dk, bool wide) {
  constexpr int kPer = 16 / (int)sizeof(T), kRounds = C * (KD / kPer) / kThreads;
  uint4 raw[kRounds];
#pragma unroll
  for (int x = 0; x < kRounds; ++x) {
    const int i = threadIdx.x + x * kThreads, row = i / (KD / kPer), col = i % (KD / kPer) * kPer;
    raw[x] = make_uint4(0u, 0u, 0u, 0u);
    if (row < rows && col < Dk) {
      if (wide) {
        raw[x] = *reinterpret_cast<const uint4*>(p + row * t_stride + col);
      } else {
        T v[kPer];
#pragma unroll
        for (int e = 0; e < kPer; ++e) v[e] = col + e < Dk ? p[row * t_stride + col + e] : from_f32<T>(0.0f);
        raw[x] = *reinterpret_cast<const uint4*>(v);
      }
    }
  }
#pragma unroll
  for (int x = 0; x < kRounds; ++x) {
    const int i = threadIdx.x + x * kThreads, row = i / (KD / kPer), col = i % (KD / kPer) * kPer;
    if constexpr (std::is_same_v<T, bf16>) {
      *reinterpret_cast<uint4*>(to.p + to.at(row, col)) = raw[x];
    } else {
      const typename Pair<T>::Raw* h = reinterpret_cast<const typename Pair<T>::Raw*>(&raw[x]);
#pragma unroll
      for (int e = 0; e < kPer / 2; ++e) {
        const float2 f = Pair<T>::get(h[e]);
        to.put(row, col + 2 * e, f.x, f.y);
      }
    }
  }
}

// high + low, low at most half a unit of high in its last place.  (A sum's rounding: what the terms lack of their own part of it.)
struct TwoFloats {
  float high, low;
  __device__ __forceinline__ TwoFloats operator+(const TwoFloats& o) const {
    const float s = __fadd_rn(high, o.high), mine = __fsub_rn(s, o.high);
    const float rest = __fadd_rn(__fadd_rn(__fsub_rn(high, mine), __fsub_rn(o.high, __fsub_rn(s, mine))), __fadd_rn(low, o.low));
    const float t = __fadd_rn(s, rest);
    return {t, __fsub_rn(rest, __fsub_rn(t, s))};
  }
};

// One warp: a chunk's sums of g, the decays that follow, beta (rows lane and lane + 32).  The sums are of two parts, so that
// differences of far ones keep their digits, and begin anew at a reset, whose own g counts as zero.
struct RawGates {
  float g[2], beta[2];
  unsigned char reset[2];
  __device__ __forceinline__ void load(const DeltaArgs& a, int t0, int rows, int b, int h) {
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const int row = (threadIdx.x & 31) + 32 * s;
      const long long t = t0 + row;
      const bool in = row < rows;
      g[s] = in ? a.g[t * a.gt + b * a.gb + h] : 0.0f;
      beta[s] = in ? a.beta[t * a.bt + b * a.bb + h] : 0.0f;
      reset[s] = in && a.reset ? a.reset[t * a.B + b] : 0;
    }
  }
};
__device__ __forceinline__ void make_gates(const RawGates& raw, Gates& gates) {
  const int lane = threadIdx.x & 31;
  TwoFloats G[2];
  unsigned cut[2];
#pragma unroll
  for (int s = 0; s < 2; ++s) {
    const int row = lane + 32 * s;
    const float g = raw.g[s] < kLeastG ? kLeastG : raw.g[s];
    const bool reset = raw.reset[s] != 0;
    gates.beta[row] = raw.beta[s];
    cut[s] = __ballot_sync(0xffffffffu, reset);
    const unsigned before = cut[s] & (2u << lane) - 1u;
    const int start = before ? 31 - __clz((int)before) : 0;
    TwoFloats x{reset ? 0.0f : g, 0.0f};
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
      const TwoFloats y{__shfl_up_sync(0xffffffffu, x.high, d), __shfl_up_sync(0xffffffffu, x.low, d)};
      if (lane - d >= start) x = y + x;
    }
    G[s] = x;
  }
  const TwoFloats first{__shfl_sync(0xffffffffu, G[0].high, 31), __shfl_sync(0xffffffffu, G[0].low, 31)};
  if (!(cut[1] & (2u << lane) - 1u)) G[1] = first + G[1];
  const TwoFloats last{__shfl_sync(0xffffffffu, G[1].high, 31), __shfl_sync(0xffffffffu, G[1].low, 31)};
  const unsigned long long cuts = cut[0] | (unsigned long long)cut[1] << 32;
#pragma unroll
  for (int s = 0; s < 2; ++s) {
    const int row = lane + 32 * s;
    const float e = expf(G[s].high);
    gates.g_high[row] = G[s].high;
    gates.g_low[row] = G[s].low;
    gates.gam[row] = cut_before(cuts, row) ? 0.0f : fmaf(e, G[s].low, e);
    gates.dec[row] = row < 63 && cuts >> (row + 1) ? 0.0f : expf((last.high - G[s].high) + (last.low - G[s].low));
  }
  if (lane == 0) gates.cuts = cuts, gates.pad = 0ull;
}

// Two blocks to an SM, so that one's loads and barriers lie behind the other's products: 2048 chunks of 128 wide bf16 keys 82 us, in
// which 212 MB move (31 us at a copy's rate).  (With 16 warps to a block registers spill: 88 us where 8 took 77.)
template <typename T, int KD>
__global__ void __launch_bounds__(kThreads, 2) delta_prepare_kernel(const DeltaArgs a) {
  extern __shared__ __align__(128) unsigned char smem[];
  constexpr int P = kParts<T>;
  using Sh = PrepareShared<T, KD>;
  constexpr int kPitch = Sh::kPitch;
  const Sh sh(smem);
  Gates& gates = *sh.gates;
  begin_op();
  const int Hk = a.H / a.share, hk = (int)(blockIdx.x % Hk), b = (int)(blockIdx.x / Hk % a.B), n = (int)(blockIdx.x / Hk / a.B);
  const int t0 = n * C, rows = min(length_of(a, b) - t0, C);
  if (rows <= 0) return;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane_g(), t = lane_t();
  const int i0 = (warp & 3) * 16, side = (warp >> 2) * 32;  // a warp's 16 rows and 32 columns
  RawGates raw;
  if (warp == 7) raw.load(a, t0, rows, b, hk * a.share);
  fill_keys<T, KD>(sh.K, static_cast<const T*>(a.k) + t0 * a.ks.t + b * a.ks.b + hk * a.ks.h, a.ks.t, rows, a.Dk, a.wide);
  fill_keys<T, KD>(sh.Q, static_cast<const T*>(a.q) + t0 * a.qs.t + b * a.qs.b + hk * a.qs.h, a.qs.t, rows, a.Dk, a.wide);
  if (warp == 7) make_gates(raw, gates);
  fence_proxy_async_shared();
  __syncthreads();
  if (threadIdx.x == 0)
    bulk_copy_s2g(a.keys + (size_t)blockIdx.x * kKeysBytes<T, KD>, smem_u32(smem), (uint32_t)kKeysBytes<T, KD>);
  __syncwarp();

  float kk[4][4] = {}, qk[4][4] = {};  // K K^T and Q K^T
  if (side < i0 + 16) {
    float ke[4][4] = {}, qe[4][4] = {};
#pragma unroll
    for (int k0 = 0; k0 < KD; k0 += 16) {
      uint32_t fk[P][4], fq[P][4], fb[2][P][2][2];
      load_a<P>(sh.K, i0, k0, fk);
      load_a<P>(sh.Q, i0, k0, fq);
      load_b<P>(sh.K, side, k0, fb[0]);
      load_b<P>(sh.K, side + 16, k0, fb[1]);
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        mma(kk[x], ke[x], fk, fb[x >> 1], x & 1);
        mma(qk[x], qe[x], fq, fb[x >> 1], x & 1);
      }
    }
#pragma unroll
    for (int x = 0; x < 4; ++x)
#pragma unroll
      for (int r = 0; r < 4; ++r) kk[x][r] += ke[x][r], qk[x][r] += qe[x][r];
  }

  for (int h = hk * a.share; h < (hk + 1) * a.share; ++h) {
    if (threadIdx.x == 0) bulk_wait_read();  // of K and Q, or of the head before
    __syncthreads();
    if (h > hk * a.share) {
      if (warp == 7) {
        raw.load(a, t0, rows, b, h);
        make_gates(raw, gates);
      }
      __syncthreads();
    }
    const unsigned long long cuts = gates.cuts;
#pragma unroll
    for (int x = 0; x < 4; ++x)
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        const int i = i0 + g + 8 * r, j = side + x * 8 + 2 * t;
        if (!LowerMat::has(i0, side)) continue;
        if (side + x * 8 >= i0 + 16) {
          sh.M.put(i, j, 0.0f, 0.0f);
          sh.N.put(i, j, 0.0f, 0.0f);
          continue;
        }
        float m[2], v[2], w[2];
#pragma unroll
        for (int y = 0; y < 2; ++y) {
          const float dist = (gates.g_high[i] - gates.g_high[j + y]) + (gates.g_low[i] - gates.g_low[j + y]);
          const bool same = i >= j + y && !(cuts && cut_between(cuts, j + y, i));
          const float D = same ? expf(dist) : 0.0f;
          m[y] = same ? D * qk[x][2 * r + y] : 0.0f;
          v[y] = same && i > j + y ? D * kk[x][2 * r + y] : 0.0f;
          w[y] = v[y] != 0.0f ? v[y] * gates.beta[j + y] : 0.0f;  // (beta of another document: anything)
        }
        sh.M.put(i, j, m[0], m[1]);
        if (side + x * 8 < i0) sh.AB.put(i, j, w[0], w[1]);
        *reinterpret_cast<float2*>(sh.A + i * kPitch + j) = make_float2(v[0], v[1]);
      }
    __syncthreads();

    // N = A - A B N.  16 x 16 blocks on the diagonal: a lane has a column, whose rows follow one another
    if (warp < 4 && lane < 16) {
      const int o = warp * 16;
      float* D = sh.A + o * kPitch + o;
      float x[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) x[i] = i > lane ? D[i * kPitch + lane] : 0.0f;
#pragma unroll
      for (int j = 0; j < 15; ++j) {
        const float bx = j > lane ? gates.beta[o + j] * x[j] : 0.0f;
#pragma unroll
        for (int i = j + 1; i < 16; ++i) x[i] = fmaf(-D[i * kPitch + j], bx, x[i]);
      }
      __syncwarp(0xffffu);
#pragma unroll
      for (int i = 0; i < 16; ++i) D[i * kPitch + lane] = i > lane ? x[i] : 0.0f;
    }
    __syncthreads();
    auto put_n = [&](int i, int j, float x, float y) {
      if (cuts) x = cut_between(cuts, j, i) ? 0.0f : x, y = cut_between(cuts, j + 1, i) ? 0.0f : y;
      sh.N.put(i, j, x, y);
    };
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      const int p = threadIdx.x + x * kThreads, o = p / 128 * 16, i = o + p % 128 / 8, j = o + p % 8 * 2;
      const float2 v = *reinterpret_cast<const float2*>(sh.A + i * kPitch + j);
      put_n(i, j, v.x, v.y);
    }
    __syncthreads();
    // for [L 0; X R]: N_X = H - N_R B H with H = X - X B N_L; tiles of 16 x 8
#pragma unroll
    for (int half = 16; half < C; half *= 2) {
      const bool mine = half == 32 || warp < 4;
      const int o = half == 16 ? (warp >> 1 & 1) * 32 : 0;               // the block's first row
      const int r0 = half == 16 ? 0 : (warp & 1) * 16;                   // the tile in X
      const int c0 = half == 16 ? (warp & 1) * 8 : (warp >> 1) * 8;
      const int h0 = half == 16 ? (warp >> 1 & 1) * 16 : 0;              // H's first row in BH
      float H[4];
      if (mine) {
        float d[4] = {}, e[4] = {}, e2[4] = {};
#pragma unroll
        for (int k0 = 0; k0 < half; k0 += 16) {
          uint32_t fa[3][4], fb[3][2][2];
          load_a<3>(sh.AB, o + half + r0, o + k0, fa);
          load_bt<3>(sh.N, o + (c0 & ~8), o + k0, fb);
          if (c0 & 8) mma(d, e, e2, fa, fb, 1);
          else mma(d, e, e2, fa, fb, 0);
        }
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          const int i = o + half + r0 + g + 8 * r, j = o + c0 + 2 * t;
          float bh[2];
#pragma unroll
          for (int y = 0; y < 2; ++y) {
            const float v = sh.A[i * kPitch + j + y] - (d[2 * r + y] + (e[2 * r + y] + e2[2 * r + y]));
            H[2 * r + y] = cuts && cut_between(cuts, j + y, i) ? 0.0f : v;
            bh[y] = H[2 * r + y] != 0.0f ? gates.beta[i] * H[2 * r + y] : 0.0f;
          }
          sh.BH.put(h0 + r0 + g + 8 * r, c0 + 2 * t, bh[0], bh[1]);
        }
      }
      __syncthreads();
      if (mine) {
        float d[4] = {}, e[4] = {}, e2[4] = {};
#pragma unroll
        for (int k0 = 0; k0 < half; k0 += 16) {
          uint32_t fa[3][4], fb[3][2][2];
          load_a<3>(sh.N, o + half + r0, o + half + k0, fa);
          load_bt<3>(sh.BH, c0 & ~8, h0 + k0, fb);
          if (c0 & 8) mma(d, e, e2, fa, fb, 1);
          else mma(d, e, e2, fa, fb, 0);
        }
#pragma unroll
        for (int r = 0; r < 2; ++r)
          put_n(o + half + r0 + g + 8 * r, o + c0 + 2 * t, H[2 * r] - (d[2 * r] + (e[2 * r] + e2[2 * r])),
                H[2 * r + 1] - (d[2 * r + 1] + (e[2 * r + 1] + e2[2 * r + 1])));
      }
      __syncthreads();
    }
    fence_proxy_async_shared();
    __syncthreads();
    if (threadIdx.x == 0) {
      unsigned char* head = a.heads + ((size_t)((long long)n * a.B + b) * a.H + h) * kHeadBytes;
      bulk_copy_s2g(head, smem_u32(sh.N.p), LowerMat::kBytes);
      bulk_copy_s2g(head + LowerMat::kBytes, smem_u32(sh.gates), Sh::kTail);
    }
  }
  if (threadIdx.x == 0) bulk_wait_all();
}

// ---- along the chunks -------------------------------------------------------------

// What a chunk brings along: parts of K and Q, N, gates, M.  Every block asks for its own copy: the blocks of a head read the same
// 69 KB (bf16, 128 wide keys) from L2.
template <typename T, int KD>
struct Stage {
  KeyMat<T, KD> K, Q;
  LowerMat N;
  Gates* gates;
  LowerMat M;
  static constexpr uint32_t kKeys = (uint32_t)kKeysBytes<T, KD>, kHead = kHeadBytes;
  static constexpr size_t kBytes = kKeys + kHead;
  __device__ __forceinline__ explicit Stage(unsigned char* p)
      : K{reinterpret_cast<bf16*>(p)}, Q{K.p + K.kSize * kParts<T>}, N{Q.p + Q.kSize * kParts<T>},
        gates(reinterpret_cast<Gates*>(N.p + N.kSize * 3)), M{reinterpret_cast<bf16*>(gates + 1)} {}
  // One thread; nobody reads the stage any more.
  __device__ __forceinline__ void load(const DeltaArgs& a, int n, int b, int h, uint32_t bar) const {
    const size_t at = (size_t)n * a.B + b;
    mbar_arrive_expect_tx(bar, kKeys + kHead);
    if (n == a.withheld) return;
    bulk_copy_g2s(smem_u32(K.p), a.keys + (at * (a.H / a.share) + h / a.share) * kKeysBytes<T, KD>, kKeys, bar);
    bulk_copy_g2s(smem_u32(N.p), a.heads + (at * a.H + h) * kHeadBytes, kHead, bar);
  }
};
// Chunks in shared memory at a time: two, or one where the parts of wide keys fill it.
template <typename T, int KD>
constexpr int kStages = kParts<T> > 1 && KD == 128 ? 1 : 2;

// The kernels along the chunks have 8 warps for what leads from one state to the next, 4 that work beside them and one that asks
// for the chunks.  Barriers among them:
constexpr int kChainThreads = 256, kSideThreads = 128, kBothThreads = kChainThreads + kSideThreads, kAllThreads = kBothThreads + 32;
constexpr uint32_t kChain = 1, kSide = 2, kToSide = 3, kToChain = 4, kStateToSide = 5;

// Two rings of barriers: a stage's chunk has come; all warps have read it.
template <int kN>
struct Ring {
  uint32_t full, empty;  // addresses
  uint64_t limit;
  bool ok;
  __device__ __forceinline__ Ring(uint64_t* bars, uint64_t limit_) : full(smem_u32(bars)), empty(smem_u32(bars + kN)), limit(limit_), ok(true) {}
  __device__ __forceinline__ void init() const {  // one thread
#pragma unroll
    for (int i = 0; i < kN; ++i) mbar_init(full + 8 * i, 1), mbar_init(empty + 8 * i, kBothThreads / 32);
    fence_mbarrier_init_cluster();
  }
  __device__ __forceinline__ bool full_by(int k) const {
    return mbar_wait_bounded<false>(full + k % kN * 8, (uint32_t)(k / kN) & 1u, limit, &g_never);
  }
  // The k-th chunk (once a wait has run out, no further one is waited for).  What follows a wait takes the same branches either way:
  // warps whose waits end differently meet at the same barriers.
  __device__ __forceinline__ bool wait_full(int k) {
    ok = ok && full_by(k);
    return ok;
  }
  // The thread that asks for the chunks: the k-th one's stage has been read, and what was asked for last has come.
  __device__ __forceinline__ bool wait_empty(int k) {
    ok = ok && (k < kN || (mbar_wait_bounded<false>(empty + k % kN * 8, (uint32_t)(k / kN - 1) & 1u, limit, &g_never) && full_by(k - kN)));
    return ok;
  }
  // The same, when it has asked for `asked` of them: a block does not end while its copies are under way.
  __device__ __forceinline__ void wait_rest(int asked) const {
    for (int k = max(asked - kN, 0); k < asked; ++k) full_by(k);
  }
  __device__ __forceinline__ void release(int k) const {  // a whole warp
    __syncwarp();
    if ((threadIdx.x & 31) == 0) mbar_arrive(empty + k % kN * 8);
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
  __device__ __forceinline__ void each(F f) {  // f(row, column, its value, the next column's)
#pragma unroll
    for (int n = 0; n < kTiles; ++n)
#pragma unroll
      for (int r = 0; r < 2; ++r) f(row0() + lane_g() + 8 * r, col0() + n * 8 + 2 * lane_t(), x[n][2 * r], x[n][2 * r + 1]);
  }
  __device__ __forceinline__ void load(const float* p, const DeltaArgs& a, int v0) {
    each([&](int r, int c, float& x, float& y) {
      const float2 v = p && r < a.Dk ? get2(p + (long long)r * a.Dv, v0 + c, a.Dv, a.even) : make_float2(0.0f, 0.0f);
      x = v.x, y = v.y;
    });
  }
  __device__ __forceinline__ void store(float* p, const DeltaArgs& a, int v0) {
    each([&](int r, int c, float& x, float& y) {
      if (r < a.Dk) put2(p + (long long)r * a.Dv, v0 + c, a.Dv, a.even, x, y);
    });
  }
  __device__ __forceinline__ void split(const Mat<KD, NV, 3>& to) {
    each([&](int r, int c, float& x, float& y) { to.put(r, c, x, y); });
  }
};

// d + e += rows m0 of A (kLength columns from k0 on) times columns n0.. of B: kTiles times 8 columns, PA and PB parts.  The
// operands of a step are asked for before the MMAs of the one before.
template <int PA, int PB, int kTiles, bool kTransA>
struct Operands {
  static constexpr int kDepthOf = kTiles == 1 ? 32 : 16;  // rows of k to a step
  uint32_t a[kDepthOf / 16][PA][4], b[kTiles == 1 ? 1 : kTiles / 2][PB][2][2];
  template <typename MatA, typename MatB>
  __device__ __forceinline__ void load(const MatA& A, int m0, const MatB& B, int n0, int k0) {
#pragma unroll
    for (int s = 0; s < kDepthOf / 16; ++s) {
      if constexpr (kTransA) load_at<PA>(A, m0, k0 + 16 * s, a[s]);
      else load_a<PA>(A, m0, k0 + 16 * s, a[s]);
    }
    if constexpr (kTiles == 1) {
      load_bt_tall<PB>(B, n0, k0, b[0]);
    } else {
#pragma unroll
      for (int n = 0; n < kTiles / 2; ++n) load_bt<PB>(B, n0 + 16 * n, k0, b[n]);
    }
  }
  __device__ __forceinline__ void multiply(float (&d)[kTiles][4], float (&e)[kTiles][4], float (&f)[4]) {
    if constexpr (kTiles == 1) {
#pragma unroll
      for (int s = 0; s < 2; ++s) mma(d[0], e[0], f, a[s], b[0], s);
    } else {
#pragma unroll
      for (int n = 0; n < kTiles; ++n) mma(d[n], e[n], a[0], b[n / 2], n & 1);
    }
  }
};
template <int PA, int PB, int kTiles, int kLength, bool kTransA, typename MatA, typename MatB>
__device__ __forceinline__ void product(float (&d)[kTiles][4], float (&e)[kTiles][4], const MatA& A, int m0, const MatB& B, int n0, int k0) {
  using Ops = Operands<PA, PB, kTiles, kTransA>;
  constexpr int kSteps = kLength / Ops::kDepthOf;
  Ops ops[2];
  float f[4] = {};  // (a third chain of sums where there is one tile)
  ops[0].load(A, m0, B, n0, k0);
#pragma unroll
  for (int k = 0; k < kSteps; ++k) {
    if (k + 1 < kSteps) ops[(k + 1) & 1].load(A, m0, B, n0, k0 + (k + 1) * Ops::kDepthOf);
    ops[k & 1].multiply(d, e, f);
  }
  if constexpr (kTiles == 1)
#pragma unroll
    for (int r = 0; r < 4; ++r) e[0][r] += f[r];
}
// What a chunk adds to S, keys^T rows (P parts of the keys).  It is summed from zero and added once: an MMA's sum is cut, not rounded,
// to 24 bits, and a state that went through the MMAs would drift towards zero by two units of its last place a chunk (4 MMAs).
template <int KD, int NV>
struct StateSum {
  using Part = StatePart<KD, NV>;
  float d[Part::kTiles][4] = {}, e[Part::kTiles][4] = {};
  template <int P, int kHas>
  __device__ __forceinline__ void add(const Mat<C, KD, kHas>& keys, const Mat<C, NV, 3>& rows) {
    product<P, 3, Part::kTiles, C, true>(d, e, keys, Part::row0(), rows, Part::col0(), 0);
  }
  __device__ __forceinline__ void add_to(Part& s) const {
#pragma unroll
    for (int c = 0; c < Part::kTiles; ++c)
#pragma unroll
      for (int r = 0; r < 4; ++r) s.x[c][r] += d[c][r] + e[c][r];
  }
};
// The same for a matrix [64][64] that is zero above the diagonal.
template <int PA, int PB, int kTiles, bool kTransA, typename MatA, typename MatB>
__device__ __forceinline__ void product_lower(float (&d)[kTiles][4], float (&e)[kTiles][4], const MatA& A, int m0, const MatB& B, int n0) {
  if (kTransA ? m0 >= C / 2 : m0 < C / 2) product<PA, PB, kTiles, C / 2, kTransA>(d, e, A, m0, B, n0, kTransA ? C / 2 : 0);
  else product<PA, PB, kTiles, C, kTransA>(d, e, A, m0, B, n0, 0);
}

template <typename T, int KD, int NV>
struct ForwardShared {
  static constexpr int kN = kStages<T, KD>;
  using St = Stage<T, KD>;
  using SMat = Mat<KD, NV, 3>;
  SMat S;  // before the chunk; the next one's behind it
  Mat<C, NV, 3> X, Ud, U;
  uint64_t* bars;  // [2 kN]
  static constexpr size_t kBytes = kN * St::kBytes + 2 * SMat::kBytes + 3 * decltype(X)::kBytes + 16 * kN;
  __device__ __forceinline__ explicit ForwardShared(unsigned char* p)
      : S{reinterpret_cast<bf16*>(p + kN * St::kBytes)}, X{S.p + 2 * S.kSize * 3}, Ud{X.p + X.kSize * 3}, U{Ud.p + Ud.kSize * 3},
        bars(reinterpret_cast<uint64_t*>(U.p + U.kSize * 3)) {}
  __device__ __forceinline__ SMat state(int n) const { return SMat{S.p + (n & 1) * S.kSize * 3}; }
};

// Warps 0 to 7: X, Y and the next state.  Warps 8 to 11: O, from the state and U.  (When 8 warps did all of it, a chunk of 64 x 128
// x 16 took 2.8 us instead of 2.2.)
template <typename T, int KD, int NV>
__global__ void __launch_bounds__(kAllThreads, 1) delta_forward_kernel(const DeltaArgs a) {
  extern __shared__ __align__(128) unsigned char smem[];
  constexpr int P = kParts<T>;
  using Sh = ForwardShared<T, KD, NV>;
  using St = typename Sh::St;
  constexpr int kN = Sh::kN;
  const Sh sh(smem);
  begin_op();
  const int v0 = (int)(blockIdx.x % a.tiles) * NV, bh = blockIdx.x / a.tiles, h = bh % a.H, b = bh / a.H;
  const int len = length_of(a, b), chunks = (len + C - 1) / C;
  const int warp = threadIdx.x >> 5, g = lane_g(), t = lane_t();
  const long long DD = (long long)a.Dk * a.Dv;
  T* o = static_cast<T*>(a.o) + b * a.os.b + h * a.os.h;
  Ring<kN> ring(sh.bars, a.wait_ns);
  StatePart<KD, NV> s;
  if (warp < 8) {
    s.load(a.h0 ? a.h0 + (long long)bh * DD : nullptr, a, v0);
    s.split(sh.S);
  }
  if (threadIdx.x == kBothThreads) ring.init();
  __syncthreads();

  if (warp == kBothThreads / 32) {
    if (threadIdx.x == kBothThreads) {
      int n = 0;
      for (; n < chunks && ring.wait_empty(n); ++n) St(smem + n % kN * St::kBytes).load(a, n, b, h, ring.full + n % kN * 8);
      ring.wait_rest(n);
    }
  } else if (warp < 8) {
    constexpr int kTiles = NV / 16;  // a warp's 16 rows of the chunk and half of the columns
    const int rb = (warp < 4 ? warp : 7 - warp) * 16;  // warps w and w + 4 share a part of the SM: of triangles, a short and a long row
    const int cb = (warp >> 2) * (NV / 2);
    const T* v = static_cast<const T*>(a.v) + b * a.vs.b + h * a.vs.h;
    Raw2<T> vx[kTiles][2];
    auto fetch_v = [&](int n) {
#pragma unroll
      for (int x = 0; x < kTiles; ++x)
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          const int time = n * C + rb + g + 8 * r;
          vx[x][r].load(v + time * a.vs.t, v0 + cb + x * 8 + 2 * t, a.Dv, a.pairs, time < len);
        }
    };
    fetch_v(0);
    unsigned long long cuts_ahead = cuts_of(a, 0, chunks, b, h);
    for (int n = 0; n < chunks; ++n) {
      const bool came = ring.wait_full(n);
      __syncwarp();
      const unsigned long long cuts = cuts_ahead;
      cuts_ahead = cuts_of(a, n + 1, chunks, b, h);
      const St now(smem + n % kN * St::kBytes);
      const auto S0 = sh.state(n);
      const Gates& gate = *now.gates;
      float2 vn[kTiles][2];
#pragma unroll
      for (int x = 0; x < kTiles; ++x)
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          vn[x][r] = vx[x][r].get();
          if (!came) vn[x][r] = make_float2(kNaN, kNaN);
        }
      fetch_v(n + 1);
      // S0 and Y for the backward pass
      float* kept = a.states ? a.states + (((long long)n * a.B + b) * a.H + h) * (a.Dk + C) * a.Dv : nullptr;
      if (kept) s.store(kept, a, v0);

      for (int lo = 0; lo < C;) {
        const int hi = piece_end(cuts, lo);
        float x[kTiles][4];  // X
        __syncwarp();
        {
          float d[kTiles][4] = {}, e[kTiles][4] = {};
          if (!cut_before(cuts, lo)) product<P, 3, kTiles, KD, false>(d, e, now.K, rb, S0, cb, 0);
#pragma unroll
          for (int r = 0; r < 2; ++r) {
            const int i = rb + g + 8 * r;
            const float gam = gate.gam[i], beta = gate.beta[i];
            const bool in = i >= lo && i < hi;
#pragma unroll
            for (int c = 0; c < kTiles; ++c) {
              x[c][2 * r] = vn[c][r].x - gam * (d[c][2 * r] + e[c][2 * r]);
              x[c][2 * r + 1] = vn[c][r].y - gam * (d[c][2 * r + 1] + e[c][2 * r + 1]);
              sh.X.put(i, cb + c * 8 + 2 * t, in ? beta * x[c][2 * r] : 0.0f, in ? beta * x[c][2 * r + 1] : 0.0f);
            }
          }
        }
        named_sync(kChain, kChainThreads);
        {
          float d[kTiles][4] = {}, e[kTiles][4] = {};
          product_lower<3, 3, kTiles, false>(d, e, now.N, rb, sh.X, cb);
          named_sync(kToChain, kBothThreads);  // the U before has been read
#pragma unroll
          for (int r = 0; r < 2; ++r) {
            const int i = rb + g + 8 * r;
            const bool in = i >= lo && i < hi;
            const float beta = gate.beta[i], dec = gate.dec[i];
#pragma unroll
            for (int c = 0; c < kTiles; ++c) {
              const float y = x[c][2 * r] - (d[c][2 * r] + e[c][2 * r]), z = x[c][2 * r + 1] - (d[c][2 * r + 1] + e[c][2 * r + 1]);
              const float p = in ? beta * y : 0.0f, q = in ? beta * z : 0.0f;
              if (kept && in) put2(kept + (long long)(a.Dk + i) * a.Dv, v0 + cb + c * 8 + 2 * t, a.Dv, a.even, y, z);
              sh.U.put(i, cb + c * 8 + 2 * t, p, q);
              if (hi == C) sh.Ud.put(i, cb + c * 8 + 2 * t, in ? dec * p : 0.0f, in ? dec * q : 0.0f);
            }
          }
        }
        if (hi == C && lo > 0) {  // the last piece's keys alone reach the next chunk
          for (int i = threadIdx.x; i < lo * KD; i += kChainThreads)
#pragma unroll
            for (int q = 0; q < P; ++q) now.K.p[q * now.K.kSize + i] = from_f32<bf16>(0.0f);
          fence_proxy_async_shared();  // (before a copy overwrites them)
        }
        named_arrive(kToSide, kBothThreads);
        named_sync(kChain, kChainThreads);
        lo = hi;
      }
      const float keep = gate.gam[C - 1];
      s.each([&](int, int, float& p, float& q) { p = cuts ? 0.0f : keep * p, q = cuts ? 0.0f : keep * q; });
      StateSum<KD, NV> more;
      more.template add<P>(now.K, sh.Ud);
      ring.release(n);
      more.add_to(s);
      s.split(sh.state(n + 1));
      if (n + 1 < chunks) named_arrive(kStateToSide, kBothThreads);
      named_sync(kChain, kChainThreads);
    }
    s.store(a.h_last + (long long)bh * DD, a, v0);
  } else {
    constexpr int kTiles = NV / 8;
    const int rb = (warp - 8) * 16;
    unsigned long long cuts_ahead = cuts_of(a, 0, chunks, b, h);
    for (int n = 0; n < chunks; ++n) {
      const bool came = ring.wait_full(n);
      __syncwarp();
      const unsigned long long cuts = cuts_ahead;
      cuts_ahead = cuts_of(a, n + 1, chunks, b, h);
      if (n > 0) named_sync(kStateToSide, kBothThreads);
      const St now(smem + n % kN * St::kBytes);
      const Gates& gate = *now.gates;
      for (int lo = 0; lo < C;) {
        const int hi = piece_end(cuts, lo);
        float d[kTiles][4] = {}, e[kTiles][4] = {};
        __syncwarp();
        if (!cut_before(cuts, lo)) {
          product<P, 3, kTiles, KD, false>(d, e, now.Q, rb, sh.state(n), 0, 0);
#pragma unroll
          for (int c = 0; c < kTiles; ++c)
#pragma unroll
            for (int r = 0; r < 4; ++r) d[c][r] = gate.gam[rb + g + 8 * (r >> 1)] * (d[c][r] + e[c][r]), e[c][r] = 0.0f;
        }
        named_arrive(kToChain, kBothThreads);
        named_sync(kToSide, kBothThreads);
        product_lower<3, 3, kTiles, false>(d, e, now.M, rb, sh.U, 0);
        if (hi == C) ring.release(n);
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          const int i = rb + g + 8 * r, time = n * C + i;
          if (i < lo || i >= hi || time >= len) continue;
#pragma unroll
          for (int c = 0; c < kTiles; ++c) {
            const float p = a.scale * (d[c][2 * r] + e[c][2 * r]), q = a.scale * (d[c][2 * r + 1] + e[c][2 * r + 1]);
            put2(o + time * a.os.t, v0 + c * 8 + 2 * t, a.Dv, a.pairs, came ? p : kNaN, came ? q : kNaN);
          }
        }
        lo = hi;
      }
    }
    for (long long i = (long long)len * NV + (threadIdx.x - kChainThreads); i < (long long)a.T * NV; i += kSideThreads) {
      const int c = v0 + (int)(i % NV);
      if (c < a.Dv) o[i / NV * a.os.t + c] = from_f32<T>(0.0f);
    }
  }
}

template <typename T, int KD, int NV>
struct BackwardShared {
  static constexpr int kN = kStages<T, KD>, kLPitch = NV + 4;
  using St = Stage<T, KD>;
  Mat<KD, NV, 3> S;                // dS
  Mat<C, NV, 3> Od, Z;             // scale gam dO; B dU, then - gam B R
  Mat<C, NV, kParts<T>> O;         // dO
  float* L;                        // scale M^T dO, [C][kLPitch]
  uint64_t* bars;                  // [2 kN]
  float* sums;                     // [8]
  static constexpr size_t kBytes = kN * St::kBytes + decltype(S)::kBytes + 2 * decltype(Z)::kBytes + decltype(O)::kBytes + C * kLPitch * 4 + 16 * kN + 32;
  __device__ __forceinline__ explicit BackwardShared(unsigned char* p)
      : S{reinterpret_cast<bf16*>(p + kN * St::kBytes)}, Od{S.p + S.kSize * 3}, Z{Od.p + Od.kSize * 3}, O{Z.p + Z.kSize * 3},
        L(reinterpret_cast<float*>(O.p + O.kSize * kParts<T>)), bars(reinterpret_cast<uint64_t*>(L + C * kLPitch)),
        sums(reinterpret_cast<float*>(bars + 2 * kN)) {}
};

// dS before a chunk from dS behind it; keeps the latter, R and <dS0, S0> for the gradients of the rest, and writes dV.  Warps 8 to
// 11 go ahead with what dO alone gives.
template <typename T, int KD, int NV>
__global__ void __launch_bounds__(kAllThreads, 1) delta_backward_kernel(const DeltaArgs a) {
  extern __shared__ __align__(128) unsigned char smem[];
  constexpr int P = kParts<T>;
  using Sh = BackwardShared<T, KD, NV>;
  using St = typename Sh::St;
  constexpr int kN = Sh::kN;
  const Sh sh(smem);
  begin_op();
  const int v0 = (int)(blockIdx.x % a.tiles) * NV, bh = blockIdx.x / a.tiles, h = bh % a.H, b = bh / a.H;
  const int len = length_of(a, b), chunks = (len + C - 1) / C;
  const int warp = threadIdx.x >> 5, g = lane_g(), t = lane_t();
  const long long DD = (long long)a.Dk * a.Dv;
  Ring<kN> ring(sh.bars, a.wait_ns);
  StatePart<KD, NV> s;
  if (warp < 8) {
    s.load(a.dh_last ? a.dh_last + (long long)bh * DD : nullptr, a, v0);
    s.split(sh.S);
  }
  if (threadIdx.x == kBothThreads) ring.init();
  __syncthreads();

  if (warp == kBothThreads / 32) {
    if (threadIdx.x == kBothThreads) {
      int k = 0;
      for (; k < chunks && ring.wait_empty(k); ++k)
        St(smem + k % kN * St::kBytes).load(a, chunks - 1 - k, b, h, ring.full + k % kN * 8);
      ring.wait_rest(k);
    }
  } else if (warp < 8) {
    constexpr int kTiles = NV / 16;
    const int rb = (warp < 4 ? warp : 7 - warp) * 16, cb = (warp >> 2) * (NV / 2);
    T* dv = static_cast<T*>(a.dv) + b * a.dvs.b + h * a.dvs.h;
    unsigned long long cuts_ahead = cuts_of(a, chunks - 1, chunks, b, h);
    for (int k = 0; k < chunks; ++k) {
      const int n = chunks - 1 - k;
      const bool came = ring.wait_full(k);
      __syncwarp();
      const unsigned long long cuts = cuts_ahead;
      cuts_ahead = cuts_of(a, n - 1, chunks, b, h);
      const St now(smem + k % kN * St::kBytes);
      const Gates& gate = *now.gates;
      const long long chunk = ((long long)n * a.B + b) * a.H + h;
      s.store(a.dS + chunk * DD, a, v0);
      StatePart<KD, NV> before;
      before.load(a.states + chunk * (a.Dk + C) * a.Dv, a, v0);
      float* R = a.R + chunk * C * a.Dv;

      for (int hi = C; hi > 0;) {  // pieces, the last first
        int lo = 0;
        for (int next = piece_end(cuts, lo); next < hi; next = piece_end(cuts, lo)) lo = next;
        float du[kTiles][4];
        __syncwarp();
        {  // dU = scale M^T dO + dec K dS
          float d[kTiles][4] = {}, e[kTiles][4] = {};
          if (hi == C) product<P, 3, kTiles, KD, false>(d, e, now.K, rb, sh.S, cb, 0);
          named_sync(kToChain, kBothThreads);  // this piece's L and Od
#pragma unroll
          for (int r = 0; r < 2; ++r) {
            const int i = rb + g + 8 * r;
            const bool in = i >= lo && i < hi;
            const float beta = gate.beta[i], dec = gate.dec[i];
#pragma unroll
            for (int c = 0; c < kTiles; ++c) {
              const int col = cb + c * 8 + 2 * t;
              const float2 l = *reinterpret_cast<const float2*>(sh.L + i * Sh::kLPitch + col);
#pragma unroll
              for (int y = 0; y < 2; ++y) {
                const float far = hi == C ? dec * (d[c][2 * r + y] + e[c][2 * r + y]) : 0.0f;
                du[c][2 * r + y] = in ? came ? (y ? l.y : l.x) + far : kNaN : 0.0f;
              }
              sh.Z.put(i, col, in ? beta * du[c][2 * r] : 0.0f, in ? beta * du[c][2 * r + 1] : 0.0f);
            }
          }
        }
        named_sync(kChain, kChainThreads);
        {  // R = dU - N^T B dU, dV = B R
          float d[kTiles][4] = {}, e[kTiles][4] = {};
          product_lower<3, 3, kTiles, true>(d, e, now.N, rb, sh.Z, cb);
          named_sync(kChain, kChainThreads);
#pragma unroll
          for (int r = 0; r < 2; ++r) {
            const int i = rb + g + 8 * r, time = n * C + i;
            const bool in = i >= lo && i < hi;
            const float beta = gate.beta[i], back = -gate.gam[i];
#pragma unroll
            for (int c = 0; c < kTiles; ++c) {
              const int col = cb + c * 8 + 2 * t;
              const float p = in ? du[c][2 * r] - (d[c][2 * r] + e[c][2 * r]) : 0.0f;
              const float q = in ? du[c][2 * r + 1] - (d[c][2 * r + 1] + e[c][2 * r + 1]) : 0.0f;
              const float bp = in ? beta * p : 0.0f, bq = in ? beta * q : 0.0f;
              if (lo == 0) sh.Z.put(i, col, in ? back * bp : 0.0f, in ? back * bq : 0.0f);
              if (!in) continue;
              put2(R + (long long)i * a.Dv, v0 + col, a.Dv, a.even, p, q);
              if (time < len) put2(dv + time * a.dvs.t, v0 + col, a.Dv, a.pairs, bp, bq);
            }
          }
        }
        if (lo == 0 && cuts) {  // rows behind the first reset do not reach the state before
          for (int i = threadIdx.x + hi * KD; i < C * KD; i += kChainThreads)
#pragma unroll
            for (int q = 0; q < P; ++q) now.K.p[q * now.K.kSize + i] = now.Q.p[q * now.Q.kSize + i] = from_f32<bf16>(0.0f);
          fence_proxy_async_shared();
        }
        named_sync(kChain, kChainThreads);
        if (lo > 0) named_arrive(kToSide, kBothThreads);  // L and Od have been read
        hi = lo;
      }
      // dS = gam_63 dS + Q^T scale gam dO - K^T gam dV
      const float keep = gate.gam[C - 1];
      s.each([&](int, int, float& p, float& q) { p = cuts ? 0.0f : keep * p, q = cuts ? 0.0f : keep * q; });
      StateSum<KD, NV> more;
      if (!(cuts & 1ull)) {
        more.template add<P>(now.Q, sh.Od);
        more.template add<P>(now.K, sh.Z);
      }
      ring.release(k);
      more.add_to(s);
      s.split(sh.S);
      float dot = 0.0f;
#pragma unroll
      for (int c = 0; c < s.kTiles; ++c)
#pragma unroll
        for (int r = 0; r < 4; ++r) dot = cuts & 1ull ? 0.0f : fmaf(s.x[c][r], before.x[c][r], dot);
#pragma unroll
      for (int d = 16; d > 0; d /= 2) dot += __shfl_xor_sync(0xffffffffu, dot, d);
      if ((threadIdx.x & 31) == 0) sh.sums[warp] = dot;
      if (k + 1 < chunks) named_arrive(kToSide, kBothThreads);
      named_sync(kChain, kChainThreads);
      if (threadIdx.x == 0) {
        dot = 0.0f;
#pragma unroll
        for (int w = 0; w < 8; ++w) dot += sh.sums[w];
        a.dots[chunk * a.tiles + blockIdx.x % a.tiles] = dot;
      }
    }
    s.store(a.dh0 + (long long)bh * DD, a, v0);
    for (long long i = (long long)len * NV + threadIdx.x; i < (long long)a.T * NV; i += kChainThreads) {
      const int c = v0 + (int)(i % NV);
      if (c < a.Dv) dv[i / NV * a.dvs.t + c] = from_f32<T>(0.0f);
    }
  } else {
    constexpr int kTiles = NV / 8;
    const int rb = (warp - 8) * 16;
    const T* d_o = static_cast<const T*>(a.d_o) + b * a.dos.b + h * a.dos.h;
    Raw2<T> ox[kTiles][2];
    auto fetch_o = [&](int n) {
#pragma unroll
      for (int c = 0; c < kTiles; ++c)
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          const int time = n * C + rb + g + 8 * r;
          ox[c][r].load(d_o + time * a.dos.t, v0 + c * 8 + 2 * t, a.Dv, a.pairs, n >= 0 && time < len);
        }
    };
    fetch_o(chunks - 1);
    unsigned long long cuts_ahead = cuts_of(a, chunks - 1, chunks, b, h);
    for (int k = 0; k < chunks; ++k) {
      const int n = chunks - 1 - k;
      const bool came = ring.wait_full(k);
      __syncwarp();
      const unsigned long long cuts = cuts_ahead;
      cuts_ahead = cuts_of(a, n - 1, chunks, b, h);
      const St now(smem + k % kN * St::kBytes);
      const Gates& gate = *now.gates;
      float2 on[kTiles][2];
#pragma unroll
      for (int c = 0; c < kTiles; ++c) on[c][0] = ox[c][0].get(), on[c][1] = ox[c][1].get();
      fetch_o(n - 1);
      for (int hi = C; hi > 0;) {
        int lo = 0;
        for (int next = piece_end(cuts, lo); next < hi; next = piece_end(cuts, lo)) lo = next;
#pragma unroll
        for (int c = 0; c < kTiles; ++c)
#pragma unroll
          for (int r = 0; r < 2; ++r) {
            const int i = rb + g + 8 * r;
            const bool in = i >= lo && i < hi;
            sh.O.put(i, c * 8 + 2 * t, in ? on[c][r].x : 0.0f, in ? on[c][r].y : 0.0f);
          }
        named_sync(kSide, kSideThreads);
        float d[kTiles][4] = {}, e[kTiles][4] = {};
        product_lower<3, P, kTiles, true>(d, e, now.M, rb, sh.O, 0);
        if (lo == 0) ring.release(k);  // (the gates below are read before the chain is done with the chunk)
        if (k > 0 || hi < C) named_sync(kToSide, kBothThreads);  // the L and Od before have been read
        else named_sync(kSide, kSideThreads);                    // (O has been read by all, as behind the other barrier)
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          const int i = rb + g + 8 * r;
          const bool in = i >= lo && i < hi;
          const float scale = came ? a.scale : kNaN, gam = in ? scale * gate.gam[i] : 0.0f;
#pragma unroll
          for (int c = 0; c < kTiles; ++c) {
            const int col = c * 8 + 2 * t;
            *reinterpret_cast<float2*>(sh.L + i * Sh::kLPitch + col) =
                make_float2(scale * (d[c][2 * r] + e[c][2 * r]), scale * (d[c][2 * r + 1] + e[c][2 * r + 1]));
            if (lo == 0) sh.Od.put(i, col, in ? gam * on[c][r].x : 0.0f, in ? gam * on[c][r].y : 0.0f);
          }
        }
        named_arrive(kToChain, kBothThreads);
        hi = lo;
      }
    }
  }
}

// ---- per chunk and key head: the gradients of q, k, g and beta ---------------------

// Columns of S to a round: fewer where the parts of 32-bit keys fill the shared memory.
template <typename T, int KD>
constexpr int kSlice = sizeof(T) == 4 && KD == 128 ? 16 : 32;
constexpr int kGradThreads = 512;

template <typename T, int KD>
struct GradShared {
  static constexpr int W = kSlice<T, KD>, P = kParts<T>;
  KeyMat<T, KD> K, Q;
  Gates* gates;
  float* sums;                                // [6][C]
  float *next_S, *next_dS, *next_R, *next_Y;  // the next round's, as they come
  // one round's: S0, dS, dO, R, U; after the last, P and E.  (Two rounds in turn, so that a warp splits one while others multiply the
  // one before, leave the L1 little: 612 us where this took 602, forward and backward of 4 streams of 8 heads and 2048 timesteps.)
  Mat<KD, W, 3> S, dS;
  Mat<C, W, P> dO;
  Mat<C, W, 3> R, U;
  SquareMat Pm, E;
  static constexpr size_t kFixed = kKeysBytes<T, KD> + sizeof(Gates) + 6 * C * 4 + 2 * (KD + C) * W * 4;
  static constexpr size_t kRound = decltype(S)::kBytes + decltype(dS)::kBytes + decltype(dO)::kBytes + decltype(R)::kBytes + decltype(U)::kBytes;
  static constexpr size_t kAfter = decltype(Pm)::kBytes + decltype(E)::kBytes;
  static constexpr size_t kBytes = kFixed + (kRound > kAfter ? kRound : kAfter);
  __device__ __forceinline__ explicit GradShared(unsigned char* p)
      : K{reinterpret_cast<bf16*>(p)}, Q{K.p + K.kSize * P}, gates(reinterpret_cast<Gates*>(Q.p + Q.kSize * P)),
        sums(reinterpret_cast<float*>(gates + 1)), next_S(sums + 6 * C), next_dS(next_S + KD * W), next_R(next_dS + KD * W),
        next_Y(next_R + C * W), S{reinterpret_cast<bf16*>(next_Y + C * W)}, dS{S.p + S.kSize * 3}, dO{dS.p + dS.kSize * 3},
        R{dO.p + dO.kSize * P}, U{R.p + R.kSize * 3}, Pm{S.p}, E{Pm.p + Pm.kSize * 3} {}
};

// [kRows][W] values of a matrix [rows][Dv] from column v0 on, as they come (zeros past its ends).  Each thread asks for the four
// neighbours that it reads itself; `quads`: as one piece of 16 bytes.
template <int kRows, int W, typename F>
__device__ __forceinline__ void each_piece(F f) {  // f(row, column)
#pragma unroll
  for (int i = threadIdx.x; i < kRows * W / 4; i += kGradThreads) f(i / (W / 4), i % (W / 4) * 4);
}
template <int kRows, int W>
__device__ __forceinline__ void fetch_slice(float* to, const float* from, int v0, int rows, int Dv, bool quads) {
  each_piece<kRows, W>([&](int r, int c) {
    const float* at = from + (long long)r * Dv + v0 + c;
    float* into = to + r * W + c;
    if (quads) {
      const bool in = r < rows && v0 + c < Dv;
      copy16(into, in ? at : from, in ? 16 : 0);
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const bool in = r < rows && v0 + c + e < Dv;
        copy4(into + e, in ? at + e : from, in ? 4 : 0);
      }
    }
  });
}

// x += A times the transposed rows n0.. of M (three parts), over kLength columns; two tiles of 8 rows of M at a time, summed apart first
// (an MMA's sum is cut, not rounded, to 24 bits).
template <int kTiles, int kLength, int PA, typename MatM>
__device__ __forceinline__ void add_rows(float (&x)[kTiles][4], const uint32_t (&fa)[kLength / 16][PA][4], const MatM& M, int n0) {
#pragma unroll
  for (int n = 0; n < kTiles; n += 2) {
    float d[2][4] = {}, e[2][4] = {};
#pragma unroll
    for (int k = 0; k < kLength / 16; ++k) {
      uint32_t m[3][2][2];
      load_b<3>(M, n0 + n * 8, k * 16, m);
      mma(d[0], e[0], fa[k], m, 0);
      mma(d[1], e[1], fa[k], m, 1);
    }
#pragma unroll
    for (int z = 0; z < 2; ++z)
#pragma unroll
      for (int r = 0; r < 4; ++r) x[n + z][r] += d[z][r] + e[z][r];
  }
}

// x += a b, of 16 rows of k.
template <int kPA, int kPB>
__device__ __forceinline__ void add_mma(float (&x)[4], const uint32_t (&a)[kPA][4], const uint32_t (&b)[kPB][2][2], int tile) {
  float d[4] = {}, e[4] = {};
  mma(d, e, a, b, tile);
#pragma unroll
  for (int r = 0; r < 4; ++r) x[r] += d[r] + e[r];
}

// By columns of S, 32 at a time: the next ones come as copies while 16 warps multiply.  1024 chunks of bf16, 128 x 128: 251 us, of
// which the products take 90 of the tensor pipes; the rest is splitting, the first slices and barriers (one block fills an SM).  dO
// and R each go through S by themselves: both at once, S read once, spills more registers and takes 10 us longer.
template <typename T, int KD>
__global__ void __launch_bounds__(kGradThreads, 1) delta_gradients_kernel(const DeltaArgs a) {
  extern __shared__ __align__(128) unsigned char smem[];
  constexpr int W = kSlice<T, KD>, P = kParts<T>;
  constexpr int kPart = KD / 4, kTiles = kPart / 8;  // a warp has 16 rows and a quarter of the columns
  using Sh = GradShared<T, KD>;
  const Sh sh(smem);
  const Gates& gate = *sh.gates;
  begin_op();
  const int Hk = a.H / a.share;
  const int hk = (int)(blockIdx.x % Hk), b = (int)(blockIdx.x / Hk % a.B), n = (int)(blockIdx.x / Hk / a.B);
  const int len = length_of(a, b), t0 = n * C, rows = min(len - t0, C), all = min(a.T - t0, C);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane_g(), t = lane_t();
  const int side = warp >> 2, rb = (side & 1 ? 3 - (warp & 3) : warp & 3) * 16;  // (long rows of triangles beside short ones)
  T* dq = static_cast<T*>(a.dq) + t0 * a.dqs.t + b * a.dqs.b + hk * a.dqs.h;
  T* dk = static_cast<T*>(a.dk) + t0 * a.dks.t + b * a.dks.b + hk * a.dks.h;
  for (int i = threadIdx.x + max(rows, 0) * a.Dk; i < all * a.Dk; i += kGradThreads) {  // past the stream's length
    dq[i / a.Dk * a.dqs.t + i % a.Dk] = from_f32<T>(0.0f);
    dk[i / a.Dk * a.dks.t + i % a.Dk] = from_f32<T>(0.0f);
  }
  for (int i = threadIdx.x + max(rows, 0) * a.share; i < all * a.share; i += kGradThreads) {
    const long long row = t0 + i / a.share;
    const int h = hk * a.share + i % a.share;
    a.dg[row * a.dgt + b * a.dgb + h] = 0.0f;
    a.dbeta[row * a.dbt + b * a.dbb + h] = 0.0f;
  }
  if (rows <= 0) return;
  const long long DD = (long long)a.Dk * a.Dv;
  const size_t where = ((size_t)n * a.B + b) * Hk + hk;
  const float2 zero = make_float2(0.0f, 0.0f);

  for (int h = hk * a.share; h < (hk + 1) * a.share; ++h) {
    const long long chunk = ((long long)n * a.B + b) * a.H + h;
    const T* v = static_cast<const T*>(a.v) + t0 * a.vs.t + b * a.vs.b + h * a.vs.h;
    const T* d_o = static_cast<const T*>(a.d_o) + t0 * a.dos.t + b * a.dos.b + h * a.dos.h;
    const float *S = a.states + chunk * (a.Dk + C) * a.Dv, *Y = S + DD, *dS = a.dS + chunk * DD, *R = a.R + chunk * C * a.Dv;
    __syncthreads();
    fetch<(int)sizeof(Gates), kGradThreads>(sh.gates, a.heads + (size_t)chunk * kHeadBytes + LowerMat::kBytes);
    if (h == hk * a.share) fetch<(int)kKeysBytes<T, KD>, kGradThreads>(sh.K.p, a.keys + where * kKeysBytes<T, KD>);
    // (R and Y as copies too: held in registers while a round is multiplied, the forward and backward passes took 636 us, not 611.)
    auto fetch_slices = [&](int v0) {
      fetch_slice<KD, W>(sh.next_S, S, v0, a.Dk, a.Dv, a.quads);
      fetch_slice<KD, W>(sh.next_dS, dS, v0, a.Dk, a.Dv, a.quads);
      fetch_slice<C, W>(sh.next_R, R, v0, rows, a.Dv, a.quads);
      fetch_slice<C, W>(sh.next_Y, Y, v0, rows, a.Dv, a.quads);
      copies_commit();
    };
    fetch_slices(0);
    // The same piece of v and dO as of R and Y.
    const bool mine = threadIdx.x < C * W / 4;
    const int row = threadIdx.x / (W / 4), col = threadIdx.x % (W / 4) * 4;
    Raw2<T> vx[2], ox[2];
    auto fetch_rows = [&](int v0) {
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        vx[x].load(v + row * a.vs.t, v0 + col + 2 * x, a.Dv, a.pairs, mine && row < rows);
        ox[x].load(d_o + row * a.dos.t, v0 + col + 2 * x, a.Dv, a.pairs, mine && row < rows);
      }
    };
    fetch_rows(0);
    copies_wait<0>();
    __syncthreads();
    const unsigned long long cuts = gate.cuts;

    for (int lo = 0; lo < rows;) {
      const int hi = min(piece_end(cuts, lo), rows);
      const bool fresh = cut_before(cuts, lo), last = hi == rows;  // the state before counts as zero; the one behind goes on
      if (cuts) {  // this piece's keys and the first slices anew
        __syncthreads();
        fetch<(int)kKeysBytes<T, KD>, kGradThreads>(sh.K.p, a.keys + where * kKeysBytes<T, KD>);
        fetch_slices(0);
        copies_wait<0>();
        __syncthreads();
        for (int i = threadIdx.x; i < C * KD; i += kGradThreads)
          if (i / KD < lo || i / KD >= hi)
#pragma unroll
            for (int q = 0; q < P; ++q) sh.K.p[q * sh.K.kSize + i] = sh.Q.p[q * sh.Q.kSize + i] = from_f32<bf16>(0.0f);
      }
      float acc_q[kTiles][4] = {}, acc_w[kTiles][4] = {}, acc_t[kTiles][4] = {};  // dO S0^T, R S0^T, U dS^T
      float acc_p[2][4] = {}, acc_e[2][4] = {};                                  // dO U^T, R U^T
      float rv = 0.0f, ry = 0.0f;                                                // R . V, R . Y
      if (lo > 0) fetch_rows(0);

      for (int v0 = 0; v0 < a.Dv; v0 += W) {
        copies_wait<0>();
        __syncthreads();  // nobody reads the round before
        const float4 none = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        each_piece<KD, W>([&](int r, int c) {
          sh.S.put4(r, c, fresh ? none : *reinterpret_cast<const float4*>(sh.next_S + r * W + c));
          sh.dS.put4(r, c, last ? *reinterpret_cast<const float4*>(sh.next_dS + r * W + c) : none);
        });
        if (mine) {
          const bool in = row >= lo && row < hi;
          const float beta = gate.beta[row];
          const float2 va = vx[0].get(), vb = vx[1].get(), oa = ox[0].get(), ob = ox[1].get();
          const float4 rn = in ? *reinterpret_cast<const float4*>(sh.next_R + row * W + col) : none;
          const float4 yn = in ? *reinterpret_cast<const float4*>(sh.next_Y + row * W + col) : none;
          const float4 vn = in ? make_float4(va.x, va.y, vb.x, vb.y) : none;
          rv = fmaf(rn.x, vn.x, fmaf(rn.y, vn.y, fmaf(rn.z, vn.z, fmaf(rn.w, vn.w, rv))));
          ry = fmaf(rn.x, yn.x, fmaf(rn.y, yn.y, fmaf(rn.z, yn.z, fmaf(rn.w, yn.w, ry))));
          sh.R.put4(row, col, rn);
          sh.dO.put4(row, col, in ? make_float4(oa.x, oa.y, ob.x, ob.y) : none);
          sh.U.put4(row, col, in ? make_float4(beta * yn.x, beta * yn.y, beta * yn.z, beta * yn.w) : none);
        }
        __syncthreads();
        if (v0 + W < a.Dv) {
          fetch_slices(v0 + W);
          fetch_rows(v0 + W);
        }
        __syncwarp();
        const bool below = side * 16 <= rb;  // else the warp's part of P and E lies above the diagonal
        {
          uint32_t fa[W / 16][P][4];
#pragma unroll
          for (int k = 0; k < W / 16; ++k) load_a<P>(sh.dO, rb, k * 16, fa[k]);
          if (below) add_rows<2, W>(acc_p, fa, sh.U, side * 16);
          if (!fresh) add_rows<kTiles, W>(acc_q, fa, sh.S, side * kPart);
        }
        {
          uint32_t fa[W / 16][3][4];
#pragma unroll
          for (int k = 0; k < W / 16; ++k) load_a<3>(sh.R, rb, k * 16, fa[k]);
          if (below) add_rows<2, W>(acc_e, fa, sh.U, side * 16);
          if (!fresh) add_rows<kTiles, W>(acc_w, fa, sh.S, side * kPart);
        }
        if (last) {
          uint32_t fa[W / 16][3][4];
#pragma unroll
          for (int k = 0; k < W / 16; ++k) load_a<3>(sh.U, rb, k * 16, fa[k]);
          add_rows<kTiles, W>(acc_t, fa, sh.dS, side * kPart);
        }
      }
      __syncthreads();

#pragma unroll
      for (int r = 0; r < 2; ++r) {
        const int i = rb + g + 8 * r;
        const bool in = i >= lo && i < hi;
        const float beta = gate.beta[i];
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          const int j = side * 16 + x * 8 + 2 * t;
          float p[2], e[2];
#pragma unroll
          for (int y = 0; y < 2; ++y) {
            const float dist = (gate.g_high[i] - gate.g_high[j + y]) + (gate.g_low[i] - gate.g_low[j + y]);
            const bool both = in && i >= j + y && j + y >= lo;
            const float D = both ? expf(dist) : 0.0f;
            p[y] = both ? a.scale * D * acc_p[x][2 * r + y] : 0.0f;
            e[y] = both && i > j + y ? beta * D * acc_e[x][2 * r + y] : 0.0f;
          }
          sh.Pm.put(i, j, p[0], p[1]);
          sh.E.put(i, j, e[0], e[1]);
        }
      }
      __syncthreads();
      // acc_q: diag(scale gam) dO S0^T + P K; acc_t: diag(dec) U dS^T - diag(gam) dV S0^T + P^T Q; acc_w: E K + E^T K
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        const int i = rb + g + 8 * r;
        const float gam = gate.gam[i], dec = gate.dec[i], back = -gate.beta[i] * gam;
#pragma unroll
        for (int x = 0; x < kTiles; ++x)
#pragma unroll
          for (int y = 2 * r; y < 2 * r + 2; ++y) {
            acc_q[x][y] = fresh ? 0.0f : a.scale * gam * acc_q[x][y];
            acc_t[x][y] = (last ? dec * acc_t[x][y] : 0.0f) + (fresh ? 0.0f : back * acc_w[x][y]);
            acc_w[x][y] = 0.0f;
          }
      }
#pragma unroll
      for (int k0 = 0; k0 < C; k0 += 16) {
        if (k0 > rb) continue;
        uint32_t fp[3][4], fe[3][4];
        load_a<3>(sh.Pm, rb, k0, fp);
        load_a<3>(sh.E, rb, k0, fe);
#pragma unroll
        for (int x = 0; x < kTiles; x += 2) {
          uint32_t fb[P][2][2];
          load_bt<P>(sh.K, side * kPart + x * 8, k0, fb);
#pragma unroll
          for (int y = 0; y < 2; ++y) {
            add_mma(acc_q[x + y], fp, fb, y);
            add_mma(acc_w[x + y], fe, fb, y);
          }
        }
      }
#pragma unroll
      for (int k0 = 0; k0 < C; k0 += 16) {
        if (k0 < rb) continue;
        uint32_t fp[3][4], fe[3][4];
        load_at<3>(sh.Pm, rb, k0, fp);
        load_at<3>(sh.E, rb, k0, fe);
#pragma unroll
        for (int x = 0; x < kTiles; x += 2) {
          uint32_t fk[P][2][2], fq[P][2][2];
          load_bt<P>(sh.K, side * kPart + x * 8, k0, fk);
          load_bt<P>(sh.Q, side * kPart + x * 8, k0, fq);
#pragma unroll
          for (int y = 0; y < 2; ++y) {
            add_mma(acc_t[x + y], fp, fq, y);
            add_mma(acc_w[x + y], fe, fk, y);
          }
        }
      }
      float dot_q[2] = {};
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        const int i = rb + g + 8 * r;
        const bool in = i >= lo && i < hi;
        float* sum_q = a.sum_q + (where * C + i) * KD;
        float* sum_k = a.sum_k + (where * C + i) * KD;
#pragma unroll
        for (int x = 0; x < kTiles; ++x) {
          const int c = side * kPart + x * 8 + 2 * t;
          const float2 qx = sh.Q.pair(i, c);
          float gq[2], gk[2];
#pragma unroll
          for (int y = 0; y < 2; ++y) {
            gq[y] = acc_q[x][2 * r + y];
            gk[y] = acc_t[x][2 * r + y] - acc_w[x][2 * r + y];
            dot_q[r] = fmaf(y ? qx.y : qx.x, gq[y], dot_q[r]);
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
      // sums over a row's columns: of neighbouring lanes, and for dot_q of four warps
#pragma unroll
      for (int d = 1; d < W / 4; d *= 2) {
        rv += __shfl_xor_sync(0xffffffffu, rv, d);
        ry += __shfl_xor_sync(0xffffffffu, ry, d);
      }
      if (mine && col == 0) sh.sums[row] = rv, sh.sums[C + row] = ry;
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        dot_q[r] += __shfl_xor_sync(0xffffffffu, dot_q[r], 1);
        dot_q[r] += __shfl_xor_sync(0xffffffffu, dot_q[r], 2);
        if (t == 0) sh.sums[(2 + side) * C + rb + g + 8 * r] = dot_q[r];
      }
      __syncthreads();
      if (warp == 0) {  // dbeta, and dg: what the state before gives, less the rows before (rows lane and lane + 32)
        float start = 0.0f;
        if (!fresh)
          for (int i = 0; i < a.tiles; ++i) start += a.dots[chunk * a.tiles + i];
        float G[2], own[2];
#pragma unroll
        for (int s = 0; s < 2; ++s) {
          const int row = lane + 32 * s;
          const bool in = row >= lo && row < hi;
          const float* x = sh.sums + 2 * C + row;
          own[s] = in ? ((x[0] + x[C]) + (x[2 * C] + x[3 * C])) - gate.beta[row] * sh.sums[row] : 0.0f;
          if (in) a.dbeta[(long long)(t0 + row) * a.dbt + b * a.dbb + h] = sh.sums[C + row];
          float sum = own[s];
#pragma unroll
          for (int d = 1; d < 32; d *= 2) {
            const float y = __shfl_up_sync(0xffffffffu, sum, d);
            if (lane >= d) sum += y;
          }
          G[s] = sum;
        }
        G[1] += __shfl_sync(0xffffffffu, G[0], 31);
#pragma unroll
        for (int s = 0; s < 2; ++s) {
          const int row = lane + 32 * s;
          if (row < lo || row >= hi) continue;
          const float g_in = a.g[(long long)(t0 + row) * a.gt + b * a.gb + h];
          const bool none = (cuts >> row & 1ull) || g_in < kLeastG;  // a decay that nothing passes through
          a.dg[(long long)(t0 + row) * a.dgt + b * a.dgb + h] = none ? 0.0f : start - (G[s] - own[s]);
        }
      }
      lo = hi;
    }
  }
}

// ---- host ----------------------------------------------------------------------

// For tests: how long a copy is waited for, and a chunk that the next call does not copy.
std::atomic<int> g_wait_us{kWaitUs}, g_withheld{-1};

struct Workspace {
  size_t keys, heads, dS, R, dots, sum_q, sum_k, bytes;
};
Workspace workspace_of(size_t es, bool exact, long long T, long long B, long long H, long long Hk, long long Dk, long long Dv, bool backward) {
  const size_t chunks = (size_t)((T + C - 1) / C) * B, KD = Dk <= 64 ? 64 : 128;
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t from = at;
    at += (bytes + 255) / 256 * 256;
    return from;
  };
  Workspace w{};
  w.keys = take(chunks * Hk * 2 * C * KD * 2 * (es == 4 ? 3 : exact ? 1 : 2));
  w.heads = take(chunks * H * kHeadBytes);
  if (backward) {
    w.dS = take(chunks * H * Dk * Dv * 4);
    w.R = take(chunks * H * C * Dv * 4);
    w.dots = take(chunks * H * ((Dv + 15) / 16) * 4);
    if (H > Hk) {
      w.sum_q = take(chunks * Hk * C * KD * 4);
      w.sum_k = take(chunks * Hk * C * KD * 4);
    }
  }
  w.bytes = at + 256;
  return w;
}

// Columns of S to a block: 16 while that fits the device in one wave, and for 32-bit keys, whose parts fill the shared memory.  A
// block of 32 takes less than two of 16: 2048 timesteps in bf16, 128 x 128 states, forward alone: 19 heads 113 us by 16; 20 heads 168
// us by 32 and 202 by 16, 38 heads 186 and 221; 39 heads, where those of 32 take a second wave and those of 16 a third, 319 and 310.
int columns_of(long long heads, int Dv, size_t es) {
  return heads * ((Dv + 15) / 16) <= 152 || es == 4 ? 16 : 32;
}

template <auto kKern>
cudaError_t launch_big(dim3 grid, size_t smem, cudaStream_t s, const DeltaArgs& a, int threads = kThreads) {
  static thread_local DeviceSet ready;  // of this kernel
  const cudaError_t e =
      once_per_device(&ready, [&] { return cudaFuncSetAttribute(kKern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem); });
  return e != cudaSuccess ? e : op_launch(kKern, grid, dim3(threads), smem, s, a);
}

template <typename F>
cudaError_t for_shape(int dtype, int Dk, F f) {
  return op_for_type(dtype, [&](auto* t) {
    if (Dk <= 64) return f(t, std::integral_constant<int, 64>());
    return f(t, std::integral_constant<int, 128>());
  });
}

cudaError_t prepare(int dtype, const DeltaArgs& a, cudaStream_t s) {
  const long long blocks = (long long)((a.T + C - 1) / C) * a.B * (a.H / a.share);
  if (blocks == 0) return cudaSuccess;
  return for_shape(dtype, a.Dk, [&](auto* t, auto kd) {
    using T = std::remove_pointer_t<decltype(t)>;
    constexpr int KD = decltype(kd)::value;
    return launch_big<delta_prepare_kernel<T, KD>>(dim3((unsigned)blocks), PrepareShared<T, KD>::kBytes, s, a);
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

extern "C" int lstm_approx_delta_scan_set_waits(int limit_us, int withheld) {
  if (limit_us < 0 || withheld < -1) return LSTM_APPROX_EINVAL;
  g_wait_us = limit_us ? limit_us : kWaitUs;
  g_withheld = withheld;
  return LSTM_APPROX_OK;
}

extern "C" size_t lstm_approx_delta_scan_workspace_bytes(int dtype, int T, int B, int H, int Hk, int Dk, int Dv, int backward) {
  if (check(dtype, nullptr, nullptr, nullptr, nullptr, nullptr, 0, B, H, Hk, Dk, Dv, nullptr, 0, nullptr, 0) || T < 0 ||
      (long long)((T + 63ll) / 64) * B > 0x7fffffffll / H)
    return 0;
  return workspace_of(op_dtype_bytes(dtype), dtype == LSTM_APPROX_OP_BF16, T, B, H, Hk, Dk, Dv, backward != 0).bytes;
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
  const Workspace w = workspace_of(es, dtype == LSTM_APPROX_OP_BF16, T, B, H, Hk, Dk, Dv, false);
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
  a.even = Dv % 2 == 0 && op_aligned(h0, 8) && op_aligned(h_last, 8) && op_aligned(states, 8);
  a.h_last = h_last, a.states = states;
  a.wait_ns = 1000ull * (uint64_t)g_wait_us.load(), a.withheld = g_withheld.exchange(-1);
  char* ws = reinterpret_cast<char*>((reinterpret_cast<uintptr_t>(workspace) + 255) / 256 * 256);
  a.keys = reinterpret_cast<unsigned char*>(ws + w.keys), a.heads = reinterpret_cast<unsigned char*>(ws + w.heads);
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  if (int rc = op_launched(prepare(dtype, a, s), "delta scan launch", msg, msg_len)) return rc;
  const int NV = columns_of((long long)B * H, Dv, es);
  a.tiles = (Dv + NV - 1) / NV;
  const dim3 grid((unsigned)(B * H * a.tiles));
  const cudaError_t e = for_shape(dtype, Dk, [&](auto* t, auto kd) {
    using Ty = std::remove_pointer_t<decltype(t)>;
    constexpr int KD = decltype(kd)::value;
    if constexpr (sizeof(Ty) == 2)
      if (NV == 32) return launch_big<delta_forward_kernel<Ty, KD, 32>>(grid, ForwardShared<Ty, KD, 32>::kBytes, s, a, kAllThreads);
    return launch_big<delta_forward_kernel<Ty, KD, 16>>(grid, ForwardShared<Ty, KD, 16>::kBytes, s, a, kAllThreads);
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
  const Workspace w = workspace_of(es, dtype == LSTM_APPROX_OP_BF16, T, B, H, Hk, Dk, Dv, true);
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
  a.even = Dv % 2 == 0 && op_aligned(states, 8) && op_aligned(dh_last, 8) && op_aligned(dh0, 8);
  a.quads = Dv % 4 == 0 && op_aligned(states, 16);
  a.states = const_cast<float*>(states), a.dh_last = dh_last;
  a.dq = dq, a.dk = dk, a.dv = dv, a.dg = dg, a.dbeta = dbeta, a.dh0 = dh0;
  a.wait_ns = 1000ull * (uint64_t)g_wait_us.load(), a.withheld = g_withheld.exchange(-1);
  char* ws = reinterpret_cast<char*>((reinterpret_cast<uintptr_t>(workspace) + 255) / 256 * 256);
  a.keys = reinterpret_cast<unsigned char*>(ws + w.keys), a.heads = reinterpret_cast<unsigned char*>(ws + w.heads);
  a.dS = reinterpret_cast<float*>(ws + w.dS), a.R = reinterpret_cast<float*>(ws + w.R);
  a.dots = reinterpret_cast<float*>(ws + w.dots);
  a.sum_q = reinterpret_cast<float*>(ws + w.sum_q), a.sum_k = reinterpret_cast<float*>(ws + w.sum_k);
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  if (int rc = op_launched(prepare(dtype, a, s), "delta scan launch", msg, msg_len)) return rc;
  const int NV = columns_of((long long)B * H, Dv, es);
  a.tiles = (Dv + NV - 1) / NV;
  const dim3 grid((unsigned)(B * H * a.tiles));
  cudaError_t e = for_shape(dtype, Dk, [&](auto* t, auto kd) {
    using Ty = std::remove_pointer_t<decltype(t)>;
    constexpr int KD = decltype(kd)::value;
    if constexpr (sizeof(Ty) == 2)
      if (NV == 32) return launch_big<delta_backward_kernel<Ty, KD, 32>>(grid, BackwardShared<Ty, KD, 32>::kBytes, s, a, kAllThreads);
    return launch_big<delta_backward_kernel<Ty, KD, 16>>(grid, BackwardShared<Ty, KD, 16>::kBytes, s, a, kAllThreads);
  });
  if (int rc = op_launched(e, "delta scan backward launch", msg, msg_len)) return rc;
  if (T == 0) return LSTM_APPROX_OK;
  const dim3 blocks((unsigned)((T + C - 1) / C * B * Hk));
  e = for_shape(dtype, Dk, [&](auto* t, auto kd) {
    using Ty = std::remove_pointer_t<decltype(t)>;
    constexpr int KD = decltype(kd)::value;
    return launch_big<delta_gradients_kernel<Ty, KD>>(blocks, GradShared<Ty, KD>::kBytes, s, a, kGradThreads);
  });
  return op_launched(e, "delta gradients launch", msg, msg_len);
}
