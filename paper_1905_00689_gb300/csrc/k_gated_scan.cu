// The gated linear recurrence over a sequence, its gradients, and one
// timestep of it on a pool of states (include/lstm_approx_ops.h):
//
//   log a_t = -c softplus(decay) sigma(r_t),   m_t = sqrt(1 - a_t^2)
//   h_t = k_t a_t h_{t-1} + m_t sigma(i_t) x_t        (k_t = 0 at a reset)
//
// Over a run of timesteps the state before it and the one after it are joined
// by h -> A h + U, where A is the product of the a_t and U the state that a
// zero start leads to; two runs join to (A2 A1, A2 U1 + U2).  A block owns 64
// channels of one stream and takes the sequence in tiles of 64 timesteps: each
// of its 8 warps forms (A, U) of 8 timesteps, two channels to a lane, the
// block joins them in their order (so the result does not depend on timing),
// and each warp goes over its 8 timesteps once more from the state it starts
// with.  a_t and m_t sigma(i_t) x_t are computed once and stay in registers.
//
// Few streams over few channels leave most of the GPU idle in that form, so the
// blocks of a cluster of up to 16 share a stream's 64 channels: block k of n
// takes tiles k, n + k, ..., writes its tile's (A, U) into every block's shared
// memory, and after one cluster barrier per n tiles each block joins all of
// them in order.  That keeps the sequence at one pass over memory in one
// launch, with no flags in memory and no waits but the barrier.
//
// Backward, with p_t = k_t a_t g_t the gradient of h_{t-1}:
//   g_t = dy_t + p_{t+1}  (p after the last timestep: dh_last; before the first: dh0)
//   dx = g m si,  di = g m x si (1 - si)                       (si = sigma(i))
//   E_t = g (k a la h_{t-1} + si x a^2 q),  q = -la / m          (la = log a)
//   dr = E (1 - sigma(r)),  ddecay = sigma(decay) / softplus(decay) sum E
// E is dL/d(la) la.  It is formed in this way because d m / d la = -a^2 / m
// has no bound as la -> 0, where every gradient has the limit 0 (q ~ sqrt(-la/2)).
// The run of p is joined the same way from the end (p -> A p + V).
//
// Timesteps past a stream's length are the identity in both directions; they
// and the state before a reset are left out by selection, never by a product
// with zero, so what they hold (NaN, infinities) reaches nothing.
#include <algorithm>

#include "ops_common.cuh"
#include "ptx.cuh"

namespace lstm_approx_impl {
namespace {

using namespace lstm_approx_dev;

constexpr int kWarps = 8;
constexpr int kSteps = 8;                 // timesteps of a warp in a tile
constexpr int kTile = kWarps * kSteps;    // timesteps of a tile
constexpr int kLanes = 64;                // channels of a block: two to a lane
static_assert(kTile == LSTM_APPROX_SCAN_CHUNK, "one saved state per tile");

// softplus(d) = log(1 + e^d) and sigma(d) / softplus(d), both to fp32 accuracy
// over the whole range (the ratio tends to 1 for d -> -inf).
__device__ __forceinline__ float softplus_f(float d) { return d > 20.0f ? d : log1pf(expf(d)); }
__device__ __forceinline__ float softplus_ratio_f(float d) {
  const float e = expf(-fabsf(d));
  const float sig = d >= 0.0f ? 1.0f / (1.0f + e) : e / (1.0f + e);
  const float sp = softplus_f(d);
  return sp > 0.0f ? sig / sp : 1.0f;
}

__device__ __forceinline__ float rsqrt_approx(float x) {
  float r;
  asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
__device__ __forceinline__ float sqrt_approx(float x) {
  float r;
  asm("sqrt.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
__device__ __forceinline__ uint64_t both(float v) { return f32x2(v, v); }
__device__ __forceinline__ uint64_t sub2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("sub.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
// The constants of the loops below, kept in registers: an instruction on two
// values takes no immediate, and left to itself the compiler forms the pairs
// anew at every use (a third of all instructions).
struct Constants {
  uint64_t one, minus_log2e, c1, c2, c3, c4;
};
__device__ __forceinline__ uint64_t held(float v) {
  uint64_t r;
  asm volatile("mov.b64 %0, {%1, %1};" : "=l"(r) : "f"(v));
  return r;
}
__device__ __forceinline__ Constants constants() {
  return {held(1.0f), held(-kLog2E), held(-0.5f), held(1.0f / 6.0f), held(-1.0f / 24.0f), held(1.0f / 120.0f)};
}
__device__ __forceinline__ uint64_t sigmoid2(uint64_t z, const Constants& k) {
  float a, b;
  f32x2_split(mul2(z, k.minus_log2e), a, b);
  f32x2_split(add2(f32x2(ex2_approx(a), ex2_approx(b)), k.one), a, b);
  return f32x2(rcp_approx(a), rcp_approx(b));
}

// The gates of a lane's two channels (pairs of fp32, two per instruction where
// there is one for two): sigma(r), sigma(i) and 1 - a, from which a and m
// follow.  rate = c softplus(decay), the largest -log a; far: it is above 1/8.
//
// 1 - a = 1 - e^-t by its Taylor series: no cancellation, a = 1 - (1 - a)
// comes out correctly rounded, which matters where a state decays over hundreds
// of timesteps, and 1 - a^2 = (1 - a)(1 + a) keeps its digits.  Up to t = 1/8
// (decays down to 0.88 where the gate is open) five terms do (the sixth is
// below 4.3e-8 of the first); beyond, eight up to t = 0.35 (the ninth is below
// 7e-10), and the exponential itself above that.
struct Gates {
  uint64_t sr, si, low;
};
template <bool kFar>
__device__ __forceinline__ Gates gates_of(uint64_t r, uint64_t i, uint64_t rate, const Constants& k) {
  Gates g;
  g.sr = sigmoid2(r, k);
  g.si = sigmoid2(i, k);
  const uint64_t t = mul2(rate, g.sr);
  uint64_t p = k.c4;
  if constexpr (kFar) {
    p = both(-1.0f / 40320.0f);
    p = fma2(p, t, both(1.0f / 5040.0f));
    p = fma2(p, t, both(-1.0f / 720.0f));
    p = fma2(p, t, k.c4);
  }
  p = fma2(p, t, k.c3);
  p = fma2(p, t, k.c2);
  p = fma2(p, t, k.c1);
  p = fma2(p, t, k.one);
  g.low = mul2(t, p);
  if constexpr (kFar) {
    float t0, t1, l0, l1;
    f32x2_split(t, t0, t1);
    f32x2_split(g.low, l0, l1);
    if (t0 > 0.35f) l0 = 1.0f - ex2_approx(-t0 * kLog2E);
    if (t1 > 0.35f) l1 = 1.0f - ex2_approx(-t1 * kLog2E);
    g.low = f32x2(l0, l1);
  }
  return g;
}
__device__ __forceinline__ uint64_t decay_of(uint64_t low, const Constants& k) { return sub2(k.one, low); }
// 1 - a^2
__device__ __forceinline__ uint64_t m2_of(uint64_t low, uint64_t a, const Constants& k) {
  return mul2(low, add2(a, k.one));
}
__device__ __forceinline__ uint64_t sqrt2(uint64_t v) {
  float a, b;
  f32x2_split(v, a, b);
  return f32x2(sqrt_approx(a), sqrt_approx(b));
}
// 1 / sqrt(v), at most 2^63
__device__ __forceinline__ uint64_t rsqrt2(uint64_t v) {
  float a, b;
  f32x2_split(add2(v, both(1.17549435e-38f)), a, b);
  return f32x2(rsqrt_approx(a), rsqrt_approx(b));
}

// The pair of channels (ch, ch + 1) at p; kVec: both exist and lie in one
// aligned access.
template <typename T, bool kVec>
__device__ __forceinline__ float2 load_pair(const T* p, int left) {
  if constexpr (kVec) return Pair<T>::get(*reinterpret_cast<const typename Pair<T>::Raw*>(p));
  return make_float2(left > 0 ? to_f32<T>(p[0]) : 0.0f, left > 1 ? to_f32<T>(p[1]) : 0.0f);
}
template <typename T, bool kVec>
__device__ __forceinline__ void store_pair(T* p, int left, float a, float b) {
  if constexpr (kVec) {
    *reinterpret_cast<typename Pair<T>::Raw*>(p) = Pair<T>::put(a, b);
  } else {
    if (left > 0) p[0] = from_f32<T>(a);
    if (left > 1) p[1] = from_f32<T>(b);
  }
}

// A lane's two channels of one staged timestep.
template <typename T>
__device__ __forceinline__ uint64_t staged_pair(const T* p) {
  if constexpr (sizeof(T) == 4) {
    return *reinterpret_cast<const uint64_t*>(p);
  } else {
    const float2 f = Pair<T>::get(*reinterpret_cast<const typename Pair<T>::Raw*>(p));
    return f32x2(f.x, f.y);
  }
}

struct Strides {
  long long t, b;
};

// How a tile comes into shared memory: by asynchronous copies of kCopy bytes
// where every address is a multiple of it (16: everything aligned, D a multiple
// of 8; 4: an even D, or 32-bit values), else value by value (2).
//
// A warp stages its own 8 timesteps of a tile, [kSteps][64] for each tensor,
// and reads nothing else, so its copies need no barrier of the block.
// Timesteps past `len` and channels past D come out as zeros, nothing of
// theirs is read.
template <typename T, int kCopy>
__device__ __forceinline__ void stage(T* dst, const T* src, long long stride, int ts, int len, int ch0, int D) {
  const int lane = threadIdx.x & 31;
  if constexpr (kCopy >= 4) {
    constexpr int kPer = kCopy / (int)sizeof(T);          // values of a copy
    constexpr int kRow = kLanes / kPer;                   // copies of a row
    constexpr int kRows = kRow >= 32 ? 1 : 32 / kRow;     // rows of one turn of the warp
    constexpr int kTurns = kRow >= 32 ? kRow / 32 : 1;    // turns of one row
    const int row0 = kRow >= 32 ? 0 : lane / kRow;
    auto copy = [&](uint32_t to, const T* from, int bytes) {
      if constexpr (kCopy == 16)
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(bytes) : "memory");
      else
        asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(to), "l"(from), "r"(bytes) : "memory");
    };
    const T* from = src + (ts + row0) * stride + lane % kRow * kPer;
    const uint32_t to = smem_u32(dst + row0 * kLanes + lane % kRow * kPer);
    if (ts + kSteps <= len && ch0 + kLanes <= D) {
#pragma unroll
      for (int s = 0; s < kSteps; s += kRows, from += kRows * stride) {
#pragma unroll
        for (int q = 0; q < kTurns; ++q)
          copy(to + (s * kLanes + 32 * q * kPer) * (int)sizeof(T), from + 32 * q * kPer, kCopy);
      }
    } else {
#pragma unroll 1
      for (int s = 0; s < kSteps; s += kRows, from += kRows * stride) {
#pragma unroll
        for (int q = 0; q < kTurns; ++q) {
          const bool in = ts + s + row0 < len && ch0 + (lane % kRow + 32 * q) * kPer < D;
          copy(to + (s * kLanes + 32 * q * kPer) * (int)sizeof(T), in ? from + 32 * q * kPer : src, in ? kCopy : 0);
        }
      }
    }
  } else {
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        const int col = lane + 32 * q;
        dst[s * kLanes + col] = ts + s < len && ch0 + col < D ? src[(ts + s) * stride + col] : from_f32<T>(0.0f);
      }
    }
  }
}
__device__ __forceinline__ void stage_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void stage_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
  __syncwarp();
}

struct ScanArgs {
  const void *x, *r, *i;
  void* y;
  Strides sx, sr, si, sy;
  const float* decay;
  float c;
  const float* h0;
  const int* lengths;
  const unsigned char* reset;
  int T, B, D, slabs, cluster;
  float* h_last;
  float* states;
};

__device__ __forceinline__ int length_of(const int* lengths, int b, int T) {
  return lengths ? min(max(lengths[b], 0), T) : T;
}

// Bit s: reset at timestep ts + s of this warp (the same in all lanes).
__device__ __forceinline__ unsigned reset_bits(const unsigned char* reset, int ts, int len, int b, int B) {
  const int lane = threadIdx.x & 31, t = ts + lane;
  const bool on = lane < kSteps && t < len && reset[(long long)t * B + b] != 0;
  return __ballot_sync(0xffffffffu, on);
}

constexpr int kMaxCluster = 16;

// Runs of several timesteps, of the warps of a tile or the tiles of a
// cluster's blocks: state after run k = cut[k] ? U : A h + U.
struct Runs {
  ulonglong2* AU;  // [runs][32]: A and U of a lane's two channels
  unsigned* cut;   // [runs]
};
struct WarpRuns {
  ulonglong2 AU[kWarps][32];
  unsigned cut[kWarps];
};
__device__ __forceinline__ Runs runs_of(WarpRuns& w) { return {&w.AU[0][0], w.cut}; }

// h after run k; kCuts: some run may have a reset.
template <bool kCuts>
__device__ __forceinline__ uint64_t after(const Runs& r, int k, uint64_t h) {
  const ulonglong2 v = r.AU[k * 32 + (threadIdx.x & 31)];
  if (kCuts && r.cut[k] != 0) h = 0ull;
  return fma2(v.x, h, v.y);
}

// The exchange buffer of parity `turn` behind the staged tiles: a run for each block of the cluster.
__device__ __forceinline__ Runs tile_runs(unsigned char* base, int cluster, int turn) {
  ulonglong2* AU = reinterpret_cast<ulonglong2*>(base);
  unsigned* cut = reinterpret_cast<unsigned*>(AU + 2 * cluster * 32);
  return {AU + turn * cluster * 32, cut + turn * cluster};
}
__host__ __device__ constexpr size_t exchange_bytes(int cluster) {
  return cluster > 1 ? (size_t)2 * cluster * (32 * sizeof(ulonglong2) + sizeof(unsigned)) : 0;
}

// Writes this block's tile run into slot `rank` of `mine` in every block of the
// cluster, one block to a warp (the blocks past the eighth in a second turn).
__device__ __forceinline__ void send_run(const Runs& mine, int rank, int size, ulonglong2 run, bool cut) {
  const int lane = threadIdx.x & 31;
  for (int to = threadIdx.x >> 5; to < size; to += kWarps) {
    const uint32_t at = mapa_shared(smem_u32(mine.AU + rank * 32 + lane), to);
    asm volatile("st.shared::cluster.v2.u64 [%0], {%1, %2};" ::"r"(at), "l"(run.x), "l"(run.y) : "memory");
    if (lane == 0) {
      const uint32_t c = mapa_shared(smem_u32(mine.cut + rank), to);
      asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(c), "r"((unsigned)cut) : "memory");
    }
  }
}

// Tiles in flight or in use at once, of kTensors tensors: as many as let two
// blocks share an SM's shared memory (32-bit values backward, and forward in a
// cluster of 16: one block).
template <typename T, int kTensors>
constexpr int kStages = 2;
template <typename T, int kTensors>
constexpr size_t kStageBytes = (size_t)kTensors * kTile * kLanes * sizeof(T);

__device__ __forceinline__ uint64_t load_f32x2(const float* p, int left) {
  return f32x2(left > 0 ? p[0] : 0.0f, left > 1 ? p[1] : 0.0f);
}
__device__ __forceinline__ void store_f32x2(float* p, int left, uint64_t v) {
  float a, b;
  f32x2_split(v, a, b);
  if (left > 0) p[0] = a;
  if (left > 1) p[1] = b;
}

template <typename T, bool kVec>
__device__ __forceinline__ void store_both(T* p, int left, uint64_t v) {
  float a, b;
  f32x2_split(v, a, b);
  store_pair<T, kVec>(p, left, a, b);
}

// a_t and m_t sigma(i_t) x_t of a warp's staged timesteps.
template <typename T, bool kFar>
__device__ __forceinline__ void form_runs(const T* here, uint64_t rate, const Constants& k, uint64_t (&A)[kSteps],
                                          uint64_t (&U)[kSteps]) {
#pragma unroll
  for (int s = 0; s < kSteps; ++s) {
    const T* p = here + s * kLanes;
    const Gates g =
        gates_of<kFar>(staged_pair<T>(p + kTile * kLanes), staged_pair<T>(p + 2 * kTile * kLanes), rate, k);
    A[s] = decay_of(g.low, k);
    U[s] = mul2(mul2(sqrt2(m2_of(g.low, A[s], k)), g.si), staged_pair<T>(p));
  }
}

// The run of a warp's timesteps (kCuts: with resets at the set bits).
template <bool kCuts>
__device__ __forceinline__ ulonglong2 join_steps(const uint64_t (&A)[kSteps], const uint64_t (&U)[kSteps], unsigned resets,
                                                 const Constants& k) {
  uint64_t PA = k.one, PU = 0ull;
#pragma unroll
  for (int s = 0; s < kSteps; ++s) {
    if (kCuts && (resets >> s & 1u)) PU = 0ull;
    PU = fma2(A[s], PU, U[s]);
    PA = mul2(PA, A[s]);
  }
  return make_ulonglong2(PA, PU);
}

// c softplus(decay) of a lane's channels, zero for one that does not exist.
__device__ __forceinline__ uint64_t rate_of(const float* decay, int left, float c) {
  return f32x2(left > 0 ? c * softplus_f(decay[0]) : 0.0f, left > 1 ? c * softplus_f(decay[1]) : 0.0f);
}
// Whether -log a of some lane may be above 1/8.
__device__ __forceinline__ bool any_far(uint64_t rate) {
  float r0, r1;
  f32x2_split(rate, r0, r1);
  return __any_sync(0xffffffffu, !(r0 <= 0.125f && r1 <= 0.125f));
}

template <typename T, int kCopy, bool kCuts>
__global__ void __launch_bounds__(kWarps * 32, sizeof(T) == 4 ? 2 : 3) gated_scan_kernel(const ScanArgs a) {
  extern __shared__ __align__(16) unsigned char staged[];
  __shared__ WarpRuns runs[2];
  constexpr int kN = kStages<T, 3>;
  unsigned char* exchange = staged + kN * kStageBytes<T, 3>;
  constexpr bool kVec = kCopy >= 2 * (int)sizeof(T);  // a lane's two channels of y in one store
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rank = blockIdx.x % a.cluster, item = blockIdx.x / a.cluster;
  const int slab = item % a.slabs, b = item / a.slabs;
  const int ch0 = slab * kLanes, ch = ch0 + 2 * lane, left = a.D - ch;  // channels of this lane that exist: min(left, 2)
  const int len = length_of(a.lengths, b, a.T);
  const T* x = static_cast<const T*>(a.x) + b * a.sx.b + ch0;
  const T* r = static_cast<const T*>(a.r) + b * a.sr.b + ch0;
  const T* in = static_cast<const T*>(a.i) + b * a.si.b + ch0;
  T* y = static_cast<T*>(a.y) + b * a.sy.b + ch;
  const long long state_at = (long long)b * a.D + ch;
  const int stride = a.cluster * kTile;
  auto buffer = [&](int n) { return reinterpret_cast<T*>(staged + n * kStageBytes<T, 3>) + warp * kSteps * kLanes; };
  auto fetch = [&](int n, int first) {  // this warp's part of the tile that starts at `first` + rank tiles, if there is one
    T* to = buffer(n);
    const int ts = first + rank * kTile + warp * kSteps;
    if (ts < len) {
      stage<T, kCopy>(to, x, a.sx.t, ts, len, ch0, a.D);
      stage<T, kCopy>(to + kTile * kLanes, r, a.sr.t, ts, len, ch0, a.D);
      stage<T, kCopy>(to + 2 * kTile * kLanes, in, a.si.t, ts, len, ch0, a.D);
    }
    stage_commit();
  };
#pragma unroll
  for (int n = 0; n < kN - 1; ++n) fetch(n, n * stride);
  const uint64_t rate = rate_of(a.decay + ch, left, a.c);
  const bool far = any_far(rate);
  const Constants k = constants();
  uint64_t h = a.h0 ? load_f32x2(a.h0 + state_at, left) : 0ull;
  // shared memory of another block is written only after that block has started
  if (a.cluster > 1) cluster_sync_all();
  int turn = 0, at = 0, next = kN - 1;  // parity of the exchange buffers; stage in use, stage to fill
  // every block of the cluster makes the same number of turns (they meet in the barrier)
  for (int first = 0; first < a.T; first += stride, turn ^= 1) {
    const int t0 = first + rank * kTile, ts = t0 + warp * kSteps;
    const unsigned resets = kCuts ? reset_bits(a.reset, ts, len, b, a.B) : 0u;
    const T* here = buffer(at) + 2 * lane;
    stage_wait<kN - 2>();
    fetch(next, first + (kN - 1) * stride);  // into the stage that the last turn read
    at = at + 1 == kN ? 0 : at + 1;
    next = next + 1 == kN ? 0 : next + 1;
    uint64_t A[kSteps], U[kSteps];
    const bool whole = ts + kSteps <= len;  // and `some` of its timesteps are the stream's
    const bool some = ts < len;
    if (some) {
      if (far) form_runs<T, true>(here, rate, k, A, U);
      else form_runs<T, false>(here, rate, k, A, U);
    }
    if (!whole) {
#pragma unroll
      for (int s = 0; s < kSteps; ++s)
        if (ts + s >= len) A[s] = k.one, U[s] = 0ull;
    }
    const ulonglong2 PR = resets ? join_steps<true>(A, U, resets, k) : join_steps<false>(A, U, 0u, k);
    runs[turn].AU[warp][lane] = PR;  // the other parity's may still be read
    if (lane == 0) runs[turn].cut[warp] = resets;
    __syncthreads();
    const Runs run = runs_of(runs[turn]), tiles = tile_runs(exchange, a.cluster, turn);
    if (a.cluster > 1) {
      ulonglong2 all = make_ulonglong2(k.one, 0ull);
      bool cut = false;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) {
        all.x = mul2(all.x, run.AU[w * 32 + lane].x);
        all.y = after<kCuts>(run, w, all.y);
        cut = cut || run.cut[w] != 0;
      }
      send_run(tiles, rank, a.cluster, all, cut);
      cluster_sync_all();
    }
    uint64_t hs = h;  // the state before this block's tile, then before this warp's timesteps
    if (a.cluster > 1) {
      for (int n = 0; n < a.cluster; ++n) {
        if (n == rank) hs = h;
        h = after<kCuts>(tiles, n, h);
      }
    }
    if (a.states && warp == 0 && t0 < a.T)
      store_f32x2(a.states + (long long)(t0 / kTile) * a.B * a.D + state_at, left, hs);
    if (a.cluster > 1) {
      for (int w = 0; w < warp; ++w) hs = after<kCuts>(run, w, hs);
    } else {
#pragma unroll
      for (int w = 0; w < kWarps; ++w) {
        if (w == warp) hs = h;
        h = after<kCuts>(run, w, h);
      }
    }
    if (resets) {
#pragma unroll
      for (int s = 0; s < kSteps; ++s) {
        if (resets >> s & 1u) hs = 0ull;
        hs = U[s] = fma2(A[s], hs, U[s]);
      }
    } else {
#pragma unroll
      for (int s = 0; s < kSteps; ++s) hs = U[s] = fma2(A[s], hs, U[s]);
    }
    if (left > 0) {
      T* to = y + ts * a.sy.t;
      if (whole) {
#pragma unroll
        for (int s = 0; s < kSteps; ++s, to += a.sy.t) store_both<T, kVec>(to, left, U[s]);
      } else {
#pragma unroll
        for (int s = 0; s < kSteps; ++s, to += a.sy.t)
          if (ts + s < a.T) store_both<T, kVec>(to, left, ts + s < len ? U[s] : 0ull);
      }
    }
  }
  if (warp == 0 && rank == 0) store_f32x2(a.h_last + state_at, left, h);
  // no block leaves while another may still write into its shared memory
  if (a.cluster > 1) cluster_sync_all();
}

struct ScanBackwardArgs {
  const void *dy, *x, *r, *i;
  void *dx, *dr, *di;
  Strides sdy, sx, sr, si, sdx, sdr, sdi;
  const float* dh_last;
  const float* decay;
  float c;
  const float* states;
  const int* lengths;
  const unsigned char* reset;
  int T, B, D, slabs, cluster;
  float* dh0;
  float* partial;  // [B][cluster][D]: each block's sum of E over its timesteps
};

// 1 - a_t, the gates and m_t sigma(i_t) x_t of a warp's staged timesteps.
template <typename T, bool kFar>
__device__ __forceinline__ void form_gates(const T* here, uint64_t rate, const Constants& k, uint64_t (&low)[kSteps],
                                           uint64_t (&sr)[kSteps], uint64_t (&si)[kSteps], uint64_t (&U)[kSteps]) {
#pragma unroll
  for (int s = 0; s < kSteps; ++s) {
    const T* p = here + s * kLanes;
    const Gates g =
        gates_of<kFar>(staged_pair<T>(p + kTile * kLanes), staged_pair<T>(p + 2 * kTile * kLanes), rate, k);
    low[s] = g.low;
    sr[s] = g.sr;
    si[s] = g.si;
    U[s] = mul2(mul2(sqrt2(m2_of(g.low, decay_of(g.low, k), k)), g.si), staged_pair<T>(p));
  }
}

// The runs of a warp's timesteps, h -> A h + U forward and p -> A p + V back
// (staged dy is zero past the stream's length).
template <typename T, bool kCuts>
__device__ __forceinline__ void join_both(const T* here, const uint64_t (&low)[kSteps], const uint64_t (&U)[kSteps],
                                          unsigned resets, const Constants& k, uint64_t& PA, uint64_t& PU, uint64_t& PV) {
#pragma unroll
  for (int s = 0; s < kSteps; ++s) {
    const uint64_t A = decay_of(low[s], k);
    if (kCuts && (resets >> s & 1u)) PU = 0ull;
    PU = fma2(A, PU, U[s]);
    PA = mul2(PA, A);
  }
#pragma unroll
  for (int s = kSteps - 1; s >= 0; --s) {
    PV = mul2(decay_of(low[s], k), add2(PV, staged_pair<T>(here + 3 * kTile * kLanes + s * kLanes)));
    if (kCuts && (resets >> s & 1u)) PV = 0ull;
  }
}

struct Gradients {
  uint64_t x, r, i, E;
};
// The gradients of the staged timestep at `here`, from p after it, which
// becomes p before it; h: the state before it.
template <typename T>
__device__ __forceinline__ Gradients gradients_of(const T* here, uint64_t low, uint64_t sr, uint64_t si, uint64_t h,
                                                  uint64_t rate, const Constants& k, uint64_t& p) {
  const uint64_t A = decay_of(low, k), xs = staged_pair<T>(here);
  const uint64_t g = add2(p, staged_pair<T>(here + 3 * kTile * kLanes));
  p = mul2(g, A);
  const uint64_t m2 = m2_of(low, A, k), inv_m = rsqrt2(m2);
  const uint64_t t = mul2(rate, sr);  // -log a
  Gradients d;
  d.E = mul2(mul2(p, t), sub2(mul2(mul2(mul2(si, xs), A), inv_m), h));  // g a t (si x a / m - h)
  d.x = mul2(g, mul2(mul2(m2, inv_m), si));
  d.r = mul2(d.E, sub2(k.one, sr));
  d.i = mul2(mul2(d.x, xs), sub2(k.one, si));
  return d;
}

template <typename T, int kCopy, bool kCuts>
__global__ void __launch_bounds__(kWarps * 32, sizeof(T) == 4 ? 1 : 2) gated_scan_backward_kernel(const ScanBackwardArgs a) {
  extern __shared__ __align__(16) unsigned char staged[];
  __shared__ WarpRuns runs[2];  // h -> A h + U
  __shared__ WarpRuns back[2];  // p -> A p + V
  constexpr int kN = kStages<T, 4>;
  unsigned char* exchange = staged + kN * kStageBytes<T, 4>;
  constexpr bool kVec = kCopy >= 2 * (int)sizeof(T);
  constexpr int kOne = kTile * kLanes;  // values of one staged tensor
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rank = blockIdx.x % a.cluster, item = blockIdx.x / a.cluster;
  const int slab = item % a.slabs, b = item / a.slabs;
  const int ch0 = slab * kLanes, ch = ch0 + 2 * lane, left = a.D - ch;
  const int len = length_of(a.lengths, b, a.T);
  const T* dy = static_cast<const T*>(a.dy) + b * a.sdy.b + ch0;
  const T* x = static_cast<const T*>(a.x) + b * a.sx.b + ch0;
  const T* r = static_cast<const T*>(a.r) + b * a.sr.b + ch0;
  const T* in = static_cast<const T*>(a.i) + b * a.si.b + ch0;
  T* dx = static_cast<T*>(a.dx) + b * a.sdx.b + ch;
  T* dr = static_cast<T*>(a.dr) + b * a.sdr.b + ch;
  T* di = static_cast<T*>(a.di) + b * a.sdi.b + ch;
  const long long state_at = (long long)b * a.D + ch;
  const int stride = a.cluster * kTile;
  auto buffer = [&](int n) { return reinterpret_cast<T*>(staged + n * kStageBytes<T, 4>) + warp * kSteps * kLanes; };
  auto fetch = [&](int n, int first) {
    T* to = buffer(n);
    const int ts = first + rank * kTile + warp * kSteps;
    if (first >= 0 && ts < len) {
      stage<T, kCopy>(to, x, a.sx.t, ts, len, ch0, a.D);
      stage<T, kCopy>(to + kOne, r, a.sr.t, ts, len, ch0, a.D);
      stage<T, kCopy>(to + 2 * kOne, in, a.si.t, ts, len, ch0, a.D);
      stage<T, kCopy>(to + 3 * kOne, dy, a.sdy.t, ts, len, ch0, a.D);
    }
    stage_commit();
  };
  const int last = a.T > 0 ? (a.T - 1) / stride * stride : -1;
#pragma unroll
  for (int n = 0; n < kN - 1; ++n) fetch(n, last - n * stride);
  const uint64_t rate = rate_of(a.decay + ch, left, a.c);
  const bool far = any_far(rate);
  const Constants k = constants();
  uint64_t p = a.dh_last ? load_f32x2(a.dh_last + state_at, left) : 0ull, sum = 0ull;
  if (a.cluster > 1) cluster_sync_all();
  int turn = 0, at = 0, next = kN - 1;
  for (int first = last; first >= 0; first -= stride, turn ^= 1) {
    const int t0 = first + rank * kTile, ts = t0 + warp * kSteps;
    const unsigned resets = kCuts ? reset_bits(a.reset, ts, len, b, a.B) : 0u;
    const T* here = buffer(at) + 2 * lane;
    uint64_t h = t0 < a.T ? load_f32x2(a.states + (long long)(t0 / kTile) * a.B * a.D + state_at, left) : 0ull;
    stage_wait<kN - 2>();
    fetch(next, first - (kN - 1) * stride);
    at = at + 1 == kN ? 0 : at + 1;
    next = next + 1 == kN ? 0 : next + 1;
    const bool whole = ts + kSteps <= len;
    const bool some = ts < len;
    uint64_t low[kSteps], sr[kSteps], si[kSteps], U[kSteps], PA = k.one, PU = 0ull, PV = 0ull;
    if (some) {
      if (far) form_gates<T, true>(here, rate, k, low, sr, si, U);
      else form_gates<T, false>(here, rate, k, low, sr, si, U);
      if (!whole) {
#pragma unroll
        for (int s = 0; s < kSteps; ++s)
          if (ts + s >= len) low[s] = U[s] = 0ull;
      }
      if (resets) join_both<T, true>(here, low, U, resets, k, PA, PU, PV);
      else join_both<T, false>(here, low, U, 0u, k, PA, PU, PV);
    }
    runs[turn].AU[warp][lane] = make_ulonglong2(PA, PU);
    back[turn].AU[warp][lane] = make_ulonglong2(PA, PV);
    if (lane == 0) runs[turn].cut[warp] = back[turn].cut[warp] = resets;
    __syncthreads();
    const Runs run = runs_of(runs[turn]), rev = runs_of(back[turn]), tiles = tile_runs(exchange, a.cluster, turn);
    if (a.cluster > 1) {
      ulonglong2 all = make_ulonglong2(k.one, 0ull);
      bool cut = false;
#pragma unroll
      for (int w = kWarps - 1; w >= 0; --w) {
        all.x = mul2(all.x, rev.AU[w * 32 + lane].x);
        all.y = after<kCuts>(rev, w, all.y);
        cut = cut || rev.cut[w] != 0;
      }
      send_run(tiles, rank, a.cluster, all, cut);
      cluster_sync_all();
    }
    for (int w = 0; w < warp; ++w) h = after<kCuts>(run, w, h);
    uint64_t ps = p;  // p after this block's tile, then after this warp's timesteps
    if (a.cluster > 1) {
      for (int n = a.cluster - 1; n >= 0; --n) {
        if (n == rank) ps = p;
        p = after<kCuts>(tiles, n, p);
      }
      for (int w = kWarps - 1; w > warp; --w) ps = after<kCuts>(rev, w, ps);
    } else {
#pragma unroll
      for (int w = kWarps - 1; w >= 0; --w) {
        if (w == warp) ps = p;
        p = after<kCuts>(rev, w, p);
      }
    }
    if (some) {
      // U becomes the state before each timestep
      if (resets) {
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
          if (resets >> s & 1u) h = 0ull;
          const uint64_t u = U[s];
          U[s] = h;
          h = fma2(decay_of(low[s], k), h, u);
        }
      } else {
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
          const uint64_t u = U[s];
          U[s] = h;
          h = fma2(decay_of(low[s], k), h, u);
        }
      }
      // from the warp's last timestep back
      T* to_x = dx + (ts + kSteps - 1) * a.sdx.t;
      T* to_r = dr + (ts + kSteps - 1) * a.sdr.t;
      T* to_i = di + (ts + kSteps - 1) * a.sdi.t;
      if (whole && left > 0) {
#pragma unroll
        for (int s = kSteps - 1; s >= 0; --s) {
          const Gradients g = gradients_of<T>(here + s * kLanes, low[s], sr[s], si[s], U[s], rate, k, ps);
          if (resets && (resets >> s & 1u)) ps = 0ull;
          sum = add2(sum, g.E);
          store_both<T, kVec>(to_x, left, g.x);
          store_both<T, kVec>(to_r, left, g.r);
          store_both<T, kVec>(to_i, left, g.i);
          to_x -= a.sdx.t;
          to_r -= a.sdr.t;
          to_i -= a.sdi.t;
        }
      } else {
#pragma unroll
        for (int s = kSteps - 1; s >= 0; --s) {
          Gradients g = {0ull, 0ull, 0ull, 0ull};
          if (ts + s < len) g = gradients_of<T>(here + s * kLanes, low[s], sr[s], si[s], U[s], rate, k, ps);
          if (resets >> s & 1u) ps = 0ull;
          sum = add2(sum, g.E);
          if (left > 0 && ts + s < a.T) {
            store_both<T, kVec>(to_x, left, g.x);
            store_both<T, kVec>(to_r, left, g.r);
            store_both<T, kVec>(to_i, left, g.i);
          }
          to_x -= a.sdx.t;
          to_r -= a.sdr.t;
          to_i -= a.sdi.t;
        }
      }
    } else if (left > 0) {
      for (int t = ts; t < min(ts + kSteps, a.T); ++t) {
        store_pair<T, kVec>(dx + t * a.sdx.t, left, 0.0f, 0.0f);
        store_pair<T, kVec>(dr + t * a.sdr.t, left, 0.0f, 0.0f);
        store_pair<T, kVec>(di + t * a.sdi.t, left, 0.0f, 0.0f);
      }
    }
  }
  __syncthreads();
  runs[0].AU[warp][lane].x = sum;
  __syncthreads();
  if (warp == 0) {
    for (int w = 1; w < kWarps; ++w) sum = add2(sum, runs[0].AU[w][lane].x);
    store_f32x2(a.partial + ((long long)b * a.cluster + rank) * a.D + ch, left, sum);
    if (rank == 0) store_f32x2(a.dh0 + state_at, left, p);
  }
  if (a.cluster > 1) cluster_sync_all();
}

// ddecay from partial [n][D], summed in a fixed order.
__global__ void __launch_bounds__(1024) decay_gradient_kernel(const float* partial, int n, int D, const float* decay,
                                                              float* ddecay) {
  __shared__ float acc[32][33];
  const int col = blockIdx.x * 32 + threadIdx.x;
  float v = 0.0f;
  if (col < D)
    for (int k = threadIdx.y; k < n; k += 32) v += partial[(long long)k * D + col];
  acc[threadIdx.y][threadIdx.x] = v;
  __syncthreads();
  v = acc[threadIdx.x][threadIdx.y];
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  const int c = blockIdx.x * 32 + threadIdx.y;
  if (threadIdx.x == 0 && c < D) ddecay[c] = v * softplus_ratio_f(decay[c]);
}

struct StepArgs {
  const void *x, *r, *i;
  long long x_pitch, r_pitch, i_pitch;
  const float* decay;
  float c;
  float* state;
  int n_slots;
  const int* slots;
  const unsigned char* reset;
  int B, D;
  void* y;
};

// One timestep: a thread per pair of channels of one stream.  A few
// thousand values at most take longer to launch than to compute.
template <typename T, bool kVec>
__global__ void __launch_bounds__(256) gated_step_kernel(const StepArgs a) {
  const int ch = 2 * (blockIdx.x * blockDim.x + threadIdx.x), left = a.D - ch;
  if (left <= 0) return;
  const uint64_t rate = rate_of(a.decay + ch, left, a.c);
  const Constants k = constants();
  for (int b = blockIdx.y; b < a.B; b += gridDim.y) {
    T* y = static_cast<T*>(a.y) + (long long)b * a.D + ch;
    const int slot = a.slots ? a.slots[b] : b;
    if (slot < 0 || slot >= a.n_slots) {
      store_pair<T, kVec>(y, left, 0.0f, 0.0f);
      continue;
    }
    const float2 x = load_pair<T, kVec>(static_cast<const T*>(a.x) + b * a.x_pitch + ch, left);
    const float2 r = load_pair<T, kVec>(static_cast<const T*>(a.r) + b * a.r_pitch + ch, left);
    const float2 i = load_pair<T, kVec>(static_cast<const T*>(a.i) + b * a.i_pitch + ch, left);
    float* st = a.state + (long long)slot * a.D + ch;
    uint64_t h = load_f32x2(st, left);
    if (a.reset && a.reset[b] != 0) h = 0ull;
    const Gates g = gates_of<true>(f32x2(r.x, r.y), f32x2(i.x, i.y), rate, k);
    const uint64_t A = decay_of(g.low, k);
    h = fma2(A, h, mul2(mul2(sqrt2(m2_of(g.low, A, k)), g.si), f32x2(x.x, x.y)));
    store_f32x2(st, left, h);
    float h0, h1;
    f32x2_split(h, h0, h1);
    store_pair<T, kVec>(y, left, h0, h1);
  }
}

bool aligned_to(size_t bytes, const void* p, size_t es, const Strides& s) {
  return op_aligned(p, bytes) && s.t * es % bytes == 0 && s.b * es % bytes == 0;
}

// The widest copy (see `stage`) that every tensor's addresses allow.
int copy_bytes(int D, size_t es, const void* const* p, const Strides* s, int n) {
  auto all = [&](size_t bytes) {
    for (int k = 0; k < n; ++k)
      if (!aligned_to(bytes, p[k], es, s[k])) return false;
    return D * es % bytes == 0;
  };
  return all(16) ? 16 : (all(4) ? 4 : 2);
}

int check_sizes(int dtype, int T, int B, int D, float c, char* msg, int msg_len) {
  if (!op_float_dtype(dtype)) return op_report(msg, msg_len, LSTM_APPROX_EINVAL, "dtype %d", dtype);
  if (T < 0 || B < 0 || D < 1 || T > 0x7fffff00 || (long long)B * ((D + kLanes - 1) / kLanes) > 0x7fffffffll || (long long)B * kMaxCluster > 0x7fffffffll)
    return op_report(msg, msg_len, LSTM_APPROX_EINVAL, "need T, B >= 0, D >= 1 and B ceil(D / 64) below 2^31");
  if (!(c > 0.0f)) return op_report(msg, msg_len, LSTM_APPROX_EINVAL, "c must be positive");
  return LSTM_APPROX_OK;
}

// Blocks of a cluster that share a stream's 64 channels: doubled while all
// blocks still run at once (two to an SM; clusters of 8 or 16 leave some of a
// processor group's slots empty) and each has a tile to itself.
int cluster_size(int T, int B, int D) {
  const long long items = (long long)B * ((D + kLanes - 1) / kLanes);
  int n = 1;
  while (n < kMaxCluster && items * 2 * n <= 256 && (long long)n * kTile < T) n *= 2;
  return n;
}

template <typename T, int kCopy, bool kCuts, int kTensors, typename A>
cudaError_t launch_scan(void (*kern)(A), int cluster, int blocks, cudaStream_t s, const A& args) {
  static thread_local DeviceSet ready;  // of the one kernel that this instance launches
  constexpr size_t smem = kStages<T, kTensors> * kStageBytes<T, kTensors>;
  constexpr int most = (int)(smem + exchange_bytes(kMaxCluster));
  const cudaError_t e = once_per_device(&ready, [&] {
    const cudaError_t e1 = cudaFuncSetAttribute(kern, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    return e1 != cudaSuccess ? e1 : cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, most);
  });
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(blocks);
  cfg.blockDim = dim3(kWarps * 32);
  cfg.dynamicSmemBytes = smem + exchange_bytes(cluster);
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = cluster;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = cluster > 1 ? 1 : 0;
  return cudaLaunchKernelEx(&cfg, kern, args);
}

// Strides of n tensors: HOST [2n], or all contiguous [T][B][D].
bool read_strides(const long long* strides, int n, int B, int D, Strides* out) {
  for (int k = 0; k < n; ++k) {
    out[k] = strides ? Strides{strides[2 * k], strides[2 * k + 1]} : Strides{(long long)B * D, D};
    if (out[k].t < 0 || out[k].b < 0) return false;
  }
  return true;
}

}  // namespace
}  // namespace lstm_approx_impl

using namespace lstm_approx_impl;

extern "C" int lstm_approx_gated_scan(int dtype, const void* x, const void* r, const void* i, const float* decay,
                                      float c, const float* h0, const int32_t* lengths, const unsigned char* reset,
                                      int T, int B, int D, void* y, const long long* strides, float* h_last,
                                      float* states, void* cuda_stream, char* msg, int msg_len) {
  if (msg && msg_len > 0) msg[0] = '\0';
  if (int rc = check_sizes(dtype, T, B, D, c, msg, msg_len)) return rc;
  if (B > 0 && (!decay || !h_last || (T > 0 && (!x || !r || !i || !y))))
    return op_report(msg, msg_len, LSTM_APPROX_EINVAL, "x, r, i, decay, y and h_last must not be NULL");
  const size_t es = op_dtype_bytes(dtype);
  if (!op_aligned(x, es) || !op_aligned(r, es) || !op_aligned(i, es) || !op_aligned(y, es) || !op_aligned(decay, 4) ||
      !op_aligned(h0, 4) || !op_aligned(lengths, 4) || !op_aligned(h_last, 4) || !op_aligned(states, 4))
    return op_report(msg, msg_len, LSTM_APPROX_EINVAL, "a pointer is not aligned to its type");
  Strides st[4];
  if (!read_strides(strides, 4, B, D, st))
    return op_report(msg, msg_len, LSTM_APPROX_EINVAL, "strides must not be negative");
  if (int rc = op_check_device(msg, msg_len)) return rc;
  if (B == 0) return LSTM_APPROX_OK;
  const int slabs = (D + kLanes - 1) / kLanes, n = cluster_size(T, B, D);
  ScanArgs a{x, r, i, y, st[0], st[1], st[2], st[3], decay, c, h0, lengths, reset, T, B, D, slabs, n,
             h_last, states};
  const void* tensors[4] = {x, r, i, y};
  const int copy = copy_bytes(D, es, tensors, st, 4);
  const cudaError_t e = op_for_type(dtype, [&](auto* t) {
    using E = std::remove_pointer_t<decltype(t)>;
    cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
    auto go = [&](auto bytes) {
      constexpr int kCopy = decltype(bytes)::value;
      return reset ? launch_scan<E, kCopy, true, 3>(gated_scan_kernel<E, kCopy, true>, n, slabs * B * n, s, a)
                   : launch_scan<E, kCopy, false, 3>(gated_scan_kernel<E, kCopy, false>, n, slabs * B * n, s, a);
    };
    if (copy == 16) return go(std::integral_constant<int, 16>());
    if (copy == 4 || sizeof(E) == 4) return go(std::integral_constant<int, 4>());
    return go(std::integral_constant<int, sizeof(E) == 4 ? 4 : 2>());  // 32-bit values are always copied
  });
  return op_launched(e, "scan launch", msg, msg_len);
}

extern "C" size_t lstm_approx_gated_scan_workspace_bytes(int T, int B, int D) {
  if (T < 0 || B < 0 || D < 1) return 0;
  return ((size_t)B * cluster_size(T, B, D) * D * sizeof(float) + 15) / 16 * 16 + 16;
}

extern "C" int lstm_approx_gated_scan_backward(int dtype, const void* dy, const float* dh_last, const void* x,
                                               const void* r, const void* i, const float* decay, float c,
                                               const float* states, const int32_t* lengths,
                                               const unsigned char* reset, int T, int B, int D, void* dx, void* dr,
                                               void* di, const long long* strides, float* ddecay, float* dh0,
                                               void* workspace, size_t workspace_bytes, void* cuda_stream, char* msg,
                                               int msg_len) {
  if (msg && msg_len > 0) msg[0] = '\0';
  if (int rc = check_sizes(dtype, T, B, D, c, msg, msg_len)) return rc;
  if (!decay || !ddecay || !workspace ||
      (B > 0 && (!dh0 || (T > 0 && (!dy || !x || !r || !i || !states || !dx || !dr || !di)))))
    return op_report(msg, msg_len, LSTM_APPROX_EINVAL,
                     "dy, x, r, i, decay, states, dx, dr, di, ddecay, dh0 and workspace must not be NULL");
  const size_t es = op_dtype_bytes(dtype);
  if (!op_aligned(dy, es) || !op_aligned(x, es) || !op_aligned(r, es) || !op_aligned(i, es) || !op_aligned(dx, es) ||
      !op_aligned(dr, es) || !op_aligned(di, es) || !op_aligned(decay, 4) || !op_aligned(dh_last, 4) ||
      !op_aligned(lengths, 4) || !op_aligned(states, 4) || !op_aligned(ddecay, 4) || !op_aligned(dh0, 4))
    return op_report(msg, msg_len, LSTM_APPROX_EINVAL, "a pointer is not aligned to its type");
  Strides st[7];
  if (!read_strides(strides, 7, B, D, st))
    return op_report(msg, msg_len, LSTM_APPROX_EINVAL, "strides must not be negative");
  const size_t need = lstm_approx_gated_scan_workspace_bytes(T, B, D);
  if (!op_aligned(workspace, 16) || workspace_bytes < need)
    return op_report(msg, msg_len, LSTM_APPROX_EINVAL, "needs a 16-byte aligned workspace of %zu bytes", need);
  if (int rc = op_check_device(msg, msg_len)) return rc;
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  float* partial = static_cast<float*>(workspace);
  const int n = cluster_size(T, B, D);
  if (B > 0) {
    const int slabs = (D + kLanes - 1) / kLanes;
    ScanBackwardArgs a{dy,    x,     r,      i,       dx,    dr, di, st[0], st[1], st[2], st[3], st[4], st[5], st[6],
                       dh_last, decay, c, states, lengths, reset, T,  B,  D,     slabs, n, dh0,   partial};
    const void* tensors[7] = {dy, x, r, i, dx, dr, di};
    const int copy = copy_bytes(D, es, tensors, st, 7);
    const cudaError_t e = op_for_type(dtype, [&](auto* t) {
      using E = std::remove_pointer_t<decltype(t)>;
      auto go = [&](auto bytes) {
        constexpr int kCopy = decltype(bytes)::value;
        return reset
                   ? launch_scan<E, kCopy, true, 4>(gated_scan_backward_kernel<E, kCopy, true>, n, slabs * B * n, s, a)
                   : launch_scan<E, kCopy, false, 4>(gated_scan_backward_kernel<E, kCopy, false>, n, slabs * B * n, s, a);
      };
      if (copy == 16) return go(std::integral_constant<int, 16>());
      if (copy == 4 || sizeof(E) == 4) return go(std::integral_constant<int, 4>());
      return go(std::integral_constant<int, sizeof(E) == 4 ? 4 : 2>());
    });
    if (int rc = op_launched(e, "scan backward launch", msg, msg_len)) return rc;
  }
  const cudaError_t e = op_launch(decay_gradient_kernel, dim3((D + 31) / 32), dim3(32, 32), 0, s,
                                  static_cast<const float*>(partial), B * n, D, decay, ddecay);
  return op_launched(e, "decay gradient launch", msg, msg_len);
}

extern "C" int lstm_approx_gated_step(int dtype, const void* x, long long x_pitch, const void* r, long long r_pitch,
                                      const void* i, long long i_pitch, const float* decay, float c, float* state,
                                      int n_slots, const int32_t* slots, const unsigned char* reset, int B, int D,
                                      void* y, void* cuda_stream, char* msg, int msg_len) {
  if (msg && msg_len > 0) msg[0] = '\0';
  if (int rc = check_sizes(dtype, 1, B, D, c, msg, msg_len)) return rc;
  if (n_slots < 0 || (!slots && B > n_slots))
    return op_report(msg, msg_len, LSTM_APPROX_EINVAL, "%d streams and %d states without slots", B, n_slots);
  if (B > 0 && (!x || !r || !i || !decay || !y || (n_slots > 0 && !state)))
    return op_report(msg, msg_len, LSTM_APPROX_EINVAL, "x, r, i, decay, state and y must not be NULL");
  const size_t es = op_dtype_bytes(dtype);
  if (x_pitch < 0 || r_pitch < 0 || i_pitch < 0 || !op_aligned(x, es) || !op_aligned(r, es) || !op_aligned(i, es) ||
      !op_aligned(y, es) || !op_aligned(decay, 4) || !op_aligned(state, 4) || !op_aligned(slots, 4))
    return op_report(msg, msg_len, LSTM_APPROX_EINVAL, "a negative pitch, or a pointer not aligned to its type");
  if (int rc = op_check_device(msg, msg_len)) return rc;
  if (B == 0) return LSTM_APPROX_OK;
  StepArgs a{x, r, i, x_pitch, r_pitch, i_pitch, decay, c, state, n_slots, slots, reset, B, D, y};
  const bool vec = D % 2 == 0 && aligned_to(2 * es, x, es, {0, x_pitch}) && aligned_to(2 * es, r, es, {0, r_pitch}) &&
                   aligned_to(2 * es, i, es, {0, i_pitch}) && op_aligned(y, 2 * es);
  const int threads = D >= 512 ? 256 : 64;
  const dim3 grid((D + 2 * threads - 1) / (2 * threads), std::min(B, 65535));
  const cudaError_t e = op_for_type(dtype, [&](auto* t) {
    using E = std::remove_pointer_t<decltype(t)>;
    return op_launch(vec ? gated_step_kernel<E, true> : gated_step_kernel<E, false>, grid, dim3(threads), 0,
                     static_cast<cudaStream_t>(cuda_stream), a);
  });
  return op_launched(e, "step launch", msg, msg_len);
}
