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

// 1 - e^t for t <= 0: above -0.35 by its Taylor series to t^8 (the first
// term left out is t^8 / 9! < 7e-10 of the first), which has no cancellation.
__device__ __forceinline__ float one_minus_exp(float t) {
  float p = 1.0f / 40320.0f;
  p = fmaf(p, t, 1.0f / 5040.0f);
  p = fmaf(p, t, 1.0f / 720.0f);
  p = fmaf(p, t, 1.0f / 120.0f);
  p = fmaf(p, t, 1.0f / 24.0f);
  p = fmaf(p, t, 1.0f / 6.0f);
  p = fmaf(p, t, 0.5f);
  p = fmaf(p, t, 1.0f);
  return t > -0.35f ? -t * p : 1.0f - ex2_approx(t * kLog2E);
}

__device__ __forceinline__ float sqrt_approx(float x) {
  float r;
  asm("sqrt.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}

struct Gates {
  float sr, si, la, a, m;
};
// rate = -c softplus(decay)
__device__ __forceinline__ Gates gates_of(float r, float i, float rate) {
  Gates g;
  g.sr = sigmoid_f(r);
  g.si = sigmoid_f(i);
  g.la = rate * g.sr;
  // a = 1 - (1 - a) and m^2 = (1 - a)(1 + a): a decay near 1, which acts over
  // hundreds of timesteps, comes out correctly rounded, and m keeps its digits
  const float low = one_minus_exp(g.la);
  g.a = 1.0f - low;
  g.m = sqrt_approx(low * (1.0f + g.a));
  return g;
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

struct Strides {
  long long t, b;
};

struct ScanArgs {
  const void *x, *r, *i;
  void* y;
  Strides sx, sr, si, sy;
  const float* decay;
  float c;
  const float* h0;
  const int* lengths;
  const unsigned char* reset;
  int T, B, D, slabs;
  float* h_last;
  float* states;
};

__device__ __forceinline__ int length_of(const int* lengths, int b, int T) {
  return lengths ? min(max(lengths[b], 0), T) : T;
}

// Bit s: reset at timestep ts + s of this warp (the same in all lanes).
__device__ __forceinline__ unsigned reset_bits(const unsigned char* reset, int ts, int len, int b, int B) {
  if (!reset) return 0u;
  const int lane = threadIdx.x & 31, t = ts + lane;
  const bool on = lane < kSteps && t < len && reset[(long long)t * B + b] != 0;
  return __ballot_sync(0xffffffffu, on);
}

// One warp's run: state after it = cut ? U : A h + U.
struct Run {
  float2 A[kWarps][32], U[kWarps][32];
  unsigned cut[kWarps];
};

template <typename T, bool kVec>
__global__ void __launch_bounds__(kWarps * 32) gated_scan_kernel(const ScanArgs a) {
  __shared__ Run runs[2];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int slab = blockIdx.x % a.slabs, b = blockIdx.x / a.slabs;
  const int ch = slab * kLanes + 2 * lane, left = a.D - ch;  // channels of this lane that exist: min(left, 2)
  const bool any = left > 0;
  const int len = length_of(a.lengths, b, a.T);
  const T* x = static_cast<const T*>(a.x) + b * a.sx.b + ch;
  const T* r = static_cast<const T*>(a.r) + b * a.sr.b + ch;
  const T* in = static_cast<const T*>(a.i) + b * a.si.b + ch;
  T* y = static_cast<T*>(a.y) + b * a.sy.b + ch;
  const long long state_at = (long long)b * a.D + ch;
  float2 rate = make_float2(0.0f, 0.0f), h = make_float2(0.0f, 0.0f);
  if (any) {
    const float2 d = load_pair<float, false>(a.decay + ch, left);
    rate = make_float2(-a.c * softplus_f(d.x), -a.c * softplus_f(d.y));
    if (a.h0) h = load_pair<float, false>(a.h0 + state_at, left);
  }
  int turn = 0;
  for (int t0 = 0; t0 < a.T; t0 += kTile, turn ^= 1) {
    const int ts = t0 + warp * kSteps;
    const unsigned resets = reset_bits(a.reset, ts, len, b, a.B);
    float2 A[kSteps], U[kSteps];
    float2 xs[kSteps], rs[kSteps], is[kSteps];
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
      xs[s] = rs[s] = is[s] = make_float2(0.0f, 0.0f);
      if (any && ts + s < len) {
        xs[s] = load_pair<T, kVec>(x + (ts + s) * a.sx.t, left);
        rs[s] = load_pair<T, kVec>(r + (ts + s) * a.sr.t, left);
        is[s] = load_pair<T, kVec>(in + (ts + s) * a.si.t, left);
      }
    }
    float2 PA = make_float2(1.0f, 1.0f), PU = make_float2(0.0f, 0.0f);
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
      const Gates g0 = gates_of(rs[s].x, is[s].x, rate.x), g1 = gates_of(rs[s].y, is[s].y, rate.y);
      const bool live = ts + s < len, cut = resets >> s & 1u;
      A[s] = live ? make_float2(g0.a, g1.a) : make_float2(1.0f, 1.0f);
      U[s] = live ? make_float2(g0.m * g0.si * xs[s].x, g1.m * g1.si * xs[s].y) : make_float2(0.0f, 0.0f);
      PU.x = cut ? U[s].x : fmaf(A[s].x, PU.x, U[s].x);
      PU.y = cut ? U[s].y : fmaf(A[s].y, PU.y, U[s].y);
      PA.x *= A[s].x;
      PA.y *= A[s].y;
    }
    Run& run = runs[turn];  // the other one may still be read
    run.A[warp][lane] = PA;
    run.U[warp][lane] = PU;
    if (lane == 0) run.cut[warp] = resets;
    __syncthreads();
    float2 hs = h;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
      const float2 wa = run.A[w][lane], wu = run.U[w][lane];
      const bool cut = run.cut[w] != 0;
      if (w == warp) hs = h;
      h.x = cut ? wu.x : fmaf(wa.x, h.x, wu.x);
      h.y = cut ? wu.y : fmaf(wa.y, h.y, wu.y);
    }
    if (a.states && warp == 0 && any)
      store_pair<float, false>(a.states + (long long)(t0 / kTile) * a.B * a.D + state_at, left, hs.x, hs.y);
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
      const bool cut = resets >> s & 1u;
      hs.x = cut ? U[s].x : fmaf(A[s].x, hs.x, U[s].x);
      hs.y = cut ? U[s].y : fmaf(A[s].y, hs.y, U[s].y);
      const bool live = ts + s < len;
      if (any && ts + s < a.T)
        store_pair<T, kVec>(y + (ts + s) * a.sy.t, left, live ? hs.x : 0.0f, live ? hs.y : 0.0f);
    }
  }
  if (warp == 0 && any) store_pair<float, false>(a.h_last + state_at, left, h.x, h.y);
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
  int T, B, D, slabs;
  float* dh0;
  float* partial;  // [B][D]: sum of E over the stream's timesteps
};

template <typename T, bool kVec>
__global__ void __launch_bounds__(kWarps * 32) gated_scan_backward_kernel(const ScanBackwardArgs a) {
  __shared__ Run runs[2];
  __shared__ float2 back[2][kWarps][32];  // V of p -> A p + V (A: as forward)
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int slab = blockIdx.x % a.slabs, b = blockIdx.x / a.slabs;
  const int ch = slab * kLanes + 2 * lane, left = a.D - ch;
  const bool any = left > 0;
  const int len = length_of(a.lengths, b, a.T);
  const T* dy = static_cast<const T*>(a.dy) + b * a.sdy.b + ch;
  const T* x = static_cast<const T*>(a.x) + b * a.sx.b + ch;
  const T* r = static_cast<const T*>(a.r) + b * a.sr.b + ch;
  const T* in = static_cast<const T*>(a.i) + b * a.si.b + ch;
  T* dx = static_cast<T*>(a.dx) + b * a.sdx.b + ch;
  T* dr = static_cast<T*>(a.dr) + b * a.sdr.b + ch;
  T* di = static_cast<T*>(a.di) + b * a.sdi.b + ch;
  const long long state_at = (long long)b * a.D + ch;
  float2 rate = make_float2(0.0f, 0.0f), p = make_float2(0.0f, 0.0f), sum = make_float2(0.0f, 0.0f);
  if (any) {
    const float2 d = load_pair<float, false>(a.decay + ch, left);
    rate = make_float2(-a.c * softplus_f(d.x), -a.c * softplus_f(d.y));
    if (a.dh_last) p = load_pair<float, false>(a.dh_last + state_at, left);
  }
  int turn = 0;
  for (int t0 = (a.T - 1) / kTile * kTile; t0 >= 0 && a.T > 0; t0 -= kTile, turn ^= 1) {
    const int ts = t0 + warp * kSteps;
    const unsigned resets = reset_bits(a.reset, ts, len, b, a.B);
    float2 ys[kSteps], xs[kSteps], rs[kSteps], is[kSteps];
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
      ys[s] = xs[s] = rs[s] = is[s] = make_float2(0.0f, 0.0f);
      if (any && ts + s < len) {
        xs[s] = load_pair<T, kVec>(x + (ts + s) * a.sx.t, left);
        rs[s] = load_pair<T, kVec>(r + (ts + s) * a.sr.t, left);
        is[s] = load_pair<T, kVec>(in + (ts + s) * a.si.t, left);
        ys[s] = load_pair<T, kVec>(dy + (ts + s) * a.sdy.t, left);
      }
    }
    float2 h = make_float2(0.0f, 0.0f);
    if (any) h = load_pair<float, false>(a.states + (long long)(t0 / kTile) * a.B * a.D + state_at, left);
    float2 A[kSteps], U[kSteps];
    float2 PA = make_float2(1.0f, 1.0f), PU = make_float2(0.0f, 0.0f), PV = make_float2(0.0f, 0.0f);
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
      const Gates g0 = gates_of(rs[s].x, is[s].x, rate.x), g1 = gates_of(rs[s].y, is[s].y, rate.y);
      const bool live = ts + s < len, cut = resets >> s & 1u;
      A[s] = live ? make_float2(g0.a, g1.a) : make_float2(1.0f, 1.0f);
      U[s] = live ? make_float2(g0.m * g0.si * xs[s].x, g1.m * g1.si * xs[s].y) : make_float2(0.0f, 0.0f);
      PU.x = cut ? U[s].x : fmaf(A[s].x, PU.x, U[s].x);
      PU.y = cut ? U[s].y : fmaf(A[s].y, PU.y, U[s].y);
      PA.x *= A[s].x;
      PA.y *= A[s].y;
    }
#pragma unroll
    for (int s = kSteps - 1; s >= 0; --s) {
      const bool cut = resets >> s & 1u;
      PV.x = cut ? 0.0f : A[s].x * (ys[s].x + PV.x);
      PV.y = cut ? 0.0f : A[s].y * (ys[s].y + PV.y);
    }
    Run& run = runs[turn];
    run.A[warp][lane] = PA;
    run.U[warp][lane] = PU;
    back[turn][warp][lane] = PV;
    if (lane == 0) run.cut[warp] = resets;
    __syncthreads();
    for (int w = 0; w < warp; ++w) {
      const float2 wa = run.A[w][lane], wu = run.U[w][lane];
      const bool cut = run.cut[w] != 0;
      h.x = cut ? wu.x : fmaf(wa.x, h.x, wu.x);
      h.y = cut ? wu.y : fmaf(wa.y, h.y, wu.y);
    }
    float2 ps = p;
#pragma unroll
    for (int w = kWarps - 1; w >= 0; --w) {
      const float2 wa = run.A[w][lane], wv = back[turn][w][lane];
      const bool cut = run.cut[w] != 0;
      if (w == warp) ps = p;
      p.x = cut ? wv.x : fmaf(wa.x, p.x, wv.x);
      p.y = cut ? wv.y : fmaf(wa.y, p.y, wv.y);
    }
    float2 before[kSteps];
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
      const bool cut = resets >> s & 1u;
      before[s] = cut ? make_float2(0.0f, 0.0f) : h;
      h.x = cut ? U[s].x : fmaf(A[s].x, h.x, U[s].x);
      h.y = cut ? U[s].y : fmaf(A[s].y, h.y, U[s].y);
    }
#pragma unroll
    for (int s = kSteps - 1; s >= 0; --s) {
      const bool live = ts + s < len, cut = resets >> s & 1u;
      float gx[2], gr[2], gi[2];
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const float rr = e ? rs[s].y : rs[s].x, ii = e ? is[s].y : is[s].x, xx = e ? xs[s].y : xs[s].x;
        const float hh = e ? before[s].y : before[s].x, dd = e ? ys[s].y : ys[s].x;
        float& pp = e ? ps.y : ps.x;
        const Gates g = gates_of(rr, ii, e ? rate.y : rate.x);
        const float grad = dd + pp;
        if (live) pp = cut ? 0.0f : g.a * grad;
        const float q = g.m > 0.0f ? -g.la * rcp_approx(g.m) : 0.0f;
        const float E = grad * g.a * fmaf(g.la, hh, g.si * xx * g.a * q);
        const float gm = grad * g.m * g.si;
        gx[e] = live ? gm : 0.0f;
        gr[e] = live ? E * (1.0f - g.sr) : 0.0f;
        gi[e] = live ? gm * xx * (1.0f - g.si) : 0.0f;
        if (live) (e ? sum.y : sum.x) += E;
      }
      if (any && ts + s < a.T) {
        store_pair<T, kVec>(dx + (ts + s) * a.sdx.t, left, gx[0], gx[1]);
        store_pair<T, kVec>(dr + (ts + s) * a.sdr.t, left, gr[0], gr[1]);
        store_pair<T, kVec>(di + (ts + s) * a.sdi.t, left, gi[0], gi[1]);
      }
    }
  }
  __syncthreads();
  back[0][warp][lane] = sum;
  __syncthreads();
  if (warp == 0 && any) {
    for (int w = 1; w < kWarps; ++w) {
      sum.x += back[0][w][lane].x;
      sum.y += back[0][w][lane].y;
    }
    store_pair<float, false>(a.partial + state_at, left, sum.x, sum.y);
    store_pair<float, false>(a.dh0 + state_at, left, p.x, p.y);
  }
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
  const float2 d = load_pair<float, false>(a.decay + ch, left);
  const float2 rate = make_float2(-a.c * softplus_f(d.x), -a.c * softplus_f(d.y));
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
    const bool cut = a.reset && a.reset[b] != 0;
    const float2 h = load_pair<float, false>(st, left);
    const Gates g0 = gates_of(r.x, i.x, rate.x), g1 = gates_of(r.y, i.y, rate.y);
    const float u0 = g0.m * g0.si * x.x, u1 = g1.m * g1.si * x.y;
    const float h0 = cut ? u0 : fmaf(g0.a, h.x, u0), h1 = cut ? u1 : fmaf(g1.a, h.y, u1);
    store_pair<float, false>(st, left, h0, h1);
    store_pair<T, kVec>(y, left, h0, h1);
  }
}

bool pair_ok(const void* p, size_t es, const Strides& s) {
  return op_aligned(p, 2 * es) && s.t % 2 == 0 && s.b % 2 == 0;
}

int check_sizes(int dtype, int T, int B, int D, float c, char* msg, int msg_len) {
  if (!op_float_dtype(dtype)) return op_report(msg, msg_len, LSTM_APPROX_EINVAL, "dtype %d", dtype);
  if (T < 0 || B < 0 || D < 1 || T > 0x7fffff00 || (long long)B * ((D + kLanes - 1) / kLanes) > 0x7fffffffll)
    return op_report(msg, msg_len, LSTM_APPROX_EINVAL, "need T, B >= 0, D >= 1 and B ceil(D / 64) below 2^31");
  if (!(c > 0.0f)) return op_report(msg, msg_len, LSTM_APPROX_EINVAL, "c must be positive");
  return LSTM_APPROX_OK;
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
  const int slabs = (D + kLanes - 1) / kLanes;
  ScanArgs a{x, r, i, y, st[0], st[1], st[2], st[3], decay, c, h0, lengths, reset, T, B, D, slabs, h_last, states};
  const bool vec = D % 2 == 0 && pair_ok(x, es, st[0]) && pair_ok(r, es, st[1]) && pair_ok(i, es, st[2]) &&
                   pair_ok(y, es, st[3]);
  const cudaError_t e = op_for_type(dtype, [&](auto* t) {
    using E = std::remove_pointer_t<decltype(t)>;
    return op_launch(vec ? gated_scan_kernel<E, true> : gated_scan_kernel<E, false>, dim3(slabs * B),
                     dim3(kWarps * 32), 0, static_cast<cudaStream_t>(cuda_stream), a);
  });
  return op_launched(e, "scan launch", msg, msg_len);
}

extern "C" size_t lstm_approx_gated_scan_workspace_bytes(int T, int B, int D) {
  if (T < 0 || B < 0 || D < 1) return 0;
  return ((size_t)B * D * sizeof(float) + 15) / 16 * 16 + 16;
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
  if (B > 0) {
    const int slabs = (D + kLanes - 1) / kLanes;
    ScanBackwardArgs a{dy,    x,     r,      i,       dx,    dr, di, st[0], st[1], st[2], st[3], st[4], st[5], st[6],
                       dh_last, decay, c, states, lengths, reset, T,  B,  D,     slabs, dh0,   partial};
    const bool vec = D % 2 == 0 && pair_ok(dy, es, st[0]) && pair_ok(x, es, st[1]) && pair_ok(r, es, st[2]) &&
                     pair_ok(i, es, st[3]) && pair_ok(dx, es, st[4]) && pair_ok(dr, es, st[5]) &&
                     pair_ok(di, es, st[6]);
    const cudaError_t e = op_for_type(dtype, [&](auto* t) {
      using E = std::remove_pointer_t<decltype(t)>;
      return op_launch(vec ? gated_scan_backward_kernel<E, true> : gated_scan_backward_kernel<E, false>,
                       dim3(slabs * B), dim3(kWarps * 32), 0, s, a);
    });
    if (int rc = op_launched(e, "scan backward launch", msg, msg_len)) return rc;
  }
  const cudaError_t e = op_launch(decay_gradient_kernel, dim3((D + 31) / 32), dim3(32, 32), 0, s,
                                  static_cast<const float*>(partial), B, D, decay, ddecay);
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
  const bool vec = D % 2 == 0 && pair_ok(x, es, {0, x_pitch}) && pair_ok(r, es, {0, r_pitch}) &&
                   pair_ok(i, es, {0, i_pitch}) && op_aligned(y, 2 * es);
  const int threads = D >= 512 ? 256 : 64;
  const dim3 grid((D + 2 * threads - 1) / (2 * threads), std::min(B, 65535));
  const cudaError_t e = op_for_type(dtype, [&](auto* t) {
    using E = std::remove_pointer_t<decltype(t)>;
    return op_launch(vec ? gated_step_kernel<E, true> : gated_step_kernel<E, false>, grid, dim3(threads), 0,
                     static_cast<cudaStream_t>(cuda_stream), a);
  });
  return op_launched(e, "step launch", msg, msg_len);
}
