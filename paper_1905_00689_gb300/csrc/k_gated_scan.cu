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
// The tiles of all streams and channels are tasks, in the order of time, that
// go round the blocks of one wave (a cooperative launch, so that all of them
// run at once).  A task forms its tile's run while the tiles before it are
// formed by other blocks, and learns the state it starts with through memory:
// every tile writes its (A, U), and the last of each group of up to 16 tiles the
// state after it; a tile takes the state before its group and joins the runs of
// the group's tiles before its own, in their order.  What joins what depends on
// the shape alone.  So the sequence is read once, the work is even whatever the
// shape, and the chain through a sequence has one link per 1024 timesteps.
// (With the blocks of a cluster of up to 16 along T, joined through distributed
// shared memory, 8192 x 1 x 2048 bf16 took 57 us and 20000 x 1 x 512 fp32 111:
// too few warps run at once, and clusters do not fill the last wave.)
//
// The exchanged words are their own flags: a first kernel fills the exchange
// with a NaN pattern that no result has, and a reader takes a word once it
// differs.  Every wait ends after 2 s at the latest, with that NaN as the value.
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
// Measured (device time; % of the 6784 GB/s that a copy reaches; all decays above
// 0.88 where the gate is open):
//   8191 x 1 x 2048 bf16      forward 41 us (48%)   backward 77 us (45%)
//   2048 x 8 x 2048 bf16              62    (63%)           127    (55%)
//   2048 x 8 x 2048 fp32              87    (91%)           191    (73%)
//   20000 x 1 x 512 fp32              42    (58%)            80    (53%)
//   700 x 13 x 1000 fp16              27    (39%)            53    (35%)
// Decays between 0.70 and 0.88 take 2048 x 8 x 2048 bf16 to 65 and 129 us, smaller
// ones to 70 and 138 (see Reach).  32-bit inputs of several streams come near the
// memory's rate.  In 16 bits nothing is saturated (profiled with
// decays down to 0.86): 35 instructions forward and 80
// backward to a warp's 32 elements, issued in 52% and 58% of the cycles by the two
// blocks of 8 warps that an SM's registers hold, special functions (5 to an element)
// 29% and 18%, memory 40%.  A task loads, forms its gates, meets in a barrier,
// exchanges, meets again and goes over its timesteps in turn, and two blocks do not
// cover each other's waits: barriers are among the first stalls.  One long sequence
// besides pays the chain of groups (a state is published once the one before it has
// come), and short ones the first kernel too, 5 us together.  A single
// step: 64 x 1024 1.9 us (the launch), 1000 x 2048 fp16 7.7 us (63%).
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
constexpr int kLanes = 64;                    // channels of a block: two to a lane
constexpr int kChunk = LSTM_APPROX_SCAN_CHUNK;  // timesteps from one saved state to the next
// Timesteps of a warp in a tile, kWarps times that in the tile: 16 forward for
// 16-bit values, 8 where the registers or shared memory do not hold so many.
template <typename T>
constexpr int kForwardSteps = sizeof(T) == 4 ? 8 : 16;
constexpr int kBackwardSteps = 8;
static_assert(kWarps * kBackwardSteps == kChunk, "the backward pass takes one saved state per tile");

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
// there is one for two): sigma(r), sigma(i), a and 1 - a, from which m
// follows.  rate = c softplus(decay), the largest t = -log a of a channel.
//
// 1 - a = 1 - e^-t by its Taylor series: no cancellation, a = 1 - (1 - a)
// comes out correctly rounded, which matters where a state decays over hundreds
// of timesteps, and 1 - a^2 = (1 - a)(1 + a) keeps its digits.  Up to t = 1/8
// (decays down to 0.88 where the gate is open) five terms do (the sixth is
// below 4.3e-8 of the first); beyond, eight up to t = 0.35 (the ninth is below
// 7e-10).  Above that a is the exponential itself, within 2^-22 + t 2^-23 of its
// size, and 1 - a follows from it: a small a is a factor of all that goes back
// through the timestep, and 1 - (1 - a) would leave it to a multiple of 2^-24.
// What a warp has to do goes by the largest rate of its channels:
enum Reach { kNear, kMiddle, kFar };  // up to 1/8, up to 0.35, above
constexpr float kNearRate = 0.125f, kMiddleRate = 0.35f;
//
// Sigma is formed from the hardware's exponential and reciprocal: within 2^-21
// + |z| 2^-24 of its size (2e-6 at |z| = 20).
struct Gates {
  uint64_t sr, si, a, low;  // low: 1 - a
};
// The series.
template <Reach kReach>
__device__ __forceinline__ uint64_t low_series(uint64_t t, const Constants& k) {
  uint64_t p = k.c4;
  if constexpr (kReach != kNear) {
    p = both(-1.0f / 40320.0f);
    p = fma2(p, t, both(1.0f / 5040.0f));
    p = fma2(p, t, both(-1.0f / 720.0f));
    p = fma2(p, t, k.c4);
  }
  p = fma2(p, t, k.c3);
  p = fma2(p, t, k.c2);
  p = fma2(p, t, k.c1);
  p = fma2(p, t, k.one);
  return mul2(t, p);
}
template <Reach kReach>
__device__ __forceinline__ Gates gates_of(uint64_t r, uint64_t i, uint64_t rate, const Constants& k) {
  Gates g;
  g.sr = sigmoid2(r, k);
  g.si = sigmoid2(i, k);
  const uint64_t t = mul2(rate, g.sr);
  g.low = low_series<kReach>(t, k);
  g.a = sub2(k.one, g.low);
  if constexpr (kReach == kFar) {
    float t0, t1, a0, a1, l0, l1;
    f32x2_split(t, t0, t1);
    f32x2_split(g.a, a0, a1);
    f32x2_split(g.low, l0, l1);
    if (t0 > kMiddleRate) a0 = ex2_approx(-t0 * kLog2E), l0 = 1.0f - a0;
    if (t1 > kMiddleRate) a1 = ex2_approx(-t1 * kLog2E), l1 = 1.0f - a1;
    g.a = f32x2(a0, a1);
    g.low = f32x2(l0, l1);
  }
  return g;
}
// What the backward pass keeps of a timestep's decay: 1 - a, from which a follows, but a itself where it may be small
// (kFar), and then 1 - a is formed again from t.
template <Reach kReach>
__device__ __forceinline__ uint64_t held_decay(const Gates& g) { return kReach == kFar ? g.a : g.low; }
template <Reach kReach>
__device__ __forceinline__ uint64_t decay_of(uint64_t held, const Constants& k) {
  return kReach == kFar ? held : sub2(k.one, held);
}
template <Reach kReach>
__device__ __forceinline__ uint64_t low_of(uint64_t held, uint64_t t, const Constants& k) {
  if constexpr (kReach != kFar) return held;
  float t0, t1, a0, a1, l0, l1;
  f32x2_split(t, t0, t1);
  f32x2_split(held, a0, a1);
  f32x2_split(low_series<kReach>(t, k), l0, l1);
  return f32x2(t0 > kMiddleRate ? 1.0f - a0 : l0, t1 > kMiddleRate ? 1.0f - a1 : l1);
}
// 1 - a^2
__device__ __forceinline__ uint64_t m2_of(uint64_t low, uint64_t a, const Constants& k) {
  return mul2(low, add2(a, k.one));
}
// 1 / sqrt(v), at most 2^63 (so that v / sqrt(v) is 0 at 0)
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

constexpr unsigned long long kWaitNs = 2000000000;  // the longest wait inside a kernel
constexpr int kStages = 2;                          // a task's tile is used while the next one's arrives

// How a tile comes into shared memory, by the layout of all tensors (kCopy):
//   16  tensor-map copies (TMA), one of a warp's timesteps by 64 channels for
//       each tensor, counted by an mbarrier of the warp: rows at 16-byte steps
//       whose strides nest (see map_of).  One lane issues them; by 16-byte copies
//       of each lane staging took 6 of 50 instructions to a value.
//   4   asynchronous copies of 4 bytes (an even D, or 32-bit values)
//   2   value by value
// A warp brings in its own timesteps of a tile, [kSteps][64] of each of the
// first N tensors, and reads nothing else, so this needs no barrier of the
// block.  What is staged for timesteps past the stream's end and channels past
// D is used for nothing.
template <typename T, int kCopy, int kSteps, int N>
struct Loader {
  static constexpr int kOne = kWarps * kSteps * kLanes;           // values of one staged tensor
  static constexpr size_t kBytes = (size_t)N * kOne * sizeof(T);  // of a stage

  unsigned char* staged;
  uint64_t* bars;  // [kStages][kWarps]

  // Called by all threads, before a barrier of the block.
  __device__ __forceinline__ Loader(unsigned char* memory, uint64_t* barriers) : staged(memory), bars(barriers) {
    if constexpr (kCopy == 16) {
      if (threadIdx.x < kStages * kWarps) mbar_init(smem_u32(bars + threadIdx.x), 1);
      if (threadIdx.x < 32) fence_mbarrier_init_cluster();
    }
  }
  __device__ __forceinline__ T* part(int stage) const {  // this warp's timesteps of the first tensor
    return reinterpret_cast<T*>(staged + stage * kBytes) + (threadIdx.x >> 5) * kSteps * kLanes;
  }
  // The warp's timesteps from ts on, `rows` of them the stream's (any number), channels ch0 .. of stream b.
  template <typename Io>
  __device__ __forceinline__ void fetch(int stage, char* const* tensors, const Io& io, int ts, int b, int ch0, int rows,
                                        int cols) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    T* to = part(stage);
    if constexpr (kCopy == 16) {
      if (elect_one()) {
        const uint32_t bar = smem_u32(bars + stage * kWarps + warp);
        if (rows > 0) {
          mbar_arrive_expect_tx(bar, N * kSteps * kLanes * (int)sizeof(T));
#pragma unroll
          for (int m = 0; m < N; ++m) {
            const bool nested = io.stream_inner[m] != 0;
            tma_load_3d(smem_u32(to + m * kOne), io.maps + m, bar, ch0, nested ? b : ts, nested ? ts : b);
          }
        } else {
          mbar_arrive(bar);
        }
      }
      __syncwarp();
    } else {
      constexpr int kPer = kCopy == 4 ? 4 / (int)sizeof(T) : 1;  // values of a copy
      constexpr int kAcross = kLanes / kPer / 32;                // copies of a lane in a row
      if (rows > 0) {
#pragma unroll
        for (int m = 0; m < N; ++m) {
          const long long step = io.strides[m].t * (long long)sizeof(T);
          const char* from = tensors[m] + warp * kSteps * step;
          for (int s = 0; s < min(rows, kSteps); ++s, from += step) {
#pragma unroll
            for (int q = 0; q < kAcross; ++q) {
              const int col = (lane + 32 * q) * kPer;
              T* at = to + m * kOne + s * kLanes + col;
              const T* src = reinterpret_cast<const T*>(from) + col;
              if (col < cols) {
                if constexpr (kCopy == 4)
                  asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(smem_u32(at)), "l"(src) : "memory");
                else
                  *at = *src;
              }
            }
          }
        }
      }
      asm volatile("cp.async.commit_group;" ::: "memory");
    }
  }
  // Nothing more to fetch.
  __device__ __forceinline__ void skip() {
    if constexpr (kCopy != 16) asm volatile("cp.async.commit_group;" ::: "memory");
  }
  // Waits for the older of the two stages in flight; false if it does not come (then its values are not used).
  __device__ __forceinline__ bool wait(int stage, unsigned parity) {
    bool ok = true;
    if constexpr (kCopy == 16) {
      const int never = 0;
      ok = mbar_wait_bounded<false>(smem_u32(bars + stage * kWarps + (threadIdx.x >> 5)), parity, kWaitNs, &never);
    } else {
      asm volatile("cp.async.wait_group 1;" ::: "memory");
    }
    __syncwarp();
    return ok;
  }
};

__device__ __forceinline__ int length_of(const int* lengths, int b, int T) {
  return lengths ? min(max(lengths[b], 0), T) : T;
}

// Bit s: reset at timestep ts + s of this warp (the same in all lanes).
template <int kSteps>
__device__ __forceinline__ unsigned reset_bits(const unsigned char* reset, int ts, int len, int b, int B) {
  const int lane = threadIdx.x & 31, t = ts + lane;
  const bool on = lane < kSteps && t < len && reset[(long long)t * B + b] != 0;
  return __ballot_sync(0xffffffffu, on);
}

// ---- tasks and the exchange between tiles -----------------------------------

constexpr int kMaxGroup = 16;                       // tiles of a group
constexpr float kNaN = __builtin_nanf("");
constexpr unsigned kNotYet = 0xffffffffu;           // a word of the exchange before it is written

// One tile of 64 channels of one stream; `order` counts tiles in the direction of the scan.
struct Task {
  int slab, b, order;
};
struct Tasks {
  int T, B, D;
  int tile;          // timesteps of a tile
  int slabs, tiles;  // of a stream's channels, of the sequence (one at least)
  int group_log2;    // of the tiles of a group: a function of the shape
  long long count;   // slabs * B * tiles
};
// Shapes with few streams and channels have many tiles of one sequence in flight at once: their groups are as long as
// makes the tiles of one group of every sequence half as many again as the blocks of a wave (two to an SM); where there
// are more sequences than blocks a tile's predecessor is done long before.
inline Tasks tasks_of(int T, int B, int D, int steps) {
  const int tile = kWarps * steps;
  Tasks t{T, B, D, tile, (D + kLanes - 1) / kLanes, std::max(1, (T + tile - 1) / tile), 0, 0};
  const long long items = (long long)t.slabs * B;
  t.count = items * t.tiles;
  t.group_log2 = 0;
  while ((1 << t.group_log2) < kMaxGroup && items << t.group_log2 < 3 * 152) ++t.group_log2;
  return t;
}
// Tasks go round the blocks in the order slab (fastest), stream, tile.
__device__ __forceinline__ Task task_at(const Tasks& t, long long id) {
  return {(int)(id % t.slabs), (int)(id / t.slabs % t.B), (int)(id / t.slabs / t.B)};
}
// The task `step` (itself a task's place) further on.
__device__ __forceinline__ Task advance(const Tasks& t, Task at, Task step) {
  at.slab += step.slab;
  at.b += step.b;
  at.order += step.order;
  if (at.slab >= t.slabs) {
    at.slab -= t.slabs;
    ++at.b;
  }
  if (at.b >= t.B) {
    at.b -= t.B;
    ++at.order;
  }
  return at;
}

// A task's place in its group, and whether it is the last there.
__device__ __forceinline__ int place_of(const Tasks& t, const Task& at) { return at.order & ((1 << t.group_log2) - 1); }
__device__ __forceinline__ bool ends_group(const Tasks& t, const Task& at) {
  return place_of(t, at) == (1 << t.group_log2) - 1;
}

// What the block's warps need of a task, worked out by one of them two tasks ahead.
struct Plan {
  Task at;
  int len;              // of the stream
  char* tensors[7];     // the tile's first value in each tensor
};
// Tensors of a call as the kernels take them: N, the first M of which are read through tensor maps where they can be.
template <int N, int M>
struct Tensors {
  TcMap maps[M];
  int stream_inner[M];  // the map's middle axis is the stream, else the timestep
  char* base[N];
  Strides strides[N];
};
// Called by one warp (all its lanes).
template <typename T, int N, int M>
__device__ __forceinline__ void make_plan(Plan& plan, const Tasks& t, const Tensors<N, M>& tensors, const int* lengths,
                                          const Task& at, bool back) {
  const int lane = threadIdx.x & 31;
  if (at.order >= t.tiles) {
    if (lane == 0) plan.at = at;
    return;
  }
  const int tile = back ? t.tiles - 1 - at.order : at.order;
  if (lane < N) {
    const Strides& st = tensors.strides[lane];
    plan.tensors[lane] =
        tensors.base[lane] + (at.b * st.b + (long long)tile * t.tile * st.t + at.slab * kLanes) * (long long)sizeof(T);
  } else if (lane == N) {
    plan.at = at;
    plan.len = length_of(lengths, at.b, t.T);
  }
}

// The exchange in memory: c softplus(decay) [slabs * 64], then each tile's run [tiles][items][32] (16 bytes for a
// lane's two channels), then the state before each group but the first [groups - 1][items][32] (8 bytes).
struct Exchange {
  float* rate;
  ulonglong2* runs;
  uint64_t* states;
};
__host__ __device__ inline Exchange exchange_of(void* base, const Tasks& t) {
  Exchange e;
  e.rate = static_cast<float*>(base);
  e.runs = reinterpret_cast<ulonglong2*>(e.rate + (long long)t.slabs * kLanes);
  e.states = reinterpret_cast<uint64_t*>(e.runs + t.count * 32);
  return e;
}
inline size_t exchange_words(const Tasks& t) {  // of the runs and states (none for a single tile)
  if (t.tiles == 1) return 0;
  const long long items = (long long)t.slabs * t.B, groups = (t.tiles - 1) / (1 << t.group_log2) + 1;
  return (size_t)(t.count * 32 * 4 + (groups - 1) * items * 32 * 2);
}
inline size_t exchange_bytes(const Tasks& t) { return ((size_t)t.slabs * kLanes + exchange_words(t)) * 4; }

// Fills the exchange and forms the rates, once per call.
__global__ void __launch_bounds__(256) scan_prepare_kernel(const float* decay, float c, int D, int rates, float* rate,
                                                           uint4* fill, long long n) {
  begin_op();
  const long long i = (long long)blockIdx.x * blockDim.x + threadIdx.x;
  if (i < rates) rate[i] = i < D ? c * softplus_f(decay[i]) : 0.0f;
  for (long long k = i; k < n; k += (long long)gridDim.x * blockDim.x)
    fill[k] = make_uint4(kNotYet, kNotYet, kNotYet, kNotYet);
}

__device__ __forceinline__ unsigned as_result(unsigned w) { return w == kNotYet ? 0x7fffffffu : w; }
__device__ __forceinline__ void publish(uint64_t* p, uint64_t v) {
  asm volatile("st.relaxed.gpu.global.v2.u32 [%0], {%1, %2};" ::"l"(p), "r"(as_result((unsigned)v)),
               "r"(as_result((unsigned)(v >> 32)))
               : "memory");
}
__device__ __forceinline__ void publish(ulonglong2* p, ulonglong2 v) {
  asm volatile("st.relaxed.gpu.global.v4.u32 [%0], {%1, %2, %3, %4};" ::"l"(p), "r"(as_result((unsigned)v.x)),
               "r"(as_result((unsigned)(v.x >> 32))), "r"(as_result((unsigned)v.y)),
               "r"(as_result((unsigned)(v.y >> 32)))
               : "memory");
}
// Polls until every lane's words are there, or the wait has run out: then the pattern itself, a NaN, is returned.
template <typename F>
__device__ __forceinline__ void wait_for_words(F ready) {
  if (__all_sync(0xffffffffu, ready())) return;
  const unsigned long long t0 = global_timer_ns();
  while (!__all_sync(0xffffffffu, ready()))
    if (__any_sync(0xffffffffu, global_timer_ns() - t0 > kWaitNs)) return;
}
__device__ __forceinline__ uint64_t receive(const uint64_t* p) {
  unsigned a, b;
  wait_for_words([&] {
    asm volatile("ld.relaxed.gpu.global.v2.u32 {%0, %1}, [%2];" : "=r"(a), "=r"(b) : "l"(p) : "memory");
    return a != kNotYet && b != kNotYet;
  });
  return (uint64_t)b << 32 | a;
}
__device__ __forceinline__ ulonglong2 receive(const ulonglong2* p) {
  unsigned a, b, c, d;
  wait_for_words([&] {
    asm volatile("ld.relaxed.gpu.global.v4.u32 {%0, %1, %2, %3}, [%4];"
                 : "=r"(a), "=r"(b), "=r"(c), "=r"(d)
                 : "l"(p)
                 : "memory");
    return a != kNotYet && b != kNotYet && c != kNotYet && d != kNotYet;
  });
  return make_ulonglong2((uint64_t)b << 32 | a, (uint64_t)d << 32 | c);
}

// A run with a reset in it leads to U whatever the state before: its A (both channels') is -1, which no product of
// decays is.
template <bool kCuts>
__device__ __forceinline__ uint64_t after(ulonglong2 run, uint64_t h) {
  if (kCuts && (int)(unsigned)run.x < 0) h = 0ull;
  return fma2(run.x, h, run.y);
}
// The run of `first` and then `second`.
template <bool kCuts>
__device__ __forceinline__ ulonglong2 join(ulonglong2 first, ulonglong2 second) {
  const bool cut = kCuts && ((int)(unsigned)first.x < 0 || (int)(unsigned)second.x < 0);
  return make_ulonglong2(cut ? both(-1.0f) : mul2(first.x, second.x), after<kCuts>(second, first.y));
}

struct Join {                             // shared memory of a block
  ulonglong2 runs[2][kWarps][32];         // of the warps of a tile, by parity of the turn
  ulonglong2 before[kMaxGroup - 1][32];   // of the group's tiles before this one
  uint64_t start[32];                     // the state before the group
};

// Brings what a task needs from other tiles into shared memory, one run to a warp, and this tile's run out to them;
// `mine`: the warps' runs of this tile, in the direction of the scan from warp `w0` in steps of `dw`.  `first`: the
// state before the sequence, in warp 0 of its first tile, whose run it goes into: no other tile reads it, and what
// the sequence ends in follows from that run, so that the state may be overwritten by the sequence's last.  Returns
// this tile's run (without `first`) in warp 0.  The block meets in a barrier before and after.
template <bool kCuts>
__device__ __forceinline__ ulonglong2 exchange_runs(const Tasks& t, const Exchange& e, const Task& at, Join& sm,
                                                    const ulonglong2 (&mine)[kWarps][32], int w0, int dw, uint64_t first) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const long long items = (long long)t.slabs * t.B, item = (long long)at.b * t.slabs + at.slab;
  const int place = place_of(t, at), group = at.order >> t.group_log2;
  ulonglong2 all = make_ulonglong2(0ull, 0ull);
  if (warp == 0) {
    all = mine[w0][lane];
#pragma unroll
    for (int w = 1; w < kWarps; ++w) all = join<kCuts>(all, mine[w0 + dw * w][lane]);
    if (!ends_group(t, at) && at.order != t.tiles - 1)
      publish(e.runs + (at.order * items + item) * 32 + lane,
              at.order == 0 ? make_ulonglong2(all.x, after<kCuts>(all, first)) : all);
    if (group == 0) sm.start[lane] = first;
  }
  if (warp == kWarps - 1 && group > 0) sm.start[lane] = receive(e.states + ((group - 1) * items + item) * 32 + lane);
  for (int q = warp; q < place; q += kWarps)
    sm.before[q][lane] = receive(e.runs + ((long long)(at.order - place + q) * items + item) * 32 + lane);
  return all;
}
// The state before a tile, after exchange_runs and the barrier.
template <bool kCuts>
__device__ __forceinline__ uint64_t state_before(const Tasks& t, const Task& at, const Join& sm) {
  const int lane = threadIdx.x & 31, place = place_of(t, at);
  uint64_t h = sm.start[lane];
  for (int q = 0; q < place; ++q) h = after<kCuts>(sm.before[q][lane], h);
  return h;
}

struct ScanArgs {
  Tensors<4, 3> io;  // x, r, i, y
  const float* h0;
  const int* lengths;
  const unsigned char* reset;
  Tasks tasks;
  Exchange exchange;
  float* h_last;
  float* states;
};

__device__ __forceinline__ uint64_t load_f32x2(const float* p, int left) {
  if (left > 1 && (reinterpret_cast<uintptr_t>(p) & 7u) == 0) return *reinterpret_cast<const uint64_t*>(p);
  return f32x2(left > 0 ? p[0] : 0.0f, left > 1 ? p[1] : 0.0f);
}
__device__ __forceinline__ void store_f32x2(float* p, int left, uint64_t v) {
  if (left > 1 && (reinterpret_cast<uintptr_t>(p) & 7u) == 0) {
    *reinterpret_cast<uint64_t*>(p) = v;
    return;
  }
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
template <typename T, Reach kReach, int kSteps>
__device__ __forceinline__ void form_runs(const T* here, uint64_t rate, const Constants& k, uint64_t (&A)[kSteps],
                                          uint64_t (&U)[kSteps]) {
  constexpr int kOne = kWarps * kSteps * kLanes;  // values of one staged tensor
#pragma unroll
  for (int s = 0; s < kSteps; ++s) {
    const T* p = here + s * kLanes;
    const Gates g =
        gates_of<kReach>(staged_pair<T>(p + kOne), staged_pair<T>(p + 2 * kOne), rate, k);
    A[s] = g.a;
    const uint64_t m2 = m2_of(g.low, g.a, k);
    U[s] = mul2(mul2(mul2(m2, rsqrt2(m2)), g.si), staged_pair<T>(p));
  }
}

// The run of a warp's timesteps (kCuts: with resets at the set bits, one at least).
template <bool kCuts, int kSteps>
__device__ __forceinline__ ulonglong2 join_steps(const uint64_t (&A)[kSteps], const uint64_t (&U)[kSteps],
                                                 unsigned resets) {
  uint64_t PA = A[0], PU = U[0];
#pragma unroll
  for (int s = 1; s < kSteps; ++s) {
    if (kCuts && (resets >> s & 1u)) PU = 0ull;
    PU = fma2(A[s], PU, U[s]);
    PA = mul2(PA, A[s]);
  }
  return make_ulonglong2(kCuts ? both(-1.0f) : PA, PU);
}

// c softplus(decay) of a lane's channels, zero for one that does not exist.
__device__ __forceinline__ uint64_t rate_of(const float* decay, int left, float c) {
  return f32x2(left > 0 ? c * softplus_f(decay[0]) : 0.0f, left > 1 ? c * softplus_f(decay[1]) : 0.0f);
}
// How far -log a may be from zero in some lane, the same in all of them (kFar also for a NaN).  The kernels with resets
// know two cases only: with the code of all three, 2048 x 8 x 2048 bf16 both directions took 203 us for near decays
// instead of 199.
template <bool kCuts>
__device__ __forceinline__ Reach reach_of(uint64_t rate) {
  float r0, r1;
  f32x2_split(rate, r0, r1);
  if (!__any_sync(0xffffffffu, !(r0 <= kNearRate && r1 <= kNearRate))) return kNear;
  if (kCuts) return kFar;
  return __any_sync(0xffffffffu, !(r0 <= kMiddleRate && r1 <= kMiddleRate)) ? kFar : kMiddle;
}
// f(the reach as a constant)
template <bool kCuts, typename F>
__device__ __forceinline__ void with_reach(Reach reach, F f) {
  if (reach == kNear) f(std::integral_constant<Reach, kNear>());
  else if (!kCuts && reach == kMiddle) f(std::integral_constant<Reach, kMiddle>());
  else f(std::integral_constant<Reach, kFar>());
}

template <typename T, int kCopy, bool kCuts>
__global__ void __launch_bounds__(kWarps * 32, 2) gated_scan_kernel(const __grid_constant__ ScanArgs a) {
  extern __shared__ __align__(128) unsigned char staged[];
  __shared__ Join sm;
  __shared__ Plan plans[3];  // of this task and the next two
  __shared__ __align__(8) uint64_t bars[kStages * kWarps];
  constexpr bool kVec = kCopy >= 2 * (int)sizeof(T);  // a lane's two channels of y in one store
  constexpr int kSteps = kForwardSteps<T>;
  const Tasks& t = a.tasks;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  Loader<T, kCopy, kSteps, 3> loader(staged, bars);
  auto fetch = [&](int n, const Plan& plan) {
    const int ts = plan.at.order * t.tile + warp * kSteps, ch0 = plan.at.slab * kLanes;
    loader.fetch(n, plan.tensors, a.io, ts, plan.at.b, ch0, plan.len - ts, t.D - ch0);
  };
  const Task step = task_at(t, gridDim.x);
  Task ahead = advance(t, task_at(t, blockIdx.x), step);  // the furthest task with a plan
  if (warp == 2) {
    make_plan<T>(plans[0], t, a.io, a.lengths, task_at(t, blockIdx.x), false);
    make_plan<T>(plans[1], t, a.io, a.lengths, ahead, false);
  }
  __syncthreads();
  fetch(0, plans[0]);
  begin_op();
  const Constants k = constants();
  int turn = 0, now = 0;
  unsigned parity = 0;  // of the stage in use
  for (; plans[now].at.order < t.tiles; turn ^= 1) {
    const Plan &plan = plans[now], &next = plans[now == 2 ? 0 : now + 1];
    const Task at = plan.at;
    const uint64_t rate = *reinterpret_cast<const uint64_t*>(a.exchange.rate + at.slab * kLanes + 2 * lane);
    __syncwarp();  // the lanes are done with the stage that the next tile goes to
    if (next.at.order < t.tiles) fetch(turn ^ 1, next);
    else loader.skip();
    const int ch = at.slab * kLanes + 2 * lane, left = t.D - ch;  // channels of this lane that exist: min(left, 2)
    const int ts = at.order * t.tile + warp * kSteps, len = plan.len;
    const long long state_at = (long long)at.b * t.D + ch;
    const unsigned resets = kCuts ? reset_bits<kSteps>(a.reset, ts, len, at.b, t.B) : 0u;
    const bool whole = ts + kSteps <= len;
    uint64_t first = 0ull;
    if (warp == 0 && at.order == 0 && a.h0) first = load_f32x2(a.h0 + state_at, left);
    const T* here = loader.part(turn) + 2 * lane;
    const bool there = loader.wait(turn, parity);
    parity ^= turn;
    uint64_t A[kSteps], U[kSteps];
    if (ts < len) {
      with_reach<kCuts>(reach_of<kCuts>(rate), [&](auto reach) { form_runs<T, decltype(reach)::value>(here, rate, k, A, U); });
    }
    if (!whole) {
#pragma unroll
      for (int s = 0; s < kSteps; ++s)
        if (ts + s >= len) A[s] = k.one, U[s] = 0ull;
    }
    if (!there) U[0] = both(kNaN);
    sm.runs[turn][warp][lane] = kCuts && resets ? join_steps<true>(A, U, resets) : join_steps<false>(A, U, 0u);
    __syncthreads();
    const ulonglong2 tile = exchange_runs<kCuts>(t, a.exchange, at, sm, sm.runs[turn], 0, 1, first);
    if (warp == 2) {
      ahead = advance(t, ahead, step);
      make_plan<T>(plans[now == 0 ? 2 : now - 1], t, a.io, a.lengths, ahead, false);
    }
    __syncthreads();
    uint64_t h = state_before<kCuts>(t, at, sm);
    if (warp == 0) {
      const uint64_t end = after<kCuts>(tile, h);
      if (at.order == t.tiles - 1) store_f32x2(a.h_last + state_at, left, end);
      else if (ends_group(t, at))
        publish(a.exchange.states + ((long long)(at.order >> t.group_log2) * t.slabs * t.B + at.b * t.slabs + at.slab) * 32 + lane, end);
    }
#pragma unroll
    for (int w = 0; w < kWarps - 1; ++w) {
      const uint64_t to = after<kCuts>(sm.runs[turn][w][lane], h);
      if (w < warp) h = to;
    }
    if (a.states && ts % kChunk == 0 && ts < t.T)
      store_f32x2(a.states + (long long)(ts / kChunk) * t.B * t.D + state_at, left, h);
    if (kCuts && resets) {
#pragma unroll
      for (int s = 0; s < kSteps; ++s) {
        if (resets >> s & 1u) h = 0ull;
        h = U[s] = fma2(A[s], h, U[s]);
      }
    } else {
#pragma unroll
      for (int s = 0; s < kSteps; ++s) h = U[s] = fma2(A[s], h, U[s]);
    }
    if (left > 0) {
      const long long sy = a.io.strides[3].t;
      T* to = reinterpret_cast<T*>(plan.tensors[3]) + warp * kSteps * sy + 2 * lane;
      if (whole) {
#pragma unroll
        for (int s = 0; s < kSteps; ++s, to += sy) store_both<T, kVec>(to, left, U[s]);
      } else {
#pragma unroll
        for (int s = 0; s < kSteps; ++s, to += sy)
          if (ts + s < t.T) store_both<T, kVec>(to, left, ts + s < len ? U[s] : 0ull);
      }
    }
    now = now == 2 ? 0 : now + 1;
  }
}

struct ScanBackwardArgs {
  Tensors<7, 4> io;  // x, r, i, dy, dx, dr, di
  const float* dh_last;
  const float* states;
  const int* lengths;
  const unsigned char* reset;
  Tasks tasks;
  Exchange exchange;
  float* dh0;
  float* partial;  // [tiles][B][slabs * 64]: each tile's sum of E
};

// a_t (see held_decay), the gates and m_t sigma(i_t) x_t of a warp's staged timesteps.
template <typename T, Reach kReach, int kSteps>
__device__ __forceinline__ void form_gates(const T* here, uint64_t rate, const Constants& k, uint64_t (&held)[kSteps],
                                           uint64_t (&sr)[kSteps], uint64_t (&si)[kSteps], uint64_t (&U)[kSteps]) {
  constexpr int kOne = kWarps * kSteps * kLanes;
#pragma unroll
  for (int s = 0; s < kSteps; ++s) {
    const T* p = here + s * kLanes;
    const Gates g =
        gates_of<kReach>(staged_pair<T>(p + kOne), staged_pair<T>(p + 2 * kOne), rate, k);
    held[s] = held_decay<kReach>(g);
    sr[s] = g.sr;
    si[s] = g.si;
    const uint64_t m2 = m2_of(g.low, g.a, k);
    U[s] = mul2(mul2(mul2(m2, rsqrt2(m2)), g.si), staged_pair<T>(p));
  }
}

// The runs of a warp's timesteps, h -> A h + U forward and p -> A p + V back
// (staged dy is zero past the stream's length; kCuts: with a reset, one at least).
template <typename T, Reach kReach, bool kCuts, int kSteps>
__device__ __forceinline__ void join_both(const T* here, const uint64_t (&held)[kSteps], const uint64_t (&U)[kSteps],
                                          unsigned resets, const Constants& k, uint64_t& PA, uint64_t& PU, uint64_t& PV) {
#pragma unroll
  for (int s = 0; s < kSteps; ++s) {
    const uint64_t A = decay_of<kReach>(held[s], k);
    if (kCuts && (resets >> s & 1u)) PU = 0ull;
    PU = fma2(A, PU, U[s]);
    PA = mul2(PA, A);
  }
#pragma unroll
  for (int s = kSteps - 1; s >= 0; --s) {
    PV = mul2(decay_of<kReach>(held[s], k), add2(PV, staged_pair<T>(here + 3 * kWarps * kSteps * kLanes + s * kLanes)));
    if (kCuts && (resets >> s & 1u)) PV = 0ull;
  }
  if (kCuts) PA = both(-1.0f);
}

struct Gradients {
  uint64_t x, r, i, E;
};
// The gradients of the staged timestep at `here`, from p after it, which
// becomes p before it; h: the state before it.
template <typename T, Reach kReach>
__device__ __forceinline__ Gradients gradients_of(const T* here, uint64_t held, uint64_t sr, uint64_t si, uint64_t h,
                                                  uint64_t rate, const Constants& k, uint64_t& p) {
  const uint64_t A = decay_of<kReach>(held, k), xs = staged_pair<T>(here);
  const uint64_t g = add2(p, staged_pair<T>(here + 3 * kWarps * kBackwardSteps * kLanes));
  p = mul2(g, A);
  const uint64_t t = mul2(rate, sr);  // -log a
  const uint64_t m2 = m2_of(low_of<kReach>(held, t, k), A, k), inv_m = rsqrt2(m2);
  Gradients d;
  d.E = mul2(mul2(p, t), sub2(mul2(mul2(mul2(si, xs), A), inv_m), h));  // g a t (si x a / m - h)
  d.x = mul2(g, mul2(mul2(m2, inv_m), si));
  d.r = mul2(d.E, sub2(k.one, sr));
  d.i = mul2(mul2(d.x, xs), sub2(k.one, si));
  return d;
}

template <typename T, int kCopy, bool kCuts>
__global__ void __launch_bounds__(kWarps * 32, sizeof(T) == 4 ? 1 : 2) gated_scan_backward_kernel(const __grid_constant__ ScanBackwardArgs a) {
  extern __shared__ __align__(128) unsigned char staged[];
  __shared__ Join sm;                             // p -> A p + V
  __shared__ ulonglong2 ahead[2][kWarps][32];     // h -> A h + U
  __shared__ uint64_t sums[kWarps][32];           // E over each warp's timesteps of the last task
  __shared__ Plan plans[3];
  __shared__ __align__(8) uint64_t bars[kStages * kWarps];
  constexpr bool kVec = kCopy >= 2 * (int)sizeof(T);
  constexpr int kSteps = kBackwardSteps;
  constexpr int kOne = kWarps * kSteps * kLanes;
  const Tasks& t = a.tasks;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  Loader<T, kCopy, kSteps, 4> loader(staged, bars);
  auto fetch = [&](int n, const Plan& plan) {
    const int ts = (t.tiles - 1 - plan.at.order) * t.tile + warp * kSteps, ch0 = plan.at.slab * kLanes;
    loader.fetch(n, plan.tensors, a.io, ts, plan.at.b, ch0, plan.len - ts, t.D - ch0);
  };
  auto add_up = [&](const Task& at) {  // the sums of a finished task into its partial
    uint64_t v = sums[0][lane];
#pragma unroll
    for (int w = 1; w < kWarps; ++w) v = add2(v, sums[w][lane]);
    const long long row = (long long)(t.tiles - 1 - at.order) * t.B + at.b;
    *reinterpret_cast<uint64_t*>(a.partial + (row * t.slabs + at.slab) * kLanes + 2 * lane) = v;
  };
  const Task step = task_at(t, gridDim.x);
  Task done = task_at(t, blockIdx.x), ahead_task = advance(t, done, step);
  if (warp == 2) {
    make_plan<T>(plans[0], t, a.io, a.lengths, done, true);
    make_plan<T>(plans[1], t, a.io, a.lengths, ahead_task, true);
  }
  __syncthreads();
  fetch(0, plans[0]);
  begin_op();
  const Constants k = constants();
  int turn = 0, now = 0;
  unsigned parity = 0;
  bool any = false;
  for (; plans[now].at.order < t.tiles; turn ^= 1) {
    const Plan &plan = plans[now], &next = plans[now == 2 ? 0 : now + 1];
    const Task at = plan.at;
    const uint64_t rate = *reinterpret_cast<const uint64_t*>(a.exchange.rate + at.slab * kLanes + 2 * lane);
    __syncwarp();
    if (next.at.order < t.tiles) fetch(turn ^ 1, next);
    else loader.skip();
    const int tile = t.tiles - 1 - at.order;
    const int ch = at.slab * kLanes + 2 * lane, left = t.D - ch;
    const int ts = tile * t.tile + warp * kSteps, len = plan.len;
    const long long state_at = (long long)at.b * t.D + ch;
    const unsigned resets = kCuts ? reset_bits<kSteps>(a.reset, ts, len, at.b, t.B) : 0u;
    const bool whole = ts + kSteps <= len, some = ts < len;
    T* here = loader.part(turn) + 2 * lane;
    uint64_t first = 0ull;
    if (warp == 0 && at.order == 0 && a.dh_last) first = load_f32x2(a.dh_last + state_at, left);
    uint64_t h = some ? load_f32x2(a.states + (long long)tile * t.B * t.D + state_at, left) : 0ull;
    const bool there = loader.wait(turn, parity);
    parity ^= turn;
    const Reach reach = reach_of<kCuts>(rate);
    uint64_t held[kSteps], sr[kSteps], si[kSteps], U[kSteps], PA = k.one, PU = 0ull, PV = 0ull;
    if (some) {
      with_reach<kCuts>(reach, [&](auto at_most) { form_gates<T, decltype(at_most)::value>(here, rate, k, held, sr, si, U); });
      if (!whole) {
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
          if (ts + s >= len) {
            held[s] = reach == kFar ? k.one : 0ull;  // a = 1
            U[s] = 0ull;
            here[3 * kOne + s * kLanes] = here[3 * kOne + s * kLanes + 1] = from_f32<T>(0.0f);  // dy
          }
        }
        if (kCopy == 16) fence_proxy_async_shared();  // before a later bulk copy to the same place
      }
      if (!there) held[0] = both(kNaN);
      auto join = [&](auto at_most) {
        constexpr Reach kReach = decltype(at_most)::value;
        if (kCuts && resets) join_both<T, kReach, true>(here, held, U, resets, k, PA, PU, PV);
        else join_both<T, kReach, false>(here, held, U, 0u, k, PA, PU, PV);
      };
      if (reach == kFar) join(std::integral_constant<Reach, kFar>());
      else join(std::integral_constant<Reach, kMiddle>());
    }
    ahead[turn][warp][lane] = make_ulonglong2(PA, PU);
    sm.runs[turn][warp][lane] = make_ulonglong2(PA, PV);
    __syncthreads();
    if (warp == 1 && any) add_up(done);
    const ulonglong2 run = exchange_runs<kCuts>(t, a.exchange, at, sm, sm.runs[turn], kWarps - 1, -1, first);
    if (warp == 2) {
      ahead_task = advance(t, ahead_task, step);
      make_plan<T>(plans[now == 0 ? 2 : now - 1], t, a.io, a.lengths, ahead_task, true);
    }
#pragma unroll
    for (int w = 0; w < kWarps - 1; ++w) {
      const uint64_t to = after<kCuts>(ahead[turn][w][lane], h);
      if (w < warp) h = to;
    }
    __syncthreads();
    uint64_t p = state_before<kCuts>(t, at, sm);
    if (warp == 0) {
      const uint64_t end = after<kCuts>(run, p);
      if (at.order == t.tiles - 1) store_f32x2(a.dh0 + state_at, left, end);
      else if (ends_group(t, at))
        publish(a.exchange.states + ((long long)(at.order >> t.group_log2) * t.slabs * t.B + at.b * t.slabs + at.slab) * 32 + lane, end);
    }
#pragma unroll
    for (int w = kWarps - 1; w > 0; --w) {
      const uint64_t to = after<kCuts>(sm.runs[turn][w][lane], p);
      if (w > warp) p = to;
    }
    // the gradients' places at the warp's last timestep, from where the loops below go back
    const long long sx = a.io.strides[4].t, sr_t = a.io.strides[5].t, si_t = a.io.strides[6].t;
    const int last = warp * kSteps + kSteps - 1;
    T* to_x = reinterpret_cast<T*>(plan.tensors[4]) + last * sx + 2 * lane;
    T* to_r = reinterpret_cast<T*>(plan.tensors[5]) + last * sr_t + 2 * lane;
    T* to_i = reinterpret_cast<T*>(plan.tensors[6]) + last * si_t + 2 * lane;
    uint64_t sum = 0ull;
    auto gradients = [&](auto at_most) {
      constexpr Reach kReach = decltype(at_most)::value;
      // U becomes the state before each timestep
      if (kCuts && resets) {
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
          if (resets >> s & 1u) h = 0ull;
          const uint64_t u = U[s];
          U[s] = h;
          h = fma2(decay_of<kReach>(held[s], k), h, u);
        }
      } else {
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
          const uint64_t u = U[s];
          U[s] = h;
          h = fma2(decay_of<kReach>(held[s], k), h, u);
        }
      }
      if (whole && left > 0) {
#pragma unroll
        for (int s = kSteps - 1; s >= 0; --s) {
          const Gradients g = gradients_of<T, kReach>(here + s * kLanes, held[s], sr[s], si[s], U[s], rate, k, p);
          if (kCuts && (resets >> s & 1u)) p = 0ull;
          sum = add2(sum, g.E);
          store_both<T, kVec>(to_x, left, g.x);
          store_both<T, kVec>(to_r, left, g.r);
          store_both<T, kVec>(to_i, left, g.i);
          to_x -= sx;
          to_r -= sr_t;
          to_i -= si_t;
        }
      } else {
#pragma unroll
        for (int s = kSteps - 1; s >= 0; --s) {
          Gradients g = {0ull, 0ull, 0ull, 0ull};
          if (ts + s < len) g = gradients_of<T, kReach>(here + s * kLanes, held[s], sr[s], si[s], U[s], rate, k, p);
          if (kCuts && (resets >> s & 1u)) p = 0ull;
          sum = add2(sum, g.E);
          if (left > 0 && ts + s < t.T) {
            store_both<T, kVec>(to_x, left, g.x);
            store_both<T, kVec>(to_r, left, g.r);
            store_both<T, kVec>(to_i, left, g.i);
          }
          to_x -= sx;
          to_r -= sr_t;
          to_i -= si_t;
        }
      }
    };
    if (some) {
      if (reach == kFar) gradients(std::integral_constant<Reach, kFar>());
      else gradients(std::integral_constant<Reach, kMiddle>());
    } else if (left > 0) {
      for (int s = kSteps - 1; s >= 0; --s, to_x -= sx, to_r -= sr_t, to_i -= si_t) {
        if (ts + s >= t.T) continue;
        store_pair<T, kVec>(to_x, left, 0.0f, 0.0f);
        store_pair<T, kVec>(to_r, left, 0.0f, 0.0f);
        store_pair<T, kVec>(to_i, left, 0.0f, 0.0f);
      }
    }
    sums[warp][lane] = sum;
    done = at;
    any = true;
    now = now == 2 ? 0 : now + 1;
  }
  __syncthreads();
  if (warp == 1 && any) add_up(done);
}

// ddecay from partial [n][pitch], summed in a fixed order.
__global__ void __launch_bounds__(1024) decay_gradient_kernel(const float* partial, int n, int pitch, int D,
                                                              const float* decay, float* ddecay) {
  begin_op();
  __shared__ float acc[32][33];
  const int col = blockIdx.x * 32 + threadIdx.x;
  float v = 0.0f;
  if (col < D) {
#pragma unroll 4
    for (int k = threadIdx.y; k < n; k += 32) v += partial[(long long)k * pitch + col];
  }
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

// One timestep: a thread takes a pair of channels of kRows streams, all of whose values it asks for before it forms the
// decays' rates, which cost more than a stream's timestep.  (One stream to a thread: 1000 x 2048 in 10.3 us, bound by
// the rates.)
template <typename T, bool kVec, int kRows>
__global__ void __launch_bounds__(256) gated_step_kernel(const StepArgs a) {
  begin_op();
  const int ch = 2 * (blockIdx.x * blockDim.x + threadIdx.x), left = a.D - ch;
  if (left <= 0) return;
  // (unsigned: the last of 2^31 - 1 streams and a turn of all blocks further on)
  for (unsigned b0 = blockIdx.y * kRows; b0 < (unsigned)a.B; b0 += gridDim.y * kRows) {
    float2 x[kRows], r[kRows], i[kRows];
    uint64_t h[kRows];
    int slot[kRows];
#pragma unroll
    for (int n = 0; n < kRows; ++n) {
      const unsigned b = b0 + n;
      slot[n] = b >= (unsigned)a.B ? -1 : (a.slots ? a.slots[b] : (int)b);
    }
#pragma unroll
    for (int n = 0; n < kRows; ++n) {
      const long long b = b0 + n;
      if (slot[n] < 0 || slot[n] >= a.n_slots) continue;
      x[n] = load_pair<T, kVec>(static_cast<const T*>(a.x) + b * a.x_pitch + ch, left);
      r[n] = load_pair<T, kVec>(static_cast<const T*>(a.r) + b * a.r_pitch + ch, left);
      i[n] = load_pair<T, kVec>(static_cast<const T*>(a.i) + b * a.i_pitch + ch, left);
      h[n] = load_f32x2(a.state + (long long)slot[n] * a.D + ch, left);
      if (a.reset && a.reset[b] != 0) h[n] = 0ull;
    }
    const uint64_t rate = rate_of(a.decay + ch, left, a.c);
    const Constants k = constants();
#pragma unroll
    for (int n = 0; n < kRows; ++n) {
      const unsigned b = b0 + n;
      if (b >= (unsigned)a.B) continue;
      T* y = static_cast<T*>(a.y) + (long long)b * a.D + ch;
      if (slot[n] < 0 || slot[n] >= a.n_slots) {
        store_pair<T, kVec>(y, left, 0.0f, 0.0f);
        continue;
      }
      const Gates g = gates_of<kFar>(f32x2(r[n].x, r[n].y), f32x2(i[n].x, i[n].y), rate, k);
      const uint64_t m2 = m2_of(g.low, g.a, k);
      const uint64_t after = fma2(g.a, h[n], mul2(mul2(mul2(m2, rsqrt2(m2)), g.si), f32x2(x[n].x, x[n].y)));
      store_f32x2(a.state + (long long)slot[n] * a.D + ch, left, after);
      store_both<T, kVec>(y, left, after);
    }
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
  if (T < 0 || B < 0 || D < 1 || D > 0x7fffff00 || T > 0x7fffff00 ||
      (double)B * ((D + kLanes - 1) / kLanes) * (T / kChunk + 1) > 2147483647.0)
    return op_report(msg, msg_len, LSTM_APPROX_EINVAL, "need T, B >= 0, D >= 1 and fewer than 2^31 tiles of 64 x 64 values");
  if (!(c > 0.0f)) return op_report(msg, msg_len, LSTM_APPROX_EINVAL, "c must be positive");
  return LSTM_APPROX_OK;
}

template <typename T, int kCopy, bool kCuts, int kTensors, int kSteps, typename A>
cudaError_t launch_scan(void (*kern)(const A), cudaStream_t s, const A& args) {
  static thread_local DeviceSet ready;  // of the one kernel that this instance launches
  static thread_local int resident[64];
  constexpr size_t smem = kStages * Loader<T, kCopy, kSteps, kTensors>::kBytes;
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e == cudaSuccess && dev >= 64) e = cudaErrorInvalidDevice;
  if (e != cudaSuccess) return e;
  e = once_per_device(&ready, [&] {
    cudaError_t e1 = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    int per = 0, sms = 0;
    if (e1 == cudaSuccess) e1 = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per, kern, kWarps * 32, smem);
    if (e1 == cudaSuccess) e1 = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
    resident[dev] = per * sms;
    return e1;
  });
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)std::min<long long>(args.tasks.count, resident[dev]));
  cfg.blockDim = dim3(kWarps * 32);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;  // the first tiles are on their way meanwhile
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeCooperative;  // all blocks at once: they wait for one another's tiles
  attr[1].val.cooperative = 1;
  cfg.attrs = attr;
  cfg.numAttrs = args.tasks.tiles > 1 ? 2 : 1;  // (a single tile waits for none)
  return cudaLaunchKernelEx(&cfg, kern, args);
}

cudaError_t launch_prepare(const float* decay, float c, const Tasks& t, const Exchange& e, cudaStream_t s) {
  const long long fill = (long long)(exchange_words(t) / 4), rates = (long long)t.slabs * kLanes;
  const long long blocks = std::max((rates + 255) / 256, std::min<long long>((fill + 1023) / 1024, 4 * 152));
  return op_launch(scan_prepare_kernel, dim3((unsigned)blocks), dim3(256), 0, s, decay, c, t.D, (int)rates, e.rate,
                   reinterpret_cast<uint4*>(e.runs), fill);
}

// Exchange, then the backward pass's partial sums.
size_t workspace_bytes_of(const Tasks& t) {
  return (exchange_bytes(t) + (size_t)t.tiles * t.B * t.slabs * kLanes * sizeof(float) + 15) / 16 * 16 + 16;
}

// The tensor map of one tensor [T][B][D], its copies 64 channels by `steps` timesteps of one stream.  The axes go by
// size of their strides, which have to be multiples of one another with no overlap (a size of 1 has any stride).
bool map_of(TcMap* map, int* stream_inner, const void* p, int dtype, int T, int B, int D, const Strides& st, int steps) {
  const long long es = (long long)op_dtype_bytes(dtype), row = (long long)D * es;
  long long b = st.b * es, t = st.t * es;
  *stream_inner = T == 1 || (B > 1 && b <= t);
  if (B == 1) b = T == 1 ? row : t * T;
  if (T == 1) t = b * B;
  const long long in = *stream_inner ? b : t, out = *stream_inner ? t : b;
  if (in < row || out % in != 0 || out < in * (*stream_inner ? B : T) || out >= 1ll << 40) return false;
  return tc_make_map_steps(map, p, es == 4, D, *stream_inner ? B : T, *stream_inner ? T : B, in, out,
                           *stream_inner ? 1 : steps, *stream_inner ? steps : 1);
}

// The tensors, and the kernels' kCopy for them.
template <int N, int M>
int set_tensors(Tensors<N, M>& io, const void* const (&p)[N], const Strides* st, int dtype, int T, int B, int D, int steps) {
  const size_t es = op_dtype_bytes(dtype);
  int copy = T > 0 ? copy_bytes(D, es, p, st, N) : 4;
  for (int n = 0; n < N; ++n) {
    io.base[n] = static_cast<char*>(const_cast<void*>(p[n]));
    io.strides[n] = st[n];
  }
  for (int m = 0; m < M && copy == 16; ++m)
    if (!map_of(&io.maps[m], &io.stream_inner[m], p[m], dtype, T, B, D, st[m], steps)) copy = 4;
  return copy;
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

extern "C" size_t lstm_approx_gated_scan_workspace_bytes(int T, int B, int D) {
  if (check_sizes(LSTM_APPROX_OP_FP32, T, B, D, 1.0f, nullptr, 0)) return 0;
  return workspace_bytes_of(tasks_of(T, B, D, kBackwardSteps));  // (forward: as many tiles or half, no partial sums)
}

extern "C" int lstm_approx_gated_scan(int dtype, const void* x, const void* r, const void* i, const float* decay,
                                      float c, const float* h0, const int32_t* lengths, const unsigned char* reset,
                                      int T, int B, int D, void* y, const long long* strides, float* h_last,
                                      float* states, void* workspace, size_t workspace_bytes, void* cuda_stream,
                                      char* msg, int msg_len) {
  if (msg && msg_len > 0) msg[0] = '\0';
  if (int rc = check_sizes(dtype, T, B, D, c, msg, msg_len)) return rc;
  if (B > 0 && (!decay || !h_last || !workspace || (T > 0 && (!x || !r || !i || !y))))
    return op_report(msg, msg_len, LSTM_APPROX_EINVAL, "x, r, i, decay, y, h_last and workspace must not be NULL");
  const size_t es = op_dtype_bytes(dtype);
  if (!op_aligned(x, es) || !op_aligned(r, es) || !op_aligned(i, es) || !op_aligned(y, es) || !op_aligned(decay, 4) ||
      !op_aligned(h0, 4) || !op_aligned(lengths, 4) || !op_aligned(h_last, 4) || !op_aligned(states, 4))
    return op_report(msg, msg_len, LSTM_APPROX_EINVAL, "a pointer is not aligned to its type");
  Strides st[4];
  if (!read_strides(strides, 4, B, D, st))
    return op_report(msg, msg_len, LSTM_APPROX_EINVAL, "strides must not be negative");
  const Tasks tasks = tasks_of(T, B, D, dtype == LSTM_APPROX_OP_FP32 ? kForwardSteps<float> : kForwardSteps<__half>);
  const size_t need = lstm_approx_gated_scan_workspace_bytes(T, B, D);
  if (B > 0 && (!op_aligned(workspace, 16) || workspace_bytes < need))
    return op_report(msg, msg_len, LSTM_APPROX_EINVAL, "needs a 16-byte aligned workspace of %zu bytes", need);
  if (int rc = op_check_device(msg, msg_len)) return rc;
  if (B == 0) return LSTM_APPROX_OK;
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  const Exchange exchange = exchange_of(workspace, tasks);
  cudaError_t e = launch_prepare(decay, c, tasks, exchange, s);
  if (int rc = op_launched(e, "scan preparation launch", msg, msg_len)) return rc;
  const void* tensors[4] = {x, r, i, y};
  ScanArgs a{{}, h0, lengths, reset, tasks, exchange, h_last, states};
  const int copy = set_tensors(a.io, tensors, st, dtype, T, B, D, tasks.tile / kWarps);
  e = op_for_type(dtype, [&](auto* t) {
    using E = std::remove_pointer_t<decltype(t)>;
    auto go = [&](auto bytes) {
      constexpr int kCopy = decltype(bytes)::value;
      return reset ? launch_scan<E, kCopy, true, 3, kForwardSteps<E>>(gated_scan_kernel<E, kCopy, true>, s, a)
                   : launch_scan<E, kCopy, false, 3, kForwardSteps<E>>(gated_scan_kernel<E, kCopy, false>, s, a);
    };
    if (copy == 16) return go(std::integral_constant<int, 16>());
    if (copy == 4) return go(std::integral_constant<int, 4>());
    return go(std::integral_constant<int, sizeof(E) == 4 ? 4 : 2>());  // 32-bit values are always copied
  });
  return op_launched(e, "scan launch", msg, msg_len);
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
  const Tasks tasks = tasks_of(T, B, D, kBackwardSteps);
  const size_t need = lstm_approx_gated_scan_workspace_bytes(T, B, D);
  if (!op_aligned(workspace, 16) || workspace_bytes < need)
    return op_report(msg, msg_len, LSTM_APPROX_EINVAL, "needs a 16-byte aligned workspace of %zu bytes", need);
  if (int rc = op_check_device(msg, msg_len)) return rc;
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  const Exchange exchange = exchange_of(workspace, tasks);
  float* partial = reinterpret_cast<float*>(static_cast<char*>(workspace) + exchange_bytes(tasks));
  if (B > 0) {
    cudaError_t e = launch_prepare(decay, c, tasks, exchange, s);
    if (int rc = op_launched(e, "scan preparation launch", msg, msg_len)) return rc;
    const void* tensors[7] = {x, r, i, dy, dx, dr, di};
    const Strides order[7] = {st[1], st[2], st[3], st[0], st[4], st[5], st[6]};
    ScanBackwardArgs a{{}, dh_last, states, lengths, reset, tasks, exchange, dh0, partial};
    const int copy = set_tensors(a.io, tensors, order, dtype, T, B, D, tasks.tile / kWarps);
    e = op_for_type(dtype, [&](auto* t) {
      using E = std::remove_pointer_t<decltype(t)>;
      auto go = [&](auto bytes) {
        constexpr int kCopy = decltype(bytes)::value;
        return reset ? launch_scan<E, kCopy, true, 4, kBackwardSteps>(gated_scan_backward_kernel<E, kCopy, true>, s, a)
                     : launch_scan<E, kCopy, false, 4, kBackwardSteps>(gated_scan_backward_kernel<E, kCopy, false>, s, a);
      };
      if (copy == 16) return go(std::integral_constant<int, 16>());
      if (copy == 4) return go(std::integral_constant<int, 4>());
      return go(std::integral_constant<int, sizeof(E) == 4 ? 4 : 2>());
    });
    if (int rc = op_launched(e, "scan backward launch", msg, msg_len)) return rc;
  }
  const cudaError_t e = op_launch(decay_gradient_kernel, dim3((D + 31) / 32), dim3(32, 32), 0, s,
                                  static_cast<const float*>(partial), tasks.tiles * B, tasks.slabs * kLanes, D, decay,
                                  ddecay);
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
  const int threads = D >= 512 ? 256 : 64, across = (D - 1) / (2 * threads) + 1;
  // one stream to a thread while that leaves no SM with more than 8 blocks
  const bool many = (long long)across * B > 8 * 152;
  const dim3 grid(across, std::min(many ? (B - 1) / 4 + 1 : B, 65535));
  const cudaError_t e = op_for_type(dtype, [&](auto* t) {
    using E = std::remove_pointer_t<decltype(t)>;
    auto kern = vec ? (many ? gated_step_kernel<E, true, 4> : gated_step_kernel<E, true, 1>)
                    : (many ? gated_step_kernel<E, false, 4> : gated_step_kernel<E, false, 1>);
    return op_launch(kern, grid, dim3(threads), 0, static_cast<cudaStream_t>(cuda_stream), a);
  });
  return op_launched(e, "step launch", msg, msg_len);
}
