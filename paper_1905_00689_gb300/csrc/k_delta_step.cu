// One timestep of the gated delta rule on a pool of matrix states
// (include/lstm_approx_ops.h).
//
//   W = e^g S;  u = beta (v - W^T k);  S = W + k u^T
//   o = scale S^T q = scale (W^T q + (k . q) u)
//
// Bound by memory: the state is read and written once.  The second form of o
// needs W only, so that both sums over Dk (with k and with q) come from one pass
// over values that stay in registers until they are written back.  The columns of
// S do not see one another: a block takes 32 of them, a thread 4 (16 bytes) of
// every 16th row, all of them asked for at once.
//
// Measured, 16 heads of 128 x 128: 64 streams 24.9 us (80% of the 6790 GB/s of a
// copy), one stream 5.6 us a call, the time of a launch.
#include "ops_common.cuh"

namespace lstm_approx_impl {
namespace {

constexpr int kThreads = 128, kColumns = 32, kRowGroups = 16;
constexpr float kLeastG = -200.0f;

struct StepArgs {
  const void *q, *k, *v;
  const float *g, *beta;
  float scale;
  float* state;
  int n_slots;
  const int32_t* slots;
  const unsigned char* reset;
  int H, share, Dk, Dv, column_tiles;
  void* o;
  long long qb, qh, kb, kh, vb, vh, ob, oh, gb, bb;
};

// kRows: rows of S to a thread, at most (Dk <= 16 kRows).  kWide: rows of S at 16-byte boundaries, 4 neighbouring columns
// to a thread; else 4 columns that lie 8 apart.
template <typename T, int kRows, bool kWide>
__global__ void __launch_bounds__(kThreads) delta_step_kernel(const StepArgs a) {
  __shared__ float sums[4][8][9];
  begin_op();
  const int tile = blockIdx.x % a.column_tiles, bh = blockIdx.x / a.column_tiles, h = bh % a.H, b = bh / a.H;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, quad = lane & 7;
  const int row0 = warp * 4 + (lane >> 3);
  auto column = [&](int e) { return tile * kColumns + (kWide ? quad * 4 + e : quad + 8 * e); };
  const int slot = a.slots ? a.slots[b] : b;
  T* o = static_cast<T*>(a.o) + b * a.ob + h * a.oh;
  if (slot < 0 || slot >= a.n_slots) {
    if (threadIdx.x < 8)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (column(e) < a.Dv) o[column(e)] = from_f32<T>(0.0f);
    return;
  }
  float* S = a.state + ((long long)slot * a.H + h) * a.Dk * a.Dv;
  const T* q = static_cast<const T*>(a.q) + b * a.qb + (h / a.share) * a.qh;
  const T* k = static_cast<const T*>(a.k) + b * a.kb + (h / a.share) * a.kh;
  const bool fresh = a.reset && a.reset[b];
  // At a reset g may be anything.  (Left out here, where it is asked for: 16.6 us for 64 streams whose states lie in L2; left out
  // where the decay is made, 18.5.)
  const float g = fresh ? 0.0f : a.g[b * a.gb + h], beta = a.beta[b * a.bb + h];

  float w[kRows][4], kr[kRows], qr[kRows];
#pragma unroll
  for (int i = 0; i < kRows; ++i) {
    const int row = row0 + i * kRowGroups;
    const float* s = S + (long long)row * a.Dv;
    if constexpr (kWide) {
      float4 x = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
      if (row < a.Dk && column(0) < a.Dv && !fresh) x = *reinterpret_cast<const float4*>(s + column(0));
      w[i][0] = x.x, w[i][1] = x.y, w[i][2] = x.z, w[i][3] = x.w;
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) w[i][e] = row < a.Dk && column(e) < a.Dv && !fresh ? s[column(e)] : 0.0f;
    }
    kr[i] = row < a.Dk ? to_f32(k[row]) : 0.0f;
    qr[i] = row < a.Dk ? to_f32(q[row]) : 0.0f;
  }
  float vc[4];
#pragma unroll
  for (int e = 0; e < 4; ++e)
    vc[e] = column(e) < a.Dv ? to_f32(static_cast<const T*>(a.v)[b * a.vb + h * a.vh + column(e)]) : 0.0f;

  const float decay = expf(g < kLeastG ? kLeastG : g);
  float part[9] = {};  // W^T k and W^T q of 4 columns, k . q
#pragma unroll
  for (int i = 0; i < kRows; ++i) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      w[i][e] *= decay;
      part[e] = fmaf(w[i][e], kr[i], part[e]);
      part[4 + e] = fmaf(w[i][e], qr[i], part[4 + e]);
    }
    part[8] = fmaf(kr[i], qr[i], part[8]);
  }
#pragma unroll
  for (int j = 0; j < 9; ++j) {
    part[j] += __shfl_xor_sync(0xffffffffu, part[j], 8);
    part[j] += __shfl_xor_sync(0xffffffffu, part[j], 16);
    if (lane < 8) sums[warp][quad][j] = part[j];
  }
  __syncthreads();
#pragma unroll
  for (int j = 0; j < 9; ++j) part[j] = sums[0][quad][j] + sums[1][quad][j] + sums[2][quad][j] + sums[3][quad][j];

  float u[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) u[e] = beta * (vc[e] - part[e]);
#pragma unroll
  for (int i = 0; i < kRows; ++i) {
    const int row = row0 + i * kRowGroups;
    float* s = S + (long long)row * a.Dv;
#pragma unroll
    for (int e = 0; e < 4; ++e) w[i][e] = fmaf(kr[i], u[e], w[i][e]);
    if (row >= a.Dk) continue;
    if constexpr (kWide) {
      if (column(0) < a.Dv) *reinterpret_cast<float4*>(s + column(0)) = make_float4(w[i][0], w[i][1], w[i][2], w[i][3]);
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (column(e) < a.Dv) s[column(e)] = w[i][e];
    }
  }
  if (threadIdx.x < 8)
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (column(e) < a.Dv) o[column(e)] = from_f32<T>(a.scale * fmaf(part[8], u[e], part[4 + e]));
}

}  // namespace
}  // namespace lstm_approx_impl

using namespace lstm_approx_impl;

extern "C" int lstm_approx_delta_step(int dtype, const void* q, const void* k, const void* v, const float* g,
                                      const float* beta, float scale, float* state, int n_slots, const int32_t* slots,
                                      const unsigned char* reset, int B, int H, int Hk, int Dk, int Dv, void* o,
                                      const long long* strides, void* cuda_stream, char* msg, int msg_len) {
  if (msg && msg_len > 0) msg[0] = '\0';
  if (!op_float_dtype(dtype)) return op_report(msg, msg_len, LSTM_APPROX_EINVAL, "dtype %d", dtype);
  if (int rc = delta_check_sizes(1, B, H, Hk, Dk, Dv, msg, msg_len)) return rc;
  if (n_slots < 0 || (!slots && n_slots < B))
    return op_report(msg, msg_len, LSTM_APPROX_EINVAL, "without slots every stream needs a row of state");
  const long long tiles = (Dv + kColumns - 1) / kColumns, blocks = (long long)B * H * tiles;
  if (blocks > 0x7fffffffll) return op_report(msg, msg_len, LSTM_APPROX_EINVAL, "B H ceil(Dv / 32) must be below 2^31");
  if (blocks > 0 && (!q || !k || !v || !g || !beta || !o || (n_slots > 0 && !state)))
    return op_report(msg, msg_len, LSTM_APPROX_EINVAL, "q, k, v, g, beta, state and o must not be NULL");
  const size_t es = op_dtype_bytes(dtype);
  if (!op_aligned(q, es) || !op_aligned(k, es) || !op_aligned(v, es) || !op_aligned(o, es) || !op_aligned(g, 4) ||
      !op_aligned(beta, 4) || !op_aligned(state, 4) || !op_aligned(slots, 4))
    return op_report(msg, msg_len, LSTM_APPROX_EINVAL, "a pointer not aligned to its type");
  const long long dense[10] = {(long long)Hk * Dk, Dk, (long long)Hk * Dk, Dk, (long long)H * Dv, Dv, (long long)H * Dv, Dv, H, H};
  const long long* p = strides ? strides : dense;
  for (int i = 0; i < 10; ++i)
    if (p[i] < 0) return op_report(msg, msg_len, LSTM_APPROX_EINVAL, "strides must not be negative");
  if (int rc = op_check_device(msg, msg_len)) return rc;
  if (blocks == 0) return LSTM_APPROX_OK;
  const StepArgs a{q, k, v, g, beta, scale, state, n_slots, slots, reset, H, H / Hk, Dk, Dv, (int)tiles, o,
                   p[0], p[1], p[2], p[3], p[4], p[5], p[6], p[7], p[8], p[9]};
  const bool wide = Dv % 4 == 0 && op_aligned(state, 16);
  const cudaError_t e = op_for_type(dtype, [&](auto* t) {
    using T = std::remove_pointer_t<decltype(t)>;
    auto kern = Dk <= 64 ? (wide ? delta_step_kernel<T, 4, true> : delta_step_kernel<T, 4, false>)
                         : (wide ? delta_step_kernel<T, 8, true> : delta_step_kernel<T, 8, false>);
    return op_launch(kern, dim3((unsigned)blocks), dim3(kThreads), 0, static_cast<cudaStream_t>(cuda_stream), a);
  });
  return op_launched(e, "delta step launch", msg, msg_len);
}
