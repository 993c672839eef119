// Gated delta rule: one decoding step on cached states,
//     u = b (v - a H^T k)      H <- a H + k u^T      y = s H^T q = s (a H^T q + (q . k) u)
// (q, k divided by their lengths if asked).  Bound by the state's bytes, read once and written once: both products with
// the old state come from one pass over it, held in registers, and y needs no second one.
//
// A unit is one (b, n).  A lane holds 16 bytes of a row (4 or 8 columns), so L = V / 4 or V / 8 lanes share a row and
// a warp takes 32 / L rows at a time; sixteen 16-byte loads of a lane are in flight at once (fewer where the state is
// smaller).  W warps share a unit: the sums over rows go through shuffles, then (W > 1) through shared memory.  Everything
// is fp32, whatever the types in memory.
// 512 rows of 32 bf16 states of 128 x 128: 198 us, 5.4 TB/s; 48 rows of 84 fp32 states of 64 x 16: 7.1 us (4.7 TB/s with the launch);
// one row of these: 3.9 us, a launch and a memory round trip.
#include "delta_common.cuh"

namespace m2rnn {
namespace {

// 16 bytes of a state, as they lie in memory, and as floats
template <typename TS> struct Vec16;
template <> struct Vec16<float> {
  static constexpr int n = 4;
  __device__ static void open(const uint4 &r, float (&x)[4]) {
    x[0] = __uint_as_float(r.x); x[1] = __uint_as_float(r.y); x[2] = __uint_as_float(r.z); x[3] = __uint_as_float(r.w);
  }
  __device__ static uint4 close(const float (&x)[4]) { return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3])); }
};
template <> struct Vec16<__nv_bfloat16> {
  static constexpr int n = 8;
  __device__ static void open(const uint4 &r, float (&x)[8]) {
    const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { const float2 f = unpack_bf16(w[i]); x[2 * i] = f.x; x[2 * i + 1] = f.y; }
  }
  __device__ static uint4 close(const float (&x)[8]) { return make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7])); }
};

// R: 16-byte pieces of a lane, most; W warps to a unit, kWarps to a CTA
template <typename TIO, typename TS, int V, int R, int kWarps>
__global__ void __launch_bounds__(32 * kWarps, (R > 8 ? 16 : sizeof(TS) == 2 ? 32 : 28) / kWarps) delta_step_kernel(DeltaStepArgs a, int W) {
  using X = Vec16<TS>;
  constexpr int E = X::n, L = V / E, G = 32 / L;     // lanes to a row, rows of a warp at a time
  __shared__ float part[kWarps][2][V];               // sums over a warp's rows; then [unit's first warp][0]: u
  __shared__ float ksm[kWarps][128], qsm[kWarps][128];
  begin_dependent();
  const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31, col = (lane % L) * E;
  const int unit0 = warp / W, sub = warp % W;        // the CTA's unit, this warp's share of it
  const long long unit = (long long)blockIdx.x * (kWarps / W) + unit0;
  const int K = a.K, N = a.N;
  const bool in = unit < (long long)a.B * N;
  const int b = in ? (int)(unit / N) : 0, n = in ? (int)(unit % N) : 0;
  const size_t bn = (size_t)b * N + n;
  int slot = b;
  if (a.slots && in) slot = a.slots[b];
  // what does not hang on the slot is asked for first
  const TIO *kg = static_cast<const TIO *>(a.k) + ((size_t)b * a.Nk + n / (N / a.Nk)) * K, *qg = static_cast<const TIO *>(a.q) + ((size_t)b * a.Nq + n / (N / a.Nq)) * K;
  float kx[4] = {}, qx[4] = {};
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (in && lane + 32 * i < K) { kx[i] = to_f32(kg[lane + 32 * i]); qx[i] = to_f32(qg[lane + 32 * i]); }
  const float gate = in ? to_f32(static_cast<const TIO *>(a.gate)[bn]) : 0.f, step_in = in ? to_f32(static_cast<const TIO *>(a.step)[bn]) : 0.f;
  const bool psi = a.gate_kind == M2RNN_GATE_PSI;
  const float alpha = psi && in ? a.alpha[n] : 1.f, beta = psi && in ? a.beta[n] : 0.f;
  // a negative slot is a padding row: no state, y = 0.  One outside the pool is reported.
  const bool live = in && slot >= 0 && slot < a.nslots;
  if (in && slot >= a.nslots && a.dev_status && lane == 0) atomicExch(a.dev_status, (int32_t)M2RNN_ERR_SHAPE);
  const int per = K / (G * W), row0 = sub * per * G + lane / L;      // this lane's rows: row0 + r G
  TS *st = static_cast<TS *>(a.state) + ((size_t)(live ? slot : 0) * N + n) * K * V + (size_t)row0 * V + col;
  uint4 H[R];
  if (live) {
#pragma unroll
    for (int r = 0; r < R; ++r)
      if (r < per) H[r] = __ldcs(reinterpret_cast<const uint4 *>(st + (size_t)(r * G) * V));
  }
  // q and k of the unit: every warp keeps its own copy in shared memory
  float kk = 0.f, qq = 0.f, qk = 0.f;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (lane + 32 * i < K) { ksm[warp][lane + 32 * i] = kx[i]; qsm[warp][lane + 32 * i] = qx[i]; }
    kk = fmaf(kx[i], kx[i], kk);
    qq = fmaf(qx[i], qx[i], qq);
    qk = fmaf(qx[i], kx[i], qk);
  }
#pragma unroll
  for (int d = 16; d; d /= 2) {
    kk += __shfl_xor_sync(0xffffffffu, kk, d);
    qq += __shfl_xor_sync(0xffffffffu, qq, d);
    qk += __shfl_xor_sync(0xffffffffu, qk, d);
  }
  __syncwarp();
  const float rk = a.qk_norm ? 1.f / sqrtf(kk + a.eps) : 1.f, rq = a.scale * (a.qk_norm ? 1.f / sqrtf(qq + a.eps) : 1.f);
  float unused;
  const float decay = expf(delta_log_decay(a.gate_kind, gate, alpha, beta, unused)), step = delta_step_of(a.step_kind, step_in, unused);
  float sk[E], sq[E];      // H^T k, H^T q
#pragma unroll
  for (int e = 0; e < E; ++e) sk[e] = sq[e] = 0.f;
  if (live) {
#pragma unroll
    for (int r = 0; r < R; ++r)
      if (r < per) {
        const float k = ksm[warp][row0 + r * G], q = qsm[warp][row0 + r * G];
        float h[E];
        X::open(H[r], h);
#pragma unroll
        for (int e = 0; e < E; ++e) {
          sk[e] = fmaf(h[e], k, sk[e]);
          sq[e] = fmaf(h[e], q, sq[e]);
        }
      }
  }
#pragma unroll
  for (int d = L; d < 32; d *= 2)
#pragma unroll
    for (int e = 0; e < E; ++e) {
      sk[e] += __shfl_xor_sync(0xffffffffu, sk[e], d);
      sq[e] += __shfl_xor_sync(0xffffffffu, sq[e], d);
    }
  // the sums of the unit's warps, its u and y: a column a lane (one pass over the sums by every warp took as long as the state's bytes)
  if (lane < L) {
#pragma unroll
    for (int e = 0; e < E; e += 4) {
      *reinterpret_cast<float4 *>(&part[warp][0][col + e]) = make_float4(sk[e], sk[e + 1], sk[e + 2], sk[e + 3]);
      *reinterpret_cast<float4 *>(&part[warp][1][col + e]) = make_float4(sq[e], sq[e + 1], sq[e + 2], sq[e + 3]);
    }
  }
  if (W > 1) __syncthreads();
  else __syncwarp();
  for (int x = sub * 32 + lane; x < V; x += 32 * W) {
    float s = 0.f, t = 0.f;
    for (int w = unit0 * W; w < unit0 * W + W; ++w) { s += part[w][0][x]; t += part[w][1][x]; }
    const float u = in ? step * fmaf(-decay * rk, s, to_f32(static_cast<const TIO *>(a.v)[bn * V + x])) : 0.f;
    part[unit0 * W][0][x] = u;      // (its place is read, by this lane)
    if (in) static_cast<TIO *>(a.y)[bn * V + x] = from_f32<TIO>(live ? rq * fmaf(decay, t, rk * qk * u) : 0.f);
  }
  if (W > 1) __syncthreads();
  else __syncwarp();
  if (!live) return;
  float u[E];
#pragma unroll
  for (int e = 0; e < E; e += 4) {
    const float4 f = *reinterpret_cast<const float4 *>(&part[unit0 * W][0][col + e]);
    u[e] = f.x; u[e + 1] = f.y; u[e + 2] = f.z; u[e + 3] = f.w;
  }
#pragma unroll
  for (int r = 0; r < R; ++r)
    if (r < per) {
      const float k = rk * ksm[warp][row0 + r * G];
      float h[E];
      X::open(H[r], h);
#pragma unroll
      for (int e = 0; e < E; ++e) h[e] = fmaf(k, u[e], decay * h[e]);
      __stcs(reinterpret_cast<uint4 *>(st + (size_t)(r * G) * V), X::close(h));
    }
}

template <typename TIO, typename TS, int V> cudaError_t launch_v(const DeltaStepArgs &a, cudaStream_t s) {
  constexpr int E = Vec16<TS>::n, G = 32 / (V / E), R = sizeof(TS) == 4 ? 16 : 8;      // 64 entries of a state a lane, most
  // warps to a unit: a power of two that leaves whole groups of rows and at most R pieces a lane
  constexpr int most = 8;
  int W = 1;
  while (W < most && a.K / (G * W) > R) W *= 2;
  const long long units = (long long)a.B * a.N;
  // few units: more warps to each, while every one has a group of rows
  while (W < most && a.K % (2 * W * G) == 0 && units * W * 2 <= (long long)sm_count() * 8) W *= 2;
  // CTAs of four warps fill an SM's registers closer than those of eight (28 warps against 24: the units of 48 sequences of 84 heads at
  // once instead of in two rounds)
  const int warps = W > 4 ? 8 : 4;
  const dim3 g((unsigned)((units * W + warps - 1) / warps)), t(32 * warps);
  const bool half = a.K / (G * W) <= R / 2;
  if (warps == 8) return half ? launch_early(delta_step_kernel<TIO, TS, V, R / 2, 8>, g, t, 0, s, a, W) : launch_early(delta_step_kernel<TIO, TS, V, R, 8>, g, t, 0, s, a, W);
  return half ? launch_early(delta_step_kernel<TIO, TS, V, R / 2, 4>, g, t, 0, s, a, W) : launch_early(delta_step_kernel<TIO, TS, V, R, 4>, g, t, 0, s, a, W);
}
template <typename TIO, typename TS> cudaError_t launch_t(const DeltaStepArgs &a, cudaStream_t s) {
  switch (a.V) {
    case 16: return launch_v<TIO, TS, 16>(a, s);
    case 32: return launch_v<TIO, TS, 32>(a, s);
    case 64: return launch_v<TIO, TS, 64>(a, s);
    default: return launch_v<TIO, TS, 128>(a, s);
  }
}

}  // namespace

cudaError_t launch_delta_step(const DeltaStepArgs &a, int io_dtype, int state_dtype, cudaStream_t s) {
  if (io_dtype == M2RNN_F32) return state_dtype == M2RNN_F32 ? launch_t<float, float>(a, s) : launch_t<float, __nv_bfloat16>(a, s);
  return state_dtype == M2RNN_F32 ? launch_t<__nv_bfloat16, float>(a, s) : launch_t<__nv_bfloat16, __nv_bfloat16>(a, s);
}

}  // namespace m2rnn
