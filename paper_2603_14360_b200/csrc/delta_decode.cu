// Gated delta rule: one decoding step on cached states,
//     u = b (v - a H^T k)      H <- a H + k u^T      y = s H^T q = s (a H^T q + (q . k) u)
// (q, k divided by their lengths if asked).  Bound by the state's bytes, read once and written once: both products with
// the old state come from one pass over it, held in registers, and y needs no second one.
//
// A unit is one (b, n).  A lane holds 16 bytes of a row (4 or 8 columns), so L = V / 4 or V / 8 lanes share a row and
// a warp takes 32 / L rows at a time; sixteen 16-byte loads of a lane are in flight at once (fewer where the state is
// smaller).  W warps share a unit: the sums over rows go through shuffles, then (W > 1) through shared memory.  Everything
// is fp32, whatever the types in memory.
#include "delta_common.cuh"

namespace m2rnn {
namespace {

constexpr int kWarps = 8;      // of a CTA

template <typename TS> struct Vec16;      // 16 bytes of a state
template <> struct Vec16<float> {
  static constexpr int n = 4;
  __device__ static void load(const float *p, float (&x)[4]) { const float4 v = __ldcs(reinterpret_cast<const float4 *>(p)); x[0] = v.x; x[1] = v.y; x[2] = v.z; x[3] = v.w; }
  __device__ static void store(float *p, const float (&x)[4]) { __stcs(reinterpret_cast<float4 *>(p), make_float4(x[0], x[1], x[2], x[3])); }
};
template <> struct Vec16<__nv_bfloat16> {
  static constexpr int n = 8;
  __device__ static void load(const __nv_bfloat16 *p, float (&x)[8]) {
    const uint4 v = __ldcs(reinterpret_cast<const uint4 *>(p));
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { const float2 f = unpack_bf16(w[i]); x[2 * i] = f.x; x[2 * i + 1] = f.y; }
  }
  __device__ static void store(__nv_bfloat16 *p, const float (&x)[8]) {
    __stcs(reinterpret_cast<uint4 *>(p), make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7])));
  }
};

// R: 16-byte pieces of a lane, most; W warps to a unit
template <typename TIO, typename TS, int V, int R>
__global__ void __launch_bounds__(32 * kWarps) delta_step_kernel(DeltaStepArgs a, int W) {
  using X = Vec16<TS>;
  constexpr int E = X::n, L = V / E, G = 32 / L;     // lanes to a row, rows of a warp at a time
  __shared__ float part[kWarps][2][V];
  __shared__ float ksm[kWarps][128], qsm[kWarps][128];
  begin_dependent();
  const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31, col = (lane % L) * E;
  const int unit0 = warp / W, sub = warp % W;        // the CTA's unit, this warp's share of it
  const long long unit = (long long)blockIdx.x * (kWarps / W) + unit0;
  const int K = a.K, N = a.N;
  const bool in = unit < (long long)a.B * N;
  const int b = in ? (int)(unit / N) : 0, n = in ? (int)(unit % N) : 0;
  int slot = b;
  if (a.slots && in) slot = a.slots[b];
  // a negative slot is a padding row: no state, y = 0.  One outside the pool is reported.
  const bool live = in && slot >= 0 && slot < a.nslots;
  if (in && slot >= a.nslots && a.dev_status && lane == 0) atomicExch(a.dev_status, (int32_t)M2RNN_ERR_SHAPE);
  TS *st = static_cast<TS *>(a.state) + ((size_t)(live ? slot : 0) * N + n) * K * V;
  const int per = K / (G * W);      // rows groups of this warp: rows (sub per + r) G + lane / L
  float H[R][E];
  const int row0 = sub * per * G + lane / L;
  if (live) {
#pragma unroll
    for (int r = 0; r < R; ++r)
      if (r < per) X::load(st + (size_t)(row0 + r * G) * V + col, H[r]);
  }
  // q and k of the unit: every warp keeps its own copy in shared memory
  const TIO *kg = static_cast<const TIO *>(a.k) + ((size_t)b * a.Nk + n / (N / a.Nk)) * K, *qg = static_cast<const TIO *>(a.q) + ((size_t)b * a.Nq + n / (N / a.Nq)) * K;
  float kk = 0.f, qq = 0.f, qk = 0.f;
  if (in) {
    for (int f = lane; f < K; f += 32) {
      const float k = to_f32(kg[f]), q = to_f32(qg[f]);
      ksm[warp][f] = k;
      qsm[warp][f] = q;
      kk = fmaf(k, k, kk);
      qq = fmaf(q, q, qq);
      qk = fmaf(q, k, qk);
    }
  }
#pragma unroll
  for (int d = 16; d; d /= 2) {
    kk += __shfl_xor_sync(0xffffffffu, kk, d);
    qq += __shfl_xor_sync(0xffffffffu, qq, d);
    qk += __shfl_xor_sync(0xffffffffu, qk, d);
  }
  __syncwarp();
  const float rk = a.qk_norm ? 1.f / sqrtf(kk + a.eps) : 1.f, rq = a.scale * (a.qk_norm ? 1.f / sqrtf(qq + a.eps) : 1.f);
  float sk[E], sq[E];      // H^T k, H^T q
#pragma unroll
  for (int e = 0; e < E; ++e) sk[e] = sq[e] = 0.f;
  if (live) {
#pragma unroll
    for (int r = 0; r < R; ++r)
      if (r < per) {
        const float k = ksm[warp][row0 + r * G], q = qsm[warp][row0 + r * G];
#pragma unroll
        for (int e = 0; e < E; ++e) {
          sk[e] = fmaf(H[r][e], k, sk[e]);
          sq[e] = fmaf(H[r][e], q, sq[e]);
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
  if (W > 1) {
    if (lane < L) {
#pragma unroll
      for (int e = 0; e < E; ++e) {
        part[warp][0][col + e] = sk[e];
        part[warp][1][col + e] = sq[e];
      }
    }
    __syncthreads();
#pragma unroll
    for (int e = 0; e < E; ++e) sk[e] = sq[e] = 0.f;
    for (int w = unit0 * W; w < unit0 * W + W; ++w)
#pragma unroll
      for (int e = 0; e < E; ++e) {
        sk[e] += part[w][0][col + e];
        sq[e] += part[w][1][col + e];
      }
  }
  if (!in) return;
  TIO *yg = static_cast<TIO *>(a.y) + ((size_t)b * N + n) * V + col;
  if (!live) {
    if (sub == 0 && lane < L)
#pragma unroll
      for (int e = 0; e < E; ++e) yg[e] = from_f32<TIO>(0.f);
    return;
  }
  const size_t bn = (size_t)b * N + n;
  const bool psi = a.gate_kind == M2RNN_GATE_PSI;
  float unused;
  const float decay = expf(delta_log_decay(a.gate_kind, to_f32(static_cast<const TIO *>(a.gate)[bn]), psi ? a.alpha[n] : 1.f, psi ? a.beta[n] : 0.f, unused));
  const float step = delta_step_of(a.step_kind, to_f32(static_cast<const TIO *>(a.step)[bn]), unused);
  const TIO *vg = static_cast<const TIO *>(a.v) + bn * V + col;
  float u[E];
#pragma unroll
  for (int e = 0; e < E; ++e) u[e] = step * fmaf(-decay * rk, sk[e], to_f32(vg[e]));
  if (sub == 0 && lane < L) {
    const float s = rq * rk * qk, d = decay * rq;
#pragma unroll
    for (int e = 0; e < E; ++e) yg[e] = from_f32<TIO>(fmaf(d, sq[e], s * u[e]));
  }
#pragma unroll
  for (int r = 0; r < R; ++r)
    if (r < per) {
      const float k = rk * ksm[warp][row0 + r * G];
#pragma unroll
      for (int e = 0; e < E; ++e) H[r][e] = fmaf(k, u[e], decay * H[r][e]);
      X::store(st + (size_t)(row0 + r * G) * V + col, H[r]);
    }
}

template <typename TIO, typename TS, int V> cudaError_t launch_v(const DeltaStepArgs &a, cudaStream_t s) {
  constexpr int E = Vec16<TS>::n, G = 32 / (V / E), R = 64 / E;      // 64 floats of state a lane, most
  // warps to a unit: a power of two that leaves whole groups of rows and at most R pieces a lane
  int W = 1;
  while (W < kWarps && a.K / (G * W) > R) W *= 2;
  const long long units = (long long)a.B * a.N;
  // few units: more warps to each, while every one has a group of rows
  while (W < kWarps && a.K % (2 * W * G) == 0 && units * W * 2 <= (long long)sm_count() * kWarps) W *= 2;
  const long long grid = (units + kWarps / W - 1) / (kWarps / W);
  return launch_early(delta_step_kernel<TIO, TS, V, R>, dim3((unsigned)grid), dim3(32 * kWarps), 0, s, a, W);
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
