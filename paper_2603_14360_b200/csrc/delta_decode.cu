// Gated delta rule: one decoding step on cached states,
//     u = b (v - a H^T k)      H <- a H + k u^T      y = s H^T q = s (a H^T q + (q . k) u)
// (q, k divided by their lengths if asked).  Bound by the state's bytes, read once and written once: both products with
// the old state come from one pass over it, held in registers, and y needs no second one.
//
// A unit is one (b, n).  A lane holds 16 bytes of a row (4 or 8 columns), so L = V / 4 or V / 8 lanes share a row and
// a warp takes 32 / L rows at a time; sixteen 16-byte loads of a lane are in flight at once (fewer where the state is
// smaller).  W warps share a unit: the sums over rows go through shuffles, then (W > 1) through shared memory.  Everything
// is fp32, whatever the types in memory.
// What is the same for a unit (lengths, decay, step) its first warp works out for the others, a warp loads the rows of k and q that it has rows of
// the state for, and v is asked for before anything is waited for: with every warp working all of it out, and loops of a length not known to
// the compiler, the kernel was bound by its instructions (81 % of the issue slots, 1 440 a warp: 198, 7.1 and 3.9 us below).
// 512 rows of 32 bf16 states of 128 x 128: 178 us, 6.0 TB/s; 48 rows of 84 fp32 states of 64 x 16 (33 MB): 5.2 us a step
// on one pool, which stays in the L2, 7.3 on sixteen by turns, 4.6 TB/s; one row of these: 3.0 us, a launch
// and a memory round trip.
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

// k and q of a row, side by side in shared memory; the sums of both products over a piece's columns
template <typename TIO, typename TS> struct Pair {
  float k, q;
  __device__ Pair(TIO k, TIO q) : k(to_f32(k)), q(to_f32(q)) {}
  __device__ float key() const { return k; }
  template <int E> __device__ void add(const uint4 &r, float (&sk)[E], float (&sq)[E]) const {
    float h[E];
    Vec16<TS>::open(r, h);
#pragma unroll
    for (int e = 0; e < E; ++e) {
      sk[e] = fmaf(h[e], k, sk[e]);
      sq[e] = fmaf(h[e], q, sq[e]);
    }
  }
};
template <> struct Pair<__nv_bfloat16, __nv_bfloat16> {      // (as they are: products of 16-bit operands in fp32, nothing to unpack)
  uint32_t kq;
  __device__ Pair(__nv_bfloat16 k, __nv_bfloat16 q) : kq((uint32_t)__bfloat16_as_ushort(q) << 16 | __bfloat16_as_ushort(k)) {}
  __device__ float key() const { return __uint_as_float(kq << 16); }
  __device__ void add(const uint4 &r, float (&sk)[8], float (&sq)[8]) const {
    const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      sk[2 * i] = fma_bf16<0, 0>(w[i], kq, sk[2 * i]);
      sk[2 * i + 1] = fma_bf16<1, 0>(w[i], kq, sk[2 * i + 1]);
      sq[2 * i] = fma_bf16<0, 1>(w[i], kq, sq[2 * i]);
      sq[2 * i + 1] = fma_bf16<1, 1>(w[i], kq, sq[2 * i + 1]);
    }
  }
};

// R: 16-byte pieces of a lane (FULL: as many, else at most); 2^log_w warps to a unit, kWarps to a CTA
template <typename TIO, typename TS, int V, int R, int kWarps, bool FULL>
__global__ void __launch_bounds__(32 * kWarps, (R > 8 ? 16 : sizeof(TS) == 2 ? 32 : 28) / kWarps) delta_step_kernel(DeltaStepArgs a, int log_w) {
  using X = Vec16<TS>;
  using KQ = Pair<TIO, TS>;
  constexpr int E = X::n, L = V / E, G = 32 / L, NX = (V + 31) / 32;     // lanes to a row, rows of a warp at a time; columns of u a lane, most
  __shared__ float part[kWarps][2][V];               // sums over a warp's rows; then [unit's first warp][0]: u / |k|
  __shared__ float scalars[kWarps][6];               // of a unit, at its first warp
  __shared__ alignas(8) unsigned char kq_of[kWarps][128 * sizeof(KQ)];      // a warp's rows
  begin_dependent();
  const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31, col = (lane % L) * E;
  const int W = 1 << log_w, first = warp & -W, sub = warp & (W - 1);      // the unit's first warp, this one's share of it
  const unsigned unit = blockIdx.x * (unsigned)(kWarps >> log_w) + (unsigned)(warp >> log_w);
  const int K = a.K, N = a.N;
  const bool in = unit < (unsigned)a.B * (unsigned)N;
  const unsigned bn = in ? unit : 0u, b = bn / (unsigned)N, n = bn - b * (unsigned)N;
  const int slot = a.slots ? a.slots[b] : (int)b;
  // what does not hang on the slot is asked for first: this warp's rows of k and q (the first one's: all, for their lengths), gates, v
  const int rows = K >> log_w, row0 = sub * rows, count = !in ? 0 : sub ? rows : K;
  const TIO *kg = static_cast<const TIO *>(a.k) + ((size_t)b * a.Nk + n / (unsigned)a.per_k) * K + row0 + lane;
  const TIO *qg = static_cast<const TIO *>(a.q) + ((size_t)b * a.Nq + n / (unsigned)a.per_q) * K + row0 + lane;
  TIO kx[4], qx[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    kx[i] = qx[i] = from_f32<TIO>(0.f);
    if (lane + 32 * i < count) { kx[i] = kg[32 * i]; qx[i] = qg[32 * i]; }
  }
  float gate = 0.f, step_in = 0.f, alpha = 1.f, beta = 0.f;
  if (in && sub == 0) {
    gate = to_f32(static_cast<const TIO *>(a.gate)[bn]);
    step_in = to_f32(static_cast<const TIO *>(a.step)[bn]);
    if (a.gate_kind == M2RNN_GATE_PSI) { alpha = a.alpha[n]; beta = a.beta[n]; }
  }
  float vx[NX];
#pragma unroll
  for (int i = 0; i < NX; ++i) {
    const int x = 32 * (sub + (i << log_w)) + lane;
    vx[i] = in && x < V ? to_f32(static_cast<const TIO *>(a.v)[(size_t)bn * V + x]) : 0.f;
  }
  // a negative slot is a padding row: no state, y = 0.  One outside the pool is reported.
  const bool live = in && slot >= 0 && slot < a.nslots;
  if (in && slot >= a.nslots && a.dev_status && lane == 0) atomicExch(a.dev_status, (int32_t)M2RNN_ERR_SHAPE);
  const int per = rows / G, mine = lane / L;      // pieces of a lane, its place in a group of rows
  TS *st = static_cast<TS *>(a.state) + ((size_t)(live ? slot : 0) * N + n) * K * V + (size_t)(row0 + mine) * V + col;
  uint4 H[R];
  if (live) {
#pragma unroll
    for (int r = 0; r < R; ++r)
      if (FULL || r < per) H[r] = __ldcs(reinterpret_cast<const uint4 *>(st + r * G * V));
  }
  KQ *kq = reinterpret_cast<KQ *>(kq_of[warp]);
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (lane + 32 * i < rows) kq[lane + 32 * i] = KQ(kx[i], qx[i]);
  if (sub == 0) {      // lengths, decay and step
    float kk = 0.f, qq = 0.f, qk = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float k = to_f32(kx[i]), q = to_f32(qx[i]);
      kk = fmaf(k, k, kk);
      qq = fmaf(q, q, qq);
      qk = fmaf(q, k, qk);
    }
#pragma unroll
    for (int d = 16; d; d /= 2) {
      kk += __shfl_xor_sync(0xffffffffu, kk, d);
      qq += __shfl_xor_sync(0xffffffffu, qq, d);
      qk += __shfl_xor_sync(0xffffffffu, qk, d);
    }
    const float rk = a.qk_norm ? 1.f / sqrtf(kk + a.eps) : 1.f, rq = a.scale * (a.qk_norm ? 1.f / sqrtf(qq + a.eps) : 1.f);
    float unused;
    const float decay = expf(delta_log_decay(a.gate_kind, gate, alpha, beta, unused)), step = delta_step_of(a.step_kind, step_in, unused);
    if (lane == 0) {
      float *f = scalars[warp];
      f[0] = decay; f[1] = step; f[2] = -decay * rk; f[3] = rq * decay; f[4] = rq * (rk * qk); f[5] = rk;
    }
  }
  __syncwarp();
  float sk[E], sq[E];      // H^T k, H^T q
#pragma unroll
  for (int e = 0; e < E; ++e) sk[e] = sq[e] = 0.f;
  if (live) {
#pragma unroll
    for (int r = 0; r < R; ++r)
      if (FULL || r < per) kq[mine + r * G].add(H[r], sk, sq);
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
  const float *f = scalars[first];
#pragma unroll
  for (int i = 0; i < NX; ++i) {
    const int x = 32 * (sub + (i << log_w)) + lane;
    if (x >= V) break;
    float s = 0.f, t = 0.f;
    for (int w = first; w < first + W; ++w) { s += part[w][0][x]; t += part[w][1][x]; }
    const float u = f[1] * fmaf(f[2], s, vx[i]);
    part[first][0][x] = f[5] * u;      // (its place is read, by this lane)
    if (in) static_cast<TIO *>(a.y)[(size_t)bn * V + x] = from_f32<TIO>(live ? fmaf(f[3], t, f[4] * u) : 0.f);
  }
  if (W > 1) __syncthreads();
  else __syncwarp();
  if (!live) return;
  const float decay = f[0];
  float u[E];
#pragma unroll
  for (int e = 0; e < E; e += 4) {
    const float4 p = *reinterpret_cast<const float4 *>(&part[first][0][col + e]);
    u[e] = p.x; u[e + 1] = p.y; u[e + 2] = p.z; u[e + 3] = p.w;
  }
#pragma unroll
  for (int r = 0; r < R; ++r)
    if (FULL || r < per) {
      const float k = kq[mine + r * G].key();
      float h[E];
      X::open(H[r], h);
#pragma unroll
      for (int e = 0; e < E; ++e) h[e] = fmaf(k, u[e], decay * h[e]);
      __stcs(reinterpret_cast<uint4 *>(st + r * G * V), X::close(h));
    }
}

template <typename TIO, typename TS, int V, int R, int kWarps> cudaError_t launch_r(const DeltaStepArgs &a, int log_w, int per, cudaStream_t s) {
  const dim3 g((unsigned)((((long long)a.B * a.N << log_w) + kWarps - 1) / kWarps)), t(32 * kWarps);
  return per == R ? launch_early(delta_step_kernel<TIO, TS, V, R, kWarps, true>, g, t, 0, s, a, log_w) : launch_early(delta_step_kernel<TIO, TS, V, R, kWarps, false>, g, t, 0, s, a, log_w);
}
template <typename TIO, typename TS, int V> cudaError_t launch_v(const DeltaStepArgs &a, cudaStream_t s) {
  constexpr int E = Vec16<TS>::n, G = 32 / (V / E), R = sizeof(TS) == 4 ? 16 : 8;      // 64 entries of a state a lane, most
  // warps to a unit: a power of two that leaves whole groups of rows and at most R pieces a lane
  constexpr int most = 3;
  int log_w = 0;
  while (log_w < most && a.K >> log_w > G * R) ++log_w;
  const long long units = (long long)a.B * a.N;
  // few units: more warps to each, while every one has a group of rows
  while (log_w < most && a.K % (G << (log_w + 1)) == 0 && units << (log_w + 1) <= (long long)sm_count() * 8) ++log_w;
  // CTAs of four warps fill an SM's registers closer than those of eight (28 warps against 24: the units of 48 sequences of 84 heads at
  // once instead of in two rounds)
  const int per = (a.K >> log_w) / G;
  if (log_w > 2) return per <= R / 2 ? launch_r<TIO, TS, V, R / 2, 8>(a, log_w, per, s) : launch_r<TIO, TS, V, R, 8>(a, log_w, per, s);
  return per <= R / 2 ? launch_r<TIO, TS, V, R / 2, 4>(a, log_w, per, s) : launch_r<TIO, TS, V, R, 4>(a, log_w, per, s);
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
