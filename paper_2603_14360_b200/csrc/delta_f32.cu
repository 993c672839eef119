// Gated delta rule, fp32 (the accuracy path): everything in fp32 FMA, chunks of 16 tokens (the formulas: delta_chain.cu,
// delta_grad.cu).  A CTA takes one (b, n) and walks its chunks; a chunk's operands lie in shared memory and every
// product is a loop of FMAs, a column or an entry a thread.  The forward call keeps a state per chunk for the backward
// call, which recomputes U from it.
#include "delta_common.cuh"

namespace m2rnn {
namespace {

constexpr int C = kDeltaChunkF32, kThreads = 256;

// Shared memory of a chunk (floats).  PK, PV: pitches (odd, so that a column's entries fall into different banks).
struct Lay {
  int PK, PV, k, q, v, dy, x, u, l, S, D, A, P, m[4], vec, total;
  __host__ __device__ Lay(int K, int V, bool backward) {
    PK = K + 1; PV = V + 1;
    int o = 0;
    auto take = [&](int n) { const int at = o; o += (n + 3) / 4 * 4; return at; };
    k = take(C * PK); q = take(C * PK); v = take(C * PV);
    u = take(C * PV); S = take(K * PV);
    A = take(C * (C + 1)); P = take(C * (C + 1));
    vec = take(16 * C);
    dy = x = l = D = m[0] = m[1] = m[2] = m[3] = 0;
    if (backward) {
      dy = take(C * PV); l = take(C * PV); D = take(K * PV);
      for (int i = 0; i < 4; ++i) m[i] = take(C * PK);
      x = take(2 * C * (C + 1));
    }
    total = o;
  }
};
enum { EG = 0, EK = 1, BT = 2, GS = 3, RK = 4, RQ = 5, DL = 6, DB = 7, SUM = 8 };   // rows of C in vec; SUM ..: sums of the gradient's rows

// Loads a chunk's k^, q^ (divided by their lengths), v; the gates; A_ij = e^(g_i - g_j) k^_i . k^_j (j < i), P_ij likewise with s q^ (j <= i)
__device__ void load_chunk(const DeltaArgs &a, const Lay &y, float *sm, long long tok, int have, int n) {
  const int K = a.K, V = a.V, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const float *kg = static_cast<const float *>(a.k) + tok * a.ks + (long long)(n / (a.N / a.Nk)) * K;
  const float *qg = static_cast<const float *>(a.q) + tok * a.qs + (long long)(n / (a.N / a.Nq)) * K;
  const float *vg = static_cast<const float *>(a.v) + tok * a.vs + (long long)n * V;
  for (int x = tid; x < C * K; x += kThreads) {
    const int r = x / K, f = x % K;
    sm[y.k + r * y.PK + f] = r < have ? kg[r * a.ks + f] : 0.f;
    sm[y.q + r * y.PK + f] = r < have ? qg[r * a.qs + f] : 0.f;
  }
  for (int x = tid; x < C * V; x += kThreads) {
    const int r = x / V, f = x % V;
    sm[y.v + r * y.PV + f] = r < have ? vg[r * a.vs + f] : 0.f;
  }
  float *vec = sm + y.vec;
  if (warp == 0) {
    float la = 0.f, bt = 0.f, dl = 0.f, db = 0.f;
    if (lane < have) {
      const size_t at = (size_t)(tok + lane) * a.N + n;
      const bool psi = a.gate_kind == M2RNN_GATE_PSI;
      la = delta_log_decay(a.gate_kind, static_cast<const float *>(a.gate)[at], psi ? a.alpha[n] : 1.f, psi ? a.beta[n] : 0.f, dl);
      bt = delta_step_of(a.step_kind, static_cast<const float *>(a.step)[at], db);
    }
    float gs = la;
#pragma unroll
    for (int d = 1; d < C; d *= 2) {
      const float o = __shfl_up_sync(0xffffffffu, gs, d);
      if (lane >= d) gs += o;
    }
    const float last = __shfl_sync(0xffffffffu, gs, C - 1);
    if (lane < C) {
      vec[C * EG + lane] = expf(gs);
      vec[C * EK + lane] = expf(last - gs);
      vec[C * BT + lane] = bt;
      vec[C * GS + lane] = gs;
      vec[C * DL + lane] = dl;
      vec[C * DB + lane] = db;
      vec[C * RK + lane] = vec[C * RQ + lane] = 1.f;
    }
  }
  __syncthreads();
  if (a.qk_norm) {      // a warp a row
    for (int r = warp; r < 2 * C; r += kThreads / 32) {
      float *row = sm + (r < C ? y.k + r * y.PK : y.q + (r - C) * y.PK);
      float s = 0.f;
      for (int f = lane; f < K; f += 32) s = fmaf(row[f], row[f], s);
#pragma unroll
      for (int d = 16; d; d /= 2) s += __shfl_xor_sync(0xffffffffu, s, d);
      const float ri = 1.f / sqrtf(s + a.eps);
      for (int f = lane; f < K; f += 32) row[f] *= ri;
      if (lane == 0) vec[C * (r < C ? RK : RQ) + r % C] = ri;
    }
    __syncthreads();
  }
  for (int x = tid; x < 2 * C * C; x += kThreads) {
    const int i = x / C % C, j = x % C;
    const bool p = x >= C * C;
    float s = 0.f;
    if (p ? j <= i : j < i) {
      const float *r = sm + (p ? y.q : y.k) + i * y.PK, *o = sm + y.k + j * y.PK;
      for (int f = 0; f < K; ++f) s = fmaf(r[f], o[f], s);
      s *= expf(vec[C * GS + i] - vec[C * GS + j]) * (p ? a.scale : 1.f);
    }
    sm[(p ? y.P : y.A) + i * (C + 1) + j] = s;
  }
  __syncthreads();
}

// U: a group of 256 / V threads has a column; k^ S first, then the 16 rows one after the other
__device__ void solve(const Lay &y, float *sm, int K, int V) {
  const float *vec = sm + y.vec;
  for (int x = threadIdx.x; x < C * V; x += kThreads) {
    const int i = x / V, v = x % V;
    float s0 = 0.f, s1 = 0.f;
    for (int f = 0; f < K; f += 2) {
      s0 = fmaf(sm[y.k + i * y.PK + f], sm[y.S + f * y.PV + v], s0);
      s1 = fmaf(sm[y.k + i * y.PK + f + 1], sm[y.S + (f + 1) * y.PV + v], s1);
    }
    sm[y.u + i * y.PV + v] = fmaf(-vec[C * EG + i], s0 + s1, sm[y.v + i * y.PV + v]);
  }
  __syncthreads();
  for (int v = threadIdx.x; v < V; v += kThreads) {
    float u[C];
#pragma unroll
    for (int i = 0; i < C; ++i) {
      float s = sm[y.u + i * y.PV + v];
#pragma unroll
      for (int j = 0; j < i; ++j) s = fmaf(-sm[y.A + i * (C + 1) + j], u[j], s);
      u[i] = vec[C * BT + i] * s;
    }
#pragma unroll
    for (int i = 0; i < C; ++i) sm[y.u + i * y.PV + v] = u[i];
  }
  __syncthreads();
}

__device__ __forceinline__ float load_state(const void *p, size_t x, int bf16) {
  return bf16 ? __bfloat162float(static_cast<const __nv_bfloat16 *>(p)[x]) : static_cast<const float *>(p)[x];
}
__device__ __forceinline__ void store_state(void *p, size_t x, int bf16, float v) {
  if (bf16) static_cast<__nv_bfloat16 *>(p)[x] = __float2bfloat16_rn(v);
  else static_cast<float *>(p)[x] = v;
}

__global__ void __launch_bounds__(kThreads) delta_fwd_f32_kernel(DeltaArgs a) {
  extern __shared__ __align__(16) float sm[];
  begin_dependent();
  const int K = a.K, V = a.V, tid = threadIdx.x, b = blockIdx.x / a.N, n = blockIdx.x % a.N;
  const Lay y(K, V, false);
  const DeltaSpan sp = delta_span<C>(a, b);
  const size_t at = ((size_t)b * a.N + n) * K * V;
  const float *vec = sm + y.vec;
  for (int x = tid; x < K * V; x += kThreads) sm[y.S + x / V * y.PV + x % V] = a.h0 ? load_state(a.h0, at + x, a.state_bf16) : 0.f;
  __syncthreads();
  for (int ch = 0; ch < sp.n; ++ch) {
    const long long tok = sp.tok0 + ch * C;
    const int have = min(C, sp.T - ch * C);
    if (a.states) {
      float *o = reinterpret_cast<float *>(a.states) + ((size_t)(sp.slot0 + ch) * a.N + n) * K * V;
      for (int x = tid; x < K * V; x += kThreads) o[x] = sm[y.S + x / V * y.PV + x % V];
    }
    load_chunk(a, y, sm, tok, have, n);
    solve(y, sm, K, V);
    if (a.y)
      for (int x = tid; x < have * V; x += kThreads) {
        const int i = x / V, v = x % V;
        float s = 0.f, p = 0.f;
        for (int f = 0; f < K; ++f) s = fmaf(sm[y.q + i * y.PK + f], sm[y.S + f * y.PV + v], s);
        for (int j = 0; j <= i; ++j) p = fmaf(sm[y.P + i * (C + 1) + j], sm[y.u + j * y.PV + v], p);
        static_cast<float *>(a.y)[((size_t)(tok + i) * a.N + n) * V + v] = fmaf(a.scale * vec[C * EG + i], s, p);
      }
    __syncthreads();
    const float ec = vec[C * EG + C - 1];
    for (int x = tid; x < K * V; x += kThreads) {
      const int f = x / V, v = x % V;
      float s = ec * sm[y.S + f * y.PV + v];
#pragma unroll
      for (int j = 0; j < C; ++j) s = fmaf(vec[C * EK + j] * sm[y.k + j * y.PK + f], sm[y.u + j * y.PV + v], s);
      sm[y.S + f * y.PV + v] = s;
    }
    __syncthreads();
  }
  if (a.hT)
    for (int x = tid; x < K * V; x += kThreads) store_state(a.hT, at + x, a.state_bf16, sm[y.S + x / V * y.PV + x % V]);
}

__global__ void __launch_bounds__(kThreads) delta_bwd_f32_kernel(DeltaArgs a) {
  extern __shared__ __align__(16) float sm[];
  begin_dependent();
  const int K = a.K, V = a.V, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, b = blockIdx.x / a.N, n = blockIdx.x % a.N;
  const Lay y(K, V, true);
  const DeltaSpan sp = delta_span<C>(a, b);
  const size_t at = ((size_t)b * a.N + n) * K * V;
  float *vec = sm + y.vec;
  for (int x = tid; x < K * V; x += kThreads) sm[y.D + x / V * y.PV + x % V] = a.d_hT ? load_state(a.d_hT, at + x, a.state_bf16) : 0.f;
  __syncthreads();
  for (int ch = sp.n - 1; ch >= 0; --ch) {
    const long long tok = sp.tok0 + ch * C;
    const int have = min(C, sp.T - ch * C);
    const float *sg = reinterpret_cast<const float *>(a.states) + ((size_t)(sp.slot0 + ch) * a.N + n) * K * V;
    for (int x = tid; x < K * V; x += kThreads) sm[y.S + x / V * y.PV + x % V] = sg[x];
    for (int x = tid; x < C * V; x += kThreads) {
      const int r = x / V, v = x % V;
      sm[y.dy + r * y.PV + v] = r < have ? static_cast<const float *>(a.dy)[((size_t)(tok + r) * a.N + n) * V + v] : 0.f;
    }
    load_chunk(a, y, sm, tok, have, n);
    solve(y, sm, K, V);
    // dU, then L = (I + b A)^-T dU from the last row up
    for (int x = tid; x < C * V; x += kThreads) {
      const int j = x / V, v = x % V;
      float s = 0.f, p = 0.f;
      for (int f = 0; f < K; ++f) s = fmaf(sm[y.k + j * y.PK + f], sm[y.D + f * y.PV + v], s);
      for (int i = j; i < C; ++i) p = fmaf(sm[y.P + i * (C + 1) + j], sm[y.dy + i * y.PV + v], p);
      sm[y.l + j * y.PV + v] = fmaf(vec[C * EK + j], s, p);
    }
    __syncthreads();
    for (int v = tid; v < V; v += kThreads) {
      float l[C];      // b L below: what row j takes of the rows behind it
#pragma unroll
      for (int j = C - 1; j >= 0; --j) {
        float s = sm[y.l + j * y.PV + v];
#pragma unroll
        for (int i = j + 1; i < C; ++i) s = fmaf(-sm[y.A + i * (C + 1) + j], l[i], s);
        sm[y.l + j * y.PV + v] = s;
        l[j] = vec[C * BT + j] * s;
      }
    }
    __syncthreads();
    for (int x = tid; x < have * V; x += kThreads) {
      const int i = x / V, v = x % V;
      static_cast<float *>(a.dv)[((size_t)(tok + i) * a.N + n) * V + v] = vec[C * BT + i] * sm[y.l + i * y.PV + v];
    }
    // E dP (s in it) and E N
    for (int x = tid; x < 2 * C * C; x += kThreads) {
      const int i = x / C % C, j = x % C;
      const bool p = x < C * C;
      float s = 0.f;
      if (p ? j <= i : j < i) {
        const float *r = sm + (p ? y.dy : y.l) + i * y.PV, *u = sm + y.u + j * y.PV;
        for (int v = 0; v < V; ++v) s = fmaf(r[v], u[v], s);
        s *= expf(vec[C * GS + i] - vec[C * GS + j]) * (p ? a.scale : -1.f);
      }
      sm[y.x + (p ? 0 : C * (C + 1)) + i * (C + 1) + j] = s;
    }
    __syncthreads();
    // dQ^, dK-, dK+
    for (int x = tid; x < C * K; x += kThreads) {
      const int i = x / K, f = x % K;
      float ys = 0.f, ls = 0.f, us = 0.f;
      for (int v = 0; v < V; ++v) {
        const float S = sm[y.S + f * y.PV + v];
        ys = fmaf(sm[y.dy + i * y.PV + v], S, ys);
        ls = fmaf(sm[y.l + i * y.PV + v], S, ls);
        us = fmaf(sm[y.u + i * y.PV + v], sm[y.D + f * y.PV + v], us);
      }
      ys *= a.scale * vec[C * EG + i];
      ls *= -vec[C * EG + i];
      us *= vec[C * EK + i];
      const float first = us;
      for (int j = 0; j <= i; ++j) {
        ys = fmaf(sm[y.x + i * (C + 1) + j], sm[y.k + j * y.PK + f], ys);
        ls = fmaf(sm[y.x + C * (C + 1) + i * (C + 1) + j], sm[y.k + j * y.PK + f], ls);
      }
      for (int j = i; j < C; ++j) {
        us = fmaf(sm[y.x + j * (C + 1) + i], sm[y.q + j * y.PK + f], us);
        us = fmaf(vec[C * BT + j] * sm[y.x + C * (C + 1) + j * (C + 1) + i], sm[y.k + j * y.PK + f], us);
      }
      sm[y.m[0] + i * y.PK + f] = ys;
      sm[y.m[1] + i * y.PK + f] = ls;
      sm[y.m[2] + i * y.PK + f] = us;
      sm[y.m[3] + i * y.PK + f] = first;
    }
    float ss = 0.f;      // <S, dS'>
    for (int x = tid; x < K * V; x += kThreads) ss = fmaf(sm[y.S + x / V * y.PV + x % V], sm[y.D + x / V * y.PV + x % V], ss);
    __syncthreads();
    // sums of a row: q^ . dQ^, k^ . dK-, k^ . dK+, k^ . (e^(g_last - g) dS' U), L . v
    for (int i = warp; i < C; i += kThreads / 32) {
      float d[5] = {};
      for (int f = lane; f < K; f += 32) {
        const float q = sm[y.q + i * y.PK + f], k = sm[y.k + i * y.PK + f];
        d[0] = fmaf(q, sm[y.m[0] + i * y.PK + f], d[0]);
#pragma unroll
        for (int m = 1; m < 4; ++m) d[m] = fmaf(k, sm[y.m[m] + i * y.PK + f], d[m]);
      }
      for (int v = lane; v < V; v += 32) d[4] = fmaf(sm[y.l + i * y.PV + v], sm[y.v + i * y.PV + v], d[4]);
#pragma unroll
      for (int m = 0; m < 5; ++m) {
#pragma unroll
        for (int o = 16; o; o /= 2) d[m] += __shfl_xor_sync(0xffffffffu, d[m], o);
        if (lane == 0) vec[C * (SUM + m) + i] = d[m];
      }
    }
#pragma unroll
    for (int o = 16; o; o /= 2) ss += __shfl_xor_sync(0xffffffffu, ss, o);
    if (lane == 0) vec[C * (SUM + 5) + warp] = ss;
    __syncthreads();
    const float ec = vec[C * EG + C - 1];
    if (warp == 0) {
      const int i = lane & (C - 1);
      float part = lane < C ? vec[C * SUM + i] + vec[C * BT + i] * vec[C * (SUM + 1) + i] - vec[C * (SUM + 2) + i] : 0.f, all = lane < C ? vec[C * (SUM + 3) + i] : 0.f;
      float sd = lane < kThreads / 32 ? vec[C * (SUM + 5) + lane] : 0.f;
#pragma unroll
      for (int o = 16; o; o /= 2) {
        all += __shfl_xor_sync(0xffffffffu, all, o);
        sd += __shfl_xor_sync(0xffffffffu, sd, o);
      }
#pragma unroll
      for (int o = 1; o < C; o *= 2) {
        const float t = __shfl_down_sync(0xffffffffu, part, o);
        if (lane + o < C) part += t;
      }
      if (lane < have) {
        const size_t x = (size_t)(tok + lane) * a.N + n;
        static_cast<float *>(a.dgate)[x] = (part + all + ec * sd) * vec[C * DL + lane];
        static_cast<float *>(a.dstep)[x] = (vec[C * (SUM + 4) + lane] + vec[C * (SUM + 1) + lane]) * vec[C * DB + lane];
      }
    }
    // dq, dk through the division by the lengths
    for (int x = tid; x < have * K; x += kThreads) {
      const int i = x / K, f = x % K;
      const float bt = vec[C * BT + i];
      float dq = sm[y.m[0] + i * y.PK + f], dk = fmaf(bt, sm[y.m[1] + i * y.PK + f], sm[y.m[2] + i * y.PK + f]);
      if (a.qk_norm) {
        dq = vec[C * RQ + i] * fmaf(-sm[y.q + i * y.PK + f], vec[C * SUM + i], dq);
        dk = vec[C * RK + i] * fmaf(-sm[y.k + i * y.PK + f], fmaf(bt, vec[C * (SUM + 1) + i], vec[C * (SUM + 2) + i]), dk);
      }
      const size_t t = (size_t)(tok + i);
      if (a.dq_part) a.dq_part[(t * a.N + n) * K + f] = dq;
      else static_cast<float *>(a.dq)[(t * a.N + n) * K + f] = dq;
      if (a.dk_part) a.dk_part[(t * a.N + n) * K + f] = dk;
      else static_cast<float *>(a.dk)[(t * a.N + n) * K + f] = dk;
    }
    // dS
    for (int x = tid; x < K * V; x += kThreads) {
      const int f = x / V, v = x % V;
      float s = ec * sm[y.D + f * y.PV + v];
#pragma unroll
      for (int j = 0; j < C; ++j) {
        s = fmaf(a.scale * vec[C * EG + j] * sm[y.q + j * y.PK + f], sm[y.dy + j * y.PV + v], s);
        s = fmaf(-vec[C * EG + j] * vec[C * BT + j] * sm[y.k + j * y.PK + f], sm[y.l + j * y.PV + v], s);
      }
      sm[y.D + f * y.PV + v] = s;
    }
    __syncthreads();
  }
  if (a.dh0)
    for (int x = tid; x < K * V; x += kThreads) store_state(a.dh0, at + x, a.state_bf16, sm[y.D + x / V * y.PV + x % V]);
}

cudaError_t launch(void (*kernel)(DeltaArgs), const DeltaArgs &a, bool backward, cudaStream_t s) {
  const size_t smem = (size_t)Lay(a.K, a.V, backward).total * sizeof(float);
  const cudaError_t e = allow_smem(kernel, smem);
  if (e != cudaSuccess) return e;
  return launch_early(kernel, dim3((unsigned)((long long)a.B * a.N)), dim3(kThreads), smem, s, a);
}

}  // namespace

cudaError_t launch_delta_fwd_f32(const DeltaArgs &a, cudaStream_t s) { return launch(delta_fwd_f32_kernel, a, false, s); }
cudaError_t launch_delta_bwd_f32(const DeltaArgs &a, cudaStream_t s) { return launch(delta_bwd_f32_kernel, a, true, s); }

}  // namespace m2rnn
