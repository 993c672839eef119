// Gated delta rule, fp32 (the accuracy path): the formulas of delta_prep.cu, delta_chain.cu and delta_grad.cu in chunks of
// 16 tokens, everything in fp32 FMA.
//
//   prep : a CTA a chunk of one head: M, T = (I + M)^-1 by substitution, P, the tokens' factors.
//   chain: columns of the state are independent recurrences.  Sixteen lanes have a column, K/16 rows each in registers.  Their
//          sixteen partial products with the chunk's tokens are added by recursive halving, which leaves token t's sum in
//          lane t: the products with T and P and with the tokens are then FMAs on shuffled values.  A CTA's warps share the
//          chunk's rows in shared memory (stages that a warp of its own fills by cp.async); few columns to a CTA where there are few units.
//   grad : a CTA a chunk of one head, everything of it in shared memory; four tokens' entries of a feature to a thread.
// States of chunks are kept column after column, [V][K], so that a column's lanes write contiguous floats.
// Bound by the latency of FMAs, shuffles and shared memory: 2 x 512 tokens of 8 heads of 64 x 64 take 11.2 (prep), 42.2 and 38.3 (chains, 1.3 us
// and 1.2 a chunk) and 33.1 us (grad, two CTAs to an SM), against 2.7 for the bytes.
#include "delta_common.cuh"

namespace m2rnn {
namespace {

constexpr int C = kDeltaChunkF32;
constexpr int kT = 0, kP = C * C, kM = 2 * C * C, kVec = 3 * C * C, kRec = kRecF32Bytes / 4;      // floats of a record
// a token's factors: of kVec* of delta.h those of the numbers 0 .. 3, 5 and 6, and these.  (The chains copy the first eight arrays.)
enum {
  kBeta = kVecBeta,
  kEg = kVecG,      // e^g
  kEl = kVecDlog,   // e^(g_last - g)
  kGHigh = 8, kGLow = 9, kDlog = 10
};
static_assert(kVec + 11 * C == kRec && kP == C * C && kEg == 4 && kEl == 7, "");

// Running sums of log a are kept as pairs of floats, kGHigh and what that leaves out (kGLow), and differences of two are taken in 64 bits: a
// dropped state (kLogFloor) or a strong decay stays in every later sum, and behind sixteen of them a float is 1.2e-4 from the next, where
// the decay between two tokens needs 2^-24 of itself.  e^d is that of d's nearest float times 1 + what is left of d.
__device__ __forceinline__ float exp_of(double d) {
  const float h = (float)d, e = expf(h);
  return fmaf(e, (float)(d - h), e);
}
__device__ __forceinline__ double sum_at(const float *vec, int i) { return (double)vec[C * kGHigh + i] + vec[C * kGLow + i]; }

// ---- prep

__global__ void __launch_bounds__(128) delta_prep_f32_kernel(DeltaArgs a) {
  extern __shared__ __align__(16) float sm[];
  begin_dependent();
  const int K = a.K, PK = K + 4, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const unsigned at = blockIdx.x / (unsigned)a.N;
  const int n = (int)(blockIdx.x - at * a.N), b = a.cu ? delta_entry<C, true>(a, at) : delta_entry<C, false>(a, at);
  const DeltaSpan sp = delta_span<C>(a, b);
  const int ch = (int)(at - sp.slot0);
  if ((unsigned)ch >= (unsigned)sp.n) return;      // (of a packed batch: a slot that is no sequence's)
  const long long tok = sp.tok0 + ch * C;
  const int have = min(C, sp.T - ch * C);
  float *ks = sm, *qs = ks + C * PK, *Ms = qs + C * PK, *vec = Ms + C * (C + 4);
  const float *kg = static_cast<const float *>(a.k) + tok * a.ks + (long long)(n / (a.N / a.Nk)) * K;
  const float *qg = static_cast<const float *>(a.q) + tok * a.qs + (long long)(n / (a.N / a.Nq)) * K;
  for (int x = tid; x < C * (K / 4); x += 128) {
    const int r = x / (K / 4), o = 4 * (x % (K / 4));
    const bool ok = r < have;
    cp16_or_zero(smem_u32(ks + r * PK + o), kg + (ok ? r * a.ks : 0) + o, ok);
    cp16_or_zero(smem_u32(qs + r * PK + o), qg + (ok ? r * a.qs : 0) + o, ok);
  }
  if (warp == 0) {
    float la = 0.f, bt = 0.f, dl = 0.f, unused;
    if (lane < have) {
      const size_t at = (size_t)(tok + lane) * a.N + n;
      const bool psi = a.gate_kind == M2RNN_GATE_PSI;
      la = delta_log_decay(a.gate_kind, static_cast<const float *>(a.gate)[at], psi ? a.alpha[n] : 1.f, psi ? a.beta[n] : 0.f, dl);
      bt = delta_step_of(a.step_kind, static_cast<const float *>(a.step)[at], unused);
    }
    double gs = la;
#pragma unroll
    for (int d = 1; d < C; d *= 2) {
      const double o = __shfl_up_sync(0xffffffffu, gs, d);
      if (lane >= d) gs += o;
    }
    if (lane < C) {
      const float high = (float)gs;
      vec[C * kGHigh + lane] = high;
      vec[C * kGLow + lane] = (float)(gs - high);
      vec[C * kBeta + lane] = bt;
      vec[C * kDlog + lane] = dl;
    }
  }
  cp_wait_all();
  __syncthreads();
  for (int r = warp; r < 2 * C; r += 4) {      // reciprocal lengths
    const float *row = sm + r * PK;
    float s = 0.f;
    for (int f = lane; f < K; f += 32) s = fmaf(row[f], row[f], s);
#pragma unroll
    for (int d = 16; d; d /= 2) s += __shfl_xor_sync(0xffffffffu, s, d);
    if (lane == 0) vec[C * (r < C ? kVecRk : kVecRq) + r % C] = !a.qk_norm ? 1.f : r % C < have ? 1.f / sqrtf(s + a.eps) : 0.f;      // (rows behind the last token: eps may be 0)
  }
  __syncthreads();
  float *rec = reinterpret_cast<float *>(a.rec) + ((size_t)(sp.slot0 + ch) * a.N + n) * kRec;
  if (tid < C) {
    const double gs = sum_at(vec, tid);
    const float eg = exp_of(gs), el = exp_of(sum_at(vec, C - 1) - gs), rk = vec[C * kVecRk + tid], rq = vec[C * kVecRq + tid];
    vec[C * kVecEgk + tid] = eg * rk;
    vec[C * kVecEq + tid] = a.scale * eg * rq;
    vec[C * kEg + tid] = eg;
    vec[C * kEl + tid] = el;
    vec[C * kVecEk + tid] = el * rk;
  }
  for (int x = tid; x < 2 * C * C; x += 128) {
    const int i = x / C % C, j = x % C;
    const bool p = x >= C * C;
    float s = 0.f;
    if (p ? j <= i : j < i) {
      const float4 *r = reinterpret_cast<const float4 *>((p ? qs : ks) + i * PK), *o = reinterpret_cast<const float4 *>(ks + j * PK);
      float s0 = 0.f, s1 = 0.f;
      for (int f = 0; f < K / 4; ++f) {
        const float4 u = r[f], w = o[f];
        s0 = fmaf(u.x, w.x, fmaf(u.y, w.y, s0));
        s1 = fmaf(u.z, w.z, fmaf(u.w, w.w, s1));
      }
      s = (s0 + s1) * exp_of(sum_at(vec, i) - sum_at(vec, j)) * vec[C * kVecRk + j] *
          (p ? a.scale * vec[C * kVecRq + i] : vec[C * kBeta + i] * vec[C * kVecRk + i]);
    }
    rec[(p ? kP : kM) + i * C + j] = s;
    if (!p) Ms[i * (C + 4) + j] = s;
  }
  __syncthreads();
  if (tid < C) {      // column tid of T
    float t[C];
#pragma unroll
    for (int i = 0; i < C; ++i) {
      float s = i == tid ? 1.f : 0.f;
#pragma unroll
      for (int m = 0; m < i; ++m) s = fmaf(-Ms[i * (C + 4) + m], t[m], s);
      t[i] = s;
    }
#pragma unroll
    for (int i = 0; i < C; ++i) rec[kT + i * C + tid] = t[i];
  }
  for (int x = tid; x < 11 * C; x += 128) rec[kVec + x] = vec[x];
}

// ---- chains

__device__ __forceinline__ float load_state(const void *p, size_t x, int bf16) {
  return bf16 ? __bfloat162float(static_cast<const __nv_bfloat16 *>(p)[x]) : static_cast<const float *>(p)[x];
}
__device__ __forceinline__ void store_state(void *p, size_t x, int bf16, float v) {
  if (bf16) static_cast<__nv_bfloat16 *>(p)[x] = __float2bfloat16_rn(v);
  else static_cast<float *>(p)[x] = v;
}

// M adjacent floats
template <int M> __device__ __forceinline__ void rows_of(const float *p, float (&x)[M]) {
  if constexpr (M % 4 == 0) {
#pragma unroll
    for (int i = 0; i < M; i += 4) { const float4 v = *reinterpret_cast<const float4 *>(p + i); x[i] = v.x; x[i + 1] = v.y; x[i + 2] = v.z; x[i + 3] = v.w; }
  } else if constexpr (M % 2 == 0) {
#pragma unroll
    for (int i = 0; i < M; i += 2) { const float2 v = *reinterpret_cast<const float2 *>(p + i); x[i] = v.x; x[i + 1] = v.y; }
  } else {
#pragma unroll
    for (int i = 0; i < M; ++i) x[i] = p[i];
  }
}
template <int M> __device__ __forceinline__ void rows_to(float *p, const float (&x)[M]) {
  if constexpr (M % 4 == 0) {
#pragma unroll
    for (int i = 0; i < M; i += 4) *reinterpret_cast<float4 *>(p + i) = make_float4(x[i], x[i + 1], x[i + 2], x[i + 3]);
  } else if constexpr (M % 2 == 0) {
#pragma unroll
    for (int i = 0; i < M; i += 2) *reinterpret_cast<float2 *>(p + i) = make_float2(x[i], x[i + 1]);
  } else {
#pragma unroll
    for (int i = 0; i < M; ++i) p[i] = x[i];
  }
}
// Sums of p[t] over the sixteen lanes of a column; lane t keeps p[t]'s
template <int H> __device__ __forceinline__ float halve(const float (&p)[2 * H], int l) {
  const bool up = l & H;
  float q[H];
#pragma unroll
  for (int i = 0; i < H; ++i) {
    const float send = up ? p[i] : p[H + i], keep = up ? p[H + i] : p[i];
    q[i] = keep + __shfl_xor_sync(0xffffffffu, send, H);
  }
  if constexpr (H > 1) return halve<H / 2>(q, l);
  else return q[0];
}
// token t's product rows . S of this lane's column
template <int M> __device__ __forceinline__ float dots(const float *rows, int pitch, const float (&S)[M], int l) {
  float p[C];
#pragma unroll
  for (int t = 0; t < C; ++t) {
    float x[M];
    rows_of<M>(rows + t * pitch + M * l, x);
    p[t] = 0.f;
#pragma unroll
    for (int m = 0; m < M; ++m) p[t] = fmaf(x[m], S[m], p[t]);
  }
  return halve<C / 2>(p, l);
}

constexpr int kStages = 4, kPM = 20;      // pitch of T and P in shared memory: rows as float4 and columns without conflicts
// Shared memory of a stage (floats): k, q rows, T, P, vectors, nc columns of v (dy)
constexpr int kSP = C * kPM, kSVec = 2 * C * kPM, kSRec = kSVec + 8 * C;
__host__ __device__ constexpr int f32_stage(int K, int nc) { return 2 * C * K + kSRec + C * nc; }

// The copying warp's loop; nc (columns of the CTA) 4, 8 or 16.  A lane has a place in a row for good.
template <int K>
__device__ __forceinline__ void f32_fill(const DeltaArgs &a, const DeltaSpan &sp, int n, int col0, int nc, float *ring, const float *vg, long long vs, uint64_t *full,
                                         uint64_t *empty, int lane, bool backward) {
  constexpr int P = K / 4, LR = P % 32 == 0 ? 32 : P % 16 == 0 ? 16 : P % 8 == 0 ? 8 : 4, RP = 32 / LR;      // pieces, lanes to a row; rows to a pass
  const int lv = nc / 4, rv = 32 / lv, r0 = lane / LR, rv0 = lane / lv;
  const float *kp = static_cast<const float *>(a.k) + (sp.tok0 + r0) * a.ks + n / a.per_k * K + 4 * (lane % LR);
  const float *qp = static_cast<const float *>(a.q) + (sp.tok0 + r0) * a.qs + n / a.per_q * K + 4 * (lane % LR);
  const float *vp = vg + (sp.tok0 + rv0) * vs + (long long)n * a.V + col0 + 4 * (lane % lv);
  const float *rp = reinterpret_cast<const float *>(a.rec) + ((size_t)sp.slot0 * a.N + n) * kRec + 4 * lane;
  for (int i = 0; i < sp.n; ++i) {
    const int ch = backward ? sp.n - 1 - i : i, st = i % kStages, have = min(C, sp.T - ch * C);
    if (i >= kStages && !mbar_wait<64>(empty + st, (uint32_t)((i / kStages - 1) & 1))) {
      if (lane == 0) report_timeout(a.dev_status);
      for (int o = i - kStages; o < i; ++o) (void)mbar_wait(full + o % kStages, (uint32_t)((o / kStages) & 1));   // its copies on their way
      return;
    }
    float *base = ring + st * f32_stage(K, nc), *sr = base + 2 * C * K;
    const uint32_t kd = smem_u32(base + r0 * K + 4 * (lane % LR));
    const float *ks = kp + (long long)ch * C * a.ks, *qs = qp + (long long)ch * C * a.qs, *vv = vp + (long long)ch * C * vs, *rs = rp + (size_t)ch * a.N * kRec;
#pragma unroll
    for (int p = 0; p < C / RP; ++p, ks += RP * a.ks, qs += RP * a.qs) {
      const bool ok = r0 + p * RP < have;      // rows behind the last token are zeros
#pragma unroll
      for (int x = 0; x < P / LR; ++x) {
        cp16_or_zero(kd + 4 * (p * RP * K + 4 * LR * x), ok ? ks + 4 * LR * x : static_cast<const float *>(a.k), ok);
        cp16_or_zero(kd + 4 * ((C + p * RP) * K + 4 * LR * x), ok ? qs + 4 * LR * x : static_cast<const float *>(a.q), ok);
      }
    }
#pragma unroll
    for (int x = 0; x < 4; ++x) cp16(smem_u32(sr + (8 * x + (lane >> 2)) * kPM + 4 * (lane & 3)), rs + 128 * x);      // (T, then P)
    cp16(smem_u32(sr + kSVec + 4 * lane), rs + kVec);
#pragma unroll 1
    for (int r = rv0; r < C; r += rv, vv += rv * vs) cp16_or_zero(smem_u32(sr + kSRec + r * nc + 4 * (lane % lv)), r < have ? vv : vg, r < have);
    cp_arrive(full + st);
  }
}

template <int M, bool BWD>
__global__ void __launch_bounds__(288) delta_chain_f32_kernel(DeltaArgs a, int nc) {
  extern __shared__ __align__(16) float sm[];
  __shared__ uint64_t full[kStages], empty[kStages];
  if (threadIdx.x == 0) {
    for (int i = 0; i < kStages; ++i) { mbar_init(full + i, 32); mbar_init(empty + i, nc / 2); }
    fence_mbar_init();
  }
  begin_dependent();
  __syncthreads();
  constexpr int K = 16 * M;
  const int V = a.V, slabs = V / nc, lane = threadIdx.x & 31, l = lane & 15, base = lane & 16;
  const int unit = blockIdx.x / slabs, b = unit / a.N, n = unit % a.N, col0 = blockIdx.x % slabs * nc, mine = threadIdx.x / 16, v = col0 + mine;
  const DeltaSpan sp = delta_span<C>(a, b);
  if (mine >= nc) {      // (the last warp)
    f32_fill<K>(a, sp, n, col0, nc, sm, static_cast<const float *>(BWD ? a.dy : a.v), BWD ? (long long)a.N * V : a.vs, full, empty, lane, BWD);
    return;
  }
  const size_t at = ((size_t)b * a.N + n) * K * V + v;
  const void *in = BWD ? a.d_hT : a.h0;
  void *out = BWD ? a.dh0 : a.hT;
  float S[M];      // rows M l ..
#pragma unroll
  for (int m = 0; m < M; ++m) S[m] = in ? load_state(in, at + (size_t)(M * l + m) * V, a.state_bf16) : 0.f;
  for (int i = 0; i < sp.n; ++i) {
    const int ch = BWD ? sp.n - 1 - i : i, st = i % kStages, have = min(C, sp.T - ch * C);
    if (!mbar_wait(full + st, (uint32_t)((i / kStages) & 1))) {
      if (lane == 0) report_timeout(a.dev_status);
      return;
    }
    const float *ks = sm + st * f32_stage(K, nc), *qs = ks + C * K, *rec = qs + C * K, *vec = rec + kSVec, *vt = rec + kSRec;
    const long long tok = sp.tok0 + ch * C;
    const size_t slot = (size_t)(sp.slot0 + ch) * a.N + n;
    const float x0 = vt[l * nc + mine], ec = vec[C * kEg + C - 1];
    float *states = reinterpret_cast<float *>(BWD ? a.dstates : a.states);
    if (states) rows_to<M>(states + slot * K * V + (size_t)v * K + M * l, S);
    if constexpr (!BWD) {
      float T[C], P[C];      // this lane's token's rows
      rows_of<C>(rec + l * kPM, T);
      rows_of<C>(rec + kSP + l * kPM, P);
      const float x = vec[C * kBeta + l] * fmaf(-vec[C * kVecEgk + l], dots<M>(ks, K, S, l), x0);
      float u = 0.f;
#pragma unroll
      for (int j = 0; j < C; ++j) u = fmaf(T[j], __shfl_sync(0xffffffffu, x, base + j), u);      // (T_lj = 0 for j > l)
      float y = 0.f;
      if (a.y) y = vec[C * kVecEq + l] * dots<M>(qs, K, S, l);
      const float qS = y;
#pragma unroll
      for (int m = 0; m < M; ++m) S[m] *= ec;
#pragma unroll
      for (int j = 0; j < C; ++j) {
        const float uj = __shfl_sync(0xffffffffu, u, base + j), e = uj * vec[C * kVecEk + j];
        y = fmaf(P[j], uj, y);
        float k[M];
        rows_of<M>(ks + j * K + M * l, k);
#pragma unroll
        for (int m = 0; m < M; ++m) S[m] = fmaf(k[m], e, S[m]);
      }
      // 0 x NaN above carried a token's NaN to the tokens before it: y without them.  (S has it in the whole column either way.)
      if (__any_sync(0xffffffffu, !(fabsf(u) < __int_as_float(0x7f800000)))) {
        u = 0.f;
        y = qS;
        for (int j = 0; j < C; ++j) {
          const float xj = __shfl_sync(0xffffffffu, x, base + j);
          if (j <= l) u = fmaf(rec[l * kPM + j], xj, u);
        }
        for (int j = 0; j < C; ++j) {
          const float uj = __shfl_sync(0xffffffffu, u, base + j);
          if (j <= l) y = fmaf(rec[kSP + l * kPM + j], uj, y);
        }
      }
      if (a.y && l < have) static_cast<float *>(a.y)[((size_t)(tok + l) * a.N + n) * V + v] = y;
      if (a.upd) reinterpret_cast<float *>(a.upd)[slot * C * V + l * V + v] = u;
    } else {
      // x0: dY
      float du = vec[C * kVecEk + l] * dots<M>(ks, K, S, l);
#pragma unroll
      for (int i2 = 0; i2 < C; ++i2) du = fmaf(rec[kSP + i2 * kPM + l], __shfl_sync(0xffffffffu, x0, base + i2), du);      // (P_il = 0 for i < l)
      float L = 0.f;
#pragma unroll
      for (int i2 = 0; i2 < C; ++i2) L = fmaf(rec[i2 * kPM + l], __shfl_sync(0xffffffffu, du, base + i2), L);
      const float dv = vec[C * kBeta + l] * L;
      if (l < have) static_cast<float *>(a.dv)[((size_t)(tok + l) * a.N + n) * V + v] = dv;
      reinterpret_cast<float *>(a.lam)[slot * C * V + l * V + v] = L;
      const float e = vec[C * kVecEq + l] * x0, f = -vec[C * kVecEgk + l] * dv;
#pragma unroll
      for (int m = 0; m < M; ++m) S[m] *= ec;
#pragma unroll
      for (int j = 0; j < C; ++j) {
        const float ej = __shfl_sync(0xffffffffu, e, base + j), fj = __shfl_sync(0xffffffffu, f, base + j);
        float k[M], q[M];
        rows_of<M>(ks + j * K + M * l, k);
        rows_of<M>(qs + j * K + M * l, q);
#pragma unroll
        for (int m = 0; m < M; ++m) S[m] = fmaf(q[m], ej, fmaf(k[m], fj, S[m]));
      }
    }
    __syncwarp();
    if (lane == 0) mbar_arrive(empty + st);
  }
  if (out)
#pragma unroll
    for (int m = 0; m < M; ++m) store_state(out, at + (size_t)(M * l + m) * V, a.state_bf16, S[m]);
}

// ---- grad

constexpr int kThreads = 256;
// Shared memory (floats): S, dS' [V][K]; dY, L, U [V][kPM]; k, q [C][K + 1]; five arrays [C][K + 1]; four matrices; the vectors; sums
__host__ __device__ constexpr int grad_floats(int K, int V) { return 2 * K * V + 3 * V * kPM + 7 * C * (K + 1) + 4 * C * C + 11 * C + 8 * C + 16; }
static_assert(grad_floats(128, 128) * 4 <= 227 * 1024, "");

__global__ void __launch_bounds__(kThreads) delta_grad_f32_kernel(DeltaArgs a) {
  extern __shared__ __align__(16) float sm[];
  begin_dependent();
  const int K = a.K, V = a.V, PK = K + 1, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const unsigned at = blockIdx.x / (unsigned)a.N;
  const int n = (int)(blockIdx.x - at * a.N), b = a.cu ? delta_entry<C, true>(a, at) : delta_entry<C, false>(a, at);
  const DeltaSpan sp = delta_span<C>(a, b);
  const int ch = (int)(at - sp.slot0);
  if ((unsigned)ch >= (unsigned)sp.n) return;      // (of a packed batch: a slot that is no sequence's)
  const long long tok = sp.tok0 + ch * C;
  const int have = min(C, sp.T - ch * C);
  const size_t slot = (size_t)(sp.slot0 + ch) * a.N + n;
  float *S = sm, *D = S + K * V, *yt = D + K * V, *lt = yt + V * kPM, *ut = lt + V * kPM;
  float *XP = ut + V * kPM, *XPt = XP + C * C, *XN = XPt + C * C, *XNt = XN + C * C, *vec = XNt + C * C, *sums = vec + 11 * C;
  float *ks = sums + 8 * C + 16, *qs = ks + C * PK, *m0 = qs + C * PK;      // five arrays from m0: dQ^, dK-, dK+, and R's and W's parts
  const float *rec = reinterpret_cast<const float *>(a.rec) + slot * kRec;
  {
    const float *sg = reinterpret_cast<const float *>(a.states) + slot * K * V, *dg = reinterpret_cast<const float *>(a.dstates) + slot * K * V;
    for (int x = tid; x < K * V / 4; x += kThreads) {
      cp16(smem_u32(S + 4 * x), sg + 4 * x);
      cp16(smem_u32(D + 4 * x), dg + 4 * x);
    }
    if (tid < 11 * C / 4) cp16(smem_u32(vec + 4 * tid), rec + kVec + 4 * tid);
    const float *yg = static_cast<const float *>(a.dy) + ((size_t)tok * a.N + n) * V;
    const float *ug = reinterpret_cast<const float *>(a.upd) + slot * C * V, *lg = reinterpret_cast<const float *>(a.lam) + slot * C * V;
    const int log_v = 31 - __clz(V);
    for (int x = tid; x < C * V; x += kThreads) {
      const int r = x >> log_v, v = x & (V - 1);
      yt[v * kPM + r] = r < have ? yg[(size_t)r * a.N * V + v] : 0.f;
      ut[v * kPM + r] = ug[x];
      lt[v * kPM + r] = lg[x];
    }
    const float *kg = static_cast<const float *>(a.k) + tok * a.ks + (long long)(n / (a.N / a.Nk)) * K;
    const float *qg = static_cast<const float *>(a.q) + tok * a.qs + (long long)(n / (a.N / a.Nq)) * K;
    for (int x = tid; x < C * K; x += kThreads) {
      const int r = x / K, f = x % K;
      ks[r * PK + f] = r < have ? kg[r * a.ks + f] : 0.f;
      qs[r * PK + f] = r < have ? qg[r * a.qs + f] : 0.f;
    }
    cp_wait_all();
  }
  __syncthreads();
  float ss = 0.f;      // <S, dS'>
  for (int x = tid; x < K * V; x += kThreads) ss = fmaf(S[x], D[x], ss);
#pragma unroll
  for (int o = 16; o; o /= 2) ss += __shfl_xor_sync(0xffffffffu, ss, o);
  if (lane == 0) sums[8 * C + warp] = ss;
  // dP, N: one entry a thread; G
  {
    const int i = tid / C, j = tid % C;
    float p = 0.f, m = 0.f, gg = 0.f, xp = 0.f, xn = 0.f;
    if (j <= i) {
      for (int v = 0; v < V; ++v) {
        p = fmaf(yt[v * kPM + i], ut[v * kPM + j], p);
        m = fmaf(-lt[v * kPM + i], ut[v * kPM + j], m);
      }
      const float e = exp_of(sum_at(vec, i) - sum_at(vec, j));
      xp = a.scale * e * p;
      if (j < i) {
        xn = e * m;
        gg = fmaf(rec[kP + i * C + j], p, rec[kM + i * C + j] * m);
      }
    }
    XP[i * C + j] = XPt[j * C + i] = xp;
    XN[i * C + j] = XNt[j * C + i] = xn;
    // sums of G's rows (a half warp has one), and of its columns through shared memory
    float r = gg;
#pragma unroll
    for (int o = 8; o; o /= 2) r += __shfl_xor_sync(0xffffffffu, r, o);
    if (j == 0) sums[5 * C + i] = r;
    m0[i * PK + j] = gg;
  }
  __syncthreads();
  if (tid < C) {
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < C; ++i) s += m0[i * PK + tid];
    sums[6 * C + tid] = s;
  }
  __syncthreads();
  const int AR = C * PK;      // one of the five arrays
  for (int x = tid; x < 4 * K; x += kThreads) {
    const int f = x % K, i0 = 4 * (x / K);
    float y[4] = {}, ls[4] = {}, us[4] = {};
    for (int v = 0; v < V; ++v) {
      const float s = S[v * K + f], d = D[v * K + f];
      const float4 y4 = *reinterpret_cast<const float4 *>(yt + v * kPM + i0), l4 = *reinterpret_cast<const float4 *>(lt + v * kPM + i0), u4 = *reinterpret_cast<const float4 *>(ut + v * kPM + i0);
      const float yy[4] = {y4.x, y4.y, y4.z, y4.w}, ll[4] = {l4.x, l4.y, l4.z, l4.w}, uu[4] = {u4.x, u4.y, u4.z, u4.w};
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        y[e] = fmaf(yy[e], s, y[e]);
        ls[e] = fmaf(ll[e], s, ls[e]);
        us[e] = fmaf(uu[e], d, us[e]);
      }
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int i = i0 + e;
      const float rk = vec[C * kVecRk + i], rq = vec[C * kVecRq + i];
      y[e] *= a.scale * vec[C * kEg + i];
      ls[e] *= -vec[C * kEg + i];
      us[e] *= vec[C * kEl + i];
      m0[3 * AR + i * PK + f] = fmaf(rq * qs[i * PK + f], y[e], vec[C * kBeta + i] * rk * ks[i * PK + f] * ls[e]);
      m0[4 * AR + i * PK + f] = rk * ks[i * PK + f] * us[e];
    }
    for (int j = 0; j < C; ++j) {
      const float kj = ks[j * PK + f], kr = vec[C * kVecRk + j] * kj, kb = vec[C * kBeta + j] * kr, qr = vec[C * kVecRq + j] * qs[j * PK + f];
      const float4 a4 = *reinterpret_cast<const float4 *>(XPt + j * C + i0), b4 = *reinterpret_cast<const float4 *>(XNt + j * C + i0);
      const float4 c4 = *reinterpret_cast<const float4 *>(XP + j * C + i0), d4 = *reinterpret_cast<const float4 *>(XN + j * C + i0);
      const float aa[4] = {a4.x, a4.y, a4.z, a4.w}, bb[4] = {b4.x, b4.y, b4.z, b4.w}, cc[4] = {c4.x, c4.y, c4.z, c4.w}, dd[4] = {d4.x, d4.y, d4.z, d4.w};
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        y[e] = fmaf(aa[e], kr, y[e]);
        ls[e] = fmaf(bb[e], kr, ls[e]);
        us[e] = fmaf(cc[e], qr, fmaf(dd[e], kb, us[e]));
      }
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      m0[(i0 + e) * PK + f] = y[e];
      m0[AR + (i0 + e) * PK + f] = ls[e];
      m0[2 * AR + (i0 + e) * PK + f] = us[e];
    }
  }
  __syncthreads();
  for (int i = warp; i < C; i += kThreads / 32) {      // q^ . dQ^, k^ . dK-, k^ . dK+, R, W, L . v
    float d[6] = {};
    for (int f = lane; f < K; f += 32) {
      const float q = vec[C * kVecRq + i] * qs[i * PK + f], k = vec[C * kVecRk + i] * ks[i * PK + f];
      d[0] = fmaf(q, m0[i * PK + f], d[0]);
      d[1] = fmaf(k, m0[AR + i * PK + f], d[1]);
      d[2] = fmaf(k, m0[2 * AR + i * PK + f], d[2]);
      d[3] += m0[3 * AR + i * PK + f];
      d[4] += m0[4 * AR + i * PK + f];
    }
    if (i < have) {
      const float *vg = static_cast<const float *>(a.v) + (tok + i) * a.vs + (long long)n * V;
      for (int v = lane; v < V; v += 32) d[5] = fmaf(lt[v * kPM + i], vg[v], d[5]);
    }
#pragma unroll
    for (int m = 0; m < 6; ++m) {
#pragma unroll
      for (int o = 16; o; o /= 2) d[m] += __shfl_xor_sync(0xffffffffu, d[m], o);
      if (lane == 0) sums[C * (m < 5 ? m : 7) + i] = d[m];
    }
  }
  __syncthreads();
  if (warp == 0) {
    const int i = lane & (C - 1);
    const float w = sums[4 * C + i];
    float all = lane < C ? w : 0.f, part = lane < C ? sums[3 * C + i] + sums[5 * C + i] - w - sums[6 * C + i] : 0.f, sd = lane < kThreads / 32 ? sums[8 * C + lane] : 0.f;
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
      float db;
      (void)delta_step_of(a.step_kind, static_cast<const float *>(a.step)[x], db);
      static_cast<float *>(a.dgate)[x] = (part + all + vec[C * kEg + C - 1] * sd) * vec[C * kDlog + lane];
      static_cast<float *>(a.dstep)[x] = (sums[7 * C + lane] + sums[C + lane]) * db;
    }
  }
  // dq, dk through the division by the lengths
  for (int x = tid; x < have * K; x += kThreads) {
    const int i = x / K, f = x % K;
    const float bt = vec[C * kBeta + i], rk = vec[C * kVecRk + i], rq = vec[C * kVecRq + i];
    float dq = m0[i * PK + f], dk = fmaf(bt, m0[AR + i * PK + f], m0[2 * AR + i * PK + f]);
    if (a.qk_norm) {
      dq = rq * fmaf(-rq * qs[i * PK + f], sums[i], dq);
      dk = rk * fmaf(-rk * ks[i * PK + f], fmaf(bt, sums[C + i], sums[2 * C + i]), dk);
    }
    const size_t t = (size_t)(tok + i);
    (a.dq_part ? a.dq_part : static_cast<float *>(a.dq))[(t * a.N + n) * K + f] = dq;      // (N shares, or N heads)
    (a.dk_part ? a.dk_part : static_cast<float *>(a.dk))[(t * a.N + n) * K + f] = dk;
  }
}

template <int M, bool BWD> cudaError_t chain_m(const DeltaArgs &a, cudaStream_t s) {
  // columns of a CTA: sixteen, fewer where that leaves SMs without one
  const long long units = (long long)a.B * a.N;
  int nc = 16;
  while (nc > 4 && units * (a.V / nc) < sm_count()) nc /= 2;
  const size_t smem = (size_t)kStages * f32_stage(a.K, nc) * sizeof(float);
  const cudaError_t e = allow_smem(delta_chain_f32_kernel<M, BWD>, smem);
  if (e != cudaSuccess) return e;
  return launch_early(delta_chain_f32_kernel<M, BWD>, dim3((unsigned)(units * (a.V / nc))), dim3(16 * nc + 32), smem, s, a, nc);
}
template <bool BWD> cudaError_t chain(const DeltaArgs &a, cudaStream_t s) {
  switch (a.K) {
    case 16: return chain_m<1, BWD>(a, s);
    case 32: return chain_m<2, BWD>(a, s);
    case 48: return chain_m<3, BWD>(a, s);
    case 64: return chain_m<4, BWD>(a, s);
    case 80: return chain_m<5, BWD>(a, s);
    case 96: return chain_m<6, BWD>(a, s);
    case 112: return chain_m<7, BWD>(a, s);
    default: return chain_m<8, BWD>(a, s);
  }
}

}  // namespace

cudaError_t launch_delta_fwd_f32(const DeltaArgs &a, cudaStream_t s) {
  const size_t smem = (size_t)(2 * C * (a.K + 4) + C * (C + 4) + 11 * C) * sizeof(float);
  const cudaError_t e = launch_early(delta_prep_f32_kernel, dim3((unsigned)(a.slots * a.N)), dim3(128), smem, s, a);
  return e != cudaSuccess ? e : chain<false>(a, s);
}
cudaError_t launch_delta_bwd_f32(const DeltaArgs &a, cudaStream_t s) {
  cudaError_t e = chain<true>(a, s);
  const size_t smem = (size_t)grad_floats(a.K, a.V) * sizeof(float);
  if (e == cudaSuccess) e = allow_smem(delta_grad_f32_kernel, smem);
  return e != cudaSuccess ? e : launch_early(delta_grad_f32_kernel, dim3((unsigned)(a.slots * a.N)), dim3(kThreads), smem, s, a);
}

}  // namespace m2rnn
