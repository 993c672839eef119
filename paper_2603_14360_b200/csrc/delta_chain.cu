// Gated delta rule, bf16: the two chains over the chunks of a sequence, forward and backward.
//
// With S the K x V state at a chunk's start, T and P of delta_prep.cu, and per token the factors of DeltaVec,
//     X = b (V - e^g K^ S)      U = T X      Y = s e^g Q^ S + P U      S' = e^g_last S + (e^(g_last - g) K^)^T U
// and backward, from dS' at a chunk's end (K^, Q^: the rows divided by their lengths),
//     dU = P^T dY + e^(g_last - g) K^ dS'      L = T^T dU      dV = b L
//     dS = e^g_last dS' + (s e^g Q^)^T dY - (e^g K^)^T dV
// Columns of S are independent recurrences: a warp owns 16 of them and walks the chunks alone.  Everything it holds is
// transposed, S^T [16 x K] as accumulators of mma.sync m16n8k16: an accumulator tile has the thread <-> element map of
// the next product's A operand, so S, X, U (and dS, dU, L) never leave registers.  K, Q, V, dY, T and P come as B
// operands (V, dY as accumulators and A operands) from a ring of shared-memory stages that one warp fills:
// a record by one untiled bulk copy, rows by cp.async, padded to an odd number of 16 bytes so that ldmatrix has no
// conflicts.  (Rows by bulk copies, one a lane, were bound by the copies' number: 3.4 us a chunk of K = V = 64.)
// A chunk's chain is S -> X -> U -> S', each step a product whose last results the next one waits for.  What is not on it fills the
// waits: forward the products of the chunk before's Y (S and U of that chunk as operands from shared memory), backward those with Q.
// (Y after its own chunk's chain: 1 680 cycles a chunk of K = 64 for a warp alone; Y in warps of its own: as much registers as the
// chains have, so half the chains to an SM.)
// Roundings to bf16: the operands S, X, U (dS, dU, L), the factored e^(g_last - g) U and the like, and T and P.  S itself
// is held and updated in fp32.
#include "delta_common.cuh"

namespace m2rnn {
namespace {

constexpr int C = kDeltaChunk;

// Bytes of a stage: K, Q rows, rows of 16 nw columns of V (dY), nw / wv records
__host__ __device__ constexpr int pitch_k(int K) { return 2 * K + 16; }
__host__ __device__ constexpr int pitch_v(int nw) { return 32 * nw + 16; }
__host__ __device__ constexpr int stage_bytes(int K, int nw, int heads) { return C * (2 * pitch_k(K) + pitch_v(nw)) + heads * kRecChain; }

// A chain warp's results on their way out: S as an operand and U (dS, L), blocks as they lie in memory; two of them
constexpr int kOuts = 2;
__host__ __device__ constexpr int out_bytes(int K) { return 32 * K + 1024; }

struct ChainPlan { int hpc, wv, slabs, stages; size_t smem; };

// What a CTA has to do: batch entry, heads n0 .. n0 + hpc, columns from col0 on (of head n0)
struct ChainWork { int b, n0, slab; };
__device__ __forceinline__ ChainWork chain_work(const DeltaArgs &a, void *scratch) {
  const int slabs = a.V / (16 * a.wv), per = (a.N / a.hpc) * slabs;
  ChainWork w;
  w.b = (int)(blockIdx.x / per);
  const int r = (int)(blockIdx.x % per);
  w.n0 = r / slabs * a.hpc;
  w.slab = r % slabs;
  return w;
}

// The copying warp's loop, in the order that `backward` says.  vg: the tensor whose columns the warps own.  It has a chunk's time
// for some 40 copies an instruction each and their addresses (with the address of each worked out from its number it was what bound
// the chains, 1.1 us a chunk of K = 128): a lane has a place in a row for good, passes are a fixed number of rows apart.
template <int K>
__device__ __forceinline__ void chain_fill(const DeltaArgs &a, const ChainWork &w, const DeltaSpan &sp, const void *vg, long long vs, int nw, int stages, uint32_t ring,
                                           uint64_t *full, uint64_t *empty, int lane, bool backward) {
  constexpr int P = K / 8, LR = P % 16 == 0 ? 16 : P % 8 == 0 ? 8 : P % 4 == 0 ? 4 : 2, RP = 32 / LR;      // pieces, lanes to a row; rows to a pass
  const int pv = pitch_v(nw), lv = 2 * nw, rv = 32 / lv;                                                    // of v: lanes to a row, rows to a pass
  const uint32_t sb = (uint32_t)stage_bytes(K, nw, a.hpc);
  const int r0 = lane / LR, rv0 = lane / lv;
  const char *kp = static_cast<const char *>(a.k) + 2 * ((sp.tok0 + r0) * a.ks + w.n0 / a.per_k * K) + 16 * (lane % LR);
  const char *qp = static_cast<const char *>(a.q) + 2 * ((sp.tok0 + r0) * a.qs + w.n0 / a.per_q * K) + 16 * (lane % LR);
  const char *vp = static_cast<const char *>(vg) + 2 * ((sp.tok0 + rv0) * vs + (long long)w.n0 * a.V + w.slab * 16 * a.wv) + 16 * (lane % lv);
  const long long kc = 2 * C * a.ks, qc = 2 * C * a.qs, vc = 2 * C * vs, kr = 2 * RP * a.ks, qr = 2 * RP * a.qs, vr = 2 * rv * vs;      // bytes to the next chunk, the next pass
  const uint32_t k_at = r0 * pitch_k(K) + 16 * (lane % LR), v_at = 2 * C * pitch_k(K) + rv0 * pv + 16 * (lane % lv);
  const size_t rec_step = (size_t)a.N * kRecBytes;
  const char *rp = a.rec + ((size_t)sp.slot0 * a.N + w.n0) * kRecBytes;
  if (backward) {
    kp += (sp.n - 1) * kc; qp += (sp.n - 1) * qc; vp += (sp.n - 1) * vc; rp += (sp.n - 1) * rec_step;
  }
  int st = 0;
  uint32_t phase = 1;      // (the first pass over the stages waits for nothing)
  for (int i = 0; i < sp.n; ++i) {
    const int have = backward ? min(C, sp.T - (sp.n - 1 - i) * C) : min(C, sp.T - i * C);
    if (i >= stages && !mbar_wait<64>(empty + st, phase)) {
      if (lane == 0) report_timeout(a.dev_status);
      for (int o = i - stages; o < i; ++o) (void)mbar_wait(full + o % stages, (uint32_t)((o / stages) & 1));   // its copies on their way
      return;
    }
    const uint32_t base = ring + st * sb, kd = base + k_at, vd = base + v_at, rd = base + C * (2 * pitch_k(K) + pv);
    if (lane == 0) {
      mbar_expect(full + st, (uint32_t)(a.hpc * kRecChain));
      for (int h = 0; h < a.hpc; ++h) bulk_load(rd + h * kRecChain, rp + (size_t)h * kRecBytes, kRecChain, full + st);
    }
    const char *ks = kp, *qs = qp, *vv = vp;
    if (have == C) {
#pragma unroll
      for (int p = 0; p < LR; ++p, ks += kr, qs += qr)
#pragma unroll
        for (int x = 0; x < P / LR; ++x) {
          cp16(kd + p * RP * pitch_k(K) + 16 * LR * x, ks + 16 * LR * x);
          cp16(kd + (C + p * RP) * pitch_k(K) + 16 * LR * x, qs + 16 * LR * x);
        }
      for (int p = 0; p < lv; ++p, vv += vr) cp16(vd + p * rv * pv, vv);
    } else {      // the last tokens: rows behind them are zeros
#pragma unroll 1
      for (int p = 0; p < LR; ++p, ks += kr, qs += qr) {
        const bool ok = r0 + p * RP < have;
        for (int x = 0; x < P / LR; ++x) {
          cp16_or_zero(kd + p * RP * pitch_k(K) + 16 * LR * x, ok ? ks + 16 * LR * x : static_cast<const char *>(a.k), ok);
          cp16_or_zero(kd + (C + p * RP) * pitch_k(K) + 16 * LR * x, ok ? qs + 16 * LR * x : static_cast<const char *>(a.q), ok);
        }
      }
      for (int p = 0; p < lv; ++p, vv += vr) {
        const bool ok = rv0 + p * rv < have;
        cp16_or_zero(vd + p * rv * pv, ok ? vv : static_cast<const char *>(vg), ok);
      }
    }
    cp_arrive(full + st);
    if (backward) { kp -= kc; qp -= qc; vp -= vc; rp -= rec_step; }
    else { kp += kc; qp += qc; vp += vc; rp += rec_step; }
    if (++st == stages) { st = 0; phase ^= 1; }
  }
}

// S^T [16 columns from v0 on][K] between memory ([K][V], fp32 or bf16) and accumulators
template <int K>
__device__ __forceinline__ void state_in(float (&S)[K / 8][4], const void *p, size_t at, int bf16, int V, int g, int c) {
#pragma unroll
  for (int nt = 0; nt < K / 8; ++nt)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const size_t x = at + (size_t)(8 * nt + 2 * c + (r & 1)) * V + g + 8 * (r >> 1);
      S[nt][r] = bf16 ? __bfloat162float(static_cast<const __nv_bfloat16 *>(p)[x]) : static_cast<const float *>(p)[x];
    }
}
template <int K>
__device__ __forceinline__ void state_out(const float (&S)[K / 8][4], void *p, size_t at, int bf16, int V, int g, int c) {
#pragma unroll
  for (int nt = 0; nt < K / 8; ++nt)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const size_t x = at + (size_t)(8 * nt + 2 * c + (r & 1)) * V + g + 8 * (r >> 1);
      if (bf16) static_cast<__nv_bfloat16 *>(p)[x] = __float2bfloat16_rn(S[nt][r]);
      else static_cast<float *>(p)[x] = S[nt][r];
    }
}
// ldmatrix addresses of a lane
struct Lanes {
  uint32_t row, mat_lo, mat_hi;   // row of an 8 x 8 matrix, and which of two matrices in each direction
  __device__ explicit Lanes(int lane) : row(lane & 7), mat_lo((lane >> 3) & 1), mat_hi(lane >> 4) {}
};

// B operands are asked for kAhead at a time before they are needed
constexpr int kAhead = 4;
// acc[4 token tiles] += A (16 x K) . rows^T over k-tiles k0 .. k1: rows [32 tokens][K] in shared memory; `a` gives the A operand of k-tile kt
template <int K> struct RowsT {
  uint32_t at, b[kAhead][4];
  __device__ __forceinline__ void load(int x) { ldmatrix_x4(at + 16 * (x & 1) * pitch_k(K) + 32 * (x >> 1), b[x % kAhead]); }
  template <int K0, int K1> __device__ __forceinline__ void start(uint32_t rows, const Lanes &l) {
    at = rows + (l.row + 8 * l.mat_hi) * pitch_k(K) + 16 * l.mat_lo;
#pragma unroll
    for (int x = 2 * K0; x < 2 * K1 && x < 2 * K0 + kAhead; ++x) load(x);
  }
  template <int K0, int K1, typename A> __device__ __forceinline__ void run(float (&acc)[4][4], A a) {
#pragma unroll
    for (int kt = K0; kt < K1; ++kt) {
      uint32_t f[4];
      a(kt, f);
#pragma unroll
      for (int np = 0; np < 2; ++np) {
        const int x = 2 * kt + np;
        mma_add(acc[2 * np], f, b[x % kAhead][0], b[x % kAhead][1]);
        mma_add(acc[2 * np + 1], f, b[x % kAhead][2], b[x % kAhead][3]);
        if (x + kAhead < 2 * K1) load(x + kAhead);
      }
    }
  }
};
// S (16 x K) += A (16 x 32 tokens) . rows
template <int K> struct Rows {
  static constexpr int N = K / 16;      // pairs of feature tiles
  uint32_t at, b[kAhead][4];
  __device__ __forceinline__ void load(int x) { ldmatrix_x4_t(at + 16 * (x / N) * pitch_k(K) + 32 * (x % N), b[x % kAhead]); }
  __device__ __forceinline__ void start(uint32_t rows, const Lanes &l) {
    at = rows + (l.row + 8 * l.mat_lo) * pitch_k(K) + 16 * l.mat_hi;
#pragma unroll
    for (int x = 0; x < 2 * N && x < kAhead; ++x) load(x);
  }
  // k-tiles (16 tokens each) T0 .. T1
  template <int T0, int T1> __device__ __forceinline__ void run(float (&S)[K / 8][4], const uint32_t (&A)[2][4]) {
#pragma unroll
    for (int x = T0 * N; x < T1 * N; ++x) {
      const int np = x % N;
      mma_add(S[2 * np], A[x / N], b[x % kAhead][0], b[x % kAhead][1]);
      mma_add(S[2 * np + 1], A[x / N], b[x % kAhead][2], b[x % kAhead][3]);
      if (x + kAhead < 2 * N) load(x + kAhead);
    }
  }
};
// A lower triangular 32 x 32 matrix, blocks in shared memory, as B operands of a product with its transpose, or with itself
__device__ __forceinline__ void lower_t_in(uint32_t (&b)[3][4], uint32_t M, const Lanes &l) {
  const uint32_t at = M + 16 * l.row + 128 * (4 * l.mat_hi + l.mat_lo);
  ldmatrix_x4(at, b[0]);
  ldmatrix_x4(at + 128 * 8, b[1]);
  ldmatrix_x4(at + 128 * 10, b[2]);
}
__device__ __forceinline__ void lower_in(uint32_t (&b)[3][4], uint32_t M, const Lanes &l) {
  const uint32_t at = M + 16 * l.row + 128 * (4 * l.mat_lo + l.mat_hi);
  ldmatrix_x4_t(at, b[0]);
  ldmatrix_x4_t(at + 128 * 8, b[1]);
  ldmatrix_x4_t(at + 128 * 10, b[2]);
}
// acc (16 x 32) += A (16 x 32) . M^T
__device__ __forceinline__ void mul_lower_t(float (&acc)[4][4], const uint32_t (&A)[2][4], const uint32_t (&b)[3][4]) {
  mma_add(acc[0], A[0], b[0][0], b[0][1]);
  mma_add(acc[1], A[0], b[0][2], b[0][3]);
  mma_add(acc[2], A[0], b[1][0], b[1][1]);
  mma_add(acc[3], A[0], b[1][2], b[1][3]);
  mma_add(acc[2], A[1], b[2][0], b[2][1]);
  mma_add(acc[3], A[1], b[2][2], b[2][3]);
}
// acc (16 x 32) += A (16 x 32) . M
__device__ __forceinline__ void mul_lower(float (&acc)[4][4], const uint32_t (&A)[2][4], const uint32_t (&b)[3][4]) {
  mma_add(acc[0], A[0], b[0][0], b[0][1]);
  mma_add(acc[1], A[0], b[0][2], b[0][3]);
  mma_add(acc[2], A[1], b[2][0], b[2][1]);
  mma_add(acc[3], A[1], b[2][2], b[2][3]);
  mma_add(acc[0], A[1], b[1][0], b[1][1]);
  mma_add(acc[1], A[1], b[1][2], b[1][3]);
}
__device__ __forceinline__ void zero(float (&x)[4][4]) {
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) x[i][j] = 0.f;
}
// the 16 x 32 tile of a row tensor that a warp owns (transposed), as packed accumulators [token tile][column half]
__device__ __forceinline__ void rows_in(uint32_t (&p)[2][4], uint32_t at, int pv) {
  ldmatrix_x4_t(at, p[0]);
  ldmatrix_x4_t(at + 16 * pv, p[1]);
}
// A operand tiles (16 columns x 16 tokens or features) to blocks [column tile][tile], `n` tiles a column tile, from tile 2 kt on
__device__ __forceinline__ void blocks_out(const uint32_t (&f)[4], uint32_t at, int n, int kt, const Lanes &l) {
  stmatrix_x4(at + 16 * l.row + 128 * (l.mat_lo * n + 2 * kt + l.mat_hi), f);
}

// Barriers of a CTA: stages filled and free, and per chain warp results there and gone
struct ChainBars { uint64_t full[8], empty[8], there[4][kOuts], gone[4][kOuts]; };
__device__ __forceinline__ void chain_bars(ChainBars &b, int stages, int nw, int readers) {
  if (threadIdx.x == 0) {
    for (int i = 0; i < stages; ++i) { mbar_init(b.full + i, 33); mbar_init(b.empty + i, readers); }
    for (int w = 0; w < nw; ++w)
      for (int i = 0; i < kOuts; ++i) { mbar_init(&b.there[w][i], 1); mbar_init(&b.gone[w][i], 1); }
    fence_mbar_init();
  }
}
__device__ __forceinline__ void bulk_store(void *dst, uint32_t src, uint32_t bytes) {
  asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;" ::"l"(dst), "r"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void bulk_commit() { asm volatile("cp.async.bulk.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void bulk_wait_read() { asm volatile("cp.async.bulk.wait_group.read %0;" ::"n"(N) : "memory"); }
__device__ __forceinline__ void bulk_wait_all() { asm volatile("cp.async.bulk.wait_group 0;" ::: "memory"); }
__device__ __forceinline__ void fence_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// Both phases over (the second only if `also`): asked for together, which costs one round trip where neither has to be waited for
__device__ __forceinline__ bool wait_both(uint64_t *x, uint32_t px, uint64_t *y, uint32_t py, bool also) {
  const bool okx = mbar_try_wait(x, px), oky = !also || mbar_try_wait(y, py);
  if (__all_sync(0xffffffffu, okx && oky)) return true;
  return mbar_wait(x, px) && (!also || mbar_wait(y, py));
}

// Y: y is asked for; KEEP: states and updates are kept for the gradient
template <int K, bool Y, bool KEEP>
__global__ void __launch_bounds__(160, 2) delta_chain_fwd_kernel(DeltaArgs a, int stages) {
  extern __shared__ __align__(128) unsigned char smem[];
  __shared__ ChainBars bars;
  const int nw = a.hpc * a.wv, warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31, g = lane >> 2, c = lane & 3;
  chain_bars(bars, stages, 0, nw);
  begin_dependent();
  __syncthreads();
  const ChainWork w = chain_work(a, smem);
  const DeltaSpan sp = delta_span<C>(a, w.b);
  const uint32_t ring = smem_u32(smem), sb = (uint32_t)stage_bytes(K, nw, a.hpc);
  if (warp == nw) {
    chain_fill<K>(a, w, sp, a.v, a.vs, nw, stages, ring, bars.full, bars.empty, lane, false);
    return;
  }
  const int n = w.n0 + warp / a.wv, v0 = 16 * (w.slab * a.wv + warp % a.wv), V = a.V, pv = pitch_v(nw);
  const Lanes l(lane);
  const uint32_t outs = ring + stages * sb + warp * (kOuts * out_bytes(K));
  const uint32_t v_off = 2 * C * pitch_k(K), r_off = v_off + C * pv + (warp / a.wv) * kRecChain, v_at = v_off + 32 * warp + (l.row + 8 * l.mat_hi) * pv + 16 * l.mat_lo;
  const size_t st_at = ((size_t)w.b * a.N + n) * K * V + v0;
  float S[K / 8][4];
  if (a.h0) state_in<K>(S, a.h0, st_at, a.state_bf16, V, g, c);
  else
#pragma unroll
    for (int nt = 0; nt < K / 8; ++nt)
#pragma unroll
      for (int r = 0; r < 4; ++r) S[nt][r] = 0.f;
  __nv_bfloat16 *yg = Y ? static_cast<__nv_bfloat16 *>(a.y) + ((size_t)(sp.tok0 + lane) * a.N + n) * V + v0 : nullptr;
  char *sg = KEEP ? a.states + ((size_t)sp.slot0 * a.N + n) * (2 * K * V) + 2 * K * v0 : nullptr, *ug = KEEP ? a.upd + ((size_t)sp.slot0 * a.N + n) * (2 * C * V) + 2 * C * v0 : nullptr;
  // Y of a chunk from its stage and its results
  float y[4][4];
  auto y_states = [&](uint32_t stage, uint32_t out) {
    RowsT<K> yb;
    yb.template start<0, K / 16>(stage + C * pitch_k(K), l);
    zero(y);
    yb.template run<0, K / 16>(y, [&](int kt, uint32_t (&f)[4]) { ldmatrix_x4(out + 16 * l.row + 128 * (l.mat_lo * (K / 8) + 2 * kt + l.mat_hi), f); });
  };
  auto y_rest = [&](uint32_t stage, uint32_t out) {
    uint32_t P[3][4], A[2][4];
    lower_t_in(P, stage + r_off + kRecP, l);
#pragma unroll
    for (int kt = 0; kt < 2; ++kt) ldmatrix_x4(out + 32 * K + 16 * l.row + 128 * (l.mat_lo * 4 + 2 * kt + l.mat_hi), A[kt]);
#pragma unroll
    for (int nt = 0; nt < 4; ++nt) {
      const float2 e = lds64(stage + r_off + kRecVec + 8 * c + 128 * kVecEq + 32 * nt);
      y[nt][0] *= e.x; y[nt][1] *= e.y; y[nt][2] *= e.x; y[nt][3] *= e.y;
    }
    mul_lower_t(y, A, P);
  };
  // ... through V's place (V has been read) to rows of 32 bytes, a token a lane
  auto y_out = [&](uint32_t stage, int have) {
    uint32_t yt[2][4];
#pragma unroll
    for (int nt = 0; nt < 4; ++nt) {
      yt[nt >> 1][2 * (nt & 1)] = pack_bf16(y[nt][0], y[nt][1]);
      yt[nt >> 1][2 * (nt & 1) + 1] = pack_bf16(y[nt][2], y[nt][3]);
    }
    const uint32_t mine = stage + v_off + 32 * warp + lane * pv;
    stmatrix_x4_trans(stage + v_at, yt[0]);
    stmatrix_x4_trans(stage + v_at + 16 * pv, yt[1]);
    __syncwarp();
    const float4 x = lds128(mine), z = lds128(mine + 16);
    if (lane < have) {
      reinterpret_cast<float4 *>(yg)[0] = x;
      reinterpret_cast<float4 *>(yg)[1] = z;
    }
  };
  // One pass works on a chunk's chain and on the chunk before's Y, in one stretch of code without branches in which the
  // compiler lets one fill the other's waits.  (The first pass's Y is made of what there is, and not stored.)
  int st = 0, before = 0;
  uint32_t phase = 0;
  bool ready = sp.n > 0 && mbar_try_wait(bars.full, 0);
  for (int ch = 0; ch < sp.n; ++ch) {
    if (!__all_sync(0xffffffffu, ready) && !mbar_wait(bars.full + st, phase)) {
      if (lane == 0) report_timeout(a.dev_status);
      return;
    }
    const uint32_t stage = ring + st * sb, last = ring + before * sb, vec = stage + r_off + kRecVec + 8 * c;
    const uint32_t out = outs + (ch & 1) * out_bytes(K), last_out = outs + (~ch & 1) * out_bytes(K);
    if (KEEP) {      // the results of the chunk before the last have been read on their way to memory
      bulk_wait_read<kOuts - 1>();
      __syncwarp();
    }
    RowsT<K> kb;
    kb.template start<0, K / 16>(stage, l);
    uint32_t vt[2][4], T[3][4];
    rows_in(vt, stage + v_at, pv);
    lower_t_in(T, stage + r_off + kRecT, l);
    const float ec = __expf(lds32(stage + r_off + kRecVec + 128 * kVecG + 124));
    float acc[4][4];
    zero(acc);
    if (Y) y_states(last, last_out);
    kb.template run<0, K / 16>(acc, [&](int kt, uint32_t (&f)[4]) {
      pack_a<K / 8>(S, kt, f);
      blocks_out(f, out, K / 8, kt, l);
#pragma unroll
      for (int r = 0; r < 4; ++r) { S[2 * kt][r] *= ec; S[2 * kt + 1][r] *= ec; }
    });
    // X
#pragma unroll
    for (int nt = 0; nt < 4; ++nt) {
      const float2 e = lds64(vec + 128 * kVecEgk + 32 * nt), b = lds64(vec + 128 * kVecBeta + 32 * nt);
      const float2 x0 = unpack_bf16(vt[nt >> 1][2 * (nt & 1)]), x1 = unpack_bf16(vt[nt >> 1][2 * (nt & 1) + 1]);
      acc[nt][0] = b.x * fmaf(-e.x, acc[nt][0], x0.x);
      acc[nt][1] = b.y * fmaf(-e.y, acc[nt][1], x0.y);
      acc[nt][2] = b.x * fmaf(-e.x, acc[nt][2], x1.x);
      acc[nt][3] = b.y * fmaf(-e.y, acc[nt][3], x1.y);
    }
    uint32_t A[2][4];
    pack_a<4>(acc, 0, A[0]);
    pack_a<4>(acc, 1, A[1]);
    float U[4][4];
    zero(U);
    mul_lower_t(U, A, T);
    if (Y) y_rest(last, last_out);
    Rows<K> rb;
    rb.start(stage, l);
#pragma unroll
    for (int kt = 0; kt < 2; ++kt) {
      uint32_t f[4];
      pack_a<4>(U, kt, f);
      blocks_out(f, out + 32 * K, 4, kt, l);
#pragma unroll
      for (int nt = 2 * kt; nt < 2 * kt + 2; ++nt) {
        const float2 e = lds64(vec + 128 * kVecEk + 32 * nt);
        U[nt][0] *= e.x; U[nt][1] *= e.y; U[nt][2] *= e.x; U[nt][3] *= e.y;
      }
      pack_a<4>(U, kt, A[kt]);
    }
    const int next = st + 1 == stages ? 0 : st + 1;
    const uint32_t next_phase = phase ^ (next == 0);
    ready = ch + 1 < sp.n && mbar_try_wait(bars.full + next, next_phase);
    // S'
    rb.template run<0, 2>(S, A);
    if (Y) {
      y_out(last, ch > 0 ? C : 0);
      if (ch > 0) yg += (size_t)C * a.N * V;
    }
    if (KEEP) fence_async();
    __syncwarp();
    if (lane == 0) {
      if (KEEP) {
        bulk_store(sg, out, 32 * K);
        bulk_store(ug, out + 32 * K, 1024);
        bulk_commit();
      }
      if (ch > 0) mbar_arrive(bars.empty + before);      // (a chunk's stage is Y's too, a chunk later)
    }
    if (KEEP) { sg += (size_t)a.N * (2 * K * V); ug += (size_t)a.N * (2 * C * V); }
    before = st;
    st = next;
    phase = next_phase;
  }
  if (Y && sp.n > 0) {
    const uint32_t last = ring + before * sb, last_out = outs + (~sp.n & 1) * out_bytes(K);
    y_states(last, last_out);
    y_rest(last, last_out);
    y_out(last, sp.T - (sp.n - 1) * C);
  }
  if (a.hT) state_out<K>(S, a.hT, st_at, a.state_bf16, V, g, c);
  if (KEEP && lane == 0) bulk_wait_all();
}

template <int K>
__global__ void __launch_bounds__(192, 2) delta_chain_bwd_kernel(DeltaArgs a, int stages) {
  extern __shared__ __align__(128) unsigned char smem[];
  __shared__ ChainBars bars;
  const int nw = a.hpc * a.wv, warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31, g = lane >> 2, c = lane & 3;
  chain_bars(bars, stages, nw, nw + 1);
  begin_dependent();
  __syncthreads();
  const ChainWork w = chain_work(a, smem);
  const DeltaSpan sp = delta_span<C>(a, w.b);
  const uint32_t ring = smem_u32(smem), sb = (uint32_t)stage_bytes(K, nw, a.hpc), outs = ring + stages * sb;
  const int V = a.V, pv = pitch_v(nw);
  if (warp == nw + 1) {
    chain_fill<K>(a, w, sp, a.dy, (long long)a.N * V, nw, stages, ring, bars.full, bars.empty, lane, true);
    return;
  }
  auto give_up = [&] { if (lane == 0) report_timeout(a.dev_status); };
  const int cols = 16 * nw, col0 = w.n0 * V + 16 * w.slab * a.wv;      // the CTA's columns: adjacent in a token's row
  if (warp == nw) {      // results out: dS', L as they are, dV by rows from dY's place
    for (int i = 0; i < sp.n; ++i) {
      const int ch = sp.n - 1 - i, st = i % stages, os = i % kOuts, have = min(C, sp.T - ch * C);
      for (int cw = 0; cw < nw; ++cw) {
        if (!mbar_wait(&bars.there[cw][os], (uint32_t)((i / kOuts) & 1))) return give_up();
        if (lane == 0) {
          fence_async();      // (written by the chain warp's lanes, seen here through the barrier)
          const int n = w.n0 + cw / a.wv, v0 = 16 * (w.slab * a.wv + cw % a.wv);
          const size_t slot = (size_t)(sp.slot0 + ch) * a.N + n;
          const uint32_t out = outs + (cw * kOuts + os) * out_bytes(K);
          bulk_store(a.dstates + slot * (2 * K * V) + 2 * K * v0, out, 32 * K);
          bulk_store(a.lam + slot * (2 * C * V) + 2 * C * v0, out + 32 * K, 1024);
        }
        __syncwarp();
      }
      if (lane == 0) bulk_commit();
      const uint32_t vsa = ring + st * sb + 2 * C * pitch_k(K);
      __nv_bfloat16 *dvg = static_cast<__nv_bfloat16 *>(a.dv) + (size_t)(sp.tok0 + ch * C) * a.N * V + col0;
      const int log_p = 28 - __clz(cols);      // pieces of a row
      for (int x = lane; x < have << log_p; x += 32) {
        const int r = x >> log_p, p = x & ((1 << log_p) - 1);
        *reinterpret_cast<float4 *>(dvg + (size_t)r * a.N * V + 8 * p) = lds128(vsa + r * pv + 16 * p);
      }
      __syncwarp();
      if (lane == 0) {
        mbar_arrive(bars.empty + st);
        bulk_wait_read<0>();
        for (int cw = 0; cw < nw; ++cw) mbar_arrive(&bars.gone[cw][os]);
      }
    }
    if (lane == 0) bulk_wait_all();
    return;
  }
  const int n = w.n0 + warp / a.wv, v0 = 16 * (w.slab * a.wv + warp % a.wv);
  const size_t st_at = ((size_t)w.b * a.N + n) * K * V + v0;
  const Lanes l(lane);
  float S[K / 8][4];    // dS
  if (a.d_hT) state_in<K>(S, a.d_hT, st_at, a.state_bf16, V, g, c);
  else
#pragma unroll
    for (int nt = 0; nt < K / 8; ++nt)
#pragma unroll
      for (int r = 0; r < 4; ++r) S[nt][r] = 0.f;
  for (int i = 0; i < sp.n; ++i) {
    const int st = i % stages, os = i % kOuts;
    if (!wait_both(bars.full + st, (uint32_t)((i / stages) & 1), &bars.gone[warp][os], (uint32_t)((i / kOuts - 1) & 1), i >= kOuts)) return give_up();
    const uint32_t ksa = ring + st * sb, qsa = ksa + C * pitch_k(K), vsa = qsa + C * pitch_k(K), rec = vsa + C * pv + (warp / a.wv) * kRecChain;
    const uint32_t vec = rec + kRecVec + 8 * c, out = outs + (warp * kOuts + os) * out_bytes(K);
    // what does not hang on dS' is asked for first
    const uint32_t vat = vsa + 32 * warp + (l.row + 8 * l.mat_hi) * pv + 16 * l.mat_lo;
    RowsT<K> kb;
    kb.template start<0, K / 16>(ksa, l);
    uint32_t yt[2][4], A[2][4], T[3][4], P[3][4];
    rows_in(yt, vat, pv);
    lower_in(P, rec + kRecP, l);
    float2 ek[4], eq[4];
#pragma unroll
    for (int nt = 0; nt < 4; ++nt) {
      ek[nt] = lds64(vec + 128 * kVecEk + 32 * nt);
      eq[nt] = lds64(vec + 128 * kVecEq + 32 * nt);
    }
    const float ec = __expf(lds32(rec + kRecVec + 128 * kVecG + 124));
    float acc[4][4];
    zero(acc);
    kb.template run<0, K / 16>(acc, [&](int kt, uint32_t (&f)[4]) {
      pack_a<K / 8>(S, kt, f);
      blocks_out(f, out, K / 8, kt, l);
#pragma unroll
      for (int r = 0; r < 4; ++r) { S[2 * kt][r] *= ec; S[2 * kt + 1][r] *= ec; }
    });
    Rows<K> rb;
    rb.start(qsa, l);
    // dU
#pragma unroll
    for (int nt = 0; nt < 4; ++nt) { acc[nt][0] *= ek[nt].x; acc[nt][1] *= ek[nt].y; acc[nt][2] *= ek[nt].x; acc[nt][3] *= ek[nt].y; }
    mul_lower(acc, yt, P);     // (packed accumulators [2kt], [2kt + 1] are the A operand of k-tile kt)
    lower_in(T, rec + kRecT, l);
    // meanwhile what does not hang on dS': + (s e^g Q)^T dY
    {
      float E[4][4];
#pragma unroll
      for (int nt = 0; nt < 4; ++nt) {
        const float2 x0 = unpack_bf16(yt[nt >> 1][2 * (nt & 1)]), x1 = unpack_bf16(yt[nt >> 1][2 * (nt & 1) + 1]);
        E[nt][0] = eq[nt].x * x0.x; E[nt][1] = eq[nt].y * x0.y; E[nt][2] = eq[nt].x * x1.x; E[nt][3] = eq[nt].y * x1.y;
      }
      pack_a<4>(E, 0, A[0]);
      pack_a<4>(E, 1, A[1]);
    }
    rb.template run<0, 1>(S, A);
    uint32_t D[2][4];
    pack_a<4>(acc, 0, D[0]);
    pack_a<4>(acc, 1, D[1]);
    float2 be[4], eg[4];
#pragma unroll
    for (int nt = 0; nt < 4; ++nt) {
      be[nt] = lds64(vec + 128 * kVecBeta + 32 * nt);
      eg[nt] = lds64(vec + 128 * kVecEgk + 32 * nt);
    }
    float L[4][4];
    zero(L);
    mul_lower(L, D, T);
    rb.template run<1, 2>(S, A);
    rb.start(ksa, l);
    uint32_t dvt[2][4];
#pragma unroll
    for (int kt = 0; kt < 2; ++kt) {
      uint32_t f[4];
      pack_a<4>(L, kt, f);
      blocks_out(f, out + 32 * K, 4, kt, l);
#pragma unroll
      for (int nt = 2 * kt; nt < 2 * kt + 2; ++nt) {
        L[nt][0] *= be[nt].x; L[nt][1] *= be[nt].y; L[nt][2] *= be[nt].x; L[nt][3] *= be[nt].y;
        dvt[nt >> 1][2 * (nt & 1)] = pack_bf16(L[nt][0], L[nt][1]);
        dvt[nt >> 1][2 * (nt & 1) + 1] = pack_bf16(L[nt][2], L[nt][3]);
        L[nt][0] *= -eg[nt].x; L[nt][1] *= -eg[nt].y; L[nt][2] *= -eg[nt].x; L[nt][3] *= -eg[nt].y;
      }
      pack_a<4>(L, kt, A[kt]);
    }
    stmatrix_x4_trans(vat, dvt[0]);      // (dY is in registers)
    stmatrix_x4_trans(vat + 16 * pv, dvt[1]);
    __syncwarp();
    if (lane == 0) mbar_arrive(&bars.there[warp][os]);
    // dS
    rb.template run<0, 2>(S, A);
    __syncwarp();
    if (lane == 0) mbar_arrive(bars.empty + st);
  }
  if (a.dh0) state_out<K>(S, a.dh0, st_at, a.state_bf16, V, g, c);
}

// 16-column warps of a CTA.  A state's columns stay together (they share the copies of k, q and the records), up to four,
// while there are CTAs for all SMs; with fewer units they are spread.
ChainPlan plan_chain(const DeltaArgs &a) {
  const int cols = a.V / 16;
  const long long units = (long long)a.B * a.N, sms = sm_count();
  ChainPlan p{1, cols < 4 ? cols : 4, 1, 4, 0};
  while (p.wv > 1 && units * (cols / p.wv) < sms) p.wv /= 2;
  p.slabs = cols / p.wv;
  const int nw = p.hpc * p.wv;
  // two CTAs to an SM where there are that many
  const size_t room = (size_t)(units * p.slabs > sms ? 113 : 226) * 1024, fixed = (size_t)nw * kOuts * out_bytes(a.K), sb = (size_t)stage_bytes(a.K, nw, p.hpc);
  while (p.stages > 3 && fixed + p.stages * sb > room) --p.stages;
  p.smem = fixed + p.stages * sb;
  return p;
}

template <int K> cudaError_t launch_k(const DeltaArgs &args, bool backward, cudaStream_t s) {
  DeltaArgs a = args;
  const ChainPlan p = plan_chain(a);
  a.hpc = p.hpc; a.wv = p.wv;
  void (*kernel)(DeltaArgs, int) = backward ? delta_chain_bwd_kernel<K> : !a.states ? delta_chain_fwd_kernel<K, true, false> : a.y ? delta_chain_fwd_kernel<K, true, true> : delta_chain_fwd_kernel<K, false, true>;
  const cudaError_t e = allow_smem(kernel, p.smem);
  if (e != cudaSuccess) return e;
  return launch_early(kernel, dim3((unsigned)((long long)a.B * (a.N / p.hpc) * p.slabs)), dim3(32 * (p.hpc * p.wv + (backward ? 2 : 1))), p.smem, s, a, p.stages);
}
cudaError_t launch(const DeltaArgs &a, bool backward, cudaStream_t s) {
  switch (a.K) {
    case 16: return launch_k<16>(a, backward, s);
    case 32: return launch_k<32>(a, backward, s);
    case 48: return launch_k<48>(a, backward, s);
    case 64: return launch_k<64>(a, backward, s);
    case 80: return launch_k<80>(a, backward, s);
    case 96: return launch_k<96>(a, backward, s);
    case 112: return launch_k<112>(a, backward, s);
    default: return launch_k<128>(a, backward, s);
  }
}

}  // namespace

cudaError_t launch_delta_chain_fwd(const DeltaArgs &a, cudaStream_t s) { return launch(a, false, s); }
cudaError_t launch_delta_chain_bwd(const DeltaArgs &a, cudaStream_t s) { return launch(a, true, s); }

}  // namespace m2rnn
