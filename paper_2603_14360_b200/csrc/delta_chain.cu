// Gated delta rule, bf16: the two chains over the chunks of a sequence, forward and backward.
//
// With S the K x V state at a chunk's start, T and P of delta_prep.cu, and per token the record's factors,
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
// waits, in one stretch of code without branches that the compiler orders: forward the products of the chunk before's Y (S of that
// chunk as operands from shared memory, tile by tile before the new ones take their places), backward those with Q.
// (Y after its own chunk's chain: 1 680 cycles a chunk of K = 64 for a warp alone.)  Where SMs have warps to spare, Y is a warp's of its own beside
// each chain: it finds the chunk's S and U in one of two buffers that the chain fills.  (plan_chain; where they have not, those warps would halve
// the chains to an SM.)  What is kept for the gradient goes from registers to memory, 128 bytes an instruction.
// Roundings to bf16: the operands S, X, U (dS, dU, L), the factored e^(g_last - g) U and the like, and P.  S itself
// is held and updated in fp32.  T comes as bf16 and what that leaves, two products: keys that are much alike (a token that is repeated) make its
// entries near -1, many of one value, and what their roundings add to U, all to the same side, sums up in S (one token throughout, b = 0.98,
// decay e^-0.002: dstep 1e-1 off, hT 6e-2; with both products 1.4e-2 and 1.8e-2, for 2 to 4 % of a pass).
// Bound by the chain's latency where an SM has a chain to a scheduler (1 001 tokens, 84 heads of 64 x 16: 16.9 us, 0.48 a chunk; 65 536 tokens,
// 32 heads of 128 x 128, two chains to an SM: 1 417 us, 0.69 a chunk; 8 x 2 048 tokens, 16 heads of 64 x 64, four: 51.9 us, 0.81), by shared memory's
// bandwidth where it has more (two to a scheduler: LSU data pipe 83 % busy).
#include <algorithm>

#include "delta_common.cuh"

namespace m2rnn {
namespace {

constexpr int C = kDeltaChunk;

// Bytes of a stage: K, Q rows, rows of 16 nw columns of V (dY), a record
__host__ __device__ constexpr int pitch_k(int K) { return 2 * K + 16; }
__host__ __device__ constexpr int pitch_v(int nw) { return 32 * nw + 16; }
__host__ __device__ constexpr int stage_bytes(int K, int nw) { return C * (2 * pitch_k(K) + pitch_v(nw)) + kRecChain; }

// Forward, a chain warp's S as operands of the next chunk's pass (Y): in registers where K leaves them, else in shared memory, blocks
// [column tile][feature tile].  (Shared memory's bandwidth is what chains of an SM compete for: 324 of its cycles a chain and chunk of K = 64.)
__host__ __device__ constexpr int out_bytes(int K) { return K <= 64 ? 0 : 32 * K; }

// S and U of a chunk for a warp that does Y
__host__ __device__ constexpr int apart_bytes(int K) { return 32 * K + 1024; }

struct ChainPlan { int nw, slabs, stages, apart; size_t smem; };      // nw: 16-column warps of a CTA

// What a CTA has to do: batch entry, head, and which slab of its columns
struct ChainWork { int b, n, slab; };
template <bool PACKED> __device__ __forceinline__ ChainWork chain_work(const DeltaArgs &a, void *scratch) {
  const int slabs = a.V / (16 * a.nw), per = a.N * slabs;
  ChainWork w;
  w.b = (int)(blockIdx.x / per);
  // sequences of a packed batch longest first: a long one that starts last keeps the others' SMs idle.  (Every CTA ranks for itself, B^2
  // comparisons over its threads: up to 64 sequences.  Kernels of their own: the call alone costs the others 3 %.)
  if (PACKED) w.b = __shfl_sync(0xffffffffu, a.B > 1 && a.B <= 64 ? longest_first(a.cu, a.B, w.b, static_cast<int *>(scratch)) : w.b, 0);
  const int r = (int)(blockIdx.x % per);
  w.n = r / slabs;
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
  const uint32_t sb = (uint32_t)stage_bytes(K, nw);
  const int r0 = lane / LR, rv0 = lane / lv;
  const char *kp = static_cast<const char *>(a.k) + 2 * ((sp.tok0 + r0) * a.ks + w.n / a.per_k * K) + 16 * (lane % LR);
  const char *qp = static_cast<const char *>(a.q) + 2 * ((sp.tok0 + r0) * a.qs + w.n / a.per_q * K) + 16 * (lane % LR);
  const char *vp = static_cast<const char *>(vg) + 2 * ((sp.tok0 + rv0) * vs + (long long)w.n * a.V + w.slab * 16 * nw) + 16 * (lane % lv);
  const long long kc = 2 * C * a.ks, qc = 2 * C * a.qs, vc = 2 * C * vs, kr = 2 * RP * a.ks, qr = 2 * RP * a.qs, vr = 2 * rv * vs;      // bytes to the next chunk, the next pass
  const uint32_t k_at = r0 * pitch_k(K) + 16 * (lane % LR), v_at = 2 * C * pitch_k(K) + rv0 * pv + 16 * (lane % lv);
  const size_t rec_step = (size_t)a.N * kRecBytes;
  const char *rp = a.rec + ((size_t)sp.slot0 * a.N + w.n) * kRecBytes;
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
      mbar_expect(full + st, (uint32_t)kRecChain);
      bulk_load(rd, rp, kRecChain, full + st);
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
// acc[4 token tiles] += A (16 x K) . rows^T, k-tile by k-tile: rows [32 tokens][K] in shared memory
template <int K> struct RowsT {
  uint32_t at, b[kAhead][4];
  __device__ __forceinline__ void load(int x) { ldmatrix_x4(at + 16 * (x & 1) * pitch_k(K) + 32 * (x >> 1), b[x % kAhead]); }
  __device__ __forceinline__ void start(uint32_t rows, const Lanes &l) {
    at = rows + (l.row + 8 * l.mat_hi) * pitch_k(K) + 16 * l.mat_lo;
#pragma unroll
    for (int x = 0; x < K / 8 && x < kAhead; ++x) load(x);
  }
  __device__ __forceinline__ void step(float (&acc)[4][4], const uint32_t (&f)[4], int kt) {
#pragma unroll
    for (int np = 0; np < 2; ++np) {
      const int x = 2 * kt + np;
      mma_add(acc[2 * np], f, b[x % kAhead][0], b[x % kAhead][1]);
      mma_add(acc[2 * np + 1], f, b[x % kAhead][2], b[x % kAhead][3]);
      if (x + kAhead < K / 8) load(x + kAhead);
    }
  }
};
// S (16 x K) += A (16 x 32 tokens) . rows, a pair of feature tiles after the other
template <int K> struct Rows {
  static constexpr int N = K / 16;      // pairs
  uint32_t at, b[kAhead][4];
  __device__ __forceinline__ void load(int x) { ldmatrix_x4_t(at + 16 * (x & 1) * pitch_k(K) + 32 * (x >> 1), b[x % kAhead]); }
  __device__ __forceinline__ void start(uint32_t rows, const Lanes &l) {
    at = rows + (l.row + 8 * l.mat_lo) * pitch_k(K) + 16 * l.mat_hi;
#pragma unroll
    for (int x = 0; x < 2 * N && x < kAhead; ++x) load(x);
  }
  __device__ __forceinline__ void step(float (&S)[K / 8][4], const uint32_t (&A)[2][4], int np) {
#pragma unroll
    for (int kt = 0; kt < 2; ++kt) {
      const int x = 2 * np + kt;
      mma_add(S[2 * np], A[kt], b[x % kAhead][0], b[x % kAhead][1]);
      mma_add(S[2 * np + 1], A[kt], b[x % kAhead][2], b[x % kAhead][3]);
      if (x + kAhead < 2 * N) load(x + kAhead);
    }
  }
  // pairs two at a time: four products in flight
  __device__ __forceinline__ void run(float (&S)[K / 8][4], const uint32_t (&A)[2][4]) {
#pragma unroll
    for (int p = 0; p < N; p += 2) {
#pragma unroll
      for (int kt = 0; kt < 2; ++kt)
#pragma unroll
        for (int np = p; np < p + 2 && np < N; ++np) {
          const int x = 2 * np + kt;
          mma_add(S[2 * np], A[kt], b[x % kAhead][0], b[x % kAhead][1]);
          mma_add(S[2 * np + 1], A[kt], b[x % kAhead][2], b[x % kAhead][3]);
          if (x + kAhead < 2 * N) load(x + kAhead);
        }
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
// What T lost as bf16, in a record's three places
__device__ __forceinline__ void low_t_in(uint32_t (&b)[3][4], uint32_t rec, const Lanes &l) {
  const uint32_t at = rec + 16 * l.row + 128 * l.mat_lo, diag = at + 512 * l.mat_hi + kRecTLDiag;
  ldmatrix_x4(diag + kRecT, b[0]);
  ldmatrix_x4(at + 256 * l.mat_hi + kRecTL, b[1]);
  ldmatrix_x4(diag + kRecP, b[2]);
}
__device__ __forceinline__ void low_in(uint32_t (&b)[3][4], uint32_t rec, const Lanes &l) {
  const uint32_t at = rec + 16 * l.row + 128 * l.mat_hi, diag = at + 512 * l.mat_lo + kRecTLDiag;
  ldmatrix_x4_t(diag + kRecT, b[0]);
  ldmatrix_x4_t(at + 256 * l.mat_lo + kRecTL, b[1]);
  ldmatrix_x4_t(diag + kRecP, b[2]);
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
// Causality and what is not finite: in a product with a lower triangular matrix 0 x NaN would carry a token's NaN to the tokens before it, of
// its block of 16.  Where U has such entries they are taken out of the operands, and per column the first such token is kept; from that one on
// results are NaN.
__device__ __forceinline__ bool any_odd(const uint32_t (&f)[2][4]) {
  __nv_bfloat162 s = __floats2bfloat162_rn(0.f, 0.f), t = s;
  const __nv_bfloat162 z = s;
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    s = __hfma2(reinterpret_cast<const __nv_bfloat162 &>(f[0][r]), z, s);
    t = __hfma2(reinterpret_cast<const __nv_bfloat162 &>(f[1][r]), z, t);
  }
  s = __hadd2(s, t);
  return __any_sync(0xffffffffu, (reinterpret_cast<const uint32_t &>(s) & 0x7fff7fffu) != 0u);
}
struct FirstOdd { int at[2]; };      // of columns g, g + 8; 32: none
__device__ __forceinline__ FirstOdd take_odd(uint32_t (&f)[2][4], int c) {
  FirstOdd o{{32, 32}};
#pragma unroll
  for (int kt = 0; kt < 2; ++kt)
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int e = 0; e < 2; ++e)
        if ((f[kt][r] >> (16 * e) & 0x7f80u) == 0x7f80u) {
          f[kt][r] &= e ? 0xffffu : 0xffff0000u;
          o.at[r & 1] = min(o.at[r & 1], 16 * kt + 8 * (r >> 1) + 2 * c + e);
        }
#pragma unroll
  for (int h = 0; h < 2; ++h)
#pragma unroll
    for (int d = 1; d < 4; d *= 2) o.at[h] = min(o.at[h], __shfl_xor_sync(0xffffffffu, o.at[h], d));
  return o;
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
// A operand tiles (16 columns x 16 tokens or features) to blocks [column tile][tile] in memory, `n` tiles a column tile, tiles 2 kt, 2 kt + 1
__device__ __forceinline__ void blocks_to(const uint32_t (&f)[4], char *p, int n, int kt) {
#pragma unroll
  for (int r = 0; r < 4; ++r) *reinterpret_cast<uint32_t *>(p + 128 * ((r & 1) * n + 2 * kt + (r >> 1))) = f[r];
}
// a tile of 16 columns x 32 tokens, packed accumulators, through its place in shared memory to rows of 32 bytes, a token a lane
__device__ __forceinline__ void rows_out(const float (&x)[4][4], uint32_t at, uint32_t mine, int pv, __nv_bfloat16 *out, bool ok) {
  uint32_t t[2][4];
#pragma unroll
  for (int nt = 0; nt < 4; ++nt) {
    t[nt >> 1][2 * (nt & 1)] = pack_bf16(x[nt][0], x[nt][1]);
    t[nt >> 1][2 * (nt & 1) + 1] = pack_bf16(x[nt][2], x[nt][3]);
  }
  stmatrix_x4_trans(at, t[0]);
  stmatrix_x4_trans(at + 16 * pv, t[1]);
  __syncwarp();
  const float4 u = lds128(mine), v = lds128(mine + 16);
  if (ok) {
    reinterpret_cast<float4 *>(out)[0] = u;
    reinterpret_cast<float4 *>(out)[1] = v;
  }
}

// Barriers of a CTA: stages filled and free; a chain's S and U there for its Y's warp, and taken
struct ChainBars { uint64_t full[8], empty[8], ready[8], taken[8]; };      // (ready, taken: two buffers of a chain)

// A warp's part: 0 .. nw - 1 a chain, nw copies, above that none; apart: nw .. 2 nw - 1 the chains' Y, 2 nw copies (with one chain the middle
// warp, with two the seventh, the fifth and sixth doing nothing: so that chains and Y have schedulers of their own, of two CTAs too).  An SM's CTAs come a layer after the other, and warp w of the SM's
// belongs to scheduler w % 4: with CTAs of two warps (a chain) or four (two) the parts of every second pair of layers, or layer, change
// places, so that chains share a scheduler only where there are more than four to the SM.
__device__ __forceinline__ int chain_role(const DeltaArgs &a, int nw, bool apart) {
  const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), layer = (int)(blockIdx.x / (unsigned)a.sms);
  if (apart) return nw == 1 ? (3 - warp) % 3 : nw == 2 && warp >= 4 ? (warp == 6 ? 4 : 5) : warp;
  if (nw == 1) return warp ^ (layer >> 1 & 1);
  if (nw == 2) return warp ^ (layer & 1) << 1;
  return warp;
}

// What both kernels' chain warps begin with
#define CHAIN_BEGIN(tensor, stride, back, apart)                                                                                               \
  extern __shared__ __align__(128) unsigned char smem[];                                                                                      \
  __shared__ ChainBars bars;                                                                                                                  \
  const int nw = a.nw, users = (apart) ? 2 * nw : nw, warp = chain_role(a, nw, apart), lane = threadIdx.x & 31, g = lane >> 2, c = lane & 3;                                         \
  if (threadIdx.x == 0) {                                                                                                                     \
    for (int i = 0; i < stages; ++i) { mbar_init(bars.full + i, 33); mbar_init(bars.empty + i, users); }                                      \
    for (int i = 0; i < 8; ++i) { mbar_init(bars.ready + i, 1); mbar_init(bars.taken + i, 1); }                                               \
    fence_mbar_init();                                                                                                                        \
  }                                                                                                                                           \
  begin_dependent();                                                                                                                          \
  __syncthreads();                                                                                                                            \
  const ChainWork w = chain_work<PACKED>(a, smem);                                                                                            \
  const DeltaSpan sp = delta_span<C>(a, w.b);                                                                                                 \
  const uint32_t ring = smem_u32(smem), sb = (uint32_t)stage_bytes(K, nw);                                                                    \
  if (warp > users) return;                                                                                                                   \
  if (warp == users) {                                                                                                                        \
    chain_fill<K>(a, w, sp, tensor, stride, nw, stages, ring, bars.full, bars.empty, lane, back);                                             \
    return;                                                                                                                                   \
  }                                                                                                                                           \
  const int mine = warp < nw ? warp : warp - nw, n = w.n, v0 = 16 * (w.slab * nw + mine), V = a.V, pv = pitch_v(nw);                          \
  const Lanes l(lane);                                                                                                                        \
  const uint32_t v_off = 2 * C * pitch_k(K), r_off = v_off + C * pv;                                                                          \
  const uint32_t v_at = v_off + 32 * mine + (l.row + 8 * l.mat_hi) * pv + 16 * l.mat_lo, v_mine = v_off + 32 * mine + lane * pv;              \
  const size_t st_at = ((size_t)w.b * a.N + n) * K * V + v0

// Where a chain finds things in a stage
struct ChainAt { uint32_t v_at, v_mine, r_off; int pv, c; };
// X from K S, as operands; T and what it lost as bf16
__device__ __forceinline__ void x_of(const ChainAt &t, const Lanes &l, uint32_t stage, float (&acc)[4][4], uint32_t (&A)[2][4], uint32_t (&T)[3][4], uint32_t (&TL)[3][4]) {
  const uint32_t vec = stage + t.r_off + kRecVec + 8 * t.c;
  uint32_t vt[2][4];
  rows_in(vt, stage + t.v_at, t.pv);
  lower_t_in(T, stage + t.r_off + kRecT, l);
  low_t_in(TL, stage + t.r_off, l);
#pragma unroll
  for (int nt = 0; nt < 4; ++nt) {
    const float2 e = lds64(vec + 128 * kVecEgk + 32 * nt), b = lds64(vec + 128 * kVecBeta + 32 * nt);
    const float2 x0 = unpack_bf16(vt[nt >> 1][2 * (nt & 1)]), x1 = unpack_bf16(vt[nt >> 1][2 * (nt & 1) + 1]);
    acc[nt][0] = b.x * fmaf(-e.x, acc[nt][0], x0.x);
    acc[nt][1] = b.y * fmaf(-e.y, acc[nt][1], x0.y);
    acc[nt][2] = b.x * fmaf(-e.x, acc[nt][2], x1.x);
    acc[nt][3] = b.y * fmaf(-e.y, acc[nt][3], x1.y);
  }
  pack_a<4>(acc, 0, A[0]);
  pack_a<4>(acc, 1, A[1]);
}
// Y from q S: scaled, + P U
__device__ __forceinline__ void y_rest(const ChainAt &t, const Lanes &l, uint32_t stage, float (&y)[4][4], const uint32_t (&Ub)[2][4]) {
  uint32_t P[3][4];
  lower_t_in(P, stage + t.r_off + kRecP, l);
#pragma unroll
  for (int nt = 0; nt < 4; ++nt) {
    const float2 e = lds64(stage + t.r_off + kRecVec + 8 * t.c + 128 * kVecEq + 32 * nt);
    y[nt][0] *= e.x; y[nt][1] *= e.y; y[nt][2] *= e.x; y[nt][3] *= e.y;
  }
  mul_lower_t(y, Ub, P);
}
// Where a chunk's U has what is not finite, before its Y: U once more from the S that Y is going to read (operand kt: s_of), and y begun with
// NaN from the first such token on.
template <int K, typename F>
__device__ __forceinline__ void mend(const ChainAt &t, const Lanes &l, uint32_t stage, F s_of, uint32_t (&Ub)[2][4], float (&y)[4][4]) {
  RowsT<K> kb;
  kb.start(stage, l);
  float acc[4][4], U[4][4];
  zero(acc);
#pragma unroll
  for (int kt = 0; kt < K / 16; ++kt) {
    uint32_t f[4];
    s_of(kt, f);
    kb.step(acc, f, kt);
  }
  uint32_t A[2][4], T[3][4], TL[3][4];
  x_of(t, l, stage, acc, A, T, TL);
  const FirstOdd x = take_odd(A, t.c);
  zero(U);
  mul_lower_t(U, A, TL);
  mul_lower_t(U, A, T);
  pack_a<4>(U, 0, Ub[0]);
  pack_a<4>(U, 1, Ub[1]);
  const FirstOdd u = take_odd(Ub, t.c);      // (T's rows may have such entries where X has none)
#pragma unroll
  for (int nt = 0; nt < 4; ++nt)
#pragma unroll
    for (int r = 0; r < 4; ++r)
      if (8 * nt + 2 * t.c + (r & 1) >= min(x.at[r >> 1], u.at[r >> 1])) y[nt][r] = __int_as_float(0x7fffffff);
}

// Y: y is asked for; KEEP: states and updates are kept for the gradient; APART: Y is a warp's of its own, beside each chain (1: up to two of
// these, seven warps at most; 2: four, nine warps, which leaves a thread fewer registers)
template <int K, bool Y, bool KEEP, bool PACKED, int APART>
__global__ void __launch_bounds__(APART == 2 ? 288 : APART ? 224 : 160, APART ? 1 : 2) delta_chain_fwd_kernel(DeltaArgs a, int stages) {
  CHAIN_BEGIN(a.v, a.vs, false, APART != 0);
  const ChainAt t{v_at, v_mine, r_off, pv, c};
  constexpr bool WITH = Y && !APART;      // the chain does Y too
  const uint32_t out = ring + stages * sb + (APART ? 2 * mine * apart_bytes(K) : warp * out_bytes(K));
  const uint32_t spare = ring + stages * sb + nw * out_bytes(K) - v_off;      // (as if a stage, its columns of V)
  const uint32_t s_lane = 16 * l.row + 128 * (l.mat_lo * (K / 8) + l.mat_hi), u_lane = 32 * K + 16 * l.row + 128 * (4 * l.mat_lo + l.mat_hi);      // blocks [column tile][tile]
  __nv_bfloat16 *yg = Y ? static_cast<__nv_bfloat16 *>(a.y) + ((size_t)(sp.tok0 + lane) * a.N + n) * V + v0 : nullptr;
  if (APART && warp >= nw) {      // S and U of chunk after chunk from the chain's two buffers
    int st = 0;
    uint32_t phase = 0;
    for (int ch = 0; ch < sp.n; ++ch) {
      const int buf = 2 * mine + (ch & 1);
      if (!mbar_wait(bars.full + st, phase) || !mbar_wait(bars.ready + buf, (ch >> 1) & 1)) {
        if (lane == 0) report_timeout(a.dev_status);
        return;
      }
      const uint32_t stage = ring + st * sb, at = out + (ch & 1) * apart_bytes(K);
      RowsT<K> qb;
      qb.start(stage + C * pitch_k(K), l);
      uint32_t Ub[2][4], f[2][4];
      ldmatrix_x4(at + u_lane, Ub[0]);
      ldmatrix_x4(at + u_lane + 256, Ub[1]);
      ldmatrix_x4(at + s_lane, f[0]);
      float y[4][4];
      zero(y);
      if (any_odd(Ub)) mend<K>(t, l, stage, [&](int kt, uint32_t (&x)[4]) { ldmatrix_x4(at + s_lane + 256 * kt, x); }, Ub, y);
#pragma unroll
      for (int kt = 0; kt < K / 16; ++kt) {
        if (kt + 1 < K / 16) ldmatrix_x4(at + s_lane + 256 * (kt + 1), f[(kt + 1) & 1]);
        qb.step(y, f[kt & 1], kt);
      }
      y_rest(t, l, stage, y, Ub);
      __syncwarp();
      if (lane == 0) mbar_arrive(bars.taken + buf);
      rows_out(y, stage + v_at, stage + v_mine, pv, yg, lane < sp.T - ch * C);      // (through V's place: the chain has read it)
      yg += (size_t)C * a.N * V;
      __syncwarp();
      if (lane == 0) mbar_arrive(bars.empty + st);
      if (++st == stages) { st = 0; phase ^= 1; }
    }
    return;
  }
  float S[K / 8][4];
  if (a.h0) state_in<K>(S, a.h0, st_at, a.state_bf16, V, g, c);
  else
#pragma unroll
    for (int nt = 0; nt < K / 8; ++nt)
#pragma unroll
      for (int r = 0; r < 4; ++r) S[nt][r] = 0.f;
  char *sg = KEEP ? a.states + ((size_t)sp.slot0 * a.N + n) * (2 * K * V) + 2 * K * v0 + 4 * lane : nullptr, *ug = KEEP ? a.upd + ((size_t)sp.slot0 * a.N + n) * (2 * C * V) + 2 * C * v0 + 4 * lane : nullptr;
  const uint32_t s_at = out + s_lane;      // tiles of S: 256 bytes apart
  uint32_t Ub[2][4] = {}, Sb[K <= 64 ? K / 16 : 1][4] = {};      // U, S as operands
  float y[4][4];
  bool odd = false;
  // operand kt of the S that Y reads
  auto s_of = [&](int kt, uint32_t (&f)[4]) {
    if constexpr (K > 64) ldmatrix_x4(s_at + 256 * kt, f);
    else {
#pragma unroll
      for (int r = 0; r < 4; ++r) f[r] = Sb[kt][r];
    }
  };
  // One pass works on a chunk's chain and (WITH) on the chunk before's Y.  (The first pass's Y is made of what there is, and not stored.)
  int st = 0, before = 0;
  uint32_t phase = 0;
  bool ready = sp.n > 0 && mbar_try_wait(bars.full, 0);
  for (int ch = 0; ch < sp.n; ++ch) {
    const int buf = 2 * mine + (ch & 1);
    if ((!__all_sync(0xffffffffu, ready) && !mbar_wait(bars.full + st, phase)) || (APART && ch > 1 && !mbar_wait(bars.taken + buf, ((ch >> 1) - 1) & 1))) {
      if (lane == 0) report_timeout(a.dev_status);
      return;
    }
    const uint32_t stage = ring + st * sb, last = ring + before * sb, vec = stage + r_off + kRecVec + 8 * c, to = APART ? s_at + (ch & 1) * apart_bytes(K) : s_at;
    zero(y);
    if (WITH && odd) mend<K>(t, l, last, s_of, Ub, y);
    RowsT<K> kb, qb;
    kb.start(stage, l);
    if (WITH) qb.start(last + C * pitch_k(K), l);
    const float ec = __expf(lds32(stage + r_off + kRecVec + 128 * kVecG + 124));
    float acc[4][4];
    zero(acc);
    uint32_t fo[2][4];      // the chunk before's S
    if (WITH && K > 64) ldmatrix_x4(s_at, fo[0]);
#pragma unroll
    for (int kt = 0; kt < K / 16; ++kt) {
      uint32_t f[4];
      pack_a<K / 8>(S, kt, f);
      if (WITH && K > 64 && kt + 1 < K / 16) ldmatrix_x4(s_at + 256 * (kt + 1), fo[(kt + 1) & 1]);
      if (APART || (WITH && K > 64)) stmatrix_x4(to + 256 * kt, f);
      if (KEEP) blocks_to(f, sg, K / 8, kt);
#pragma unroll
      for (int r = 0; r < 4; ++r) { S[2 * kt][r] *= ec; S[2 * kt + 1][r] *= ec; }
      kb.step(acc, f, kt);
      if (WITH) {
        if constexpr (K > 64) {
          qb.step(y, fo[kt & 1], kt);
        } else {
          qb.step(y, Sb[kt], kt);
#pragma unroll
          for (int r = 0; r < 4; ++r) Sb[kt][r] = f[r];
        }
      }
    }
    if (WITH) y_rest(t, l, last, y, Ub);
    uint32_t A[2][4], T[3][4], TL[3][4];
    x_of(t, l, stage, acc, A, T, TL);
    float U[4][4];
    zero(U);
    mul_lower_t(U, A, TL);
    mul_lower_t(U, A, T);
    Rows<K> rb;
    rb.start(stage, l);
#pragma unroll
    for (int kt = 0; kt < 2; ++kt) {
      pack_a<4>(U, kt, Ub[kt]);
      if (APART) stmatrix_x4(out + (ch & 1) * apart_bytes(K) + u_lane + 256 * kt, Ub[kt]);
      if (KEEP) blocks_to(Ub[kt], ug, 4, kt);
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
    rb.run(S, A);
    if (WITH) {
      odd = any_odd(Ub);
      const uint32_t y_to = ch > 0 ? last : spare;      // (through V's place, which has been read)
      rows_out(y, y_to + v_at, y_to + v_mine, pv, yg, ch > 0);
      if (ch > 0) yg += (size_t)C * a.N * V;
    }
    __syncwarp();
    if (WITH) {
      if (lane == 0 && ch > 0) mbar_arrive(bars.empty + before);      // (a chunk's stage is Y's too, a chunk later)
    } else if (lane == 0) {
      if (APART) mbar_arrive(bars.ready + buf);
      mbar_arrive(bars.empty + st);
    }
    if (KEEP) { sg += (size_t)a.N * (2 * K * V); ug += (size_t)a.N * (2 * C * V); }
    before = st;
    st = next;
    phase = next_phase;
  }
  if (WITH && sp.n > 0) {
    const uint32_t last = ring + before * sb;
    zero(y);
    if (odd) mend<K>(t, l, last, s_of, Ub, y);
    RowsT<K> qb;
    qb.start(last + C * pitch_k(K), l);
#pragma unroll
    for (int kt = 0; kt < K / 16; ++kt) {
      uint32_t f[4];
      s_of(kt, f);
      qb.step(y, f, kt);
    }
    y_rest(t, l, last, y, Ub);
    rows_out(y, last + v_at, last + v_mine, pv, yg, lane < sp.T - (sp.n - 1) * C);
  }
  if (a.hT) state_out<K>(S, a.hT, st_at, a.state_bf16, V, g, c);
}

template <int K, bool PACKED>
__global__ void __launch_bounds__(160, 2) delta_chain_bwd_kernel(DeltaArgs a, int stages) {
  CHAIN_BEGIN(a.dy, (long long)a.N * a.V, true, false);
  float S[K / 8][4];    // dS
  if (a.d_hT) state_in<K>(S, a.d_hT, st_at, a.state_bf16, V, g, c);
  else
#pragma unroll
    for (int nt = 0; nt < K / 8; ++nt)
#pragma unroll
      for (int r = 0; r < 4; ++r) S[nt][r] = 0.f;
  const size_t slot = (size_t)(sp.slot0 + sp.n - 1) * a.N + n;
  char *sg = a.dstates + slot * (2 * K * V) + 2 * K * v0 + 4 * lane, *lg = a.lam + slot * (2 * C * V) + 2 * C * v0 + 4 * lane;
  __nv_bfloat16 *dvg = static_cast<__nv_bfloat16 *>(a.dv) + ((size_t)(sp.tok0 + (sp.n - 1) * C + lane) * a.N + n) * V + v0;
  int st = 0;
  uint32_t phase = 0;
  bool ready = sp.n > 0 && mbar_try_wait(bars.full, 0);
  for (int i = 0; i < sp.n; ++i) {
    const int ch = sp.n - 1 - i;
    if (!__all_sync(0xffffffffu, ready) && !mbar_wait(bars.full + st, phase)) {
      if (lane == 0) report_timeout(a.dev_status);
      return;
    }
    const uint32_t stage = ring + st * sb, qsa = stage + C * pitch_k(K), vec = stage + r_off + kRecVec + 8 * c;
    RowsT<K> kb;
    kb.start(stage, l);
    Rows<K> rb;
    rb.start(qsa, l);
    uint32_t yt[2][4], A[2][4], T[3][4], TL[3][4], P[3][4];
    rows_in(yt, stage + v_at, pv);
    const float ec = __expf(lds32(stage + r_off + kRecVec + 128 * kVecG + 124));
    {      // s e^g dY
      float E[4][4];
#pragma unroll
      for (int nt = 0; nt < 4; ++nt) {
        const float2 e = lds64(vec + 128 * kVecEq + 32 * nt);
        const float2 x0 = unpack_bf16(yt[nt >> 1][2 * (nt & 1)]), x1 = unpack_bf16(yt[nt >> 1][2 * (nt & 1) + 1]);
        E[nt][0] = e.x * x0.x; E[nt][1] = e.y * x0.y; E[nt][2] = e.x * x1.x; E[nt][3] = e.y * x1.y;
      }
      pack_a<4>(E, 0, A[0]);
      pack_a<4>(E, 1, A[1]);
    }
    float acc[4][4];
    zero(acc);
#pragma unroll
    for (int kt = 0; kt < K / 16; ++kt) {      // K^ dS', and e^g_last dS' + (s e^g Q^)^T dY
      uint32_t f[4];
      pack_a<K / 8>(S, kt, f);
      blocks_to(f, sg, K / 8, kt);
#pragma unroll
      for (int r = 0; r < 4; ++r) { S[2 * kt][r] *= ec; S[2 * kt + 1][r] *= ec; }
      kb.step(acc, f, kt);
      rb.step(S, A, kt);
    }
    // dU
    lower_in(P, stage + r_off + kRecP, l);
#pragma unroll
    for (int nt = 0; nt < 4; ++nt) {
      const float2 e = lds64(vec + 128 * kVecEk + 32 * nt);
      acc[nt][0] *= e.x; acc[nt][1] *= e.y; acc[nt][2] *= e.x; acc[nt][3] *= e.y;
    }
    mul_lower(acc, yt, P);     // (packed accumulators [2kt], [2kt + 1] are the A operand of k-tile kt)
    lower_in(T, stage + r_off + kRecT, l);
    low_in(TL, stage + r_off, l);
    pack_a<4>(acc, 0, A[0]);
    pack_a<4>(acc, 1, A[1]);
    float L[4][4];
    zero(L);
    mul_lower(L, A, TL);
    mul_lower(L, A, T);
    rb.start(stage, l);
    float dv[4][4];
#pragma unroll
    for (int kt = 0; kt < 2; ++kt) {
      uint32_t f[4];
      pack_a<4>(L, kt, f);
      blocks_to(f, lg, 4, kt);
#pragma unroll
      for (int nt = 2 * kt; nt < 2 * kt + 2; ++nt) {
        const float2 b = lds64(vec + 128 * kVecBeta + 32 * nt), e = lds64(vec + 128 * kVecEgk + 32 * nt);
        dv[nt][0] = L[nt][0] * b.x; dv[nt][1] = L[nt][1] * b.y; dv[nt][2] = L[nt][2] * b.x; dv[nt][3] = L[nt][3] * b.y;
        L[nt][0] = -e.x * dv[nt][0]; L[nt][1] = -e.y * dv[nt][1]; L[nt][2] = -e.x * dv[nt][2]; L[nt][3] = -e.y * dv[nt][3];
      }
      pack_a<4>(L, kt, A[kt]);
    }
    const int next = st + 1 == stages ? 0 : st + 1;
    const uint32_t next_phase = phase ^ (next == 0);
    ready = i + 1 < sp.n && mbar_try_wait(bars.full + next, next_phase);
    // dS
    rb.run(S, A);
    rows_out(dv, stage + v_at, stage + v_mine, pv, dvg, lane < sp.T - ch * C);      // (through dY's place, which has been read)
    dvg -= (size_t)C * a.N * V;
    sg -= (size_t)a.N * (2 * K * V);
    lg -= (size_t)a.N * (2 * C * V);
    __syncwarp();
    if (lane == 0) mbar_arrive(bars.empty + st);
    st = next;
    phase = next_phase;
  }
  if (a.dh0) state_out<K>(S, a.dh0, st_at, a.state_bf16, V, g, c);
}

// (The figures in here were taken with T in one part; the second adds 2 to 4 % to either side of each.)
// 16-column warps of a CTA: four (they share the copies of k, q and the records), two or one where that leaves a quarter fewer chains to
// the SM that has the most: chains of an SM share its shared memory's bandwidth (65 536 tokens, 32 heads of 128 x 128: 64 CTAs of four
// 2 354 us, 128 of two 1 576, both with Y in the chains).
ChainPlan plan_chain(const DeltaArgs &a, bool with_y) {
  const int cols = a.V / 16;
  const long long units = (long long)a.B * a.N, sms = sm_count();
  ChainPlan p{1, 1, 4, 0, 0};
  long long least = 0;
  for (int nw = cols < 4 ? cols : 4; nw >= 1; nw /= 2) {
    const long long chains = (units * (cols / nw) + sms - 1) / sms * nw;
    if (!least || 4 * chains <= 3 * least) { least = chains; p.nw = nw; }
  }
  p.slabs = cols / p.nw;
  // Two CTAs to an SM where there are that many, but above K = 64 one: four chains of K = 128 take 1.5 us a chunk, eight 2.9, and a batch
  // is done no sooner than its longest sequence (12 of up to 4 000 tokens, 16 heads: 370 us with two, 266 with one).  These are CTAs of four
  // chains; those of one (V = 16) follow the rule too, which was not measured where there are more of them than SMs.
  const bool one = a.K > 64;
  const long long per = (units * p.slabs + sms - 1) / sms;
  // Y in warps of their own where an SM has one CTA, or up to four of one chain (2 001 tokens a sequence, us without and with): 84 heads of 128 x 16
  // 52, 40; 32 heads of 128 x 128 (two chains to an SM) 54, 49; the ragged batch of 128 x 128 (four) 270, 242; 84 heads of 64 x 16, 1 sequence 34,
  // 29, with the states kept 36, 31, 2 sequences 46, 43, 4 (three to an SM) 67, 61, 6 (four) 95, 79.  But four chains of 64 x 64 in a CTA 49.5, 55.7, and
  // K = 16 20.9, 22.8.
  p.apart = !with_y ? 0 : p.nw == 4 ? (one ? 2 : 0) : one || (a.K > 16 && per <= (p.nw == 1 ? 4 : 1)) ? 1 : 0;
  const size_t room = (size_t)(226 / (one || per <= 1 ? 1 : p.apart ? (int)per : 2)) * 1024, sb = (size_t)stage_bytes(a.K, p.nw);
  const size_t fixed = p.apart ? (size_t)p.nw * 2 * apart_bytes(a.K) : (size_t)p.nw * out_bytes(a.K) + C * pitch_v(p.nw);
  while (p.stages > 3 && fixed + p.stages * sb > room) --p.stages;
  p.smem = std::max(fixed + p.stages * sb, one ? (size_t)115 * 1024 : 0);
  return p;
}

template <int K, bool PACKED, int APART> auto fwd_kernel(bool keep) {
  return keep ? delta_chain_fwd_kernel<K, true, true, PACKED, APART> : delta_chain_fwd_kernel<K, true, false, PACKED, APART>;
}
template <int K, bool PACKED> cudaError_t launch_kp(const DeltaArgs &args, bool backward, cudaStream_t s) {
  DeltaArgs a = args;
  const ChainPlan p = plan_chain(a, !backward && a.y);
  a.nw = p.nw; a.sms = sm_count();
  void (*kernel)(DeltaArgs, int) = backward ? delta_chain_bwd_kernel<K, PACKED> : !a.y ? delta_chain_fwd_kernel<K, false, true, PACKED, 0>
                                   : p.apart == 0 ? fwd_kernel<K, PACKED, 0>(a.states) : p.apart == 1 ? fwd_kernel<K, PACKED, 1>(a.states)
                                                                                                     : fwd_kernel<K, PACKED, (K > 64 ? 2 : 1)>(a.states);
  const cudaError_t e = allow_smem(kernel, p.smem);
  if (e != cudaSuccess) return e;
  return launch_early(kernel, dim3((unsigned)((long long)a.B * a.N * p.slabs)), dim3(p.apart ? (p.nw == 2 ? 224 : 32 * (2 * p.nw + 1)) : p.nw == 2 ? 128 : 32 * (p.nw + 1)), p.smem, s, a, p.stages);
}
template <int K> cudaError_t launch_k(const DeltaArgs &a, bool backward, cudaStream_t s) {
  return a.cu ? launch_kp<K, true>(a, backward, s) : launch_kp<K, false>(a, backward, s);
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
