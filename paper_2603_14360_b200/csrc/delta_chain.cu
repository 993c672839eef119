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

// The copying warp's loop, in the order that `backward` says.  V: the tensor whose columns the warps own.
template <int K>
__device__ __forceinline__ void chain_fill(const DeltaArgs &a, const ChainWork &w, const DeltaSpan &sp, const __nv_bfloat16 *vg, long long vs, int nw,
                                           int stages, uint32_t ring, uint64_t *full, uint64_t *empty, int lane, bool backward) {
  const int hq = w.n0 / (a.N / a.Nq), hk = w.n0 / (a.N / a.Nk), pv = pitch_v(nw);
  const uint32_t sb = (uint32_t)stage_bytes(K, nw, a.hpc);
  const __nv_bfloat16 *kp = static_cast<const __nv_bfloat16 *>(a.k) + sp.tok0 * a.ks + (long long)hk * K;
  const __nv_bfloat16 *qp = static_cast<const __nv_bfloat16 *>(a.q) + sp.tok0 * a.qs + (long long)hq * K;
  const __nv_bfloat16 *vp = vg + sp.tok0 * vs + (long long)w.n0 * a.V + w.slab * 16 * a.wv;
  for (int i = 0; i < sp.n; ++i) {
    const int ch = backward ? sp.n - 1 - i : i, st = i % stages, have = min(C, sp.T - ch * C);
    if (i >= stages && !mbar_wait<64>(empty + st, (uint32_t)((i / stages - 1) & 1))) {
      if (lane == 0) report_timeout(a.dev_status);
      for (int o = i - stages; o < i; ++o) (void)mbar_wait(full + o % stages, (uint32_t)((o / stages) & 1));   // its copies on their way
      return;
    }
    const uint32_t base = ring + st * sb, vd = base + 2 * C * pitch_k(K), rd = vd + C * pv;
    if (lane == 0) {
      mbar_expect(full + st, (uint32_t)(a.hpc * kRecChain));
      const char *rec = a.rec + ((size_t)(sp.slot0 + ch) * a.N + w.n0) * kRecBytes;
      for (int h = 0; h < a.hpc; ++h) bulk_load(rd + h * kRecChain, rec + (size_t)h * kRecBytes, kRecChain, full + st);
    }
    // 16 bytes a lane and copy, neighbouring lanes in a row; rows behind the last token are zeros
    const long long t0 = (long long)ch * C;
#pragma unroll 4
    for (int x = lane; x < C * (K / 8); x += 32) {
      const int r = x / (K / 8), o = x % (K / 8);
      const bool ok = r < have;
      cp16_or_zero(base + r * pitch_k(K) + 16 * o, kp + (t0 + (ok ? r : 0)) * a.ks + 8 * o, ok);
      cp16_or_zero(base + (C + r) * pitch_k(K) + 16 * o, qp + (t0 + (ok ? r : 0)) * a.qs + 8 * o, ok);
    }
    const int log_v = 31 - __clz(2 * nw);      // pieces of a row of V: a power of two
#pragma unroll 4
    for (int x = lane; x < C << log_v; x += 32) {
      const int r = x >> log_v, o = x & (2 * nw - 1);
      const bool ok = r < have;
      cp16_or_zero(vd + r * pv + 16 * o, vp + (t0 + (ok ? r : 0)) * vs + 8 * o, ok);
    }
    cp_arrive(full + st);
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
// A operands of S^T to memory as 8 x 8 blocks (block (vb, kb) at 128 (vb K/8 + kb) bytes, rows of columns v)
template <int K>
__device__ __forceinline__ void blocks_out(const uint32_t (&f)[K / 16][4], char *p, int vb, int lane) {
  uint32_t *o = reinterpret_cast<uint32_t *>(p) + lane;
#pragma unroll
  for (int kt = 0; kt < K / 16; ++kt)
#pragma unroll
    for (int r = 0; r < 4; ++r) o[32 * ((vb + (r & 1)) * (K / 8) + 2 * kt + (r >> 1))] = f[kt][r];
}

// ldmatrix addresses of a lane
struct Lanes {
  uint32_t row, mat_lo, mat_hi;   // row of an 8 x 8 matrix, and which of two matrices in each direction
  __device__ explicit Lanes(int lane) : row(lane & 7), mat_lo((lane >> 3) & 1), mat_hi(lane >> 4) {}
};

// acc[4 token tiles] += A (16 x K) . rows^T: rows [32 tokens][K] in shared memory
template <int K>
__device__ __forceinline__ void mul_rows_t(float (&acc)[4][4], const uint32_t (&A)[K / 16][4], uint32_t rows, const Lanes &l) {
  const uint32_t at = rows + (l.row + 8 * l.mat_hi) * pitch_k(K) + 16 * l.mat_lo;
#pragma unroll
  for (int kt = 0; kt < K / 16; ++kt)
#pragma unroll
    for (int np = 0; np < 2; ++np) {
      uint32_t b[4];
      ldmatrix_x4(at + 16 * np * pitch_k(K) + 32 * kt, b);
      mma_bf16_16816(acc[2 * np], A[kt], b[0], b[1]);
      mma_bf16_16816(acc[2 * np + 1], A[kt], b[2], b[3]);
    }
}
// S (16 x K) += A (16 x 32 tokens) . rows
template <int K>
__device__ __forceinline__ void mul_rows(float (&S)[K / 8][4], const uint32_t (&A)[2][4], uint32_t rows, const Lanes &l) {
  const uint32_t at = rows + (l.row + 8 * l.mat_lo) * pitch_k(K) + 16 * l.mat_hi;
#pragma unroll
  for (int np = 0; np < K / 16; ++np)
#pragma unroll
    for (int kt = 0; kt < 2; ++kt) {
      uint32_t b[4];
      ldmatrix_x4_t(at + 16 * kt * pitch_k(K) + 32 * np, b);
      mma_bf16_16816(S[2 * np], A[kt], b[0], b[1]);
      mma_bf16_16816(S[2 * np + 1], A[kt], b[2], b[3]);
    }
}
// acc (16 x 32) += A (16 x 32) . M^T, M lower triangular as blocks
__device__ __forceinline__ void mul_lower_t(float (&acc)[4][4], const uint32_t (&A)[2][4], uint32_t M, const Lanes &l) {
  const uint32_t at = M + 16 * l.row + 128 * (4 * l.mat_hi + l.mat_lo);
#pragma unroll
  for (int np = 0; np < 2; ++np)
#pragma unroll
    for (int kt = 0; kt <= np; ++kt) {
      uint32_t b[4];
      ldmatrix_x4(at + 128 * (8 * np + 2 * kt), b);
      mma_bf16_16816(acc[2 * np], A[kt], b[0], b[1]);
      mma_bf16_16816(acc[2 * np + 1], A[kt], b[2], b[3]);
    }
}
// acc (16 x 32) += A (16 x 32) . M, M lower triangular as blocks
__device__ __forceinline__ void mul_lower(float (&acc)[4][4], const uint32_t (&A)[2][4], uint32_t M, const Lanes &l) {
  const uint32_t at = M + 16 * l.row + 128 * (4 * l.mat_lo + l.mat_hi);
#pragma unroll
  for (int np = 0; np < 2; ++np)
#pragma unroll
    for (int kt = np; kt < 2; ++kt) {
      uint32_t b[4];
      ldmatrix_x4_t(at + 128 * (8 * kt + 2 * np), b);
      mma_bf16_16816(acc[2 * np], A[kt], b[0], b[1]);
      mma_bf16_16816(acc[2 * np + 1], A[kt], b[2], b[3]);
    }
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
// ... and back to memory through its place in shared memory: rows of 32 bytes, a token a lane
__device__ __forceinline__ void rows_out(const uint32_t (&p)[2][4], uint32_t at, uint32_t mine, int pv, __nv_bfloat16 *out, bool ok) {
  stmatrix_x4_trans(at, p[0]);
  stmatrix_x4_trans(at + 16 * pv, p[1]);
  __syncwarp();
  if (ok) {
    const float4 x = lds128(mine), y = lds128(mine + 16);
    reinterpret_cast<float4 *>(out)[0] = x;
    reinterpret_cast<float4 *>(out)[1] = y;
  }
}

template <int K>
__global__ void __launch_bounds__(160) delta_chain_fwd_kernel(DeltaArgs a, int stages) {
  extern __shared__ __align__(128) unsigned char smem[];
  __shared__ uint64_t full[8], empty[8];
  const int nw = a.hpc * a.wv, warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31, g = lane >> 2, c = lane & 3;
  if (threadIdx.x == 0) {
    for (int i = 0; i < stages; ++i) { mbar_init(full + i, 33); mbar_init(empty + i, nw); }
    fence_mbar_init();
  }
  begin_dependent();
  __syncthreads();
  const ChainWork w = chain_work(a, smem);
  const DeltaSpan sp = delta_span<C>(a, w.b);
  const uint32_t ring = smem_u32(smem);
  if (warp == nw) {
    chain_fill<K>(a, w, sp, static_cast<const __nv_bfloat16 *>(a.v), a.vs, nw, stages, ring, full, empty, lane, false);
    return;
  }
  const int n = w.n0 + warp / a.wv, v0 = 16 * (w.slab * a.wv + warp % a.wv), V = a.V, pv = pitch_v(nw);
  const size_t st_at = ((size_t)w.b * a.N + n) * K * V + v0;
  const Lanes l(lane);
  float S[K / 8][4];
  if (a.h0) state_in<K>(S, a.h0, st_at, a.state_bf16, V, g, c);
  else
#pragma unroll
    for (int nt = 0; nt < K / 8; ++nt)
#pragma unroll
      for (int r = 0; r < 4; ++r) S[nt][r] = 0.f;
  const uint32_t sb = (uint32_t)stage_bytes(K, nw, a.hpc);
  __nv_bfloat16 *yg = a.y ? static_cast<__nv_bfloat16 *>(a.y) + ((size_t)(sp.tok0 + lane) * a.N + n) * V + v0 : nullptr;
  const size_t y_step = (size_t)C * a.N * V;
  for (int ch = 0; ch < sp.n; ++ch) {
    const int st = ch % stages, have = min(C, sp.T - ch * C);
    if (!mbar_wait(full + st, (uint32_t)((ch / stages) & 1))) {
      if (lane == 0) report_timeout(a.dev_status);
      return;
    }
    const uint32_t ksa = ring + st * sb, qsa = ksa + C * pitch_k(K), vsa = qsa + C * pitch_k(K), rec = vsa + C * pv + (warp / a.wv) * kRecChain;
    const uint32_t vec = rec + kRecVec + 8 * c;
    uint32_t Sb[K / 16][4];
#pragma unroll
    for (int kt = 0; kt < K / 16; ++kt) pack_a<K / 8>(S, kt, Sb[kt]);
    const size_t slot = (size_t)(sp.slot0 + ch) * a.N + n;
    if (a.states) blocks_out<K>(Sb, a.states + slot * (2 * K * V), v0 / 8, lane);
    float acc[4][4];
    zero(acc);
    mul_rows_t<K>(acc, Sb, ksa, l);
    // X
    const uint32_t vat = vsa + 32 * warp + (l.row + 8 * l.mat_hi) * pv + 16 * l.mat_lo;
    uint32_t vt[2][4];
    rows_in(vt, vat, pv);
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
    mul_lower_t(U, A, rec + kRecT, l);
    pack_a<4>(U, 0, A[0]);
    pack_a<4>(U, 1, A[1]);
    if (a.upd) {
      uint32_t *o = reinterpret_cast<uint32_t *>(a.upd + slot * (2 * C * V)) + lane;
#pragma unroll
      for (int kt = 0; kt < 2; ++kt)
#pragma unroll
        for (int r = 0; r < 4; ++r) o[32 * ((v0 / 8 + (r & 1)) * 4 + 2 * kt + (r >> 1))] = A[kt][r];
    }
    // S'
    {
      const float ec = expf(lds32(rec + kRecVec + 128 * kVecG + 124));
#pragma unroll
      for (int nt = 0; nt < 4; ++nt) {
        const float2 e = lds64(vec + 128 * kVecEk + 32 * nt);
        U[nt][0] *= e.x; U[nt][1] *= e.y; U[nt][2] *= e.x; U[nt][3] *= e.y;
      }
      uint32_t E[2][4];
      pack_a<4>(U, 0, E[0]);
      pack_a<4>(U, 1, E[1]);
#pragma unroll
      for (int nt = 0; nt < K / 8; ++nt)
#pragma unroll
        for (int r = 0; r < 4; ++r) S[nt][r] *= ec;
      mul_rows<K>(S, E, ksa, l);
    }
    if (yg) {
      zero(acc);
      mul_rows_t<K>(acc, Sb, qsa, l);
#pragma unroll
      for (int nt = 0; nt < 4; ++nt) {
        const float2 e = lds64(vec + 128 * kVecEq + 32 * nt);
        acc[nt][0] *= e.x; acc[nt][1] *= e.y; acc[nt][2] *= e.x; acc[nt][3] *= e.y;
      }
      mul_lower_t(acc, A, rec + kRecP, l);
      uint32_t yt[2][4];
#pragma unroll
      for (int nt = 0; nt < 4; ++nt) {
        yt[nt >> 1][2 * (nt & 1)] = pack_bf16(acc[nt][0], acc[nt][1]);
        yt[nt >> 1][2 * (nt & 1) + 1] = pack_bf16(acc[nt][2], acc[nt][3]);
      }
      rows_out(yt, vat, vsa + 32 * warp + lane * pv, pv, yg, lane < have);
      yg += y_step;
    }
    __syncwarp();
    if (lane == 0) mbar_arrive(empty + st);
  }
  if (a.hT) state_out<K>(S, a.hT, st_at, a.state_bf16, V, g, c);
}

template <int K>
__global__ void __launch_bounds__(160) delta_chain_bwd_kernel(DeltaArgs a, int stages) {
  extern __shared__ __align__(128) unsigned char smem[];
  __shared__ uint64_t full[8], empty[8];
  const int nw = a.hpc * a.wv, warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31, g = lane >> 2, c = lane & 3;
  if (threadIdx.x == 0) {
    for (int i = 0; i < stages; ++i) { mbar_init(full + i, 33); mbar_init(empty + i, nw); }
    fence_mbar_init();
  }
  begin_dependent();
  __syncthreads();
  const ChainWork w = chain_work(a, smem);
  const DeltaSpan sp = delta_span<C>(a, w.b);
  const uint32_t ring = smem_u32(smem);
  const int V = a.V;
  if (warp == nw) {
    chain_fill<K>(a, w, sp, static_cast<const __nv_bfloat16 *>(a.dy), (long long)a.N * V, nw, stages, ring, full, empty, lane, true);
    return;
  }
  const int n = w.n0 + warp / a.wv, v0 = 16 * (w.slab * a.wv + warp % a.wv), pv = pitch_v(nw);
  const size_t st_at = ((size_t)w.b * a.N + n) * K * V + v0;
  const Lanes l(lane);
  float S[K / 8][4];    // dS
  if (a.d_hT) state_in<K>(S, a.d_hT, st_at, a.state_bf16, V, g, c);
  else
#pragma unroll
    for (int nt = 0; nt < K / 8; ++nt)
#pragma unroll
      for (int r = 0; r < 4; ++r) S[nt][r] = 0.f;
  const uint32_t sb = (uint32_t)stage_bytes(K, nw, a.hpc);
  __nv_bfloat16 *dvg = static_cast<__nv_bfloat16 *>(a.dv) + ((size_t)(sp.tok0 + lane) * a.N + n) * V + v0;
  for (int i = 0; i < sp.n; ++i) {
    const int ch = sp.n - 1 - i, st = i % stages, have = min(C, sp.T - ch * C);
    if (!mbar_wait(full + st, (uint32_t)((i / stages) & 1))) {
      if (lane == 0) report_timeout(a.dev_status);
      return;
    }
    const uint32_t ksa = ring + st * sb, qsa = ksa + C * pitch_k(K), vsa = qsa + C * pitch_k(K), rec = vsa + C * pv + (warp / a.wv) * kRecChain;
    const uint32_t vec = rec + kRecVec + 8 * c;
    const size_t slot = (size_t)(sp.slot0 + ch) * a.N + n;
    float acc[4][4];
    zero(acc);
    {
      uint32_t Sb[K / 16][4];
#pragma unroll
      for (int kt = 0; kt < K / 16; ++kt) pack_a<K / 8>(S, kt, Sb[kt]);
      blocks_out<K>(Sb, a.dstates + slot * (2 * K * V), v0 / 8, lane);
      mul_rows_t<K>(acc, Sb, ksa, l);
    }
    // dU
    const uint32_t vat = vsa + 32 * warp + (l.row + 8 * l.mat_hi) * pv + 16 * l.mat_lo;
    uint32_t yt[2][4];
    rows_in(yt, vat, pv);
#pragma unroll
    for (int nt = 0; nt < 4; ++nt) {
      const float2 e = lds64(vec + 128 * kVecEk + 32 * nt);
      acc[nt][0] *= e.x; acc[nt][1] *= e.y; acc[nt][2] *= e.x; acc[nt][3] *= e.y;
    }
    mul_lower(acc, yt, rec + kRecP, l);     // (packed accumulators [2kt], [2kt + 1] are the A operand of k-tile kt)
    uint32_t A[2][4];
    pack_a<4>(acc, 0, A[0]);
    pack_a<4>(acc, 1, A[1]);
    float L[4][4];
    zero(L);
    mul_lower(L, A, rec + kRecT, l);
    {
      uint32_t *o = reinterpret_cast<uint32_t *>(a.lam + slot * (2 * C * V)) + lane;
#pragma unroll
      for (int nt = 0; nt < 4; ++nt)
#pragma unroll
        for (int h = 0; h < 2; ++h) o[32 * ((v0 / 8 + h) * 4 + nt)] = pack_bf16(L[nt][2 * h], L[nt][2 * h + 1]);
    }
    // dS
    {
      const float ec = expf(lds32(rec + kRecVec + 128 * kVecG + 124));
#pragma unroll
      for (int nt = 0; nt < K / 8; ++nt)
#pragma unroll
        for (int r = 0; r < 4; ++r) S[nt][r] *= ec;
      float E[4][4];
#pragma unroll
      for (int nt = 0; nt < 4; ++nt) {
        const float2 e = lds64(vec + 128 * kVecEq + 32 * nt);
        const float2 x0 = unpack_bf16(yt[nt >> 1][2 * (nt & 1)]), x1 = unpack_bf16(yt[nt >> 1][2 * (nt & 1) + 1]);
        E[nt][0] = e.x * x0.x; E[nt][1] = e.y * x0.y; E[nt][2] = e.x * x1.x; E[nt][3] = e.y * x1.y;
      }
      pack_a<4>(E, 0, A[0]);
      pack_a<4>(E, 1, A[1]);
      mul_rows<K>(S, A, qsa, l);
      uint32_t dvt[2][4];
#pragma unroll
      for (int nt = 0; nt < 4; ++nt) {
        const float2 b = lds64(vec + 128 * kVecBeta + 32 * nt), e = lds64(vec + 128 * kVecEgk + 32 * nt);
        L[nt][0] *= b.x; L[nt][1] *= b.y; L[nt][2] *= b.x; L[nt][3] *= b.y;
        dvt[nt >> 1][2 * (nt & 1)] = pack_bf16(L[nt][0], L[nt][1]);
        dvt[nt >> 1][2 * (nt & 1) + 1] = pack_bf16(L[nt][2], L[nt][3]);
        L[nt][0] *= -e.x; L[nt][1] *= -e.y; L[nt][2] *= -e.x; L[nt][3] *= -e.y;
      }
      pack_a<4>(L, 0, A[0]);
      pack_a<4>(L, 1, A[1]);
      mul_rows<K>(S, A, ksa, l);
      rows_out(dvt, vat, vsa + 32 * warp + lane * pv, pv, dvg + (size_t)ch * C * a.N * V, lane < have);
    }
    __syncwarp();
    if (lane == 0) mbar_arrive(empty + st);
  }
  if (a.dh0) state_out<K>(S, a.dh0, st_at, a.state_bf16, V, g, c);
}

// Heads and 16-column warps of a CTA.  A state's columns stay together (they share the copies of k, q and the records)
// while there are CTAs for all SMs; with fewer units they are spread.
ChainPlan plan_chain(const DeltaArgs &a) {
  const int cols = a.V / 16;
  const long long units = (long long)a.B * a.N, sms = sm_count();
  ChainPlan p{1, cols < 4 ? cols : 4, 1, 2, 0};
  while (p.wv > 1 && units * (cols / p.wv) < sms) p.wv /= 2;
  p.slabs = cols / p.wv;
  const size_t sb = (size_t)stage_bytes(a.K, p.hpc * p.wv, p.hpc);
  p.stages = 4;
  p.smem = p.stages * sb;
  return p;
}

template <int K> cudaError_t launch_k(const DeltaArgs &args, bool backward, cudaStream_t s) {
  DeltaArgs a = args;
  const ChainPlan p = plan_chain(a);
  a.hpc = p.hpc; a.wv = p.wv;
  void (*kernel)(DeltaArgs, int) = backward ? delta_chain_bwd_kernel<K> : delta_chain_fwd_kernel<K>;
  const cudaError_t e = allow_smem(kernel, p.smem);
  if (e != cudaSuccess) return e;
  return launch_early(kernel, dim3((unsigned)((long long)a.B * (a.N / p.hpc) * p.slabs)), dim3(32 * (p.hpc * p.wv + 1)), p.smem, s, a, p.stages);
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
