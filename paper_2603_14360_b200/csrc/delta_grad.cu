// Gated delta rule, bf16: gradients of q, k, the gate and the step, chunk by chunk, from what the chains kept
// (delta_chain.cu: S at a chunk's start, U; dS' at its end, L = dU through T^T).  With r_q, r_k the reciprocal lengths,
// E_ij = e^(g_i - g_j), dP_ij = dY_i . U_j and N_ij = -L_i . U_j, two 32 x 32 matrices
//     X1_ij = s r_q,i r_k,j E_ij dP_ij   (j <= i)        X2_ij = b_i r_k,i r_k,j E_ij N_ij   (j < i)
// serve both sides of their products:
//     dq' = s e^g r_q dY S^T + X1 K                                          (r_q times the gradient of q r_q)
//     dk' = -b e^g r_k L S^T + e^(g_last - g) r_k U dS'^T + (X2 + X2^T) K + X1^T Q
// Every sum over features that is needed comes from three of the products with the states, a1 = q . dY S^T, a2 = k . L S^T,
// a3 = k . U dS'^T, and from the rows and columns of X1 (.) Q K^T and X2 (.) K K^T:
//     dx = x' - r^2 x (x . x')  (the division by the lengths)        db_i = L_i . v_i - e^g r_k a2 + sum_j X2_ij k_i . k_j / b_i
// The decays' gradient sums what crosses token t's decay: what tokens from t on read of S, what tokens before t write
// into S', the pairs on either side of it, and S on its way to S':
//     R_i = s e^g r_q a1 - b e^g r_k a2        W_j = e^(g_last - g) r_k a3        G_ij = X1_ij q_i . k_j + X2_ij k_i . k_j   (j < i)
//     d log a_t = e^g_last <S, dS'> + sum_{i >= t} R_i + sum_{j < t} W_j + sum_{j < t <= i} G_ij
// (With q . dq - k . dk in place of R, W and G the pairs on one side of t would cancel only up to the roundings of
// the matrices to bf16: 2.5e-2 off where states decay within a few tokens.  Here the same fp32 value is added and taken away.)
//
// 2 KG warps: 16 tokens x one of KG parts of the K features each; the products over V in slabs of 64 columns (32 where K > 64 or where
// heads share q and k).  (Four parts: half the accumulators a thread, but every warp loads all of dY, L and U; slower at three CTAs to an SM.)
// A job is a chunk of `hpc` heads that share q and k, one after the other: their X1, X2, dq', dk' are added up in registers, and the products
// with Q and K, which are the same for all of them, taken once.  Two or three CTAs to an SM (delta_grad_plan) walk over the jobs, the next slab
// (and the next job's rows) on its way while one is worked on: with a CTA a job the loads' latency stood between a third of the cycles.  Where
// both buffers of a slab leave no room for a third CTA (V = 64, heads of their own) there is one buffer: 469 us for the second shape below, 497
// with two and two.  What the chains wrote is contiguous and comes by untiled bulk copies; rows of q, k, v and dY by cp.async; results go straight to
// memory, 16 bytes of a row an instruction.
// 16 384 tokens, 84 heads of 64 x 16 on one q and k: 351 us; 32 768 tokens, 32 heads of 64 x 64: 469 us, 49 KB a chunk and head or 3.4 TB/s;
// 25 026 packed tokens, 16 heads of 128 x 128: 425 us.  Bound by the latency of its products, shuffles and shared-memory reads.
#include "delta_common.cuh"

namespace m2rnn {
namespace {

constexpr int C = kDeltaChunk, KG = 2;

template <int K> struct GradCfg {
  static constexpr int kThreads = 64 * KG;
  static constexpr int kPK = 2 * K + 16;
  static constexpr int kRows = 2 * C * kPK, kMat = 2 * kRows;            // q, k rows, twice; X1, X2 as blocks
  static constexpr int kRed = kMat + 2 * 2048;                           // sums: rows as named below
  static constexpr int kSlab = kRed + (5 * KG + 7) * 128;                // slabs: the vectors, dY, V rows, then U, L, S, dS' blocks
  static constexpr int NT = (K / 8 + KG - 1) / KG;                       // 8-feature tiles of a warp, most
  static constexpr int JT = 4 / KG;                                      // 8-token tiles of a warp's part of a 16 x 32 product
  // rows of 32 floats: a1, a2, a3 by part of the features; sums of X1 (.) QK^T and X2 (.) KK^T / b over a row's entries by part of
  // the tokens; over a column's by half; X1 (.) QK^T's diagonal; L . v; the factors of the division by the lengths; <S, dS'>
  static constexpr int kA = 0, kRow1 = 3 * KG, kRow2 = 4 * KG, kCol = 5 * KG, kDiag = kCol + 2, kLv = kCol + 3, kUq = kCol + 4, kUk = kCol + 5, kSds = kCol + 6;
  static_assert(kSlab % 16 == 0, "");
};
__host__ __device__ constexpr int slab_bytes(int K, int VS) { return 1024 + 2 * C * (2 * VS + 16) + 2 * 2 * C * VS + 2 * 2 * K * VS; }

struct GradJob { long long tok; size_t slot; int have, n0, run, hq, hk; };      // have = 0: no more

// MULTI: several heads to a job; VS: columns of a slab
template <int K, bool MULTI, int VS, int BUFS, int CTAS>
__global__ void __launch_bounds__(64 * KG, CTAS) delta_grad_kernel(DeltaArgs a, unsigned jobs) {
  using Cfg = GradCfg<K>;
  constexpr int NT = Cfg::NT, JT = Cfg::JT, kThreads = Cfg::kThreads, kIdle = 2 * (KG - 1);
  constexpr int pv = 2 * VS + 16, P = VS / 8, slab = slab_bytes(K, VS), UB = 2 * C * VS, SB = 2 * K * VS;      // P: pieces of a row; bytes of U, of S
  extern __shared__ __align__(128) unsigned char smem[];
  __shared__ uint64_t full[2];
  const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = tid & 31, g = lane >> 2, c = lane & 3;
  if (tid == 0) {
    mbar_init(full, 1);
    mbar_init(full + 1, 1);
    fence_mbar_init();
  }
  const int mh = warp & 1, kq = warp >> 1, i0 = 16 * mh, f0 = 8 * NT * kq;      // tokens i0 .., features f0 ..
  const int tiles = K % (8 * KG) == 0 ? NT : min(NT, max(0, K / 8 - NT * kq));  // 8-feature tiles that this warp has
  const int V = a.V, parts = (unsigned)V / VS;
  const uint32_t base = smem_u32(smem), mat = base + Cfg::kMat;
  float *red = reinterpret_cast<float *>(smem + Cfg::kRed);
  const uint32_t mrow = lane & 7, mlo = (lane >> 3) & 1, mhi = lane >> 4;
  const unsigned runs = (unsigned)(a.N / a.hpc);
  begin_dependent();
  __syncthreads();

  // the first job from number j on that there is (of a packed batch a slot may be no sequence's)
  int entry = -1;      // the batch entry of the last one
  auto find = [&](unsigned &j) {
    GradJob o{};
    for (; j < jobs; j += gridDim.x) {
      const unsigned slot = j / runs, run = j - slot * runs;
      if (!a.cu) entry = delta_entry<C, false>(a, slot);
      else if (entry < 0) entry = delta_entry<C, true>(a, slot);
      DeltaSpan sp = delta_span<C>(a, entry);
      while (a.cu && entry + 1 < a.B) {      // (slots only grow)
        const DeltaSpan after = delta_span<C>(a, entry + 1);
        if (after.slot0 > slot) break;
        ++entry;
        sp = after;
      }
      const int ch = (int)(slot - sp.slot0);
      if ((unsigned)ch >= (unsigned)sp.n) continue;
      o.tok = sp.tok0 + ch * C;
      o.slot = (size_t)slot * a.N;
      o.have = min(C, sp.T - ch * C);
      o.run = (int)run;
      o.n0 = (int)run * a.hpc;
      o.hq = (int)((unsigned)o.n0 / (unsigned)a.per_q);
      o.hk = (int)((unsigned)o.n0 / (unsigned)a.per_k);
      break;
    }
    return o;
  };
  // rows of q and k of a job, and slab `part` of its head n, on their way.
  constexpr int NR = (C * (K / 8) + kThreads - 1) / kThreads, NV = (C * P + kThreads - 1) / kThreads;
  auto fetch_rows = [&](const GradJob &o, int qb) {
    const __nv_bfloat16 *kg = static_cast<const __nv_bfloat16 *>(a.k) + o.tok * a.ks + o.hk * K;
    const __nv_bfloat16 *qg = static_cast<const __nv_bfloat16 *>(a.q) + o.tok * a.qs + o.hq * K;
#pragma unroll
    for (int y = 0; y < NR; ++y) {
      const int x = tid + y * kThreads, r = x / (K / 8), p = x % (K / 8);
      if (C * (K / 8) % kThreads && x >= C * (K / 8)) break;
      const bool ok = r < o.have;
      const uint32_t at = base + qb * Cfg::kRows + r * Cfg::kPK + 16 * p;
      cp16_or_zero(at, qg + (ok ? r * a.qs : 0) + 8 * p, ok);
      cp16_or_zero(at + C * Cfg::kPK, kg + (ok ? r * a.ks : 0) + 8 * p, ok);
    }
  };
  auto fetch = [&](const GradJob &o, int n, int part, int buf) {
    const int vb = part * VS;
    const uint32_t at = base + Cfg::kSlab + buf * slab, ysa = at + 1024, vsa = ysa + C * pv, usa = vsa + C * pv;
    if (tid == 0) {
      const size_t slot = o.slot + n, u = slot * (2 * C * V) + 2 * C * vb, x = slot * (2 * K * V) + 2 * K * vb;
      mbar_expect(full + buf, 1024 + 2 * (UB + SB));
      bulk_load(at, a.rec + slot * kRecBytes + kRecVec, 1024, full + buf);
      bulk_load(usa, a.upd + u, UB, full + buf);
      bulk_load(usa + UB, a.lam + u, UB, full + buf);
      bulk_load(usa + 2 * UB, a.states + x, SB, full + buf);
      bulk_load(usa + 2 * UB + SB, a.dstates + x, SB, full + buf);
    }
    const __nv_bfloat16 *yg = static_cast<const __nv_bfloat16 *>(a.dy) + (o.tok * a.N + n) * V + vb, *vg = static_cast<const __nv_bfloat16 *>(a.v) + o.tok * a.vs + (long long)n * V + vb;
#pragma unroll
    for (int y = 0; y < NV; ++y) {
      const int x = tid + y * kThreads, r = x / P, p = x % P;
      if (C * P % kThreads && x >= C * P) break;
      const bool ok = r < o.have;
      cp16_or_zero(ysa + r * pv + 16 * p, yg + (ok ? (long long)r * a.N * V : 0) + 8 * p, ok);
      cp16_or_zero(vsa + r * pv + 16 * p, vg + (ok ? r * a.vs : 0) + 8 * p, ok);
    }
  };
  unsigned j = blockIdx.x;
  GradJob o = find(j);
  if (!o.have) return;
  fetch_rows(o, 0);
  fetch(o, o.n0, 0, 0);
  bool fine = true;
  unsigned cnt = 0;      // slabs so far: the buffer's parity and its barrier's phase
  float qk[JT][4], kk[JT][4];                 // q k^T and k k^T, tiles (16 mh, 8 (JT kq + u))
  float dq[NT][4], dm[NT][4], dp[NT][4];      // dY S^T, L S^T, U dS'^T
  float yu[JT][4], lu[JT][4], ld[JT][4];      // dY U^T, L U^T, L V^T, tiles as of qk
  float dqs[NT][4], dks[NT][4], x1s[JT][4], x2s[JT][4];      // dq', dk', X1, X2, summed over a job's heads
  float pqs = 0.f, pks = 0.f;                 // (warp 0) of q . dq', k . dk'
  for (int qb = 0;; qb ^= 1) {
    const uint32_t qsa = base + qb * Cfg::kRows, ksa = qsa + C * Cfg::kPK, qat = qsa + (i0 + g) * Cfg::kPK + 2 * (f0 + 2 * c), kat = qat + C * Cfg::kPK;   // (at: this thread's entries)
    GradJob next{};
    for (int h = 0; h < a.hpc; ++h) {
      const int n = o.n0 + h;
#pragma unroll
      for (int r = 0; r < 4; ++r) {
#pragma unroll
        for (int u = 0; u < JT; ++u) yu[u][r] = lu[u][r] = ld[u][r] = 0.f;
#pragma unroll
        for (int t = 0; t < NT; ++t) dq[t][r] = dm[t][r] = dp[t][r] = 0.f;
      }
      float ss = 0.f, ss1 = 0.f;      // this thread's part of <S, dS'>
      const float *vec = nullptr;
      for (int part = 0; part < parts; ++part, ++cnt) {
        const int bi = BUFS > 1 ? cnt & 1 : 0;
        cp_wait_all();
        if (fine) {      // (after a wait that ran out the rest is worked through with whatever there is: every access is in bounds)
          fine = mbar_wait(full + bi, (BUFS > 1 ? cnt >> 1 : cnt) & 1);
          if (!fine && lane == 0) report_timeout(a.dev_status);
        }
        __syncthreads();
        if (BUFS > 1 && part + 1 < parts) fetch(o, n, part + 1, bi ^ 1);
        else if (BUFS > 1 && h + 1 < a.hpc) fetch(o, n + 1, 0, bi ^ 1);
        else if (part + 1 == parts && h + 1 == a.hpc) {
          j += gridDim.x;
          next = find(j);
          if (next.have) {
            fetch_rows(next, qb ^ 1);
            if (BUFS > 1) fetch(next, next.n0, 0, bi ^ 1);
          }
        }
        unsigned char *buf = smem + Cfg::kSlab + bi * slab;
        const uint32_t at0 = base + Cfg::kSlab + bi * slab, ysa = at0 + 1024, vsa = ysa + C * pv, usa = vsa + C * pv, ssa = usa + 2 * UB;
        vec = reinterpret_cast<const float *>(buf);
        if (h == 0 && part == 0) {
#pragma unroll
          for (int u = 0; u < JT; ++u)
#pragma unroll
            for (int r = 0; r < 4; ++r) qk[u][r] = kk[u][r] = 0.f;
#pragma unroll
          for (int kt = 0; kt < K / 16; ++kt) {
            uint32_t qa[4], ka[4];
            const uint32_t ra = (i0 + (lane & 15)) * Cfg::kPK + 32 * kt + 16 * mhi;
            ldmatrix_x4(qsa + ra, qa);
            ldmatrix_x4(ksa + ra, ka);
#pragma unroll
            for (int u = 0; u < JT; ++u)
              if (JT * kq + u <= 2 * mh + 1) {
                uint32_t kb[2];
                ldmatrix_x2(ksa + (8 * (JT * kq + u) + mrow) * Cfg::kPK + 32 * kt + 16 * mlo, kb);
                mma_add(qk[u], qa, kb[0], kb[1]);
                mma_add(kk[u], ka, kb[0], kb[1]);
              }
          }
        }
        // products over the slab's columns
        const uint32_t y_at = ysa + (i0 + mrow + 8 * mlo) * pv + 16 * mhi, v_at = vsa + (8 * JT * kq + mrow) * pv + 16 * mlo;
        const uint32_t b_at = usa + 16 * mrow + 128 * (4 * mhi + 2 * mh + mlo), u_at = usa + 16 * mrow + 128 * (4 * mlo + JT * kq);   // blocks [column tile][token tile]
        const uint32_t s_one = ssa + 16 * mrow + 128 * (mlo * (K / 8) + f0 / 8), s_at = s_one + 128 * mhi;
#pragma unroll
        for (int kt = 0; kt < VS / 16; ++kt) {
          uint32_t ya[4], la[4], ua[4];     // A operands: 16 tokens x 16 columns
          ldmatrix_x4(y_at + 32 * kt, ya);
          ldmatrix_x4_t(b_at + 1024 * kt, ua);
          ldmatrix_x4_t(b_at + UB + 1024 * kt, la);
#pragma unroll
          for (int u = 0; u < JT; ++u)
            if (JT * kq + u <= 2 * mh + 1) {
              uint32_t ub[2];               // B operands: 16 columns x 8 tokens
              ldmatrix_x2_t(u_at + 1024 * kt + 128 * u, ub);
              mma_add(yu[u], ya, ub[0], ub[1]);
              mma_add(lu[u], la, ub[0], ub[1]);
              if (JT * kq + u >= 2 * mh) {
                ldmatrix_x2(v_at + 32 * kt + 8 * u * pv, ub);
                mma_add(ld[u], la, ub[0], ub[1]);
              }
            }
#pragma unroll
          for (int t = 0; t < NT; t += 2) {
            // B operands: 16 columns x 16 features (of a last tile alone the second is not used)
            if (t >= tiles) continue;
            const uint32_t at = (t + 1 < tiles ? s_at : s_one) + 32 * K * kt + 128 * t;
            uint32_t sb[4], db[4];
            ldmatrix_x4_t(at, sb);
            ldmatrix_x4_t(at + SB, db);
            mma_add(dq[t], ya, sb[0], sb[1]);
            mma_add(dm[t], la, sb[0], sb[1]);
            mma_add(dp[t], ua, db[0], db[1]);
            if (t + 1 < NT && t + 1 < tiles) {
              mma_add(dq[t + 1], ya, sb[2], sb[3]);
              mma_add(dm[t + 1], la, sb[2], sb[3]);
              mma_add(dp[t + 1], ua, db[2], db[3]);
            }
          }
        }
        if (warp == kIdle) {      // <S, dS'>: the warp without a part of X1, X2 has the time
          const unsigned char *sp = buf + (ssa - at0);
#pragma unroll 4
          for (int x = lane; x < K * P; x += 32) {
            const uint4 p = *reinterpret_cast<const uint4 *>(sp + 16 * x), d = *reinterpret_cast<const uint4 *>(sp + SB + 16 * x);
            ss = fma_bf16<0, 0>(p.x, d.x, fma_bf16<1, 1>(p.x, d.x, ss));
            ss1 = fma_bf16<0, 0>(p.y, d.y, fma_bf16<1, 1>(p.y, d.y, ss1));
            ss = fma_bf16<0, 0>(p.z, d.z, fma_bf16<1, 1>(p.z, d.z, ss));
            ss1 = fma_bf16<0, 0>(p.w, d.w, fma_bf16<1, 1>(p.w, d.w, ss1));
          }
        }
        if (BUFS == 1 && part + 1 < parts) {
          __syncthreads();      // (the slab's place is the next one's)
          fetch(o, n, part + 1, 0);
        }
      }
      // X1, X2; rows i of this thread: i0 + g, i0 + g + 8
      float bt[2], r1[2] = {}, r2[2] = {};
#pragma unroll
      for (int x = 0; x < 2; ++x) bt[x] = vec[32 * kVecBeta + i0 + g + 8 * x];
#pragma unroll
      for (int u = 0; u < JT; ++u) {
        const int jt = JT * kq + u, jj = 8 * jt + 2 * c;
        if (jt > 2 * mh + 1) continue;
        const float2 gj = *reinterpret_cast<const float2 *>(vec + 32 * kVecG + jj), rj = *reinterpret_cast<const float2 *>(vec + 32 * kVecRk + jj);
        float c0 = 0.f, c1 = 0.f;
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          const int i = i0 + g + 8 * x;
          const float gi = vec[32 * kVecG + i], rk = vec[32 * kVecRk + i], rq = a.scale * vec[32 * kVecRq + i];
          const float e0 = i >= jj ? __expf(gi - gj.x) * rj.x : 0.f, e1 = i > jj ? __expf(gi - gj.y) * rj.y : 0.f;
          const float x10 = rq * e0 * yu[u][2 * x], x11 = rq * e1 * yu[u][2 * x + 1];
          const float m0 = i > jj ? -rk * e0 * lu[u][2 * x] : 0.f, m1 = i > jj + 1 ? -rk * e1 * lu[u][2 * x + 1] : 0.f;
          const float t0 = x10 * qk[u][2 * x], t1 = x11 * qk[u][2 * x + 1], u0 = m0 * kk[u][2 * x], u1 = m1 * kk[u][2 * x + 1];
          c0 += fmaf(bt[x], u0, i > jj ? t0 : 0.f);
          c1 += fmaf(bt[x], u1, i > jj + 1 ? t1 : 0.f);
          if (jt == 2 * mh + x && c == g >> 1) {      // the diagonal's entry of row i
            red[32 * Cfg::kDiag + i] = g & 1 ? t1 : t0;
            red[32 * Cfg::kLv + i] = g & 1 ? ld[u][2 * x + 1] : ld[u][2 * x];
          }
          r1[x] += t0 + t1;
          r2[x] += u0 + u1;
          x1s[u][2 * x] = x10 + (MULTI && h ? x1s[u][2 * x] : 0.f);
          x1s[u][2 * x + 1] = x11 + (MULTI && h ? x1s[u][2 * x + 1] : 0.f);
          x2s[u][2 * x] = fmaf(bt[x], m0, MULTI && h ? x2s[u][2 * x] : 0.f);
          x2s[u][2 * x + 1] = fmaf(bt[x], m1, MULTI && h ? x2s[u][2 * x + 1] : 0.f);
        }
#pragma unroll
        for (int d = 4; d < 32; d *= 2) {
          c0 += __shfl_xor_sync(0xffffffffu, c0, d);
          c1 += __shfl_xor_sync(0xffffffffu, c1, d);
        }
        if (g == 0) *reinterpret_cast<float2 *>(red + 32 * (Cfg::kCol + mh) + jj) = make_float2(c0, c1);
      }
      if (mh == 0 && JT * kq + JT > 2 && g == 0)      // (columns that the upper half of the rows does not reach)
#pragma unroll
        for (int u = 0; u < JT; ++u)
          if (JT * kq + u >= 2) *reinterpret_cast<float2 *>(red + 32 * Cfg::kCol + 8 * (JT * kq + u) + 2 * c) = make_float2(0.f, 0.f);
      // a1, a2, a3; the products with the states scaled and put together
      float a1[2] = {}, a2[2] = {}, a3[2] = {};
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const int i = i0 + g + 8 * x;
        const float eq = vec[32 * kVecEq + i], be = -bt[x] * vec[32 * kVecEgk + i], ek = vec[32 * kVecEk + i];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          if (t >= tiles) continue;
          const float2 qv = unpack_bf16(__float_as_uint(lds32(qat + 8 * x * Cfg::kPK + 16 * t))), kv = unpack_bf16(__float_as_uint(lds32(kat + 8 * x * Cfg::kPK + 16 * t)));
          a1[x] = fmaf(qv.x, dq[t][2 * x], fmaf(qv.y, dq[t][2 * x + 1], a1[x]));
          a2[x] = fmaf(kv.x, dm[t][2 * x], fmaf(kv.y, dm[t][2 * x + 1], a2[x]));
          a3[x] = fmaf(kv.x, dp[t][2 * x], fmaf(kv.y, dp[t][2 * x + 1], a3[x]));
#pragma unroll
          for (int e = 2 * x; e < 2 * x + 2; ++e) {
            dqs[t][e] = fmaf(eq, dq[t][e], MULTI && h ? dqs[t][e] : 0.f);
            dks[t][e] = fmaf(be, dm[t][e], fmaf(ek, dp[t][e], MULTI && h ? dks[t][e] : 0.f));
          }
        }
#pragma unroll
        for (int d = 1; d < 4; d *= 2) {
          a1[x] += __shfl_xor_sync(0xffffffffu, a1[x], d);
          a2[x] += __shfl_xor_sync(0xffffffffu, a2[x], d);
          a3[x] += __shfl_xor_sync(0xffffffffu, a3[x], d);
          r1[x] += __shfl_xor_sync(0xffffffffu, r1[x], d);
          r2[x] += __shfl_xor_sync(0xffffffffu, r2[x], d);
        }
        red[32 * (Cfg::kA + KG * c + kq) + i] = c == 0 ? a1[x] : c == 1 ? a2[x] : c == 2 ? a3[x] : r1[x];      // (kRow1 follows a3)
        if (c == 0) red[32 * (Cfg::kRow2 + kq) + i] = r2[x];
      }
      if (warp == kIdle) {
        ss += ss1;
#pragma unroll
        for (int d = 16; d; d /= 2) ss += __shfl_xor_sync(0xffffffffu, ss, d);
        if (lane == 0) red[32 * Cfg::kSds] = ss;
      }
      if (!MULTI || h + 1 == a.hpc) {
#pragma unroll
        for (int u = 0; u < JT; ++u) {
          if (JT * kq + u > 2 * mh + 1) continue;
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            const uint32_t at = mat + 128 * (4 * (2 * mh + x) + JT * kq + u) + 4 * lane;
            sts32(at, __uint_as_float(pack_bf16(x1s[u][2 * x], x1s[u][2 * x + 1])));
            sts32(at + 2048, __uint_as_float(pack_bf16(x2s[u][2 * x], x2s[u][2 * x + 1])));
          }
        }
      }
      __syncthreads();
      if (warp == 0) {      // a token a lane
        auto sum = [&](int r) {
          const float *p = red + 32 * r + lane;
          float s = p[0];
#pragma unroll
          for (int x = 1; x < KG; ++x) s += p[32 * x];
          return s;
        };
        const float b = vec[32 * kVecBeta + lane];
        const float s1 = vec[32 * kVecEq + lane] * sum(Cfg::kA), s2 = vec[32 * kVecEgk + lane] * sum(Cfg::kA + KG), W = vec[32 * kVecEk + lane] * sum(Cfg::kA + 2 * KG);
        const float r1 = sum(Cfg::kRow1), r2 = sum(Cfg::kRow2), col = red[32 * Cfg::kCol + lane] + red[32 * Cfg::kCol + 32 + lane], diag = red[32 * Cfg::kDiag + lane];
        pqs = s1 + r1 + (MULTI && h ? pqs : 0.f);      // q . dq', k . dk'
        pks = fmaf(b, r2 - s2, W + col + diag) + (MULTI && h ? pks : 0.f);
        if (!MULTI || h + 1 == a.hpc) {
          const float rk = vec[32 * kVecRk + lane], rq = vec[32 * kVecRq + lane];
          red[32 * Cfg::kUq + lane] = a.qk_norm ? -rq * rq * pqs : 0.f;
          red[32 * Cfg::kUk + lane] = a.qk_norm ? -rk * rk * pks : 0.f;
        }
        float all = W, part = s1 + (r1 - diag) + b * (r2 - s2) - W - col;
#pragma unroll
        for (int d = 16; d; d /= 2) all += __shfl_xor_sync(0xffffffffu, all, d);
#pragma unroll
        for (int d = 1; d < 32; d *= 2) {
          const float t = __shfl_down_sync(0xffffffffu, part, d);
          if (lane + d < 32) part += t;
        }
        if (lane < o.have) {
          const size_t at = (size_t)(o.tok + lane) * a.N + n;
          const float dlog = fmaf(expf(vec[32 * kVecG + 31]), red[32 * Cfg::kSds], part + all);
          static_cast<__nv_bfloat16 *>(a.dgate)[at] = __float2bfloat16_rn(dlog * vec[32 * kVecDlog + lane]);
          static_cast<__nv_bfloat16 *>(a.dstep)[at] = __float2bfloat16_rn((red[32 * Cfg::kLv + lane] - s2 + r2) * (a.step_kind == M2RNN_STEP_LOGIT ? b * (1.f - b) : 1.f));
        }
      }
    }
#pragma unroll
    for (int kt = 0; kt < 2; ++kt) {
      // rows of this warp's tokens against tokens 16 kt (k-tile): lower parts, and transposed ones
      const bool lo = kt <= mh, up = kt >= mh;
      uint32_t x1[4], x2[4], t1[4], t2[4];
      if (lo) {
        const uint32_t at = mat + 16 * mrow + 128 * (4 * (2 * mh + mlo) + 2 * kt + mhi);
        ldmatrix_x4(at, x1);
        ldmatrix_x4(at + 2048, x2);
      }
      if (up) {
        const uint32_t at = mat + 16 * mrow + 128 * (4 * (2 * kt + mhi) + 2 * mh + mlo);
        ldmatrix_x4_t(at, t1);
        ldmatrix_x4_t(at + 2048, t2);
      }
#pragma unroll
      for (int t = 0; t < NT; t += 2) {
        if (t >= tiles) continue;
        const uint32_t at = (16 * kt + mrow + 8 * mlo) * Cfg::kPK + 2 * f0 + 16 * (t + (t + 1 < tiles ? mhi : 0));
        uint32_t kb[4], qb4[4];
        ldmatrix_x4_t(ksa + at, kb);
        if (up) ldmatrix_x4_t(qsa + at, qb4);
#pragma unroll
        for (int e = 0; e < 2; ++e)
          if (t + e < NT && t + e < tiles) {
            if (lo) {
              mma_add(dqs[t + e], x1, kb[2 * e], kb[2 * e + 1]);
              mma_add(dks[t + e], x2, kb[2 * e], kb[2 * e + 1]);
            }
            if (up) {
              mma_add(dks[t + e], t1, qb4[2 * e], qb4[2 * e + 1]);
              mma_add(dks[t + e], t2, kb[2 * e], kb[2 * e + 1]);
            }
          }
      }
    }
    __syncthreads();      // the factors are there; X1, X2, q and k are read
    if (BUFS == 1 && next.have) fetch(next, next.n0, 0, 0);
    // through the division by the lengths: to the shares, or to memory as they are (16 bytes of a row an instruction, two make a sector)
    auto emit = [&](const float (&x)[NT][4], uint32_t at, int factors, float *part, void *out, int heads, int head) {
      const size_t t = (size_t)(o.tok + i0 + g), step = (size_t)8 * (part ? a.shares : heads) * K;
      float *pp = part + (t * a.shares + o.run) * K + f0 + 2 * c;
      __nv_bfloat16 *po = static_cast<__nv_bfloat16 *>(out) + (t * heads + head) * K + f0 + 2 * c;
#pragma unroll
      for (int y = 0; y < 2; ++y) {
        const float f = red[32 * factors + i0 + g + 8 * y];
        if (i0 + g + 8 * y >= o.have) continue;
#pragma unroll
        for (int u = 0; u < NT; ++u) {
          if (u >= tiles) continue;
          const float2 was = unpack_bf16(__float_as_uint(lds32(at + 8 * y * Cfg::kPK + 16 * u)));
          const float v0 = fmaf(f, was.x, x[u][2 * y]), v1 = fmaf(f, was.y, x[u][2 * y + 1]);
          if (part) *reinterpret_cast<float2 *>(pp + y * step + 8 * u) = make_float2(v0, v1);
          else *reinterpret_cast<uint32_t *>(po + y * step + 8 * u) = pack_bf16(v0, v1);
        }
      }
    };
    emit(dqs, qat, Cfg::kUq, a.dq_part, a.dq, a.Nq, o.hq);
    emit(dks, kat, Cfg::kUk, a.dk_part, a.dk, a.Nk, o.hk);
    if (!next.have) break;
    o = next;
  }
}

template <int K, bool MULTI, int VS, int CTAS> cudaError_t launch_kmvc(const DeltaArgs &a, cudaStream_t s) {
  using Cfg = GradCfg<K>;
  constexpr int room = 227 * 1024 / CTAS - 1024, BUFS = MULTI || Cfg::kSlab + 2 * slab_bytes(K, VS) <= room ? 2 : 1;
  constexpr size_t smem = Cfg::kSlab + BUFS * (size_t)slab_bytes(K, VS);
  static_assert(smem <= room, "CTAs to an SM");
  const auto kernel = delta_grad_kernel<K, MULTI, VS, BUFS, CTAS>;
  const cudaError_t e = allow_smem(kernel, smem);
  if (e != cudaSuccess) return e;
  const unsigned jobs = (unsigned)(a.slots * (a.N / a.hpc)), most = CTAS * (unsigned)sm_count();
  return launch_early(kernel, dim3(jobs < most ? jobs : most), dim3(Cfg::kThreads), smem, s, a, jobs);
}
template <int K, bool MULTI, int VS> cudaError_t launch_kmv(const DeltaArgs &a, cudaStream_t s) {
  if constexpr (K > 64) return launch_kmvc<K, MULTI, VS, 2>(a, s);
  else if constexpr (!MULTI) return launch_kmvc<K, MULTI, VS, 3>(a, s);
  else return a.grad_ctas == 2 ? launch_kmvc<K, MULTI, VS, 2>(a, s) : launch_kmvc<K, MULTI, VS, 3>(a, s);
}
template <int K, bool MULTI> cudaError_t launch_km(const DeltaArgs &a, cudaStream_t s) {
  constexpr int VS = MULTI || K > 64 ? 32 : 64;
  if (a.V == 16) return launch_kmv<K, MULTI, 16>(a, s);
  if (a.V == 32 || VS == 32) return launch_kmv<K, MULTI, 32>(a, s);
  return launch_kmv<K, MULTI, VS>(a, s);
}
template <int K> cudaError_t launch_k(const DeltaArgs &a, cudaStream_t s) { return a.hpc > 1 ? launch_km<K, true>(a, s) : launch_km<K, false>(a, s); }

}  // namespace

// Heads of a job, of those that share q and k, and CTAs to an SM: what leaves an SM the least to do, a job counted as its heads and half a
// head for what it does once.  Above K = 64 registers and shared memory have room for two CTAs; up to there three fill an SM, but of several
// heads two do 6 % more (16 384 tokens, 84 heads of 64 x 16: 351 us against 371), unless the jobs come out as one round of three.
GradPlan delta_grad_plan(const m2rnn_delta_params *p, size_t slots) {
  int run = p->N / p->Nq, o = p->N / p->Nk;
  while (o) { const int t = run % o; run = o; o = t; }
  GradPlan best{1, 2};
  size_t least = ~(size_t)0;
  for (int d = run; d >= 1; --d)
    for (int ctas = 2; ctas <= 3; ++ctas) {
      if (run % d || (p->K > 64 ? ctas == 3 : d == 1 && ctas == 2)) continue;
      const size_t round = (size_t)ctas * sm_count(), cost = (slots * (p->N / d) + round - 1) / round * ctas * (2 * d + 1) * (d > 1 && ctas == 3 ? 17 : 16);
      if (cost + cost / 32 < least) { least = cost; best = GradPlan{d, ctas}; }      // (fewer heads only where that saves 3 %: more shares to add up)
    }
  return best;
}

cudaError_t launch_delta_grad(const DeltaArgs &a, cudaStream_t s) {
  switch (a.K) {
    case 16: return launch_k<16>(a, s);
    case 32: return launch_k<32>(a, s);
    case 48: return launch_k<48>(a, s);
    case 64: return launch_k<64>(a, s);
    case 80: return launch_k<80>(a, s);
    case 96: return launch_k<96>(a, s);
    case 112: return launch_k<112>(a, s);
    default: return launch_k<128>(a, s);
  }
}

}  // namespace m2rnn
