// Gated delta rule, bf16: gradients of q, k, the gate and the step, chunk by chunk, from what the chains kept
// (delta_chain.cu: S at a chunk's start, U; dS' at its end, L = dU through T^T).  With K^, Q^ the rows divided by
// their lengths, E_ij = e^(g_i - g_j), and dP_ij = dY_i . U_j (j <= i), N_ij = -L_i . U_j (j < i):
//     dQ^ = s (e^g dY S^T + (E dP) K^)
//     dK- = -e^g L S^T + (E N) K^                     its step b_i left out: k's part in what the update reads
//     dK+ = e^(g_last - g) U dS'^T + (b E N)^T K^ + s (E dP)^T Q^        k's part in what it writes
//     dK^ = b dK- + dK+        db_i = L_i . v_i + k^_i . dK-_i
// The decays' gradient sums what crosses token t's decay: what tokens from t on read of S, what tokens before t write
// into S', the pairs on either side of it, and S on its way to S':
//     R_i = q^_i . (s e^g S dY)_i - b_i k^_i . (e^g S L)_i        W_j = k^_j . (e^(g_last - g) dS' U)_j
//     G_ij = E_ij (s (q^_i . k^_j) dP_ij + b_i (k^_i . k^_j) N_ij)      (j < i)
//     d log a_t = e^g_last <S, dS'> + sum_{i >= t} R_i + sum_{j < t} W_j + sum_{j < t <= i} G_ij
// (With q . dQ^ - k . dK+ in place of R, W and G the pairs on one side of t would cancel only up to the roundings of
// the matrices to bf16: 2.5e-2 off where states decay within a few tokens.  Here the same fp32 value is added and taken away.)
// Four warps: 16 tokens x half of the K features each; the products over V in slabs of 64 columns.  A CTA takes a chunk
// of `hpc` heads that share q and k, one after the other, and adds up their dq and dk in registers.
#include "delta_common.cuh"

namespace m2rnn {
namespace {

constexpr int C = kDeltaChunk;

template <int K> struct GradCfg {
  static constexpr int kPK = 2 * K + 16;
  static constexpr int kQ = 0, kK = C * kPK, kMat = 2 * C * kPK;        // q, k rows; four 32 x 32 matrices as blocks
  static constexpr int kVec = kMat + 4 * 2048;                           // the record's vectors
  static constexpr int kRed = kVec + 1024;                               // float [8][32] sums of the two halves; [2][32] each of G's rows and columns; [32] L.v; [4] <S, dS'>
  static constexpr int kSlab = kRed + (10 * 32 + 4 * 32 + 32 + 16) * 4;        // dY, V rows, then U, L, S, dS' blocks of a slab
  static_assert(kSlab % 16 == 0, "");
};
__host__ __device__ constexpr int slab_bytes(int K, int VS) { return 2 * C * (2 * VS + 16) + 2 * 2 * C * VS + 2 * 2 * K * VS; }

// MULTI: several heads to a CTA
template <int K, bool MULTI>
__global__ void __launch_bounds__(128, 2) delta_grad_kernel(DeltaArgs a) {
  using Cfg = GradCfg<K>;
  constexpr int NT = K / 16;     // 8-feature tiles of a warp
  extern __shared__ __align__(128) unsigned char smem[];
  begin_dependent();
  const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = tid & 31, g = lane >> 2, c = lane & 3;
  const int mh = warp & 1, kh = warp >> 1, i0 = 16 * mh, f0 = kh * (K / 2);
  const int runs = a.N / a.hpc;
  const long long bc = blockIdx.x / runs;
  const int run = (int)(blockIdx.x % runs), n0 = run * a.hpc;
  const int b = (int)(bc / a.nch), ch = (int)(bc % a.nch);
  const DeltaSpan sp = delta_span<C>(a, b);
  if (ch >= sp.n) return;
  const long long tok = sp.tok0 + ch * C;
  const int have = min(C, sp.T - ch * C), V = a.V, VS = V < 64 ? V : 64, pv = 2 * VS + 16;
  const int hq = n0 / (a.N / a.Nq), hk = n0 / (a.N / a.Nk);
  const uint32_t base = smem_u32(smem), qsa = base + Cfg::kQ, ksa = base + Cfg::kK, mat = base + Cfg::kMat;
  const uint32_t ysa = base + Cfg::kSlab, vsa = ysa + C * pv, usa = vsa + C * pv, lsa = usa + 2 * C * VS, ssa = lsa + 2 * C * VS, dsa = ssa + 2 * K * VS;
  const float *vec = reinterpret_cast<const float *>(smem + Cfg::kVec);
  float *red = reinterpret_cast<float *>(smem + Cfg::kRed), *grow = red + 10 * 32, *gcol = grow + 64, *lv = gcol + 64, *sds = lv + 32;
  const uint32_t mrow = lane & 7, mlo = (lane >> 3) & 1, mhi = lane >> 4;

  {
    const __nv_bfloat16 *kg = static_cast<const __nv_bfloat16 *>(a.k) + tok * a.ks + (long long)hk * K;
    const __nv_bfloat16 *qg = static_cast<const __nv_bfloat16 *>(a.q) + tok * a.qs + (long long)hq * K;
    for (int x = tid; x < C * (K / 8); x += 128) {
      const int r = x / (K / 8), o = x % (K / 8);
      const bool ok = r < have;
      cp16_or_zero(ksa + r * Cfg::kPK + 16 * o, kg + (ok ? r * a.ks : 0) + 8 * o, ok);
      cp16_or_zero(qsa + r * Cfg::kPK + 16 * o, qg + (ok ? r * a.qs : 0) + 8 * o, ok);
    }
  }
  const uint32_t qat = qsa + (i0 + g) * Cfg::kPK + 2 * (f0 + 2 * c), kat = ksa + (i0 + g) * Cfg::kPK + 2 * (f0 + 2 * c);   // this thread's entries
  // results: to their shares, or to the places of q and k
  auto emit = [&](const float (&oq)[NT][4], const float (&ok)[NT][4]) {
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const int i = i0 + g + 8 * x;
        const size_t at = ((size_t)(tok + i) * a.shares + run) * K + f0 + 8 * t + 2 * c;
        if (!a.dq_part) sts32(qat + 8 * x * Cfg::kPK + 16 * t, __uint_as_float(pack_bf16(oq[t][2 * x], oq[t][2 * x + 1])));
        else if (i < have) *reinterpret_cast<float2 *>(a.dq_part + at) = make_float2(oq[t][2 * x], oq[t][2 * x + 1]);
        if (!a.dk_part) sts32(kat + 8 * x * Cfg::kPK + 16 * t, __uint_as_float(pack_bf16(ok[t][2 * x], ok[t][2 * x + 1])));
        else if (i < have) *reinterpret_cast<float2 *>(a.dk_part + at) = make_float2(ok[t][2 * x], ok[t][2 * x + 1]);
      }
  };
  float dqs[MULTI ? NT : 1][4], dks[MULTI ? NT : 1][4];
  if constexpr (MULTI)
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) dqs[t][r] = dks[t][r] = 0.f;

  for (int h = 0; h < a.hpc; ++h) {
    const int n = n0 + h;
    const size_t slot = (size_t)(sp.slot0 + ch) * a.N + n;
    const char *rec = a.rec + slot * kRecBytes;
    if (tid < 64) cp16(base + Cfg::kVec + 16 * tid, rec + kRecVec + 16 * tid);
    float dq[NT][4], dm[NT][4], dp[NT][4];      // dY S^T, L S^T, U dS'^T; then dQ^, dK-, dK+
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) dq[t][r] = dm[t][r] = dp[t][r] = 0.f;
    float yu[2][4] = {}, lu[2][4] = {}, ld[2][4] = {};    // tiles (16 mh, 16 kh): dY U^T, L U^T, L V^T
    float ss = 0.f;                                        // this thread's part of <S, dS'>
    for (int vb = 0; vb < V; vb += VS) {
      {
        const __nv_bfloat16 *yg = static_cast<const __nv_bfloat16 *>(a.dy) + ((size_t)tok * a.N + n) * V + vb;
        const __nv_bfloat16 *vg = static_cast<const __nv_bfloat16 *>(a.v) + tok * a.vs + (long long)n * V + vb;
        const long long ys = (long long)a.N * V;
        const int per = VS / 8;
        for (int x = tid; x < C * per; x += 128) {
          const int r = x / per, o = x % per;
          const bool ok = r < have;
          cp16_or_zero(ysa + r * pv + 16 * o, yg + (ok ? r * ys : 0) + 8 * o, ok);
          cp16_or_zero(vsa + r * pv + 16 * o, vg + (ok ? r * a.vs : 0) + 8 * o, ok);
        }
        const char *ug = a.upd + slot * (2 * C * V) + 2 * C * vb, *lg = a.lam + slot * (2 * C * V) + 2 * C * vb;
        for (int x = tid; x < C * VS / 8; x += 128) {
          cp16(usa + 16 * x, ug + 16 * x);
          cp16(lsa + 16 * x, lg + 16 * x);
        }
        const char *sg = a.states + slot * (2 * K * V) + 2 * K * vb, *dg = a.dstates + slot * (2 * K * V) + 2 * K * vb;
        for (int x = tid; x < K * VS / 8; x += 128) {
          cp16(ssa + 16 * x, sg + 16 * x);
          cp16(dsa + 16 * x, dg + 16 * x);
        }
        cp_wait_all();
        __syncthreads();
      }
      // <S, dS'>
      for (int x = tid; x < K * VS / 8; x += 128) {
        const uint4 p = *reinterpret_cast<const uint4 *>(smem + (ssa - base) + 16 * x), d = *reinterpret_cast<const uint4 *>(smem + (dsa - base) + 16 * x);
        ss = fma_bf16<0, 0>(p.x, d.x, fma_bf16<1, 1>(p.x, d.x, ss));
        ss = fma_bf16<0, 0>(p.y, d.y, fma_bf16<1, 1>(p.y, d.y, ss));
        ss = fma_bf16<0, 0>(p.z, d.z, fma_bf16<1, 1>(p.z, d.z, ss));
        ss = fma_bf16<0, 0>(p.w, d.w, fma_bf16<1, 1>(p.w, d.w, ss));
      }
      // products over the slab's columns
      for (int kt = 0; kt < VS / 16; ++kt) {
        uint32_t ya[4], la[4], ua[4];     // A operands: 16 tokens x 16 columns
        ldmatrix_x4(ysa + (i0 + mrow + 8 * mlo) * pv + 32 * kt + 16 * mhi, ya);
        // blocks [column tile][token tile]; transposed: rows are tokens
        const uint32_t ba = 16 * mrow + 128 * (4 * (2 * kt + mhi) + 2 * mh + mlo);
        ldmatrix_x4_t(lsa + ba, la);
        ldmatrix_x4_t(usa + ba, ua);
        if (kh <= mh) {
          uint32_t ub[4], wb[4];          // B operands: 16 columns x 16 tokens from 16 kh
          ldmatrix_x4_t(usa + 16 * mrow + 128 * (4 * (2 * kt + mlo) + 2 * kh + mhi), ub);
          mma_bf16_16816(yu[0], ya, ub[0], ub[1]);
          mma_bf16_16816(yu[1], ya, ub[2], ub[3]);
          mma_bf16_16816(lu[0], la, ub[0], ub[1]);
          mma_bf16_16816(lu[1], la, ub[2], ub[3]);
          if (kh == mh) {
            ldmatrix_x4(vsa + (i0 + mrow + 8 * mhi) * pv + 32 * kt + 16 * mlo, wb);
            mma_bf16_16816(ld[0], la, wb[0], wb[1]);
            mma_bf16_16816(ld[1], la, wb[2], wb[3]);
          }
        }
#pragma unroll
        for (int t = 0; t < NT; t += 2) {
          // B operands: 16 columns x 16 features (the last pair of an odd number of tiles: the second is not used)
          const uint32_t fb = f0 / 8 + t + (t + 1 < NT ? mhi : 0);
          const uint32_t at = 16 * mrow + 128 * ((2 * kt + mlo) * (K / 8) + fb);
          uint32_t sb[4], db[4];
          ldmatrix_x4_t(ssa + at, sb);
          ldmatrix_x4_t(dsa + at, db);
          mma_bf16_16816(dq[t], ya, sb[0], sb[1]);
          mma_bf16_16816(dm[t], la, sb[0], sb[1]);
          mma_bf16_16816(dp[t], ua, db[0], db[1]);
          if (t + 1 < NT) {
            mma_bf16_16816(dq[t + 1], ya, sb[2], sb[3]);
            mma_bf16_16816(dm[t + 1], la, sb[2], sb[3]);
            mma_bf16_16816(dp[t + 1], ua, db[2], db[3]);
          }
        }
      }
      if (vb + VS < V) __syncthreads();     // (the slab's place is the next one's)
    }
    // rows i of this thread: i0 + g, i0 + g + 8
    const float *vg = vec + 32 * kVecG, *vb_ = vec + 32 * kVecBeta, *vrk = vec + 32 * kVecRk, *vrq = vec + 32 * kVecRq;
    const float glast = vg[31];
    float eg[2], ek[2], bt[2], rk[2], rq[2], gi[2];
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      const int i = i0 + g + 8 * x;
      gi[x] = vg[i]; bt[x] = vb_[i]; rk[x] = vrk[i]; rq[x] = vrq[i];
      eg[x] = expf(gi[x]);
      ek[x] = expf(glast - gi[x]);
    }
    // q k^T and k k^T, tiles (16 mh, 16 kh)
    float qk[2][4] = {}, kk[2][4] = {};
    if (kh <= mh) {
#pragma unroll
      for (int kt = 0; kt < K / 16; ++kt) {
        uint32_t qa[4], ka[4], kb[4];
        const uint32_t ra = (i0 + (lane & 15)) * Cfg::kPK + 32 * kt + 16 * mhi;
        ldmatrix_x4(qsa + ra, qa);
        ldmatrix_x4(ksa + ra, ka);
        ldmatrix_x4(ksa + (16 * kh + mrow + 8 * mhi) * Cfg::kPK + 32 * kt + 16 * mlo, kb);
        mma_bf16_16816(qk[0], qa, kb[0], kb[1]);
        mma_bf16_16816(qk[1], qa, kb[2], kb[3]);
        mma_bf16_16816(kk[0], ka, kb[0], kb[1]);
        mma_bf16_16816(kk[1], ka, kb[2], kb[3]);
      }
    }
    float gr[2] = {}, gc[2][2] = {};      // sums of G over this thread's entries of a row, of a column
    // the four 32 x 32 matrices: 0: s E dP r_k,j   1: s E dP r_q,i   2: E N r_k,j   3: b_i E N r_k,i
    if (kh <= mh) {
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          const int i = i0 + g + 8 * x, j = 16 * kh + 8 * t + 2 * c;
          const float e0 = i >= j ? __expf(gi[x] - vg[j]) : 0.f, e1 = i >= j + 1 ? __expf(gi[x] - vg[j + 1]) : 0.f;
          const float p0 = a.scale * e0 * yu[t][2 * x], p1 = a.scale * e1 * yu[t][2 * x + 1];
          const float m0 = i > j ? -e0 * lu[t][2 * x] : 0.f, m1 = i > j + 1 ? -e1 * lu[t][2 * x + 1] : 0.f;
          const uint32_t at = mat + 128 * (4 * (2 * mh + x) + 2 * kh + t) + 4 * lane;
          const float r0 = vrk[j], r1 = vrk[j + 1];
          const uint32_t w[4] = {pack_bf16(p0 * r0, p1 * r1), pack_bf16(p0 * rq[x], p1 * rq[x]), pack_bf16(m0 * r0, m1 * r1),
                                 pack_bf16(m0 * bt[x] * rk[x], m1 * bt[x] * rk[x])};
#pragma unroll
          for (int m = 0; m < 4; ++m) sts32(at + 2048 * m, __uint_as_float(w[m]));
          const float b = bt[x] * rk[x];
          const float t0 = i > j ? r0 * fmaf(p0 * rq[x], qk[t][2 * x], m0 * b * kk[t][2 * x]) : 0.f;
          const float t1 = i > j + 1 ? r1 * fmaf(p1 * rq[x], qk[t][2 * x + 1], m1 * b * kk[t][2 * x + 1]) : 0.f;
          gr[x] += t0 + t1;
          gc[t][0] += t0;
          gc[t][1] += t1;
        }
      if (kh == mh)      // L_i . v_i: the diagonal
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int r = 0; r < 4; ++r)
            if (g + 8 * (r >> 1) == 8 * t + 2 * c + (r & 1)) lv[i0 + g + 8 * (r >> 1)] = ld[t][r];
    }
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      gr[x] += __shfl_xor_sync(0xffffffffu, gr[x], 1);
      gr[x] += __shfl_xor_sync(0xffffffffu, gr[x], 2);
      if (c == 0) grow[32 * kh + i0 + g + 8 * x] = gr[x];
    }
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
#pragma unroll
        for (int d = 4; d < 32; d *= 2) gc[t][e] += __shfl_xor_sync(0xffffffffu, gc[t][e], d);
        if (g == 0) gcol[32 * mh + 16 * kh + 8 * t + 2 * c + e] = gc[t][e];
      }
    // the parts from S and dS' scaled; W and R
    float d0[2] = {}, dr[2] = {};
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const float sq = a.scale * eg[x];
        dq[t][2 * x] *= sq; dq[t][2 * x + 1] *= sq;
        dm[t][2 * x] *= -eg[x]; dm[t][2 * x + 1] *= -eg[x];
        dp[t][2 * x] *= ek[x]; dp[t][2 * x + 1] *= ek[x];
        const float2 kv = unpack_bf16(__float_as_uint(lds32(kat + 8 * x * Cfg::kPK + 16 * t))), qv = unpack_bf16(__float_as_uint(lds32(qat + 8 * x * Cfg::kPK + 16 * t)));
        const float b = bt[x] * rk[x];
        d0[x] = fmaf(kv.x, dp[t][2 * x], fmaf(kv.y, dp[t][2 * x + 1], d0[x]));
        dr[x] = fmaf(rq[x], fmaf(qv.x, dq[t][2 * x], qv.y * dq[t][2 * x + 1]), fmaf(b, fmaf(kv.x, dm[t][2 * x], kv.y * dm[t][2 * x + 1]), dr[x]));
      }
    __syncthreads();
#pragma unroll
    for (int kt = 0; kt < 2; ++kt) {
      // rows of this warp's tokens against tokens 16 kt (k-tile): lower for dQ^, dK-, its transpose for dK+
      const bool lo = kt <= mh, up = kt >= mh;
      uint32_t m0[4], m1[4], m2[4], m3[4];
      if (lo) {
        const uint32_t at = mat + 16 * mrow + 128 * (4 * (2 * mh + mlo) + 2 * kt + mhi);
        ldmatrix_x4(at, m0);
        ldmatrix_x4(at + 2 * 2048, m2);
      }
      if (up) {
        const uint32_t at = mat + 16 * mrow + 128 * (4 * (2 * kt + mhi) + 2 * mh + mlo);
        ldmatrix_x4_t(at + 2048, m1);
        ldmatrix_x4_t(at + 3 * 2048, m3);
      }
#pragma unroll
      for (int t = 0; t < NT; t += 2) {
        const uint32_t at = (16 * kt + mrow + 8 * mlo) * Cfg::kPK + 2 * f0 + 16 * (t + (t + 1 < NT ? mhi : 0));
        uint32_t kb[4], qb[4];
        ldmatrix_x4_t(ksa + at, kb);
        if (up) ldmatrix_x4_t(qsa + at, qb);
#pragma unroll
        for (int e = 0; e < 2; ++e)
          if (t + e < NT) {
            if (lo) {
              mma_bf16_16816(dq[t + e], m0, kb[2 * e], kb[2 * e + 1]);
              mma_bf16_16816(dm[t + e], m2, kb[2 * e], kb[2 * e + 1]);
            }
            if (up) {
              mma_bf16_16816(dp[t + e], m1, qb[2 * e], qb[2 * e + 1]);
              mma_bf16_16816(dp[t + e], m3, kb[2 * e], kb[2 * e + 1]);
            }
          }
      }
    }
    // sums over the features: q . dQ^, k . dK-, k . dK+ and the two above, then over the two halves of the features
    float d1[2] = {}, d2[2] = {}, d3[2] = {};
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const float2 qv = unpack_bf16(__float_as_uint(lds32(qat + 8 * x * Cfg::kPK + 16 * t))), kv = unpack_bf16(__float_as_uint(lds32(kat + 8 * x * Cfg::kPK + 16 * t)));
        d1[x] = fmaf(qv.x, dq[t][2 * x], fmaf(qv.y, dq[t][2 * x + 1], d1[x]));
        d2[x] = fmaf(kv.x, dm[t][2 * x], fmaf(kv.y, dm[t][2 * x + 1], d2[x]));
        d3[x] = fmaf(kv.x, dp[t][2 * x], fmaf(kv.y, dp[t][2 * x + 1], d3[x]));
      }
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      float *v5[5] = {&d0[x], &d1[x], &d2[x], &d3[x], &dr[x]};
#pragma unroll
      for (int y = 0; y < 5; ++y) {
        float &v = *v5[y];
        v += __shfl_xor_sync(0xffffffffu, v, 1);
        v += __shfl_xor_sync(0xffffffffu, v, 2);
        v *= y == 4 ? 1.f : y == 1 ? rq[x] : rk[x];
        if (c == 0) red[(2 * y + kh) * 32 + i0 + g + 8 * x] = v;
      }
    }
#pragma unroll
    for (int d = 16; d; d /= 2) ss += __shfl_xor_sync(0xffffffffu, ss, d);
    if (lane == 0) sds[warp] = ss;
    __syncthreads();
    if (warp == 0) {
      const float w = red[lane] + red[32 + lane], e2 = red[128 + lane] + red[160 + lane], r = red[256 + lane] + red[288 + lane];
      float all = w, part = r + grow[lane] + grow[32 + lane] - w - gcol[lane] - gcol[32 + lane];
#pragma unroll
      for (int d = 16; d; d /= 2) all += __shfl_xor_sync(0xffffffffu, all, d);
#pragma unroll
      for (int d = 1; d < 32; d *= 2) {
        const float o = __shfl_down_sync(0xffffffffu, part, d);
        if (lane + d < 32) part += o;
      }
      if (lane < have) {
        const size_t at = (size_t)(tok + lane) * a.N + n;
        const float dlog = part + all + expf(glast) * (sds[0] + sds[1] + sds[2] + sds[3]);
        float ds;
        (void)delta_step_of(a.step_kind, __bfloat162float(static_cast<const __nv_bfloat16 *>(a.step)[at]), ds);
        static_cast<__nv_bfloat16 *>(a.dgate)[at] = __float2bfloat16_rn(dlog * vec[32 * kVecDlog + lane]);
        static_cast<__nv_bfloat16 *>(a.dstep)[at] = __float2bfloat16_rn((lv[lane] + e2) * ds);
      }
    }
    // through the division by the lengths: dx = r (dx^ - x^ (x^ . dx^))
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      const int i = i0 + g + 8 * x;
      float pq = 0.f, pk = 0.f;
      if (a.qk_norm) {
        pq = red[64 + i] + red[96 + i];
        pk = bt[x] * (red[128 + i] + red[160 + i]) + red[192 + i] + red[224 + i];
      }
      const float uq = -pq * rq[x] * rq[x], uk = -pk * rk[x] * rk[x];
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        const float2 qv = unpack_bf16(__float_as_uint(lds32(qat + 8 * x * Cfg::kPK + 16 * t))), kv = unpack_bf16(__float_as_uint(lds32(kat + 8 * x * Cfg::kPK + 16 * t)));
        const float q0 = fmaf(uq, qv.x, rq[x] * dq[t][2 * x]), q1 = fmaf(uq, qv.y, rq[x] * dq[t][2 * x + 1]);
        const float k0 = fmaf(uk, kv.x, rk[x] * fmaf(bt[x], dm[t][2 * x], dp[t][2 * x])), k1 = fmaf(uk, kv.y, rk[x] * fmaf(bt[x], dm[t][2 * x + 1], dp[t][2 * x + 1]));
        if constexpr (MULTI) {
          dqs[t][2 * x] += q0; dqs[t][2 * x + 1] += q1;
          dks[t][2 * x] += k0; dks[t][2 * x + 1] += k1;
        } else {
          dq[t][2 * x] = q0; dq[t][2 * x + 1] = q1;
          dm[t][2 * x] = k0; dm[t][2 * x + 1] = k1;
        }
      }
    }
    __syncthreads();      // the vectors, matrices and sums are read, and (at the last head) q and k
    if constexpr (!MULTI) emit(dq, dm);
  }
  if constexpr (MULTI) emit(dqs, dks);
  __syncthreads();
  for (int x = tid; x < have * (K / 8); x += 128) {
    const int r = x / (K / 8), o = x % (K / 8);
    if (!a.dq_part) *reinterpret_cast<float4 *>(static_cast<__nv_bfloat16 *>(a.dq) + ((size_t)(tok + r) * a.Nq + hq) * K + 8 * o) = lds128(qsa + r * Cfg::kPK + 16 * o);
    if (!a.dk_part) *reinterpret_cast<float4 *>(static_cast<__nv_bfloat16 *>(a.dk) + ((size_t)(tok + r) * a.Nk + hk) * K + 8 * o) = lds128(ksa + r * Cfg::kPK + 16 * o);
  }
}

template <int K, bool MULTI> cudaError_t launch_km(const DeltaArgs &a, cudaStream_t s) {
  const size_t smem = GradCfg<K>::kSlab + slab_bytes(K, a.V < 64 ? a.V : 64);
  const cudaError_t e = allow_smem(delta_grad_kernel<K, MULTI>, smem);
  if (e != cudaSuccess) return e;
  return launch_early(delta_grad_kernel<K, MULTI>, dim3((unsigned)((long long)a.B * a.nch * (a.N / a.hpc))), dim3(128), smem, s, a);
}
template <int K> cudaError_t launch_k(const DeltaArgs &a, cudaStream_t s) { return a.hpc > 1 ? launch_km<K, true>(a, s) : launch_km<K, false>(a, s); }

}  // namespace

// Heads of a CTA: as many of those that share q and k as leave four CTAs for every SM
int delta_grad_heads(const m2rnn_delta_params *p, size_t slots) {
  int run = p->N / p->Nq, o = p->N / p->Nk;
  while (o) { const int t = run % o; run = o; o = t; }
  for (int d = run; d > 1; --d)
    if (run % d == 0 && slots * (p->N / d) >= (size_t)4 * sm_count()) return d;
  return 1;
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
