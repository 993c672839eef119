// Gated delta rule, bf16: what does not depend on the state, chunk by chunk (see delta_chain.cu for the rule in chunks).
//
// For a chunk of 32 tokens of one head, with g the running sum of log a, r_k, r_q the reciprocal lengths:
//     M_ij = b_i e^(g_i - g_j) r_k,i r_k,j (k_i . k_j)   (j < i)        T = (I + M)^-1
//     P_ij = s   e^(g_i - g_j) r_q,i r_k,j (q_i . k_j)   (j <= i)
// Differences g_i - g_j are formed before the exponential: no e^-g that could overflow.
//
// A warp does a chunk for all heads that share its q and k: the two products of 32 x 32 are taken once (mma.sync, fp32
// accumulators that stay in registers), then for each head the gates, M, its inverse and P.  q and k go from memory
// straight into operands: a lane of an operand's row takes eight neighbouring features (16 bytes) for four k slots; which
// slot a feature has does not matter as long as both operands agree, and a row's words are the same as row of A
// and as column of B.  T is inverted in fp32:
// the two 16 x 16 blocks on the diagonal by forward substitution, a column a lane (a series of powers of M would
// cancel digits where keys point the same way), then T_21 = -(T_22 M_21) T_11 with tf32 operands (2^-12 of each).  T goes out as bf16
// and what that leaves.
// (65 536 tokens of 32 heads, K = 128, 1.45 GB: 270 us, 5.4 TB/s; a form with q and k through shared memory, the lengths by FMA and T's
// last block too took 361.)
#include "delta_common.cuh"

namespace m2rnn {
namespace {

constexpr int kWarps = 4, kPM = 36, kPT = 20;   // pitches (floats) of M and of the diagonal blocks of T
constexpr int kTHalf = 16 * kPT + 16;           // the second block, half the banks on
constexpr int kWarpFloats = 32 * kPM + 2 * kTHalf;

__device__ __forceinline__ uint32_t tf32(float x) {
  uint32_t r;
  asm("cvt.rna.tf32.f32 %0, %1;" : "=r"(r) : "f"(x));
  return r;
}
__device__ __forceinline__ void mma_tf32(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k8.row.col.f32.tf32.tf32.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};\n"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

template <int K, bool PACKED>
__global__ void __launch_bounds__(32 * kWarps, 4) delta_prep_kernel(DeltaArgs a, int run) {
  __shared__ __align__(16) float sm[kWarps][kWarpFloats];
  begin_dependent();
  const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31, g = lane >> 2, c = lane & 3;
  const unsigned runs = (unsigned)(a.N / run), job = blockIdx.x * kWarps + warp, slot = job / runs;
  if (slot >= a.slots) return;
  const int n0 = (int)(job - slot * runs) * run, b = delta_entry<kDeltaChunk, PACKED>(a, slot);
  const DeltaSpan sp = delta_span<kDeltaChunk>(a, b);
  const int ch = PACKED ? (int)(slot - sp.slot0) : (int)(slot - (unsigned)b * a.nch);
  if ((unsigned)ch >= (unsigned)sp.n) return;      // (of a packed batch: a slot that is no sequence's)
  const long long tok = sp.tok0 + ch * kDeltaChunk;
  const int have = min(kDeltaChunk, sp.T - ch * kDeltaChunk);
  const char *kg = static_cast<const char *>(a.k) + 2 * ((tok + g) * a.ks + (unsigned)n0 / (unsigned)a.per_k * K);
  const char *qg = static_cast<const char *>(a.q) + 2 * ((tok + g) * a.qs + (unsigned)n0 / (unsigned)a.per_q * K);
  const long long k8 = 16 * a.ks, q8 = 16 * a.qs;      // bytes to a row eight tokens on

  // a head's gate and step entries (this lane's token's), asked for a head ahead
  float gate_in = 0.f, step_in = 0.f, alpha = 1.f, beta = 0.f;
  const bool mine = lane < have, psi = a.gate_kind == M2RNN_GATE_PSI;
  auto gates = [&](int n) {
    if (!mine) return;
    const size_t at = (size_t)(tok + lane) * a.N + n;
    gate_in = __bfloat162float(static_cast<const __nv_bfloat16 *>(a.gate)[at]);
    step_in = __bfloat162float(static_cast<const __nv_bfloat16 *>(a.step)[at]);
    if (psi) { alpha = a.alpha[n]; beta = a.beta[n]; }
  };
  gates(n0);
  // the rows' 64-byte parts on their way to the L2, one a lane, while the first is waited for
  if (64 * c < 2 * K && K > 32)
#pragma unroll
    for (int x = 0; x < 4; ++x)
      if (8 * x + g < have) {
        asm volatile("prefetch.global.L2 [%0];" ::"l"(kg + x * k8 + 64 * c));
        asm volatile("prefetch.global.L2 [%0];" ::"l"(qg + x * q8 + 64 * c));
      }
  // k k^T and q k^T, tiles (mt, nt) of 16 x 8 on and below the diagonal: mt = 0: nt 0, 1; mt = 1: nt 0 .. 3; of q q^T
  // those on the diagonal
  float kk[6][4] = {}, qk[6][4] = {}, qq[4][4] = {};
  auto half = [&](const uint32_t (&k0)[4], const uint32_t (&k1)[4], const uint32_t (&q0)[4], const uint32_t (&q1)[4]) {      // 16 features: two words of each row
    const uint32_t A0[4] = {k0[0], k0[1], k1[0], k1[1]}, A1[4] = {k0[2], k0[3], k1[2], k1[3]}, Q0[4] = {q0[0], q0[1], q1[0], q1[1]}, Q1[4] = {q0[2], q0[3], q1[2], q1[3]};
#pragma unroll
    for (int nt = 0; nt < 2; ++nt) { mma_add(kk[nt], A0, k0[nt], k1[nt]); mma_add(qk[nt], Q0, k0[nt], k1[nt]); mma_add(qq[nt], Q0, q0[nt], q1[nt]); mma_add(qq[2 + nt], Q1, q0[2 + nt], q1[2 + nt]); }
#pragma unroll
    for (int nt = 0; nt < 4; ++nt) { mma_add(kk[2 + nt], A1, k0[nt], k1[nt]); mma_add(qk[2 + nt], Q1, k0[nt], k1[nt]); }
  };
#pragma unroll
  for (int f = 0; f + 32 <= K; f += 32) {
    uint4 kx[4], qx[4];
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      kx[x] = qx[x] = make_uint4(0u, 0u, 0u, 0u);
      if (8 * x + g < have) {
        kx[x] = *reinterpret_cast<const uint4 *>(kg + x * k8 + 2 * f + 16 * c);
        qx[x] = *reinterpret_cast<const uint4 *>(qg + x * q8 + 2 * f + 16 * c);
      }
    }
    half({kx[0].x, kx[1].x, kx[2].x, kx[3].x}, {kx[0].y, kx[1].y, kx[2].y, kx[3].y}, {qx[0].x, qx[1].x, qx[2].x, qx[3].x}, {qx[0].y, qx[1].y, qx[2].y, qx[3].y});
    half({kx[0].z, kx[1].z, kx[2].z, kx[3].z}, {kx[0].w, kx[1].w, kx[2].w, kx[3].w}, {qx[0].z, qx[1].z, qx[2].z, qx[3].z}, {qx[0].w, qx[1].w, qx[2].w, qx[3].w});
  }
  if constexpr (K % 32) {
    uint2 kx[4], qx[4];
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      kx[x] = qx[x] = make_uint2(0u, 0u);
      if (8 * x + g < have) {
        kx[x] = *reinterpret_cast<const uint2 *>(kg + x * k8 + 2 * (K - 16) + 8 * c);
        qx[x] = *reinterpret_cast<const uint2 *>(qg + x * q8 + 2 * (K - 16) + 8 * c);
      }
    }
    half({kx[0].x, kx[1].x, kx[2].x, kx[3].x}, {kx[0].y, kx[1].y, kx[2].y, kx[3].y}, {qx[0].x, qx[1].x, qx[2].x, qx[3].x}, {qx[0].y, qx[1].y, qx[2].y, qx[3].y});
  }
  // reciprocal lengths: of rows 8 x + g, of columns 8 x + 2c, + 1, and of this lane's token
  float rki[4], rqi[4], rkj[4][2], rk = 1.f, rq = 1.f;
#pragma unroll
  for (int x = 0; x < 4; ++x) {
    rki[x] = rqi[x] = 1.f;
    if (a.qk_norm) {      // entry (g, g) of the diagonal's tile x is lane (g, g / 2)'s
      const int tile = x < 2 ? x : 2 + x, r = 2 * (x & 1);
      const float sk = __shfl_sync(0xffffffffu, g & 1 ? kk[tile][r + 1] : kk[tile][r], 4 * g + (g >> 1));
      const float sq = __shfl_sync(0xffffffffu, g & 1 ? qq[x][r + 1] : qq[x][r], 4 * g + (g >> 1));
      const bool row = 8 * x + g < have;      // (rows behind the last token: eps may be 0)
      rki[x] = rsqrtf(row ? sk + a.eps : 1.f);
      rqi[x] = rsqrtf(row ? sq + a.eps : 1.f);
    }
    rkj[x][0] = __shfl_sync(0xffffffffu, rki[x], 8 * c);
    rkj[x][1] = __shfl_sync(0xffffffffu, rki[x], 8 * c + 4);
    const float tk = __shfl_sync(0xffffffffu, rki[x], 4 * (lane & 7)), tq = __shfl_sync(0xffffffffu, rqi[x], 4 * (lane & 7));
    if (lane >> 3 == x) { rk = tk; rq = tq; }
    rqi[x] *= a.scale;
  }
  float *M = sm[warp], *Td = M + 32 * kPM, *T22 = Td + kTHalf;
  const uint32_t Msa = smem_u32(M);

  for (int n = n0; n < n0 + run; ++n) {
    float la = 0.f, bt = 0.f, dlog = 0.f;
    if (mine) {
      float unused;
      la = delta_log_decay(a.gate_kind, gate_in, alpha, beta, dlog);
      bt = delta_step_of(a.step_kind, step_in, unused);
    }
    if (n + 1 < n0 + run) gates(n + 1);
    float gs = la;
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
      const float o = __shfl_up_sync(0xffffffffu, gs, d);
      if (lane >= d) gs += o;
    }
    const float glast = __shfl_sync(0xffffffffu, gs, 31);
    char *rec = a.rec + ((size_t)(sp.slot0 + ch) * a.N + n) * kRecBytes;
    {
      float *vec = reinterpret_cast<float *>(rec + kRecVec) + lane;
      const float eg = expf(gs);
      vec[32 * kVecEgk] = eg * rk;
      vec[32 * kVecEq] = a.scale * eg * rq;
      vec[32 * kVecEk] = expf(glast - gs) * rk;
      vec[32 * kVecBeta] = bt;
      vec[32 * kVecG] = gs;
      vec[32 * kVecRk] = rk;
      vec[32 * kVecRq] = rq;
      vec[32 * kVecDlog] = dlog;
    }
    // M to shared memory, P straight out as blocks
    float gi[4], bi[4];
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      gi[x] = __shfl_sync(0xffffffffu, gs, g + 8 * x);
      bi[x] = __shfl_sync(0xffffffffu, bt, g + 8 * x) * rki[x];
    }
    uint32_t *Pg = reinterpret_cast<uint32_t *>(rec + kRecP) + lane;
    float odd = 0.f;      // NaN where M_21 has what is not finite
#pragma unroll
    for (int nt = 0; nt < 4; ++nt) {
      const float g0 = __shfl_sync(0xffffffffu, gs, 8 * nt + 2 * c), g1 = __shfl_sync(0xffffffffu, gs, 8 * nt + 2 * c + 1);
      const int j = 8 * nt + 2 * c;
#pragma unroll
      for (int mt = nt < 2 ? 0 : 1; mt < 2; ++mt) {
        const int tile = mt ? 2 + nt : nt;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int x = 2 * mt + h, i = g + 8 * x;      // (8 x 8 blocks below the diagonal are whole, those above it zeros)
          uint32_t p = 0u;
          if (x >= nt) {
            const float e0 = __expf(gi[x] - g0) * rkj[nt][0], e1 = __expf(gi[x] - g1) * rkj[nt][1];
            const float m0 = x > nt || i > j ? bi[x] * e0 * kk[tile][2 * h] : 0.f, m1 = x > nt || i > j + 1 ? bi[x] * e1 * kk[tile][2 * h + 1] : 0.f;
            sts64(Msa + 4u * (i * kPM + j), make_float2(m0, m1));
            if (x > 1 && nt < 2) odd = fmaf(0.f, m0, fmaf(0.f, m1, odd));
            p = pack_bf16(x > nt || i >= j ? rqi[x] * e0 * qk[tile][2 * h] : 0.f, x > nt || i > j ? rqi[x] * e1 * qk[tile][2 * h + 1] : 0.f);
          }
          Pg[(4 * x + nt) * 32] = p;
        }
      }
    }
    __syncwarp();
    // the diagonal blocks: lane (half, j) has column j of block `half`
    {
      const int half = lane >> 4, j = lane & 15;
      float t[16];
      const float *Mb = M + half * (16 * kPM + 16);
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        float s0 = i == j ? 1.f : 0.f, s1 = 0.f;
#pragma unroll
        for (int m4 = 0; m4 < i; m4 += 4) {
          const float4 w = *reinterpret_cast<const float4 *>(Mb + i * kPM + m4);
          if (m4 + 0 < i) s0 = fmaf(-w.x, t[m4 + 0], s0);
          if (m4 + 1 < i) s1 = fmaf(-w.y, t[m4 + 1], s1);
          if (m4 + 2 < i) s0 = fmaf(-w.z, t[m4 + 2], s0);
          if (m4 + 3 < i) s1 = fmaf(-w.w, t[m4 + 3], s1);
        }
        t[i] = s0 + s1;
        Td[half * kTHalf + i * kPT + j] = t[i];
      }
    }
    __syncwarp();
    uint32_t *Tg = reinterpret_cast<uint32_t *>(rec + kRecT) + lane;
    auto t_out = [&](int block, int low, float x, float y) {      // as bf16, and what that leaves, `low` bytes into the record
      const uint32_t high = pack_bf16(x, y);
      const float2 h = unpack_bf16(high);
      Tg[32 * block] = high;
      Tg[(low - kRecT) / 4] = pack_bf16(x - h.x, y - h.y);
    };
#pragma unroll
    for (int d = 0; d < 2; ++d)
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        const float2 t = *reinterpret_cast<const float2 *>(Td + d * kTHalf + (8 * (x >> 1) + g) * kPT + 8 * (x & 1) + 2 * c);
        t_out(4 * (2 * d + (x >> 1)) + 2 * d + (x & 1), (d ? kRecP : kRecT) + kRecTLDiag + 128 * (4 * (x >> 1) + (x & 1)), t.x, t.y);
      }
    // W = T_22 M_21; its accumulators are the next product's A operand with columns 2c, 2c + 1 in k slots c, c + 4
    float W[2][4] = {}, Z[2][4] = {};
#pragma unroll
    for (int kt = 0; kt < 2; ++kt) {
      const float *t = T22 + g * kPT + 8 * kt + c, *m = M + (16 + 8 * kt + c) * kPM + g;
      const uint32_t A[4] = {tf32(t[0]), tf32(t[8 * kPT]), tf32(t[4]), tf32(t[8 * kPT + 4])};
#pragma unroll
      for (int nt = 0; nt < 2; ++nt) mma_tf32(W[nt], A, tf32(m[8 * nt]), tf32(m[4 * kPM + 8 * nt]));
    }
#pragma unroll
    for (int kt = 0; kt < 2; ++kt) {
      const float *t = Td + (8 * kt + 2 * c) * kPT + g;
      const uint32_t A[4] = {tf32(-W[kt][0]), tf32(-W[kt][2]), tf32(-W[kt][1]), tf32(-W[kt][3])};
#pragma unroll
      for (int nt = 0; nt < 2; ++nt) mma_tf32(Z[nt], A, tf32(t[8 * nt]), tf32(t[kPT + 8 * nt]));
    }
    if (__any_sync(0xffffffffu, odd != 0.f)) {      // (0 x NaN: the products would carry a token's NaN to rows before it.  By substitution, T_21 taking M_21's place.)
#pragma unroll 1
      for (int i = 16; i < 32; ++i) {
        const int j = lane & 15;
        float s = 0.f;
        for (int m = 0; m < i; ++m) s = fmaf(-M[i * kPM + m], m < 16 ? Td[m * kPT + j] : M[m * kPM + j], s);
        __syncwarp();
        if (lane < 16) M[i * kPM + j] = s;
        __syncwarp();
      }
#pragma unroll
      for (int nt = 0; nt < 2; ++nt)
#pragma unroll
        for (int r = 0; r < 4; ++r) Z[nt][r] = M[(16 + g + 8 * (r >> 1)) * kPM + 8 * nt + 2 * c + (r & 1)];
    }
#pragma unroll
    for (int nt = 0; nt < 2; ++nt) {
      t_out(4 * 2 + nt, kRecTL + 128 * nt, Z[nt][0], Z[nt][1]);
      t_out(4 * 3 + nt, kRecTL + 128 * (2 + nt), Z[nt][2], Z[nt][3]);
    }
    __syncwarp();
  }
}

template <int K> cudaError_t launch_k(const DeltaArgs &a, cudaStream_t s) {
  const int dq = a.N / a.Nq, dk = a.N / a.Nk;
  int run = dq, o = dk;
  while (o) { const int t = run % o; run = o; o = t; }          // heads in a row that share both q and k
  // a run is cut where that makes warps for the SMs to work on
  const long long want = (long long)sm_count() * 8;
  int per = run;
  for (int d = run; d >= 1; --d)
    if (run % d == 0) {
      per = d;
      if (a.slots * (a.N / d) >= want) break;
    }
  const long long jobs = a.slots * (a.N / per);
  return launch_early(a.cu ? delta_prep_kernel<K, true> : delta_prep_kernel<K, false>, dim3((unsigned)((jobs + kWarps - 1) / kWarps)), dim3(32 * kWarps), 0, s, a, per);
}

}  // namespace

cudaError_t launch_delta_prep(const DeltaArgs &a, cudaStream_t s) {
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
