// Gated delta rule, bf16: what does not depend on the state, chunk by chunk (see delta_chain.cu for the rule in chunks).
//
// For a chunk of 32 tokens of one head, with g the running sum of log a, r_k, r_q the reciprocal lengths:
//     M_ij = b_i e^(g_i - g_j) r_k,i r_k,j (k_i . k_j)   (j < i)        T = (I + M)^-1
//     P_ij = s   e^(g_i - g_j) r_q,i r_k,j (q_i . k_j)   (j <= i)
// Differences g_i - g_j are formed before the exponential: no e^-g that could overflow.
//
// A warp does a chunk for all heads that share its q and k: the two products of 32 x 32 are taken once (mma.sync, fp32
// accumulators that stay in registers), then for each head the gates, M, its inverse and P.  T is inverted in fp32:
// the two 16 x 16 blocks on the diagonal by forward substitution, a column a lane (a series of powers of M would
// cancel digits where keys point the same way), then T_21 = -T_22 M_21 T_11.
#include "delta_common.cuh"

namespace m2rnn {
namespace {

constexpr int kWarps = 4, kPM = 36;   // pitch of M (floats)

template <int K> struct PrepCfg {
  static constexpr int kPitch = 2 * K + 16;                     // bytes; an odd number of 16: ldmatrix without conflicts
  static constexpr int kTile = 32 * kPitch;
  static constexpr int kScratch = (32 + 16) * kPM * 4 + 2048;   // M, T_22; then T as blocks (over the tiles, dead by then)
  static constexpr int kWarpBytes = 2 * kTile > kScratch ? 2 * kTile : kScratch;
};

template <int K>
__global__ void __launch_bounds__(32 * kWarps) delta_prep_kernel(DeltaArgs a, int run) {
  using Cfg = PrepCfg<K>;
  extern __shared__ __align__(128) unsigned char smem[];
  begin_dependent();
  const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31, g = lane >> 2, c = lane & 3;
  const int runs = a.N / run;
  // (a packed batch's sequences are of different lengths: blocks of chunks that a sequence does not have leave at once)
  const long long job = (long long)blockIdx.x * kWarps + warp;
  const long long bc = job / runs;
  const int n0 = (int)(job % runs) * run;
  const int b = (int)(bc / a.nch), ch = (int)(bc % a.nch);
  if (b >= a.B) return;
  const DeltaSpan sp = delta_span<kDeltaChunk>(a, b);
  if (ch >= sp.n) return;
  const long long tok = sp.tok0 + ch * kDeltaChunk;
  const int have = min(kDeltaChunk, sp.T - ch * kDeltaChunk);
  const int hq = n0 / (a.N / a.Nq), hk = n0 / (a.N / a.Nk);

  unsigned char *mine = smem + warp * Cfg::kWarpBytes;
  const uint32_t ksa = smem_u32(mine), qsa = ksa + Cfg::kTile;
  {
    const __nv_bfloat16 *kg = static_cast<const __nv_bfloat16 *>(a.k) + tok * a.ks + (long long)hk * K;
    const __nv_bfloat16 *qg = static_cast<const __nv_bfloat16 *>(a.q) + tok * a.qs + (long long)hq * K;
    for (int x = lane; x < 32 * (K / 8); x += 32) {
      const int r = x / (K / 8), o = x % (K / 8);
      const bool ok = r < have;
      cp16_or_zero(ksa + r * Cfg::kPitch + 16 * o, kg + (ok ? r * a.ks : 0) + 8 * o, ok);
      cp16_or_zero(qsa + r * Cfg::kPitch + 16 * o, qg + (ok ? r * a.qs : 0) + 8 * o, ok);
    }
    cp_wait_all();
    __syncwarp();
  }
  // reciprocal lengths of this lane's token's rows
  float rk = 1.f, rq = 1.f;
  if (a.qk_norm) {
    float sk = 0.f, sq = 0.f;
    for (int o = 0; o < K / 8; ++o) {
      const uint4 x = *reinterpret_cast<const uint4 *>(mine + lane * Cfg::kPitch + 16 * o);
      const uint4 z = *reinterpret_cast<const uint4 *>(mine + Cfg::kTile + lane * Cfg::kPitch + 16 * o);
      const uint32_t xs[4] = {x.x, x.y, x.z, x.w}, zs[4] = {z.x, z.y, z.z, z.w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float2 u = unpack_bf16(xs[i]), w = unpack_bf16(zs[i]);
        sk = fmaf(u.x, u.x, fmaf(u.y, u.y, sk));
        sq = fmaf(w.x, w.x, fmaf(w.y, w.y, sq));
      }
    }
    rk = 1.f / sqrtf(sk + a.eps);
    rq = 1.f / sqrtf(sq + a.eps);
  }
  // k k^T and q k^T, tiles (mt, nt) of 16 x 8 on and below the diagonal: mt = 0: nt 0, 1; mt = 1: nt 0 .. 3
  float kk[6][4] = {}, qk[6][4] = {};
#pragma unroll
  for (int kt = 0; kt < K / 16; ++kt) {
    const uint32_t ra = (uint32_t)((lane & 15) * Cfg::kPitch + 32 * kt + 16 * (lane >> 4));                                 // A: rows lane % 16
    const uint32_t rb = (uint32_t)(((lane & 7) + 8 * (lane >> 4)) * Cfg::kPitch + 32 * kt + 16 * ((lane >> 3) & 1));      // B: two tiles of tokens
    uint32_t a0[4], a1[4], q0[4], q1[4], b0[4], b1[4];
    ldmatrix_x4(ksa + ra, a0);
    ldmatrix_x4(ksa + ra + 16 * Cfg::kPitch, a1);
    ldmatrix_x4(qsa + ra, q0);
    ldmatrix_x4(qsa + ra + 16 * Cfg::kPitch, q1);
    ldmatrix_x4(ksa + rb, b0);
    ldmatrix_x4(ksa + rb + 16 * Cfg::kPitch, b1);
    mma_add(kk[0], a0, b0[0], b0[1]);
    mma_add(kk[1], a0, b0[2], b0[3]);
    mma_add(kk[2], a1, b0[0], b0[1]);
    mma_add(kk[3], a1, b0[2], b0[3]);
    mma_add(kk[4], a1, b1[0], b1[1]);
    mma_add(kk[5], a1, b1[2], b1[3]);
    mma_add(qk[0], q0, b0[0], b0[1]);
    mma_add(qk[1], q0, b0[2], b0[3]);
    mma_add(qk[2], q1, b0[0], b0[1]);
    mma_add(qk[3], q1, b0[2], b0[3]);
    mma_add(qk[4], q1, b1[0], b1[1]);
    mma_add(qk[5], q1, b1[2], b1[3]);
  }
  __syncwarp();   // the tiles are read: their place is M's now
  // the factors that no head changes
  float rkj[4][2], rki[4], rqi[4];
#pragma unroll
  for (int x = 0; x < 4; ++x) {
    rki[x] = __shfl_sync(0xffffffffu, rk, g + 8 * x);
    rqi[x] = a.scale * __shfl_sync(0xffffffffu, rq, g + 8 * x);
    rkj[x][0] = __shfl_sync(0xffffffffu, rk, 8 * x + 2 * c);
    rkj[x][1] = __shfl_sync(0xffffffffu, rk, 8 * x + 2 * c + 1);
  }
  float *M = reinterpret_cast<float *>(mine), *T22 = M + 32 * kPM;
  unsigned char *Tb = reinterpret_cast<unsigned char *>(T22 + 16 * kPM);
  const uint32_t Msa = smem_u32(M);

  for (int n = n0; n < n0 + run; ++n) {
    float la = 0.f, bt = 0.f, dlog = 0.f;
    if (lane < have) {
      const size_t at = (size_t)(tok + lane) * a.N + n;
      const bool psi = a.gate_kind == M2RNN_GATE_PSI;
      float unused;
      la = delta_log_decay(a.gate_kind, __bfloat162float(static_cast<const __nv_bfloat16 *>(a.gate)[at]), psi ? a.alpha[n] : 1.f, psi ? a.beta[n] : 0.f, dlog);
      bt = delta_step_of(a.step_kind, __bfloat162float(static_cast<const __nv_bfloat16 *>(a.step)[at]), unused);
    }
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
#pragma unroll
    for (int nt = 0; nt < 4; ++nt) {
      const float g0 = __shfl_sync(0xffffffffu, gs, 8 * nt + 2 * c), g1 = __shfl_sync(0xffffffffu, gs, 8 * nt + 2 * c + 1);
      const int j = 8 * nt + 2 * c;
#pragma unroll
      for (int mt = nt < 2 ? 0 : 1; mt < 2; ++mt) {
        const int tile = mt ? 2 + nt : nt;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int x = 2 * mt + h, i = g + 8 * x;
          const float e0 = i >= j ? __expf(gi[x] - g0) * rkj[nt][0] : 0.f, e1 = i >= j + 1 ? __expf(gi[x] - g1) * rkj[nt][1] : 0.f;
          const float m0 = i > j ? bi[x] * e0 * kk[tile][2 * h] : 0.f, m1 = i > j + 1 ? bi[x] * e1 * kk[tile][2 * h + 1] : 0.f;
          sts64(Msa + 4u * (i * kPM + j), make_float2(m0, m1));
          const float p0 = i >= j ? rqi[x] * e0 * qk[tile][2 * h] : 0.f, p1 = i >= j + 1 ? rqi[x] * e1 * qk[tile][2 * h + 1] : 0.f;
          reinterpret_cast<uint32_t *>(rec + kRecP)[(4 * x + nt) * 32 + lane] = pack_bf16(p0, p1);
        }
      }
    }
    __syncwarp();
    // the diagonal blocks: lane (half, j) has column j of block `half`
    const int half = lane >> 4, j = lane & 15;
    float t[16];
    {
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
      }
    }
    if (half) {
#pragma unroll
      for (int i = 0; i < 16; ++i) T22[i * kPM + j] = t[i];
    }
    __nv_bfloat16 *tb = reinterpret_cast<__nv_bfloat16 *>(Tb);
#pragma unroll
    for (int i = 0; i < 16; ++i) tb[(4 * (2 * half + (i >> 3)) + 2 * half + (j >> 3)) * 64 + (i & 7) * 8 + (j & 7)] = __float2bfloat16_rn(t[i]);
    // Z = M_21 T_11: lane (half, j) rows 8 half .. of column j
    float z[8];
    {
      float c11[16];
#pragma unroll
      for (int m = 0; m < 16; ++m) c11[m] = __shfl_sync(0xffffffffu, t[m], j);
      const float *Mz = M + (16 + 8 * half) * kPM;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        float s0 = 0.f, s1 = 0.f;
#pragma unroll
        for (int m4 = 0; m4 < 16; m4 += 4) {
          const float4 w = *reinterpret_cast<const float4 *>(Mz + i * kPM + m4);
          s0 = fmaf(w.x, c11[m4], s0);
          s1 = fmaf(w.y, c11[m4 + 1], s1);
          s0 = fmaf(w.z, c11[m4 + 2], s0);
          s1 = fmaf(w.w, c11[m4 + 3], s1);
        }
        z[i] = s0 + s1;
      }
    }
    __syncwarp();
    {
      float zz[16];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float o = __shfl_xor_sync(0xffffffffu, z[i], 16);
        zz[i] = half ? o : z[i];
        zz[8 + i] = half ? z[i] : o;
      }
      const float *Tz = T22 + 8 * half * kPM;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        float s0 = 0.f, s1 = 0.f;
#pragma unroll
        for (int m4 = 0; m4 < 16; m4 += 4) {
          const float4 w = *reinterpret_cast<const float4 *>(Tz + i * kPM + m4);
          s0 = fmaf(w.x, zz[m4], s0);
          s1 = fmaf(w.y, zz[m4 + 1], s1);
          s0 = fmaf(w.z, zz[m4 + 2], s0);
          s1 = fmaf(w.w, zz[m4 + 3], s1);
        }
        tb[(4 * (2 + half) + (j >> 3)) * 64 + i * 8 + (j & 7)] = __float2bfloat16_rn(-(s0 + s1));
      }
    }
    __syncwarp();
    {
      // blocks 0, 1, 4, 5 and 8 .. 15
      uint4 *out = reinterpret_cast<uint4 *>(rec + kRecT);
      const uint4 *in = reinterpret_cast<const uint4 *>(Tb);
      const int first = (lane & 7) + 8 * ((lane >> 3) & 1) + 32 * (lane >> 4);
      out[first] = in[first];
      out[64 + lane] = in[64 + lane];
      out[96 + lane] = in[96 + lane];
    }
    __syncwarp();
  }
}

template <int K> cudaError_t launch_k(const DeltaArgs &a, cudaStream_t s) {
  using Cfg = PrepCfg<K>;
  constexpr size_t smem = (size_t)kWarps * Cfg::kWarpBytes;
  cudaError_t e = allow_smem(delta_prep_kernel<K>, smem);
  if (e != cudaSuccess) return e;
  const int dq = a.N / a.Nq, dk = a.N / a.Nk;
  int run = dq, o = dk;
  while (o) { const int t = run % o; run = o; o = t; }          // heads in a row that share both q and k
  // a run is cut where that makes warps for the SMs to work on
  const long long chunks = a.cu ? a.TT / kDeltaChunk + a.B : (long long)a.B * a.nch, want = (long long)sm_count() * 8;
  int per = run;
  for (int d = run; d >= 1; --d)
    if (run % d == 0) {
      per = d;
      if (chunks * (a.N / d) >= want) break;
    }
  const long long jobs = (long long)a.B * a.nch * (a.N / per);
  return launch_early(delta_prep_kernel<K>, dim3((unsigned)((jobs + kWarps - 1) / kWarps)), dim3(32 * kWarps), smem, s, a, per);
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
