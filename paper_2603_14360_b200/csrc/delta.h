// Internal declarations of the gated delta rule (delta_*.cu) and of the state copy.
#pragma once

#include <cuda_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "m2rnn.h"

namespace m2rnn {

constexpr int kDeltaChunk = 32;        // tokens of a chunk (bf16 kernels)
constexpr int kDeltaChunkF32 = 16;     // (fp32 kernels)

// What the chains and the gradient kernel need of one chunk of one head (delta_prep.cu):
//   T, P: 32 x 32 bf16 as 8 x 8 blocks, block (bi, bj) at 128 (4 bi + bj) bytes, its rows 16 bytes each; blocks
//         above the diagonal of 16 x 16 blocks are not written
//   TL  : what T's entries lose as bf16: its blocks of 16 x 16 on the diagonal in the places above T's and P's (kRecTLDiag bytes into each),
//         that below it as four 8 x 8 blocks in a row
//   vec : eight fp32 values per token, array after array
constexpr int kRecT = 0, kRecP = 2048, kRecTLDiag = 2 * 128, kRecTL = 4096, kRecVec = 4608, kRecBytes = 5632;
enum {
  kVecEgk = 0,   // e^g r_k             g: running sum of log a in the chunk, r: 1 / length of the row
  kVecEq = 1,    // s e^g r_q
  kVecEk = 2,    // e^(g_last - g) r_k
  kVecBeta = 3,  // step b
  kVecG = 4, kVecRk = 5, kVecRq = 6,
  kVecDlog = 7   // d log a / d gate entry
};
constexpr int kRecChain = kRecVec + 4 * 128 + 128;     // what the chains read of it: up to and with kVecG
constexpr int kRecF32Bytes = (3 * 256 + 11 * 16) * 4;   // fp32: T, P, M 16 x 16, then eleven vectors (delta_f32.cu)

struct DeltaArgs {
  int B, T, N, Nq, Nk, K, V;
  int gate_kind, step_kind, qk_norm;
  float eps, scale;
  int state_bf16;              // element type of h0, hT, d_hT, dh0
  const void *q, *k, *v, *gate, *step, *h0;
  const float *alpha, *beta;
  void *y, *hT;
  char *rec;                   // [slots][N] records
  char *states;                // [slots][N] states at a chunk's start (bf16: blocks; fp32: [V][K] floats), or null
  char *upd;                   // [slots][N] updates U of a chunk (bf16: blocks; fp32: [chunk][V]), or null
  // backward
  const void *dy, *d_hT;
  void *dq, *dk, *dv, *dgate, *dstep, *dh0;
  char *dstates, *lam;         // like states (at a chunk's end) and upd
  float *dq_part, *dk_part;    // [TT][shares][K] fp32, or null where a head's are the final ones
  int shares;                  // CTAs that a token's heads are spread over
  int32_t *dev_status;
  long long qs, ks, vs, TT;
  const int32_t *cu;
  int nch;                     // chunks of the longest sequence
  long long slots;             // chunk slots of the batch
  int per_q, per_k;            // heads to a q head, to a k head
  int sms, nw;                 // chains: SMs of the device, 16-column warps of a CTA
  int hpc, grad_ctas;          // gradient kernel: heads of a job, CTAs to an SM
};

__host__ __device__ inline int delta_chunks(int T, int C) { return T / C + (T % C != 0); }

// First token, length, first chunk slot and chunks of batch entry b.  Of a packed batch, sequence b's slots start at
// cu[b] / chunk + b: no two overlap, whatever the lengths.  Offsets are cut to 0 .. TT and lengths to T: nothing is
// addressed beyond what those sized.
struct DeltaSpan { long long tok0, slot0; int T, n; };
#ifdef __CUDACC__
template <int C> __device__ __forceinline__ DeltaSpan delta_span(const DeltaArgs &a, int b) {
  DeltaSpan s;
  if (a.cu) {
    const long long lo = min(max((long long)a.cu[b], 0ll), a.TT), hi = min(max((long long)a.cu[b + 1], lo), a.TT);
    s.tok0 = lo;
    s.T = (int)min(hi - lo, (long long)a.T);
    s.slot0 = lo / C + b;
  } else {
    s.tok0 = (long long)b * a.T;
    s.T = a.T;
    s.slot0 = (long long)b * a.nch;
  }
  s.n = delta_chunks(s.T, C);
  return s;
}
// The batch entry that chunk slot `slot` belongs to (every lane of a warp calls it): of a packed batch the last one whose slots do not start
// behind it, or entry 0 where none's do (offsets that begin behind 0): whether the slot is one of the entry's is for the caller to see, on both
// sides (of entry 0's, or of offsets that fall, it may lie before the first).  (Jobs are numbered by slots: by entry and chunk of the longest, a ragged batch's were mostly none.)
template <int C, bool PACKED> __device__ __forceinline__ int delta_entry(const DeltaArgs &a, unsigned slot) {
  if (!PACKED) return (int)(slot / (unsigned)a.nch);
  int b = 0;
  for (int x = 1; x < a.B; x += 32) {
    const int i = x + (int)(threadIdx.x & 31);
    const bool in = i < a.B && min(max((long long)a.cu[i], 0ll), a.TT) / C + i <= slot;
    b += __popc(__ballot_sync(0xffffffffu, in));
  }
  return __shfl_sync(0xffffffffu, b, 0);      // (known to be the same in all lanes: what derives from it stays in uniform registers)
}
#endif
inline size_t delta_slots(const m2rnn_delta_params *p, size_t tokens, int C) {
  return p->cu_seqlens ? tokens / C + p->B : (size_t)p->B * delta_chunks(p->T, C);
}

cudaError_t launch_delta_prep(const DeltaArgs &a, cudaStream_t s);        // delta_prep.cu
cudaError_t launch_delta_chain_fwd(const DeltaArgs &a, cudaStream_t s);   // delta_chain.cu
cudaError_t launch_delta_chain_bwd(const DeltaArgs &a, cudaStream_t s);
struct GradPlan { int heads, ctas; };
GradPlan delta_grad_plan(const m2rnn_delta_params *p, size_t slots);      // delta_grad.cu
cudaError_t launch_delta_grad(const DeltaArgs &a, cudaStream_t s);
// launch_reduce_heads (reduce.cu); of a packed batch (cu, with B and T) only rows of tokens that belong to a sequence are written
cudaError_t launch_reduce_heads_of(const float *part, void *out, int io_dtype, size_t BT, int N, int Ng, int K, const int32_t *cu, int B, int T, cudaStream_t s);
cudaError_t launch_delta_fwd_f32(const DeltaArgs &a, cudaStream_t s);     // delta_f32.cu
cudaError_t launch_delta_bwd_f32(const DeltaArgs &a, cudaStream_t s);

struct DeltaStepArgs {
  int B, N, Nq, Nk, K, V, per_q, per_k;      // per: as in DeltaArgs
  int gate_kind, step_kind, qk_norm;
  float eps, scale;
  const void *q, *k, *v, *gate, *step;
  const float *alpha, *beta;
  void *state, *y;
  const int32_t *slots;
  int nslots;
  int32_t *dev_status;
};
cudaError_t launch_delta_step(const DeltaStepArgs &a, int io_dtype, int state_dtype, cudaStream_t s);   // delta_decode.cu

struct StateCopyArgs {
  const char *src;
  char *dst;
  const int32_t *src_slots, *dst_slots;
  int n, src_rows, dst_rows, layers;
  long long row_bytes, src_layer, dst_layer;   // bytes
  int32_t *dev_status;
};
cudaError_t launch_state_copy(const StateCopyArgs &a, cudaStream_t s);   // state_copy.cu
int state_copy_limit();

}  // namespace m2rnn
