// C ABI of the gated delta rule and of the state copy: argument checks, workspace layout, dispatch.
#include <cuda_runtime.h>

#include <algorithm>

#include "delta.h"
#include "internal.h"
#include "m2rnn.h"

namespace m2rnn {
namespace {

int cuda_failed() {
  (void)cudaGetLastError();
  return M2RNN_ERR_CUDA;
}
bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

int chunk_of(const m2rnn_delta_params *p) { return p->io_dtype == M2RNN_BF16 ? kDeltaChunk : kDeltaChunkF32; }
size_t tokens_of(const m2rnn_delta_params *p) { return p->cu_seqlens ? (size_t)p->total_tokens : (size_t)p->B * p->T; }
size_t state_elem(const m2rnn_delta_params *p) { return p->state_dtype == M2RNN_BF16 ? 2 : 4; }

int check_params(const m2rnn_delta_params *p, bool step) {
  if (!p) return M2RNN_ERR_NULL;
  if (p->B < 0 || p->N <= 0 || p->K <= 0 || p->V <= 0 || (!step && p->T < 0)) return M2RNN_ERR_SHAPE;
  if (p->Nq <= 0 || p->Nk <= 0 || p->Nq > p->N || p->Nk > p->N || p->N % p->Nq || p->N % p->Nk) return M2RNN_ERR_SHAPE;
  if (p->io_dtype != M2RNN_F32 && p->io_dtype != M2RNN_BF16) return M2RNN_ERR_UNSUPPORTED;
  if (p->state_dtype != M2RNN_F32 && p->state_dtype != M2RNN_BF16) return M2RNN_ERR_UNSUPPORTED;
  if (p->gate_kind < M2RNN_GATE_LOGIT || p->gate_kind > M2RNN_GATE_LOG) return M2RNN_ERR_UNSUPPORTED;
  if (p->step_kind != M2RNN_STEP_VALUE && p->step_kind != M2RNN_STEP_LOGIT) return M2RNN_ERR_UNSUPPORTED;
  if (p->K % 16 || p->K > 128) return M2RNN_ERR_UNSUPPORTED;
  if (p->V != 16 && p->V != 32 && p->V != 64 && p->V != 128) return M2RNN_ERR_UNSUPPORTED;
  // (every element of a state tensor and every CTA of a launch has a number that the kernels can hold)
  if ((int64_t)p->B * p->N > (int64_t)0x7fffffff / 8) return M2RNN_ERR_SHAPE;
  if (step) return M2RNN_OK;
  const int64_t unit16 = p->io_dtype == M2RNN_BF16 ? 8 : 4;
  const int64_t dense[3] = {(int64_t)p->Nq * p->K, (int64_t)p->Nk * p->K, (int64_t)p->N * p->V};
  const int64_t given[3] = {p->q_stride, p->k_stride, p->v_stride};
  for (int x = 0; x < 3; ++x)
    if (given[x] != 0 && (given[x] < dense[x] || given[x] % unit16)) return M2RNN_ERR_SHAPE;
  if (p->total_tokens < 0 || (!p->cu_seqlens && p->total_tokens != 0)) return M2RNN_ERR_SHAPE;
  if (p->cu_seqlens && p->total_tokens > (int64_t)p->B * p->T) return M2RNN_ERR_SHAPE;
  if ((p->cu_seqlens ? p->total_tokens / 16 + p->B : (int64_t)p->B * (delta_chunks(p->T, 16) + 1)) > (int64_t)0x7fffffff / p->N) return M2RNN_ERR_SHAPE;
  return M2RNN_OK;
}

// What a forward call leaves for the backward one: records, states at the chunks' starts, updates
struct Ckpt { size_t rec, states, upd, total; };
Ckpt ckpt_layout(const m2rnn_delta_params *p) {
  Ckpt c{};
  const size_t units = delta_slots(p, tokens_of(p), chunk_of(p)) * p->N, KV = (size_t)p->K * p->V;
  const bool f32 = p->io_dtype == M2RNN_F32;
  const size_t e = f32 ? 4 : 2;
  c.states = align_up(units * (f32 ? kRecF32Bytes : kRecBytes));
  c.upd = c.states + align_up(units * KV * e);
  c.total = c.upd + align_up(units * chunk_of(p) * p->V * e);
  return c;
}

struct Workspace { size_t ckpt, dstates, lam, dq, dk, total; GradPlan grad; };
Workspace bwd_layout(const m2rnn_delta_params *p, bool have_ckpt) {
  Workspace w{};
  const size_t tokens = tokens_of(p), slots = delta_slots(p, tokens, chunk_of(p)), units = slots * p->N;
  size_t off = have_ckpt ? 0 : ckpt_layout(p).total;
  const bool f32 = p->io_dtype == M2RNN_F32;
  w.grad = f32 ? GradPlan{1, 0} : delta_grad_plan(p, slots);
  const int hpc = w.grad.heads;
  w.dstates = off;
  off += align_up(units * p->K * p->V * (f32 ? 4 : 2));
  w.lam = off;
  off += align_up(units * chunk_of(p) * p->V * (f32 ? 4 : 2));
  const size_t shares = tokens * (p->N / hpc) * p->K * sizeof(float);
  w.dq = off;
  if (p->N / p->Nq > hpc) off += align_up(shares);
  w.dk = off;
  if (p->N / p->Nk > hpc) off += align_up(shares);
  w.total = off;
  return w;
}

DeltaArgs base_args(const m2rnn_delta_params *p, const void *q, const void *k, const void *v, const void *gate, const void *step, const void *h0,
                    const float *alpha, const float *beta) {
  DeltaArgs a{};
  a.B = p->B; a.T = p->T; a.N = p->N; a.Nq = p->Nq; a.Nk = p->Nk; a.K = p->K; a.V = p->V;
  a.gate_kind = p->gate_kind; a.step_kind = p->step_kind; a.qk_norm = p->qk_norm != 0; a.eps = p->norm_eps; a.scale = p->q_scale;
  a.state_bf16 = p->state_dtype == M2RNN_BF16;
  a.q = q; a.k = k; a.v = v; a.gate = gate; a.step = step; a.h0 = h0; a.alpha = alpha; a.beta = beta;
  a.qs = p->q_stride ? p->q_stride : (long long)p->Nq * p->K;
  a.ks = p->k_stride ? p->k_stride : (long long)p->Nk * p->K;
  a.vs = p->v_stride ? p->v_stride : (long long)p->N * p->V;
  a.TT = (long long)tokens_of(p);
  a.cu = p->cu_seqlens;
  a.nch = delta_chunks(p->T, chunk_of(p));
  a.slots = (long long)delta_slots(p, tokens_of(p), chunk_of(p));
  a.per_q = p->N / p->Nq; a.per_k = p->N / p->Nk;
  return a;
}
// A call without tokens leaves the states as they are: `to` = `from`, or zeros
int pass_state(const m2rnn_delta_params *p, void *to, const void *from, cudaStream_t s) {
  if (!aligned16(to) || !aligned16(from)) return M2RNN_ERR_ALIGN;
  if (!to || to == from || p->B == 0) return M2RNN_OK;
  const size_t bytes = state_elem(p) * p->B * p->N * p->K * p->V;
  const cudaError_t e = from ? cudaMemcpyAsync(to, from, bytes, cudaMemcpyDeviceToDevice, s) : cudaMemsetAsync(to, 0, bytes, s);
  return e == cudaSuccess ? M2RNN_OK : cuda_failed();
}
bool empty_call(const m2rnn_delta_params *p) { return p->B == 0 || p->T == 0 || tokens_of(p) == 0; }

// the forward kernels; ckpt: where records (and, with `keep`, states and updates) go
cudaError_t run_fwd(DeltaArgs a, const m2rnn_delta_params *p, char *ckpt, bool keep, cudaStream_t s) {
  const Ckpt c = ckpt_layout(p);
  a.rec = ckpt + c.rec;
  a.states = keep ? ckpt + c.states : nullptr;
  a.upd = keep ? ckpt + c.upd : nullptr;
  if (p->io_dtype == M2RNN_F32) return launch_delta_fwd_f32(a, s);
  const cudaError_t e = launch_delta_prep(a, s);
  return e != cudaSuccess ? e : launch_delta_chain_fwd(a, s);
}

}  // namespace
}  // namespace m2rnn

using namespace m2rnn;

extern "C" {

size_t m2rnn_delta_ckpt_bytes(const m2rnn_delta_params *params) {
  if (check_params(params, false) != M2RNN_OK || empty_call(params)) return 0;
  return ckpt_layout(params).total;
}

size_t m2rnn_delta_fwd_workspace_bytes(const m2rnn_delta_params *params, int have_ckpt) {
  if (check_params(params, false) != M2RNN_OK || empty_call(params) || have_ckpt) return 0;
  return ckpt_layout(params).states;      // the records
}

int m2rnn_delta_fwd(const m2rnn_delta_params *params, const void *q, const void *k, const void *v, const void *gate, const void *step, const void *h0,
                    const float *alpha, const float *beta, void *y, void *hT, void *ckpt, void *workspace, size_t workspace_bytes, int32_t *dev_status,
                    void *stream) {
  const int rc = check_params(params, false);
  if (rc != M2RNN_OK) return rc;
  if (empty_call(params)) return pass_state(params, hT, h0, static_cast<cudaStream_t>(stream));
  if (!q || !k || !v || !gate || !step || !y) return M2RNN_ERR_NULL;
  if (params->gate_kind == M2RNN_GATE_PSI && (!alpha || !beta)) return M2RNN_ERR_NULL;
  const void *ptrs[] = {q, k, v, gate, step, h0, y, hT, ckpt};
  for (const void *p : ptrs)
    if (!aligned16(p)) return M2RNN_ERR_ALIGN;
  const size_t need = m2rnn_delta_fwd_workspace_bytes(params, ckpt != nullptr);
  if (need > 0 && (!workspace || workspace_bytes < need)) return M2RNN_ERR_WORKSPACE;
  if (reinterpret_cast<uintptr_t>(workspace) % kAlign || reinterpret_cast<uintptr_t>(ckpt) % kAlign) return M2RNN_ERR_ALIGN;
  DeltaArgs a = base_args(params, q, k, v, gate, step, h0, alpha, beta);
  a.y = y; a.hT = hT; a.dev_status = dev_status;
  const cudaError_t e = run_fwd(a, params, static_cast<char *>(ckpt ? ckpt : workspace), ckpt != nullptr, static_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? M2RNN_OK : cuda_failed();
}

size_t m2rnn_delta_bwd_workspace_bytes(const m2rnn_delta_params *params, int have_ckpt) {
  if (check_params(params, false) != M2RNN_OK || empty_call(params)) return 0;
  return bwd_layout(params, have_ckpt != 0).total;
}

int m2rnn_delta_bwd(const m2rnn_delta_params *params, const void *q, const void *k, const void *v, const void *gate, const void *step, const void *h0,
                    const float *alpha, const float *beta, const void *ckpt, const void *dy, const void *d_hT, void *dq, void *dk, void *dv, void *dgate,
                    void *dstep, void *dh0, void *workspace, size_t workspace_bytes, int32_t *dev_status, void *stream) {
  const int rc = check_params(params, false);
  if (rc != M2RNN_OK) return rc;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (empty_call(params)) return pass_state(params, dh0, d_hT, s);      // (the only defined output)
  if (!q || !k || !v || !gate || !step || !dy || !dq || !dk || !dv || !dgate || !dstep) return M2RNN_ERR_NULL;
  if (params->gate_kind == M2RNN_GATE_PSI && (!alpha || !beta)) return M2RNN_ERR_NULL;
  const void *ptrs[] = {q, k, v, gate, step, h0, ckpt, dy, d_hT, dq, dk, dv, dgate, dstep, dh0};
  for (const void *p : ptrs)
    if (!aligned16(p)) return M2RNN_ERR_ALIGN;
  const Workspace w = bwd_layout(params, ckpt != nullptr);
  if (w.total > 0 && (!workspace || workspace_bytes < w.total)) return M2RNN_ERR_WORKSPACE;
  if (reinterpret_cast<uintptr_t>(workspace) % kAlign || reinterpret_cast<uintptr_t>(ckpt) % kAlign) return M2RNN_ERR_ALIGN;
  char *ws = static_cast<char *>(workspace);
  DeltaArgs a = base_args(params, q, k, v, gate, step, h0, alpha, beta);
  a.dev_status = dev_status;
  char *kept = ckpt ? static_cast<char *>(const_cast<void *>(ckpt)) : ws + w.ckpt;
  if (!ckpt) {      // the forward pass without y
    const cudaError_t e = run_fwd(a, params, kept, true, s);
    if (e != cudaSuccess) return cuda_failed();
  }
  a.dy = dy; a.d_hT = d_hT; a.dq = dq; a.dk = dk; a.dv = dv; a.dgate = dgate; a.dstep = dstep; a.dh0 = dh0;
  a.hpc = w.grad.heads; a.grad_ctas = w.grad.ctas;
  a.shares = params->N / a.hpc;
  a.dq_part = params->N / params->Nq > a.hpc ? reinterpret_cast<float *>(ws + w.dq) : nullptr;
  a.dk_part = params->N / params->Nk > a.hpc ? reinterpret_cast<float *>(ws + w.dk) : nullptr;
  cudaError_t e;
  const Ckpt c = ckpt_layout(params);
  a.rec = kept + c.rec; a.states = kept + c.states; a.upd = kept + c.upd;
  a.dstates = ws + w.dstates; a.lam = ws + w.lam;
  if (params->io_dtype == M2RNN_F32) {
    e = launch_delta_bwd_f32(a, s);
  } else {
    e = launch_delta_chain_bwd(a, s);
    if (e == cudaSuccess) e = launch_delta_grad(a, s);
  }
  const size_t tokens = tokens_of(params);
  if (e == cudaSuccess && a.dq_part) e = launch_reduce_heads_of(a.dq_part, dq, params->io_dtype, tokens, a.shares, params->Nq, params->K, a.cu, a.B, a.T, s);
  if (e == cudaSuccess && a.dk_part) e = launch_reduce_heads_of(a.dk_part, dk, params->io_dtype, tokens, a.shares, params->Nk, params->K, a.cu, a.B, a.T, s);
  return e == cudaSuccess ? M2RNN_OK : cuda_failed();
}

int m2rnn_delta_decode_step(const m2rnn_delta_params *params, const void *q, const void *k, const void *v, const void *gate, const void *step,
                            const float *alpha, const float *beta, void *state, const int32_t *slots, int32_t n_slots, void *y, int32_t *dev_status,
                            void *stream) {
  const int rc = check_params(params, true);
  if (rc != M2RNN_OK) return rc;
  if (slots ? n_slots < 0 : n_slots != params->B) return M2RNN_ERR_SHAPE;
  if (params->B == 0) return M2RNN_OK;
  if (!q || !k || !v || !gate || !step || !state || !y) return M2RNN_ERR_NULL;
  if (params->gate_kind == M2RNN_GATE_PSI && (!alpha || !beta)) return M2RNN_ERR_NULL;
  const void *ptrs[] = {q, k, v, gate, step, state, y};
  for (const void *p : ptrs)
    if (!aligned16(p)) return M2RNN_ERR_ALIGN;
  DeltaStepArgs a{};
  a.B = params->B; a.N = params->N; a.Nq = params->Nq; a.Nk = params->Nk; a.K = params->K; a.V = params->V;
  a.per_q = params->N / params->Nq; a.per_k = params->N / params->Nk;
  a.gate_kind = params->gate_kind; a.step_kind = params->step_kind; a.qk_norm = params->qk_norm != 0; a.eps = params->norm_eps; a.scale = params->q_scale;
  a.q = q; a.k = k; a.v = v; a.gate = gate; a.step = step; a.alpha = alpha; a.beta = beta;
  a.state = state; a.y = y; a.slots = slots; a.nslots = n_slots; a.dev_status = dev_status;
  const cudaError_t e = launch_delta_step(a, params->io_dtype, params->state_dtype, static_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? M2RNN_OK : cuda_failed();
}

int m2rnn_state_copy_limit(void) { return state_copy_limit(); }

int m2rnn_state_copy(void *dst, const int32_t *dst_slots, int32_t dst_rows, int64_t dst_layer_stride, const void *src, const int32_t *src_slots,
                     int32_t src_rows, int64_t src_layer_stride, int32_t n, int64_t row_bytes, int32_t layers, int32_t *dev_status, void *stream) {
  if (n < 0 || layers < 0 || dst_rows < 0 || src_rows < 0 || row_bytes < 0 || row_bytes % 16) return M2RNN_ERR_SHAPE;
  if (n > state_copy_limit()) return M2RNN_ERR_UNSUPPORTED;
  if (n == 0 || layers == 0 || row_bytes == 0) return M2RNN_OK;
  if (!dst || !src || !dst_slots || !src_slots) return M2RNN_ERR_NULL;
  if (!aligned16(dst) || !aligned16(src)) return M2RNN_ERR_ALIGN;
  if (layers > 1) {
    if (dst_layer_stride % 16 || src_layer_stride % 16) return M2RNN_ERR_SHAPE;
    if (dst_layer_stride < (int64_t)dst_rows * row_bytes || src_layer_stride < (int64_t)src_rows * row_bytes) return M2RNN_ERR_SHAPE;
  }
  if (row_bytes / 32 + 1 > (int64_t)0x7fffffff / layers) return M2RNN_ERR_SHAPE;
  StateCopyArgs a{};
  a.src = static_cast<const char *>(src); a.dst = static_cast<char *>(dst);
  a.src_slots = src_slots; a.dst_slots = dst_slots;
  a.n = n; a.src_rows = src_rows; a.dst_rows = dst_rows; a.layers = layers;
  a.row_bytes = row_bytes; a.src_layer = src_layer_stride; a.dst_layer = dst_layer_stride;
  a.dev_status = dev_status;
  const cudaError_t e = launch_state_copy(a, static_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? M2RNN_OK : cuda_failed();
}

}  // extern "C"
