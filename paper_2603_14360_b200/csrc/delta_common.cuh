// Device helpers of the gated delta rule's kernels.
#pragma once

#include "delta.h"
#include "device_common.cuh"
#include "internal.h"
#include "mma_tile.cuh"
#include "pipeline.cuh"
#include "tile.cuh"

namespace m2rnn {

// log a of a gate entry and its derivative.  Below kLogFloor a is 0 in fp32 whatever follows (e^-104 is half the smallest
// denormal): the running sums of a chunk stay finite, and differences of two of them mean something, also after a = 0.
constexpr float kLogFloor = -104.f;
__device__ __forceinline__ float delta_log_decay(int kind, float x, float alpha, float beta, float &d) {
  float l;
  if (kind == M2RNN_GATE_LOG) {
    l = x;
    d = 1.f;
  } else {
    // sigmoid(x) = (1 + e^-x)^-1: the psi gate of -x with alpha = 1, beta = 0
    const bool psi = kind == M2RNN_GATE_PSI;
    const float u = psi ? x + beta : -x, al = psi ? alpha : 1.f;
    const float e = expf(-fabsf(u)), sp = fmaxf(u, 0.f) + log1pf(e), sg = (u >= 0.f ? 1.f : e) / (1.f + e);
    l = -al * sp;
    if (u != u) l = u;              // (fmaxf drops a NaN)
    d = psi ? -al * sg : sg;
  }
  if (l < kLogFloor) { l = kLogFloor; d = 0.f; }
  return l;
}
// step b of an entry and its derivative
__device__ __forceinline__ float delta_step_of(int kind, float x, float &d) {
  if (kind == M2RNN_STEP_VALUE) { d = 1.f; return x; }
  const float e = expf(-fabsf(x)), b = (x >= 0.f ? 1.f : e) / (1.f + e);
  d = b * (1.f - b);
  return x != x ? x : b;
}

// d += a b.  (Not volatile: where products of two chains of dependences stand side by side, the order is the compiler's.)
__device__ __forceinline__ void mma_add(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};\n"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void ldmatrix_x4_t(uint32_t addr, uint32_t (&r)[4]) { ldmatrix_x4_trans(addr, r[0], r[1], r[2], r[3]); }
__device__ __forceinline__ void ldmatrix_x2(uint32_t addr, uint32_t (&r)[2]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x2.shared.b16 {%0,%1}, [%2];" : "=r"(r[0]), "=r"(r[1]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldmatrix_x2_t(uint32_t addr, uint32_t (&r)[2]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x2.trans.shared.b16 {%0,%1}, [%2];" : "=r"(r[0]), "=r"(r[1]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void stmatrix_x4_trans(uint32_t addr, const uint32_t (&r)[4]) {
  asm volatile("stmatrix.sync.aligned.m8n8.x4.trans.shared.b16 [%0], {%1,%2,%3,%4};" ::"r"(addr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]) : "memory");
}
__device__ __forceinline__ void stmatrix_x4(uint32_t addr, const uint32_t (&r)[4]) {
  asm volatile("stmatrix.sync.aligned.m8n8.x4.shared.b16 [%0], {%1,%2,%3,%4};" ::"r"(addr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]) : "memory");
}
// A operand of k-tile kt from accumulator tiles 2kt, 2kt + 1
template <int NT> __device__ __forceinline__ void pack_a(const float (&d)[NT][4], int kt, uint32_t (&a)[4]) {
  a[0] = pack_bf16(d[2 * kt][0], d[2 * kt][1]);
  a[1] = pack_bf16(d[2 * kt][2], d[2 * kt][3]);
  a[2] = pack_bf16(d[2 * kt + 1][0], d[2 * kt + 1][1]);
  a[3] = pack_bf16(d[2 * kt + 1][2], d[2 * kt + 1][3]);
}

__device__ __forceinline__ void mbar_expect(uint64_t *bar, uint32_t bytes) {
  asm volatile("{\n .reg .b64 st;\n mbarrier.arrive.expect_tx.shared::cta.b64 st, [%0], %1;\n}" ::"r"(smem_u32(bar)), "r"(bytes) : "memory");
}
// untiled copy into shared memory: both addresses and the size are multiples of 16 bytes
__device__ __forceinline__ void bulk_load(uint32_t dst, const void *src, uint32_t bytes, uint64_t *bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src), "r"(bytes), "r"(smem_u32(bar)) : "memory");
}
// 16 bytes global -> shared, zeros where !ok (nothing is read then)
__device__ __forceinline__ void cp16_or_zero(uint32_t dst, const void *src, bool ok) {
  const int n = ok ? 16 : 0;
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(n) : "memory");
}
__device__ __forceinline__ void cp_wait_all() { asm volatile("cp.async.wait_all;" ::: "memory"); }

}  // namespace m2rnn
