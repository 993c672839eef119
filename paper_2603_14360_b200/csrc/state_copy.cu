// States moved between the slots of a cache: dst[dst_slots[i]] = src[src_slots[i]] for all i at once (a source of -1
// stands for zeros), in every layer of the cache.
//
// All sources are read before any destination is written, although sources and destinations may be slots of the same
// pool (a compaction shifts, a permutation swaps): a CTA takes a slab of P x 16 bytes of every row, the same bytes of
// each, holds the n pieces of it in registers, and writes them after a barrier.  Slabs do not touch one another, so
// nothing has to be ordered between CTAs and no byte passes through scratch.  P is as large as 64 KB of a CTA allow
// (16 pieces of 16 bytes a thread, or 8), a row's slab at least 32 bytes, a sector: that bounds n.
// Where a destination comes twice the last pair counts; each CTA finds those once (n^2 / 256 comparisons a thread) and
// walks several slabs.
// Few pairs (rows' pieces stay wide): eight pieces a thread and four CTAs to an SM, which load while others store (8 states of 344 KB in 24
// layers from one: 14.9 us, with sixteen and two 19.1); many: sixteen and two (200 of 512 states of 1 MB: 63 us, 77 the other way).
// The line between them lies between figures of 8 and of 200 pairs.  Many pairs of small rows are bound by the comparisons: 1 500 of 16 KB 79 us,
// 2 000 of them 131, where their bytes take 8 and 10.
#include "delta.h"
#include "internal.h"

namespace m2rnn {
namespace {

constexpr int kThreads = 256, kMost = kThreads * 16 / 2, kFew = 64;      // pairs: most, and up to which eight pieces a thread do

template <int kPer>
__global__ void __launch_bounds__(kThreads, 32 / kPer) state_copy_kernel(StateCopyArgs a, int log_p, int slabs) {
  __shared__ int from[kMost], to[kMost];
  begin_dependent();
  const int tid = threadIdx.x, P = 1 << log_p;      // pieces of a slab
  for (int i = tid; i < a.n; i += kThreads) {
    int s = a.src_slots[i], d = a.dst_slots[i];
    if (s >= a.src_rows || d >= a.dst_rows) {       // not a slot: the pair is left out
      if (blockIdx.x == 0 && a.dev_status) atomicExch(a.dev_status, (int32_t)M2RNN_ERR_SHAPE);
      d = -1;
    }
    from[i] = s;
    to[i] = d;
  }
  __syncthreads();
  unsigned later = 0;      // of this thread's pairs, those that a later one replaces
  for (int i = tid, x = 0; i < a.n; i += kThreads, ++x) {
    const int d = to[i];
    bool again = false;
    if (d >= 0)
      for (int o = i + 1; o < a.n; ++o) again |= to[o] == d;
    later |= (unsigned)again << x;
  }
  __syncthreads();
  for (int i = tid, x = 0; i < a.n; i += kThreads, ++x)
    if (later >> x & 1) to[i] = -1;
  __syncthreads();
  const unsigned per_row = (unsigned)((a.row_bytes + 16ll * P - 1) / (16ll * P));
  for (unsigned slab = blockIdx.x; slab < (unsigned)slabs; slab += gridDim.x) {
    const unsigned layer = a.layers > 1 ? slab / per_row : 0;
    const long long first = (long long)(slab - layer * per_row) * 16 * P;
    const char *src = a.src + layer * a.src_layer + first;
    char *dst = a.dst + layer * a.dst_layer + first;
    float4 x[kPer];
#pragma unroll
    for (int r = 0; r < kPer; ++r) {
      const int q = tid + r * kThreads, i = q >> log_p, off = (q & (P - 1)) * 16;
      x[r] = make_float4(0.f, 0.f, 0.f, 0.f);
      if (i < a.n && to[i] >= 0 && from[i] >= 0 && first + off < a.row_bytes)
        asm volatile("ld.global.cg.v4.f32 {%0,%1,%2,%3}, [%4];" : "=f"(x[r].x), "=f"(x[r].y), "=f"(x[r].z), "=f"(x[r].w)
                     : "l"(src + from[i] * a.row_bytes + off) : "memory");
    }
    __syncthreads();      // (all of the slab's sources are in registers)
#pragma unroll
    for (int r = 0; r < kPer; ++r) {
      const int q = tid + r * kThreads, i = q >> log_p, off = (q & (P - 1)) * 16;
      if (i < a.n && to[i] >= 0 && first + off < a.row_bytes) *reinterpret_cast<float4 *>(dst + to[i] * a.row_bytes + off) = x[r];
    }
  }
}

}  // namespace

int state_copy_limit() { return kMost; }

template <int kPer> static cudaError_t launch_per(const StateCopyArgs &a, cudaStream_t s) {
  // the widest slab whose n pieces a CTA holds; no wider than a row, nor (down to 512 bytes) than leaves a slab for each CTA
  const long long most = (long long)sm_count() * (32 / kPer);
  auto slabs_of = [&](int l) { return (a.row_bytes + (16ll << l) - 1) / (16ll << l) * a.layers; };
  int log_p = 1;
  while (((long long)a.n << (log_p + 1)) <= kThreads * kPer && (16ll << log_p) < a.row_bytes && (log_p < 5 || slabs_of(log_p + 1) >= most)) ++log_p;
  const long long slabs = slabs_of(log_p);
  if (slabs > 0x7fffffffll) return cudaErrorInvalidValue;
  return launch_early(state_copy_kernel<kPer>, dim3((unsigned)(slabs < most ? slabs : most)), dim3(kThreads), 0, s, a, log_p, (int)slabs);
}
cudaError_t launch_state_copy(const StateCopyArgs &a, cudaStream_t s) { return a.n <= kFew ? launch_per<8>(a, s) : launch_per<16>(a, s); }

}  // namespace m2rnn
