// Distillation loss: what its kernels share (the formulas: fw_distill.cu).
#ifndef FW_DISTILL_CUH_
#define FW_DISTILL_CUH_

#include "fw_internal.h"
#include "fw_rows.cuh"

namespace fw {
namespace distill {

using namespace rows;

constexpr int kMaxK = 1024;
constexpr int kMaxV = 1 << 20;             // a cluster's bit sets and entries stay below 48 KB of shared memory a CTA
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kLow = -3.402823466e38f;   // the lowest finite value: the largest of nothing, beside a sum of 0
// Logarithms are summed times 2^-21 (exact), so that a logit at the lowest finite value (a mask) times log2(e) / tau stays in
// fp32 for every tau; kUp = 2^21 ln 2 makes the loss of them.
constexpr float kDown = 4.76837158203125e-07f, kUp = 2097152.f * kLn2;
enum { DIST_LOSS = 0, DIST_BOTH = 1, DIST_BACKWARD = 2 };

struct Distill {
  const void* Z;
  const void* T;
  const void* I;
  const float *t_lse, *weight;
  const float* stat_in;
  float *loss, *stat;
  void* dZ;
  int64_t ldz, lddz;
  int32_t V, K;
  int32_t t_bf16, i64;
  int32_t slice;          // classes of a CTA, a multiple of the CTA's accesses
  float inv_tau;
};

// Largest logit m and the sum of exp((z - m) / tau).  Differences of logits are scaled, not logits: near the largest, where the
// mass is, their rounding is small.  c2 = log2(e) / tau.
// (The roundings are written out: the loss alone and the loss with the gradient are the same number.)
struct MaxSum { float m, l; };
__device__ __forceinline__ MaxSum merge(MaxSum a, MaxSum b, float c2) {
  const float m = fmaxf(a.m, b.m);
  return {m, fmaf(a.l, ex2((a.m - m) * c2), __fmul_rn(b.l, ex2((b.m - m) * c2)))};
}
__device__ __forceinline__ float lanes_max(float v) {
  float r;
  asm("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(v));
  return r;
}
__device__ __forceinline__ float lanes_sum(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}
// The whole warp's: its largest first, so that the chain is one exponential and five additions long (five merges took twice that)
__device__ __forceinline__ MaxSum merge_lanes(MaxSum s, float c2) {
  const float m = lanes_max(s.m);
  return {m, lanes_sum(s.l * ex2((s.m - m) * c2))};
}

// Two and three of them at once: the chains run beside each other.
__device__ __forceinline__ void merge_lanes2(MaxSum& a, MaxSum& b, float c2) {
  const float ma = lanes_max(a.m), mb = lanes_max(b.m);
  a = {ma, a.l * ex2((a.m - ma) * c2)};
  b = {mb, b.l * ex2((b.m - mb) * c2)};
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const float x = __shfl_xor_sync(0xffffffffu, a.l, o), y = __shfl_xor_sync(0xffffffffu, b.l, o);
    a.l += x;
    b.l += y;
  }
}
__device__ __forceinline__ void merge_lanes3(MaxSum& a, MaxSum& b, MaxSum& c, float c2) {
  const float ma = lanes_max(a.m), mb = lanes_max(b.m), mc = lanes_max(c.m);
  a = {ma, a.l * ex2((a.m - ma) * c2)};
  b = {mb, b.l * ex2((b.m - mb) * c2)};
  c = {mc, c.l * ex2((c.m - mc) * c2)};
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const float x = __shfl_xor_sync(0xffffffffu, a.l, o), y = __shfl_xor_sync(0xffffffffu, b.l, o), z = __shfl_xor_sync(0xffffffffu, c.l, o);
    a.l += x;
    b.l += y;
    c.l += z;
  }
}

// With P of the teacher's mass and Q of the student's on the named classes: log p_t - log q_t (base 2, times kDown), and A q_t - p_t, from the masses
// that are small.  Where both lie almost wholly on the other classes the loss is what is left of two logarithms near 0.
// log q_t comes from logarithms, and the others' exponentials are relative to the largest of the others: a named class 90 tau ahead
// takes their mass out of fp32, not the loss nor their gradient (A q_t - p_t times their shares of q_t).
__device__ __forceinline__ float log_rest(float pt, MaxSum others, MaxSum all, float c2, float P, float Q) {
  if (P < 0.5f && Q < 0.5f) return (log1pf(-P) - log1pf(-Q)) * (kLog2e * kDown);
  return kDown * log2f(pt) - fmaf(others.m - all.m, c2 * kDown, kDown * (log2f(others.l) - log2f(all.l)));
}
__device__ __forceinline__ float excess_rest(float A, float pt, float qt, float P, float Q) {
  return pt > 0.f ? (P < 0.5f && Q < 0.5f ? P - Q : fmaf(A, qt, -pt)) : A * qt;
}

// Launchers of a kernel for rows of one kind; *taken: the shape is one of its own
template <class T, int VEC, int MODE>
cudaError_t launch_ring(const Distill& p, int64_t rows, cudaStream_t s, bool* taken);      // fw_distill_ring.cu
template <class T, int VEC, int MODE>
cudaError_t launch_warp(const Distill& p, int64_t rows, cudaStream_t s, bool* taken);      // fw_distill_warp.cu

}  // namespace distill
}  // namespace fw
#endif
