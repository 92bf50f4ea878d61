// Distillation loss of short rows (see fw_distill.cu).
#include "fw_distill.cuh"

namespace fw {
namespace distill {
namespace {

// ---------------------------------------------------------------------------
// Short rows (a classifier's): a warp a row, its classes in registers, its entries four to a lane at most, no barrier but the
// warp's own.  With a CTA a row 8192 rows of 1000 classes took 55 us, most of it barriers.
// ---------------------------------------------------------------------------
constexpr int kWarpRows = 4;                // warps of a CTA
constexpr int kWarpMaxV = 2048, kWarpMaxK = 128;

template <class T, int VEC, int NV, int EPL, int MODE>
__global__ void __launch_bounds__(32 * kWarpRows) distill_warp_kernel(const Distill p, int rows) {
  __shared__ uint32_t s_bits[kWarpRows][kWarpMaxV / 32];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int row = (int)blockIdx.x * kWarpRows + warp;
  uint32_t* bits = s_bits[warp];
  dep_sync();
  if (row >= rows) return;
  const float wt = p.weight ? p.weight[row] : 1.f;
  const T* z = static_cast<const T*>(p.Z) + (int64_t)row * p.ldz;
  T* dz = MODE == DIST_LOSS ? nullptr : static_cast<T*>(p.dZ) + (int64_t)row * p.lddz;
  const float c2 = p.inv_tau * kLog2e;
  if (wt == 0.f) {
    if (MODE != DIST_LOSS) {
      const float zero[VEC] = {};
#pragma unroll 4
      for (int c = lane * VEC; c < p.V; c += 32 * VEC) store<VEC>(dz + c, p.V - c, zero);
    }
    if (MODE != DIST_BACKWARD && lane == 0) {
      p.loss[row] = 0.f;
      if (p.stat) { p.stat[2 * (int64_t)row] = 0.f; p.stat[2 * (int64_t)row + 1] = 0.f; }
    }
    return;
  }
  float e[NV][VEC];
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int c = (k * 32 + lane) * VEC;
    load<VEC>(z + c, p.V - c, -INFINITY, e[k]);
  }
  const float s0 = MODE == DIST_BACKWARD ? p.stat_in[2 * (int64_t)row] : 0.f, s1 = MODE == DIST_BACKWARD ? p.stat_in[2 * (int64_t)row + 1] : 0.f;
  if (MODE == DIST_BACKWARD && coarse(s0, s1)) {
    coarse_row<T, VEC, false>(p, row, bits, nullptr);
    return;
  }
  // ---- entries: a class named twice counts once, with its first logit: in the groups of 32 in order, in a group the lowest lane ----
  int cls[EPL];
  float tv[EPL], zv[EPL];
#pragma unroll
  for (int j = 0; j < EPL; ++j) {
    const int k = j * 32 + lane;
    cls[j] = -1;
    tv[j] = 0.f;
    if (k < p.K) {
      const int64_t at = (int64_t)row * p.K + k;
      const int64_t i = p.i64 ? static_cast<const int64_t*>(p.I)[at] : static_cast<const int32_t*>(p.I)[at];
      cls[j] = i >= 0 && i < p.V ? (int)i : -1;
      tv[j] = p.t_bf16 ? to_f(static_cast<const __nv_bfloat16*>(p.T)[at]) : static_cast<const float*>(p.T)[at];
    }
  }
  const float t_lse = p.t_lse ? p.t_lse[row] : 0.f;
  for (int i = lane; i < (p.V + 31) / 32; i += 32) bits[i] = 0;
  __syncwarp();
#pragma unroll
  for (int j = 0; j < EPL; ++j) {
    const unsigned same = __match_any_sync(0xffffffffu, cls[j]);
    bool out = cls[j] < 0 || (int)__ffs(same) - 1 != lane;
    if (!out) out = (atomicOr(&bits[cls[j] >> 5], 1u << (cls[j] & 31)) >> (cls[j] & 31)) & 1u;
    __syncwarp();
    if (out) cls[j] = -1;
    zv[j] = cls[j] >= 0 ? to_f(z[cls[j]]) : 0.f;
  }
  // ---- sums of the classes that are not named, of those that are, of the teacher's ----
  MaxSum sum = {kLow, 0.f}, named = {kLow, 0.f}, t = {kLow, 0.f};
#pragma unroll
  for (int j = 0; j < EPL; ++j) {
    if (cls[j] >= 0) {
      t.m = fmaxf(t.m, tv[j]);
      if (MODE != DIST_BACKWARD) named.m = fmaxf(named.m, zv[j]);
    }
  }
  t.m = lanes_max(t.m);
  auto teacher2 = [&](float v) { return p.t_lse ? fmaf(v, p.inv_tau, -t_lse) * kLog2e : (v - t.m) * c2; };
  MaxSum others = {kLow, 0.f};
  if (MODE != DIST_BACKWARD) {
    named.m = lanes_max(named.m);
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int c = (k * 32 + lane) * VEC;
      const uint32_t is = c < p.V ? (bits[c >> 5] >> (c & 31)) & (VEC < 32 ? (1u << VEC) - 1u : ~0u) : 0u;
#pragma unroll
      for (int v = 0; v < VEC; ++v) {
        if ((is >> v) & 1u) e[k][v] = -INFINITY;
        sum.m = fmaxf(sum.m, e[k][v]);
      }
    }
    sum.m = lanes_max(sum.m);                 // the others' largest: one reference for all lanes
#pragma unroll
    for (int k = 0; k < NV; ++k) {
#pragma unroll
      for (int v = 0; v < VEC; ++v) {
        e[k][v] = ex2((e[k][v] - sum.m) * c2);
        sum.l += e[k][v];
      }
    }
  }
#pragma unroll
  for (int j = 0; j < EPL; ++j) {
    if (cls[j] >= 0) {
      t.l += ex2(teacher2(tv[j]));
      if (MODE != DIST_BACKWARD) named.l += ex2((zv[j] - named.m) * c2);
    }
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    t.l += __shfl_xor_sync(0xffffffffu, t.l, o);
    if (MODE != DIST_BACKWARD) {
      sum.l += __shfl_xor_sync(0xffffffffu, sum.l, o);
      named.l += __shfl_xor_sync(0xffffffffu, named.l, o);
    }
  }
  const float ts = t.l;
  const float scale_p = p.t_lse ? 1.f : (ts > 0.f ? 1.f / ts : (ts == 0.f ? 0.f : ts));       // a NaN goes on
  const float whole = ts * scale_p;
  float pt = 0.f;
  if (p.t_lse) pt = 1.f - whole < 0.f ? 0.f : 1.f - whole;
  const float A = whole + pt;
  float ref, inv, qt, Q = 1.f;
  bool empty;
  MaxSum all = {kLow, 0.f};
  if (MODE != DIST_BACKWARD) {
    others = sum;
    all = merge(others, named, c2);
    empty = all.l == 0.f;
    ref = all.m;
    inv = 1.f / all.l;
    qt = others.l * ex2((others.m - all.m) * c2) * inv;
    Q = named.l * ex2((named.m - all.m) * c2) * inv;
  } else {
    ref = s0;
    inv = 1.f;
    empty = false;
    qt = ex2((s1 - ref) * kLog2e);
  }
  auto student = [&](float v) { return ex2(MODE == DIST_BACKWARD ? fmaf(v, p.inv_tau, -ref) * kLog2e : (v - ref) * c2) * inv; };
  if (MODE != DIST_BACKWARD) {
    float kl = 0.f;
    const float log_all = log2f(all.l), log_p = log2f(scale_p);
#pragma unroll
    for (int j = 0; j < EPL; ++j) {
      if (cls[j] < 0) continue;
      const float lp = teacher2(tv[j]), pk = ex2(lp) * scale_p;
      if (pk > 0.f || pk != pk) kl += pk * (kDown * (lp + log_p) - fmaf(zv[j] - all.m, c2 * kDown, -kDown * log_all));
    }
    kl = lanes_sum(kl);
    if (lane == 0) {
      if (pt > 0.f) kl += pt * log_rest(pt, others, all, c2, whole, Q);
      if (whole != whole) kl = whole;
      p.loss[row] = empty ? 0.f : wt * kl * kUp;
      if (p.stat) {
        p.stat[2 * (int64_t)row] = empty ? -INFINITY : fmaf(all.m, p.inv_tau, logf(all.l));
        p.stat[2 * (int64_t)row + 1] = others.l == 0.f ? -INFINITY : fmaf(others.m, p.inv_tau, logf(others.l));
      }
    }
  }
  if (MODE != DIST_LOSS) {
    const float ws = empty ? 0.f : wt * p.inv_tau;
    const float other = ws == 0.f ? 0.f : ws * excess_rest(A, pt, qt, whole, Q);
    const float f = MODE == DIST_BACKWARD ? other : (others.l == 0.f ? 0.f : other / others.l);
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int c = (k * 32 + lane) * VEC;
      if (c >= p.V) continue;
#pragma unroll
      for (int v = 0; v < VEC; ++v) e[k][v] = MODE != DIST_BACKWARD ? e[k][v] * f : f == 0.f ? 0.f : f * ex2(fmaf(e[k][v], p.inv_tau, -s1) * kLog2e);
      store<VEC>(dz + c, p.V - c, e[k]);
    }
    __syncwarp();                             // the named classes are written over
#pragma unroll
    for (int j = 0; j < EPL; ++j)
      if (cls[j] >= 0) put(dz + cls[j], ws == 0.f ? 0.f : ws * (A * student(zv[j]) - ex2(teacher2(tv[j])) * scale_p));
  }
}

template <class T, int VEC, int NV, int MODE>
cudaError_t launch_few(const Distill& p, int64_t rows, cudaStream_t s) {
  const dim3 grid((unsigned)((rows + kWarpRows - 1) / kWarpRows));
  if (p.K <= 32) return launch_dep(distill_warp_kernel<T, VEC, NV, 1, MODE>, grid, 32 * kWarpRows, 0, s, p, (int)rows);
  return launch_dep(distill_warp_kernel<T, VEC, NV, kWarpMaxK / 32, MODE>, grid, 32 * kWarpRows, 0, s, p, (int)rows);
}
template <class T, int VEC, int MODE>
cudaError_t launch_lanes(const Distill& p, int64_t rows, cudaStream_t s) {
  // accesses a lane: a quarter, half or all of what it can hold
  constexpr int most = VEC == 1 ? 32 : 64 / VEC;
  if (p.V <= 32 * VEC * most / 4) return launch_few<T, VEC, most / 4, MODE>(p, rows, s);
  if (p.V <= 32 * VEC * most / 2) return launch_few<T, VEC, most / 2, MODE>(p, rows, s);
  return launch_few<T, VEC, most, MODE>(p, rows, s);
}

}  // namespace

template <class T, int VEC, int MODE>
cudaError_t launch_warp(const Distill& p, int64_t rows, cudaStream_t s, bool* taken) {
  // its lanes hold the row: up to 64 classes each (32 where rows are not aligned)
  *taken = p.V <= (VEC == 1 ? kWarpMaxV / 2 : kWarpMaxV) && p.K <= kWarpMaxK;
  return *taken ? launch_lanes<T, VEC, MODE>(p, rows, s) : cudaSuccess;
}

template cudaError_t launch_warp<float, 4, DIST_LOSS>(const Distill&, int64_t, cudaStream_t, bool*);
template cudaError_t launch_warp<float, 4, DIST_BOTH>(const Distill&, int64_t, cudaStream_t, bool*);
template cudaError_t launch_warp<float, 4, DIST_BACKWARD>(const Distill&, int64_t, cudaStream_t, bool*);
template cudaError_t launch_warp<float, 1, DIST_LOSS>(const Distill&, int64_t, cudaStream_t, bool*);
template cudaError_t launch_warp<float, 1, DIST_BOTH>(const Distill&, int64_t, cudaStream_t, bool*);
template cudaError_t launch_warp<float, 1, DIST_BACKWARD>(const Distill&, int64_t, cudaStream_t, bool*);
template cudaError_t launch_warp<__nv_bfloat16, 8, DIST_LOSS>(const Distill&, int64_t, cudaStream_t, bool*);
template cudaError_t launch_warp<__nv_bfloat16, 8, DIST_BOTH>(const Distill&, int64_t, cudaStream_t, bool*);
template cudaError_t launch_warp<__nv_bfloat16, 8, DIST_BACKWARD>(const Distill&, int64_t, cudaStream_t, bool*);
template cudaError_t launch_warp<__nv_bfloat16, 1, DIST_LOSS>(const Distill&, int64_t, cudaStream_t, bool*);
template cudaError_t launch_warp<__nv_bfloat16, 1, DIST_BOTH>(const Distill&, int64_t, cudaStream_t, bool*);
template cudaError_t launch_warp<__nv_bfloat16, 1, DIST_BACKWARD>(const Distill&, int64_t, cudaStream_t, bool*);

}  // namespace distill
}  // namespace fw
