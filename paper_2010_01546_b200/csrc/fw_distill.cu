// Distillation loss against a teacher's top logits, with its gradient.
//
// z = Z / tau, q = softmax(z).  The teacher names K classes i_k of a row with logits t_k: p = softmax(t / tau) over them, or, where
// t_lse gives its whole normaliser, p_k = exp(t_k / tau - t_lse) and p_t = 1 - sum p for all classes it does not name, with
// q_t the student's mass on those.
//
//   loss = w [sum_k p_k (log p_k - log q_ik) + p_t (log p_t - log q_t)]
//   dZ_j = w / tau (A q_j - p_j)            named classes,  A = sum p + p_t
//        = w / tau (A q_t - p_t) q_j / q_t  the others
//
// The mass of the others is summed by itself, never as 1 - sum of the named: a trained student leaves little there.
//
// One pass: a row (2 to 4 bytes a class, read once) stays in the registers of a CTA, or of a cluster where it is long, as
// exponentials relative to each thread's own largest logit; the sums go through shared memory of the cluster; then the
// gradient is written.  HBM bandwidth bounds long rows.
//
//   distill_warp_kernel  rows of up to 2048 classes (a classifier's) and 128 entries: a warp a row
//   distill_ring_kernel  long aligned rows of up to 256 entries: resident clusters walk the rows, two rows ahead of themselves
//   distill_kernel       everything else: a CTA or cluster a row; rows beyond what a cluster holds are read twice
#include <cstdio>

#include <cooperative_groups.h>

#include "fw_distill.cuh"

namespace fw {
namespace {

using namespace distill;

// VEC classes an access, NV accesses a thread and trip.  KEEP: the CTA's slice is one trip, its exponentials stay in registers.
template <class T, int VEC, int NV, int MODE, bool KEEP>
__global__ void __launch_bounds__(512, 2) distill_kernel(const Distill p) {
  namespace cg = cooperative_groups;
  extern __shared__ uint32_t dyn[];
  __shared__ float red_m[16], red_l[16], red_p[16], red_x[16];
  __shared__ MaxSum cta_sum;                 // of this CTA's slice, without the named classes
  const int tid = threadIdx.x, nt = blockDim.x, warp = tid >> 5, lane = tid & 31, nw = nt >> 5;
  cg::cluster_group cluster = cg::this_cluster();
  const int C = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
  const int64_t row = blockIdx.x / C;
  // shared: bit set of the slice's named classes, then class, teacher's and student's logit of each entry
  const int words = (p.slice + 31) >> 5;
  uint32_t* bits = dyn;
  int* cls = reinterpret_cast<int*>(dyn + words);
  float* tv = reinterpret_cast<float*>(cls + p.K);
  float* zv = tv + p.K;
  const float c2 = p.inv_tau * kLog2e;
  const int first = rank * p.slice, last = min(p.V, first + p.slice);
  dep_sync();
  const float wt = p.weight ? p.weight[row] : 1.f;
  const T* z = static_cast<const T*>(p.Z) + row * p.ldz;
  T* dz = MODE == DIST_LOSS ? nullptr : static_cast<T*>(p.dZ) + row * p.lddz;
  // the row's sums are formed here, not taken from the forward call (the same decision in all CTAs of the row)
  const bool sums = MODE != DIST_BACKWARD || (wt != 0.f && coarse(p.stat_in[2 * row], p.stat_in[2 * row + 1]));
  if (wt == 0.f) {                            // the row does not count: it is not read (the same decision in all CTAs of the row)
    if (MODE != DIST_LOSS) {
      const float zero[VEC] = {};
      for (int c = first + tid * VEC; c < last; c += nt * VEC) store<VEC>(dz + c, last - c, zero);
    }
    if (MODE != DIST_BACKWARD && rank == 0 && tid == 0) {
      p.loss[row] = 0.f;
      if (p.stat) { p.stat[2 * row] = 0.f; p.stat[2 * row + 1] = 0.f; }
    }
    return;
  }
  for (int i = tid; i < words; i += nt) bits[i] = 0;
  for (int k = tid; k < p.K; k += nt) {
    const int64_t at = row * p.K + k;
    const int64_t i = p.i64 ? static_cast<const int64_t*>(p.I)[at] : static_cast<const int32_t*>(p.I)[at];
    cls[k] = i >= 0 && i < p.V ? (int)i : -1;
    tv[k] = p.t_bf16 ? to_f(static_cast<const __nv_bfloat16*>(p.T)[at]) : static_cast<const float*>(p.T)[at];
  }
  __syncthreads();
  // a class named twice counts once, with its first logit
  bool mine_twice[(kMaxK + 127) / 128];
#pragma unroll
  for (int q = 0; q < (kMaxK + 127) / 128; ++q) {
    const int k = tid + q * nt;
    mine_twice[q] = false;
    if (k < p.K && cls[k] >= 0)
      for (int j = 0; j < k; ++j) mine_twice[q] |= cls[j] == cls[k];
  }
  __syncthreads();
#pragma unroll
  for (int q = 0; q < (kMaxK + 127) / 128; ++q) {
    const int k = tid + q * nt;
    if (k < p.K && mine_twice[q]) cls[k] = -1;
  }
  __syncthreads();
  for (int k = tid; k < p.K; k += nt) {
    const int i = cls[k];
    // without sums those of its slice are enough, and dZ may be Z: another CTA's are being written over
    const bool here = i >= first && i < last;
    zv[k] = (sums ? i >= 0 : here) ? to_f(z[i]) : 0.f;
    if (here) atomicOr(&bits[(i - first) >> 5], 1u << ((i - first) & 31));
  }
  __syncthreads();

  // ---- the slice: largest logit and sum of exponentials of the classes that are not named ----
  float e[NV][VEC];
  MaxSum sum = {kLow, 0.f};
  if (sums) {
    for (int base = first; base < last; base += nt * NV * VEC) {
      MaxSum now = {kLow, 0.f};
#pragma unroll
      for (int k = 0; k < NV; ++k) {
        const int c = base + (k * nt + tid) * VEC;
        load<VEC>(z + c, last - c, -INFINITY, e[k]);
      }
#pragma unroll
      for (int k = 0; k < NV; ++k) {
        const int c = base + (k * nt + tid) * VEC - first;
        uint32_t named = 0;
        if (c + first < last) {
          named = bits[c >> 5] >> (c & 31);
          if (VEC < 32) named &= (1u << VEC) - 1u;
        }
        if (named) {
#pragma unroll
          for (int v = 0; v < VEC; ++v)
            if ((named >> v) & 1u) e[k][v] = -INFINITY;
        }
#pragma unroll
        for (int v = 0; v < VEC; ++v) now.m = fmaxf(now.m, e[k][v]);
      }
#pragma unroll
      for (int k = 0; k < NV; ++k) {
#pragma unroll
        for (int v = 0; v < VEC; ++v) {
          e[k][v] = ex2((e[k][v] - now.m) * c2);
          now.l += e[k][v];
        }
      }
      sum = KEEP ? now : merge(sum, now, c2);
    }
    // lanes, warps, CTAs of the cluster
    const MaxSum s = merge_lanes(sum, c2);
    if (lane == 0) { red_m[warp] = s.m; red_l[warp] = s.l; }
  }
  // ---- the teacher: normaliser, probabilities (every CTA for itself; warps in order) ----
  float tm = kLow;
  for (int k = tid; k < p.K; k += nt)
    if (cls[k] >= 0) tm = fmaxf(tm, tv[k]);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) tm = fmaxf(tm, __shfl_xor_sync(0xffffffffu, tm, o));
  if (lane == 0) red_x[warp] = tm;
  __syncthreads();
  for (int k = 0; k < nw; ++k) tm = fmaxf(tm, red_x[k]);
  // exp(t / tau - normaliser): relative to the largest here, or to the normaliser that the caller has
  const float t_lse = p.t_lse ? p.t_lse[row] : 0.f;
  auto teacher2 = [&](float t) { return p.t_lse ? fmaf(t, p.inv_tau, -t_lse) * kLog2e : (t - tm) * c2; };
  float ts = 0.f;
  for (int k = tid; k < p.K; k += nt)
    if (cls[k] >= 0) ts += ex2(teacher2(tv[k]));
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) ts += __shfl_xor_sync(0xffffffffu, ts, o);
  if (lane == 0) red_p[warp] = ts;
  if (sums && tid == 0) {
    MaxSum s = {red_m[0], red_l[0]};
    for (int k = 1; k < nw; ++k) s = merge(s, {red_m[k], red_l[k]}, c2);
    cta_sum = s;
  }
  if (sums) cluster.sync();
  else __syncthreads();
  ts = 0.f;
  for (int k = 0; k < nw; ++k) ts += red_p[k];
  // whole: the teacher's mass on the named classes; pt: on the others
  const float scale_p = p.t_lse ? 1.f : (ts > 0.f ? 1.f / ts : (ts == 0.f ? 0.f : ts));     // a NaN goes on
  const float whole = ts * scale_p;
  float pt = 0.f;
  if (p.t_lse) pt = 1.f - whole < 0.f ? 0.f : 1.f - whole;
  const float A = whole + pt;

  // ---- the student's normalisers: the others' over the cluster in order, then the named classes ----
  // q_j = exp((z_j - ref) / tau) inv, or, from what the forward call left, exp(z_j / tau - ref)
  float ref, inv, qt, Q = 1.f;                // qt: the mass of the classes that are not named, Q: of those that are (with sums)
  bool empty;                                 // no class has any
  MaxSum all = {kLow, 0.f}, others = {kLow, 0.f};
  if (sums) {
    others = *cluster.map_shared_rank(&cta_sum, 0);
    for (int r = 1; r < C; ++r) others = merge(others, *cluster.map_shared_rank(&cta_sum, r), c2);
    MaxSum n = {kLow, 0.f};
    for (int k = tid; k < p.K; k += nt)
      if (cls[k] >= 0) n = merge(n, {fmaxf(zv[k], kLow), zv[k] == -INFINITY ? 0.f : zv[k] != zv[k] ? zv[k] : 1.f}, c2);
    n = merge_lanes(n, c2);
    __syncthreads();                          // red_m, red_l have been read
    if (lane == 0) { red_m[warp] = n.m; red_l[warp] = n.l; }
    __syncthreads();
    MaxSum named = {red_m[0], red_l[0]};
    for (int k = 1; k < nw; ++k) named = merge(named, {red_m[k], red_l[k]}, c2);
    all = merge(others, named, c2);
    empty = all.l == 0.f;
    ref = all.m;
    inv = 1.f / all.l;
    qt = others.l * ex2((others.m - all.m) * c2) * inv;
    Q = named.l * ex2((named.m - all.m) * c2) * inv;
  } else {
    ref = p.stat_in[2 * row];
    inv = 1.f;
    empty = false;
    qt = ex2((p.stat_in[2 * row + 1] - ref) * kLog2e);
  }
  auto student = [&](float v) { return ex2(sums ? (v - ref) * c2 : fmaf(v, p.inv_tau, -ref) * kLog2e) * inv; };

  // ---- loss ----
  if (MODE != DIST_BACKWARD) {
    float kl = 0.f;
    if (rank == 0) {
      for (int k = tid; k < p.K; k += nt) {
        if (cls[k] < 0) continue;
        const float lp = teacher2(tv[k]), pk = ex2(lp) * scale_p;
        if (pk > 0.f || pk != pk) kl += pk * (kDown * (lp + log2f(scale_p)) - fmaf(zv[k] - all.m, c2 * kDown, -kDown * log2f(all.l)));
      }
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) kl += __shfl_xor_sync(0xffffffffu, kl, o);
      if (lane == 0) red_x[warp] = kl;
      __syncthreads();
      if (tid == 0) {
        kl = 0.f;
        for (int k = 0; k < nw; ++k) kl += red_x[k];
        if (pt > 0.f) kl += pt * log_rest(pt, others, all, c2, whole, Q);
        if (whole != whole) kl = whole;
        p.loss[row] = empty ? 0.f : wt * kl * kUp;
        if (p.stat) {
          p.stat[2 * row] = empty ? -INFINITY : fmaf(all.m, p.inv_tau, logf(all.l));
          p.stat[2 * row + 1] = others.l == 0.f ? -INFINITY : fmaf(others.m, p.inv_tau, logf(others.l));
        }
      }
    }
  }
  // ---- gradient ----
  if (MODE != DIST_LOSS) {
    const float ws = empty ? 0.f : wt * p.inv_tau;
    // (A q_t - p_t) q_j / q_t of the others: the first factor, and q_j / q_t relative to the others' largest or their normaliser
    const float other = ws == 0.f ? 0.f : ws * excess_rest(A, pt, qt, whole, Q);
    const float other_ref = sums ? others.m : p.stat_in[2 * row + 1];
    if (KEEP && sums) {
      const float f = others.l == 0.f ? 0.f : other * ex2((sum.m - others.m) * c2) / others.l;
#pragma unroll
      for (int k = 0; k < NV; ++k) {
        const int c = first + (k * nt + tid) * VEC;
#pragma unroll
        for (int v = 0; v < VEC; ++v) e[k][v] *= f;
        if (c < last) store<VEC>(dz + c, last - c, e[k]);
      }
    } else {
      const float f = !sums ? other : (others.l == 0.f ? 0.f : other / others.l);
      for (int base = first; base < last; base += nt * NV * VEC) {
#pragma unroll
        for (int k = 0; k < NV; ++k) {
          const int c = base + (k * nt + tid) * VEC;
          load<VEC>(z + c, last - c, -INFINITY, e[k]);
        }
#pragma unroll
        for (int k = 0; k < NV; ++k) {
          const int c = base + (k * nt + tid) * VEC;
#pragma unroll
          for (int v = 0; v < VEC; ++v)
            e[k][v] = f == 0.f ? 0.f : f * ex2(sums ? (e[k][v] - other_ref) * c2 : fmaf(e[k][v], p.inv_tau, -other_ref) * kLog2e);
          if (c < last) store<VEC>(dz + c, last - c, e[k]);
        }
      }
    }
    __syncthreads();                          // the named classes are written over, by the same CTA, after its stores
    for (int k = tid; k < p.K; k += nt) {
      const int i = cls[k];
      if (i < first || i >= last) continue;
      put(dz + i, empty ? 0.f : ws * (A * student(zv[k]) - ex2(teacher2(tv[k])) * scale_p));
    }
  }
  if (sums) cluster.sync();                   // no CTA of the cluster leaves while its sum may still be read
}

fw_status desc_check(const fw_distill_desc* d) {
  if (!d) return FW_ERR_INVALID_ARG;
  if (d->V < 1 || d->V > kMaxV || d->K < 1 || d->K > kMaxK || d->K > d->V) return FW_ERR_SHAPE;
  if ((d->z_dtype != FW_F32 && d->z_dtype != FW_BF16) || (d->t_dtype != FW_F32 && d->t_dtype != FW_BF16)) return FW_ERR_INVALID_ARG;
  if (d->index_bits != 32 && d->index_bits != 64) return FW_ERR_INVALID_ARG;
  if (!(d->tau >= 1e-6f && d->tau <= 1e6f)) return FW_ERR_INVALID_ARG;
  return FW_OK;
}

template <class T, int VEC, int NV, int MODE, bool KEEP>
cudaError_t launch(const Distill& p, int C, int threads, int64_t rows, cudaStream_t s) {
  const size_t smem = (size_t)((p.slice + 31) / 32) * 4 + (size_t)p.K * 12;   // below 48 KB: see kMaxV
  return launch_dep_cluster(C, distill_kernel<T, VEC, NV, MODE, KEEP>, dim3((unsigned)(rows * C)), threads, smem, s, p);
}

template <class T, int VEC, int MODE>
cudaError_t launch_mode(Distill p, int64_t rows, cudaStream_t s) {
  bool taken = false;
  cudaError_t e = launch_warp<T, VEC, MODE>(p, rows, s, &taken);
  if (taken) return e;
  if constexpr (VEC > 1) {                                  // rows on 16 bytes
    e = launch_ring<T, VEC, MODE>(p, rows, s, &taken);
    if (taken) return e;
  }
  constexpr int NV = VEC == 1 ? 16 : 32 / VEC;              // 32 classes of a thread in registers (16 single ones)
  constexpr int few = VEC == 1 ? 4 : 1;
  // threads and CTAs of a row: enough that the row is one trip, as far as 8 CTAs of 512 threads go
  const int need = (p.V + VEC * few - 1) / (VEC * few);     // threads at `few` accesses each
  int threads = 128, C = 1;
  if (need > 128) threads = 256;
  const int per_small = threads * few * VEC;
  if (p.V > per_small) {
    threads = 512;
    while (threads > 128 && (threads / 2) * NV * VEC >= p.V) threads /= 2;
    while (C < 8 && C * threads * NV * VEC < p.V) C *= 2;
    const int unit = threads * VEC;
    p.slice = ((p.V + C - 1) / C + unit - 1) / unit * unit;
    if (p.slice <= threads * NV * VEC) return launch<T, VEC, NV, MODE, true>(p, C, threads, rows, s);
    return launch<T, VEC, NV, MODE, false>(p, C, threads, rows, s);
  }
  p.slice = per_small;
  return launch<T, VEC, few, MODE, true>(p, 1, threads, rows, s);
}

template <class T, int VEC>
cudaError_t launch_vec(const Distill& p, int mode, int64_t rows, cudaStream_t s) {
  if (mode == DIST_LOSS) return launch_mode<T, VEC, DIST_LOSS>(p, rows, s);
  if (mode == DIST_BOTH) return launch_mode<T, VEC, DIST_BOTH>(p, rows, s);
  return launch_mode<T, VEC, DIST_BACKWARD>(p, rows, s);
}

fw_status run(const fw_distill_desc* d, const void* Z, int64_t rows, int64_t ldz, const void* T, const void* I, const float* t_lse,
              const float* weight, float* loss, float* stat, const float* stat_in, void* dZ, int64_t lddz, int mode, cudaStream_t s) {
  fw_status st = desc_check(d);
  if (st != FW_OK) return st;
  if (!Z || !T || !I) return FW_ERR_INVALID_ARG;
  if (mode == DIST_BACKWARD ? (!stat_in || !dZ) : !loss) return FW_ERR_INVALID_ARG;
  if (rows < 1 || rows >= (1 << 28) || ldz < d->V || ldz > ((int64_t)1 << 30)) return FW_ERR_SHAPE;
  if (dZ && (lddz < d->V || lddz > ((int64_t)1 << 30))) return FW_ERR_SHAPE;
  const int es = d->z_dtype == FW_F32 ? 4 : 2, ts = d->t_dtype == FW_F32 ? 4 : 2, is = d->index_bits / 8;
  if (!aligned_to(Z, es) || !aligned_to(dZ, es) || !aligned_to(T, ts) || !aligned_to(I, is) || !aligned_to(t_lse, 4) ||
      !aligned_to(weight, 4) || !aligned_to(loss, 4) || !aligned_to(stat, 4) || !aligned_to(stat_in, 4))
    return FW_ERR_INVALID_ARG;
  const uint64_t nz = matrix_span(rows, d->V, ldz, es), nd = dZ ? matrix_span(rows, d->V, lddz, es) : 0;
  const uint64_t nk = (uint64_t)rows * d->K, nr = (uint64_t)rows * 4;
  if (overlap(dZ, nd, Z, nz) && !(dZ == Z && lddz == ldz)) return FW_ERR_INVALID_ARG;
  const void* out[3] = {dZ, loss, stat};
  const uint64_t no[3] = {nd, nr, 2 * nr};
  for (int i = 0; i < 3; ++i) {
    if (overlap(out[i], no[i], T, nk * ts) || overlap(out[i], no[i], I, nk * is) || overlap(out[i], no[i], t_lse, nr) ||
        overlap(out[i], no[i], weight, nr) || overlap(out[i], no[i], stat_in, 2 * nr) || (i > 0 && overlap(out[i], no[i], Z, nz)))
      return FW_ERR_INVALID_ARG;
    for (int j = 0; j < i; ++j)
      if (overlap(out[i], no[i], out[j], no[j])) return FW_ERR_INVALID_ARG;
  }
  Distill p;
  p.Z = Z; p.T = T; p.I = I; p.t_lse = t_lse; p.weight = weight; p.stat_in = stat_in; p.loss = loss; p.stat = stat; p.dZ = dZ;
  p.ldz = ldz; p.lddz = lddz; p.V = d->V; p.K = d->K; p.t_bf16 = d->t_dtype == FW_BF16; p.i64 = d->index_bits == 64;
  p.slice = 0; p.inv_tau = 1.f / d->tau;
  const bool vec = aligned_to(Z, 16) && (ldz * es) % 16 == 0 && (!dZ || (aligned_to(dZ, 16) && (lddz * es) % 16 == 0));
  ProfScope ps(FW_PROF_MISC, s);
  cudaError_t e;
  if (d->z_dtype == FW_F32) e = vec ? launch_vec<float, 4>(p, mode, rows, s) : launch_vec<float, 1>(p, mode, rows, s);
  else e = vec ? launch_vec<__nv_bfloat16, 8>(p, mode, rows, s) : launch_vec<__nv_bfloat16, 1>(p, mode, rows, s);
  if (e == cudaSuccess) return FW_OK;
  fprintf(stderr, "[fw] distillation loss: %s\n", cudaGetErrorString(e));
  return FW_ERR_CUDA;
}

}  // namespace
}  // namespace fw

using namespace fw;

extern "C" {

void fw_distill_desc_default(fw_distill_desc* d, int32_t V, int32_t K) {
  if (!d) return;
  d->V = V; d->K = K; d->z_dtype = FW_BF16; d->t_dtype = FW_BF16; d->index_bits = 32; d->tau = 1.f;
}

fw_status fw_distill_forward(const fw_distill_desc* d, const void* Z, int64_t rows, int64_t ldz, const void* T, const void* I,
                             const float* t_lse, const float* weight, float* loss, float* stat, void* dZ, int64_t lddz,
                             void* cuda_stream) {
  return run(d, Z, rows, ldz, T, I, t_lse, weight, loss, stat, nullptr, dZ, lddz, dZ ? DIST_BOTH : DIST_LOSS, (cudaStream_t)cuda_stream);
}

fw_status fw_distill_backward(const fw_distill_desc* d, const void* Z, int64_t rows, int64_t ldz, const void* T, const void* I,
                              const float* t_lse, const float* weight, const float* stat, void* dZ, int64_t lddz, void* cuda_stream) {
  return run(d, Z, rows, ldz, T, I, t_lse, weight, nullptr, nullptr, stat, dZ, lddz, DIST_BACKWARD, (cudaStream_t)cuda_stream);
}

}  // extern "C"
