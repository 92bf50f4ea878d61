// Log-probabilities of given classes with their gradient, and the clipped policy loss made from them.
//
//   z = Z / tau, q = softmax(z)      logp = z_id - log sum exp z      dZ_j = dlogp / tau ([j = id] - q_j)
//   r = exp(logp - old), k = ref - logp
//   loss = w [-min(r A, clip(r) A) + kl (exp(k) - 1 - k)]    dlogp = w [-(r A if it is the smaller) - kl (exp(k) - 1)]
//
// The classes other than id are summed by themselves: dZ_id = dlogp / tau (sum of the others) / (sum of all), not 1 - q_id, and logp
// = -log(1 + others / own) where a class has most of the mass.
//
// HBM bandwidth bounds it: a row is read once and its gradient written once.  4096 x 131072 bf16: log-probabilities 181-188 us (5.7-5.9 TB/s),
// gradient from statistics 329 (6.5), loss and gradient in one pass, an eighth of the rows out, 383-417 (4.8-5.3, the exponentials twice).
#include <cstdio>
#include <type_traits>

#include "fw_logprob.cuh"

namespace fw {
namespace {

using namespace logprob;

// Sums of the groups t, t + width ... of a row, U at a time
template <class T, int U, bool LONG>
__device__ __forceinline__ MaxSum sums_of(const Place<T>& z, int id, int t, int width, float c2) {
  MaxSum s = {kLow, 0.f};
  int g = t;
  auto take = [&](auto whole) {
    uint4 raw[U];
    bool any = false;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      raw[u] = make_uint4(Group<T>::kNone, Group<T>::kNone, Group<T>::kNone, Group<T>::kNone);
      if (whole.value || g + u * width < z.groups) raw[u] = *z.at(g + u * width);
      any |= z.special(g + u * width);
    }
    if (any) {
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (z.special(g + u * width)) raw[u] = z.others(raw[u], g + u * width, id);
    }
    s = add_groups<T, U>(s, raw, c2);
    g += width * U;
  };
  if (LONG)
    while (g - t + U * width <= z.groups) take(std::true_type());
  while (g - t < z.groups) take(std::false_type());
  return s;
}
// Their gradient
template <class T, bool SAME, int U>
__device__ __forceinline__ void gradient_of(const Logprob& p, const Place<T>& z, int64_t row, int id, int t, int width, float c2, const Scale& s) {
  constexpr int VEC = Group<T>::VEC;
  T* out = static_cast<T*>(p.dZ) + row * p.lddz;
  uint4* d = reinterpret_cast<uint4*>(reinterpret_cast<uintptr_t>(out) & ~(uintptr_t)15);
  if (s.zero) {
    for (int g = t; g < z.groups; g += width) {
      if (SAME && !z.edge(g)) d[g] = make_uint4(0, 0, 0, 0);
      else put_singly<T>(z, g, make_uint4(0, 0, 0, 0), s, c2, out);
    }
    return;
  }
  for (int g = t; g < z.groups; g += width * U) {
    uint4 raw[U];
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (g + u * width < z.groups) raw[u] = *z.at(g + u * width);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int at = g + u * width;
      if (SAME) {
        float v[VEC];
        slopes<T, VEC>(raw[u], s, c2, v);
        if (at < z.groups && !z.edge(at)) d[at] = Group<T>::close(v);
      }
    }
    bool any = !SAME;
#pragma unroll
    for (int u = 0; u < U; ++u) any |= z.edge(g + u * width);
    if (any) {
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (g + u * width < z.groups && (!SAME || z.edge(g + u * width))) put_singly<T>(z, g + u * width, raw[u], s, c2, out);
    }
  }
  if (z.own % width == t) put(out + id, s.own);             // over what this thread has put there
}

// A CTA takes a row, its last warp the row's numbers.  SAME: Z and dZ lie equally past 16 bytes in every row.
template <class T, int MODE, bool SAME, int TH>
__global__ void __launch_bounds__(TH, 1024 / TH) logprob_kernel(const Logprob p) {
  constexpr int nw = TH / 32 - 1, width = TH - 32;
  __shared__ MaxSum red[2 * 32];
  __shared__ Scale scale[2];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, t = threadIdx.x, unit = blockIdx.x, units = gridDim.x;
  const float c2 = p.inv_tau * kLog2e;
  dep_wait();
  if (warp == nw) {
    numbers<T, MODE>(p, unit, units, TH, nw, red, scale, true, [](MaxSum s, int) { return s; });
  } else {
    int64_t later = row_at(0, unit, units);
    int next = id_of<MODE>(p, later), n = 0;
    for (int it = 0; (int64_t)it * units < p.rows; ++it) {
      const int id = next;
      const int64_t row = later;
      later = row_at(it + 1, unit, units);
      next = id_of<MODE>(p, later);
      if (row >= p.rows) continue;                           // (in the last turn)
      const Place<T> z(p.Z, row, p.ldz, p.V, id);
      Scale s = {0.f, 0.f, 0.f, 1};
      if (id >= 0) {
        if (MODE != LP_BACKWARD) {
          const MaxSum sum = merge_lanes(sums_of<T, 6, true>(z, id, t, width, c2), c2);
          if (MODE == LP_FORWARD && n >= 2) meet<BAR_READ>(n, TH);
          if (lane == 0) red[(n & 1) * 32 + warp] = sum;
          tell<BAR_SUMS>(n, TH);
        }
        if (MODE != LP_FORWARD) {
          meet<BAR_SCALE>(n, TH);
          s = scale[n & 1];
          if (MODE == LP_BACKWARD) tell<BAR_READ>(n, TH);
        }
        ++n;
      }
      if (MODE != LP_FORWARD) gradient_of<T, SAME, 4>(p, z, row, id, t, width, c2, s);
    }
    if (MODE == LP_FORWARD)                                  // what the last warp has told is taken in
      for (int k = n > 2 ? n - 2 : 0; k < n; ++k) meet<BAR_READ>(k, TH);
  }
  dep_trigger();
}

// A warp takes `batch` rows: their sums one after the other, their numbers a lane each, their gradients one after the other (the rows come
// from L1 or L2 then).
template <class T, int MODE, bool SAME>
__global__ void __launch_bounds__(128, 8) logprob_warp_kernel(const Logprob p, int batch) {
  const int lane = threadIdx.x & 31, unit = (int)blockIdx.x * 4 + (threadIdx.x >> 5), units = (int)gridDim.x * 4;
  const float c2 = p.inv_tau * kLog2e;
  dep_wait();
  const int64_t none = p.rows;
  auto mine = [&](int it) { return lane < batch ? row_at(it + lane, unit, units) : none; };
  int64_t row = mine(0);
  Head next = head_of<T, MODE>(p, row);
  for (int it = 0; (int64_t)it * units < p.rows; it += batch) {
    const Head h = next;
    const int64_t later = mine(it + batch);
    next = head_of<T, MODE>(p, later);
    Row r = {0.f, 0.f, 0.f, 0.f, true};
    if (MODE == LP_BACKWARD) {
      if (h.id >= 0) r = row_of_stat(h, c2);
    } else {
      MaxSum s = {kLow, 0.f};
      for (int i = 0; i < batch; ++i) {
        const int id = __shfl_sync(0xffffffffu, h.id, i);
        const int64_t at = __shfl_sync(0xffffffffu, row, i);
        if (id < 0) continue;
        const MaxSum sum = merge_lanes(sums_of<T, 4, false>(Place<T>(p.Z, at, p.ldz, p.V, id), id, lane, 32, c2), c2);
        if (lane == i) s = sum;
      }
      if (h.id >= 0) r = row_of(s, h.z, c2, p.inv_tau);
    }
    float dlogp = 0.f;
    if (row < p.rows) dlogp = finish<MODE>(p, row, h, r, true);
    if (MODE != LP_FORWARD) {
      const Scale s = scale_of(r, h.id >= 0 ? dlogp : 0.f, p.inv_tau);
      for (int i = 0; i < batch; ++i) {
        const int id = __shfl_sync(0xffffffffu, h.id, i);
        const int64_t at = __shfl_sync(0xffffffffu, row, i);
        const Scale si = {__shfl_sync(0xffffffffu, s.m, i), __shfl_sync(0xffffffffu, s.f, i), __shfl_sync(0xffffffffu, s.own, i),
                          __shfl_sync(0xffffffffu, s.zero, i)};
        if (at < p.rows) gradient_of<T, SAME, 4>(p, Place<T>(p.Z, at, p.ldz, p.V, id), at, id, lane, 32, c2, si);
      }
    }
    row = later;
  }
  dep_trigger();
}

fw_status desc_check(const fw_logprob_desc* d) {
  if (!d) return FW_ERR_INVALID_ARG;
  if (d->V < 1 || d->V > kMaxV) return FW_ERR_SHAPE;
  if (d->z_dtype != FW_F32 && d->z_dtype != FW_BF16) return FW_ERR_INVALID_ARG;
  if (d->index_bits != 32 && d->index_bits != 64) return FW_ERR_INVALID_ARG;
  if (!(d->tau >= 1e-6f && d->tau <= 1e6f)) return FW_ERR_INVALID_ARG;
  return FW_OK;
}

// Rows of up to 8 KB by a warp (8192 x 1000 bf16, loss and gradient, 11.4 us; by CTAs 55.9).
constexpr int kWarpGroups = 512, kWarpRows = 8;

template <class T, int MODE, bool SAME, int TH>
cudaError_t launch_ctas(const Logprob& p, cudaStream_t s) {
  const int64_t most = (int64_t)(1024 / TH) * sm_count(), turns = (p.rows + most - 1) / most;
  // of the gradient alone no more CTAs than take equal turns (2451 x 50257 bf16 84.5 us against 87; the sums would be slower: 57 against 51)
  const int64_t ctas = MODE == LP_BACKWARD ? (p.rows + turns - 1) / turns : most;
  return launch_dep(logprob_kernel<T, MODE, SAME, TH>, (unsigned)(p.rows < ctas ? p.rows : ctas), TH, 0, s, p);
}
template <class T, int MODE, bool SAME>
cudaError_t launch(const Logprob& p, cudaStream_t s) {
  if (p.V <= kWarpGroups * Group<T>::VEC) {
    const int64_t want = (p.rows + 3) / 4, most = 8 * (int64_t)sm_count(), ctas = want < most ? want : most;
    const int64_t each = (p.rows + ctas * 4 - 1) / (ctas * 4);                // rows of a warp
    return launch_dep(logprob_warp_kernel<T, MODE, SAME>, (unsigned)ctas, 128, 0, s, p, (int)(each < kWarpRows ? each : kWarpRows));
  }
  // the gradient alone: long rows by large CTAs (131072 bf16 329 us, by four of 256 threads a SM 353), others by small ones (8000 fp32 43
  // against 58)
  if constexpr (MODE == LP_BACKWARD)
    if ((int64_t)p.V * (int)sizeof(T) > 128 * 1024) return launch_ctas<T, MODE, SAME, 1024>(p, s);
  return launch_ctas<T, MODE, SAME, 256>(p, s);
}
template <class T, int MODE>
cudaError_t launch_mode(const Logprob& p, cudaStream_t s) {
  if constexpr (MODE == LP_FORWARD) {
    return launch<T, MODE, true>(p, s);
  } else {
    const bool same = ((reinterpret_cast<uintptr_t>(p.Z) ^ reinterpret_cast<uintptr_t>(p.dZ)) & 15) == 0 && ((p.ldz - p.lddz) * (int64_t)sizeof(T)) % 16 == 0;
    if (MODE == LP_BOTH && same && p.V > kWarpGroups * Group<T>::VEC) {
      bool taken = false;
      const cudaError_t e = launch_resident<T>(p, s, &taken);
      if (taken) return e;
    }
    return same ? launch<T, MODE, true>(p, s) : launch<T, MODE, false>(p, s);
  }
}
template <class T>
cudaError_t launch_type(const Logprob& p, int mode, cudaStream_t s) {
  if (mode == LP_FORWARD) return launch_mode<T, LP_FORWARD>(p, s);
  if (mode == LP_BOTH) return launch_mode<T, LP_BOTH>(p, s);
  return launch_mode<T, LP_BACKWARD>(p, s);
}

struct Range { const void* p; uint64_t n; };

// Checks what all calls share, then launches.
fw_status run(const fw_logprob_desc* d, Logprob p, int mode, cudaStream_t s, const char* where) {
  const int es = d->z_dtype == FW_F32 ? 4 : 2, is = d->index_bits / 8;
  if (!p.Z || !p.id) return FW_ERR_INVALID_ARG;
  if (p.rows < 1 || p.rows >= (1 << 28) || p.ldz < d->V || p.ldz > ((int64_t)1 << 30)) return FW_ERR_SHAPE;
  if (p.dZ && (p.lddz < d->V || p.lddz > ((int64_t)1 << 30))) return FW_ERR_SHAPE;
  if (!aligned_to(p.Z, es) || !aligned_to(p.dZ, es) || !aligned_to(p.id, is)) return FW_ERR_INVALID_ARG;
  const uint64_t nz = matrix_span(p.rows, d->V, p.ldz, es), nd = p.dZ ? matrix_span(p.rows, d->V, p.lddz, es) : 0, nr = (uint64_t)p.rows * 4;
  const Range in[] = {{p.id, (uint64_t)p.rows * is}, {p.stat_in, 2 * nr}, {p.dlogp_in, nr}, {p.logp_old, nr}, {p.logp_ref, nr}, {p.adv, nr},
                      {p.weight, nr}, {p.Z, nz}};
  const Range out[] = {{p.dZ, nd}, {p.logp, nr}, {p.stat, 2 * nr}, {p.loss, nr}, {p.dlogp, nr}};
  for (const Range& r : in)
    if (r.p != p.Z && r.p != p.id && !aligned_to(r.p, 4)) return FW_ERR_INVALID_ARG;
  for (int i = 0; i < 5; ++i) {
    if (i > 0 && !aligned_to(out[i].p, 4)) return FW_ERR_INVALID_ARG;
    for (const Range& r : in)
      if (overlap(out[i].p, out[i].n, r.p, r.n) && !(i == 0 && r.p == p.Z && p.dZ == p.Z && p.lddz == p.ldz)) return FW_ERR_INVALID_ARG;
    for (int j = 0; j < i; ++j)
      if (overlap(out[i].p, out[i].n, out[j].p, out[j].n)) return FW_ERR_INVALID_ARG;
  }
  if (p.kl == 0.f) p.logp_ref = nullptr;                     // the term is off: exp(k) may be infinite, and 0 times that is NaN
  p.V = d->V; p.i64 = d->index_bits == 64; p.inv_tau = 1.f / d->tau;
  ProfScope ps(FW_PROF_MISC, s);
  const cudaError_t e = d->z_dtype == FW_F32 ? launch_type<float>(p, mode, s) : launch_type<__nv_bfloat16>(p, mode, s);
  if (e == cudaSuccess) return FW_OK;
  fprintf(stderr, "[fw] %s: %s\n", where, cudaGetErrorString(e));
  return FW_ERR_CUDA;
}

}  // namespace
}  // namespace fw

using namespace fw;

extern "C" {

void fw_logprob_desc_default(fw_logprob_desc* d, int32_t V) {
  if (!d) return;
  d->V = V; d->z_dtype = FW_BF16; d->index_bits = 32; d->tau = 1.f;
}

fw_status fw_logprob_forward(const fw_logprob_desc* d, const void* Z, int64_t rows, int64_t ldz, const void* id, float* logp, float* stat,
                             void* cuda_stream) {
  const fw_status st = desc_check(d);
  if (st != FW_OK) return st;
  if (!logp) return FW_ERR_INVALID_ARG;
  Logprob p = {};
  p.Z = Z; p.rows = rows; p.ldz = ldz; p.id = id; p.logp = logp; p.stat = stat;
  return run(d, p, LP_FORWARD, (cudaStream_t)cuda_stream, "fw_logprob_forward");
}

fw_status fw_logprob_backward(const fw_logprob_desc* d, const void* Z, int64_t rows, int64_t ldz, const void* id, const float* stat,
                              const float* dlogp, void* dZ, int64_t lddz, void* cuda_stream) {
  const fw_status st = desc_check(d);
  if (st != FW_OK) return st;
  if (!stat || !dlogp || !dZ) return FW_ERR_INVALID_ARG;
  Logprob p = {};
  p.Z = Z; p.rows = rows; p.ldz = ldz; p.id = id; p.stat_in = stat; p.dlogp_in = dlogp; p.dZ = dZ; p.lddz = lddz;
  return run(d, p, LP_BACKWARD, (cudaStream_t)cuda_stream, "fw_logprob_backward");
}

void fw_policy_desc_default(fw_policy_desc* p) {
  if (!p) return;
  p->clip_low = 0.2f; p->clip_high = 0.2f; p->kl = 0.f;
}

fw_status fw_policy_forward(const fw_logprob_desc* d, const fw_policy_desc* o, const void* Z, int64_t rows, int64_t ldz, const void* id,
                            const float* logp_old, const float* logp_ref, const float* adv, const float* weight, float* loss, float* logp,
                            float* stat, float* dlogp, void* dZ, int64_t lddz, void* cuda_stream) {
  const fw_status st = desc_check(d);
  if (st != FW_OK) return st;
  if (!o || !(o->clip_low >= 0.f && o->clip_low < 1.f) || !(o->clip_high >= 0.f) || !(o->kl >= -3e38f && o->kl <= 3e38f)) return FW_ERR_INVALID_ARG;
  if (!logp_old || !adv || !loss || (!logp_ref && o->kl != 0.f)) return FW_ERR_INVALID_ARG;
  Logprob p = {};
  p.Z = Z; p.rows = rows; p.ldz = ldz; p.id = id; p.logp_old = logp_old; p.logp_ref = logp_ref; p.adv = adv; p.weight = weight;
  p.loss = loss; p.logp = logp; p.stat = stat; p.dlogp = dlogp; p.dZ = dZ; p.lddz = lddz;
  p.low = 1.f - o->clip_low; p.high = 1.f + o->clip_high; p.kl = o->kl;
  return run(d, p, dZ ? LP_BOTH : LP_FORWARD, (cudaStream_t)cuda_stream, "fw_policy_forward");
}

}  // extern "C"
