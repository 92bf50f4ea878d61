// Log-probabilities of given classes with their gradient, and the clipped policy loss made from them.
//
//   z = Z / tau, q = softmax(z)      logp = z_id - log sum exp z      dZ_j = dlogp / tau ([j = id] - q_j)
//   r = exp(logp - old), k = ref - logp
//   loss = w [-min(r A, clip(r) A) + kl (exp(k) - 1 - k)]    dlogp = w [-(r A if it is the smaller) - kl (exp(k) - 1)]
//
// The classes other than id are summed by themselves: dZ_id = dlogp / tau (sum of the others) / (sum of all), not 1 - q_id, and logp
// = -log(1 + others / own) where a class has most of the mass.
//
// HBM bandwidth bounds it: a row is read once and its gradient written once.
#include <cstdio>

#include "fw_logprob.cuh"

namespace fw {
namespace {

using namespace logprob;

// The 16 bytes of a row that begin `first` elements after its start (before it where rows are not aligned); elements that are not the
// row's read as -inf
template <class T> struct Group;
template <> struct Group<float> {
  static constexpr int VEC = 4;
  static __device__ __forceinline__ uint4 none() { return make_uint4(0xff800000u, 0xff800000u, 0xff800000u, 0xff800000u); }
  static __device__ __forceinline__ void open(uint4 q, float (&v)[4]) {
    v[0] = __uint_as_float(q.x); v[1] = __uint_as_float(q.y); v[2] = __uint_as_float(q.z); v[3] = __uint_as_float(q.w);
  }
  static __device__ __forceinline__ uint4 close(const float (&v)[4]) {
    return make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
  }
};
template <> struct Group<__nv_bfloat16> {
  static constexpr int VEC = 8;
  static __device__ __forceinline__ uint4 none() { return make_uint4(0xff80ff80u, 0xff80ff80u, 0xff80ff80u, 0xff80ff80u); }
  static __device__ __forceinline__ void open(uint4 q, float (&v)[8]) {
    v[0] = bf16_lo(q.x); v[1] = bf16_hi(q.x); v[2] = bf16_lo(q.y); v[3] = bf16_hi(q.y);
    v[4] = bf16_lo(q.z); v[5] = bf16_hi(q.z); v[6] = bf16_lo(q.w); v[7] = bf16_hi(q.w);
  }
  static __device__ __forceinline__ uint4 close(const float (&v)[8]) {
    return make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7]));
  }
};

// A row's place: its groups of 16 aligned bytes, of which the first and the last may be shared with other rows
template <class T>
struct Place {
  static constexpr int VEC = Group<T>::VEC;
  uintptr_t base;                                            // of the first group
  int shift, groups;                                         // elements before the row in it
  __device__ __forceinline__ Place(const void* matrix, int64_t row, int64_t ld, int V) {
    const uintptr_t a = reinterpret_cast<uintptr_t>(matrix) + (uint64_t)row * (uint64_t)ld * sizeof(T);
    base = a & ~(uintptr_t)15;
    shift = (int)(a & 15) / (int)sizeof(T);
    groups = (V + shift + VEC - 1) / VEC;
  }
  __device__ __forceinline__ const uint4* at(int g) const { return reinterpret_cast<const uint4*>(base) + g; }
  __device__ __forceinline__ int first(int g) const { return g * VEC - shift; }        // the group's first element
};

// Group g's values, -inf in the place of elements that are not the row's
template <class T, int VEC>
__device__ __forceinline__ void values(const Place<T>& r, uint4 raw, int g, int V, float (&v)[VEC]) {
  Group<T>::open(raw, v);
  const int c = r.first(g);
  if (c < 0 || c + VEC > V) {
#pragma unroll
    for (int e = 0; e < VEC; ++e)
      if (c + e < 0 || c + e >= V) v[e] = -INFINITY;
  }
}

// WARP: a warp takes a row, else a CTA.  SAME: Z and dZ lie equally past 16 bytes in every row.
template <class T, int MODE, bool WARP, bool SAME>
__global__ void __launch_bounds__(512) logprob_kernel(const Logprob p) {
  constexpr int VEC = Group<T>::VEC, U = 4;
  __shared__ MaxSum red[2][16];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, nw = blockDim.x >> 5;
  const int width = WARP ? 32 : blockDim.x, t = WARP ? lane : threadIdx.x;
  const int64_t first = WARP ? (int64_t)blockIdx.x * nw + warp : blockIdx.x, step = WARP ? (int64_t)gridDim.x * nw : gridDim.x;
  const float c2 = p.inv_tau * kLog2e;
  dep_wait();
  Head next = head_of<T, MODE>(p, first);
  int flip = 0;
  for (int64_t row = first; row < p.rows; row += step) {
    const Head h = next;
    next = head_of<T, MODE>(p, row + step);
    // where dZ is Z: the logit of a row's class has been read by all before it is written over
    if (MODE == LP_BACKWARD) { if (WARP) __syncwarp(); else __syncthreads(); }
    const Place<T> z(p.Z, row, p.ldz, p.V);
    Row r = {0.f, 0.f, 0.f, 0.f, true};
    float dlogp = 0.f;
    if (h.id >= 0) {
      if (MODE == LP_BACKWARD) {
        const float e = h.z == -INFINITY ? 0.f : ex2((h.z - h.b) * c2);
        r = {h.b, h.c, h.c + e, 0.f, h.c + e == 0.f};
        dlogp = h.a;
      } else {
        MaxSum s = {kLow, 0.f};
        for (int g0 = t; g0 < z.groups; g0 += width * U) {
          uint4 raw[U];
#pragma unroll
          for (int u = 0; u < U; ++u) raw[u] = g0 + u * width < z.groups ? *z.at(g0 + u * width) : Group<T>::none();
          float v[U][VEC], m = s.m;
#pragma unroll
          for (int u = 0; u < U; ++u) {
            values<T, VEC>(z, raw[u], g0 + u * width, p.V, v[u]);
            const int k = h.id - z.first(g0 + u * width);
            if ((unsigned)k < (unsigned)VEC) {
#pragma unroll
              for (int e = 0; e < VEC; ++e)
                if (e == k) v[u][e] = -INFINITY;
            }
#pragma unroll
            for (int e = 0; e < VEC; ++e) m = fmaxf(m, v[u][e]);
          }
          float l[2] = {s.l * ex2((s.m - m) * c2), 0.f};
#pragma unroll
          for (int u = 0; u < U; ++u)
#pragma unroll
            for (int e = 0; e < VEC; ++e) l[e & 1] += ex2((v[u][e] - m) * c2);
          s = {m, l[0] + l[1]};
        }
        s = merge_lanes(s, c2);
        if (!WARP) {
          if (lane == 0) red[flip][warp] = s;
          __syncthreads();
          s = lane < nw ? red[flip][lane] : MaxSum{kLow, 0.f};
          s = merge_lanes(s, c2);
          flip ^= 1;                                         // (rows that do not count have no barrier)
        }
        r = row_of(s, h.z, c2, p.inv_tau);
      }
    }
    if (MODE != LP_BACKWARD) {
      Slope sl = {0.f, 0.f};
      if (p.loss && !r.empty) sl = policy_of(p, h, r.logp);
      dlogp = sl.dlogp;
      if (t == 0) {
        if (p.logp) p.logp[row] = r.empty ? 0.f : r.logp;
        if (p.stat) {
          p.stat[2 * row] = r.empty ? 0.f : r.m;
          p.stat[2 * row + 1] = r.empty ? 0.f : r.others;
        }
        if (p.loss) p.loss[row] = sl.loss;
        if (p.dlogp) p.dlogp[row] = sl.dlogp;
      }
    }
    if (MODE != LP_FORWARD) {
      const float coef = r.empty ? 0.f : dlogp * p.inv_tau, inv = 1.f / r.all, f = -coef * inv, own = coef * (r.others * inv);
      const bool zero = r.empty || coef == 0.f;
      T* out = static_cast<T*>(p.dZ) + row * p.lddz;
      const Place<T> d(p.dZ, row, p.lddz, p.V);
      for (int g0 = t; g0 < z.groups; g0 += width * U) {
        uint4 raw[U];
        if (!zero) {
#pragma unroll
          for (int u = 0; u < U; ++u) raw[u] = g0 + u * width < z.groups ? *z.at(g0 + u * width) : Group<T>::none();
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int g = g0 + u * width, c = z.first(g), k = h.id - c;
          if (g >= z.groups) break;
          float v[VEC];
          if (zero) {
#pragma unroll
            for (int e = 0; e < VEC; ++e) v[e] = 0.f;
          } else {
            Group<T>::open(raw[u], v);
#pragma unroll
            for (int e = 0; e < VEC; ++e) v[e] = f * ex2((v[e] - r.m) * c2);
            if ((unsigned)k < (unsigned)VEC) {
#pragma unroll
              for (int e = 0; e < VEC; ++e)
                if (e == k) v[e] = own;
            }
          }
          if (SAME && c >= 0 && c + VEC <= p.V) {
            *const_cast<uint4*>(d.at(g)) = Group<T>::close(v);
          } else {
#pragma unroll
            for (int e = 0; e < VEC; ++e)
              if (c + e >= 0 && c + e < p.V) put(out + c + e, v[e]);
          }
        }
      }
    }
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

template <class T, int MODE, bool WARP, bool SAME>
cudaError_t launch(const Logprob& p, cudaStream_t s) {
  const int threads = WARP ? 128 : 512, per = WARP ? threads / 32 : 1;
  const int64_t want = (p.rows + per - 1) / per, most = (int64_t)(WARP ? 16 : 3) * sm_count();
  return launch_dep(logprob_kernel<T, MODE, WARP, SAME>, (unsigned)(want < most ? want : most), threads, 0, s, p);
}
template <class T, int MODE>
cudaError_t launch_mode(const Logprob& p, cudaStream_t s) {
  const bool same = MODE == LP_FORWARD || (((reinterpret_cast<uintptr_t>(p.Z) ^ reinterpret_cast<uintptr_t>(p.dZ)) & 15) == 0 &&
                                           ((p.ldz - p.lddz) * (int64_t)sizeof(T)) % 16 == 0);
  const bool warp = p.V <= 4096;
  if (MODE == LP_FORWARD || same) return warp ? launch<T, MODE, true, true>(p, s) : launch<T, MODE, false, true>(p, s);
  return warp ? launch<T, MODE, true, false>(p, s) : launch<T, MODE, false, false>(p, s);
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
