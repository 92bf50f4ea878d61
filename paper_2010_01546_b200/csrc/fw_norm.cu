// Residual addition and root-mean-square norm, forward and backward, a row at a time.
//
//   s = x + r, kept in the type of x      n = s / sqrt(mean(s^2) + eps)      y = n w
//   e4m3 y: c = max |y| / 448, y is held as e4m3(y / c) with c beside it
//   du = dy w     dx = (du - n mean(du n)) / sqrt(mean(s^2) + eps) + ds      dw = sum over the rows of dy n
//
// Both directions read each element once and write each result once: HBM bandwidth bounds them.  A row stays in the registers
// of the threads that share it between its sum and its output.
#include <cstdio>
#include <mutex>

#include "fw_internal.h"
#include "fw_rows.cuh"

namespace fw {
namespace {

using namespace rows;

constexpr int kNormMaxM = 16384;
constexpr float kE4m3Max = 448.f;
constexpr float kMinScale = 7.52316385e-37f;   // 2^-120: the reciprocal of a scale stays finite

struct NormFwd {
  const void *x, *res;
  const float* w;
  void *sum, *y;
  float *y_scale, *rstd;
  int64_t rows, ldx, ldr, lds, ldy;
  int32_t M, width;      // width: threads that share a row
  float eps, inv_M;
};

// what s holds of a vector
__device__ __forceinline__ void round_pairs(float (&v)[4], const float*) {}
__device__ __forceinline__ void round_pairs(float (&v)[1], const float*) {}
__device__ __forceinline__ void round_pairs(float (&v)[1], const __nv_bfloat16* p) { v[0] = held(v[0], p); }
__device__ __forceinline__ void round_pairs(float (&v)[8], const __nv_bfloat16*) {
#pragma unroll
  for (int e = 0; e < 8; e += 2) {
    const uint32_t w = pack_bf16(v[e], v[e + 1]);
    v[e] = bf16_lo(w);
    v[e + 1] = bf16_hi(w);
  }
}

// T: type of x, r and s; Y: of y.  VEC elements an access, NV accesses a thread; SLOTS rows of a CTA on their way.
// A CTA walks the rows, one at a time.  With a CTA launched for each row its loads waited for nothing but the sums, the largest
// value and the stores of the rows before it: 8192 x 4096 bf16 to e4m3 71.5 us.
template <class T, class Y, int VEC, int NV, int SLOTS, bool RES, int FILL>
__global__ void __launch_bounds__(512) norm_forward_kernel(const NormFwd p) {
  typedef Ahead<T, VEC, NV, FILL> Ring;
  extern __shared__ __align__(16) uint8_t room[];            // [slot][x, res]
  __shared__ float buf[2][2][16];
  const int t = threadIdx.x, width = blockDim.x;
  const uint32_t row_bytes = Ring::row_bytes(p.M, width, width), slot_bytes = row_bytes * (RES ? 2 : 1);
  const uint32_t base = (uint32_t)__cvta_generic_to_shared(room);
  auto x_row = [&](int64_t row) { return static_cast<const T*>(p.x) + row * p.ldx; };
  auto r_row = [&](int64_t row) { return static_cast<const T*>(p.res) + row * p.ldr; };
  auto fetch = [&](int64_t row, int i) {
    if (row < p.rows) {
      Ring::fetch(base + i * slot_bytes, x_row(row), p.M, t, width);
      if (RES) Ring::fetch(base + i * slot_bytes + row_bytes, r_row(row), p.M, t, width);
    }
    ahead_commit();
  };
  dep_wait();
#pragma unroll
  for (int i = 0; i < SLOTS; ++i) fetch((int64_t)blockIdx.x + (int64_t)i * gridDim.x, i);
  int i = 0, flip = 0;
  for (int64_t row = blockIdx.x; row < p.rows; row += gridDim.x, flip ^= 1) {
    const uint8_t* slot = room + i * slot_bytes;
    ahead_wait<SLOTS - 1>();
    if (VEC == 1) __syncthreads();
    float v[NV][VEC];
    float sq[2] = {0.f, 0.f};
    const T* x = x_row(row);
    const T* res = RES ? r_row(row) : nullptr;
    T* sum = p.sum ? static_cast<T*>(p.sum) + row * p.lds : nullptr;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const uint32_t c = (uint32_t)(t + k * width) * VEC;
      const int n = p.M - (int)c;
      Ring::get(slot, x, p.M, width, k, c, n, v[k]);
      if (RES) {
        float r[VEC];
        Ring::get(slot + row_bytes, res, p.M, width, k, c, n, r);
        vadd<VEC>(v[k], r);
        round_pairs(v[k], static_cast<const T*>(nullptr));
        if (sum) Ring::keep(sum + c, n, v[k]);
      }
      vdot<VEC>(sq, v[k], v[k]);
    }
    const float ss = over_group<Sum>(sq[0] + sq[1], width, buf[flip][0]);
    fetch(row + (int64_t)SLOTS * gridDim.x, i);              // the slot has been read: the sum of its threads depends on it
    const float rstd = rsqrtf(fmaf(ss, p.inv_M, p.eps));
    if (t == 0 && p.rstd) p.rstd[row] = rstd;
    float top = 0.f;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const uint32_t c = (uint32_t)(t + k * width) * VEC;
      float w[VEC];
      Ring::plain(p.w + c, p.M - (int)c, w);
      if (sizeof(Y) != 1) vscale<VEC>(v[k], rstd);           // the scale takes rstd out of an 8-bit y again: y / c = 448 s w / max |s w|
      vmul<VEC>(v[k], w);
      if (sizeof(Y) == 1) {
#pragma unroll
        for (int e = 0; e < VEC; ++e) top = max_keep_nan(top, fabsf(v[k][e]));
      }
    }
    float inv = 1.f;
    if (sizeof(Y) == 1) {
      top = over_group<MaxAbs>(top, width, buf[flip][1]);
      const float size = top * rstd;                         // max |y|; NaN where the row has a NaN or an infinity
      const bool tiny = size < kMinScale * kE4m3Max;
      if (t == 0) p.y_scale[row] = size == 0.f ? 1.f : tiny ? kMinScale : size / kE4m3Max;
      const bool by_size = tiny || top < 2e-36f;              // 448 / top may be beyond fp32 (below 1.32e-36)
      // an exact quotient: its error moves every code of the row the same way
      inv = tiny ? 1.f / kMinScale : size != size ? size : kE4m3Max / (by_size ? size : top);
      if (by_size) {
#pragma unroll
        for (int k = 0; k < NV; ++k) vscale<VEC>(v[k], rstd);
      }
    }
    Y* y = static_cast<Y*>(p.y) + row * p.ldy;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const uint32_t c = (uint32_t)(t + k * width) * VEC;
      if (sizeof(Y) == 1) vscale<VEC>(v[k], inv);
      Ring::keep(y + c, p.M - (int)c, v[k]);
    }
    if (++i == SLOTS) i = 0;
  }
  ahead_wait<0>();
  dep_trigger();
}

struct NormBwd {
  const void *dy, *s, *ds;
  const float *w, *rstd;
  void* dx;
  float* part;           // a row of M sums for each CTA, or null
  int64_t rows, lddy, lds, ldds, lddx;
  int32_t M, width;
  float inv_M;
};

// A CTA takes every gridDim-th group of rows and keeps its columns' share of dw in registers, so that the sums over the rows have
// a fixed order and cost one row of partial sums a CTA.  Rows are on their way as in the forward kernel.
// SOLO: a row at a time (p.width is the CTA), else several.
template <class T, int VEC, int NV, int SLOTS, bool DS, int FILL, bool SOLO>
__global__ void __launch_bounds__(512) norm_backward_kernel(const NormBwd p) {
  typedef Ahead<T, VEC, NV, FILL> Ring;
  extern __shared__ __align__(16) uint8_t room[];            // [slot][dy, s, ds], at the end the groups' sums
  __shared__ float buf[2][16];
  const int tid = threadIdx.x, nt = blockDim.x, width = SOLO ? nt : p.width, t = SOLO ? tid : tid & (width - 1);
  const int per = SOLO ? 1 : nt / width, mine = SOLO ? 0 : tid / width;
  const int64_t step = (int64_t)gridDim.x * per;
  const uint32_t row_bytes = Ring::row_bytes(p.M, nt, width), slot_bytes = row_bytes * (DS ? 3 : 2);
  const uint32_t base = (uint32_t)__cvta_generic_to_shared(room);
  auto u_row = [&](int64_t row) { return static_cast<const T*>(p.dy) + row * p.lddy; };
  auto s_row = [&](int64_t row) { return static_cast<const T*>(p.s) + row * p.lds; };
  auto d_row = [&](int64_t row) { return static_cast<const T*>(p.ds) + row * p.ldds; };
  auto fetch = [&](int64_t row, int i) {
    if (row < p.rows) {
      Ring::fetch(base + i * slot_bytes, u_row(row), p.M, t, width);
      Ring::fetch(base + i * slot_bytes + row_bytes, s_row(row), p.M, t, width);
      if (DS) Ring::fetch(base + i * slot_bytes + 2 * row_bytes, d_row(row), p.M, t, width);
    }
    ahead_commit();
  };
  dep_wait();
  float dw[NV][VEC];
#pragma unroll
  for (int k = 0; k < NV; ++k)
#pragma unroll
    for (int e = 0; e < VEC; ++e) dw[k][e] = 0.f;
  const int64_t first = (int64_t)blockIdx.x * per;
#pragma unroll
  for (int i = 0; i < SLOTS; ++i) fetch(first + mine + i * step, i);
  float rstd = first + mine < p.rows ? p.rstd[first + mine] : 0.f;
  int i = 0, flip = 0;
  for (int64_t row0 = first; row0 < p.rows; row0 += step, flip ^= 1) {
    const int64_t row = row0 + mine;
    const bool live = SOLO || row < p.rows;
    const float rstd_next = row + step < p.rows ? p.rstd[row + step] : 0.f;
    const uint8_t* slot = room + i * slot_bytes;
    ahead_wait<SLOTS - 1>();
    if (VEC == 1) __syncthreads();
    float u[NV][VEC], n[NV][VEC];
    const T *dy = u_row(row), *s = s_row(row), *ds = DS ? d_row(row) : nullptr;
    T* dx = static_cast<T*>(p.dx) + row * p.lddx;
    float dots[2] = {0.f, 0.f};
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const uint32_t c = (uint32_t)(t + k * width) * VEC;
      const int left = live ? p.M - (int)c : 0;
      Ring::get(slot, dy, p.M, width, k, c, left, u[k]);
      Ring::get(slot + row_bytes, s, p.M, width, k, c, left, n[k]);
      float w[VEC];
      Ring::plain(p.w + c, p.M - (int)c, w);
      vscale<VEC>(n[k], rstd);
      vfma<VEC>(dw[k], u[k], n[k]);
      vmul<VEC>(u[k], w);
      vdot<VEC>(dots, u[k], n[k]);
    }
    const float dot = over_group<Sum>(dots[0] + dots[1], width, buf[flip]) * -p.inv_M;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const uint32_t c = (uint32_t)(t + k * width) * VEC;
      const int left = live ? p.M - (int)c : 0;
      vfma<VEC>(u[k], n[k], dot);
      vscale<VEC>(u[k], rstd);
      if (DS) {
        float add[VEC];
        Ring::get(slot + 2 * row_bytes, ds, p.M, width, k, c, left, add);
        vadd<VEC>(u[k], add);
      }
      if (live) Ring::keep(dx + c, p.M - (int)c, u[k]);
    }
    // the slot is given away when every thread that reads it has: itself, or (VEC = 1) the row's
    if (VEC == 1 && DS) __syncthreads();
    fetch(row + SLOTS * step, i);
    rstd = rstd_next;
    if (++i == SLOTS) i = 0;
  }
  ahead_wait<0>();
  dep_trigger();
  if (!p.part) return;
  // the groups of the CTA in order, then the CTA's row of sums
  float* out = p.part + (int64_t)blockIdx.x * p.M;
  if (SOLO) {
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int c = (t + k * width) * VEC;
#pragma unroll
      for (int e = 0; e < VEC; ++e)
        if (c + e < p.M) out[c + e] = dw[k][e];
    }
    return;
  }
  float* shared = reinterpret_cast<float*>(room);
  __syncthreads();
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int c = (t + k * width) * VEC;
#pragma unroll
    for (int e = 0; e < VEC; ++e)
      if (c + e < p.M) shared[mine * p.M + c + e] = dw[k][e];
  }
  __syncthreads();
  for (int c = threadIdx.x; c < p.M; c += blockDim.x) {
    float a = 0.f;
    for (int k = 0; k < per; ++k) a += shared[k * p.M + c];
    out[c] = a;
  }
}

// dw = sum of the CTAs' rows, 32 columns a CTA: 32 warps take every 32nd row, eight of them in flight, and are added in pairs.
// (With eight warps and four rows in flight the 592 rows of M = 4096 took 14 us behind a pass of 48.)
__global__ void __launch_bounds__(1024) norm_weight_kernel(const float* part, int n, int M, float* dw) {
  __shared__ float acc[32][33];
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, c = blockIdx.x * 32 + lane;
  dep_sync();
  float a = 0.f;
  if (c < M) {
    for (int k = w; k < n; k += 256) {
      float b[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) b[j] = k + 32 * j < n ? part[(int64_t)(k + 32 * j) * M + c] : 0.f;
      a += ((b[0] + b[1]) + (b[2] + b[3])) + ((b[4] + b[5]) + (b[6] + b[7]));
    }
  }
  acc[w][lane] = a;
  __syncthreads();
  // warp w: column w of the 32, a row of sums a lane
  a = acc[lane][w];
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) a += __shfl_xor_sync(0xffffffffu, a, o);
  if (lane == 0 && blockIdx.x * 32 + w < M) dw[blockIdx.x * 32 + w] = a;
}

int pow2_at_least(int n) {
  int p = 32;
  while (p < n) p <<= 1;
  return p;
}

// Threads that share a row: about `each` accesses a thread, 32 to `most` threads.
int row_width(int accesses, int each, int most) {
  const int w = pow2_at_least((accesses + each - 1) / each);
  return w > most ? most : w;
}

bool type_ok(int32_t t) { return t == FW_F32 || t == FW_BF16; }
int type_bytes(int32_t t) { return t == FW_F32 ? 4 : t == FW_BF16 ? 2 : 1; }

fw_status desc_check(const fw_norm_desc* d) {
  if (!d) return FW_ERR_INVALID_ARG;
  if (d->M < 1 || d->M > kNormMaxM) return FW_ERR_SHAPE;
  if (!type_ok(d->dtype) || (d->y_dtype != d->dtype && d->y_dtype != FW_E4M3)) return FW_ERR_INVALID_ARG;
  if (!(d->eps > 0.f) || d->eps > 3e38f) return FW_ERR_INVALID_ARG;
  return FW_OK;
}

fw_status rows_check(int64_t rows) { return rows < 1 || rows > 0x7fffffff ? FW_ERR_SHAPE : FW_OK; }

struct Mat { const void* p; int64_t ld; int elem; };

// rows wide enough, elements aligned; *vec: whole 16-byte accesses fit too
fw_status mat_check(const Mat& m, int M, int access, bool* vec) {
  if (m.ld < M || m.ld > ((int64_t)1 << 30)) return FW_ERR_SHAPE;
  if (!aligned_to(m.p, m.elem)) return FW_ERR_INVALID_ARG;
  const size_t bytes = (size_t)access * m.elem;
  if (!aligned_to(m.p, bytes) || (m.ld * m.elem) % (int64_t)bytes != 0) *vec = false;
  return FW_OK;
}

// What a kernel of one shape is launched with: found once for each device, number of threads and size of shared memory.
struct FillCache {
  std::mutex mu;
  struct { int dev, threads, per_sm; size_t smem; } known[8] = {};
  int n = 0;
};
// CTAs of one wave, or as many as there are groups of rows
template <class F>
cudaError_t fill(F* kernel, FillCache& cache, int threads, size_t smem, int64_t groups, int most, int* ctas) {
  int dev = 0, per_sm = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  {
    std::lock_guard<std::mutex> lock(cache.mu);
    const int have = cache.n < 8 ? cache.n : 8;
    for (int i = 0; i < have && !per_sm; ++i)
      if (cache.known[i].dev == dev && cache.known[i].threads == threads && cache.known[i].smem == smem) per_sm = cache.known[i].per_sm;
    if (!per_sm) {
      // the most that any launch asks for: what is set late by one thread never undoes what another needs
      e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 227 * 1024 - 1024);
      if (e == cudaSuccess) e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, kernel, threads, smem);
      if (e != cudaSuccess) return e;
      if (per_sm < 1) return cudaErrorInvalidConfiguration;
      cache.known[cache.n % 8] = {dev, threads, per_sm, smem};
      if (++cache.n >= 16) cache.n = 8;
    }
  }
  int64_t n = (int64_t)per_sm * sm_count();
  if (n > most) n = most;
  *ctas = (int)(groups < n ? groups : n);
  return cudaSuccess;
}

// Rows on their way: 256 bytes of them a thread.  Where they are not aligned two, or one of more than 8192
// elements (three tensors of 64 KB fit a SM once)
constexpr int slots(int vec, int nv, int tensors) {
  const int n = vec > 1 ? 256 / (16 * nv * tensors) : nv > 16 ? 1 : 2;
  return n < 1 ? 1 : n > 4 ? 4 : n;
}

template <class T, class Y, int VEC, int NV, bool RES, int FILL>
cudaError_t forward_launch(const NormFwd& p, cudaStream_t s) {
  constexpr int SLOTS = slots(VEC, NV, RES ? 2 : 1);
  static FillCache cache;
  auto kernel = norm_forward_kernel<T, Y, VEC, NV, SLOTS, RES, FILL>;
  const size_t smem = (size_t)SLOTS * (RES ? 2 : 1) * Ahead<T, VEC, NV, FILL>::row_bytes(p.M, p.width, p.width);
  int ctas = 0;
  const cudaError_t e = fill(kernel, cache, p.width, smem, p.rows, 1 << 30, &ctas);
  return e != cudaSuccess ? e : launch_dep(kernel, ctas, p.width, smem, s, p);
}
template <class T, class Y, int VEC, int NV, bool RES>
cudaError_t forward_launch(const NormFwd& p, cudaStream_t s) {
  constexpr int WHOLE = VEC > 1 ? ROW_WHOLE : ROW_PART, FULL = VEC > 1 ? ROW_FULL : ROW_PART;
  if (VEC > 1 && p.M == NV * VEC * p.width) return forward_launch<T, Y, VEC, NV, RES, FULL>(p, s);
  if (VEC > 1 && p.M % VEC == 0) return forward_launch<T, Y, VEC, NV, RES, WHOLE>(p, s);
  return forward_launch<T, Y, VEC, NV, RES, ROW_PART>(p, s);
}
template <class T, class Y, int VEC, int NV>
cudaError_t forward_launch(const NormFwd& p, cudaStream_t s) {
  return p.res ? forward_launch<T, Y, VEC, NV, true>(p, s) : forward_launch<T, Y, VEC, NV, false>(p, s);
}

// Four accesses of 16 bytes a thread where there are rows for every SM, one where the chain of one row is all there is
template <class T, class Y, int VEC>
cudaError_t forward_nv(const NormFwd& p0, cudaStream_t s) {
  NormFwd p = p0;
  const int acc = (p.M + VEC - 1) / VEC;
  p.width = row_width(acc, p.rows < 2 * sm_count() ? 1 : VEC > 1 ? 4 : 8, 512);
  const int nv = (acc + p.width - 1) / p.width;
  // 512 threads take kNormMaxM elements in four accesses of eight, eight of four or thirty-two of one
  if (nv <= 1) return forward_launch<T, Y, VEC, 1>(p, s);
  if (nv <= 2) return forward_launch<T, Y, VEC, 2>(p, s);
  if (nv <= 4) return forward_launch<T, Y, VEC, 4>(p, s);
  if (nv <= 8) return forward_launch<T, Y, VEC, VEC == 8 ? 4 : 8>(p, s);
  if (nv <= 16) return forward_launch<T, Y, VEC, VEC == 8 ? 4 : VEC == 4 ? 8 : 16>(p, s);
  return forward_launch<T, Y, VEC, VEC == 8 ? 4 : VEC == 4 ? 8 : 32>(p, s);
}

template <class T, class Y>
cudaError_t forward_vec(const NormFwd& p, bool vec, cudaStream_t s) {
  return vec ? forward_nv<T, Y, 16 / sizeof(T)>(p, s) : forward_nv<T, Y, 1>(p, s);
}

int backward_ctas() { return 4 * sm_count(); }

template <class T, int VEC, int NV, bool DS, int FILL, bool SOLO>
cudaError_t backward_launch(const NormBwd& p, cudaStream_t s, int* ctas) {
  constexpr int SLOTS = slots(VEC, NV, DS ? 3 : 2);
  static FillCache cache;
  auto kernel = norm_backward_kernel<T, VEC, NV, SLOTS, DS, FILL, SOLO>;
  const int threads = SOLO ? p.width : 128, per = threads / p.width;
  size_t smem = (size_t)SLOTS * (DS ? 3 : 2) * Ahead<T, VEC, NV, FILL>::row_bytes(p.M, threads, p.width);
  if (!SOLO && p.part && smem < (size_t)per * p.M * sizeof(float)) smem = (size_t)per * p.M * sizeof(float);
  const cudaError_t e = fill(kernel, cache, threads, smem, (p.rows + per - 1) / per, backward_ctas(), ctas);
  return e != cudaSuccess ? e : launch_dep(kernel, *ctas, threads, smem, s, p);
}
template <class T, int VEC, int NV, bool DS>
cudaError_t backward_launch(const NormBwd& p, cudaStream_t s, int* ctas) {
  constexpr int WHOLE = VEC > 1 ? ROW_WHOLE : ROW_PART, FULL = VEC > 1 ? ROW_FULL : ROW_PART;
  if constexpr (NV <= 4) {                                   // more accesses a thread: 128 threads or more (see backward_nv)
    if (p.width < 128)
      return VEC > 1 && p.M % VEC == 0 ? backward_launch<T, VEC, NV, DS, WHOLE, false>(p, s, ctas)
                                       : backward_launch<T, VEC, NV, DS, ROW_PART, false>(p, s, ctas);
  }
  if (VEC > 1 && p.M == NV * VEC * p.width) return backward_launch<T, VEC, NV, DS, FULL, true>(p, s, ctas);
  if (VEC > 1 && p.M % VEC == 0) return backward_launch<T, VEC, NV, DS, WHOLE, true>(p, s, ctas);
  return backward_launch<T, VEC, NV, DS, ROW_PART, true>(p, s, ctas);
}
template <class T, int VEC, int NV>
cudaError_t backward_launch(const NormBwd& p, cudaStream_t s, int* ctas) {
  return p.ds ? backward_launch<T, VEC, NV, true>(p, s, ctas) : backward_launch<T, VEC, NV, false>(p, s, ctas);
}

template <class T, int VEC>
cudaError_t backward_nv(const NormBwd& p0, cudaStream_t s, int* ctas) {
  NormBwd p = p0;
  const int acc = (p.M + VEC - 1) / VEC;
  // rows of up to 128 accesses of 16 bytes by a warp or two (30000 x 1000: 61.9 us against 72.2), longer ones two accesses a thread
  // (8192 x 4096: 63.4 against 64.7)
  p.width = row_width(acc, VEC == 1 || acc <= 128 ? 4 : 2, 512);
  const int nv = (acc + p.width - 1) / p.width;
  if (nv <= 1) return backward_launch<T, VEC, 1>(p, s, ctas);
  if (nv <= 2) return backward_launch<T, VEC, 2>(p, s, ctas);
  if (nv <= 4) return backward_launch<T, VEC, 4>(p, s, ctas);
  if (nv <= 8) return backward_launch<T, VEC, VEC == 8 ? 4 : 8>(p, s, ctas);
  if (nv <= 16) return backward_launch<T, VEC, VEC == 8 ? 4 : VEC == 4 ? 8 : 16>(p, s, ctas);
  return backward_launch<T, VEC, VEC == 8 ? 4 : VEC == 4 ? 8 : 32>(p, s, ctas);
}

fw_status failed(cudaError_t e, const char* where) {
  if (e == cudaSuccess) return FW_OK;
  fprintf(stderr, "[fw] %s: %s\n", where, cudaGetErrorString(e));
  return FW_ERR_CUDA;
}

}  // namespace
}  // namespace fw

using namespace fw;

extern "C" {

void fw_norm_desc_default(fw_norm_desc* d, int32_t M) {
  if (!d) return;
  d->M = M; d->dtype = FW_BF16; d->y_dtype = FW_BF16; d->eps = 1e-6f;
}

size_t fw_rmsnorm_scratch_bytes(const fw_norm_desc* d) {
  if (desc_check(d) != FW_OK) return 0;
  return ((size_t)backward_ctas() * d->M * sizeof(float) + 255) / 256 * 256;
}

fw_status fw_rmsnorm_forward(const fw_norm_desc* d, int64_t rows, const void* x, int64_t ldx, const void* res, int64_t ldr,
                             const float* w, void* sum, int64_t lds, void* y, int64_t ldy, float* y_scale, float* rstd,
                             void* cuda_stream) {
  fw_status st = desc_check(d);
  if (st != FW_OK) return st;
  const bool q8 = d->y_dtype == FW_E4M3;
  if (!x || !w || !y || (q8 != (y_scale != nullptr)) || (sum && !res)) return FW_ERR_INVALID_ARG;
  if ((st = rows_check(rows)) != FW_OK) return st;
  const int es = type_bytes(d->dtype), ys = type_bytes(d->y_dtype), per16 = 16 / es;
  bool vec = aligned_to(w, 16);
  if (!aligned_to(w, 4) || (rstd && !aligned_to(rstd, 4)) || (y_scale && !aligned_to(y_scale, 4))) return FW_ERR_INVALID_ARG;
  const Mat in[2] = {{x, ldx, es}, {res, ldr, es}}, out[2] = {{sum, lds, es}, {y, ldy, ys}};
  for (const Mat& m : in)
    if (m.p && (st = mat_check(m, d->M, per16, &vec)) != FW_OK) return st;
  for (const Mat& m : out)
    if (m.p && (st = mat_check(m, d->M, per16, &vec)) != FW_OK) return st;
  // an output may be an input itself (a thread has read what it writes), any other overlap is refused
  for (const Mat& o : out)
    for (const Mat& i : in)
      if (overlap(o.p, matrix_span(rows, d->M, o.ld, o.elem), i.p, matrix_span(rows, d->M, i.ld, i.elem)) &&
          !(o.p == i.p && o.ld == i.ld && o.elem == i.elem))
        return FW_ERR_INVALID_ARG;
  const uint64_t ny = matrix_span(rows, d->M, ldy, ys), nvec = (uint64_t)rows * 4;
  if (overlap(y, ny, sum, sum ? matrix_span(rows, d->M, lds, es) : 0)) return FW_ERR_INVALID_ARG;
  for (const Mat& o : out) {
    const uint64_t n = o.p ? matrix_span(rows, d->M, o.ld, o.elem) : 0;
    if (overlap(o.p, n, w, (uint64_t)d->M * 4) || overlap(o.p, n, y_scale, nvec) || overlap(o.p, n, rstd, nvec)) return FW_ERR_INVALID_ARG;
  }
  const void* rows_out[2] = {y_scale, rstd};
  for (const void* v : rows_out) {
    if (overlap(v, nvec, w, (uint64_t)d->M * 4)) return FW_ERR_INVALID_ARG;
    for (const Mat& i : in)
      if (overlap(v, nvec, i.p, i.p ? matrix_span(rows, d->M, i.ld, i.elem) : 0)) return FW_ERR_INVALID_ARG;
  }
  if (overlap(y_scale, nvec, rstd, nvec)) return FW_ERR_INVALID_ARG;
  NormFwd p;
  p.x = x; p.res = res; p.w = w; p.sum = sum; p.y = y; p.y_scale = y_scale; p.rstd = rstd;
  p.rows = rows; p.ldx = ldx; p.ldr = ldr; p.lds = lds; p.ldy = ldy; p.M = d->M; p.width = 0;
  p.eps = d->eps; p.inv_M = 1.f / (float)d->M;
  cudaStream_t s = (cudaStream_t)cuda_stream;
  ProfScope ps(FW_PROF_MISC, s);
  cudaError_t e;
  if (d->dtype == FW_F32)
    e = q8 ? forward_vec<float, __nv_fp8_storage_t>(p, vec, s) : forward_vec<float, float>(p, vec, s);
  else
    e = q8 ? forward_vec<__nv_bfloat16, __nv_fp8_storage_t>(p, vec, s) : forward_vec<__nv_bfloat16, __nv_bfloat16>(p, vec, s);
  return failed(e, "fw_rmsnorm_forward");
}

fw_status fw_rmsnorm_backward(const fw_norm_desc* d, int64_t rows, const void* dy, int64_t lddy, const void* s, int64_t lds,
                              const void* dsum, int64_t ldds, const float* w, const float* rstd, void* dx, int64_t lddx, float* dw,
                              void* scratch, size_t scratch_bytes, void* cuda_stream) {
  fw_status st = desc_check(d);
  if (st != FW_OK) return st;
  if (!dy || !s || !w || !rstd || !dx) return FW_ERR_INVALID_ARG;
  if ((st = rows_check(rows)) != FW_OK) return st;
  if (dw) {
    if (!scratch) return FW_ERR_INVALID_ARG;
    if (!aligned_to(scratch, 256) || scratch_bytes < fw_rmsnorm_scratch_bytes(d)) return FW_ERR_WORKSPACE;
  }
  const int es = type_bytes(d->dtype), per16 = 16 / es;
  bool vec = aligned_to(w, 16);
  if (!aligned_to(w, 4) || !aligned_to(rstd, 4) || (dw && !aligned_to(dw, 4))) return FW_ERR_INVALID_ARG;
  const Mat in[3] = {{dy, lddy, es}, {s, lds, es}, {dsum, ldds, es}}, out = {dx, lddx, es};
  for (const Mat& m : in)
    if (m.p && (st = mat_check(m, d->M, per16, &vec)) != FW_OK) return st;
  if ((st = mat_check(out, d->M, per16, &vec)) != FW_OK) return st;
  const uint64_t nout = matrix_span(rows, d->M, lddx, es);
  for (const Mat& i : in)
    if (overlap(dx, nout, i.p, i.p ? matrix_span(rows, d->M, i.ld, es) : 0) && !(dx == i.p && lddx == i.ld)) return FW_ERR_INVALID_ARG;
  if (overlap(dx, nout, w, (uint64_t)d->M * 4) || overlap(dx, nout, rstd, (uint64_t)rows * 4) ||
      overlap(dx, nout, dw, (uint64_t)d->M * 4))
    return FW_ERR_INVALID_ARG;
  if (dw) {
    const uint64_t nw = (uint64_t)d->M * 4, ns = fw_rmsnorm_scratch_bytes(d);
    const void* others[2] = {w, rstd};
    const uint64_t no[2] = {nw, (uint64_t)rows * 4};
    for (int k = 0; k < 2; ++k)
      if (overlap(dw, nw, others[k], no[k]) || overlap(scratch, ns, others[k], no[k])) return FW_ERR_INVALID_ARG;
    for (const Mat& i : in) {
      const uint64_t n = i.p ? matrix_span(rows, d->M, i.ld, es) : 0;
      if (overlap(dw, nw, i.p, n) || overlap(scratch, ns, i.p, n)) return FW_ERR_INVALID_ARG;
    }
    if (overlap(scratch, ns, dx, nout) || overlap(scratch, ns, dw, nw)) return FW_ERR_INVALID_ARG;
  }
  NormBwd p;
  p.dy = dy; p.s = s; p.ds = dsum; p.w = w; p.rstd = rstd; p.dx = dx; p.part = dw ? static_cast<float*>(scratch) : nullptr;
  p.rows = rows; p.lddy = lddy; p.lds = lds; p.ldds = ldds; p.lddx = lddx; p.M = d->M; p.width = 0; p.inv_M = 1.f / (float)d->M;
  cudaStream_t str = (cudaStream_t)cuda_stream;
  int ctas = 0;
  cudaError_t e;
  {
    ProfScope ps(FW_PROF_MISC, str);
    if (d->dtype == FW_F32) e = vec ? backward_nv<float, 4>(p, str, &ctas) : backward_nv<float, 1>(p, str, &ctas);
    else e = vec ? backward_nv<__nv_bfloat16, 8>(p, str, &ctas) : backward_nv<__nv_bfloat16, 1>(p, str, &ctas);
  }
  if (e == cudaSuccess && dw) {
    ProfScope ps(FW_PROF_MISC, str);
    e = launch_dep(norm_weight_kernel, (d->M + 31) / 32, 1024, 0, str, p.part, ctas, d->M, dw);
  }
  return failed(e, "fw_rmsnorm_backward");
}

}  // extern "C"
