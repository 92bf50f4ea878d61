// Residual addition and root-mean-square norm, forward and backward, a row at a time.
//
//   s = x + r, kept in the type of x      n = s / sqrt(mean(s^2) + eps)      y = n w
//   e4m3 y: c = max |y| / 448, y is held as e4m3(y / c) with c beside it
//   du = dy w     dx = (du - n mean(du n)) / sqrt(mean(s^2) + eps) + ds      dw = sum over the rows of dy n
//
// Both directions read each element once and write each result once: HBM bandwidth bounds them.  A row stays in the registers
// of the threads that share it between its sum and its output.
#include <cstdio>

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

// T: type of x, r and s; Y: of y.  VEC elements an access, NV accesses a thread.
template <class T, class Y, int VEC, int NV>
__global__ void __launch_bounds__(1024) norm_forward_kernel(const NormFwd p) {
  __shared__ float buf[2][32];
  const int t = threadIdx.x & (p.width - 1);
  const int64_t row = (int64_t)blockIdx.x * (blockDim.x / p.width) + threadIdx.x / p.width;
  const bool live = row < p.rows;
  dep_sync();
  const T* x = static_cast<const T*>(p.x) + row * p.ldx;
  const T* res = p.res ? static_cast<const T*>(p.res) + row * p.ldr : nullptr;
  float v[NV][VEC];
  float r[NV][VEC];
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int c = (t + k * p.width) * VEC;
    const int n = live ? p.M - c : 0;
    load<VEC>(x + c, n, 0.f, v[k]);
    if (res) load<VEC>(res + c, n, 0.f, r[k]);
  }
  float ss = 0.f;
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int c = (t + k * p.width) * VEC;
    if (res) {
#pragma unroll
      for (int e = 0; e < VEC; ++e) v[k][e] = held(v[k][e] + r[k][e], x);
      if (p.sum && live) store<VEC>(static_cast<T*>(p.sum) + row * p.lds + c, p.M - c, v[k]);
    }
#pragma unroll
    for (int e = 0; e < VEC; ++e) ss = fmaf(v[k][e], v[k][e], ss);
  }
  ss = over_group<Sum>(ss, p.width, buf[0]);
  const float rstd = rsqrtf(fmaf(ss, p.inv_M, p.eps));
  if (t == 0 && live && p.rstd) p.rstd[row] = rstd;
  float top = 0.f;
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int c = (t + k * p.width) * VEC;
    float w[VEC];
    load<VEC>(p.w + c, p.M - c, 0.f, w);
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
      v[k][e] = v[k][e] * rstd * w[e];
      if (sizeof(Y) == 1) top = max_keep_nan(top, fabsf(v[k][e]));
    }
  }
  float inv = 1.f;
  if (sizeof(Y) == 1) {
    top = over_group<MaxAbs>(top, p.width, buf[1]);
    float scale = 1.f;
    if (top != 0.f) scale = top * (1.f / kE4m3Max);
    if (scale < kMinScale) scale = kMinScale;                  // a NaN stays
    if (t == 0 && live) p.y_scale[row] = scale;
    inv = 1.f / scale;
  }
  if (!live) return;
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int c = (t + k * p.width) * VEC;
    if (sizeof(Y) == 1) {
#pragma unroll
      for (int e = 0; e < VEC; ++e) v[k][e] *= inv;
    }
    store<VEC>(static_cast<Y*>(p.y) + row * p.ldy + c, p.M - c, v[k]);
  }
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
// a fixed order and cost one row of partial sums a CTA.
template <class T, int VEC, int NV>
__global__ void __launch_bounds__(VEC > 1 ? 512 : 1024) norm_backward_kernel(const NormBwd p) {
  extern __shared__ float shared[];
  __shared__ float buf[2][32];
  const int t = threadIdx.x & (p.width - 1), per = blockDim.x / p.width, mine = threadIdx.x / p.width;
  dep_sync();
  float dw[NV][VEC];
#pragma unroll
  for (int k = 0; k < NV; ++k)
#pragma unroll
    for (int e = 0; e < VEC; ++e) dw[k][e] = 0.f;
  const int64_t groups = (p.rows + per - 1) / per;
  int flip = 0;
  for (int64_t g = blockIdx.x; g < groups; g += gridDim.x, flip ^= 1) {
    const int64_t row = g * per + mine;
    const bool live = row < p.rows;
    const T* dy = static_cast<const T*>(p.dy) + row * p.lddy;
    const T* s = static_cast<const T*>(p.s) + row * p.lds;
    float u[NV][VEC], n[NV][VEC], add[NV][VEC];
    const float rstd = live ? p.rstd[row] : 0.f;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int c = (t + k * p.width) * VEC, left = live ? p.M - c : 0;
      load<VEC>(dy + c, left, 0.f, u[k]);
      load<VEC>(s + c, left, 0.f, n[k]);
      if (p.ds) load<VEC>(static_cast<const T*>(p.ds) + row * p.ldds + c, left, 0.f, add[k]);
    }
    float dot = 0.f;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int c = (t + k * p.width) * VEC;
      float w[VEC];
      load<VEC>(p.w + c, p.M - c, 0.f, w);
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        n[k][e] *= rstd;
        dw[k][e] = fmaf(u[k][e], n[k][e], dw[k][e]);
        u[k][e] *= w[e];
        dot = fmaf(u[k][e], n[k][e], dot);
      }
    }
    dot = over_group<Sum>(dot, p.width, buf[flip]) * p.inv_M;
    if (!live) continue;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int c = (t + k * p.width) * VEC;
      float out[VEC];
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        out[e] = rstd * (u[k][e] - n[k][e] * dot);
        if (p.ds) out[e] += add[k][e];
      }
      store<VEC>(static_cast<T*>(p.dx) + row * p.lddx + c, p.M - c, out);
    }
  }
  if (!p.part) return;
  // the groups of the CTA in order, then the CTA's row of sums
  float* out = p.part + (int64_t)blockIdx.x * p.M;
  if (per == 1) {
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int c = (t + k * p.width) * VEC;
#pragma unroll
      for (int e = 0; e < VEC; ++e)
        if (c + e < p.M) out[c + e] = dw[k][e];
    }
    return;
  }
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int c = (t + k * p.width) * VEC;
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

// dw = sum of the CTAs' rows, 32 columns a CTA: eight warps take every eighth row, and are added in order.
__global__ void __launch_bounds__(256) norm_weight_kernel(const float* part, int n, int M, float* dw) {
  __shared__ float acc[8][32];
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, c = blockIdx.x * 32 + lane;
  dep_sync();
  float a = 0.f;
  if (c < M) {
    float b[4] = {0.f, 0.f, 0.f, 0.f};
    int k = w;
    for (; k + 24 < n; k += 32)
#pragma unroll
      for (int j = 0; j < 4; ++j) b[j] += part[(int64_t)(k + 8 * j) * M + c];
    for (int j = 0; k < n; k += 8, ++j) b[j & 3] += part[(int64_t)k * M + c];
    a = (b[0] + b[1]) + (b[2] + b[3]);
  }
  acc[w][lane] = a;
  __syncthreads();
  if (w == 0 && c < M) {
    a = acc[0][lane];
#pragma unroll
    for (int k = 1; k < 8; ++k) a += acc[k][lane];
    dw[c] = a;
  }
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

template <class T, class Y, int VEC>
cudaError_t forward_nv(const NormFwd& p0, cudaStream_t s) {
  NormFwd p = p0;
  const int acc = (p.M + VEC - 1) / VEC;
  p.width = row_width(acc, VEC > 1 ? 2 : 8, 1024);
  const int nv = (acc + p.width - 1) / p.width;
  const int threads = p.width < 256 ? 256 : p.width;
  const dim3 grid((unsigned)((p.rows + threads / p.width - 1) / (threads / p.width)));
  if (nv <= 1) return launch_dep(norm_forward_kernel<T, Y, VEC, 1>, grid, threads, 0, s, p);
  if (nv <= 2) return launch_dep(norm_forward_kernel<T, Y, VEC, 2>, grid, threads, 0, s, p);
  // 1024 threads take kNormMaxM elements in two accesses of eight, four of four or sixteen of one
  if (nv <= 4) return launch_dep(norm_forward_kernel<T, Y, VEC, VEC == 8 ? 2 : 4>, grid, threads, 0, s, p);
  if (nv <= 8) return launch_dep(norm_forward_kernel<T, Y, VEC, VEC == 8 ? 2 : VEC == 4 ? 4 : 8>, grid, threads, 0, s, p);
  return launch_dep(norm_forward_kernel<T, Y, VEC, VEC == 8 ? 2 : VEC == 4 ? 4 : 16>, grid, threads, 0, s, p);
}

template <class T, class Y>
cudaError_t forward_vec(const NormFwd& p, bool vec, cudaStream_t s) {
  return vec ? forward_nv<T, Y, 16 / sizeof(T)>(p, s) : forward_nv<T, Y, 1>(p, s);
}

int backward_ctas() { return 2 * sm_count(); }

template <class T, int VEC, int NV>
cudaError_t backward_launch(const NormBwd& p, cudaStream_t s, int* ctas) {
  const int threads = p.width < 256 ? 256 : p.width, per = threads / p.width;
  const int64_t groups = (p.rows + per - 1) / per;
  const int most = backward_ctas();
  *ctas = groups < most ? (int)groups : most;
  // at most 8 KB: a row shared by fewer than 256 threads has an access or (VEC = 1) four for each of them
  const size_t smem = per > 1 && p.part ? (size_t)per * p.M * sizeof(float) : 0;
  return launch_dep(norm_backward_kernel<T, VEC, NV>, *ctas, threads, smem, s, p);
}

template <class T, int VEC>
cudaError_t backward_nv(const NormBwd& p0, cudaStream_t s, int* ctas) {
  NormBwd p = p0;
  const int acc = (p.M + VEC - 1) / VEC;
  p.width = row_width(acc, VEC > 1 ? 1 : 4, VEC > 1 ? 512 : 1024);
  const int nv = (acc + p.width - 1) / p.width;
  if (nv <= 1) return backward_launch<T, VEC, 1>(p, s, ctas);
  if (nv <= 2) return backward_launch<T, VEC, 2>(p, s, ctas);
  if (nv <= 4) return backward_launch<T, VEC, 4>(p, s, ctas);
  if (VEC == 8) return cudaErrorInvalidValue;            // kNormMaxM / 8 accesses by 512 threads are four each
  if (nv <= 8) return backward_launch<T, VEC, VEC == 8 ? 4 : 8>(p, s, ctas);
  return VEC == 1 ? backward_launch<T, VEC, VEC == 1 ? 16 : 4>(p, s, ctas) : cudaErrorInvalidValue;
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
    e = launch_dep(norm_weight_kernel, (d->M + 31) / 32, 256, 0, str, p.part, ctas, d->M, dw);
  }
  return failed(e, "fw_rmsnorm_backward");
}

}  // extern "C"
