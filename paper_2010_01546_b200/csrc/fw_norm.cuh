// What the norms share (fw_norm.cu, fw_sandwich.cu): rows of a matrix that stay on chip between their sums and their outputs.
#ifndef FW_NORM_CUH_
#define FW_NORM_CUH_

#include <cstdio>
#include <mutex>

#include "fw_internal.h"
#include "fw_rows.cuh"

namespace fw {
namespace norm {

using namespace rows;

constexpr int kNormMaxM = 16384;
constexpr float kE4m3Max = 448.f;
constexpr float kMinScale = 7.52316385e-37f;   // 2^-120: the reciprocal of a scale stays finite

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

// 8-bit rows, from top = max |s w|: the factor that takes s w to codes, and the scale beside them
__device__ __forceinline__ bool by_size(float top, float rstd) {
  return top * rstd < kMinScale * kE4m3Max || top < 2e-36f;  // 448 / top may be beyond fp32 (below 1.32e-36): s w rstd is taken instead
}
__device__ __forceinline__ float row_scale(float top, float rstd, float* scale) {
  const float size = top * rstd;                             // max |y|; NaN where the row has a NaN or an infinity
  const bool tiny = size < kMinScale * kE4m3Max;
  *scale = size == 0.f ? 1.f : tiny ? kMinScale : size / kE4m3Max;
  // an exact quotient: its error moves every code of the row the same way
  return tiny ? 1.f / kMinScale : size != size ? size : kE4m3Max / (by_size(top, rstd) ? size : top);
}

// ---- host ----
inline int pow2_at_least(int n) {
  int p = 32;
  while (p < n) p <<= 1;
  return p;
}

// Threads that share a row: about `each` accesses a thread, 32 to `most` threads.
inline int row_width(int accesses, int each, int most) {
  const int w = pow2_at_least((accesses + each - 1) / each);
  return w > most ? most : w;
}

inline bool type_ok(int32_t t) { return t == FW_F32 || t == FW_BF16; }
inline int type_bytes(int32_t t) { return t == FW_F32 ? 4 : t == FW_BF16 ? 2 : 1; }

inline fw_status rows_check(int64_t rows) { return rows < 1 || rows > 0x7fffffff ? FW_ERR_SHAPE : FW_OK; }

struct Mat { const void* p; int64_t ld; int elem; };

// rows wide enough, elements aligned; *vec: whole 16-byte accesses fit too
inline fw_status mat_check(const Mat& m, int M, int access, bool* vec) {
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

inline fw_status failed(cudaError_t e, const char* where) {
  if (e == cudaSuccess) return FW_OK;
  fprintf(stderr, "[fw] %s: %s\n", where, cudaGetErrorString(e));
  return FW_ERR_CUDA;
}

}  // namespace norm
}  // namespace fw
#endif
