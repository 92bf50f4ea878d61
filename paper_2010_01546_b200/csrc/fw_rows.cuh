// Rows of a matrix as vectors of VEC elements: loads into and stores from fp32 registers, and sums over the threads that
// share a row.  Used by the operators that pass over rows once (norm, distillation loss, gates of a gated block).
#ifndef FW_ROWS_CUH_
#define FW_ROWS_CUH_

#include <cuda_bf16.h>
#include <cuda_fp8.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "fw_lanes.cuh"

namespace fw {
namespace rows {

// The two halves of dep_sync (fw_internal.h) for kernels whose CTAs stay and walk over their work: the dependents of such a grid
// come when its CTAs are through.  Earlier they take places beside those that still run, and the grid after next starts
// where there is room, not where there is time: norm backward of 8192 x 4096 in a row of calls 97 us, this way 74.
__device__ __forceinline__ void dep_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void dep_trigger() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

// Two bf16 of a 32-bit word, the lower address first.
__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {          // nearest even, a NaN stays one
  const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}
// Four fp32 to e4m3 (nearest even, beyond 448 to 448, a NaN stays one), the lowest address in the lowest byte.
__device__ __forceinline__ uint32_t pack_e4m3(float a, float b, float c, float d) {
  const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3);
  const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(c, d), __NV_SATFINITE, __NV_E4M3);
  return lo | (hi << 16);
}

__device__ __forceinline__ float to_f(float x) { return x; }
__device__ __forceinline__ float to_f(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ void put(float* p, float v) { *p = v; }
__device__ __forceinline__ void put(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }
__device__ __forceinline__ void put(__nv_fp8_storage_t* p, float v) { *p = __nv_cvt_float_to_fp8(v, __NV_SATFINITE, __NV_E4M3); }

// n <= VEC elements from p on; those past n read as `none`.  With VEC > 1 a whole vector is aligned to its own size.
template <int VEC>
__device__ __forceinline__ void load(const float* p, int n, float none, float (&v)[VEC]) {
  if (VEC == 4 && n >= 4) {
    const float4 q = *reinterpret_cast<const float4*>(p);
    v[0] = q.x; v[1 % VEC] = q.y; v[2 % VEC] = q.z; v[3 % VEC] = q.w;
  } else if (VEC == 8 && n >= 8) {
    const float4 q = reinterpret_cast<const float4*>(p)[0], r = reinterpret_cast<const float4*>(p)[1];
    v[0] = q.x; v[1 % VEC] = q.y; v[2 % VEC] = q.z; v[3 % VEC] = q.w;
    v[4 % VEC] = r.x; v[5 % VEC] = r.y; v[6 % VEC] = r.z; v[7 % VEC] = r.w;
  } else {
#pragma unroll
    for (int e = 0; e < VEC; ++e) v[e] = e < n ? p[e] : none;
  }
}
template <int VEC>
__device__ __forceinline__ void load(const __nv_bfloat16* p, int n, float none, float (&v)[VEC]) {
  if (VEC == 8 && n >= 8) {
    const uint4 q = *reinterpret_cast<const uint4*>(p);
    v[0] = bf16_lo(q.x); v[1 % VEC] = bf16_hi(q.x); v[2 % VEC] = bf16_lo(q.y); v[3 % VEC] = bf16_hi(q.y);
    v[4 % VEC] = bf16_lo(q.z); v[5 % VEC] = bf16_hi(q.z); v[6 % VEC] = bf16_lo(q.w); v[7 % VEC] = bf16_hi(q.w);
  } else {
#pragma unroll
    for (int e = 0; e < VEC; ++e) v[e] = e < n ? to_f(p[e]) : none;
  }
}
template <int VEC>
__device__ __forceinline__ void store(float* p, int n, const float (&v)[VEC]) {
  if (VEC == 4 && n >= 4) {
    *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1 % VEC], v[2 % VEC], v[3 % VEC]);
  } else {
#pragma unroll
    for (int e = 0; e < VEC; ++e)
      if (e < n) p[e] = v[e];
  }
}
template <int VEC>
__device__ __forceinline__ void store(__nv_bfloat16* p, int n, const float (&v)[VEC]) {
  if (VEC == 8 && n >= 8) {
    *reinterpret_cast<uint4*>(p) = make_uint4(pack_bf16(v[0], v[1 % VEC]), pack_bf16(v[2 % VEC], v[3 % VEC]),
                                              pack_bf16(v[4 % VEC], v[5 % VEC]), pack_bf16(v[6 % VEC], v[7 % VEC]));
  } else {
#pragma unroll
    for (int e = 0; e < VEC; ++e)
      if (e < n) put(p + e, v[e]);
  }
}
template <int VEC>
__device__ __forceinline__ void store(__nv_fp8_storage_t* p, int n, const float (&v)[VEC]) {
  if (VEC == 8 && n >= 8) {
    *reinterpret_cast<uint2*>(p) = make_uint2(pack_e4m3(v[0], v[1 % VEC], v[2 % VEC], v[3 % VEC]),
                                              pack_e4m3(v[4 % VEC], v[5 % VEC], v[6 % VEC], v[7 % VEC]));
  } else if (VEC == 4 && n >= 4) {
    *reinterpret_cast<uint32_t*>(p) = pack_e4m3(v[0], v[1 % VEC], v[2 % VEC], v[3 % VEC]);
  } else {
#pragma unroll
    for (int e = 0; e < VEC; ++e)
      if (e < n) put(p + e, v[e]);
  }
}

// ---- element by element over a vector, two at a time where there are two (f32x2: half the issue slots) ----
template <int VEC>
__device__ __forceinline__ void vadd(float (&a)[VEC], const float (&b)[VEC]) {             // a += b
  if (VEC == 1) a[0] += b[0];
#pragma unroll
  for (int e = 0; e + 1 < VEC; e += 2) unpack2(add2(pack2(a[e], a[e + 1]), pack2(b[e], b[e + 1])), a[e], a[e + 1]);
}
template <int VEC>
__device__ __forceinline__ void vmul(float (&a)[VEC], const float (&b)[VEC]) {             // a *= b
  if (VEC == 1) a[0] *= b[0];
#pragma unroll
  for (int e = 0; e + 1 < VEC; e += 2) unpack2(times2(pack2(a[e], a[e + 1]), pack2(b[e], b[e + 1])), a[e], a[e + 1]);
}
template <int VEC>
__device__ __forceinline__ void vscale(float (&a)[VEC], float s) {                         // a *= s
  if (VEC == 1) a[0] *= s;
  const u64 ss = pack2(s, s);
#pragma unroll
  for (int e = 0; e + 1 < VEC; e += 2) unpack2(times2(pack2(a[e], a[e + 1]), ss), a[e], a[e + 1]);
}
template <int VEC>
__device__ __forceinline__ void vfma(float (&c)[VEC], const float (&a)[VEC], const float (&b)[VEC]) {   // c += a b
  if (VEC == 1) c[0] = fmaf(a[0], b[0], c[0]);
#pragma unroll
  for (int e = 0; e + 1 < VEC; e += 2)
    unpack2(fmadd2(pack2(a[e], a[e + 1]), pack2(b[e], b[e + 1]), pack2(c[e], c[e + 1])), c[e], c[e + 1]);
}
template <int VEC>
__device__ __forceinline__ void vfma(float (&c)[VEC], const float (&a)[VEC], float s) {    // c += a s
  if (VEC == 1) c[0] = fmaf(a[0], s, c[0]);
  const u64 ss = pack2(s, s);
#pragma unroll
  for (int e = 0; e + 1 < VEC; e += 2) unpack2(fmadd2(pack2(a[e], a[e + 1]), ss, pack2(c[e], c[e + 1])), c[e], c[e + 1]);
}
template <int VEC>
__device__ __forceinline__ void vdot(float (&c)[2], const float (&a)[VEC], const float (&b)[VEC]) {     // c: two sums of products
  if (VEC == 1) c[0] = fmaf(a[0], b[0], c[0]);
  u64 acc = pack2(c[0], c[1]);
#pragma unroll
  for (int e = 0; e + 1 < VEC; e += 2) acc = fmadd2(pack2(a[e], a[e + 1]), pack2(b[e], b[e + 1]), acc);
  if (VEC > 1) unpack2(acc, c[0], c[1]);
}

// ---- rows on their way to shared memory ahead of their use (cp.async) ----
// Aligned rows (VEC > 1): a thread copies its own accesses of 16 bytes and reads back those alone, so that no barrier stands
// between.  Other rows (VEC = 1): the threads of the row copy the aligned 16 bytes that it touches (the first of them may begin
// with the end of the row before; past its end nothing is read), and read elements after a barrier.
__device__ __forceinline__ void ahead16(uint32_t to, const void* from) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
}
__device__ __forceinline__ void ahead16(uint32_t to, const void* from, int bytes) {         // the rest is filled with zeros
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(bytes) : "memory");
}
// How a row fills its threads' accesses: it ends inside one, with one, or it fills all of them
enum { ROW_PART = 0, ROW_WHOLE = 1, ROW_FULL = 2 };
template <class T, int VEC, int NV, int FILL>
struct Ahead {
  // bytes of one row of one tensor for `threads` threads of which `width` share a row
  static __host__ __device__ __forceinline__ uint32_t row_bytes(int M, int threads, int width) {
    if (VEC > 1) return (uint32_t)(NV * threads * 16);
    return (uint32_t)((M * (int)sizeof(T) + 15) / 16 * 16 + 16) * (threads / width);
  }
  // room: shared address of this tensor's row; t: the thread's place in its group
  static __device__ __forceinline__ void fetch(uint32_t room, const T* row, int M, int t, int width) {
    const int tid = threadIdx.x, nt = blockDim.x;
    if (VEC > 1) {
#pragma unroll
      for (int k = 0; k < NV; ++k) {
        const int c = (t + k * width) * VEC;
        if (FILL == ROW_FULL || c + VEC <= M) ahead16(room + (uint32_t)(k * nt + tid) * 16u, row + (uint32_t)c);
      }
    } else {
      const uintptr_t a = reinterpret_cast<uintptr_t>(row), a0 = a & ~(uintptr_t)15, end = a + (uintptr_t)M * sizeof(T);
      const uint32_t at = room + (uint32_t)(tid / width) * row_bytes(M, 1, 1);
      for (uintptr_t p = a0 + 16 * t; p < end; p += 16 * width) {
        const int left = (int)(end - p < 16 ? end - p : 16);
        ahead16(at + (uint32_t)(p - a0), reinterpret_cast<const void*>(p), left);
      }
    }
  }
  // this thread's k-th access, elements c .. c + VEC of the row, n of them valid (zeros in place of the others)
  static __device__ __forceinline__ void get(const uint8_t* room, const T* row, int M, int width, int k, int c, int n, float (&o)[VEC]) {
    const int tid = threadIdx.x;
    if (VEC > 1) {
      if (FILL == ROW_FULL || (FILL == ROW_WHOLE ? n > 0 : n >= VEC)) load<VEC>(reinterpret_cast<const T*>(room + (k * (int)blockDim.x + tid) * 16), VEC, 0.f, o);
      else load<VEC>(row + c, FILL == ROW_WHOLE ? 0 : n, 0.f, o);
    } else {
      const uint8_t* at = room + (tid / width) * row_bytes(M, 1, 1) + (reinterpret_cast<uintptr_t>(row) & 15);
      o[0] = n > 0 ? to_f(reinterpret_cast<const T*>(at)[c]) : 0.f;
    }
  }
  // n elements at most; a whole access or none where rows are whole
  template <class Y>
  static __device__ __forceinline__ void keep(Y* p, int n, const float (&v)[VEC]) {
    if (FILL == ROW_FULL) store<VEC>(p, VEC, v);
    else if (FILL == ROW_WHOLE) { if (n > 0) store<VEC>(p, VEC, v); }
    else store<VEC>(p, n, v);
  }
  static __device__ __forceinline__ void plain(const float* p, int n, float (&v)[VEC]) {
    load<VEC>(p, FILL == ROW_FULL ? VEC : FILL == ROW_WHOLE ? (n > 0 ? VEC : 0) : n, 0.f, v);
  }
};
__device__ __forceinline__ void ahead_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void ahead_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }   // all but the last N groups

// A value as its own type holds it.
__device__ __forceinline__ float held(float v, const float*) { return v; }
__device__ __forceinline__ float held(float v, const __nv_bfloat16*) { return __bfloat162float(__float2bfloat16_rn(v)); }

// 2^x, relative error about 2^-22; 0 below 2^-126, infinity above the range, NaN for NaN.
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// 1 / x within one unit in the last place
__device__ __forceinline__ float rcp(float x) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}

// The larger of two numbers, a NaN if one of them is.
__device__ __forceinline__ float max_keep_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}

struct Sum { __device__ static float of(float a, float b) { return a + b; } };
struct MaxAbs { __device__ static float of(float a, float b) { return max_keep_nan(a, b); } };

// One value for each group of `width` threads (a power of two, 32 or more, within the CTA), the same bits in every thread: lanes
// in pairs, then warps in pairs.  Every thread of the CTA comes here; buf: a float for each warp of the CTA, not used
// again before another barrier of the CTA.
template <class Op>
__device__ __forceinline__ float over_group(float v, int width, float* buf) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v = Op::of(v, __shfl_xor_sync(0xffffffffu, v, o));
  if (width == 32) return v;
  const int w = threadIdx.x >> 5, per = width >> 5, lane = threadIdx.x & 31;
  if (lane == 0) buf[w] = v;
  __syncthreads();
  v = buf[(w & ~(per - 1)) + (lane & (per - 1))];
  for (int o = per >> 1; o > 0; o >>= 1) v = Op::of(v, __shfl_xor_sync(0xffffffffu, v, o));
  return v;
}

}  // namespace rows

// ---- host: argument checks shared by these operators ----
inline bool aligned_to(const void* p, size_t bytes) { return (reinterpret_cast<uintptr_t>(p) % bytes) == 0; }
// bytes from the first to the last element of a row-major matrix
inline uint64_t matrix_span(int64_t rows, int64_t cols, int64_t ld, int elem) {
  return ((uint64_t)(rows - 1) * (uint64_t)ld + (uint64_t)cols) * (uint64_t)elem;
}
inline bool overlap(const void* a, uint64_t na, const void* b, uint64_t nb) {
  if (!a || !b) return false;
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return x < y + nb && y < x + na;
}

}  // namespace fw
#endif
