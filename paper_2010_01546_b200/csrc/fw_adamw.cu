// AdamW over all tensors of a network: clipping by the norm of all gradients, states in 32 or 8 bits, bf16 copies.
//
//   m <- b1 m + (1 - b1) c g     v <- b2 v + (1 - b2) (c g)^2
//   p <- p (1 - lr decay) - lr m / (1 - b1^t) / (sqrt(v / (1 - b2^t)) + eps)
//
// Every element is read once and written once (the gradient twice with clipping): HBM bandwidth bounds it, with 8-bit
// states their arithmetic too.  A warp takes turns of a few blocks of 256 neighbouring elements, which are what shares a scale in 8-bit states;
// the turns of all tensors follow one another and the warps of the grid take every n-th, so that tensors of any size are one launch.
// 371M parameters with copies and clipping 1.82-1.87 ms (5.6-5.7 TB/s), without clipping 1.67-1.71; 168M with 8-bit states 0.59-0.63 ms (4.3-4.5 TB/s).
//
// 8-bit states.  An average that moves by 1 - beta a step stands still where it is rounded to the nearest code of three mantissa bits, so
// codes are taken by chance: m's in proportion to its share of the way between two codes, sqrt(v)'s in proportion to v's share
// between their squares (by its own share v would grow: a code is up to 1/8 off, whose square is 0.1 % of v a step).  Scales are powers of
// two: they leave a number on the same codes while the largest of its 256 moves.
#include <algorithm>
#include <cmath>
#include <cstdio>
#include <cstring>
#include <new>
#include <vector>

#include "fw_norm.cuh"

namespace fw {
namespace {

using namespace norm;

constexpr int kBlock = 256;              // elements of a warp's turn, and of a scale
constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kMaxTensors = 65536;
// Tensors of a launch: their gradients' addresses travel as parameters, which may be 4 KB in all
constexpr int kPerLaunch = 440;
// Blocks of a warp's turn at most.  Its tensor is looked up once for them, and in 8-bit states the scales come and go together: with a byte a
// block 168M parameters took 550 us, with two 501, four 468, eight 457 and sixteen 461.
__host__ __device__ constexpr int most_blocks(bool s8) { return s8 ? 8 : 4; }
constexpr int kNormCtasPerSm = 8;

struct __align__(16) Tensor {             // in the workspace, from fw_adamw_create
  float* p;
  __nv_bfloat16* copy;                   // or null
  int64_t n;
  int64_t first;                         // its first block among all
  int64_t runs;                          // turns up to its end, among those of its launch
  float decay;
  int32_t aligned;                       // p and copy take whole accesses
};

struct Control {                         // in the workspace
  int64_t step;                          // steps taken
  float clip;                            // factor of this step's gradients
  int32_t skip;                          // this step is left out
  int32_t status;                        // a step has been left out since the last look
  uint32_t done;                         // CTAs of the present launch that are through
};

struct Grads {
  const void* g[kPerLaunch];
  uint8_t kind[kPerLaunch];              // bit 0: bf16, bit 1: takes accesses of four elements, bit 2: of 16 bytes
};

struct Args {
  const Tensor* tensors;                 // of this launch
  Control* control;
  void *m, *v;
  uint8_t *m_scale, *v_scale;
  const float* lr_factor;
  int64_t runs;                          // this launch's
  int32_t each;                          // elements of a warp's turn
  int32_t n;
  int32_t last;                          // the step's last launch
  int32_t clipped;
  uint32_t seed;
  float lr, eps;
  double beta1, beta2;
};

struct NormArgs {
  const Tensor* tensors;
  Control* control;
  double* part;
  float* norm_out;
  int64_t runs;
  int32_t each;                          // elements of a warp's turn
  int32_t n, part0, parts;               // parts: of all launches so far and this one
  int32_t last;
  float max_norm;
};

// 1 - beta^n, the power by squares in 64 bits (1e-15)
__device__ double one_minus_power(double beta, int64_t n) {
  double r = 1.0;
  for (; n > 0; n >>= 1) {
    if (n & 1) r *= beta;
    beta *= beta;
  }
  return 1.0 - r;
}

// A published integer hash of two multiplications (C. Wellons, 2018), with its constants
__device__ __forceinline__ uint32_t mix(uint32_t x) {
  x ^= x >> 16; x *= 0x7feb352du;
  x ^= x >> 15; x *= 0x846ca68bu;
  return x ^ (x >> 16);
}

// A lane's eight of a block's 256: four from 4 lane on and four from 128 + 4 lane on, so that the accesses of a warp lie next to
// each other.
__device__ __forceinline__ int place(int e, int lane) { return (e & 4) * 32 + 4 * lane + (e & 3); }

__device__ __forceinline__ void get4(const float* p, float* o) {
  const float4 q = __ldcs(reinterpret_cast<const float4*>(p));
  o[0] = q.x; o[1] = q.y; o[2] = q.z; o[3] = q.w;
}
__device__ __forceinline__ void get4(const __nv_bfloat16* p, float* o) {
  const uint2 q = __ldcs(reinterpret_cast<const uint2*>(p));
  o[0] = bf16_lo(q.x); o[1] = bf16_hi(q.x); o[2] = bf16_lo(q.y); o[3] = bf16_hi(q.y);
}
__device__ __forceinline__ void put4(float* p, const float* v) { __stcs(reinterpret_cast<float4*>(p), make_float4(v[0], v[1], v[2], v[3])); }
__device__ __forceinline__ void put4(__nv_bfloat16* p, const float* v) {
  __stcs(reinterpret_cast<uint2*>(p), make_uint2(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])));
}
// The block at p, `left` elements of it there (0 in the place of the others); WHOLE: all, four elements at a time
template <bool WHOLE, class T>
__device__ __forceinline__ void get_block(const T* p, int64_t left, int lane, float (&o)[8]) {
  if (WHOLE) {
    get4(p + 4 * lane, o);
    get4(p + 128 + 4 * lane, o + 4);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) o[e] = place(e, lane) < left ? to_f(p[place(e, lane)]) : 0.f;
  }
}
// The launch's tensors in shared memory; the CTA meets behind it
__device__ __forceinline__ const Tensor* table_of(const Tensor* from, int n, uint8_t* room) {
  const uint4* q = reinterpret_cast<const uint4*>(from);
  uint4* to = reinterpret_cast<uint4*>(room);
  for (int i = threadIdx.x; i < n * (int)(sizeof(Tensor) / 16); i += kThreads) to[i] = q[i];
  __syncthreads();
  return reinterpret_cast<const Tensor*>(room);
}
// From tensor t on, the first that ends behind place b: 32 tensors looked at by the lanes of a warp
template <class F>
__device__ __forceinline__ int advance(int t, int n, int lane, F ended) {
  uint32_t m;
  do {
    m = __ballot_sync(0xffffffffu, t + lane < n && ended(t + lane));
    t += __popc(m);
  } while (m == 0xffffffffu);
  return t;
}

// Whether this CTA is the last of its grid; the others' writes before are then visible.  The count is back at 0 after it.
__device__ bool last_cta(uint32_t* done) {
  __shared__ bool last;
  __threadfence();
  __syncthreads();
  if (threadIdx.x == 0) {
    last = atomicAdd(done, 1u) == gridDim.x - 1;
    if (last) *done = 0;
  }
  __syncthreads();
  if (last) __threadfence();
  return last;
}

// Sum of the squares of n neighbouring elements, of whole blocks four at a time
template <class T>
__device__ __forceinline__ void squares(const T* p, int n, bool aligned, int lane, float (&acc)[2]) {
  constexpr int VEC = 16 / sizeof(T), N = kBlock / (32 * VEC);
  const int blocks = aligned ? n / kBlock : 0;
  for (int j = 0; j < blocks; j += 4) {
    uint4 q[4 * N];
#pragma unroll
    for (int k = 0; k < 4 * N; ++k) {
      q[k] = make_uint4(0, 0, 0, 0);
      if (j + k / N < blocks) q[k] = __ldcs(reinterpret_cast<const uint4*>(p + j * kBlock) + k * 32 + lane);
    }
#pragma unroll
    for (int k = 0; k < 4 * N; ++k) {
      float x[VEC];
      if (VEC == 8) {
        x[0] = bf16_lo(q[k].x); x[1] = bf16_hi(q[k].x); x[2] = bf16_lo(q[k].y); x[3] = bf16_hi(q[k].y);
        x[4 % VEC] = bf16_lo(q[k].z); x[5 % VEC] = bf16_hi(q[k].z); x[6 % VEC] = bf16_lo(q[k].w); x[7 % VEC] = bf16_hi(q[k].w);
      } else {
        x[0] = __uint_as_float(q[k].x); x[1] = __uint_as_float(q[k].y); x[2] = __uint_as_float(q[k].z); x[3] = __uint_as_float(q[k].w);
      }
      vdot<VEC>(acc, x, x);
    }
  }
  for (int c = blocks * kBlock + lane; c < n; c += 32) {
    const float x = to_f(p[c]);
    acc[0] = fmaf(x, x, acc[0]);
  }
}

// Squares of all gradients, a warp's turn at a time: fp32 sums of those, 64 bits beyond; the last CTA adds the CTAs' in order.
__global__ void __launch_bounds__(kThreads) adamw_norm_kernel(const __grid_constant__ NormArgs a, const __grid_constant__ Grads g) {
  extern __shared__ __align__(16) uint8_t room[];
  __shared__ double red[kWarps];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  dep_wait();
  const Tensor* tensors = table_of(a.tensors, a.n, room);
  double sum = 0.0;
  int t = 0;
  for (int64_t run = (int64_t)blockIdx.x * kWarps + warp; run < a.runs; run += (int64_t)gridDim.x * kWarps) {
    t = advance(t, a.n, lane, [&](int i) { return run >= tensors[i].runs; });
    const int64_t at = (run - (t > 0 ? tensors[t - 1].runs : 0)) * a.each, left = tensors[t].n - at;
    float acc[2] = {0.f, 0.f};
    const int kind = g.kind[t], n = left < a.each ? (int)left : a.each;
    if (kind & 1) squares(static_cast<const __nv_bfloat16*>(g.g[t]) + at, n, (kind & 4) != 0, lane, acc);
    else squares(static_cast<const float*>(g.g[t]) + at, n, (kind & 4) != 0, lane, acc);
    sum += (double)(acc[0] + acc[1]);
  }
  sum = warp_sum(sum);
  if (lane == 0) red[warp] = sum;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int k = 1; k < kWarps; ++k) sum += red[k];
    a.part[a.part0 + blockIdx.x] = sum;
  }
  const bool last = last_cta(&a.control->done);
  dep_trigger();
  if (!last || !a.last) return;
  double all = 0.0;
  for (int k = threadIdx.x; k < a.parts; k += kThreads) all += __ldcg(a.part + k);
  all = warp_sum(all);
  __syncthreads();
  if (lane == 0) red[warp] = all;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int k = 1; k < kWarps; ++k) all += red[k];
    const double norm = sqrt(all);
    const bool finite = norm <= 1.7976931348623157e308;
    if (a.norm_out) *a.norm_out = (float)norm;
    a.control->clip = finite && norm > (double)a.max_norm ? (float)((double)a.max_norm / norm) : 1.f;
    a.control->skip = !finite;
    if (!finite) a.control->status = 1;
  }
}

// ---- 8-bit states ----
// The least power of two 2^(b - 127) that takes top to 448 = 1.75 2^8 or less, 2^-100 at least
__device__ __forceinline__ uint32_t scale_byte(float top) {
  const uint32_t w = __float_as_uint(top);
  const int b = (int)(w >> 23) - 8 + ((w & 0x7fffffu) > 0x600000u ? 1 : 0);
  return b < 27 ? 27u : (uint32_t)b;
}
// The same for the root of top: 448^2 = 1.53125 2^17
__device__ __forceinline__ uint32_t root_scale_byte(float top) {
  const bool low = top < 0x1p-100f;                          // it may be subnormal
  const uint32_t w = __float_as_uint(low ? top * 0x1p96f : top);
  const int n = (int)(w >> 23) - (low ? 240 : 144) + ((w & 0x7fffffu) > 0x440000u ? 1 : 0), b = 127 + ((n + 1) >> 1);
  return b < 27 ? 27u : (uint32_t)b;
}
__device__ __forceinline__ float scale_of(uint32_t b) { return __uint_as_float(b << 23); }
__device__ __forceinline__ float inverse_square(uint32_t b) { return __uint_as_float((381u - 2u * b) << 23); }      // 64 <= b <= 190
// Codes of e4m3 are the upper bits of fp32 numbers times 2^-120: both have their least exponent there, and what lies below it is a
// number of smallest codes in both.
constexpr float kDown = 0x1p-120f, kUp = 0x1p120f;
constexpr uint32_t kStep = 0x100000u;    // from one code to the next
constexpr float kMost = 3.402823466e38f; // the largest finite number
// The top bytes of four words
__device__ __forceinline__ uint32_t top_bytes(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  return __byte_perm(__byte_perm(a, b, 0x0073), __byte_perm(c, d, 0x0073), 0x5410);
}
// Relative error 2^-23, of subnormal numbers too: a v of gradients below 1e-18 is one, and eps may be less than its root
__device__ __forceinline__ float root(float x) {
  float r;
  asm("sqrt.approx.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
__device__ __forceinline__ float root_ftz(float x) {
  float r;
  asm("sqrt.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
// Four of m to codes, up where the share of the way and chance / 2^16 reach 1; down: 2^-120 over the scale; x: the elements' hashes, whose
// lower halves are the chance
__device__ __forceinline__ uint32_t mean_codes(float (&m)[4], float down, const uint32_t (&x)[4]) {
  uint32_t w[4];
  vscale<4>(m, down);
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const uint32_t bits = __float_as_uint(m[e]), chance = __byte_perm(x[e] ^ (x[e] >> 16), 0, 0x4104);      // in bits 8 to 23
    w[e] = (((bits << 4) + chance) & 0x7fffffffu) | (bits & 0x80000000u);
  }
  return top_bytes(w[0], w[1], w[2], w[3]);
}
// Four v >= 0 to the codes of their roots, up where v's share of the way between the codes' squares passes (chance + 1/2) / 2^16, chance the
// hashes' upper halves; what is not 0 is not held as 0.  v: over the square of the scale, 448^2 at most (480^2: the NaN's code).  The share is
// v's own: the root, which may be a step off, tells only which two codes, and beside a code either pair gives that one.
__device__ __forceinline__ uint32_t root_codes(const float (&v)[4], const uint32_t (&x)[4]) {
  uint32_t c[4], w[4];
  float y[4], low[4], high[4], f[4], lhs[4], d[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) y[e] = root_ftz(v[e]);
  // from 2^-6 on, where almost all are, numbers and codes have their leading bits in common but for the exponent's origin
  const bool plain = fminf(fminf(y[0], y[1]), fminf(y[2], y[3])) >= 0x1p-6f;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    f[e] = __uint_as_float(0x3f800000u | ((x[e] >> 9) & 0x7fff80u));      // 1 + chance / 2^16
    lhs[e] = 0x1p-17f - 1.f;
    low[e] = y[e];
  }
  vadd<4>(f, lhs);                                           // (chance + 1/2) / 2^16
  if (!plain) vscale<4>(low, kDown);
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    c[e] = __float_as_uint(low[e]) & 0xfff00000u;
    low[e] = __uint_as_float(c[e]);
    high[e] = __uint_as_float(c[e] + kStep);
  }
  if (!plain) {
    vscale<4>(low, kUp);
    vscale<4>(high, kUp);
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) lhs[e] = -low[e];
  vmul<4>(lhs, low);                                         // - low^2, exact
#pragma unroll
  for (int e = 0; e < 4; ++e) d[e] = lhs[e];
  vfma<4>(d, high, high);                                    // high^2 - low^2, exact
  vadd<4>(lhs, v);                                           // v - low^2, rounded once
  vmul<4>(f, d);
  const uint32_t origin = plain ? 120u << 27 : 0u;           // of the exponent, four bits up
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    w[e] = lhs[e] > f[e] ? c[e] + kStep : c[e];
    if (!plain) w[e] = max(w[e], v[e] > 0.f ? kStep : 0u);
    w[e] = (w[e] << 4) - origin;
  }
  return top_bytes(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ void from_e4m3(uint32_t w, float (&o)[4]) {
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(w >> (16 * k)), __NV_E4M3);
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h));
    o[2 * k] = f.x;
    o[2 * k + 1] = f.y;
  }
}
__device__ __forceinline__ float warp_max(float v) {
  float r;
  asm("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(v));
  return r;
}
__device__ __forceinline__ float warp_max_keep_nan(float v) {
  float r;
  asm("redux.sync.max.NaN.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(v));
  return r;
}

// What a step's blocks share
struct Step {
  float lr, step, inv_root, beta1, beta2, c1, c2, eps;       // c1, c2: the clipping factor times 1 - beta1, root of 1 - beta2
  uint32_t key;
};

template <bool S8> struct StateBits;
template <> struct StateBits<false> {
  float m[8], v[8];
  __device__ __forceinline__ void load(const Args& a, int64_t b, int lane) {
    get_block<true>(static_cast<const float*>(a.m) + b * kBlock, kBlock, lane, m);
    get_block<true>(static_cast<const float*>(a.v) + b * kBlock, kBlock, lane, v);
  }
};
template <> struct StateBits<true> {
  uint32_t m[2], v[2];
  __device__ __forceinline__ void load(const Args& a, int64_t b, int lane) {
    const uint32_t* mw = static_cast<const uint32_t*>(a.m) + b * (kBlock / 4) + lane;
    const uint32_t* vw = static_cast<const uint32_t*>(a.v) + b * (kBlock / 4) + lane;
    m[0] = __ldcs(mw); m[1] = __ldcs(mw + 32); v[0] = __ldcs(vw); v[1] = __ldcs(vw + 32);
  }
};
// A block's place
struct Where {
  float* p;
  __nv_bfloat16* copy;
  const void* g;
  int left;                              // elements there, 256 at most
  float keep;
  bool half, aligned;                    // gradients in bf16; all takes accesses of four elements
  __device__ __forceinline__ bool whole() const { return aligned && left == kBlock; }
};
// A lane's part of a block as it is loaded
template <bool S8>
struct Bits {
  float p[8];
  uint32_t g[8];                         // four words of them bf16
  StateBits<S8> s;
  __device__ __forceinline__ void load(const Args& a, const Where& w, int64_t b, int lane) {
    s.load(a, b, lane);
    if (w.whole()) {
      get_block<true>(w.p, kBlock, lane, p);
      if (w.half) {
        const uint2 x = __ldcs(static_cast<const uint2*>(w.g) + lane), y = __ldcs(static_cast<const uint2*>(w.g) + 32 + lane);
        g[0] = x.x; g[1] = x.y; g[2] = y.x; g[3] = y.y;
      } else {
        const uint4 x = __ldcs(static_cast<const uint4*>(w.g) + lane), y = __ldcs(static_cast<const uint4*>(w.g) + 32 + lane);
        g[0] = x.x; g[1] = x.y; g[2] = x.z; g[3] = x.w; g[4] = y.x; g[5] = y.y; g[6] = y.z; g[7] = y.w;
      }
    } else {
      get_block<false>(w.p, w.left, lane, p);
      float v[8];
      if (w.half) {
        get_block<false>(static_cast<const __nv_bfloat16*>(w.g), w.left, lane, v);
#pragma unroll
        for (int e = 0; e < 4; ++e) g[e] = pack_bf16(v[2 * e], v[2 * e + 1]);
      } else {
        get_block<false>(static_cast<const float*>(w.g), w.left, lane, v);
#pragma unroll
        for (int e = 0; e < 8; ++e) g[e] = __float_as_uint(v[e]);
      }
    }
  }
  // the k-th four gradients
  __device__ __forceinline__ void open(bool half, int k, float (&o)[4]) const {
    if (half) {
#pragma unroll
      for (int e = 0; e < 2; ++e) { o[2 * e] = bf16_lo(g[2 * k + e]); o[2 * e + 1] = bf16_hi(g[2 * k + e]); }
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] = __uint_as_float(g[4 * k + e]);
    }
  }
};

// Four elements at p, of which n are there (or all, at once)
template <class T>
__device__ __forceinline__ void put_four(T* p, int n, bool whole, const float (&v)[4]) {
  if (whole) {
    put4(p, v);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (e < n) put(p + e, v[e]);
  }
}

// The step of block b, four elements of a lane at a time (all eight at once took 80 registers and more)
template <bool S8>
__device__ __forceinline__ void update(const Args& a, const Step& st, const Bits<S8>& in, const Where& at, int64_t b, int lane, uint32_t& scale_m, uint32_t& scale_v) {
  float m[2][4], v[2][4];
  const bool whole = at.whole();
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    float p[4], gr[4], q[4];
    in.open(at.half, k, gr);
    if constexpr (S8) {
      from_e4m3(in.s.m[k], m[k]);
      from_e4m3(in.s.v[k], v[k]);
      if ((in.s.v[k] + 0x01010101u) & 0x80808080u) {         // a NaN's code: infinity
#pragma unroll
        for (int e = 0; e < 4; ++e) v[k][e] = fminf(v[k][e], INFINITY);
      }
      vscale<4>(m[k], scale_of(scale_m) * st.beta1);         // a power of two: no rounding but beta1's product
      const float s = scale_of(scale_v);
      if (scale_v >= 70) {                                   // its square is in range
        vmul<4>(v[k], v[k]);
        vscale<4>(v[k], s * s * st.beta2);
      } else {
        vscale<4>(v[k], s);
        vmul<4>(v[k], v[k]);
        vscale<4>(v[k], st.beta2);
      }
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) { m[k][e] = in.s.m[4 * k + e]; v[k][e] = in.s.v[4 * k + e]; }
      vscale<4>(m[k], st.beta1);
      vscale<4>(v[k], st.beta2);
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) { p[e] = in.p[4 * k + e]; q[e] = gr[e]; }
    vfma<4>(m[k], gr, st.c1);
    vscale<4>(q, st.c2);
    vfma<4>(v[k], q, q);                                     // the square of a scaled gradient: a factor's own square may be out of range
    float r[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      r[e] = root(v[k][e]);
      q[e] = st.eps;
    }
    vfma<4>(q, r, st.inv_root);
#pragma unroll
    for (int e = 0; e < 4; ++e) q[e] = rcp(q[e]);
    vmul<4>(q, m[k]);
    vscale<4>(p, at.keep);
    vfma<4>(p, q, -st.step);
    const int c = 128 * k + 4 * lane;
    put_four(at.p + c, at.left - c, whole, p);
    if (at.copy) put_four(at.copy + c, at.left - c, whole, p);
    if (!S8) {
      put4(static_cast<float*>(a.m) + b * kBlock + c, m[k]);
      put4(static_cast<float*>(a.v) + b * kBlock + c, v[k]);
    }
  }
  if constexpr (S8) {
    float tm = 0.f, tv = 0.f;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      tm = fmaxf(tm, fmaxf(fabsf(m[0][e]), fabsf(m[1][e])));
      tv = max_keep_nan(tv, max_keep_nan(v[0][e], v[1][e]));
    }
    tv = warp_max_keep_nan(tv);
    const bool none = !(tv <= kMost);
    if (none) {
      // An element whose v is not finite takes no part in the scales, which would hold the others' as nothing: the code of its root is the
      // NaN's, that of its m, which takes no step any more, 0.
      tm = tv = 0.f;
#pragma unroll
      for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if (v[k][e] <= kMost) tv = fmaxf(tv, v[k][e]);
          else { v[k][e] = INFINITY; m[k][e] = 0.f; }
          tm = fmaxf(tm, fabsf(m[k][e]));
        }
      tv = warp_max(tv);
    }
    uint32_t bm = scale_byte(warp_max(tm)), bv = root_scale_byte(tv);
    scale_m = bm;
    scale_v = bv;
    if (bm > 156) {                                          // 2^-120 over the scale is out of range
      vscale<4>(m[0], 0x1p-100f);
      vscale<4>(m[1], 0x1p-100f);
      bm -= 100;
    }
    if (!none && bv - 64u < 64u) {
      vscale<4>(v[0], inverse_square(bv));
      vscale<4>(v[1], inverse_square(bv));
    } else {
      // 1 over the scale's square may be out of range; what is not 0 stays so, however far below the largest
      const float first = bv < 64 ? 0x1p80f : 1.f, second = inverse_square(bv < 64 ? bv + 40 : bv);
#pragma unroll
      for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int e = 0; e < 4; ++e) v[k][e] = fminf(fmaxf(v[k][e] * first * second, fminf(v[k][e], 0x1p-100f)), 480.f * 480.f);
    }
    const float down = __uint_as_float(bm < 134 ? (134u - bm) << 23 : 0x400000u >> (bm - 134));
    // mix(i ^ key) of this lane's elements: its first step is the same for all but the lower 8 bits
    uint32_t first = ((uint32_t)(b * kBlock) + 4u * lane) ^ st.key;
    first ^= first >> 16;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      uint32_t hash[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        uint32_t h = (first ^ (uint32_t)(128 * k + e)) * 0x7feb352du;
        h ^= h >> 15;
        hash[e] = h * 0x846ca68bu;                           // its last step: the lower half by the upper one
      }
      const int64_t w = b * (kBlock / 4) + 32 * k + lane;
      __stcs(static_cast<uint32_t*>(a.m) + w, mean_codes(m[k], down, hash));
      __stcs(static_cast<uint32_t*>(a.v) + w, root_codes(v[k], hash));
    }
  }
}

template <bool S8>
__global__ void __launch_bounds__(kThreads, S8 ? 3 : 2) adamw_step_kernel(const __grid_constant__ Args a, const __grid_constant__ Grads g) {
  extern __shared__ __align__(16) uint8_t room[];            // table of the tensors
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  dep_wait();
  const Tensor* tensors = table_of(a.tensors, a.n, room);
  const int64_t t1 = a.control->step + 1;
  const float clip = a.clipped ? a.control->clip : 1.f;
  const bool skip = a.clipped && a.control->skip;
  int64_t run = (int64_t)blockIdx.x * kWarps + warp;
  if (!skip && run < a.runs) {
    Step st;
    st.lr = a.lr_factor ? a.lr * *a.lr_factor : a.lr;
    st.step = (float)((double)st.lr / one_minus_power(a.beta1, t1));
    st.inv_root = (float)(1.0 / sqrt(one_minus_power(a.beta2, t1)));
    st.beta1 = (float)a.beta1; st.beta2 = (float)a.beta2; st.eps = a.eps;
    st.c1 = (float)((1.0 - a.beta1) * clip); st.c2 = (float)(sqrt(1.0 - a.beta2) * clip);
    st.key = mix(a.seed ^ ((uint32_t)t1 * 0x9e3779b9u));
    int t = 0;
    for (; run < a.runs; run += (int64_t)gridDim.x * kWarps) {
      t = advance(t, a.n, lane, [&](int i) { return run >= tensors[i].runs; });
      const Tensor x = tensors[t];
      const int64_t at = (run - (t > 0 ? tensors[t - 1].runs : 0)) * a.each;
      const int kind = g.kind[t];
      int left = x.n - at < a.each ? (int)(x.n - at) : a.each;
      int64_t b = x.first + at / kBlock;
      Where w;
      w.p = x.p + at;
      w.copy = x.copy ? x.copy + at : nullptr;
      w.half = kind & 1;
      w.g = static_cast<const char*>(g.g[t]) + at * (w.half ? 2 : 4);
      w.keep = fmaf(-st.lr, x.decay, 1.f);
      w.aligned = x.aligned && (kind & 2);
      // scales: a lane each, all of the turn at once (single bytes of scattered warps took a quarter of the time)
      const int blocks = (left + kBlock - 1) / kBlock;
      uint32_t bm = 0, bv = 0;
      if (S8 && lane < blocks) { bm = a.m_scale[b + lane]; bv = a.v_scale[b + lane]; }
      const int64_t b0 = b;
#pragma unroll 1
      for (int j = 0; j < blocks; ++j, ++b, left -= kBlock) {
        w.left = left < kBlock ? left : kBlock;
        uint32_t sm = S8 ? __shfl_sync(0xffffffffu, bm, j) : 0, sv = S8 ? __shfl_sync(0xffffffffu, bv, j) : 0;
        Bits<S8> in;
        in.load(a, w, b, lane);
        update<S8>(a, st, in, w, b, lane, sm, sv);
        if (lane == j) { bm = sm; bv = sv; }
        w.p += kBlock;
        if (w.copy) w.copy += kBlock;
        w.g = static_cast<const char*>(w.g) + kBlock * (w.half ? 2 : 4);
      }
      if (S8 && lane < blocks) { a.m_scale[b0 + lane] = (uint8_t)bm; a.v_scale[b0 + lane] = (uint8_t)bv; }
    }
  }
  const bool last = last_cta(&a.control->done);
  dep_trigger();
  if (last && a.last && threadIdx.x == 0 && !skip) a.control->step = t1;
}

// ---- host ----
constexpr size_t kAlign = 256;
struct Span { uintptr_t at, end; };

}  // namespace
}  // namespace fw

struct fw_adamw {
  fw_adamw_desc d;
  cudaStream_t stream;
  int device;
  int64_t blocks;
  int32_t each;
  std::vector<int64_t>* sizes;
  std::vector<int64_t>* runs;              // as in the table
  std::vector<fw::Span>* out;              // P, copies and the workspace, in order
  fw::Control* control;
  fw::Tensor* tensors;
  double* part;
  void *m, *v;
  uint8_t *m_scale, *v_scale;
};

namespace fw {
namespace {

fw_status desc_check(const fw_adamw_desc* d, const int64_t* sizes, int64_t* blocks) {
  if (!d || !sizes) return FW_ERR_INVALID_ARG;
  if (d->state != FW_F32 && d->state != FW_E4M3) return FW_ERR_INVALID_ARG;
  if (!(d->beta1 >= 0.0 && d->beta1 < 1.0) || !(d->beta2 >= 0.0 && d->beta2 < 1.0) || !(d->eps >= 1e-36f && d->eps <= 3e38f)) return FW_ERR_INVALID_ARG;
  if (d->n < 1 || d->n > kMaxTensors) return FW_ERR_SHAPE;
  const int64_t most = (int64_t)1 << (d->state == FW_E4M3 ? 32 : 40);      // the chance counts elements in 32 bits
  int64_t b = 0;
  for (int i = 0; i < d->n; ++i) {
    if (sizes[i] < 1 || sizes[i] > most) return FW_ERR_SHAPE;
    b += (sizes[i] + kBlock - 1) / kBlock;
    if (b > most / kBlock) return FW_ERR_SHAPE;
  }
  *blocks = b;
  return FW_OK;
}

int norm_ctas(int64_t runs) {
  const int64_t most = (int64_t)kNormCtasPerSm * sm_count(), want = (runs + kWarps - 1) / kWarps;
  return (int)(want < most ? want : most);
}
int launches(int n) { return (n + kPerLaunch - 1) / kPerLaunch; }

size_t carve(const fw_adamw_desc& d, int64_t blocks, char* base, fw_adamw* a) {
  size_t at = 0;
  auto take = [&](size_t bytes) {
    char* p = base ? base + at : nullptr;
    at += (bytes + kAlign - 1) / kAlign * kAlign;
    return p;
  };
  const size_t each = d.state == FW_F32 ? 4 : 1;
  char* control = take(sizeof(Control));
  char* tensors = take((size_t)d.n * sizeof(Tensor));
  char* part = take((size_t)launches(d.n) * kNormCtasPerSm * sm_count() * sizeof(double));
  char* m = take((size_t)blocks * kBlock * each);
  char* v = take((size_t)blocks * kBlock * each);
  char* ms = d.state == FW_E4M3 ? take((size_t)blocks) : nullptr;
  char* vs = d.state == FW_E4M3 ? take((size_t)blocks) : nullptr;
  if (a) {
    a->control = (Control*)control; a->tensors = (Tensor*)tensors; a->part = (double*)part; a->m = m; a->v = v;
    a->m_scale = (uint8_t*)ms; a->v_scale = (uint8_t*)vs;
  }
  return at;
}

bool meets(const std::vector<Span>& sorted, uintptr_t at, uintptr_t end) {
  auto it = std::upper_bound(sorted.begin(), sorted.end(), at, [](uintptr_t x, const Span& s) { return x < s.end; });
  return it != sorted.end() && it->at < end;
}

void release(fw_adamw* a) {
  if (!a) return;
  delete a->sizes;
  delete a->runs;
  delete a->out;
  delete a;
}

template <bool S8>
cudaError_t launch_step(const Args& q, const Grads& g, cudaStream_t s) {
  static FillCache cache;
  const size_t smem = (size_t)q.n * sizeof(Tensor);
  int ctas = 0;
  const cudaError_t e = fill(adamw_step_kernel<S8>, cache, kThreads, smem, (q.runs + kWarps - 1) / kWarps, 1 << 30, &ctas);
  return e != cudaSuccess ? e : launch_dep(adamw_step_kernel<S8>, (unsigned)ctas, kThreads, smem, s, q, g);
}

}  // namespace
}  // namespace fw

using namespace fw;

extern "C" {

void fw_adamw_desc_default(fw_adamw_desc* d, int32_t n) {
  if (!d) return;
  d->n = n; d->state = FW_F32; d->beta1 = 0.9; d->beta2 = 0.999; d->eps = 1e-8f; d->seed = 0;
}

size_t fw_adamw_workspace_bytes(const fw_adamw_desc* d, const int64_t* sizes) {
  int64_t blocks = 0;
  if (desc_check(d, sizes, &blocks) != FW_OK) return 0;
  return carve(*d, blocks, nullptr, nullptr);
}

fw_status fw_adamw_create(const fw_adamw_desc* d, const int64_t* sizes, float* const* P, void* const* copies, const float* decay,
                          void* dev_workspace, size_t bytes, void* cuda_stream, fw_adamw** out) {
  if (!out) return FW_ERR_INVALID_ARG;
  *out = nullptr;
  if (!d || !sizes || !P || !dev_workspace) return FW_ERR_INVALID_ARG;
  int64_t blocks = 0;
  const fw_status st = desc_check(d, sizes, &blocks);
  if (st != FW_OK) return st;
  const size_t need = carve(*d, blocks, nullptr, nullptr);
  if (!aligned_to(dev_workspace, kAlign) || bytes < need) return FW_ERR_WORKSPACE;
  fw_adamw* a = nullptr;
  try {
    a = new fw_adamw();
    a->sizes = new std::vector<int64_t>(sizes, sizes + d->n);
    a->runs = new std::vector<int64_t>(d->n);
    a->out = new std::vector<Span>();
    a->out->reserve(2 * (size_t)d->n + 1);
    a->d = *d;
    a->blocks = blocks;
    a->stream = (cudaStream_t)cuda_stream;
    carve(*d, blocks, (char*)dev_workspace, a);
    std::vector<Tensor> table(d->n);
    auto add = [&](const void* p, uint64_t n) { a->out->push_back({(uintptr_t)p, (uintptr_t)p + n}); };
    add(dev_workspace, need);
    // a turn for every warp of the chip first
    const int64_t turn = blocks / ((int64_t)sm_count() * 3 * kWarps), most = most_blocks(d->state == FW_E4M3);
    const int64_t each = (turn < 1 ? 1 : turn < most ? turn : most) * kBlock;
    a->each = (int32_t)each;
    int64_t b = 0;
    for (int i = 0; i < d->n; ++i) {
      Tensor& t = table[i];
      void* c = copies ? copies[i] : nullptr;
      const float wd = decay ? decay[i] : 0.f;
      if (!P[i] || !aligned_to(P[i], 4) || !aligned_to(c, 2) || !(wd >= 0.f && wd <= 3e38f)) { release(a); return FW_ERR_INVALID_ARG; }
      t.p = P[i]; t.copy = (__nv_bfloat16*)c; t.n = sizes[i]; t.decay = wd;
      t.aligned = aligned_to(P[i], 16) && aligned_to(c, 8);
      t.first = b;
      b += (sizes[i] + kBlock - 1) / kBlock;
      t.runs = (i % kPerLaunch ? table[i - 1].runs : 0) + (sizes[i] + each - 1) / each;
      (*a->runs)[i] = t.runs;
      add(P[i], (uint64_t)sizes[i] * 4);
      if (c) add(c, (uint64_t)sizes[i] * 2);
    }
    std::sort(a->out->begin(), a->out->end(), [](const Span& x, const Span& y) { return x.at < y.at; });
    for (size_t i = 1; i < a->out->size(); ++i)
      if ((*a->out)[i].at < (*a->out)[i - 1].end) { release(a); return FW_ERR_INVALID_ARG; }
    int ndev = 0;
    if (cudaGetDeviceCount(&ndev) != cudaSuccess || ndev < 1 || cudaGetDevice(&a->device) != cudaSuccess) {
      cudaGetLastError();
      fprintf(stderr, "[fw] no CUDA device: this library has no CPU path\n");
      release(a);
      return FW_ERR_CUDA;
    }
    cudaError_t e = cudaMemsetAsync(dev_workspace, 0, need, a->stream);
    if (e == cudaSuccess && d->state == FW_E4M3) e = cudaMemsetAsync(a->m_scale, 27, (size_t)blocks, a->stream);
    if (e == cudaSuccess && d->state == FW_E4M3) e = cudaMemsetAsync(a->v_scale, 27, (size_t)blocks, a->stream);
    // from pageable memory: `table` has been read when the call returns
    if (e == cudaSuccess) e = cudaMemcpyAsync(a->tensors, table.data(), table.size() * sizeof(Tensor), cudaMemcpyHostToDevice, a->stream);
    if (e != cudaSuccess) {
      release(a);
      return failed(e, "fw_adamw_create");
    }
  } catch (const std::bad_alloc&) {
    release(a);
    return FW_ERR_INVALID_ARG;
  }
  *out = a;
  return FW_OK;
}

fw_status fw_adamw_destroy(fw_adamw* a) {
  if (!a) return FW_ERR_INVALID_ARG;
  release(a);
  return FW_OK;
}

fw_status fw_adamw_step(fw_adamw* a, const void* const* G, const int32_t* g_dtype, float lr, const float* lr_factor, float max_norm,
                        float* norm_out) {
  if (!a || !G || !(lr >= 0.f && lr <= 3e38f) || !(max_norm >= 0.f) || !aligned_to(lr_factor, 4) || !aligned_to(norm_out, 4)) return FW_ERR_INVALID_ARG;
  if (norm_out && max_norm == 0.f) return FW_ERR_INVALID_ARG;
  const int n = a->d.n;
  const uintptr_t no = (uintptr_t)norm_out, lo = (uintptr_t)lr_factor;
  if ((norm_out && meets(*a->out, no, no + 4)) || (lr_factor && (meets(*a->out, lo, lo + 4) || (no && no < lo + 4 && lo < no + 4)))) return FW_ERR_INVALID_ARG;
  for (int i = 0; i < n; ++i) {
    const int kind = g_dtype ? g_dtype[i] : FW_F32;
    if (!G[i] || (kind != FW_F32 && kind != FW_BF16)) return FW_ERR_INVALID_ARG;
    const int es = kind == FW_F32 ? 4 : 2;
    const uintptr_t at = (uintptr_t)G[i], end = at + (uint64_t)(*a->sizes)[i] * es;
    if (at % es || meets(*a->out, at, end) || (no && no < end && at < no + 4)) return FW_ERR_INVALID_ARG;
  }
  int dev = -1;
  if (cudaGetDevice(&dev) != cudaSuccess) { cudaGetLastError(); return FW_ERR_CUDA; }
  if (dev != a->device) return FW_ERR_INVALID_ARG;
  const bool s8 = a->d.state == FW_E4M3;
  cudaError_t e = cudaSuccess;
  Grads g;
  auto fill = [&](int i0, int i1) {
    for (int i = i0; i < i1; ++i) {
      const bool half = g_dtype && g_dtype[i] == FW_BF16;
      g.g[i - i0] = G[i];
      g.kind[i - i0] = (uint8_t)((half ? 1 : 0) | (aligned_to(G[i], half ? 8 : 16) ? 2 : 0) | (aligned_to(G[i], 16) ? 4 : 0));
    }
  };
  const bool clipped = max_norm > 0.f;
  if (clipped) {
    int parts = 0;
    for (int i0 = 0; i0 < n && e == cudaSuccess; i0 += kPerLaunch) {
      const int i1 = std::min(n, i0 + kPerLaunch);
      fill(i0, i1);
      NormArgs q;
      q.tensors = a->tensors + i0; q.control = a->control; q.part = a->part; q.norm_out = norm_out;
      q.runs = (*a->runs)[i1 - 1]; q.each = a->each; q.n = i1 - i0;
      const int ctas = norm_ctas(q.runs);
      q.part0 = parts; parts += ctas; q.parts = parts; q.last = i1 == n; q.max_norm = max_norm;
      ProfScope ps(FW_PROF_MISC, a->stream);
      e = launch_dep(adamw_norm_kernel, ctas, kThreads, (size_t)q.n * sizeof(Tensor), a->stream, q, g);
    }
  }
  for (int i0 = 0; i0 < n && e == cudaSuccess; i0 += kPerLaunch) {
    const int i1 = std::min(n, i0 + kPerLaunch);
    if (n > kPerLaunch || !clipped) fill(i0, i1);
    Args q;
    q.tensors = a->tensors + i0; q.control = a->control; q.m = a->m; q.v = a->v; q.m_scale = a->m_scale; q.v_scale = a->v_scale;
    q.lr_factor = lr_factor; q.runs = (*a->runs)[i1 - 1]; q.each = a->each; q.n = i1 - i0; q.last = i1 == n;
    q.clipped = clipped; q.seed = a->d.seed; q.lr = lr; q.beta1 = a->d.beta1; q.beta2 = a->d.beta2; q.eps = a->d.eps;
    ProfScope ps(FW_PROF_MISC, a->stream);
    e = s8 ? launch_step<true>(q, g, a->stream) : launch_step<false>(q, g, a->stream);
  }
  return failed(e, "fw_adamw_step");
}

fw_status fw_adamw_state(fw_adamw* a, int32_t field, void** address, size_t* bytes) {
  if (!a || !address || !bytes) return FW_ERR_INVALID_ARG;
  const bool s8 = a->d.state == FW_E4M3;
  const size_t n = (size_t)a->blocks * kBlock * (s8 ? 1 : 4);
  switch (field) {
    case FW_A_M: *address = a->m; *bytes = n; return FW_OK;
    case FW_A_V: *address = a->v; *bytes = n; return FW_OK;
    case FW_A_M_SCALE:
    case FW_A_V_SCALE:
      if (!s8) return FW_ERR_UNSUPPORTED;
      *address = field == FW_A_M_SCALE ? a->m_scale : a->v_scale;
      *bytes = (size_t)a->blocks;
      return FW_OK;
    case FW_A_STEP: *address = &a->control->step; *bytes = sizeof(int64_t); return FW_OK;
  }
  return FW_ERR_INVALID_ARG;
}

fw_status fw_adamw_sync_status(fw_adamw* a) {
  if (!a) return FW_ERR_INVALID_ARG;
  int32_t code = 0;
  cudaError_t e = cudaMemcpyAsync(&code, &a->control->status, sizeof(code), cudaMemcpyDeviceToHost, a->stream);
  if (e == cudaSuccess) e = cudaStreamSynchronize(a->stream);
  if (e == cudaSuccess && code) e = cudaMemsetAsync(&a->control->status, 0, sizeof(code), a->stream);
  if (e != cudaSuccess) return failed(e, "fw_adamw_sync_status");
  return code ? FW_WARN_NONFINITE : FW_OK;
}

}  // extern "C"
