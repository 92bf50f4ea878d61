// AdamW over all tensors of a network: clipping by the norm of all gradients, states in 32 or 8 bits, bf16 copies.
//
//   m <- b1 m + (1 - b1) c g     v <- b2 v + (1 - b2) (c g)^2
//   p <- p (1 - lr decay) - lr m / (1 - b1^t) / (sqrt(v / (1 - b2^t)) + eps)
//
// Every element is read once and written once (the gradient twice with clipping): HBM bandwidth bounds it.  A warp takes 256
// neighbouring elements of one tensor at a time, which are what shares a scale in 8-bit states; CTAs take equal shares of all of them in
// order, so that tensors of any size are one launch.
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

#include "fw_internal.h"
#include "fw_rows.cuh"

namespace fw {
namespace {

using namespace rows;

constexpr int kBlock = 256;              // elements of a warp's turn, and of a scale
constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kMaxTensors = 65536;
// Tensors of a launch: their gradients' addresses travel as parameters, which may be 4 KB in all
constexpr int kPerLaunch = 440;
constexpr int kNormCtasPerSm = 8;

struct Tensor {                          // in the workspace, from fw_adamw_create
  float* p;
  __nv_bfloat16* copy;                   // or null
  int64_t n;
  int64_t first, last;                   // its blocks among all
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
  uint8_t kind[kPerLaunch];              // bit 0: bf16, bit 1: takes whole accesses
};

struct Args {
  const Tensor* tensors;                 // of this launch
  Control* control;
  void *m, *v;
  uint8_t *m_scale, *v_scale;
  const float* lr_factor;
  int64_t first, blocks;                 // this launch's
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
  int64_t first, blocks;
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
// The block at p, `left` elements of it there (0 in the place of the others); whole: 16 bytes (8 of bf16) at a time
template <class T>
__device__ __forceinline__ void get_block(const T* p, int64_t left, bool whole, int lane, float (&o)[8]) {
  if (whole && left >= kBlock) {
    get4(p + 4 * lane, o);
    get4(p + 128 + 4 * lane, o + 4);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) o[e] = place(e, lane) < left ? to_f(p[place(e, lane)]) : 0.f;
  }
}
template <class T>
__device__ __forceinline__ void put_block(T* p, int64_t left, bool whole, int lane, const float (&v)[8]) {
  if (whole && left >= kBlock) {
    put4(p + 4 * lane, v);
    put4(p + 128 + 4 * lane, v + 4);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (place(e, lane) < left) put(p + place(e, lane), v[e]);
  }
}
__device__ __forceinline__ void get_grad(const Grads& g, int t, int64_t at, int64_t left, int lane, float (&o)[8]) {
  const int kind = g.kind[t];
  if (kind & 1) get_block(static_cast<const __nv_bfloat16*>(g.g[t]) + at, left, (kind & 2) != 0, lane, o);
  else get_block(static_cast<const float*>(g.g[t]) + at, left, (kind & 2) != 0, lane, o);
}

// The tensor of block b: the last one that begins at b or before
__device__ __forceinline__ int tensor_of(const Tensor* t, int n, int64_t b) {
  int lo = 0, hi = n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (t[mid].first <= b) lo = mid;
    else hi = mid - 1;
  }
  return lo;
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

// Squares of all gradients: fp32 sums of a thread's elements, 64 bits beyond; the last CTA adds the CTAs' in order.
__global__ void __launch_bounds__(kThreads) adamw_norm_kernel(const __grid_constant__ NormArgs a, const __grid_constant__ Grads g) {
  __shared__ double red[kWarps];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  dep_wait();
  const int64_t b0 = a.first + a.blocks * blockIdx.x / gridDim.x, b1 = a.first + a.blocks * (blockIdx.x + 1) / gridDim.x;
  double sum = 0.0;
  if (b0 + warp < b1) {
    int t = tensor_of(a.tensors, a.n, b0 + warp);
    float acc[8] = {};
    for (int64_t b = b0 + warp; b < b1; b += kWarps) {
      while (b >= a.tensors[t].last) ++t;
      const int64_t at = (b - a.tensors[t].first) * kBlock;
      float x[8];
      get_grad(g, t, at, a.tensors[t].n - at, lane, x);
#pragma unroll
      for (int e = 0; e < 8; ++e) acc[e] = fmaf(x[e], x[e], acc[e]);
    }
    sum = (double)((acc[0] + acc[1]) + (acc[2] + acc[3])) + (double)((acc[4] + acc[5]) + (acc[6] + acc[7]));
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
constexpr float kTiny = 0.015625f;       // 2^-6: below it codes are 2^-9 apart; above, three bits behind the leading one
// The least power of two 2^(b - 127) that takes top to 448 = 1.75 2^8 or less, 2^-100 at least
__device__ __forceinline__ uint32_t scale_byte(float top) {
  const uint32_t w = __float_as_uint(top);
  const int b = (int)(w >> 23) - 8 + ((w & 0x7fffffu) > 0x600000u ? 1 : 0);
  return b < 27 ? 27u : (uint32_t)b;
}
__device__ __forceinline__ float scale_of(uint32_t b) { return __uint_as_float(b << 23); }
__device__ __forceinline__ float inverse_scale(uint32_t b) { return __uint_as_float((254u - b) << 23); }
// a >= 0 up or down to a code, up where the share of the way and chance / 2^16 reach 1
__device__ __forceinline__ float code_of(float a, uint32_t chance) {
  const float shift = a < kTiny ? kTiny : 0.f;               // codes 2^-9 apart up to 2^-5
  return __uint_as_float((__float_as_uint(a + shift) + (chance << 4)) & 0xfff00000u) - shift;
}
// r >= 0 up or down, up where the share of r^2 on the way between the codes' squares passes (chance + 1/2) / 2^16
__device__ __forceinline__ float root_code_of(float r, uint32_t chance) {
  const float shift = r < kTiny ? kTiny : 0.f;
  const uint32_t w = __float_as_uint(r + shift) & 0xfff00000u;
  const float low = __uint_as_float(w) - shift, high = __uint_as_float(w + 0x100000u) - shift;
  const float c = fmaf((float)chance, 0x1p-16f, 0x1p-17f);
  const float code = (r - low) * (r + low) > c * ((high - low) * (high + low)) ? high : low;
  return r > 0.f ? fmaxf(code, 0x1p-9f) : code;
}
__device__ __forceinline__ void from_e4m3(uint32_t w, float* o) {
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
// Within one unit in the last place
__device__ __forceinline__ float root(float x) {
  float r;
  asm("sqrt.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}

template <bool S8>
__global__ void __launch_bounds__(kThreads) adamw_step_kernel(const __grid_constant__ Args a, const __grid_constant__ Grads g) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  dep_wait();
  const int64_t t1 = a.control->step + 1;
  const float clip = a.clipped ? a.control->clip : 1.f;
  const bool skip = a.clipped && a.control->skip;
  const int64_t b0 = a.first + a.blocks * blockIdx.x / gridDim.x, b1 = a.first + a.blocks * (blockIdx.x + 1) / gridDim.x;
  if (!skip && b0 + warp < b1) {
    const float lr = a.lr_factor ? a.lr * *a.lr_factor : a.lr;
    const float step = (float)((double)lr / one_minus_power(a.beta1, t1));
    const float inv_root = (float)(1.0 / sqrt(one_minus_power(a.beta2, t1)));
    const float beta1 = (float)a.beta1, beta2 = (float)a.beta2, c1 = (float)(1.0 - a.beta1), c2 = (float)(1.0 - a.beta2);
    const uint32_t key = mix(a.seed ^ ((uint32_t)t1 * 0x9e3779b9u));
    int t = tensor_of(a.tensors, a.n, b0 + warp);
    Tensor x = a.tensors[t];
    for (int64_t b = b0 + warp; b < b1; b += kWarps) {
      while (b >= x.last) x = a.tensors[++t];
      const int64_t at = (b - x.first) * kBlock, left = x.n - at;
      float p[8], gr[8], m[8], v[8];
      get_block(x.p + at, left, x.aligned, lane, p);
      get_grad(g, t, at, left, lane, gr);
      if (S8) {
        const uint32_t* mw = static_cast<const uint32_t*>(a.m) + b * (kBlock / 4) + lane;
        const uint32_t* vw = static_cast<const uint32_t*>(a.v) + b * (kBlock / 4) + lane;
        const uint32_t m0 = __ldcs(mw), m1 = __ldcs(mw + 32), v0 = __ldcs(vw), v1 = __ldcs(vw + 32);
        const float sm = scale_of(a.m_scale[b]), sv = scale_of(a.v_scale[b]);
        from_e4m3(m0, m); from_e4m3(m1, m + 4);
        from_e4m3(v0, v); from_e4m3(v1, v + 4);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          m[e] *= sm;
          v[e] *= sv;
          v[e] *= v[e];
        }
      } else {
        get_block(static_cast<const float*>(a.m) + b * kBlock, kBlock, true, lane, m);
        get_block(static_cast<const float*>(a.v) + b * kBlock, kBlock, true, lane, v);
      }
      const float keep = (float)(1.0 - (double)lr * x.decay);
      float r[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float gc = gr[e] * clip;
        m[e] = fmaf(beta1, m[e], c1 * gc);
        v[e] = fmaf(beta2, v[e], c2 * gc * gc);
        r[e] = root(v[e]);
        p[e] = fmaf(-step, __fdividef(m[e], fmaf(r[e], inv_root, a.eps)), p[e] * keep);
      }
      put_block(x.p + at, left, x.aligned, lane, p);
      if (x.copy) put_block(x.copy + at, left, x.aligned, lane, p);
      if (S8) {
        float tm = 0.f, tr = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          tm = fmaxf(tm, fabsf(m[e]));
          tr = fmaxf(tr, r[e]);
        }
        const uint32_t bm = scale_byte(warp_max(tm)), bv = scale_byte(warp_max(tr));
        const float im = inverse_scale(bm), iv = inverse_scale(bv);
        const uint32_t i0 = (uint32_t)(b * kBlock);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const uint32_t chance = mix((i0 + place(e, lane)) ^ key);
          m[e] = copysignf(code_of(fabsf(m[e]) * im, chance & 0xffffu), m[e]);
          v[e] = root_code_of(r[e] * iv, chance >> 16);
        }
        uint32_t* mw = static_cast<uint32_t*>(a.m) + b * (kBlock / 4) + lane;
        uint32_t* vw = static_cast<uint32_t*>(a.v) + b * (kBlock / 4) + lane;
        __stcs(mw, pack_e4m3(m[0], m[1], m[2], m[3]));
        __stcs(mw + 32, pack_e4m3(m[4], m[5], m[6], m[7]));
        __stcs(vw, pack_e4m3(v[0], v[1], v[2], v[3]));
        __stcs(vw + 32, pack_e4m3(v[4], v[5], v[6], v[7]));
        if (lane == 0) {
          a.m_scale[b] = (uint8_t)bm;
          a.v_scale[b] = (uint8_t)bv;
        }
      } else {
        put_block(static_cast<float*>(a.m) + b * kBlock, kBlock, true, lane, m);
        put_block(static_cast<float*>(a.v) + b * kBlock, kBlock, true, lane, v);
      }
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
  std::vector<int64_t>* sizes;
  std::vector<int64_t>* first;             // first block of each tensor, and the number of all
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
  if (!(d->beta1 >= 0.0 && d->beta1 < 1.0) || !(d->beta2 >= 0.0 && d->beta2 < 1.0) || !(d->eps > 0.f && d->eps <= 3e38f)) return FW_ERR_INVALID_ARG;
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

int norm_ctas(int64_t blocks) {
  const int64_t most = (int64_t)kNormCtasPerSm * sm_count(), want = (blocks + kWarps - 1) / kWarps;
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

fw_status failed(cudaError_t e, const char* where) {
  if (e == cudaSuccess) return FW_OK;
  fprintf(stderr, "[fw] %s: %s\n", where, cudaGetErrorString(e));
  return FW_ERR_CUDA;
}

void release(fw_adamw* a) {
  if (!a) return;
  delete a->sizes;
  delete a->first;
  delete a->out;
  delete a;
}

template <bool S8>
cudaError_t step_ctas(int* per_sm) {
  static std::mutex mu;
  static int known = 0;
  std::lock_guard<std::mutex> lock(mu);
  if (!known) {
    int n = 0;
    const cudaError_t e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, adamw_step_kernel<S8>, kThreads, 0);
    if (e != cudaSuccess) return e;
    known = n > 0 ? n : 1;
  }
  *per_sm = known;
  return cudaSuccess;
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
    a->first = new std::vector<int64_t>(d->n + 1);
    a->out = new std::vector<Span>();
    a->out->reserve(2 * (size_t)d->n + 1);
    a->d = *d;
    a->blocks = blocks;
    a->stream = (cudaStream_t)cuda_stream;
    carve(*d, blocks, (char*)dev_workspace, a);
    std::vector<Tensor> table(d->n);
    auto add = [&](const void* p, uint64_t n) { a->out->push_back({(uintptr_t)p, (uintptr_t)p + n}); };
    add(dev_workspace, need);
    int64_t b = 0;
    for (int i = 0; i < d->n; ++i) {
      Tensor& t = table[i];
      void* c = copies ? copies[i] : nullptr;
      const float wd = decay ? decay[i] : 0.f;
      if (!P[i] || !aligned_to(P[i], 4) || !aligned_to(c, 2) || !(wd >= 0.f && wd <= 3e38f)) { release(a); return FW_ERR_INVALID_ARG; }
      t.p = P[i]; t.copy = (__nv_bfloat16*)c; t.n = sizes[i]; t.decay = wd;
      t.aligned = aligned_to(P[i], 16) && aligned_to(c, 8);
      t.first = (*a->first)[i] = b;
      b += (sizes[i] + kBlock - 1) / kBlock;
      t.last = b;
      add(P[i], (uint64_t)sizes[i] * 4);
      if (c) add(c, (uint64_t)sizes[i] * 2);
    }
    (*a->first)[d->n] = b;
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
  int per_sm = 0;
  cudaError_t e = s8 ? step_ctas<true>(&per_sm) : step_ctas<false>(&per_sm);
  Grads g;
  auto fill = [&](int i0, int i1) {
    for (int i = i0; i < i1; ++i) {
      const bool half = g_dtype && g_dtype[i] == FW_BF16;
      g.g[i - i0] = G[i];
      g.kind[i - i0] = (uint8_t)((half ? 1 : 0) | (aligned_to(G[i], half ? 8 : 16) ? 2 : 0));
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
      q.first = (*a->first)[i0]; q.blocks = (*a->first)[i1] - q.first; q.n = i1 - i0;
      const int ctas = norm_ctas(q.blocks);
      q.part0 = parts; parts += ctas; q.parts = parts; q.last = i1 == n; q.max_norm = max_norm;
      ProfScope ps(FW_PROF_MISC, a->stream);
      e = launch_dep(adamw_norm_kernel, ctas, kThreads, 0, a->stream, q, g);
    }
  }
  for (int i0 = 0; i0 < n && e == cudaSuccess; i0 += kPerLaunch) {
    const int i1 = std::min(n, i0 + kPerLaunch);
    if (n > kPerLaunch || !clipped) fill(i0, i1);
    Args q;
    q.tensors = a->tensors + i0; q.control = a->control; q.m = a->m; q.v = a->v; q.m_scale = a->m_scale; q.v_scale = a->v_scale;
    q.lr_factor = lr_factor; q.first = (*a->first)[i0]; q.blocks = (*a->first)[i1] - q.first; q.n = i1 - i0; q.last = i1 == n;
    q.clipped = clipped; q.seed = a->d.seed; q.lr = lr; q.beta1 = a->d.beta1; q.beta2 = a->d.beta2; q.eps = a->d.eps;
    const int64_t want = (q.blocks + kWarps - 1) / kWarps, most = (int64_t)per_sm * sm_count();
    ProfScope ps(FW_PROF_MISC, a->stream);
    e = launch_dep(s8 ? adamw_step_kernel<true> : adamw_step_kernel<false>, (unsigned)(want < most ? want : most), kThreads, 0, a->stream, q, g);
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
