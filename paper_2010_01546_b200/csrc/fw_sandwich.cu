// The norms behind a block and before the next one with the gate and the residual addition between them, forward and backward.
//
//   n1 = o rstd1 (or o)      h = alpha x + k w_post n1, kept in the type of x      n2 = h rstd2      y = n2 w_pre
//   e4m3 y: c = max |y| / 448, y is held as e4m3(y / c) with c beside it
//
//   u2 = dy w_pre     t = rstd2 (u2 - n2 mean(u2 n2)) + dh     dx = alpha t     dw_pre = sum over the rows of dy n2
//   u1 = t w_post     do = k rstd1 (u1 - n1 mean(u1 n1)) (or k u1)     dw_post = sum over the rows of k t n1     dk = sum of u1 n1
//
// Both directions read each element once and write each result once: HBM bandwidth bounds them.  A row stays on chip between its two
// sums, which depend on one another, so a CTA has the next rows on their way meanwhile, and backward forms two rows at once where they are
// short enough.  8192 x 4096 bf16: forward 49-52 us (5.2-5.5 TB/s), backward 74-79 us (5.1-5.4 TB/s), of which 7 are the
// sum of the CTAs' shares of dw; 5003 x 1537 fp32 backward 45 us (4.1 TB/s).
#include "fw_norm.cuh"

namespace fw {
namespace {

using namespace norm;

// How aligned accesses of a thread meet its rows.  Rows whose matrices all lie equally past 16 bytes (SHIFT) are taken by such accesses too:
// the first of a row may hold the row before's elements, what lies behind the row the copy fills with zeros.  How far a row lies past them repeats every 16 bytes / element rows, so a CTA
// takes rows of one residue, and its columns stay its own; the weights wait in shared memory, moved as the row is.  (Element by element,
// backward of 5003 x 1537 fp32: 82 us.)
// Aligned rows that end inside an access (TAIL) are taken the same way.  (Their last elements read one by one where
// they are used, which all warps of the row waited for: 8192 x 4095 bf16 backward 134 us, so 87.)
enum { ROW_SHIFT = 3, ROW_TAIL = 4 };
template <class T, int VEC, int NV, int FILL>
struct Way {
  static constexpr bool MOVED = FILL == ROW_SHIFT || FILL == ROW_TAIL;
  static constexpr bool ZEROS = VEC > 1 && (FILL == ROW_WHOLE || MOVED);      // in accesses behind the row, see zeros()
  typedef Ahead<T, VEC, NV, MOVED ? ROW_PART : FILL> Ring;
  int M, t, width, shift;
  // bytes of a row of one tensor
  static __host__ __device__ __forceinline__ uint32_t row_bytes(int M, int width) {
    return VEC > 1 && !ZEROS ? (uint32_t)((M + VEC - 1) / VEC * 16) : Ring::row_bytes(M, width, width);
  }
  // bytes of a row of weights, where they wait in shared memory
  static __host__ __device__ __forceinline__ uint32_t weight_bytes(int width) { return MOVED ? (uint32_t)(NV * width * VEC * sizeof(float)) : 0u; }
  __device__ __forceinline__ int column(int k) const { return (t + k * width) * VEC - (FILL == ROW_SHIFT ? shift : 0); }
  __device__ __forceinline__ bool inside(int c) const { return c >= 0 && c + VEC <= M; }
  __device__ __forceinline__ void fetch(uint32_t room, const T* row) const {
    if (!MOVED) {
      Ring::fetch(room, row, M, t, width);
    } else {
#pragma unroll
      for (int k = 0; k < NV; ++k) {
        const int c = column(k);
        const uint32_t to = room + (uint32_t)(k * (int)blockDim.x + (int)threadIdx.x) * 16u;
        if (c < M) ahead16(to, row + c, M - c < VEC ? (M - c) * (int)sizeof(T) : 16);
      }
    }
  }
  __device__ __forceinline__ void get(const uint8_t* room, const T* row, int k, float (&v)[VEC]) const {
    const int c = column(k);
    if (ZEROS) {
      load<VEC>(reinterpret_cast<const T*>(room + (k * (int)blockDim.x + (int)threadIdx.x) * 16), VEC, 0.f, v);
      if (FILL == ROW_SHIFT && k == 0 && c < 0) {            // what the row before has there
#pragma unroll
        for (int e = 0; e < VEC - 1; ++e)
          if (c + e < 0) v[e] = 0.f;
      }
    } else {
      Ring::get(room, row, M, width, k, c, M - c, v);
    }
  }
  template <class Y>
  __device__ __forceinline__ void keep(Y* row, int k, const float (&v)[VEC]) const {
    const int c = column(k);
    if (!MOVED) {
      Ring::keep(row + c, M - c, v);
    } else if (inside(c)) {
      store<VEC>(row + c, VEC, v);
    } else {
#pragma unroll
      for (int e = 0; e < VEC; ++e)
        if (c + e >= 0 && c + e < M) put(row + c + e, v[e]);
    }
  }
  // Zeros in the accesses of n rows that lie behind a row's end: once, so that no reading of them asks (8192 x 4095 bf16 backward 98 us with that)
  __device__ __forceinline__ void zeros(uint8_t* room, uint32_t stride, int n) const {
    if (!ZEROS) return;
    for (int k = 0; k < NV; ++k)
      if (column(k) >= M)
        for (int i = 0; i < n; ++i) *reinterpret_cast<uint4*>(room + i * stride + (k * (int)blockDim.x + (int)threadIdx.x) * 16) = make_uint4(0, 0, 0, 0);
  }
  // a row of weights, or its place in shared memory
  __device__ __forceinline__ void weights(const float* w, const float* moved, int k, float (&v)[VEC]) const {
    if (!MOVED) Ring::plain(w + column(k), M - column(k), v);
    else load<VEC>(moved + (t + k * width) * VEC, VEC, 0.f, v);
  }
  __device__ __forceinline__ void move(const float* w, float* moved) const {
    for (int i = t; i < NV * width * VEC; i += width) moved[i] = i - shift >= 0 && i - shift < M ? w[i - shift] : 0.f;
  }
};

struct SandwichFwd {
  const void *o, *x;
  const float *w1, *gate, *w2;   // w_post or null, a number a row or null, w_pre
  void *h, *y;
  float *y_scale, *rstd;
  int64_t rows, ldo, ldx, ldh, ldy;
  int32_t M, width, post, classes;   // classes: of rows that lie unequally past 16 bytes, 0: by other ways
  float eps, inv_M, alpha;
};

// Warps that a CTA's numbers are counted for when one warp joins them
__device__ __forceinline__ int warp_span() {
  const int warps = blockDim.x >> 5;
  return warps <= 4 ? 4 : warps <= 8 ? 8 : 16;
}
// One value over the CTA, the same bits in every thread; 0 is nothing to Op.  buf: a float for each warp, not used again before another
// barrier of the CTA
template <class Op>
__device__ __forceinline__ float over_row(float v, float* buf) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v = Op::of(v, __shfl_xor_sync(0xffffffffu, v, o));
  const int warps = blockDim.x >> 5, lane = threadIdx.x & 31, span = warp_span(), at = lane & (span - 1);
  if (warps == 1) return v;
  if (lane == 0) buf[threadIdx.x >> 5] = v;
  __syncthreads();
  v = at < warps ? buf[at] : 0.f;
  for (int o = span >> 1; o > 0; o >>= 1) v = Op::of(v, __shfl_xor_sync(0xffffffffu, v, o));
  return v;
}

// As norm_forward_kernel: T is the type of o, x and h, Y of y; VEC elements an access, NV accesses a thread, SLOTS rows of a CTA on
// their way, a row at a time.
template <class T, class Y, int VEC, int NV, int SLOTS, int FILL>
__global__ void __maxnreg__(96) sandwich_forward_kernel(const SandwichFwd p) {
  typedef Way<T, VEC, NV, FILL> Rows;
  extern __shared__ __align__(16) uint8_t room[];            // [slot][o, x], with SHIFT w_post and w_pre
  __shared__ float buf[2][3][16];
  const int t = threadIdx.x, width = blockDim.x;
  const uint32_t row_bytes = Rows::row_bytes(p.M, width), slot_bytes = row_bytes * 2;
  const uint32_t base = (uint32_t)__cvta_generic_to_shared(room);
  auto o_row = [&](int64_t row) { return static_cast<const T*>(p.o) + row * p.ldo; };
  auto x_row = [&](int64_t row) { return static_cast<const T*>(p.x) + row * p.ldx; };
  // the CTA's rows
  const int first = FILL == ROW_SHIFT ? (int)blockIdx.x % p.classes : 0;
  const int64_t step = FILL == ROW_SHIFT ? (int64_t)gridDim.x / p.classes * p.classes : gridDim.x, begin = blockIdx.x;
  const Rows way = {p.M, t, width, FILL == ROW_SHIFT ? (int)((reinterpret_cast<uintptr_t>(o_row(first)) & 15) / sizeof(T)) : 0};
  float* w1 = reinterpret_cast<float*>(room + SLOTS * slot_bytes);
  float* w2 = w1 + NV * width * VEC;
  auto fetch = [&](int64_t row, int i) {
    if (row < p.rows) {
      way.fetch(base + i * slot_bytes, o_row(row));
      way.fetch(base + i * slot_bytes + row_bytes, x_row(row));
    }
    ahead_commit();
  };
  dep_wait();
#pragma unroll
  for (int i = 0; i < SLOTS; ++i) fetch(begin + i * step, i);
  if (Rows::MOVED) {
    if (p.w1) way.move(p.w1, w1);
    way.move(p.w2, w2);
    __syncthreads();
  }
  way.zeros(room, row_bytes, 2 * SLOTS);
  int i = 0, flip = 0;
  for (int64_t row = begin; row < p.rows; row += step, flip ^= 1) {
    const uint8_t* slot = room + i * slot_bytes;
    const float k1 = p.gate ? p.gate[row] : 1.f;
    ahead_wait<SLOTS - 1>();
    if (VEC == 1) __syncthreads();
    float v[NV][VEC];
    const T *o = o_row(row), *x = x_row(row);
    T* h = static_cast<T*>(p.h) + row * p.ldh;
    float sq[2] = {0.f, 0.f};
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      way.get(slot, o, k, v[k]);
      vdot<VEC>(sq, v[k], v[k]);
    }
    float r1 = 1.f;
    if (p.post) r1 = rsqrtf(fmaf(over_row<Sum>(sq[0] + sq[1], buf[flip][0]), p.inv_M, p.eps));
    const float f = k1 * r1;
    sq[0] = sq[1] = 0.f;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      float a[VEC];
      if (p.w1) {
        way.weights(p.w1, w1, k, a);
        vmul<VEC>(v[k], a);
      }
      vscale<VEC>(v[k], f);
      way.get(slot + row_bytes, x, k, a);
      vfma<VEC>(v[k], a, p.alpha);
      round_pairs(v[k], static_cast<const T*>(nullptr));
      way.keep(h, k, v[k]);
      vdot<VEC>(sq, v[k], v[k]);
    }
    const float r2 = rsqrtf(fmaf(over_row<Sum>(sq[0] + sq[1], buf[flip][1]), p.inv_M, p.eps));
    fetch(row + SLOTS * step, i);              // the slot has been read: the sum of its threads depends on it
    if (t == 0 && p.rstd) { p.rstd[2 * row] = r1; p.rstd[2 * row + 1] = r2; }
    float top = 0.f;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      float w[VEC];
      way.weights(p.w2, w2, k, w);
      if (sizeof(Y) != 1) vscale<VEC>(v[k], r2);             // the scale takes rstd out of an 8-bit y again: y / c = 448 h w / max |h w|
      vmul<VEC>(v[k], w);
      if (sizeof(Y) == 1) {
#pragma unroll
        for (int e = 0; e < VEC; ++e) top = max_keep_nan(top, fabsf(v[k][e]));
      }
    }
    float inv = 1.f;
    if (sizeof(Y) == 1) {
      top = over_row<MaxAbs>(top, buf[flip][2]);
      float scale;
      inv = row_scale(top, r2, &scale);
      if (t == 0) p.y_scale[row] = scale;
      if (by_size(top, r2)) {
#pragma unroll
        for (int k = 0; k < NV; ++k) vscale<VEC>(v[k], r2);
      }
    }
    Y* y = static_cast<Y*>(p.y) + row * p.ldy;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      if (sizeof(Y) == 1) vscale<VEC>(v[k], inv);
      way.keep(y, k, v[k]);
    }
    if (++i == SLOTS) i = 0;
  }
  ahead_wait<0>();
  dep_trigger();
}

struct SandwichBwd {
  const void *dy, *dh, *o, *h;
  const float *w1, *gate, *w2, *rstd;
  void *dx, *d_o;
  float *part, *dgate;           // part: two rows of sums for each CTA (dw_pre, dw_post), part_row(M) apart, or null
  int64_t rows, lddy, lddh, ldo, ldh, lddx, lddo;
  int32_t M, width, post, classes;
  float inv_M, alpha;
};

__host__ __device__ constexpr int part_row(int M) { return (M + 3) / 4 * 4; }

// As norm_backward_kernel, for rows element by element (VEC = 1) and for short ones, several to a CTA: a CTA takes every gridDim-th group
// of rows, a row at a time (SOLO) or several, and keeps its columns' shares of dw_pre and dw_post in registers.  DIRECT: dh is read where it is
// needed: four rows of 64 KB do not fit a SM.
template <class T, int VEC, int NV, int SLOTS, bool DH, int FILL, bool SOLO>
__global__ void __launch_bounds__(512) sandwich_backward_kernel(const SandwichBwd p) {
  typedef Ahead<T, VEC, NV, FILL> Ring;
  constexpr bool DIRECT = DH && VEC == 1;
  constexpr int ROOMS = DH && !DIRECT ? 4 : 3;
  extern __shared__ __align__(16) uint8_t room[];            // [slot][dy, h, o, dh], at the end the groups' sums
  __shared__ float buf[2][2][16];
  const int tid = threadIdx.x, nt = blockDim.x, width = SOLO ? nt : p.width, t = SOLO ? tid : tid & (width - 1);
  const int per = SOLO ? 1 : nt / width, mine = SOLO ? 0 : tid / width;
  const int64_t step = (int64_t)gridDim.x * per;
  const uint32_t row_bytes = Ring::row_bytes(p.M, nt, width), slot_bytes = row_bytes * ROOMS;
  const uint32_t base = (uint32_t)__cvta_generic_to_shared(room);
  auto u_row = [&](int64_t row) { return static_cast<const T*>(p.dy) + row * p.lddy; };
  auto h_row = [&](int64_t row) { return static_cast<const T*>(p.h) + row * p.ldh; };
  auto o_row = [&](int64_t row) { return static_cast<const T*>(p.o) + row * p.ldo; };
  auto d_row = [&](int64_t row) { return static_cast<const T*>(p.dh) + row * p.lddh; };
  auto fetch = [&](int64_t row, int i) {
    if (row < p.rows) {
      const uint32_t at = base + i * slot_bytes;
      Ring::fetch(at, u_row(row), p.M, t, width);
      Ring::fetch(at + row_bytes, h_row(row), p.M, t, width);
      Ring::fetch(at + 2 * row_bytes, o_row(row), p.M, t, width);
      if (ROOMS == 4) Ring::fetch(at + 3 * row_bytes, d_row(row), p.M, t, width);
    }
    ahead_commit();
  };
  struct Head { float r1, r2, k; };
  auto head = [&](int64_t row) {
    Head a = {0.f, 0.f, 0.f};
    if (row < p.rows) a = {p.post ? p.rstd[2 * row] : 1.f, p.rstd[2 * row + 1], p.gate ? p.gate[row] : 1.f};
    return a;
  };
  dep_wait();
  float dw1[NV][VEC], dw2[NV][VEC];
#pragma unroll
  for (int k = 0; k < NV; ++k)
#pragma unroll
    for (int e = 0; e < VEC; ++e) dw1[k][e] = dw2[k][e] = 0.f;
  const int64_t first = (int64_t)blockIdx.x * per;
#pragma unroll
  for (int i = 0; i < SLOTS; ++i) fetch(first + mine + i * step, i);
  Head a = head(first + mine);
  int i = 0, flip = 0;
  for (int64_t row0 = first; row0 < p.rows; row0 += step, flip ^= 1) {
    const int64_t row = row0 + mine;
    const bool live = SOLO || row < p.rows;
    const Head next = head(row + step);
    const uint8_t* slot = room + i * slot_bytes;
    ahead_wait<SLOTS - 1>();
    if (VEC == 1) __syncthreads();
    float u[NV][VEC];
    const T *dy = u_row(row), *h = h_row(row), *o = o_row(row), *dh = DH ? d_row(row) : nullptr;
    float dots[2] = {0.f, 0.f};
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const uint32_t c = (uint32_t)(t + k * width) * VEC;
      const int left = live ? p.M - (int)c : 0;
      float n[VEC], w[VEC];
      Ring::get(slot, dy, p.M, width, k, c, left, u[k]);
      Ring::get(slot + row_bytes, h, p.M, width, k, c, left, n);
      Ring::plain(p.w2 + c, p.M - (int)c, w);
      vscale<VEC>(n, a.r2);
      vfma<VEC>(dw2[k], u[k], n);
      vmul<VEC>(u[k], w);
      vdot<VEC>(dots, u[k], n);
    }
    const float f2 = over_group<Sum>(dots[0] + dots[1], width, buf[flip][0]) * -p.inv_M * a.r2;
    T* dx = static_cast<T*>(p.dx) + row * p.lddx;
    dots[0] = dots[1] = 0.f;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const uint32_t c = (uint32_t)(t + k * width) * VEC;
      const int left = live ? p.M - (int)c : 0;
      float n[VEC], w[VEC];
      Ring::get(slot + row_bytes, h, p.M, width, k, c, left, n);
      vfma<VEC>(u[k], n, f2);                                // u2 - n2 mean(u2 n2)
      vscale<VEC>(u[k], a.r2);
      if (DH) {
        if (DIRECT) load<VEC>(dh + c, left, 0.f, n);
        else Ring::get(slot + 3 * row_bytes, dh, p.M, width, k, c, left, n);
        vadd<VEC>(u[k], n);
      }
#pragma unroll
      for (int e = 0; e < VEC; ++e) n[e] = u[k][e] * p.alpha;
      if (live) Ring::keep(dx + c, p.M - (int)c, n);
      Ring::get(slot + 2 * row_bytes, o, p.M, width, k, c, left, n);
      vscale<VEC>(n, a.r1);
#pragma unroll
      for (int e = 0; e < VEC; ++e) w[e] = n[e] * a.k;
      vfma<VEC>(dw1[k], u[k], w);
      if (p.w1) {
        Ring::plain(p.w1 + c, p.M - (int)c, w);
        vmul<VEC>(u[k], w);
      }
      vdot<VEC>(dots, u[k], n);
    }
    const float dot = over_group<Sum>(dots[0] + dots[1], width, buf[flip][1]);
    if (p.dgate && t == 0 && live) p.dgate[row] = dot;
    const float f1 = p.post ? -dot * p.inv_M * a.r1 : 0.f, scale = a.k * a.r1;      // (r1 = 1 without post)
    T* d_o = static_cast<T*>(p.d_o) + row * p.lddo;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const uint32_t c = (uint32_t)(t + k * width) * VEC;
      const int left = live ? p.M - (int)c : 0;
      float n[VEC];
      Ring::get(slot + 2 * row_bytes, o, p.M, width, k, c, left, n);
      if (p.post) vfma<VEC>(u[k], n, f1);
      vscale<VEC>(u[k], scale);
      if (live) Ring::keep(d_o + c, p.M - (int)c, u[k]);
    }
    // the slot is given away when every thread that reads it has: itself, or (VEC = 1) the row's
    if (VEC == 1) __syncthreads();
    fetch(row + SLOTS * step, i);
    a = next;
    if (++i == SLOTS) i = 0;
  }
  ahead_wait<0>();
  dep_trigger();
  if (!p.part) return;
  // the groups of the CTA in order, then the CTA's rows of sums
  const int apart = part_row(p.M);
  float* out = p.part + (int64_t)blockIdx.x * 2 * apart;
  float* shared = reinterpret_cast<float*>(room);
  if (!SOLO) __syncthreads();
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int c = (t + k * width) * VEC;
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
      if (c + e >= p.M) continue;
      float* to = SOLO ? out + c + e : shared + mine * 2 * apart + c + e;
      to[0] = dw2[k][e];
      to[apart] = dw1[k][e];
    }
  }
  if (SOLO) return;
  __syncthreads();
  for (int c = threadIdx.x; c < 2 * apart; c += blockDim.x) {
    float s = 0.f;
    for (int k = 0; k < per; ++k) s += shared[k * 2 * apart + c];
    out[c] = s;
  }
}

// One sum over the CTA for each of R values, the same bits in every thread; buf: R floats for each warp, not used again before another
// barrier of the CTA
template <int R>
__device__ __forceinline__ void over_cta(float (&v)[R], float* buf) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1)
#pragma unroll
    for (int r = 0; r < R; ++r) v[r] += __shfl_xor_sync(0xffffffffu, v[r], o);
  const int warps = blockDim.x >> 5, lane = threadIdx.x & 31, span = warp_span(), at = lane & (span - 1);
  if (lane == 0)
#pragma unroll
    for (int r = 0; r < R; ++r) buf[r * 16 + (threadIdx.x >> 5)] = v[r];
  __syncthreads();
#pragma unroll
  for (int r = 0; r < R; ++r) v[r] = at < warps ? buf[r * 16 + at] : 0.f;
  for (int o = span >> 1; o > 0; o >>= 1)
#pragma unroll
    for (int r = 0; r < R; ++r) v[r] += __shfl_xor_sync(0xffffffffu, v[r], o);
}

// Aligned rows by CTAs of 128 threads and more: R rows of a CTA at a time, so that their chains of two sums run beside each other and the
// weights are read once for them (a row at a time: 8192 x 4096 bf16 7 us more).  A thread asks for the next rows' elements where it has
// used up its own.
template <class T, int VEC, int NV, int R, bool DH, int FILL>
__global__ void __launch_bounds__(512) sandwich_backward_rows_kernel(const SandwichBwd p) {
  typedef Way<T, VEC, NV, FILL> Rows;
  constexpr bool DIRECT = DH && NV == 8;
  constexpr int ROOMS = DH && !DIRECT ? 4 : 3;
  extern __shared__ __align__(16) uint8_t room[];            // [row][dy, h, o, dh], with SHIFT w_pre and w_post
  __shared__ float buf[2][R * 16];
  const int t = threadIdx.x, width = blockDim.x;
  const uint32_t row_bytes = Rows::row_bytes(p.M, width);
  // rows that follow one another here are `apart` rows apart
  const int apart = FILL == ROW_SHIFT ? p.classes : 1, first = FILL == ROW_SHIFT ? (int)blockIdx.x % p.classes : 0;
  const int64_t step = (FILL == ROW_SHIFT ? (int64_t)gridDim.x / p.classes * p.classes : (int64_t)gridDim.x) * R;
  const uint32_t base = (uint32_t)__cvta_generic_to_shared(room);
  enum { DY, H, O, D };
  auto row_of = [&](int which, int64_t row) {
    return which == DY ? static_cast<const T*>(p.dy) + row * p.lddy : which == H ? static_cast<const T*>(p.h) + row * p.ldh :
           which == O ? static_cast<const T*>(p.o) + row * p.ldo : static_cast<const T*>(p.dh) + row * p.lddh;
  };
  const Rows way = {p.M, t, width, FILL == ROW_SHIFT ? (int)((reinterpret_cast<uintptr_t>(row_of(DY, first)) & 15) / sizeof(T)) : 0};
  float* w2 = reinterpret_cast<float*>(room + R * ROOMS * row_bytes);
  float* w1 = w2 + NV * width * VEC;
  auto fetch = [&](int which, int64_t row0) {
#pragma unroll
    for (int r = 0; r < R; ++r)
      if (row0 + r * apart < p.rows) way.fetch(base + (r * ROOMS + which) * row_bytes, row_of(which, row0 + r * apart));
  };
  auto get = [&](int which, int r, int64_t row0, int k, float (&v)[VEC]) {
    way.get(room + (r * ROOMS + which) * row_bytes, row_of(which, row0 + r * apart), k, v);
  };
  struct Head { float r1, r2, k; };
  auto head = [&](int64_t row) {
    Head a = {0.f, 0.f, 0.f};
    if (row < p.rows) a = {p.post ? p.rstd[2 * row] : 1.f, p.rstd[2 * row + 1], p.gate ? p.gate[row] : 1.f};
    return a;
  };
  dep_wait();
  float dw1[NV][VEC], dw2[NV][VEC];
#pragma unroll
  for (int k = 0; k < NV; ++k)
#pragma unroll
    for (int e = 0; e < VEC; ++e) dw1[k][e] = dw2[k][e] = 0.f;
  int64_t row0 = FILL == ROW_SHIFT ? first + (int64_t)(blockIdx.x / p.classes) * R * p.classes : (int64_t)blockIdx.x * R;
  fetch(DY, row0);
  fetch(H, row0);
  fetch(O, row0);
  if (ROOMS == 4) fetch(D, row0);
  ahead_commit();
  if (Rows::MOVED) {
    if (p.w1) way.move(p.w1, w1);
    way.move(p.w2, w2);
    __syncthreads();
  }
  way.zeros(room, row_bytes, R * ROOMS);
  Head a[R];
#pragma unroll
  for (int r = 0; r < R; ++r) a[r] = head(row0 + r * apart);
  for (; row0 < p.rows; row0 += step) {
    Head next[R];
#pragma unroll
    for (int r = 0; r < R; ++r) next[r] = head(row0 + step + r * apart);
    ahead_wait<0>();
    float u[R][NV][VEC], f[R];
    {
      float dots[R][2];
#pragma unroll
      for (int r = 0; r < R; ++r) dots[r][0] = dots[r][1] = 0.f;
#pragma unroll
      for (int k = 0; k < NV; ++k) {
        float w[VEC];
        way.weights(p.w2, w2, k, w);
#pragma unroll
        for (int r = 0; r < R; ++r) {
          if (r > 0 && row0 + r * apart >= p.rows) continue;
          float n[VEC];
          get(DY, r, row0, k, u[r][k]);
          get(H, r, row0, k, n);
          vscale<VEC>(n, a[r].r2);
          vfma<VEC>(dw2[k], u[r][k], n);
          vmul<VEC>(u[r][k], w);
          vdot<VEC>(dots[r], u[r][k], n);
        }
      }
      fetch(DY, row0 + step);
#pragma unroll
      for (int r = 0; r < R; ++r) f[r] = dots[r][0] + dots[r][1];
      over_cta<R>(f, buf[0]);
#pragma unroll
      for (int r = 0; r < R; ++r) {
        f[r] *= -p.inv_M * a[r].r2;
        dots[r][0] = dots[r][1] = 0.f;
      }
#pragma unroll
      for (int k = 0; k < NV; ++k) {
        float w[VEC];
        if (p.w1) way.weights(p.w1, w1, k, w);
#pragma unroll
        for (int r = 0; r < R; ++r) {
          if (r > 0 && row0 + r * apart >= p.rows) continue;
          float n[VEC];
          get(H, r, row0, k, n);
          vfma<VEC>(u[r][k], n, f[r]);                       // u2 - n2 mean(u2 n2)
          vscale<VEC>(u[r][k], a[r].r2);
          if (DH) {
            if (DIRECT) load<VEC>(row_of(D, row0 + r * apart) + way.column(k), FILL == ROW_FULL ? VEC : FILL == ROW_WHOLE ? (p.M > way.column(k) ? VEC : 0) : p.M - way.column(k), 0.f, n);
            else get(D, r, row0, k, n);
            vadd<VEC>(u[r][k], n);
          }
#pragma unroll
          for (int e = 0; e < VEC; ++e) n[e] = u[r][k][e];
          vscale<VEC>(n, p.alpha);
          way.keep(static_cast<T*>(p.dx) + (row0 + r * apart) * p.lddx, k, n);
          get(O, r, row0, k, n);
          vscale<VEC>(n, a[r].r1);
          if (p.gate) {
            float q[VEC];
#pragma unroll
            for (int e = 0; e < VEC; ++e) q[e] = n[e];
            vscale<VEC>(q, a[r].k);
            vfma<VEC>(dw1[k], u[r][k], q);
          } else {
            vfma<VEC>(dw1[k], u[r][k], n);
          }
          if (p.w1) vmul<VEC>(u[r][k], w);
          vdot<VEC>(dots[r], u[r][k], n);
        }
      }
      fetch(H, row0 + step);
      if (ROOMS == 4) fetch(D, row0 + step);
#pragma unroll
      for (int r = 0; r < R; ++r) f[r] = dots[r][0] + dots[r][1];
      over_cta<R>(f, buf[1]);
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
      if (r > 0 && row0 + r * apart >= p.rows) continue;
      if (p.dgate && t == 0) p.dgate[row0 + r * apart] = f[r];
      const float f1 = -f[r] * p.inv_M * a[r].r1, scale = a[r].k * a[r].r1;         // (r1 = 1 without post)
#pragma unroll
      for (int k = 0; k < NV; ++k) {
        if (p.post) {
          float n[VEC];
          get(O, r, row0, k, n);
          vfma<VEC>(u[r][k], n, f1);
        }
        vscale<VEC>(u[r][k], scale);
        way.keep(static_cast<T*>(p.d_o) + (row0 + r * apart) * p.lddo, k, u[r][k]);
      }
    }
    fetch(O, row0 + step);
    ahead_commit();
#pragma unroll
    for (int r = 0; r < R; ++r) a[r] = next[r];
  }
  ahead_wait<0>();
  dep_trigger();
  if (!p.part) return;
  // four sums at a time, by way of shared memory where a thread's columns do not begin on four (8192 x 4096 bf16 with single stores here and
  // single loads where they are added 82 us, so 75)
  constexpr bool EVEN = FILL == ROW_FULL || FILL == ROW_WHOLE;
  const int half = part_row(p.M);
  float* out = p.part + (int64_t)blockIdx.x * 2 * half;
  float* shared = reinterpret_cast<float*>(room);
  if (!EVEN) __syncthreads();
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int c = way.column(k);
    if (EVEN) {
#pragma unroll
      for (int e = 0; e < VEC; e += 4) {
        if (FILL == ROW_WHOLE && c >= p.M) continue;
        *reinterpret_cast<float4*>(out + c + e) = make_float4(dw2[k][e], dw2[k][e + 1], dw2[k][e + 2], dw2[k][e + 3]);
        *reinterpret_cast<float4*>(out + half + c + e) = make_float4(dw1[k][e], dw1[k][e + 1], dw1[k][e + 2], dw1[k][e + 3]);
      }
    } else {
#pragma unroll
      for (int e = 0; e < VEC; ++e)
        if (c + e >= 0 && c + e < p.M) { shared[c + e] = dw2[k][e]; shared[half + c + e] = dw1[k][e]; }
    }
  }
  if (EVEN) return;
  __syncthreads();
  for (int c = 4 * t; c < 2 * half; c += 4 * width) *reinterpret_cast<float4*>(out + c) = *reinterpret_cast<const float4*>(shared + c);
}

// dw_pre and dw_post = sums of the CTAs' rows, 32 columns a CTA: eight threads side by side take four columns each, of every 32nd row, eight
// rows in flight; then in pairs.
__global__ void __launch_bounds__(256) sandwich_weight_kernel(const float* part, int n, int M, float* dw2, float* dw1) {
  __shared__ float4 acc[32][8];
  const int t = threadIdx.x, x = t & 7, y = t >> 3, half = part_row(M), c = blockIdx.x * 32 + 4 * x;
  dep_sync();
  float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
  auto add = [](float4& s, const float4& v) { s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w; };
  if (c < 2 * half) {
    for (int k = y; k < n; k += 256) {
      float4 b[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        b[j] = make_float4(0.f, 0.f, 0.f, 0.f);
        if (k + 32 * j < n) b[j] = *reinterpret_cast<const float4*>(part + (int64_t)(k + 32 * j) * 2 * half + c);
      }
#pragma unroll
      for (int j = 4; j > 0; j >>= 1)
#pragma unroll
        for (int i = 0; i < j; ++i) add(b[i], b[i + j]);
      add(a, b[0]);
    }
  }
  acc[y][x] = a;
#pragma unroll
  for (int j = 16; j > 0; j >>= 1) {
    __syncthreads();
    if (y < j) add(acc[y][x], acc[y + j][x]);
  }
  __syncthreads();
  if (t >= 32) return;
  const int at = blockIdx.x * 32 + t, col = at < half ? at : at - half;
  float* dw = at < half ? dw2 : dw1;
  if (dw && at < 2 * half && col < M) dw[col] = reinterpret_cast<const float*>(acc[0])[t];
}

fw_status desc_check(const fw_sandwich_desc* d) {
  if (!d) return FW_ERR_INVALID_ARG;
  if (d->M < 1 || d->M > kNormMaxM) return FW_ERR_SHAPE;
  if (!type_ok(d->dtype) || (d->y_dtype != d->dtype && d->y_dtype != FW_E4M3) || (d->post != 0 && d->post != 1)) return FW_ERR_INVALID_ARG;
  if (!(d->eps > 0.f && d->eps <= 3e38f) || !(d->alpha >= -3e38f && d->alpha <= 3e38f)) return FW_ERR_INVALID_ARG;
  return FW_OK;
}

// CTAs that take rows of each residue alike
int whole_classes(int ctas, int classes) { return ctas < classes ? classes : ctas / classes * classes; }

template <class T, class Y, int VEC, int NV, int FILL>
cudaError_t forward_launch(const SandwichFwd& p, cudaStream_t s) {
  constexpr int SLOTS = slots(VEC, NV, 2);
  static FillCache cache;
  auto kernel = sandwich_forward_kernel<T, Y, VEC, NV, SLOTS, FILL>;
  typedef Way<T, VEC, NV, FILL> Rows;
  const size_t smem = (size_t)SLOTS * 2 * Rows::row_bytes(p.M, p.width) + 2 * (size_t)Rows::weight_bytes(p.width);
  int ctas = 0;
  const cudaError_t e = fill(kernel, cache, p.width, smem, p.rows, 1 << 30, &ctas);
  if (FILL == ROW_SHIFT && e == cudaSuccess) ctas = whole_classes(ctas, p.classes);
  return e != cudaSuccess ? e : launch_dep(kernel, ctas, p.width, smem, s, p);
}
template <class T, class Y, int VEC, int NV>
cudaError_t forward_launch(const SandwichFwd& p, cudaStream_t s) {
  if constexpr (VEC > 1 && NV <= 4)
    if (p.classes == 1) return forward_launch<T, Y, VEC, NV, ROW_TAIL>(p, s);
  if constexpr (VEC > 1 && NV <= 4 && sizeof(T) == sizeof(Y))
    if (p.classes) return forward_launch<T, Y, VEC, NV, ROW_SHIFT>(p, s);
  constexpr int WHOLE = VEC > 1 ? ROW_WHOLE : ROW_PART, FULL = VEC > 1 ? ROW_FULL : ROW_PART;
  if (VEC > 1 && p.M == NV * VEC * p.width) return forward_launch<T, Y, VEC, NV, FULL>(p, s);
  if (VEC > 1 && p.M % VEC == 0) return forward_launch<T, Y, VEC, NV, WHOLE>(p, s);
  return forward_launch<T, Y, VEC, NV, ROW_PART>(p, s);
}

// Threads for a row of that many accesses, no more warps than have some (powers of two: 8192 x 5120 bf16 backward 146 us, so 115)
int warps_for(int accesses, int each, int least) {
  const int warps = (accesses + 32 * each - 1) / (32 * each);
  return 32 * (warps < least ? least : warps);
}

// Four accesses of 16 bytes a thread where there are rows for every SM, one where the chain of one row is all there is
template <class T, class Y, int VEC>
cudaError_t forward_nv(const SandwichFwd& p0, cudaStream_t s) {
  SandwichFwd p = p0;
  const int acc = (p.M + VEC - 1 + (p.classes > 1 ? VEC - 1 : 0)) / VEC;
  p.width = row_width(acc, p.rows < 2 * sm_count() ? 1 : VEC > 1 ? 4 : 8, 512);
  const int nv = (acc + p.width - 1) / p.width;
  if (VEC > 1) p.width = warps_for(acc, nv <= 2 ? nv : nv <= 4 || VEC == 8 ? 4 : 8, 1);
  // 512 threads take kNormMaxM elements in four accesses of eight, eight of four or thirty-two of one
  if (nv <= 1) return forward_launch<T, Y, VEC, 1>(p, s);
  if (nv <= 2) return forward_launch<T, Y, VEC, 2>(p, s);
  if (nv <= 4) return forward_launch<T, Y, VEC, 4>(p, s);
  if (nv <= 8) return forward_launch<T, Y, VEC, VEC == 8 ? 4 : 8>(p, s);
  if (nv <= 16) return forward_launch<T, Y, VEC, VEC == 8 ? 4 : VEC == 4 ? 8 : 16>(p, s);
  return forward_launch<T, Y, VEC, VEC == 8 ? 4 : VEC == 4 ? 8 : 32>(p, s);
}
template <class T, class Y>
cudaError_t forward_vec(const SandwichFwd& p, bool vec, cudaStream_t s) {
  return vec || p.classes ? forward_nv<T, Y, 16 / sizeof(T)>(p, s) : forward_nv<T, Y, 1>(p, s);
}

int backward_ctas() { return 4 * sm_count(); }

template <class T, int VEC, int NV, bool DH, int FILL, bool SOLO>
cudaError_t backward_launch(const SandwichBwd& p, cudaStream_t s, int* ctas) {
  constexpr int ROOMS = DH && VEC > 1 ? 4 : 3;
  constexpr int SLOTS = slots(VEC, NV, ROOMS);
  static FillCache cache;
  auto kernel = sandwich_backward_kernel<T, VEC, NV, SLOTS, DH, FILL, SOLO>;
  const int threads = SOLO ? p.width : 256, per = threads / p.width;
  size_t smem = (size_t)SLOTS * ROOMS * Ahead<T, VEC, NV, FILL>::row_bytes(p.M, threads, p.width);
  const size_t sums = (size_t)per * 2 * part_row(p.M) * sizeof(float);
  if (!SOLO && p.part && smem < sums) smem = sums;
  const cudaError_t e = fill(kernel, cache, threads, smem, (p.rows + per - 1) / per, backward_ctas(), ctas);
  return e != cudaSuccess ? e : launch_dep(kernel, *ctas, threads, smem, s, p);
}
template <class T, int VEC, int NV, bool DH, int FILL>
cudaError_t backward_rows_launch(const SandwichBwd& p, cudaStream_t s, int* ctas) {
  constexpr int ROOMS = DH && NV < 8 ? 4 : 3, R = NV <= 2 ? 2 : 1;
  static FillCache cache;
  auto kernel = sandwich_backward_rows_kernel<T, VEC, NV, R, DH, FILL>;
  typedef Way<T, VEC, NV, FILL> Rows;
  size_t smem = (size_t)R * ROOMS * Rows::row_bytes(p.M, p.width) + 2 * (size_t)Rows::weight_bytes(p.width);
  const size_t sums = (size_t)2 * part_row(p.M) * sizeof(float);
  if ((FILL == ROW_PART || Rows::MOVED) && p.part && smem < sums) smem = sums;
  const cudaError_t e = fill(kernel, cache, p.width, smem, (p.rows + R - 1) / R, backward_ctas(), ctas);
  if (FILL == ROW_SHIFT && e == cudaSuccess) *ctas = whole_classes(*ctas, p.classes);
  return e != cudaSuccess ? e : launch_dep(kernel, *ctas, p.width, smem, s, p);
}
// What backward_nv comes to, and no other shapes, are built.
template <class T, int VEC, int NV, bool DH>
cudaError_t backward_launch(const SandwichBwd& p, cudaStream_t s, int* ctas) {
  if constexpr (VEC == 1) {
    if constexpr (NV <= 4)                                   // up to 512 columns
      if (p.width < 128) return backward_launch<T, VEC, NV, DH, ROW_PART, false>(p, s, ctas);
    if constexpr (NV >= 4) return backward_launch<T, VEC, NV, DH, ROW_PART, true>(p, s, ctas);
  } else {
    if constexpr (NV <= (VEC == 8 ? 2 : 4)) {                // 6144 columns at most (see classes_of)
      if (p.classes == 1) return backward_rows_launch<T, VEC, NV, DH, ROW_TAIL>(p, s, ctas);
      if (p.classes) return backward_rows_launch<T, VEC, NV, DH, ROW_SHIFT>(p, s, ctas);
    }
    if constexpr (NV <= 2) {                                 // more accesses a thread: 128 threads or more
      if (p.width < 128)
        return p.M % VEC == 0 ? backward_launch<T, VEC, NV, DH, ROW_WHOLE, false>(p, s, ctas)
                              : backward_launch<T, VEC, NV, DH, ROW_PART, false>(p, s, ctas);
    }
    if (p.M == NV * VEC * p.width) return backward_rows_launch<T, VEC, NV, DH, ROW_FULL>(p, s, ctas);
    if (p.M % VEC == 0) return backward_rows_launch<T, VEC, NV, DH, ROW_WHOLE>(p, s, ctas);
    // rows without classes that end inside an access: up to 2 KB, of one access, or of more than 6144 columns
    if constexpr (VEC == 8 || NV != 2) return backward_rows_launch<T, VEC, NV, DH, ROW_PART>(p, s, ctas);
  }
  return cudaErrorInvalidConfiguration;
}
template <class T, int VEC, int NV>
cudaError_t backward_launch(const SandwichBwd& p, cudaStream_t s, int* ctas) {
  return p.dh ? backward_launch<T, VEC, NV, true>(p, s, ctas) : backward_launch<T, VEC, NV, false>(p, s, ctas);
}

template <class T, int VEC>
cudaError_t backward_nv(const SandwichBwd& p0, cudaStream_t s, int* ctas) {
  SandwichBwd p = p0;
  const int acc = (p.M + VEC - 1 + (p.classes > 1 ? VEC - 1 : 0)) / VEC;
  // two accesses a thread; one where rows are short and many (30000 x 1000 bf16 79 us against 95, but 2000 x 1000 17.5 against 14.2), and
  // where 128 threads would take twice more than there are (8192 x 1536 bf16 39 us against 43, but 8192 x 2048 45.3 against 43.6)
  p.width = row_width(acc, VEC == 1 ? 4 : (acc <= 128 && p.rows > 32 * sm_count()) || (acc > 128 && acc <= 192) ? 1 : 2, 512);
  const int nv = (acc + p.width - 1) / p.width;
  if (VEC > 1 && p.width >= 128) p.width = warps_for(acc, nv <= 2 ? nv : nv <= 4 || VEC == 8 ? 4 : 8, 4);
  if (nv <= 1) return backward_launch<T, VEC, 1>(p, s, ctas);
  if (nv <= 2) return backward_launch<T, VEC, 2>(p, s, ctas);
  if (nv <= 4) return backward_launch<T, VEC, 4>(p, s, ctas);
  if (nv <= 8) return backward_launch<T, VEC, VEC == 8 ? 4 : 8>(p, s, ctas);
  if (nv <= 16) return backward_launch<T, VEC, VEC == 8 ? 4 : VEC == 4 ? 8 : 16>(p, s, ctas);
  return backward_launch<T, VEC, VEC == 8 ? 4 : VEC == 4 ? 8 : 32>(p, s, ctas);
}

// A range of memory that a call reads or writes; ld, elem: of a matrix (0: a vector)
struct Range { const void* p; uint64_t n; int64_t ld; int elem; };
// Rows after which matrices that all lie equally past 16 bytes do so as at their beginning (1: aligned rows that end inside 16 bytes); 0 where
// they do not, where a row is so short that a few threads take several, and beyond 6144 columns.  (At 16384 a row and its weights are more than
// a SM holds; between, up to 8191 columns, they would fit, but nothing has been measured there this way: 4096 x 7001 bf16, aligned rows, forward 71 us and
// backward 127 by the way that is taken, 57 and 83 for 7008 columns.)
int classes_of(const Mat* m, int n, int M, bool aligned) {
  const bool fits = M <= 6144 && M * m[0].elem > 2048;
  if (aligned) return fits && M * m[0].elem % 16 != 0 ? 1 : 0;
  uint64_t differ = 0;
  for (int i = 0; i < n; ++i)
    if (m[i].p) differ |= (reinterpret_cast<uintptr_t>(m[i].p) ^ reinterpret_cast<uintptr_t>(m[0].p)) | (uint64_t)((m[i].ld - m[0].ld) * m[0].elem);
  return (differ & 15) == 0 && fits ? 16 / m[0].elem : 0;
}
Range mat(const void* p, int64_t rows, int M, int64_t ld, int elem) { return {p, p ? matrix_span(rows, M, ld, elem) : 0, ld, elem}; }
Range vec4(const void* p, uint64_t n) { return {p, 4 * n, 0, 4}; }
bool meet(const Range& a, const Range& b) { return overlap(a.p, a.n, b.p, b.n); }
bool same(const Range& a, const Range& b) { return a.ld && b.ld && a.p == b.p && a.ld == b.ld && a.elem == b.elem; }

}  // namespace
}  // namespace fw

using namespace fw;

extern "C" {

void fw_sandwich_desc_default(fw_sandwich_desc* d, int32_t M) {
  if (!d) return;
  d->M = M; d->dtype = FW_BF16; d->y_dtype = FW_BF16; d->post = 1; d->eps = 1e-6f; d->alpha = 1.f;
}

size_t fw_sandwich_scratch_bytes(const fw_sandwich_desc* d) {
  if (desc_check(d) != FW_OK) return 0;
  return ((size_t)backward_ctas() * 2 * part_row(d->M) * sizeof(float) + 255) / 256 * 256;
}

fw_status fw_sandwich_forward(const fw_sandwich_desc* d, int64_t rows, const void* o, int64_t ldo, const void* x, int64_t ldx,
                              const float* w_post, const float* gate, const float* w_pre, void* h, int64_t ldh, void* y, int64_t ldy,
                              float* y_scale, float* rstd, void* cuda_stream) {
  fw_status st = desc_check(d);
  if (st != FW_OK) return st;
  const bool q8 = d->y_dtype == FW_E4M3;
  if (!o || !x || !w_pre || !h || !y || (q8 != (y_scale != nullptr))) return FW_ERR_INVALID_ARG;
  if ((st = rows_check(rows)) != FW_OK) return st;
  const int M = d->M, es = type_bytes(d->dtype), ys = type_bytes(d->y_dtype), per16 = 16 / es;
  bool vec = aligned_to(w_pre, 16) && aligned_to(w_post, 16);
  const Mat mats[4] = {{o, ldo, es}, {x, ldx, es}, {h, ldh, es}, {y, ldy, ys}};
  for (const Mat& m : mats)
    if ((st = mat_check(m, M, per16, &vec)) != FW_OK) return st;
  const Range in[5] = {mat(o, rows, M, ldo, es), mat(x, rows, M, ldx, es), vec4(w_post, M), vec4(gate, rows), vec4(w_pre, M)};
  const Range out[4] = {mat(h, rows, M, ldh, es), mat(y, rows, M, ldy, ys), vec4(y_scale, rows), vec4(rstd, 2 * rows)};
  for (int i = 2; i < 5; ++i)
    if (!aligned_to(in[i].p, 4)) return FW_ERR_INVALID_ARG;
  for (int i = 0; i < 4; ++i) {
    if (!aligned_to(out[i].p, i < 2 ? 1 : 4)) return FW_ERR_INVALID_ARG;
    // an output may be an input itself (a thread has read what it writes), any other overlap is refused
    for (const Range& r : in)
      if (meet(out[i], r) && !same(out[i], r)) return FW_ERR_INVALID_ARG;
    for (int j = 0; j < i; ++j)
      if (meet(out[i], out[j])) return FW_ERR_INVALID_ARG;
  }
  SandwichFwd p;
  p.o = o; p.x = x; p.w1 = w_post; p.gate = gate; p.w2 = w_pre; p.h = h; p.y = y; p.y_scale = y_scale; p.rstd = rstd;
  p.rows = rows; p.ldo = ldo; p.ldx = ldx; p.ldh = ldh; p.ldy = ldy; p.M = M; p.width = 0; p.post = d->post;
  p.classes = q8 && !vec ? 0 : classes_of(mats, q8 ? 3 : 4, M, vec);      // (a row of e4m3 lies otherwise past 16 bytes)
  p.eps = d->eps; p.inv_M = 1.f / (float)M; p.alpha = d->alpha;
  cudaStream_t s = (cudaStream_t)cuda_stream;
  ProfScope ps(FW_PROF_MISC, s);
  cudaError_t e;
  if (d->dtype == FW_F32)
    e = q8 ? forward_vec<float, __nv_fp8_storage_t>(p, vec, s) : forward_vec<float, float>(p, vec, s);
  else
    e = q8 ? forward_vec<__nv_bfloat16, __nv_fp8_storage_t>(p, vec, s) : forward_vec<__nv_bfloat16, __nv_bfloat16>(p, vec, s);
  return failed(e, "fw_sandwich_forward");
}

fw_status fw_sandwich_backward(const fw_sandwich_desc* d, int64_t rows, const void* dy, int64_t lddy, const void* dh, int64_t lddh,
                               const void* o, int64_t ldo, const void* h, int64_t ldh, const float* w_post, const float* gate,
                               const float* w_pre, const float* rstd, void* dx, int64_t lddx, void* d_o, int64_t lddo, float* dw_post,
                               float* dw_pre, float* dgate, void* scratch, size_t scratch_bytes, void* cuda_stream) {
  fw_status st = desc_check(d);
  if (st != FW_OK) return st;
  if (!dy || !o || !h || !w_pre || !rstd || !dx || !d_o) return FW_ERR_INVALID_ARG;
  if ((st = rows_check(rows)) != FW_OK) return st;
  const bool sums = dw_post || dw_pre;
  const size_t ns = fw_sandwich_scratch_bytes(d);
  if (sums) {
    if (!scratch) return FW_ERR_INVALID_ARG;
    if (!aligned_to(scratch, 256) || scratch_bytes < ns) return FW_ERR_WORKSPACE;
  }
  const int M = d->M, es = type_bytes(d->dtype), per16 = 16 / es;
  bool vec = aligned_to(w_pre, 16) && aligned_to(w_post, 16);
  const Mat mats[6] = {{dy, lddy, es}, {dh, lddh, es}, {o, ldo, es}, {h, ldh, es}, {dx, lddx, es}, {d_o, lddo, es}};
  for (const Mat& m : mats)
    if (m.p && (st = mat_check(m, M, per16, &vec)) != FW_OK) return st;
  const Range in[8] = {mat(dy, rows, M, lddy, es), mat(dh, rows, M, lddh, es), mat(o, rows, M, ldo, es), mat(h, rows, M, ldh, es),
                       vec4(w_post, M), vec4(gate, rows), vec4(w_pre, M), vec4(rstd, 2 * rows)};
  const Range out[6] = {mat(dx, rows, M, lddx, es), mat(d_o, rows, M, lddo, es), vec4(dw_post, M), vec4(dw_pre, M), vec4(dgate, rows),
                        {sums ? scratch : nullptr, ns, 0, 4}};
  for (int i = 4; i < 8; ++i)
    if (!aligned_to(in[i].p, 4)) return FW_ERR_INVALID_ARG;
  for (int i = 0; i < 6; ++i) {
    if (i > 1 && !aligned_to(out[i].p, 4)) return FW_ERR_INVALID_ARG;
    for (int j = 0; j < 8; ++j)
      // o is read once more after dx has been written
      if (meet(out[i], in[j]) && !(same(out[i], in[j]) && !(i == 0 && j == 2))) return FW_ERR_INVALID_ARG;
    for (int j = 0; j < i; ++j)
      if (meet(out[i], out[j])) return FW_ERR_INVALID_ARG;
  }
  SandwichBwd p;
  p.dy = dy; p.dh = dh; p.o = o; p.h = h; p.w1 = w_post; p.gate = gate; p.w2 = w_pre; p.rstd = rstd; p.dx = dx; p.d_o = d_o;
  p.part = sums ? static_cast<float*>(scratch) : nullptr; p.dgate = dgate;
  p.rows = rows; p.lddy = lddy; p.lddh = lddh; p.ldo = ldo; p.ldh = ldh; p.lddx = lddx; p.lddo = lddo; p.M = M; p.width = 0;
  p.classes = classes_of(mats, 6, M, vec);
  p.post = d->post; p.inv_M = 1.f / (float)M; p.alpha = d->alpha;
  cudaStream_t str = (cudaStream_t)cuda_stream;
  int ctas = 0;
  cudaError_t e;
  {
    ProfScope ps(FW_PROF_MISC, str);
    const bool wide = vec || p.classes;
    if (d->dtype == FW_F32) e = wide ? backward_nv<float, 4>(p, str, &ctas) : backward_nv<float, 1>(p, str, &ctas);
    else e = wide ? backward_nv<__nv_bfloat16, 8>(p, str, &ctas) : backward_nv<__nv_bfloat16, 1>(p, str, &ctas);
  }
  if (e == cudaSuccess && sums) {
    ProfScope ps(FW_PROF_MISC, str);
    e = launch_dep(sandwich_weight_kernel, (2 * part_row(M) + 31) / 32, 256, 0, str, p.part, ctas, M, dw_pre, dw_post);
  }
  return failed(e, "fw_sandwich_backward");
}

}  // extern "C"
