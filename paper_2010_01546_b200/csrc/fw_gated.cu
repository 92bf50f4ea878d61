// Gated feed-forward block H = act(X Wg^T + bg) * (X Wu^T + bu): host side, and the pass over the gates' gradients.
#include <cstdio>
#include <cstring>
#include <new>

#include "fw_gated.h"
#include "fw_gated_act.cuh"
#include "fw_rows.cuh"
#include "fw_umma.h"

using namespace fw;

struct fw_gated {
  fw_gated_desc d;
  cudaStream_t stream;
  int device;
  int32_t* status;        // first word of the workspace: code of a bounded wait that gave up
  char *Da, *Db;          // gradients of the projections, max_rows x ldd bf16
  float* part;            // partial column sums
  int64_t ldd;
};

namespace fw {
namespace {

using namespace rows;

__device__ __forceinline__ void unpack8(uint4 q, float (&v)[8]) {
  v[0] = bf16_lo(q.x); v[1] = bf16_hi(q.x); v[2] = bf16_lo(q.y); v[3] = bf16_hi(q.y);
  v[4] = bf16_lo(q.z); v[5] = bf16_hi(q.z); v[6] = bf16_lo(q.w); v[7] = bf16_hi(q.w);
}

// da = dh b act'(a), db = dh act(a), and with SUMS partial sums of both over the rows.  Both are rounded to bf16 here, as operands of the
// products that follow: half a step, 2^-8, of each term, the size of the rounding of bf16 outputs; fp32 weight gradients carry it too
// (twice the operands' bits would take twice the products).  The sums are of the values before that.  A CTA has 256 columns and a slab of rows: a
// thread eight neighbouring columns (16 bytes) of every eighth row, two rows' loads in flight.  Reads 6 bytes an element and writes 4:
// HBM bound.  (One kernel for all activations took 98 registers and two CTAs a SM: 8192 x 8192 184 us.)
template <int ACT, bool SUMS>
__global__ void __launch_bounds__(256, SUMS ? 3 : 4) gated_gates_kernel(const GatedGates g) {
  __shared__ float acc[SUMS ? 8 : 1][256];
  const int lane = threadIdx.x & 31, ty = threadIdx.x >> 5;
  const int col = blockIdx.x * 256 + lane * 8, n = g.N - col;
  const int64_t per = (g.rows + g.slabs - 1) / g.slabs;
  const int64_t r0 = blockIdx.y * per, r1 = min(g.rows, r0 + per);
  dep_sync();
  float sa[8], sb[8];
  if (SUMS) {
#pragma unroll
    for (int e = 0; e < 8; ++e) sa[e] = sb[e] = 0.f;
  }
  typedef const __nv_bfloat16* In;
  typedef __nv_bfloat16* Out;
  In dh = static_cast<In>(g.dH) + col, zg = static_cast<In>(g.Zg) + col, zu = static_cast<In>(g.Zu) + col;
  Out oa = static_cast<Out>(g.Da) + col, ob = static_cast<Out>(g.Db) + col;
  auto one = [&](int64_t r, float (&h)[8], float (&a)[8], float (&b)[8]) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      float f, df;
      Act<ACT>::both(a[e], f, df);
      a[e] = h[e] * b[e] * df;
      b[e] = h[e] * f;
      if (SUMS) { sa[e] += a[e]; sb[e] += b[e]; }
    }
    store<8>(oa + r * g.ldd, n, a);
    store<8>(ob + r * g.ldd, n, b);
  };
  int64_t r = r0 + ty;
  if (n >= 8) {
    for (; r + 8 < r1; r += 16) {
      uint4 q[6];
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        q[3 * k] = *reinterpret_cast<const uint4*>(dh + (r + 8 * k) * g.lddh);
        q[3 * k + 1] = *reinterpret_cast<const uint4*>(zg + (r + 8 * k) * g.ldz);
        q[3 * k + 2] = *reinterpret_cast<const uint4*>(zu + (r + 8 * k) * g.ldz);
      }
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        float h[8], a[8], b[8];
        unpack8(q[3 * k], h);
        unpack8(q[3 * k + 1], a);
        unpack8(q[3 * k + 2], b);
        one(r + 8 * k, h, a, b);
      }
    }
  }
  if (n > 0) {
    for (; r < r1; r += 8) {
      float h[8], a[8], b[8];
      load<8>(dh + r * g.lddh, n, 0.f, h);
      load<8>(zg + r * g.ldz, n, 0.f, a);
      load<8>(zu + r * g.ldz, n, 0.f, b);
      one(r, h, a, b);
    }
  }
  if (!SUMS) return;
  for (int k = 0; k < 2; ++k) {
    __syncthreads();
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[ty][lane * 8 + e] = k ? sb[e] : sa[e];
    __syncthreads();
    const int c = blockIdx.x * 256 + threadIdx.x;
    float s = acc[0][threadIdx.x];
#pragma unroll
    for (int w = 1; w < 8; ++w) s += acc[w][threadIdx.x];
    if (c < g.N) g.part[((int64_t)k * g.slabs + blockIdx.y) * g.N + c] = s;
  }
}

// dbg, dbu: sums over the slabs, 32 columns a CTA: eight warps take every eighth slab, all of them in flight, and are added in order
// (a thread for each column took 9 us for the 64 slabs of N = 8192)
__global__ void __launch_bounds__(256) gated_bias_kernel(const float* part, int slabs, int N, float* dbg, float* dbu) {
  __shared__ float acc[8][32];
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, c = blockIdx.x * 32 + lane;
  dep_sync();
  float* out = blockIdx.y ? dbu : dbg;
  const float* p = part + (int64_t)blockIdx.y * slabs * N + c;
  float v[kGateSlabs / 8];
#pragma unroll
  for (int k = 0; k < kGateSlabs / 8; ++k) v[k] = c < N && w + 8 * k < slabs ? p[(int64_t)(w + 8 * k) * N] : 0.f;
  float s = v[0];
#pragma unroll
  for (int k = 1; k < kGateSlabs / 8; ++k) s += v[k];
  acc[w][lane] = s;
  __syncthreads();
  if (w == 0 && c < N) {
#pragma unroll
    for (int k = 1; k < 8; ++k) s += acc[k][lane];
    out[c] = s;
  }
}

constexpr int kGatedMaxDim = 32768;
constexpr int64_t kGatedMaxRows = 1 << 26;        // tiles are counted in 32 bits
constexpr size_t kAlign = 256;
size_t align_up(size_t x) { return (x + kAlign - 1) / kAlign * kAlign; }

fw_status desc_check(const fw_gated_desc* d) {
  if (!d) return FW_ERR_INVALID_ARG;
  if (d->M < 1 || d->M > kGatedMaxDim || d->N < 1 || d->N > kGatedMaxDim) return FW_ERR_SHAPE;
  if (d->x_dtype != FW_BF16 && d->x_dtype != FW_E4M3) return d->x_dtype == FW_F32 ? FW_ERR_UNSUPPORTED : FW_ERR_INVALID_ARG;
  if (d->act < FW_ACT_SILU || d->act > FW_ACT_RELU) return FW_ERR_INVALID_ARG;
  if (d->grad != 0 && d->grad != 1) return FW_ERR_INVALID_ARG;
  if (d->grad && d->x_dtype == FW_E4M3) return FW_ERR_UNSUPPORTED;
  if (d->grad && (d->max_rows < 1 || d->max_rows > kGatedMaxRows)) return FW_ERR_SHAPE;
  return FW_OK;
}

size_t carve(const fw_gated_desc& d, char* base, fw_gated* h) {
  size_t off = kAlign;                       // status
  fw_gated tmp;
  fw_gated& g = h ? *h : tmp;
  g.status = reinterpret_cast<int32_t*>(base);
  g.Da = g.Db = nullptr;
  g.part = nullptr;
  g.ldd = ((int64_t)d.N + 7) / 8 * 8;
  if (d.grad) {
    const size_t mat = align_up((size_t)d.max_rows * (size_t)g.ldd * 2);
    g.Da = base + off; off += mat;
    g.Db = base + off; off += mat;
    g.part = reinterpret_cast<float*>(base + off); off += align_up((size_t)2 * kGateSlabs * d.N * sizeof(float));
  }
  return off;
}

struct View { const void* p; int64_t rows, cols, ld; int elem; };

// 16-byte aligned rows, wide enough: what TMA and the 16-byte accesses need
fw_status view_check(const View& v) {
  if (v.ld < v.cols || v.ld > ((int64_t)1 << 30)) return FW_ERR_SHAPE;
  if (!aligned_to(v.p, 16) || (v.ld * v.elem) % 16 != 0) return FW_ERR_INVALID_ARG;
  return FW_OK;
}
// what a matrix of one row has for a leading dimension does not matter: the next multiple of 16 bytes
int64_t pitch(int64_t rows, int64_t cols, int64_t ld, int elem) {
  const int64_t q = 16 / elem;
  return rows == 1 && ld >= cols ? (cols + q - 1) / q * q : ld;
}
uint64_t span(const View& v) { return v.p ? matrix_span(v.rows, v.cols, v.ld, v.elem) : 0; }

// no output overlaps an input or another output
bool disjoint(const View* out, int no, const View* in, int ni) {
  for (int i = 0; i < no; ++i) {
    for (int j = 0; j < ni; ++j)
      if (overlap(out[i].p, span(out[i]), in[j].p, span(in[j]))) return false;
    for (int j = 0; j < i; ++j)
      if (overlap(out[i].p, span(out[i]), out[j].p, span(out[j]))) return false;
  }
  return true;
}

// A product whose tiles of 256 x 256 do not give every pair of SMs one goes to narrower tiles that share K.  Narrow / pairs in us: forward
// 512 x 4096, 36 tiles 23.0 / 25.9, 56 tiles 34.2 / 27.4, 72 tiles 37.2 / 28.5, 74 tiles 37.8 / 29.0, 96 tiles 68.3 / 47.5; gradient of X of
// 4608 x 1024 x 1152, 72 tiles 35.8 / 31.3; weight gradients of 8192 x 512 x 1024, 16 tiles 42.5 / 62.6, of 8192 x 1024 x 1024, 32 tiles
// 55.1 / 65.0, of 512 x 1536 x 1536, 72 tiles 18.7 / 13.3.  So the narrow tiles are right up to about 40 tiles, and from 50 to 73 they
// cost up to 40 % more.
bool few_tiles(int64_t tiles) { return tiles < sm_count() / 2; }

fw_status here(const fw_gated* g) {
  int dev = -1;
  if (cudaGetDevice(&dev) != cudaSuccess) { cudaGetLastError(); return FW_ERR_CUDA; }
  return dev == g->device ? FW_OK : FW_ERR_INVALID_ARG;
}

}  // namespace

int gated_gate_slabs(int64_t rows, int N) {
  // 32 rows a slab at least, and no more CTAs than a few waves of eight a SM
  int64_t s = (rows + 31) / 32;
  const int64_t cols = (N + 255) / 256, most = (4 * 8 * (int64_t)sm_count() + cols - 1) / cols;
  if (s > most) s = most;
  return s > kGateSlabs ? kGateSlabs : (int)s;
}

cudaError_t launch_gated_gates(const GatedGates& g, cudaStream_t s) {
  cudaError_t e;
  {
    ProfScope ps(FW_PROF_MISC, s);
    const dim3 grid((g.N + 255) / 256, g.slabs);
    auto go = [&](auto with, auto without) { return launch_dep(g.part ? with : without, grid, 256, 0, s, g); };
    if (g.act == FW_ACT_SILU) e = go(gated_gates_kernel<FW_ACT_SILU, true>, gated_gates_kernel<FW_ACT_SILU, false>);
    else if (g.act == FW_ACT_GELU) e = go(gated_gates_kernel<FW_ACT_GELU, true>, gated_gates_kernel<FW_ACT_GELU, false>);
    else if (g.act == FW_ACT_GELU_TANH) e = go(gated_gates_kernel<FW_ACT_GELU_TANH, true>, gated_gates_kernel<FW_ACT_GELU_TANH, false>);
    else e = go(gated_gates_kernel<FW_ACT_RELU, true>, gated_gates_kernel<FW_ACT_RELU, false>);
  }
  if (e == cudaSuccess && g.part) {
    ProfScope ps(FW_PROF_MISC, s);
    e = launch_dep(gated_bias_kernel, dim3((g.N + 31) / 32, 2), 256, 0, s, g.part, g.slabs, g.N, g.dbg, g.dbu);
  }
  return e;
}

}  // namespace fw

extern "C" {

void fw_gated_desc_default(fw_gated_desc* d, int32_t M, int32_t N) {
  if (!d) return;
  d->M = M; d->N = N; d->x_dtype = FW_BF16; d->act = FW_ACT_SILU; d->grad = 0; d->max_rows = 0;
}

size_t fw_gated_workspace_bytes(const fw_gated_desc* d) {
  if (desc_check(d) != FW_OK) return 0;
  return carve(*d, nullptr, nullptr);
}

fw_status fw_gated_create(const fw_gated_desc* d, void* dev_workspace, size_t bytes, void* cuda_stream, fw_gated** out) {
  if (!out) return FW_ERR_INVALID_ARG;
  *out = nullptr;
  if (!d || !dev_workspace) return FW_ERR_INVALID_ARG;
  const fw_status st = desc_check(d);
  if (st != FW_OK) return st;
  if (!aligned_to(dev_workspace, kAlign) || bytes < carve(*d, nullptr, nullptr)) return FW_ERR_WORKSPACE;
  int dev = -1, ndev = 0;
  if (cudaGetDeviceCount(&ndev) != cudaSuccess || ndev < 1 || cudaGetDevice(&dev) != cudaSuccess || !umma_available()) {
    cudaGetLastError();
    fprintf(stderr, "[fw] no CUDA device: this library has no CPU path\n");
    return FW_ERR_CUDA;
  }
  fw_gated* g = new (std::nothrow) fw_gated;
  if (!g) return FW_ERR_INVALID_ARG;
  memset(g, 0, sizeof(*g));
  g->d = *d;
  g->stream = (cudaStream_t)cuda_stream;
  g->device = dev;
  carve(*d, (char*)dev_workspace, g);
  const cudaError_t e = cudaMemsetAsync(g->status, 0, kAlign, g->stream);
  if (e != cudaSuccess) {
    fprintf(stderr, "[fw] fw_gated_create: %s\n", cudaGetErrorString(e));
    delete g;
    return FW_ERR_CUDA;
  }
  *out = g;
  return FW_OK;
}

fw_status fw_gated_destroy(fw_gated* g) {
  if (!g) return FW_ERR_INVALID_ARG;
  delete g;
  return FW_OK;
}

fw_status fw_gated_forward(fw_gated* g, const void* X, int64_t rows, int64_t ldx, const float* x_scale, const void* Wg, const void* Wu,
                           int64_t ldw, const float* wg_scale, const float* wu_scale, const float* bg, const float* bu, void* H,
                           int64_t ldh, void* Zg, void* Zu, int64_t ldz) {
  if (!g || !X || !Wg || !Wu || !H || (Zg == nullptr) != (Zu == nullptr) || (bg == nullptr) != (bu == nullptr)) return FW_ERR_INVALID_ARG;
  const bool q8 = g->d.x_dtype == FW_E4M3;
  if (q8 != (x_scale != nullptr) || q8 != (wg_scale != nullptr) || q8 != (wu_scale != nullptr)) return FW_ERR_INVALID_ARG;
  if (rows < 1 || rows > kGatedMaxRows) return FW_ERR_SHAPE;
  const int M = g->d.M, N = g->d.N, es = q8 ? 1 : 2;
  ldx = pitch(rows, M, ldx, es); ldw = pitch(N, M, ldw, es); ldh = pitch(rows, N, ldh, 2); ldz = pitch(rows, N, ldz, 2);
  const View in[8] = {{X, rows, M, ldx, es}, {Wg, N, M, ldw, es}, {Wu, N, M, ldw, es}, {x_scale, 1, rows, rows, 4},
                      {wg_scale, 1, N, N, 4}, {wu_scale, 1, N, N, 4}, {bg, 1, N, N, 4}, {bu, 1, N, N, 4}};
  const View out[3] = {{H, rows, N, ldh, 2}, {Zg, rows, N, ldz, 2}, {Zu, rows, N, ldz, 2}};
  fw_status st;
  for (int i = 0; i < 3; ++i) {
    if ((st = view_check(in[i])) != FW_OK) return st;
    if (out[i].p && (st = view_check(out[i])) != FW_OK) return st;
  }
  for (int i = 3; i < 8; ++i)
    if (!aligned_to(in[i].p, 4)) return FW_ERR_INVALID_ARG;
  if (!disjoint(out, 3, in, 8)) return FW_ERR_INVALID_ARG;
  if ((st = here(g)) != FW_OK) return st;
  GatedForward f;
  f.X = X; f.Wg = Wg; f.Wu = Wu; f.xs = x_scale; f.wgs = wg_scale; f.wus = wu_scale; f.bg = bg; f.bu = bu;
  f.H = H; f.Zg = Zg; f.Zu = Zu; f.rows = rows; f.ldx = ldx; f.ldw = ldw; f.ldh = ldh; f.ldz = ldz;
  f.M = M; f.N = N; f.e4m3 = q8; f.act = g->d.act; f.status = g->status;
  return few_tiles((rows + 255) / 256 * ((N + 127) / 128)) ? launch_gated_small_forward(f, g->stream) : launch_gated_pair_forward(f, g->stream);
}

fw_status fw_gated_backward(fw_gated* g, const void* dH, int64_t rows, int64_t lddh, const void* X, int64_t ldx, const void* Wg,
                            const void* Wu, int64_t ldw, const void* Zg, const void* Zu, int64_t ldz, void* dX, int64_t lddx,
                            void* dWg, void* dWu, int32_t dw_dtype, float* dbg, float* dbu) {
  if (!g || !dH || !Zg || !Zu || (dWg == nullptr) != (dWu == nullptr) || (dbg == nullptr) != (dbu == nullptr)) return FW_ERR_INVALID_ARG;
  if (!dX && !dWg && !dbg) return FW_ERR_INVALID_ARG;
  if ((dX && (!Wg || !Wu)) || (dWg && !X)) return FW_ERR_INVALID_ARG;
  if (dWg && dw_dtype != FW_F32 && dw_dtype != FW_BF16) return FW_ERR_INVALID_ARG;
  if (!g->d.grad) return FW_ERR_WORKSPACE;
  if (rows < 1 || rows > g->d.max_rows) return FW_ERR_SHAPE;
  const int M = g->d.M, N = g->d.N, ws = dw_dtype == FW_F32 ? 4 : 2;
  lddh = pitch(rows, N, lddh, 2); ldx = pitch(rows, M, ldx, 2); ldw = pitch(N, M, ldw, 2); ldz = pitch(rows, N, ldz, 2);
  lddx = pitch(rows, M, lddx, 2);
  const View in[6] = {{dH, rows, N, lddh, 2}, {Zg, rows, N, ldz, 2}, {Zu, rows, N, ldz, 2}, {dWg ? X : nullptr, rows, M, ldx, 2},
                      {dX ? Wg : nullptr, N, M, ldw, 2}, {dX ? Wu : nullptr, N, M, ldw, 2}};
  const View out[5] = {{dX, rows, M, lddx, 2}, {dWg, N, M, M, ws}, {dWu, N, M, M, ws}, {dbg, 1, N, N, 4}, {dbu, 1, N, N, 4}};
  fw_status st;
  for (const View& v : in)
    if (v.p && (st = view_check(v)) != FW_OK) return st;
  if (dX && (st = view_check(out[0])) != FW_OK) return st;
  if (!aligned_to(dWg, ws) || !aligned_to(dWu, ws) || !aligned_to(dbg, 4) || !aligned_to(dbu, 4)) return FW_ERR_INVALID_ARG;
  if (!disjoint(out, 5, in, 6)) return FW_ERR_INVALID_ARG;
  if ((st = here(g)) != FW_OK) return st;
  GatedGates q;
  q.dH = dH; q.Zg = Zg; q.Zu = Zu; q.Da = g->Da; q.Db = g->Db; q.dbg = dbg; q.dbu = dbu; q.part = dbg ? g->part : nullptr;
  q.rows = rows; q.lddh = lddh; q.ldz = ldz; q.ldd = g->ldd; q.N = N; q.act = g->d.act; q.slabs = gated_gate_slabs(rows, N);
  const cudaError_t e = launch_gated_gates(q, g->stream);
  if (e != cudaSuccess) {
    fprintf(stderr, "[fw] fw_gated_backward: %s\n", cudaGetErrorString(e));
    return FW_ERR_CUDA;
  }
  if (!dX && !dWg) return FW_OK;
  GatedBackward b;
  b.X = X; b.Wg = Wg; b.Wu = Wu; b.Da = g->Da; b.Db = g->Db; b.dX = dX; b.dWg = dWg; b.dWu = dWu;
  b.rows = rows; b.ldx = ldx; b.ldw = ldw; b.ldd = g->ldd; b.lddx = lddx; b.M = M; b.N = N; b.w_f32 = dw_dtype == FW_F32; b.status = g->status;
  const int64_t mt = ((int64_t)M + 255) / 256;
  if (dX && few_tiles((rows + 255) / 256 * mt)) {
    if ((st = launch_gated_small_dx(b, g->stream)) != FW_OK) return st;
    b.dX = nullptr;
  }
  if (dWg && few_tiles(2 * (((int64_t)N + 255) / 256) * mt)) {
    if ((st = launch_gated_small_dw(b, g->stream)) != FW_OK) return st;
    b.dWg = b.dWu = nullptr;
  }
  return b.dX || b.dWg ? launch_gated_pair_backward(b, g->stream) : FW_OK;
}

fw_status fw_gated_sync_status(fw_gated* g) {
  if (!g) return FW_ERR_INVALID_ARG;
  int32_t code = 0;
  cudaError_t e = cudaMemcpyAsync(&code, g->status, sizeof(code), cudaMemcpyDeviceToHost, g->stream);
  if (e == cudaSuccess) e = cudaStreamSynchronize(g->stream);
  if (e == cudaSuccess && code) e = cudaMemsetAsync(g->status, 0, sizeof(code), g->stream);
  if (e != cudaSuccess) {
    fprintf(stderr, "[fw] fw_gated_sync_status: %s\n", cudaGetErrorString(e));
    return FW_ERR_CUDA;
  }
  return code ? FW_ERR_TIMEOUT : FW_OK;
}

}  // extern "C"
