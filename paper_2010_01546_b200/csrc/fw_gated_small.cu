// Products of the gated feed-forward block with few tiles: single tokens, small batches, narrow blocks.
//
// A CTA has a tile of 128 rows and 32 to 128 outputs (forward: of both projections, so twice as many accumulator columns) and
// a share of K; the CTAs of a cluster share a tile's K.  Their accumulators meet in shared memory: each CTA of the cluster
// adds all shares of its part of the outputs, in order, and finishes it (scales, bias, activation, product).
//
// With few rows the weights are read once from HBM and everything else is small: what counts is that every SM has its loads in
// flight from the first moment to the last, so the tiles are narrow and K is split until there are two CTAs a SM or more.  Of X
// only the rows that exist are staged (16 to 128); the tensor core's other rows compute on whatever lies there and are dropped.
// The products of backward passes with few tiles come here too: their operands are taken as they lie (K-major or MN-major).
#include <cstdio>
#include <cstring>

#include "fw_gated.h"
#include "fw_gated_act.cuh"
#include "fw_rows.cuh"
#include "fw_sm100.cuh"

namespace fw {
namespace {

using namespace sm100;

constexpr int GS_MAX_STAGES = 8, GS_MAX_SPLITS = 8;
constexpr int GS_THREADS = 6 * 32;                 // producer, MMA, four epilogue warps
enum { GS_FWD_BF16 = 0, GS_FWD_E4M3 = 1, GS_DX = 2, GS_DW = 3 };

struct SmallArgs {
  CUtensorMap a[2], b[2];         // forward: X, -, Wg, Wu.  dX: Da, Db, Wg, Wu.  weight gradients: Da, Db, X, -
  void* out[3];                   // forward: H, Zg, Zu.  dX.  dWg, dWu
  int64_t ld[3];
  const float *xs, *wgs, *wus, *bg, *bu;
  int64_t height;                 // rows of the outputs
  int32_t width;                  // and columns
  int32_t nk, seg;                // K blocks in all, and of the first operand pair
  int32_t splits;                 // CTAs of a tile
  int32_t a_rows;                 // rows of the left operand that are staged (K-major)
  int32_t stages, stage_bytes, a_bytes;
  int32_t act, f32, vec;          // vec: four outputs at a time may be stored as one
  int32_t* status;
};

__device__ __forceinline__ void mma_e4m3(uint32_t tmem_d, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}\n"
      ::"r"(tmem_d), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate)
      : "memory");
}
__device__ __forceinline__ float4 ld_cluster4(uint32_t addr) {
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr) : "memory");
  return v;
}
__device__ __forceinline__ void sts4(uint32_t a, const uint32_t* v) {
  asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(a), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]) : "memory");
}

// n neighbouring values of a row, as many as the matrix has, in one access where that may be
template <int n>
__device__ __forceinline__ void put_row(const SmallArgs& g, int o, int64_t row, int col, const float (&v)[n], bool f32) {
  const int left = g.width - col;
  const int64_t at = row * g.ld[o] + col;
  if (f32) {
    float* p = static_cast<float*>(g.out[o]) + at;
    if (g.vec && left >= n) {
#pragma unroll
      for (int e = 0; e < n; e += 4) *reinterpret_cast<float4*>(p + e) = make_float4(v[e], v[e + 1], v[e + 2], v[e + 3]);
    } else {
#pragma unroll
      for (int e = 0; e < n; ++e)
        if (e < left) p[e] = v[e];
    }
  } else {
    __nv_bfloat16* p = static_cast<__nv_bfloat16*>(g.out[o]) + at;
    if (g.vec && left >= n) {
#pragma unroll
      for (int e = 0; e < n; e += 4) *reinterpret_cast<uint2*>(p + e) = make_uint2(rows::pack_bf16(v[e], v[e + 1]), rows::pack_bf16(v[e + 2], v[e + 3]));
    } else {
#pragma unroll
      for (int e = 0; e < n; ++e)
        if (e < left) p[e] = __float2bfloat16_rn(v[e]);
    }
  }
}
// n neighbouring outputs from their sums: of one matrix, or of both projections
template <int KIND, int n>
__device__ __forceinline__ void finish(const SmallArgs& g, int which, int64_t row, int col, float (&a)[n], float (&b)[n]) {
  if (KIND > GS_FWD_E4M3) {
    put_row<n>(g, KIND == GS_DW ? which : 0, row, col, a, KIND == GS_DW && g.f32);
    return;
  }
  const int left = g.width - col;
  const float xs = KIND == GS_FWD_E4M3 ? g.xs[row] : 1.f;
#pragma unroll
  for (int e = 0; e < n; ++e) {
    if (e < left) {
      if (KIND == GS_FWD_E4M3) { a[e] *= xs * g.wgs[col + e]; b[e] *= xs * g.wus[col + e]; }
      if (g.bg) { a[e] += g.bg[col + e]; b[e] += g.bu[col + e]; }
    }
  }
  if (g.out[1]) { put_row<n>(g, 1, row, col, a, false); put_row<n>(g, 2, row, col, b, false); }
  with_act(g.act, [&](auto act) {
#pragma unroll
    for (int e = 0; e < n; ++e) a[e] = act.value(a[e]) * b[e];
  });
  put_row<n>(g, 0, row, col, a, false);
}

// F: outputs of a tile; the accumulator has NT columns.  Grid: (column tiles x splits, row tiles, matrices).
template <int KIND, int F>
__global__ void __launch_bounds__(GS_THREADS, KIND <= GS_FWD_E4M3 && F == 32 ? 4 : 2) gated_small_kernel(const __grid_constant__ SmallArgs g) {
  constexpr bool FWD = KIND <= GS_FWD_E4M3;
  constexpr int NT = FWD ? 2 * F : F;
  constexpr int KB = KIND == GS_FWD_E4M3 ? 128 : 64;
  constexpr bool A_MN = KIND == GS_DW, B_MN = !FWD;
  constexpr int PITCH = NT + 4;                    // floats of a row of partial sums: 16-byte stores of neighbouring rows on distinct banks
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  __shared__ __align__(8) uint64_t bar_full[GS_MAX_STAGES], bar_empty[GS_MAX_STAGES], bar_accum;
  __shared__ uint32_t tmem_base_sh;
  __shared__ int abort_flag, never;

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int S = g.splits, rank = (int)blockIdx.x % S, tile = (int)blockIdx.x / S, which = blockIdx.z;
  const int n0 = tile * F, m0 = (int)blockIdx.y * 128;
  const int k0 = (int)((int64_t)g.nk * rank / S), nk = (int)((int64_t)g.nk * (rank + 1) / S) - k0;
  const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  const int stages = g.stages;
  const bool direct = S == 1 && !(FWD && g.out[1]);

  if (threadIdx.x == 0) {
    abort_flag = never = 0;
    for (int s = 0; s < stages; ++s) {
      mbar_init(smem_u32(&bar_full[s]), 1);
      mbar_init(smem_u32(&bar_empty[s]), 1);
    }
    mbar_init(smem_u32(&bar_accum), 1);
    mbar_fence_init();
    tma_prefetch_desc(&g.a[0]);
    tma_prefetch_desc(&g.b[0]);
    if (FWD) tma_prefetch_desc(&g.b[1]);
  }
  dep_sync();
  if (warp == 1) {                                 // after the wait: a grid before this one may still need columns (see dep_sync)
    tmem_alloc(smem_u32(&tmem_base_sh), NT < 32 ? 32 : NT);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = tmem_base_sh;
  const volatile int* abortp = &abort_flag;
#define GS_ABORT(code)            \
  do {                            \
    abort_flag = 1;               \
    atomicExch(g.status, (code)); \
  } while (0)

  if (warp == 0) {
    // ---- TMA producer: a lane for each box of a stage ----
    // lane -> box: left operand (one box of a_rows, or two of 64 columns), right operand (forward: Wg, Wu; else F / 64 boxes)
    const int na = A_MN ? 2 : 1, nb = FWD ? 2 : F / 64;
    const bool issue = lane < na + nb;
    const bool left = lane < na;
    const int i = left ? lane : lane - na;
    const bool kx = left ? !A_MN : !B_MN;                                   // K along x
    const int fix = left ? (A_MN ? m0 + 64 * i : m0) : (FWD ? n0 : n0 + 64 * i);
    const uint32_t off = left ? (uint32_t)i * 8192u : (uint32_t)g.a_bytes + (uint32_t)i * (FWD ? F * 128u : 8192u);
    const uint32_t bytes = (uint32_t)g.stage_bytes;
    uint32_t ph = 0;
    int s = 0, issued = 0;
    bool ok = true;
    for (int kb = k0; kb < k0 + nk; ++kb) {
      const bool got = mbar_wait(smem_u32(&bar_empty[s]), ph ^ 1, abortp);
      if (!__all_sync(0xffffffffu, got)) {
        if (lane == 0) GS_ABORT(411);
        ok = false;
        break;
      }
      const uint32_t full = smem_u32(&bar_full[s]);
      if (lane == 0) mbar_expect_tx(full, bytes);
      __syncwarp();
      if (issue) {
        const bool second = KIND == GS_DX && kb >= g.seg;
        const int k = (second ? kb - g.seg : kb) * KB;
        const CUtensorMap* m = left ? &g.a[KIND == GS_DW ? which : second ? 1 : 0] : &g.b[FWD ? i : KIND == GS_DW ? 0 : second ? 1 : 0];
        tma_load_2d(base + s * bytes + off, m, kx ? k : fix, kx ? fix : k, full);
      }
      ++issued;
      if (++s == stages) { s = 0; ph ^= 1; }
    }
    if (!ok) {
      // given up: the copies that are still on their way land before shared memory goes to somebody else
      const int last = issued < stages ? issued : stages;
      for (int k = 1; k <= last; ++k) mbar_wait(smem_u32(&bar_full[(issued - k) % stages]), (uint32_t)((issued - k) / stages) & 1u, &never, 4096u);
    }
  } else if (warp == 1) {
    if (elect_one()) {
      const uint32_t idesc = make_idesc(KIND == GS_FWD_E4M3 ? 0 : 1, NT, A_MN, B_MN, 128);
      const uint64_t ad = make_smem_desc(base, A_MN ? 8192 : 0, 1024, kSwizzle128B);
      const uint64_t bd = make_smem_desc(base + g.a_bytes, B_MN ? 8192 : 0, 1024, kSwizzle128B);
      constexpr uint32_t astep = A_MN ? 2048 / 16 : 2, bstep = B_MN ? 2048 / 16 : 2;
      uint32_t ph = 0;
      int s = 0;
      bool ok = true;
      for (int kb = 0; kb < nk; ++kb) {
        if (!mbar_wait(smem_u32(&bar_full[s]), ph, abortp)) { GS_ABORT(412); ok = false; break; }
        tc_fence_after();
        const uint32_t so = (uint32_t)(s * g.stage_bytes) >> 4;
#pragma unroll
        for (int ks = 0; ks < 4; ++ks) {
          if (KIND == GS_FWD_E4M3) mma_e4m3(tmem_base, ad + so + ks * astep, bd + so + ks * bstep, idesc, (kb | ks) != 0);
          else mma_bf16(tmem_base, ad + so + ks * astep, bd + so + ks * bstep, idesc, (kb | ks) != 0);
        }
        mma_commit(smem_u32(&bar_empty[s]));
        if (++s == stages) { s = 0; ph ^= 1; }
      }
      if (ok) mma_commit(smem_u32(&bar_accum));
    }
    __syncwarp();
  } else {
    // ---- epilogue, a row a thread: the results themselves where the tile is this CTA's alone, else its share to shared memory
    //      (every product has read its operands).  With both projections kept they go through shared memory too: three outputs
    //      of 32 bytes a row are more stores than the way around (512 rows, 1024 x 2816: 20.9 us against 16.8). ----
    const int q = warp & 3, r = q * 32 + lane;
    const int64_t left = g.height - m0;
    if (q * 32 < left) {
      const bool got = mbar_wait(smem_u32(&bar_accum), 0, abortp);
      if (!__all_sync(0xffffffffu, got)) {
        if (lane == 0) GS_ABORT(413);
      } else {
        tc_fence_after();
        const uint32_t row = base + (uint32_t)(r * PITCH) * 4u, lanes = tmem_base + ((uint32_t)(q * 32) << 16);
        if (!direct) {
#pragma unroll
          for (int c = 0; c < NT; c += 16) {
            uint32_t v[16];
            tmem_ld16(lanes + (uint32_t)c, v);
            tmem_ld_wait();
            if (r < left) {
#pragma unroll
              for (int j = 0; j < 16; j += 4) sts4(row + (uint32_t)(c + j) * 4u, v + j);
            }
          }
        } else {
#pragma unroll 1
          for (int c = 0; c < F; c += 16) {
            float a[16], b[16];
            tmem_ld16(lanes + (uint32_t)c, reinterpret_cast<uint32_t(&)[16]>(a));
            if (FWD) tmem_ld16(lanes + (uint32_t)(F + c), reinterpret_cast<uint32_t(&)[16]>(b));
            tmem_ld_wait();
            if (r < left && n0 + c < g.width) finish<KIND, 16>(g, which, m0 + r, n0 + c, a, b);
          }
        }
      }
    }
  }
#undef GS_ABORT
  tc_fence_before();
  __syncthreads();
  if (S > 1) { cluster_arrive(); cluster_wait(); }

  // ---- four neighbouring outputs a thread, of this CTA's part of the columns: all shares in order ----
  if (!direct && !abort_flag) {
    const int part = F / S, quads = part / 4;       // a power of two
    const int have = (int)(g.height - m0 < 128 ? g.height - m0 : 128);
    for (int i = threadIdx.x; i < have * quads; i += GS_THREADS) {
      const int r = i / quads, j = rank * part + (i - r * quads) * 4, col = n0 + j;
      if (col >= g.width) continue;
      const uint32_t at = base + (uint32_t)(r * PITCH + j) * 4u;
      float a[4] = {0.f, 0.f, 0.f, 0.f}, b[4] = {0.f, 0.f, 0.f, 0.f};
      // four shares' loads before their sums: one by one the latency of another SM's shared memory was most of the kernel (333 x 1000 x
      // 1367 in eight shares: 38 us; all eight at once take registers that cost a single token one of its four CTAs a SM)
      for (int s0 = 0; s0 < S; s0 += 4) {
        float4 x[4], y[4];
#pragma unroll
        for (int s = 0; s < 4; ++s) {
          if (s0 + s < S) {
            const uint32_t from = mapa_shared(at, (uint32_t)(s0 + s));
            x[s] = ld_cluster4(from);
            if (FWD) y[s] = ld_cluster4(from + F * 4);
          }
        }
#pragma unroll
        for (int s = 0; s < 4; ++s) {
          if (s0 + s < S) {
            a[0] += x[s].x; a[1] += x[s].y; a[2] += x[s].z; a[3] += x[s].w;
            if (FWD) { b[0] += y[s].x; b[1] += y[s].y; b[2] += y[s].z; b[3] += y[s].w; }
          }
        }
      }
      finish<KIND, 4>(g, which, m0 + r, col, a, b);
    }
  }
  // no CTA leaves while its shares are being read
  if (S > 1) { cluster_arrive(); cluster_wait(); }
  else __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem_base, NT < 32 ? 32 : NT);
  }
}

int blocks(int64_t n, int each) { return (int)((n + each - 1) / each); }

template <int KIND, int F>
fw_status launch(SmallArgs& g, int matrices, cudaStream_t s, const char* what) {
  constexpr int NT = KIND <= GS_FWD_E4M3 ? 2 * F : F;
  const int mt = blocks(g.height, 128), nt = blocks(g.width, F);
  // K is shared by up to eight CTAs, four blocks of it each at least (the exchange of a cluster takes as long), until three SMs of
  // four have one; where 16 blocks each are left, until there are 1.5 a SM, with few rows two: loads in flight are what counts
  // there (64 rows, 4096 x 8192: 28.7 us against 34.7; 512 rows, 1024 x 2816, 8 blocks each: 22.7 against 16.9)
  const int64_t tiles = (int64_t)mt * nt * matrices, sms = sm_count();
  int S = 1;
  while (S < GS_MAX_SPLITS && g.nk >= 8 * S && (4 * tiles * S < 3 * sms || (g.nk >= 32 * S && 2 * tiles * S < (g.height <= 32 ? 4 : 3) * sms))) S *= 2;
  g.splits = S;
  g.a_bytes = KIND == GS_DW ? 128 * 128 : g.a_rows * 128;
  g.stage_bytes = g.a_bytes + NT * 128;
  const int most = blocks(g.nk, S);
  // four CTAs a SM with 64 accumulator columns, two with more
  const int budget = (NT <= 64 ? 48 : 104) * 1024;
  int st = budget / g.stage_bytes;
  if (st > GS_MAX_STAGES) st = GS_MAX_STAGES;
  if (st > most) st = most;
  if (st < 2) st = 2;
  g.stages = st;
  // the tensor core reads 128 rows of the left operand whatever was staged; the partial sums lie over the stages
  const int have = g.height < 128 ? (int)g.height : 128;
  size_t smem = (size_t)st * g.stage_bytes;
  if (g.stage_bytes < 128 * 128) smem += 128 * 128 - g.stage_bytes;
  const size_t part = (size_t)have * (NT + 4) * 4;
  if (smem < part) smem = part;
  smem += 1024;
  static SmemAttrCache cache;
  cudaError_t e = ensure_dyn_smem(gated_small_kernel<KIND, F>, smem, cache);
  if (e == cudaSuccess) {
    ProfScope ps(FW_PROF_MISC, s);
    e = launch_dep_cluster(S, gated_small_kernel<KIND, F>, dim3(nt * S, mt, matrices), GS_THREADS, smem, s, g);
  }
  if (e == cudaSuccess) return FW_OK;
  fprintf(stderr, "[fw] %s: %s\n", what, cudaGetErrorString(e));
  return FW_ERR_CUDA;
}

int staged_rows(int64_t rows) {
  int r = 16;
  while (r < 128 && r < rows) r *= 2;
  return r;
}

}  // namespace

fw_status launch_gated_small_forward(const GatedForward& f, cudaStream_t s) {
  SmallArgs g;
  memset(&g, 0, sizeof(g));
  const int es = f.e4m3 ? 1 : 2, F = f.rows <= 32 ? 32 : 64;
  g.a_rows = staged_rows(f.rows);
  if (!(tmap_encode_rows128(&g.a[0], es, f.X, f.M, f.rows, f.ldx, g.a_rows) && tmap_encode_rows128(&g.b[0], es, f.Wg, f.M, f.N, f.ldw, F) &&
        tmap_encode_rows128(&g.b[1], es, f.Wu, f.M, f.N, f.ldw, F))) {
    fprintf(stderr, "[fw] tensor-map encoding failed (gated block, forward)\n");
    return FW_ERR_CUDA;
  }
  g.out[0] = f.H; g.out[1] = f.Zg; g.out[2] = f.Zu; g.ld[0] = f.ldh; g.ld[1] = g.ld[2] = f.ldz;
  g.xs = f.xs; g.wgs = f.wgs; g.wus = f.wus; g.bg = f.bg; g.bu = f.bu;
  g.height = f.rows; g.width = f.N; g.nk = g.seg = blocks(f.M, f.e4m3 ? 128 : 64);
  g.act = f.act; g.vec = 1; g.status = f.status;
  const char* what = "fw_gated_forward";
  if (f.e4m3) return F == 32 ? launch<GS_FWD_E4M3, 32>(g, 1, s, what) : launch<GS_FWD_E4M3, 64>(g, 1, s, what);
  return F == 32 ? launch<GS_FWD_BF16, 32>(g, 1, s, what) : launch<GS_FWD_BF16, 64>(g, 1, s, what);
}

fw_status launch_gated_small_dx(const GatedBackward& b, cudaStream_t s) {
  SmallArgs g;
  memset(&g, 0, sizeof(g));
  g.a_rows = staged_rows(b.rows);
  if (!(tmap_encode_rows128(&g.a[0], 2, b.Da, b.N, b.rows, b.ldd, g.a_rows) && tmap_encode_rows128(&g.a[1], 2, b.Db, b.N, b.rows, b.ldd, g.a_rows) &&
        tmap_encode_rows128(&g.b[0], 2, b.Wg, b.M, b.N, b.ldw, 64) && tmap_encode_rows128(&g.b[1], 2, b.Wu, b.M, b.N, b.ldw, 64))) {
    fprintf(stderr, "[fw] tensor-map encoding failed (gated block, dX)\n");
    return FW_ERR_CUDA;
  }
  g.out[0] = b.dX; g.ld[0] = b.lddx;
  g.height = b.rows; g.width = b.M; g.seg = blocks(b.N, 64); g.nk = 2 * g.seg;
  g.vec = 1; g.status = b.status;
  return b.rows <= 32 ? launch<GS_DX, 64>(g, 1, s, "fw_gated_backward") : launch<GS_DX, 128>(g, 1, s, "fw_gated_backward");
}

fw_status launch_gated_small_dw(const GatedBackward& b, cudaStream_t s) {
  SmallArgs g;
  memset(&g, 0, sizeof(g));
  if (!(tmap_encode_rows128(&g.a[0], 2, b.Da, b.N, b.rows, b.ldd, 64) && tmap_encode_rows128(&g.a[1], 2, b.Db, b.N, b.rows, b.ldd, 64) &&
        tmap_encode_rows128(&g.b[0], 2, b.X, b.M, b.rows, b.ldx, 64))) {
    fprintf(stderr, "[fw] tensor-map encoding failed (gated block, weight gradients)\n");
    return FW_ERR_CUDA;
  }
  g.out[0] = b.dWg; g.out[1] = b.dWu; g.ld[0] = g.ld[1] = b.M;
  g.height = b.N; g.width = b.M; g.nk = g.seg = blocks(b.rows, 64);
  g.f32 = b.w_f32; g.status = b.status;
  const int need = b.w_f32 ? 16 : 8;
  g.vec = b.M % 4 == 0 && reinterpret_cast<uintptr_t>(b.dWg) % need == 0 && reinterpret_cast<uintptr_t>(b.dWu) % need == 0;
  return launch<GS_DW, 128>(g, 2, s, "fw_gated_backward");
}

}  // namespace fw
