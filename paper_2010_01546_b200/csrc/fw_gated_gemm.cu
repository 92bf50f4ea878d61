// Matrix products of the gated feed-forward block on CTA pairs (tcgen05 cta_group::2), forward and backward.
//
//   forward   [A | B] = X [Wg ; Wu]^T, H = act(A + bg) * (B + bu)
//   backward  dX = Da Wg + Db Wu;   dWg = Da^T X,  dWu = Db^T X
//
// A pair of CTAs on the two SMs of a TPC computes tiles of 256 x 256 accumulators: each CTA stages its own 128 rows of the left
// operand and half of the right one, 32 KB for 64 of K (of bf16), so the pair asks 64 bytes per clock and SM of L2 at the
// tensor cores' full rate.  Two accumulators (all 512 columns of TMEM) take turns: the epilogue of a tile runs beside the
// products of the next one.  Persistent CTAs walk the tiles eight block rows at a time, so that the operands of the tiles
// in flight stay in L2.
//
// Forward: the right operand of a tile is 128 rows of Wg (staged by the even CTA) and the same 128 of Wu (by the odd one):
// columns j and 128 + j of the accumulator are the two projections of one output, and the epilogue has both at hand.
// Backward: dX runs over the rows of Wg and then of Wu as one long K; its right operand and both operands of the weight
// gradients lie with their long side along K and are taken MN-major as TMA lays them down: no transposed copies.
// The tiles of all three products are one list: dX first, whose tiles are the longest.
#include <cstdio>
#include <cstring>

#include "fw_gated.h"
#include "fw_gated_act.cuh"
#include "fw_rows.cuh"
#include "fw_sm100.cuh"

namespace fw {
namespace {

using namespace sm100;
using rows::pack_bf16;

constexpr int GG_STAGES = 6;
constexpr int GG_OPERAND = 128 * 128;              // bytes of one operand of a stage and CTA: 128 rows of 128 bytes
constexpr int GG_STAGE = 2 * GG_OPERAND;
constexpr int GG_ROOM = 128 * 128;                 // an epilogue half's tile of results: 128 rows of 128 bytes
constexpr int GG_SMEM = GG_STAGES * GG_STAGE + 2 * GG_ROOM + 1024;
constexpr int GG_THREADS = 12 * 32;                // producer, MMA, TMEM, (idle), eight epilogue warps
constexpr int GG_GROUP = 8;                        // block rows walked together
enum { GG_FWD_BF16 = 0, GG_FWD_E4M3 = 1, GG_BWD = 2 };

struct PairProduct {
  int32_t tiles_m, tiles_n, first;                 // block rows (weight gradients: of both matrices) and columns; first tile
  int32_t seg_blocks;                              // dX: K blocks of Wg, after which Wu's come
  int32_t nk;                                      // K blocks of a tile
};
struct PairArgs {
  CUtensorMap a[2], b[2];                          // forward: X, -, Wg, Wu.  backward: Da, Db (K-major), Wg, Wu (MN-major)
  CUtensorMap at[2], bt;                           // backward: Da, Db, X as MN-major operands
  CUtensorMap out[3];                              // forward: H, Zg, Zu.  backward: dX, dWg, dWu
  PairProduct dx, dw;                              // forward: dx
  int32_t tiles;
  int32_t M, N, act, keep, w_f32;
  int32_t whole[3];                                // outputs: 1 rows are whole multiples of 16 bytes long and apart, 0 only apart, -1 neither
  int64_t rows;
  const float *xs, *wgs, *wus, *bg, *bu;
  void* to[3];                                     // the outputs of out[], as addresses
  int64_t ld[3];
  int32_t* status;
};

__device__ __forceinline__ void mma_e4m3_pair(uint32_t tmem_d, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::2.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}\n"
      ::"r"(tmem_d), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate)
      : "memory");
}
// shared -> global, the part of the box that lies inside the tensor
__device__ __forceinline__ void tma_store_2d(const CUtensorMap* m, uint32_t src, int x, int y) {
  asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.bulk_group [%0, {%2, %3}], [%1];" ::"l"(reinterpret_cast<uint64_t>(m)), "r"(src),
               "r"(x), "r"(y)
               : "memory");
}
__device__ __forceinline__ void sts16(uint32_t a, uint32_t x, uint32_t y, uint32_t z, uint32_t w) {
  asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(a), "r"(x), "r"(y), "r"(z), "r"(w) : "memory");
}

// 32 lanes x 32 consecutive 32-bit columns -> 32 registers per thread (thread = lane)
__device__ __forceinline__ void tmem_ld32(uint32_t taddr, uint32_t (&r)[32]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
      "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
        "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]),
        "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]),
        "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(taddr)
      : "memory");
}

struct Tile {
  int kind;                  // 0: forward or dX, 1: weight gradient
  int which;                 // weight gradient: 0 of Wg, 1 of Wu
  int m, n, nk;              // block row and column; K blocks
};
__device__ __forceinline__ Tile tile_at(const PairArgs& g, int t) {
  Tile r;
  const bool dw = t >= g.dw.first;
  const PairProduct& p = dw ? g.dw : g.dx;
  int i = t - p.first;
  r.kind = dw;
  r.which = 0;
  r.nk = p.nk;
  int tm = p.tiles_m;
  if (dw) {
    tm /= 2;
    const int each = tm * p.tiles_n;
    r.which = i >= each;
    i -= r.which * each;
  }
  const int group = i / (GG_GROUP * p.tiles_n);
  i -= group * GG_GROUP * p.tiles_n;
  const int gm = min(GG_GROUP, tm - group * GG_GROUP);
  r.n = i / gm;
  r.m = group * GG_GROUP + (i - r.n * gm);
  return r;
}

template <int KIND>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(GG_THREADS, 1) gated_pair_kernel(const __grid_constant__ PairArgs g) {
  constexpr bool FWD = KIND != GG_BWD;
  constexpr int KB = KIND == GG_FWD_E4M3 ? 128 : 64;   // K of a stage: 128 bytes
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  __shared__ __align__(8) uint64_t bar_full[GG_STAGES], bar_empty[GG_STAGES], bar_accum[2], bar_drained[2];
  __shared__ uint32_t tmem_base_sh;
  __shared__ int abort_flag, never;
  __shared__ int go[2];

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = cluster_ctarank();
  const int pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;
  const uint32_t stages = (smem_u32(smem_raw) + 1023u) & ~1023u;
  const uint32_t rooms = stages + GG_STAGES * GG_STAGE;

  if (threadIdx.x == 0) {
    abort_flag = never = 0;
    for (int s = 0; s < GG_STAGES; ++s) {
      mbar_init(smem_u32(&bar_full[s]), 1);
      mbar_init(smem_u32(&bar_empty[s]), 1);
    }
    for (int b = 0; b < 2; ++b) {
      mbar_init(smem_u32(&bar_accum[b]), 1);
      mbar_init(smem_u32(&bar_drained[b]), 16);        // eight warps of both CTAs
    }
    mbar_fence_init();
  }
  rows::dep_wait();
  if (warp == 2) {
    tmem_alloc_pair(smem_u32(&tmem_base_sh), 512);
    tmem_relinquish_pair();
  }
  __syncthreads();
  tc_fence_before();
  cluster_arrive();
  cluster_wait();
  tc_fence_after();
  const uint32_t tmem_base = tmem_base_sh;
  const volatile int* abortp = &abort_flag;
  const uint32_t peer_abort = mapa_shared(smem_u32(&abort_flag), rank ^ 1u);
#define GG_ABORT(code)              \
  do {                              \
    abort_flag = 1;                 \
    st_cluster_u32(peer_abort, 1u); \
    atomicExch(g.status, (code));   \
  } while (0)

  if (warp == 0) {
    // ---- TMA producer, both CTAs: up to four boxes of a stage, a lane each; bytes are counted on the even CTA's barrier ----
    int s = 0;
    uint32_t ph = 0;
    bool ok = true;
    int issued = 0;
    for (int t = pair; ok && t < g.tiles; t += pairs) {
      const Tile tl = tile_at(g, t);
      const int row0 = 256 * tl.m + 128 * (int)rank;                       // this CTA's rows of the left operand
      const int col0 = FWD ? 128 * tl.n : 256 * tl.n + 128 * (int)rank;    // and its rows (columns) of the right one
      // lane -> box: source, and how its coordinates and place depend on K
      const CUtensorMap *m0 = nullptr, *m1 = nullptr;
      int x = 0, y = 0;
      bool kx = true;                                                      // K along x (K-major) or along y
      uint32_t off = 0;
      bool issue = false;
      if (FWD) {
        issue = lane < 2;
        if (lane == 0) { m0 = &g.a[0]; y = row0; }
        else if (lane == 1) { m0 = &g.b[rank]; y = col0; off = GG_OPERAND; }
        m1 = m0;
      } else if (tl.kind == 0) {
        issue = lane < 3;
        if (lane == 0) { m0 = &g.a[0]; m1 = &g.a[1]; y = row0; }
        else { m0 = &g.b[0]; m1 = &g.b[1]; kx = false; x = col0 + 64 * (lane - 1); off = GG_OPERAND + (lane - 1) * (GG_OPERAND / 2); }
      } else {
        issue = lane < 4;
        kx = false;
        if (lane < 2) { m0 = &g.at[tl.which]; x = row0 + 64 * lane; off = lane * (GG_OPERAND / 2); }
        else { m0 = &g.bt; x = col0 + 64 * (lane - 2); off = GG_OPERAND + (lane - 2) * (GG_OPERAND / 2); }
        m1 = m0;
      }
      const int seg = !FWD && tl.kind == 0 ? g.dx.seg_blocks : tl.nk;
      for (int kb = 0; kb < tl.nk; ++kb) {
        const bool got = mbar_wait(smem_u32(&bar_empty[s]), ph ^ 1, abortp);
        if (!__all_sync(0xffffffffu, got)) {
          if (lane == 0) GG_ABORT(401);
          ok = false;
          break;
        }
        const uint32_t full = smem_u32(&bar_full[s]);
        const uint32_t bar = mapa_shared(full, 0u);
        if (lane == 0 && rank == 0) mbar_expect_tx(full, 2u * GG_STAGE);
        if (issue) {
          const bool second = kb >= seg;
          const int k0 = (second ? kb - seg : kb) * KB;
          tma_load_2d_pair(stages + s * GG_STAGE + off, second ? m1 : m0, kx ? k0 : x, kx ? y : k0, bar);
        }
        ++issued;
        if (++s == GG_STAGES) { s = 0; ph ^= 1; }
      }
    }
    if (!ok && rank == 0) {
      // given up: the copies that are still on their way land before shared memory goes to somebody else
      const int last = issued < GG_STAGES ? issued : GG_STAGES;
      for (int k = 1; k <= last; ++k) {
        const int i = issued - k;
        mbar_wait(smem_u32(&bar_full[i % GG_STAGES]), (uint32_t)(i / GG_STAGES) & 1u, &never, 4096u);
      }
    }
  } else if (warp == 1) {
    // ---- MMA issuer: one thread of the even CTA drives the tensor cores of both SMs ----
    if (rank == 0 && elect_one()) {
      int s = 0, b = 0;
      uint32_t ph = 0, bph = 0;
      bool ok = true;
      for (int t = pair; ok && t < g.tiles; t += pairs) {
        const Tile tl = tile_at(g, t);
        const bool a_mn = !FWD && tl.kind == 1, b_mn = !FWD;
        const uint32_t idesc = KIND == GG_FWD_E4M3 ? make_idesc(0, 256, 0, 0, 256) : make_idesc(1, 256, a_mn, b_mn, 256);
        // K-major: 8-row groups 1024 bytes apart, 32 bytes a step.  MN-major: 64 columns 8 KB apart, 8 K rows 1024 bytes.
        const uint64_t ad = make_smem_desc(stages, a_mn ? GG_OPERAND / 2 : 0, 1024, kSwizzle128B);
        const uint64_t bd = make_smem_desc(stages + GG_OPERAND, b_mn ? GG_OPERAND / 2 : 0, 1024, kSwizzle128B);
        const uint32_t astep = a_mn ? 2048 / 16 : 2, bstep = b_mn ? 2048 / 16 : 2;
        const uint32_t d = tmem_base + (uint32_t)(b * 256);
        if (!mbar_wait(smem_u32(&bar_drained[b]), bph ^ 1, abortp)) { GG_ABORT(402); break; }
        tc_fence_after();
        for (int kb = 0; kb < tl.nk; ++kb) {
          if (!mbar_wait(smem_u32(&bar_full[s]), ph, abortp)) { GG_ABORT(403); ok = false; break; }
          tc_fence_after();
          const uint32_t so = (uint32_t)(s * GG_STAGE) >> 4;
#pragma unroll
          for (int ks = 0; ks < 4; ++ks) {
            if (KIND == GG_FWD_E4M3) mma_e4m3_pair(d, ad + so + ks * astep, bd + so + ks * bstep, idesc, (kb | ks) != 0);
            else mma_bf16_pair(d, ad + so + ks * astep, bd + so + ks * bstep, idesc, (kb | ks) != 0);
          }
          mma_commit_pair(smem_u32(&bar_empty[s]), (uint16_t)3);
          if (++s == GG_STAGES) { s = 0; ph ^= 1; }
        }
        if (!ok) break;
        mma_commit_pair(smem_u32(&bar_accum[b]), (uint16_t)3);
        b ^= 1;
        if (b == 0) bph ^= 1;
      }
    }
  } else if (warp >= 4) {
    // ---- epilogue: a warp has 32 rows; warps 4-7 take the first half of the columns, 8-11 the second.  Results leave through
    //      shared memory in tiles of 128 rows x 128 bytes, one TMA store each. ----
    const int q = warp & 3, half = (warp - 4) >> 2;
    const int r = q * 32 + lane;
    const bool issuer = q == 0 && lane == 0;
    const uint32_t room = rooms + half * GG_ROOM;
    const uint32_t mine = room + r * 128;
    const uint32_t lanes = (uint32_t)(q * 32) << 16;
    int b = 0;
    uint32_t bph = 0;
    auto chunk = [&](int c) { return mine + ((uint32_t)(c ^ (r & 7)) << 4); };
    auto sync_half = [&]() { asm volatile("bar.sync %0, 128;" ::"r"(1 + half) : "memory"); };
    // the tile of results may be written again once the last store has read it
    auto room_free = [&]() {
      if (issuer) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
      sync_half();
    };
    // the tile of results -> output o from (row y, column x) on; it has `height` x `width` elements, of 4 bytes with f32
    auto send = [&](int o, int x, int y, int64_t height, int width, bool f32) {
      if (x + (f32 ? 32 : 64) <= width ? g.whole[o] >= 0 : g.whole[o] > 0) {
        fence_proxy_async_smem();
        sync_half();
        if (issuer && y < height && x < width) {
          tma_store_2d(&g.out[o], room, x, y);
          asm volatile("cp.async.bulk.commit_group;" ::: "memory");
        }
        return;
      }
      // TMA writes whole 16 bytes: where a row ends inside of them, or rows start anywhere (a dense matrix of odd width), a warp
      // copies its own 32 rows element by element
      __syncwarp();
      for (int i = 0; i < 32; ++i) {
        const int rr = q * 32 + i;
        if (y + rr >= height) break;
        const uint32_t at = room + rr * 128 + ((uint32_t)((lane >> 2) ^ (rr & 7)) << 4) + (lane & 3) * 4;
        uint32_t w;
        asm volatile("ld.shared.b32 %0, [%1];" : "=r"(w) : "r"(at) : "memory");
        const int64_t row = (int64_t)(y + rr) * g.ld[o];
        if (f32) {
          if (x + lane < width) static_cast<float*>(g.to[o])[row + x + lane] = __uint_as_float(w);
        } else {
          uint16_t* d = static_cast<uint16_t*>(g.to[o]) + row + x + 2 * lane;
          if (x + 2 * lane < width) d[0] = (uint16_t)w;
          if (x + 2 * lane + 1 < width) d[1] = (uint16_t)(w >> 16);
        }
      }
    };
    for (int t = pair; t < g.tiles; t += pairs) {
      const Tile tl = tile_at(g, t);
      if (!mbar_wait(smem_u32(&bar_accum[b]), bph, abortp) && lane == 0) GG_ABORT(404);
      sync_half();
      if (issuer) go[half] = *abortp == 0;          // one verdict: the half's warps take the barriers below or none does
      sync_half();
      if (!go[half]) break;
      tc_fence_after();
      const uint32_t drained = mapa_shared(smem_u32(&bar_drained[b]), 0u);
      const uint32_t acc = tmem_base + lanes + (uint32_t)(b * 256);
      // every accumulator of this warp has been read: the buffer is the next but one tile's
      auto all_read = [&]() {
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive_cluster(drained);
      };
      const int m0 = 256 * tl.m + 128 * (int)rank, row = m0 + r;
      if (FWD) {
        const int n0 = 128 * tl.n + 64 * half;      // this half's 64 outputs
        const float xs = KIND == GG_FWD_E4M3 && row < g.rows ? g.xs[row] : 1.f;
        // 32 projections of one kind from accumulator column c on (output n0 + j): scaled, with their bias
        auto project = [&](float (&v)[32], int c, int j0, const float* ws, const float* bias) {
          tmem_ld32(acc + (uint32_t)c, reinterpret_cast<uint32_t(&)[32]>(v));
          tmem_ld_wait();
          if (KIND == GG_FWD_E4M3) {
#pragma unroll
            for (int j = 0; j < 32; ++j) v[j] *= xs * (n0 + j0 + j < g.N ? ws[n0 + j0 + j] : 0.f);
          }
          if (bias) {
#pragma unroll
            for (int j = 0; j < 32; ++j) v[j] += n0 + j0 + j < g.N ? bias[n0 + j0 + j] : 0.f;
          }
        };
        auto put32 = [&](const float (&v)[32], int j0) {
#pragma unroll
          for (int c = 0; c < 4; ++c)
            sts16(chunk(j0 / 8 + c), pack_bf16(v[8 * c], v[8 * c + 1]), pack_bf16(v[8 * c + 2], v[8 * c + 3]),
                  pack_bf16(v[8 * c + 4], v[8 * c + 5]), pack_bf16(v[8 * c + 6], v[8 * c + 7]));
        };
        if (g.keep) {
          for (int k = 0; k < 2; ++k) {
            room_free();
            for (int j0 = 0; j0 < 64; j0 += 32) {
              float v[32];
              project(v, 128 * k + 64 * half + j0, j0, k ? g.wus : g.wgs, k ? g.bu : g.bg);
              put32(v, j0);
            }
            send(1 + k, n0, m0, g.rows, g.N, false);
          }
        }
        room_free();
        with_act(g.act, [&](auto a) {
          for (int j0 = 0; j0 < 64; j0 += 32) {
            float v[32], u[32];
            project(v, 64 * half + j0, j0, g.wgs, g.bg);
            project(u, 128 + 64 * half + j0, j0, g.wus, g.bu);
            if (j0 == 32) all_read();
#pragma unroll
            for (int j = 0; j < 32; ++j) v[j] = a.value(v[j]) * u[j];
            put32(v, j0);
          }
        });
        send(0, n0, m0, g.rows, g.N, false);
      } else {
        const int n0 = 256 * tl.n + 128 * half;     // this half's 128 columns
        const bool f32 = tl.kind == 1 && g.w_f32;
        const int64_t height = tl.kind == 1 ? g.N : g.rows;
        const int wide = f32 ? 32 : 64;             // columns of 128 bytes
        for (int c0 = 0; c0 < 128; c0 += wide) {
          room_free();
          for (int j0 = 0; j0 < wide; j0 += 32) {
            uint32_t v[32];
            tmem_ld32(acc + (uint32_t)(128 * half + c0 + j0), v);
            tmem_ld_wait();
            if (c0 + j0 == 96) all_read();
            if (f32) {
#pragma unroll
              for (int c = 0; c < 8; ++c) sts16(chunk(c), v[4 * c], v[4 * c + 1], v[4 * c + 2], v[4 * c + 3]);
            } else {
#pragma unroll
              for (int c = 0; c < 4; ++c) {
                const float* f = reinterpret_cast<const float*>(v) + 8 * c;
                sts16(chunk(j0 / 8 + c), pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]), pack_bf16(f[4], f[5]), pack_bf16(f[6], f[7]));
              }
            }
          }
          const int x = n0 + c0;
          send(tl.kind == 1 ? 1 + tl.which : 0, x, m0, height, g.M, f32);
        }
      }
      b ^= 1;
      if (b == 0) bph ^= 1;
    }
    if (issuer) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");       // no CTA leaves before its copies have
  }
#undef GG_ABORT
  rows::dep_trigger();
  tc_fence_before();
  cluster_arrive();
  cluster_wait();
  if (warp == 2) {
    tc_fence_after();
    tmem_dealloc_pair(tmem_base, 512);
  }
}

int resident(int tiles) {
  const int most = sm_count() / 2;
  return tiles < most ? tiles : most;
}

template <int KIND>
fw_status launch(const PairArgs& g, cudaStream_t s, const char* what) {
  static SmemAttrCache cache;
  cudaError_t e = ensure_dyn_smem(gated_pair_kernel<KIND>, GG_SMEM, cache);
  if (e == cudaSuccess) {
    ProfScope ps(FW_PROF_MISC, s);
    e = launch_dep(gated_pair_kernel<KIND>, 2 * resident(g.tiles), GG_THREADS, GG_SMEM, s, g);
  }
  if (e == cudaSuccess) return FW_OK;
  fprintf(stderr, "[fw] %s: %s\n", what, cudaGetErrorString(e));
  return FW_ERR_CUDA;
}

int blocks(int64_t n, int each) { return (int)((n + each - 1) / each); }

}  // namespace

fw_status launch_gated_pair_forward(const GatedForward& f, cudaStream_t s) {
  PairArgs g;
  memset(&g, 0, sizeof(g));
  const int es = f.e4m3 ? 1 : 2, kb = f.e4m3 ? 128 : 64;
  bool ok = tmap_encode_rows128(&g.a[0], es, f.X, f.M, f.rows, f.ldx, 128) && tmap_encode_rows128(&g.b[0], es, f.Wg, f.M, f.N, f.ldw, 128) &&
            tmap_encode_rows128(&g.b[1], es, f.Wu, f.M, f.N, f.ldw, 128) && tmap_encode_rows128(&g.out[0], 2, f.H, f.N, f.rows, f.ldh, 128);
  g.keep = f.Zg != nullptr;
  g.to[0] = f.H; g.to[1] = f.Zg; g.to[2] = f.Zu; g.ld[0] = f.ldh; g.ld[1] = g.ld[2] = f.ldz;
  g.whole[0] = g.whole[1] = g.whole[2] = f.N % 8 == 0;
  if (g.keep) ok = ok && tmap_encode_rows128(&g.out[1], 2, f.Zg, f.N, f.rows, f.ldz, 128) && tmap_encode_rows128(&g.out[2], 2, f.Zu, f.N, f.rows, f.ldz, 128);
  if (!ok) {
    fprintf(stderr, "[fw] tensor-map encoding failed (gated block, forward)\n");
    return FW_ERR_CUDA;
  }
  g.dx.tiles_m = blocks(f.rows, 256); g.dx.tiles_n = blocks(f.N, 128);
  g.dx.nk = g.dx.seg_blocks = blocks(f.M, kb);
  g.tiles = g.dw.first = g.dx.tiles_m * g.dx.tiles_n;
  g.M = f.M; g.N = f.N; g.rows = f.rows; g.act = f.act;
  g.xs = f.xs; g.wgs = f.wgs; g.wus = f.wus; g.bg = f.bg; g.bu = f.bu;
  g.status = f.status;
  return f.e4m3 ? launch<GG_FWD_E4M3>(g, s, "fw_gated_forward") : launch<GG_FWD_BF16>(g, s, "fw_gated_forward");
}

fw_status launch_gated_pair_backward(const GatedBackward& b, cudaStream_t s) {
  PairArgs g;
  memset(&g, 0, sizeof(g));
  bool ok = true;
  if (b.dX) {
    ok = ok && tmap_encode_rows128(&g.a[0], 2, b.Da, b.N, b.rows, b.ldd, 128) && tmap_encode_rows128(&g.a[1], 2, b.Db, b.N, b.rows, b.ldd, 128) &&
         tmap_encode_rows128(&g.b[0], 2, b.Wg, b.M, b.N, b.ldw, 64) && tmap_encode_rows128(&g.b[1], 2, b.Wu, b.M, b.N, b.ldw, 64) &&
         tmap_encode_rows128(&g.out[0], 2, b.dX, b.M, b.rows, b.lddx, 128);
    g.to[0] = b.dX; g.ld[0] = b.lddx; g.whole[0] = b.M % 8 == 0;
    g.dx.tiles_m = blocks(b.rows, 256); g.dx.tiles_n = blocks(b.M, 256);
    g.dx.seg_blocks = blocks(b.N, 64); g.dx.nk = 2 * g.dx.seg_blocks;
  }
  g.dw.first = g.tiles = g.dx.tiles_m * g.dx.tiles_n;
  if (b.dWg) {
    const int es = b.w_f32 ? 4 : 2;
    g.w_f32 = b.w_f32;
    g.to[1] = b.dWg; g.to[2] = b.dWu; g.ld[1] = g.ld[2] = b.M;
    const bool aligned = ((int64_t)b.M * es) % 16 == 0 && reinterpret_cast<uintptr_t>(b.dWg) % 16 == 0 && reinterpret_cast<uintptr_t>(b.dWu) % 16 == 0;
    g.whole[1] = g.whole[2] = aligned ? 1 : -1;
    ok = ok && tmap_encode_rows128(&g.at[0], 2, b.Da, b.N, b.rows, b.ldd, 64) && tmap_encode_rows128(&g.at[1], 2, b.Db, b.N, b.rows, b.ldd, 64) &&
         tmap_encode_rows128(&g.bt, 2, b.X, b.M, b.rows, b.ldx, 64);
    if (aligned)
      ok = ok && tmap_encode_rows128(&g.out[1], es, b.dWg, b.M, b.N, b.M, 128) && tmap_encode_rows128(&g.out[2], es, b.dWu, b.M, b.N, b.M, 128);
    g.dw.tiles_m = 2 * blocks(b.N, 256); g.dw.tiles_n = blocks(b.M, 256);
    g.dw.nk = blocks(b.rows, 64);
    g.tiles += g.dw.tiles_m * g.dw.tiles_n;
  }
  if (!ok) {
    fprintf(stderr, "[fw] tensor-map encoding failed (gated block, backward)\n");
    return FW_ERR_CUDA;
  }
  g.M = b.M; g.N = b.N; g.rows = b.rows;
  g.status = b.status;
  return launch<GG_BWD>(g, s, "fw_gated_backward");
}

}  // namespace fw
