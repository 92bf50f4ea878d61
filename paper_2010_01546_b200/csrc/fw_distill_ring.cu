// Distillation loss of long rows (see fw_distill.cu).
#include <cstring>
#include <mutex>

#include "fw_distill.cuh"
#include "fw_sm100.cuh"

namespace fw {
namespace distill {
namespace {

// ---------------------------------------------------------------------------
// Long rows.  A row is a chain of latencies (entries, their logits, the slice, an exchange over the cluster, stores), and with a
// CTA for each slice of each row the chains and not the bytes took the time: 4096 x 131072 bf16 1708 us.  So clusters stay and
// walk the rows, everything is on its way before it is needed, and the entries have a warp of their own:
//   eight warps   classes of the slice: cp.async two rows ahead (a thread reads back only what it copied: no barrier), exponentials
//                 in registers, each warp's sum sent to every CTA of the cluster (st.async, counted in bytes there), the gradient
//                 once the factor is known;
//   one warp      entries of the next row: repeated classes, bit set, sums of the teacher's and of the named classes;
//   one warp      all sums, the factor and the loss; the named classes' gradient of the row before over the eight warps' stores;
//                 and entries copied ahead, class and teacher's logit 2 kAheadRows + 1 rows, the student's logit kAheadRows + 1.
// They meet on mbarriers, a CTA has no common barrier.  With the entries spread over the eight warps, a barrier a row and every
// thread working out the factor, the fixed part of a row was 650 instructions a warp beside 320 for its classes: 690 us.
// ---------------------------------------------------------------------------
constexpr int kRingWarps = 8, kRingThreads = 32 * kRingWarps, kRingSlots = 3, kRingMaxK = 256, kRingMaxCtas = 16;
constexpr int kRingAll = kRingThreads + 64;
constexpr int kAheadRows = 1, kEntrySlots = 2 * kAheadRows + 4;
constexpr int kSeenBits = 16384;

// to a place in a CTA of the cluster, counted in bytes on that CTA's barrier
__device__ __forceinline__ void send_pair(uint32_t addr, MaxSum v, uint32_t bar) {
  asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.v2.f32 [%0], {%1, %2}, [%3];" ::"r"(addr), "f"(v.m), "f"(v.l), "r"(bar)
               : "memory");
}
__device__ __forceinline__ void ahead4(uint32_t to, const void* from) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(to), "l"(from) : "memory");
}
__device__ __forceinline__ void unpack16(uint4 q, float (&v)[8]) {
  v[0] = bf16_lo(q.x); v[1] = bf16_hi(q.x); v[2] = bf16_lo(q.y); v[3] = bf16_hi(q.y);
  v[4] = bf16_lo(q.z); v[5] = bf16_hi(q.z); v[6] = bf16_lo(q.w); v[7] = bf16_hi(q.w);
}
__device__ __forceinline__ void unpack16(uint4 q, float (&v)[4]) {
  v[0] = __uint_as_float(q.x); v[1] = __uint_as_float(q.y); v[2] = __uint_as_float(q.z); v[3] = __uint_as_float(q.w);
}
__device__ __forceinline__ const void* word_of(const void* at) {
  return reinterpret_cast<const void*>(reinterpret_cast<uintptr_t>(at) & ~(uintptr_t)3);
}

struct RingNumbers { float w, t_lse, s0, s1; };
// What the sums' warp says of a row: to the classes that are not named, for the gradient of those that are, and for the loss.  Without
// sums of the row inv is 1, or 0 for a row that is left for the end.
struct RingScale { float ref, other_ref, factor, ws, A, inv, scale_p; };
// Of a row's entries: the teacher's exponentials and the named classes', each relative to its largest; with w the teacher's exponentials
// and a their exponents (base 2), sum w a and sum w (z - named.m) kDown
struct RingEntries { MaxSum teacher, named; float wa, wz; };

// FILL: the last CTA's slice ends inside an access of 16 bytes, with one, or all slices fill all accesses of their threads.
template <class T, int NV, int MODE, int FILL>
__global__ void __launch_bounds__(kRingAll, 2) distill_ring_kernel(const Distill p, int rows, int C) {
  constexpr int VEC = 16 / sizeof(T);
  constexpr int words = NV * kRingThreads * VEC / 32;
  extern __shared__ __align__(16) uint8_t dyn8[];
  __shared__ RingNumbers s_num[kEntrySlots];
  __shared__ RingScale s_scale[2];
  __shared__ RingEntries s_entries[2];
  __shared__ uint32_t s_seen[kSeenBits / 32];
  __shared__ float s_w[kRingWarps][kRingSlots + 2];
  __shared__ __align__(8) uint64_t bar_sums[2], bar_bits[2], bar_scale[2], bar_done[2], bar_clear[2];
  __shared__ int s_lost;                          // a wait gave up
  __shared__ int s_coarse;                        // gradient alone: rows of this CTA are left for the end
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int rank = (int)blockIdx.x % C, row0 = (int)blockIdx.x / C, step = (int)gridDim.x / C;
  uint4* ring = reinterpret_cast<uint4*>(dyn8);                                             // [slot][k][thread]
  uint32_t* bits = reinterpret_cast<uint32_t*>(ring + kRingSlots * NV * kRingThreads);      // [2][words]
  // [slot][class, teacher's logit, student's logit, with 64 bits the class's upper half][K]
  const int kp = (p.K + 3) & ~3, slot_words = kp * (p.i64 ? 4 : 3);
  uint32_t* entries = bits + 2 * words;
  // sums of every warp of the cluster, in two places that take turns
  MaxSum* s_sum = reinterpret_cast<MaxSum*>(entries + kEntrySlots * slot_words);
  const int place = C * kRingWarps;
  const float c2 = p.inv_tau * kLog2e;
  const int first = rank * p.slice, last = min(p.V, first + p.slice);
  auto bar = [](uint64_t& b) { return sm100::smem_u32(&b); };
  // parity of the n-th wait on one of two barriers that take turns
  auto wait = [&](uint64_t* two, int n) {
    const bool ok = sm100::mbar_wait(bar(two[n & 1]), (uint32_t)(n >> 1) & 1u, &s_lost, s_lost ? 1u : sm100::kSpinLimit);
    if (__all_sync(0xffffffffu, ok)) return true;              // one verdict a warp
    s_lost = 1;
    return false;
  };
  auto zrow = [&](int row) { return static_cast<const T*>(p.Z) + (int64_t)row * p.ldz; };

  for (int i = tid; i < 2 * words; i += kRingAll) bits[i] = 0;
  for (int i = tid; i < kSeenBits / 32; i += kRingAll) s_seen[i] = 0;
  if (tid == 0) {
    s_lost = s_coarse = 0;
    for (int i = 0; i < 2; ++i) {
      sm100::mbar_init(bar(bar_sums[i]), 1);
      sm100::mbar_init(bar(bar_bits[i]), 1);
      sm100::mbar_init(bar(bar_scale[i]), 1);
      sm100::mbar_init(bar(bar_clear[i]), 1);
      sm100::mbar_init(bar(bar_done[i]), kRingWarps);
    }
    sm100::mbar_fence_init();
  }
  dep_wait();
  __syncthreads();
  // Rows whose statistics are coarse are left out of the walk; of the cluster's rows a CTA does every C-th by itself at the end.  The
  // choice rests on memory that no one writes, so all CTAs make the same one.
  auto later = [&](int row) { return MODE == DIST_BACKWARD && coarse(p.stat_in[2 * (int64_t)row], p.stat_in[2 * (int64_t)row + 1]); };
  if (MODE == DIST_BACKWARD)
    for (int64_t row = row0 + (int64_t)(rank + tid * C) * step; row < rows; row += (int64_t)kRingAll * C * step)
      if (later((int)row)) s_coarse = 1;
  // no CTA sends to another before that one has begun
  sm100::cluster_arrive();
  sm100::cluster_wait();

  if (warp < kRingWarps) {
    // ---- classes ----
    const int mine = last - first - tid * VEC;    // of the slice from this thread's first on
    // its k-th access: whole (the ring has it), or at least begun
    auto whole = [&](int k) { return FILL == ROW_FULL || (FILL == ROW_WHOLE ? mine > k * kRingThreads * VEC : mine >= (k * kRingThreads + 1) * VEC); };
    auto begun = [&](int k) { return FILL == ROW_FULL || mine > k * kRingThreads * VEC; };
    const uint32_t ring_at = sm100::smem_u32(ring) + tid * 16;
    const uint32_t push_at = sm100::mapa_shared(sm100::smem_u32(&s_sum[rank * kRingWarps + warp]), lane < C ? lane : 0);
    const uint32_t push_bar = sm100::mapa_shared(bar(bar_sums[0]), lane < C ? lane : 0);
    auto fetch = [&](int row, int slot, bool live) {
      if (live) {
        const T* z = zrow(row) + first;
        const uint32_t to = ring_at + (uint32_t)slot * (NV * kRingThreads * 16);
#pragma unroll
        for (int k = 0; k < NV; ++k)
          if (whole(k)) ahead16(to + k * kRingThreads * 16, z + (uint32_t)((k * kRingThreads + tid) * VEC));
      }
    };
    // weights, four rows ahead: a row of weight 0 is not fetched
    auto fetch_weight = [&](int row, int it) {
      if (lane == 0 && row < rows && p.weight) ahead4(sm100::smem_u32(&s_w[warp][it % (kRingSlots + 2)]), p.weight + row);
    };
    auto counts = [&](int row, int it) { return row < rows && (!p.weight || s_w[warp][it % (kRingSlots + 2)] != 0.f); };
    for (int i = 0; i < 4; ++i) fetch_weight(row0 + i * step, i);
    ahead_commit();
    ahead_wait<0>();
    __syncwarp();
    bool live0 = counts(row0, 0), live1 = counts(row0 + step, 1);
    fetch(row0, 0, live0);
    ahead_commit();
    fetch(row0 + step, 1, live1);
    ahead_commit();
    int turn = 0, slot = 0;
    int it = 0, row = row0;
    for (; row < rows; row += step, ++it) {
      ahead_wait<1>();                            // this row's classes, the weight of the row after next
      __syncwarp();
      const bool live2 = counts(row + 2 * step, it + 2);
      fetch(row + 2 * step, slot == 0 ? 2 : slot - 1, live2);       // (the slot of the row before)
      fetch_weight(row + 4 * step, it + 4);
      ahead_commit();
      T* dz = MODE == DIST_LOSS ? nullptr : static_cast<T*>(p.dZ) + (int64_t)row * p.lddz + first;
      // A row begins when its entries are ready and ends when its factor is there, whether it needs them or not: so no warp is a
      // turn of a barrier ahead of another, and a place for sums has been read in every CTA before it is written again two such
      // rows on (that takes all sums of the row between, which are sent after the factor of the row before).
      if (!wait(bar_bits, it)) break;
      if (live0) {                                // the same in all warps of the cluster
        float e[NV][VEC];
        float top = kLow;
        const uint4* at = ring + slot * NV * kRingThreads + tid;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
          if (whole(k)) {
            unpack16(at[k * kRingThreads], e[k]);
          } else if (FILL == ROW_PART) {          // the row's last few, and past them
            load<VEC>(zrow(row) + first + (k * kRingThreads + tid) * VEC, mine - k * kRingThreads * VEC, -INFINITY, e[k]);
          } else {
#pragma unroll
            for (int v = 0; v < VEC; ++v) e[k][v] = -INFINITY;
          }
        }
        if (MODE != DIST_BACKWARD) {
          float part[2] = {kLow, kLow};
          // a byte (bf16) or half of one of the bit set to an access
          const uint32_t* set = bits + (it & 1) * words + tid * VEC / 32;
#pragma unroll
          for (int k = 0; k < NV; ++k) {
            const uint32_t named = (set[k * kRingThreads * VEC / 32] >> (tid * VEC % 32)) & ((1u << VEC) - 1u);
            if (named) {
#pragma unroll
              for (int v = 0; v < VEC; ++v)
                if ((named >> v) & 1u) e[k][v] = -INFINITY;
            }
#pragma unroll
            for (int v = 0; v < VEC; v += 2) {
              part[0] = fmaxf(part[0], e[k][v]);
              part[1] = fmaxf(part[1], e[k][v + 1]);
            }
          }
          top = fmaxf(part[0], part[1]);
          part[0] = part[1] = 0.f;
          const float less[2] = {-top, -top};
#pragma unroll
          for (int k = 0; k < NV; ++k) {
#pragma unroll
            for (int v = 0; v < VEC; v += 2) {
              float two[2] = {e[k][v], e[k][v + 1]};
              vadd<2>(two, less);
              vscale<2>(two, c2);
              e[k][v] = ex2(two[0]);
              e[k][v + 1] = ex2(two[1]);
              const float ex[2] = {e[k][v], e[k][v + 1]};
              vadd<2>(part, ex);
            }
          }
          const MaxSum s = merge_lanes({top, part[0] + part[1]}, c2);
          if (lane < C) send_pair(push_at + (uint32_t)(turn * place) * (uint32_t)sizeof(MaxSum), s, push_bar + (uint32_t)turn * 8u);
          turn ^= 1;
        }
        if (MODE != DIST_LOSS) {
          if (!wait(bar_scale, it)) break;
          const RingScale& sc = s_scale[it & 1];
          const float f = MODE == DIST_BACKWARD || sc.factor == 0.f ? sc.factor : sc.factor * ex2((top - sc.other_ref) * c2);
#pragma unroll
          for (int k = 0; k < NV; ++k) {
            if (!begun(k)) continue;
            if (MODE == DIST_BACKWARD) {
#pragma unroll
              for (int v = 0; v < VEC; ++v) e[k][v] = f == 0.f ? 0.f : f * ex2(fmaf(e[k][v], p.inv_tau, -sc.other_ref) * kLog2e);
            } else {
              vscale<VEC>(e[k], f);
            }
            if (MODE != DIST_BACKWARD || sc.inv != 0.f)
              store<VEC>(dz + (uint32_t)((k * kRingThreads + tid) * VEC), FILL == ROW_PART ? mine - k * kRingThreads * VEC : VEC, e[k]);
          }
        }
      } else if (MODE != DIST_LOSS) {
        const float zero[VEC] = {};
#pragma unroll
        for (int k = 0; k < NV; ++k)
          if (begun(k)) store<VEC>(dz + (uint32_t)((k * kRingThreads + tid) * VEC), FILL == ROW_PART ? mine - k * kRingThreads * VEC : VEC, zero);
      }
      if (!wait(bar_scale, it)) break;
      __syncwarp();                               // lane 0 speaks for the stores of all lanes
      if (lane == 0) sm100::mbar_arrive(bar(bar_done[it & 1]));
      live0 = live1;
      live1 = live2;
      if (++slot == kRingSlots) slot = 0;
    }
    ahead_wait<0>();
    // given up: no row that is left is taken for a gradient
    if (MODE != DIST_LOSS)
      for (; row < rows; row += step)
        for (int c = first + tid; c < last; c += kRingThreads) put(static_cast<T*>(p.dZ) + (int64_t)row * p.lddz + c, NAN);
  } else {
    const bool t16 = p.t_bf16 != 0;
    auto slot_of = [](int it) { return it % kEntrySlots; };
    auto cls = [&](int it) { return reinterpret_cast<int*>(entries + slot_of(it) * slot_words); };
    auto weight = [&](int it) { return p.weight ? s_num[slot_of(it)].w : 1.f; };
    auto t_lse_of = [&](int it) { return p.t_lse ? s_num[slot_of(it)].t_lse : 0.f; };
    // A 16-bit element by itself cannot be copied ahead: the aligned word that holds it is; which half of it, from the element's number
    const uint32_t t_odd = (uint32_t)(reinterpret_cast<uintptr_t>(p.T) >> 1), z_odd = (uint32_t)(reinterpret_cast<uintptr_t>(p.Z) >> 1);
    auto half_of = [](uint32_t w, uint32_t n) { return (n & 1u) ? bf16_hi(w) : bf16_lo(w); };
    auto t_of = [&](int it, int row, int k) {
      const uint32_t w = entries[slot_of(it) * slot_words + kp + k];
      return t16 ? half_of(w, t_odd + (uint32_t)row * (uint32_t)p.K + (uint32_t)k) : __uint_as_float(w);
    };
    auto z_of = [&](int it, int row, int k, int c) {
      const uint32_t w = entries[slot_of(it) * slot_words + 2 * kp + k];
      return sizeof(T) == 2 ? half_of(w, z_odd + (uint32_t)row * (uint32_t)p.ldz + (uint32_t)c) : __uint_as_float(w);
    };
    auto teacher2 = [&](float t, float t_lse, float tm) { return p.t_lse ? fmaf(t, p.inv_tau, -t_lse) * kLog2e : (t - tm) * c2; };
    auto fetch_entries = [&](int row, int it) {
      if (row >= rows) return;
      RingNumbers& n = s_num[slot_of(it)];
      const uint32_t to = sm100::smem_u32(entries + slot_of(it) * slot_words);
      if (lane == 0 && p.weight) ahead4(sm100::smem_u32(&n.w), p.weight + row);
      if (lane == 1 && p.t_lse) ahead4(sm100::smem_u32(&n.t_lse), p.t_lse + row);
      if (MODE == DIST_BACKWARD && lane >= 2 && lane < 4) ahead4(sm100::smem_u32(&n.s0) + (lane - 2) * 4, p.stat_in + 2 * (int64_t)row + (lane - 2));
      const int64_t at = (int64_t)row * p.K;
      const int32_t* i = static_cast<const int32_t*>(p.I) + (p.i64 ? 2 * at : at);
      const char* t = static_cast<const char*>(p.T) + (t16 ? 2 * at : 4 * at);
#pragma unroll 2
      for (int k = lane; k < p.K; k += 32) {
        ahead4(to + k * 4, i + (uint32_t)(p.i64 ? 2 * k : k));
        if (p.i64) ahead4(to + (3 * kp + k) * 4, i + (uint32_t)(2 * k + 1));
        ahead4(to + (kp + k) * 4, word_of(t + (uint32_t)(t16 ? 2 * k : 4 * k)));
      }
    };
    // classes as they are used, and the student's logits on their way (the backward pass needs those of its slice alone: dZ may be
    // Z, and other CTAs write over theirs)
    auto fetch_logits = [&](int row, int it) {
      if (row >= rows) return;
      const bool live = weight(it) != 0.f;
      int* c = cls(it);
      const uint32_t to = sm100::smem_u32(c + 2 * kp);
      const T* z = zrow(row);
#pragma unroll 2
      for (int k = lane; k < p.K; k += 32) {
        int i = c[k];
        if (i >= p.V || (p.i64 && c[3 * kp + k] != 0)) i = -1;
        if (i < 0) i = -1;
        c[k] = i;
        const bool wanted = MODE == DIST_BACKWARD ? i >= first && i < last : i >= 0;
        if (live && wanted) ahead4(to + k * 4, word_of(z + (uint32_t)i));
      }
    };
    // a row whose stores are done: the named classes' gradient over them, its bits out
    auto finish = [&](int row, int it) {
      if (weight(it) == 0.f) return;
      const RingScale sc = s_scale[it & 1];
      T* dz = MODE == DIST_LOSS ? nullptr : static_cast<T*>(p.dZ) + (int64_t)row * p.lddz;
      const int* c = cls(it);
      const uint32_t* values = entries + slot_of(it) * slot_words + kp;      // as prepare left them
      for (int k = lane; k < p.K; k += 32) {
        const int i = c[k];
        if (i < first || i >= last) continue;
        bits[(it & 1) * words + ((i - first) >> 5)] = 0;
        if (MODE == DIST_BOTH || (MODE == DIST_BACKWARD && sc.inv != 0.f)) {
          const float z = __uint_as_float(values[kp + k]), pk = ex2(__uint_as_float(values[k])) * sc.scale_p;
          const float q = ex2(MODE == DIST_BACKWARD ? fmaf(z, p.inv_tau, -sc.ref) * kLog2e : (z - sc.ref) * c2) * sc.inv;
          put(dz + i, sc.ws == 0.f ? 0.f : sc.ws * (sc.A * q - pk));
        }
      }
    };
    if (warp == kRingWarps) {
      // ---- entries of the next row ----
      // repeated classes out, bit set, sums of the teacher's and of the named classes' exponentials
      auto prepare = [&](int row, int it) {
        MaxSum t = {kLow, 0.f}, n = {kLow, 0.f};
        float wa = 0.f, wz = 0.f;
        if (weight(it) != 0.f) {
          const float t_lse = t_lse_of(it);
          int* c = cls(it);
          // Is a class there twice?  A bit for each, by its low bits, says no for most rows (K = 64: 9 of 10): comparing all with all
          // took 3500 of 4800 clocks.
          bool seen = false;
          for (int g = 0; g < p.K; g += 64) {          // two entries of a lane beside each other
            const int k0 = g + lane, k1 = k0 + 32;
            const int i0 = k0 < p.K ? c[k0] : -1, i1 = k1 < p.K ? c[k1] : -1;
            const float t0 = i0 >= 0 ? t_of(it, row, k0) : kLow, t1 = i1 >= 0 ? t_of(it, row, k1) : kLow;
            t.m = fmaxf(t.m, fmaxf(t0, t1));
            if (MODE != DIST_BACKWARD) {
              const float z0 = i0 >= 0 ? z_of(it, row, k0, i0) : kLow, z1 = i1 >= 0 ? z_of(it, row, k1, i1) : kLow;
              n.m = fmaxf(n.m, fmaxf(z0, z1));
            }
            uint32_t was0 = 0, was1 = 0;
            if (i0 >= 0) was0 = atomicOr(&s_seen[(i0 & (kSeenBits - 1)) >> 5], 1u << (i0 & 31));
            if (i1 >= 0) was1 = atomicOr(&s_seen[(i1 & (kSeenBits - 1)) >> 5], 1u << (i1 & 31));
            uint32_t* set = bits + (it & 1) * words;
            if (i0 >= first && i0 < last) atomicOr(&set[(i0 - first) >> 5], 1u << ((i0 - first) & 31));
            if (i1 >= first && i1 < last) atomicOr(&set[(i1 - first) >> 5], 1u << ((i1 - first) & 31));
            seen |= ((was0 >> (i0 & 31)) & 1u) || ((was1 >> (i1 & 31)) & 1u);
          }
          __syncwarp();
          for (int k = lane; k < p.K; k += 32)
            if (c[k] >= 0) s_seen[(c[k] & (kSeenBits - 1)) >> 5] = 0;
          if (__any_sync(0xffffffffu, seen)) {
            bool out = false;
            for (int g = 0; g < p.K; g += 32) {
              // a lane compares with the entries before its own, four at a time (a repeated class's first is not taken out)
              const int k = g + lane, i = k < p.K ? c[k] : -1;
              bool twice = false;
              const int4* before = reinterpret_cast<const int4*>(c);
#pragma unroll 4
              for (int j = 0; j < g; j += 4) {
                const int4 q = before[j >> 2];
                twice |= q.x == i || q.y == i || q.z == i || q.w == i;
              }
#pragma unroll
              for (int j = 0; j < 32; j += 4) {
                if (g + j < p.K) {
                  const int4 q = before[(g + j) >> 2];
                  twice |= (j < lane && q.x == i) || (j + 1 < lane && q.y == i) || (j + 2 < lane && q.z == i) || (j + 3 < lane && q.w == i);
                }
              }
              __syncwarp();
              if (i >= 0 && twice) {
                c[k] = -2;
                out = true;
              }
            }
            // the teacher's largest of what counts: an ignored logit far ahead would leave no exponential of the others
            if (__any_sync(0xffffffffu, out)) {
              t.m = kLow;
              for (int k = lane; k < p.K; k += 32)
                if (c[k] >= 0) t.m = fmaxf(t.m, t_of(it, row, k));
            }
          }
          t.m = p.t_lse ? kLow : lanes_max(t.m);
          n.m = lanes_max(n.m);
          uint32_t* values = entries + slot_of(it) * slot_words + kp;
          for (int g = 0; g < p.K; g += 64) {
            const int k0 = g + lane, k1 = k0 + 32;
            const int i0 = k0 < p.K ? c[k0] : -1, i1 = k1 < p.K ? c[k1] : -1;
            const float a0 = i0 >= 0 ? teacher2(t_of(it, row, k0), t_lse, t.m) : -INFINITY, a1 = i1 >= 0 ? teacher2(t_of(it, row, k1), t_lse, t.m) : -INFINITY;
            const float z0 = i0 >= 0 ? z_of(it, row, k0, i0) : 0.f, z1 = i1 >= 0 ? z_of(it, row, k1, i1) : 0.f;
            const float w0 = ex2(a0), w1 = ex2(a1);
            t.l += w0 + w1;
            if (MODE != DIST_BACKWARD) {
              const float d0 = z0 - n.m, d1 = z1 - n.m;
              n.l += (i0 >= 0 ? ex2(d0 * c2) : 0.f) + (i1 >= 0 ? ex2(d1 * c2) : 0.f);
              if (w0 > 0.f) { wa = fmaf(w0, a0, wa); wz = fmaf(w0 * kDown, d0, wz); }
              if (w1 > 0.f) { wa = fmaf(w1, a1, wa); wz = fmaf(w1 * kDown, d1, wz); }
            }
            // the loss and the gradient take them from here
            if (i0 >= 0) { values[k0] = __float_as_uint(a0); values[kp + k0] = __float_as_uint(z0); }
            if (i1 >= 0) { values[k1] = __float_as_uint(a1); values[kp + k1] = __float_as_uint(z1); }
          }
#pragma unroll
          for (int o = 16; o > 0; o >>= 1) {
            t.l += __shfl_xor_sync(0xffffffffu, t.l, o);
            if (MODE != DIST_BACKWARD) {
              n.l += __shfl_xor_sync(0xffffffffu, n.l, o);
              wa += __shfl_xor_sync(0xffffffffu, wa, o);
              wz += __shfl_xor_sync(0xffffffffu, wz, o);
            }
          }
        }
        if (lane == 0) s_entries[it & 1] = {t, n, wa, wz};
        __syncwarp();
        if (lane == 0) sm100::mbar_arrive(bar(bar_bits[it & 1]));
      };
      asm volatile("bar.sync 1, 64;" ::: "memory");              // the first rows have landed
      prepare(row0, 0);
      int it = 0;
      for (int row = row0; row + step < rows; row += step, ++it) {
        if (it > 0 && !wait(bar_clear, it - 1)) break;
        prepare(row + step, it + 1);
      }
    } else {
      // ---- sums ----
      for (int i = 0; i <= 2 * kAheadRows; ++i) fetch_entries(row0 + i * step, i);
      ahead_commit();
      ahead_wait<0>();
      __syncwarp();
      for (int i = 0; i <= kAheadRows; ++i) fetch_logits(row0 + i * step, i);
      ahead_commit();
      ahead_wait<0>();
      asm volatile("bar.sync 1, 64;" ::: "memory");
      int sums = 0, it = 0, row = row0;            // rows that count; rows
      bool lost = false;
      for (; row < rows; row += step, ++it) {
        // the row before is through
        if (it > 0) {
          lost = !wait(bar_done, it - 1);
          if (lost) break;
          finish(row - step, it - 1);
          ahead_wait<kAheadRows - 1>();
          __syncwarp();
          if (lane == 0) sm100::mbar_arrive(bar(bar_clear[(it - 1) & 1]));
        }
        lost = !wait(bar_bits, it);
        if (lost) break;
        const float w = weight(it);
        if (w == 0.f) {
          if (lane == 0) {
            sm100::mbar_arrive(bar(bar_scale[it & 1]));
            if (MODE != DIST_BACKWARD && rank == 0) {
              p.loss[row] = 0.f;
              if (p.stat) { p.stat[2 * (int64_t)row] = 0.f; p.stat[2 * (int64_t)row + 1] = 0.f; }
            }
          }
        } else {
          const RingEntries en = s_entries[it & 1];
          const MaxSum n = en.named;
          const float ts = en.teacher.l;
          const float scale_p = p.t_lse ? 1.f : (ts > 0.f ? 1.f / ts : (ts == 0.f ? 0.f : ts));     // a NaN goes on
          const float whole = ts * scale_p;
          float pt = 0.f;
          if (p.t_lse) pt = 1.f - whole < 0.f ? 0.f : 1.f - whole;
          const float A = whole + pt;
          float ref, inv, qt, Q = 1.f;
          bool empty;
          MaxSum all = {kLow, 0.f}, others = {kLow, 0.f};
          if (MODE != DIST_BACKWARD) {
            const int count = place;
            const MaxSum* sent = s_sum + (sums & 1) * place;
            if (lane == 0) sm100::mbar_expect_tx(bar(bar_sums[sums & 1]), (uint32_t)(count * (int)sizeof(MaxSum)));
            __syncwarp();
            lost = !wait(bar_sums, sums);
            if (lost) break;
            ++sums;
            for (int i = lane; i < count; i += 32) others.m = fmaxf(others.m, sent[i].m);
            others.m = lanes_max(others.m);
            for (int i = lane; i < count; i += 32) others.l += sent[i].l * ex2((sent[i].m - others.m) * c2);
            others.l = lanes_sum(others.l);
            all = merge(others, n, c2);
            empty = all.l == 0.f;
            ref = all.m;
            inv = __fdividef(1.f, all.l);
            qt = others.l * ex2((others.m - all.m) * c2) * inv;
            Q = n.l * ex2((n.m - all.m) * c2) * inv;
          } else {
            ref = s_num[slot_of(it)].s0;
            inv = coarse(ref, s_num[slot_of(it)].s1) ? 0.f : 1.f;
            empty = false;
            qt = ex2((s_num[slot_of(it)].s1 - ref) * kLog2e);
          }
          const float ws = empty ? 0.f : w * p.inv_tau;
          // (A q_t - p_t) q_j / q_t of the others: the first factor, and q_j / q_t relative to the others' largest or their normaliser
          const float other = ws == 0.f ? 0.f : ws * excess_rest(A, pt, qt, whole, Q);
          const float other_ref = MODE == DIST_BACKWARD ? s_num[slot_of(it)].s1 : others.m;
          const bool none = MODE != DIST_BACKWARD && others.l == 0.f;
          if (lane == 0) {
            s_scale[it & 1] = {ref, other_ref, none ? 0.f : MODE == DIST_BACKWARD ? other : __fdividef(other, others.l), ws, A, inv, scale_p};
            sm100::mbar_arrive(bar(bar_scale[it & 1]));
            if (MODE != DIST_BACKWARD && rank == 0) {
              // sum p (log p - log q), p = w scale_p: from the entries' sums, relative to the named classes' largest logit
              float kl = 0.f;
              if (ts != 0.f)
                kl = scale_p * (kDown * fmaf(ts, log2f(scale_p), en.wa) - fmaf(c2, fmaf((n.m - all.m) * kDown, ts, en.wz), -kDown * (ts * log2f(all.l))));
              if (pt > 0.f) kl += pt * log_rest(pt, others, all, c2, whole, Q);
              if (whole != whole) kl = whole;
              p.loss[row] = empty ? 0.f : w * kl * kUp;
              if (p.stat) {
                p.stat[2 * (int64_t)row] = empty ? -INFINITY : fmaf(all.m, p.inv_tau, logf(all.l));
                p.stat[2 * (int64_t)row + 1] = others.l == 0.f ? -INFINITY : fmaf(others.m, p.inv_tau, logf(others.l));
              }
            }
          }
        }
        fetch_logits(row + (1 + kAheadRows) * step, it + 1 + kAheadRows);
        fetch_entries(row + (1 + 2 * kAheadRows) * step, it + 1 + 2 * kAheadRows);
        ahead_commit();
      }
      lost = lost || !wait(bar_done, it - 1);
      if (!lost) finish(row - step, it - 1);
      ahead_wait<0>();
      // given up: no barrier is touched any more, and the rows that are left say so, with the one before, whose named classes'
      // gradient may be missing
      if (lost)
        for (int r = (it > 0 ? row - step : row) + lane * step; r < rows; r += 32 * step) {
          if (MODE != DIST_BACKWARD && rank == 0) p.loss[r] = NAN;
          if (MODE != DIST_LOSS && first < last) put(static_cast<T*>(p.dZ) + (int64_t)r * p.lddz + first, NAN);
        }
    }
  }
  if (MODE == DIST_BACKWARD) {
    __syncthreads();
    if (s_coarse)
      for (int64_t row = row0 + (int64_t)rank * step; row < rows; row += (int64_t)C * step)
        if (later((int)row) && !(p.weight && p.weight[row] == 0.f))
          coarse_row<T, VEC, true>(p, row, reinterpret_cast<uint32_t*>(dyn8), reinterpret_cast<float*>(s_seen));
  }
  dep_trigger();
  // no CTA leaves while its sums may still be written by another
  __syncwarp();
  sm100::cluster_arrive();
  sm100::cluster_wait();
}

// Resident clusters of a kernel, found once for each device, cluster size and size of shared memory
struct ClusterCache {
  std::mutex mu;
  struct { int dev, C, n; size_t smem; } known[16] = {};
  int count = 0;
};

template <class T, int NV, int MODE, int FILL>
cudaError_t launch_clusters(const Distill& p, int C, int64_t rows, cudaStream_t s) {
  static ClusterCache cache;
  constexpr int threads = kRingAll;
  const size_t smem = (size_t)kRingSlots * NV * kRingThreads * 16 + 2 * (NV * kRingThreads * (16 / sizeof(T)) / 8) +
                      (size_t)kEntrySlots * ((p.K + 3) & ~3) * (p.i64 ? 16 : 12) + 2 * (size_t)C * kRingWarps * sizeof(MaxSum);
  auto kernel = distill_ring_kernel<T, NV, MODE, FILL>;
  int dev = 0, n = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  {
    std::lock_guard<std::mutex> lock(cache.mu);
    const int have = cache.count < 16 ? cache.count : 16;
    for (int i = 0; i < have && !n; ++i)
      if (cache.known[i].dev == dev && cache.known[i].C == C && cache.known[i].smem == smem) n = cache.known[i].n;
    if (!n) {
      // as much as any launch asks for
      e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 200 * 1024);
      if (e == cudaSuccess) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
      if (e != cudaSuccess) return e;
      cudaLaunchConfig_t cfg;
      memset(&cfg, 0, sizeof(cfg));
      cfg.gridDim = dim3((unsigned)(C * 1024)); cfg.blockDim = dim3(threads); cfg.dynamicSmemBytes = smem;
      cudaLaunchAttribute at[1];
      at[0].id = cudaLaunchAttributeClusterDimension;
      at[0].val.clusterDim.x = C; at[0].val.clusterDim.y = 1; at[0].val.clusterDim.z = 1;
      cfg.attrs = at; cfg.numAttrs = 1;
      if (cudaOccupancyMaxActiveClusters(&n, kernel, &cfg) != cudaSuccess || n < 1) { cudaGetLastError(); n = 1; }
      cache.known[cache.count % 16] = {dev, C, n, smem};
      if (++cache.count >= 32) cache.count = 16;
    }
  }
  if (n > rows) n = (int)rows;
  return launch_dep_cluster(C, kernel, dim3((unsigned)(n * C)), threads, smem, s, p, (int)rows, C);
}
template <class T, int NV, int MODE>
cudaError_t launch_fill(const Distill& p, int C, int64_t rows, cudaStream_t s) {
  constexpr int VEC = 16 / sizeof(T);
  if (p.slice == NV * kRingThreads * VEC && p.V == C * p.slice) return launch_clusters<T, NV, MODE, ROW_FULL>(p, C, rows, s);
  if (p.V % VEC == 0) return launch_clusters<T, NV, MODE, ROW_WHOLE>(p, C, rows, s);
  return launch_clusters<T, NV, MODE, ROW_PART>(p, C, rows, s);
}

// Rows the ring takes: fewer than 2^28 of up to 16 slices; *C CTAs a row, *nv accesses a thread
bool ring_shape(int V, int K, int vec, int* C, int* nv) {
  if (K > kRingMaxK) return false;
  const int cap = kRingThreads * 8 * vec;
  int c = 1;
  while (c <= kRingMaxCtas && c * cap < V) c *= 2;
  if (c > kRingMaxCtas) return false;
  *C = c;
  const int per = (V + c * kRingThreads * vec - 1) / (c * kRingThreads * vec);
  *nv = per <= 2 ? 2 : per <= 4 ? 4 : per <= 6 ? 6 : 8;
  return true;
}

}  // namespace

template <class T, int VEC, int MODE>
cudaError_t launch_ring(const Distill& p0, int64_t rows, cudaStream_t s, bool* taken) {
  int C = 0, nv = 0;
  *taken = ring_shape(p0.V, p0.K, VEC, &C, &nv);
  if (!*taken) return cudaSuccess;
  Distill p = p0;
  p.slice = ((p.V + C - 1) / C + 31) / 32 * 32;
  if (nv == 2) return launch_fill<T, 2, MODE>(p, C, rows, s);
  if (nv == 4) return launch_fill<T, 4, MODE>(p, C, rows, s);
  if (nv == 6) return launch_fill<T, 6, MODE>(p, C, rows, s);
  return launch_fill<T, 8, MODE>(p, C, rows, s);
}

template cudaError_t launch_ring<float, 4, DIST_LOSS>(const Distill&, int64_t, cudaStream_t, bool*);
template cudaError_t launch_ring<float, 4, DIST_BOTH>(const Distill&, int64_t, cudaStream_t, bool*);
template cudaError_t launch_ring<float, 4, DIST_BACKWARD>(const Distill&, int64_t, cudaStream_t, bool*);
template cudaError_t launch_ring<__nv_bfloat16, 8, DIST_LOSS>(const Distill&, int64_t, cudaStream_t, bool*);
template cudaError_t launch_ring<__nv_bfloat16, 8, DIST_BOTH>(const Distill&, int64_t, cudaStream_t, bool*);
template cudaError_t launch_ring<__nv_bfloat16, 8, DIST_BACKWARD>(const Distill&, int64_t, cudaStream_t, bool*);

}  // namespace distill
}  // namespace fw
