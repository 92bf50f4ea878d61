// Loss and gradient of long rows in one pass over the logits (see fw_logprob.cu).
#include <cstring>
#include <mutex>

#include "fw_logprob.cuh"
#include "fw_sm100.cuh"

namespace fw {
namespace logprob {
namespace {

// A row stays in the shared memory of a CTA, or of a cluster where it is long, between its sums and its gradient.  (From L2 it does not come
// back: with the rows of 296 CTAs, 76 MB, 400 MB were read for 235.)  A thread copies ahead its own groups of 16 bytes and reads back
// those alone, so that the exchange of the sums is all that threads wait for; where its gradient has used up a group it asks for the
// next row's, and the next sums follow the copies as they arrive.  So the memory has work while the exponentials are formed, twice for
// each logit, which takes two thirds of its time.
constexpr int kTurns = 14;               // groups of a thread in shared memory
constexpr int kMaxCtas = 8;

__device__ __forceinline__ void send_pair(uint32_t addr, MaxSum v) {
  asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(addr), "f"(v.m), "f"(v.l) : "memory");
}
// all copies but those of the last n groups are there
__device__ __forceinline__ void wait_but(int n) {
  switch (n) {
    case 0: ahead_wait<0>(); break;
    case 1: ahead_wait<1>(); break;
    case 2: ahead_wait<2>(); break;
    default: ahead_wait<3>(); break;
  }
}

// TH threads a CTA, 1024 a SM, the last warp for the rows' numbers; KEPT groups of a thread stay in registers beside those in shared
// memory; SOLO: no cluster.
template <class T, int TH, int KEPT, bool SOLO>
__global__ void __launch_bounds__(TH, 1024 / TH) logprob_resident_kernel(const Logprob p, int C, int slice, int turns) {
  constexpr int VEC = Group<T>::VEC, nw = TH / 32 - 1, width = TH - 32, kChunk = 4;
  extern __shared__ __align__(16) uint8_t room[];            // [turn][thread]
  __shared__ MaxSum red[2 * 32];
  __shared__ Scale scale[2];
  __shared__ __align__(8) MaxSum ctas[2][kMaxCtas];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int rank = SOLO ? 0 : (int)blockIdx.x % C, unit = SOLO ? blockIdx.x : blockIdx.x / C, units = SOLO ? gridDim.x : gridDim.x / C;
  const float c2 = p.inv_tau * kLog2e;
  dep_wait();
  if (!SOLO) {                                               // no CTA writes to another before that one has begun
    sm100::cluster_arrive();
    sm100::cluster_wait();
  }
  if (warp == nw) {
    const uint32_t push = SOLO ? 0 : sm100::mapa_shared(sm100::smem_u32(&ctas[0][rank]), lane < C ? lane : 0);
    // the sums of the cluster's CTAs.  Their places are written again two rows on: every thread of the cluster has come to the
    // exchange between, after this one has read them
    numbers<T, LP_BOTH>(p, unit, units, TH, nw, red, scale, rank == 0, [&](MaxSum s, int n) {
      if (SOLO) return s;
      if (lane < C) send_pair(push + (n & 1) * (uint32_t)sizeof(ctas[0]), s);
      __syncwarp();
      sm100::cluster_arrive();
      sm100::cluster_wait();
      return merge_lanes(lane < C ? ctas[n & 1][lane] : MaxSum{kLow, 0.f}, c2);
    });
  } else {
    const uint32_t mine = (uint32_t)__cvta_generic_to_shared(room) + tid * 16;
    const uint4* from = reinterpret_cast<const uint4*>(room) + tid;
    const int g0 = rank * slice, held = min(turns, kTurns), chunks = (held + kChunk - 1) / kChunk;
    uint4 kept[KEPT > 0 ? KEPT : 1];
    // the k-th group, of which n are this CTA's
    auto fetch = [&](const Place<T>& z, int n, int k) {
      const int c = k * width + tid;
      if (c < n) ahead16(mine + k * (width * 16), z.at(g0 + c));
    };
    auto fetch_kept = [&](const Place<T>& z, int n) {
#pragma unroll
      for (int j = 0; j < KEPT; ++j)
        if ((kTurns + j) * width + tid < n) kept[j] = *z.at(g0 + (kTurns + j) * width + tid);
    };
    int64_t row = row_at(0, unit, units);
    int next = id_of<LP_BOTH>(p, row), m = 0;
    {
      const Place<T> z(p.Z, next >= 0 ? row : 0, p.ldz, p.V, 0);
      const int n = next >= 0 ? min(slice, z.groups - g0) : 0;
      fetch_kept(z, n);
      for (int i = 0; i < chunks; ++i) {
#pragma unroll
        for (int u = 0; u < kChunk; ++u)
          if (i * kChunk + u < held) fetch(z, n, i * kChunk + u);
        ahead_commit();
      }
    }
    for (int it = 0; (int64_t)it * units < p.rows; ++it) {
      const int id = next;
      const int64_t later = row_at(it + 1, unit, units);
      next = id_of<LP_BOTH>(p, later);
      const Place<T> z(p.Z, row, p.ldz, p.V, id);
      const int n = min(slice, z.groups - g0);
      Scale sc = {0.f, 0.f, 0.f, 1};
      if (id >= 0) {
        MaxSum s = {kLow, 0.f};
        auto get = [&](int k) {                              // for the sums
          const int c = k * width + tid;
          uint4 q = make_uint4(Group<T>::kNone, Group<T>::kNone, Group<T>::kNone, Group<T>::kNone);
          if (c < n) q = from[k * width];
          return z.special(g0 + c) ? z.others(q, g0 + c, id) : q;
        };
        int k = 0;
        for (int i = 0; i + 1 < chunks; ++i, k += kChunk) {
          wait_but(chunks - 1 - i);
          uint4 raw[kChunk];
          bool any = false;
#pragma unroll
          for (int u = 0; u < kChunk; ++u) {
            const int c = (k + u) * width + tid;             // (only a cluster's last CTA may have fewer groups)
            raw[u] = make_uint4(Group<T>::kNone, Group<T>::kNone, Group<T>::kNone, Group<T>::kNone);
            if (SOLO || c < n) raw[u] = from[(k + u) * width];
            any |= z.special(g0 + c);
          }
          if (any) {
#pragma unroll
            for (int u = 0; u < kChunk; ++u) raw[u] = get(k + u);
          }
          s = add_groups<T, kChunk>(s, raw, c2);
        }
        wait_but(0);
        for (; k < held; ++k) {
          const uint4 raw[1] = {get(k)};
          s = add_groups<T, 1>(s, raw, c2);
        }
        if (KEPT > 0) {
          uint4 raw[KEPT > 0 ? KEPT : 1];
#pragma unroll
          for (int j = 0; j < KEPT; ++j) {
            const int c = (kTurns + j) * width + tid;
            raw[j] = make_uint4(Group<T>::kNone, Group<T>::kNone, Group<T>::kNone, Group<T>::kNone);
            if (c < n) raw[j] = z.special(g0 + c) ? z.others(kept[j], g0 + c, id) : kept[j];
          }
          s = add_groups<T, (KEPT > 0 ? KEPT : 1)>(s, raw, c2);
        }
        s = merge_lanes(s, c2);
        if (lane == 0) red[(m & 1) * 32 + warp] = s;
        tell<BAR_SUMS>(m, TH);
        if (!SOLO) sm100::cluster_arrive();
        meet<BAR_SCALE>(m, TH);
        if (!SOLO) sm100::cluster_wait();
        sc = scale[m & 1];
        ++m;
      }
      if (row < p.rows) {
        T* out = static_cast<T*>(p.dZ) + row * p.lddz;
        uint4* d = reinterpret_cast<uint4*>(reinterpret_cast<uintptr_t>(out) & ~(uintptr_t)15);
        const Place<T> zl(p.Z, next >= 0 ? later : 0, p.ldz, p.V, 0);
        const int nl = next >= 0 ? min(slice, zl.groups - g0) : 0;
        // this thread's turns of the row and of the next one, and of the groups that go one by one
        const int kn = (n - tid + width - 1) / width, kl = nl > 0 ? (nl - tid + width - 1) / width : 0;
        const int ka = tid == 0 && rank == 0 && z.edge0 == 0 ? 0 : -1;
        const int e1 = z.edge1 - g0, kb = z.edge1 >= 0 && e1 >= 0 && e1 < n && e1 % width == tid ? e1 / width : -1;
        if (!sc.zero && (ka >= 0 || kb >= 0)) {
          if (ka >= 0) put_singly<T>(z, g0 + tid, from[0], sc, c2, out);
          if (kb >= 0 && kb < held && kb != ka) put_singly<T>(z, z.edge1, from[kb * width], sc, c2, out);
          if (KEPT > 0) {
#pragma unroll
            for (int j = 0; j < KEPT; ++j)
              if (kb == kTurns + j) put_singly<T>(z, z.edge1, kept[j], sc, c2, out);
          }
        }
        d += g0 + tid;
        if (!sc.zero) {
          auto put_group = [&](int k, uint4 raw) {
            float v[VEC];
            slopes<T, VEC>(raw, sc, c2, v);
            if (k < kn && k != ka && k != kb) __stcs(d + k * width, Group<T>::close(v));
          };
          int k = 0;
          for (int i = 0; i < chunks; ++i) {
            for (const int end = min(held, k + kChunk); k < end; k += 2) {
              const uint4 raw[2] = {from[k * width], from[(k + 1 < held ? k + 1 : k) * width]};
              put_group(k, raw[0]);
              if (k + 1 < end) put_group(k + 1, raw[1]);
              if (k < kl) ahead16(mine + k * (width * 16), zl.at(g0 + k * width + tid));
              if (k + 1 < end && k + 1 < kl) ahead16(mine + (k + 1) * (width * 16), zl.at(g0 + (k + 1) * width + tid));
            }
            ahead_commit();
          }
          if (KEPT > 0) {
#pragma unroll
            for (int j = 0; j < KEPT; ++j) put_group(kTurns + j, kept[j]);
          }
          if (z.own >= g0 && z.own - g0 < n && (z.own - g0) % width == tid) put(out + id, sc.own);      // over what this thread has put there
        } else {
          int k = 0;
          for (int i = 0; i < chunks; ++i) {
            for (const int end = min(held, k + kChunk); k < end; ++k) {
              if (k < kn && k != ka && k != kb) d[k * width] = make_uint4(0, 0, 0, 0);
              if (k < kl) ahead16(mine + k * (width * 16), zl.at(g0 + k * width + tid));
            }
            ahead_commit();
          }
          for (k = held; k < kn; ++k)
            if (k != kb) d[k * width] = make_uint4(0, 0, 0, 0);
          if (ka >= 0) put_singly<T>(z, g0 + tid, make_uint4(0, 0, 0, 0), sc, c2, out);
          if (kb >= 0 && kb != ka) put_singly<T>(z, z.edge1, make_uint4(0, 0, 0, 0), sc, c2, out);
        }
        if (KEPT > 0) {
          fetch_kept(zl, nl);
        }
      }
      row = later;
    }
    ahead_wait<0>();
  }
  dep_trigger();
}

// Resident clusters of a kernel, found once for each device, cluster size and size of shared memory
struct ClusterCache {
  std::mutex mu;
  struct { int dev, C, n; size_t smem; } known[16] = {};
  int count = 0;
};

template <class T, int TH, int KEPT, bool SOLO>
cudaError_t launch_clusters(const Logprob& p, int C, int slice, int turns, cudaStream_t s) {
  static ClusterCache cache;
  const size_t smem = (size_t)(turns < kTurns ? turns : kTurns) * (TH - 32) * 16;
  auto kernel = logprob_resident_kernel<T, TH, KEPT, SOLO>;
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
      e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kTurns * (TH - 32) * 16);
      if (e != cudaSuccess) return e;
      if (SOLO) {
        e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, kernel, TH, smem);
        if (e != cudaSuccess) return e;
        n *= sm_count();
      } else {
        cudaLaunchConfig_t cfg;
        memset(&cfg, 0, sizeof(cfg));
        cfg.gridDim = dim3((unsigned)(C * 1024)); cfg.blockDim = dim3(TH); cfg.dynamicSmemBytes = smem;
        cudaLaunchAttribute at[1];
        at[0].id = cudaLaunchAttributeClusterDimension;
        at[0].val.clusterDim.x = C; at[0].val.clusterDim.y = 1; at[0].val.clusterDim.z = 1;
        cfg.attrs = at; cfg.numAttrs = 1;
        if (cudaOccupancyMaxActiveClusters(&n, kernel, &cfg) != cudaSuccess) { cudaGetLastError(); n = 1; }
      }
      if (n < 1) n = 1;
      cache.known[cache.count % 16] = {dev, C, n, smem};
      if (++cache.count >= 32) cache.count = 16;
    }
  }
  if (n > p.rows) n = (int)p.rows;
  if (SOLO) return launch_dep(kernel, dim3((unsigned)n), TH, smem, s, p, 1, slice, turns);
  return launch_dep_cluster(C, kernel, dim3((unsigned)(n * C)), TH, smem, s, p, C, slice, turns);
}

}  // namespace

template <class T>
cudaError_t launch_resident(const Logprob& p, cudaStream_t s, bool* taken) {
  constexpr int VEC = Group<T>::VEC;
  const int groups = (p.V + 2 * VEC - 2) / VEC;              // at most, wherever the row begins
  auto turns = [&](int C, int th) { return ((groups + C - 1) / C + th - 33) / (th - 32); };
  *taken = true;
  if (turns(1, 256) <= kTurns) return launch_clusters<T, 256, 0, true>(p, 1, groups, turns(1, 256), s);
  if (turns(1, 512) <= kTurns) return launch_clusters<T, 512, 0, true>(p, 1, groups, turns(1, 512), s);
  if (turns(1, 1024) <= kTurns) return launch_clusters<T, 1024, 0, true>(p, 1, groups, turns(1, 1024), s);
  if (turns(1, 1024) <= kTurns + 3) return launch_clusters<T, 1024, 3, true>(p, 1, groups, turns(1, 1024), s);
  if (turns(2, 1024) > kTurns && turns(2, 1024) <= kTurns + 3) return launch_clusters<T, 1024, 3, false>(p, 2, (groups + 1) / 2, turns(2, 1024), s);
  int C = 2;
  while (C <= kMaxCtas && turns(C, 1024) > kTurns) C *= 2;
  *taken = C <= kMaxCtas;
  return *taken ? launch_clusters<T, 1024, 0, false>(p, C, (groups + C - 1) / C, turns(C, 1024), s) : cudaSuccess;
}

template cudaError_t launch_resident<float>(const Logprob&, cudaStream_t, bool*);
template cudaError_t launch_resident<__nv_bfloat16>(const Logprob&, cudaStream_t, bool*);

}  // namespace logprob
}  // namespace fw
