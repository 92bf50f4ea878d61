// Preference loss of pairs of answers from the log-probabilities of their tokens.
//
//   s = sum of logp over an answer's rows that count (by their number with `mean`)
//   h = beta ((s_a - ref_a) - (s_b - ref_b)) - margin
//   loss = w ((1 - e) log(1 + exp(-h)) + e log(1 + exp(h)))      d loss / d s_a = beta w (e - 1 / (1 + exp(h))) = -d loss / d s_b
//
// A CTA a pair; a few bytes a row beside the rows of logits that made them: latency bounds it (16 pairs
// of up to 160 tokens: 2.9 us in a row of them, 5 between the passes over the logits).  Sums are in 64 bits in a fixed order.
#include <cstdio>

#include "fw_internal.h"
#include "fw_rows.cuh"

namespace fw {
namespace {

using namespace rows;

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kMaxPairs = 1 << 24, kMaxClasses = 1 << 20;

struct Preference {
  const float* logp;
  const void* id;                       // or null: all rows count
  const int32_t* seq;
  const float *ref, *weight;
  float *loss, *sums, *dlogp;
  int64_t rows;
  int32_t pairs, V, i64, mean;
  float beta, margin, smooth;
};

struct Sum { double s; int n; };
// Both answers' sums over the CTA, the same in every thread
__device__ __forceinline__ void over_cta(Sum (&v)[2]) {
  __shared__ Sum part[kWarps][2];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
  for (int k = 0; k < 2; ++k) v[k] = {warp_sum(v[k].s), warp_sum(v[k].n)};
  if (lane < 2) part[warp][lane] = lane == 0 ? v[0] : v[1];
  __syncthreads();
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    v[k] = part[0][k];
#pragma unroll
    for (int w = 1; w < kWarps; ++w) v[k] = {v[k].s + part[w][k].s, v[k].n + part[w][k].n};
  }
}
__device__ __forceinline__ bool counts(const Preference& p, int64_t row) {
  if (!p.id) return true;
  const int64_t i = p.i64 ? static_cast<const int64_t*>(p.id)[row] : static_cast<const int32_t*>(p.id)[row];
  return i >= 0 && i < p.V;
}
__device__ __forceinline__ int64_t border(const Preference& p, int k) {
  const int64_t at = p.seq[k];
  return at < 0 ? 0 : at > p.rows ? p.rows : at;
}

__global__ void __launch_bounds__(kThreads) preference_kernel(const Preference p) {
  dep_sync();
  const int pair = blockIdx.x;
  if (pair == p.pairs) {                // rows before the first answer and behind the last
    const int64_t first = border(p, 0), last = border(p, 2 * p.pairs);
    for (int64_t r = threadIdx.x; r < first; r += kThreads) p.dlogp[r] = 0.f;
    for (int64_t r = last + threadIdx.x; r < p.rows; r += kThreads) p.dlogp[r] = 0.f;
    return;
  }
  const int64_t edge[3] = {border(p, 2 * pair), border(p, 2 * pair + 1), border(p, 2 * pair + 2)};
  const float ref[2] = {p.ref ? p.ref[2 * pair] : 0.f, p.ref ? p.ref[2 * pair + 1] : 0.f}, weight = p.weight ? p.weight[pair] : 1.f;
  Sum v[2] = {{0.0, 0}, {0.0, 0}};
#pragma unroll
  for (int k = 0; k < 2; ++k)
    for (int64_t r = edge[k] + threadIdx.x; r < edge[k + 1]; r += kThreads) {
      const float x = p.logp[r];
      if (counts(p, r)) { v[k].s += x; ++v[k].n; }
    }
  over_cta(v);
  if (p.mean)
#pragma unroll
    for (int k = 0; k < 2; ++k) v[k].s /= v[k].n > 0 ? v[k].n : 1;
  const double h = p.beta * ((v[0].s - ref[0]) - (v[1].s - ref[1])) - p.margin, e = p.smooth, w = weight;
  const double t = exp(-fabs(h));                            // log(1 + exp(x)) = max(x, 0) + log(1 + exp(-|x|))
  if (threadIdx.x == kThreads - 1) {                         // beside the others' slopes
    const double l = log1p(t);
    p.loss[pair] = w == 0.0 ? 0.f : (float)(w * ((1.0 - e) * (fmax(-h, 0.0) + l) + (e > 0.0 ? e * (fmax(h, 0.0) + l) : 0.0)));
    if (p.sums) { p.sums[2 * pair] = (float)v[0].s; p.sums[2 * pair + 1] = (float)v[1].s; }
  }
  if (!p.dlogp) return;
  const double d = w == 0.0 ? 0.0 : p.beta * w * (e - (h > 0.0 ? t : 1.0) / (1.0 + t));           // 1 / (1 + exp(h))
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const double share = p.mean ? d / (v[k].n > 0 ? v[k].n : 1) : d;
    const float f = (float)(k == 0 ? share : -share);
    for (int64_t r = edge[k] + threadIdx.x; r < edge[k + 1]; r += kThreads) p.dlogp[r] = counts(p, r) ? f : 0.f;
  }
}

}  // namespace
}  // namespace fw

using namespace fw;

extern "C" {

void fw_preference_desc_default(fw_preference_desc* p) {
  if (!p) return;
  p->beta = 0.1f; p->margin = 0.f; p->smooth = 0.f; p->mean = 0;
}

fw_status fw_preference_loss(const fw_logprob_desc* d, const fw_preference_desc* o, const float* logp, int64_t rows, const void* id,
                             const int32_t* seq, int32_t pairs, const float* ref, const float* weight, float* loss, float* sums,
                             float* dlogp, void* cuda_stream) {
  if (!d || !o || !logp || !seq || !loss) return FW_ERR_INVALID_ARG;
  if (d->V < 1 || d->V > kMaxClasses) return FW_ERR_SHAPE;
  if (d->index_bits != 32 && d->index_bits != 64) return FW_ERR_INVALID_ARG;
  if (!(o->beta > 0.f && o->beta <= 3e38f) || !(o->margin >= -3e38f && o->margin <= 3e38f) || !(o->smooth >= 0.f && o->smooth < 1.f) ||
      (o->mean != 0 && o->mean != 1))
    return FW_ERR_INVALID_ARG;
  if (rows < 1 || rows >= (1 << 28) || pairs < 1 || pairs > kMaxPairs) return FW_ERR_SHAPE;
  const int is = d->index_bits / 8;
  const uint64_t nr = (uint64_t)rows * 4, np = (uint64_t)pairs * 4;
  const struct { const void* p; uint64_t n; int align; } in[] = {{logp, nr, 4}, {id, (uint64_t)rows * is, is}, {seq, 2 * np + 4, 4}, {ref, 2 * np, 4},
                                                                 {weight, np, 4}},
                                                         out[] = {{loss, np, 4}, {sums, 2 * np, 4}, {dlogp, nr, 4}};
  for (const auto& r : in)
    if (!aligned_to(r.p, r.align)) return FW_ERR_INVALID_ARG;
  for (int i = 0; i < 3; ++i) {
    if (!aligned_to(out[i].p, 4)) return FW_ERR_INVALID_ARG;
    for (const auto& r : in)
      if (overlap(out[i].p, out[i].n, r.p, r.n)) return FW_ERR_INVALID_ARG;
    for (int j = 0; j < i; ++j)
      if (overlap(out[i].p, out[i].n, out[j].p, out[j].n)) return FW_ERR_INVALID_ARG;
  }
  Preference p;
  p.logp = logp; p.id = id; p.seq = seq; p.ref = ref; p.weight = weight; p.loss = loss; p.sums = sums; p.dlogp = dlogp; p.rows = rows;
  p.pairs = pairs; p.V = d->V; p.i64 = d->index_bits == 64; p.mean = o->mean; p.beta = o->beta; p.margin = o->margin; p.smooth = o->smooth;
  cudaStream_t s = (cudaStream_t)cuda_stream;
  ProfScope ps(FW_PROF_MISC, s);
  const cudaError_t e = launch_dep(preference_kernel, (unsigned)(pairs + (dlogp ? 1 : 0)), kThreads, 0, s, p);
  if (e == cudaSuccess) return FW_OK;
  fprintf(stderr, "[fw] fw_preference_loss: %s\n", cudaGetErrorString(e));
  return FW_ERR_CUDA;
}

}  // extern "C"
