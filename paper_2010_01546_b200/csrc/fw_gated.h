// Gated feed-forward block: what its host side (fw_gated.cu) and its kernels share.
#ifndef FW_GATED_H_
#define FW_GATED_H_

#include <cuda.h>

#include "fw_internal.h"

namespace fw {

// 2-D row-major tensor [outer][inner] of 1-byte, 2-byte (bf16) or 4-byte (fp32) elements, leading dimension ld (elements),
// boxes of 128 bytes x box_outer rows, 128-byte swizzle; elements outside read as 0
bool tmap_encode_rows128(CUtensorMap* m, int elem_bytes, const void* base, uint64_t inner, uint64_t outer, uint64_t ld,
                         uint32_t box_outer);

struct GatedForward {
  const void *X, *Wg, *Wu;
  const float *xs, *wgs, *wus;   // e4m3: scales of the rows of X, Wg, Wu
  const float *bg, *bu;          // or null
  void *H, *Zg, *Zu;             // bf16; Zg, Zu or null
  int64_t rows, ldx, ldw, ldh, ldz;
  int32_t M, N, e4m3, act;
  int32_t* status;
};
struct GatedBackward {
  const void *X, *Wg, *Wu;
  const void *Da, *Db;           // rows x N bf16: gradients of the two projections
  void *dX, *dWg, *dWu;          // dX bf16 or null; dWg, dWu bf16 or fp32, dense N x M, or null
  int64_t rows, ldx, ldw, ldd, lddx;
  int32_t M, N, w_f32;
  int32_t* status;
};
struct GatedGates {
  const void *dH, *Zg, *Zu;
  void *Da, *Db;
  float *part, *dbg, *dbu;       // part: 2 x slabs x N; dbg, dbu or null
  int64_t rows, lddh, ldz, ldd;
  int32_t N, act, slabs;
};
int gated_gate_slabs(int64_t rows, int N);      // at most kGateSlabs
constexpr int kGateSlabs = 64;
cudaError_t launch_gated_gates(const GatedGates& g, cudaStream_t s);
// tiles of 256 x 256 accumulators by CTA pairs (fw_gated_gemm.cu): products that fill the chip
fw_status launch_gated_pair_forward(const GatedForward& f, cudaStream_t s);
fw_status launch_gated_pair_backward(const GatedBackward& b, cudaStream_t s);
// narrow tiles of 128 rows, K shared by clusters (fw_gated_small.cu): the others
fw_status launch_gated_small_forward(const GatedForward& f, cudaStream_t s);
fw_status launch_gated_small_dx(const GatedBackward& b, cudaStream_t s);
fw_status launch_gated_small_dw(const GatedBackward& b, cudaStream_t s);

}  // namespace fw
#endif
