// Host-side launch interface of the 8-bit checkpoint kernels (act8.hip) and of
// the gated, normed join of a branch into the residual stream (gated_norm.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "dcp.h"

namespace dcp {

constexpr int kActMax = 3;  // matrices of one pack or unpack launch (Q, K and V of a layer)
struct ActBatch {
  const void* src[kActMax];  // bf16 (pack) or codes (unpack)
  void* dst[kActMax];        // codes (pack) or bf16 (unpack)
  void* scales[kActMax];
  int n;
};
inline int64_t act_groups(int64_t cols) { return (cols + 31) / 32; }

// Codes and scale bytes of `n` bf16 matrices [rows, cols] (row stride ld), and back.
hipError_t launch_act8_pack(const ActBatch& b, int format, int64_t rows, int cols, int64_t ld, hipStream_t s);
hipError_t launch_act8_unpack(const ActBatch& b, int format, int64_t rows, int cols, int64_t ld, hipStream_t s);
// du = da GELU'(u), a = GELU(u) with u in `format` (bf16 of row stride ld, or
// contiguous codes); da, du, a bf16 of row stride ld.
hipError_t launch_act_gelu_bwd(const void* u, const void* scales, int format, const void* da, void* du, void* a,
                               int64_t rows, int cols, int64_t ld, hipStream_t s);

// The join (see dcp_gated_norm_fwd / _bwd for the meaning of every pointer).
struct GatedNormFwd {
  const void *x, *f, *post, *gate, *pre;
  const int32_t* cu;  // null: one gate row
  void *out, *y;
  float *rstd_f, *rstd_out;
  void *keep_f, *keep_f_scales, *keep_out, *keep_out_scales;
  int64_t rows;
  int hidden, n_seqs, format;
  float alpha, eps;
};
hipError_t launch_gated_norm_fwd(const GatedNormFwd& p, hipStream_t s);

struct GatedNormBwd {
  const void *dout, *dy, *f, *f_scales, *out, *out_scales;
  const float *rstd_f, *rstd_out;
  const void *post, *gate, *pre;
  const int32_t* cu;
  void *dx, *df, *y;
  float *dpost, *dgate, *dpre;
  int64_t rows;
  int hidden, n_seqs, format, dy_f32, accumulate;
  float alpha;
};
size_t gated_norm_bwd_workspace(int64_t rows, int hidden, int n_seqs);
hipError_t launch_gated_norm_bwd(const GatedNormBwd& p, void* workspace, hipStream_t s);

}  // namespace dcp
