// Shared by the two transformer layers of the C ABI (layer_api.cpp, block_api.cpp):
// sizes, the library's products and the rules by which the kernels of
// layer_proj.hip and layer_gemm.hip take their place.
#pragma once

#include <hip/hip_runtime.h>
#include <rocblas/rocblas.h>

#include <cstddef>
#include <cstdint>
#include <initializer_list>

#include "dcp.h"
#include "dcp_internal.h"

namespace dcp {

constexpr size_t kAlign = 256;
inline size_t up(size_t x) { return (x + kAlign - 1) / kAlign * kAlign; }
constexpr size_t kGemmWorkspace = size_t(64) << 20;  // rocBLAS scratch, carved from the caller's workspace

constexpr int kMaxHidden = 4096;

struct Dims {
  int64_t T, H, D, h;
};

// Validates the layer's descriptor and its attention's.
int dims_of(const dcp_layer_desc* L, Dims* d);
// The calling thread's rocBLAS handle on `stream`, its scratch (kGemmWorkspace) at `scratch`.
int blas(hipStream_t stream, void* scratch, rocblas_handle* out);
// Row-major C[M, N] = op(A) op(B) + beta C into Dst (see the definition).
int gemm(rocblas_handle hd, bool ta, bool tb, int64_t M, int64_t N, int64_t K, const void* A, const void* B,
         float beta, const void* C, void* Dst, bool c_f32);
int check_ptrs(std::initializer_list<const void*> ps, const char* what);
int check_weights(const dcp_layer_weights* w);

// Which projections layer_proj.hip takes.  It saves launches and passes over
// memory; the library's main loop is faster once the contraction is long, and
// where its 256-wide tiles fit the hidden size and 192-wide ones do not.
// Library / fused, us, at (hidden, tokens):
//   Q, K, V    (1152, 300) 28 / 15, (1152, 16381) 175 / 145, (2048, 1000) 61 /
//              39, (2048, 4000) 111 / 126, (3072, 1000) 89 / 66, (3072, 8192) 406 / 425
//   W_up+GELU  (1152, 300) 16 / 17, (1152, 1000) 31 / 22, (1152, 16381) 237 /
//              201, (2048, 1000) 48 / 51, (2048, 16000) 521 / 543
//   W_down^T+GELU'  (1152, 300) 14 / 18, (1152, 1000) 27 / 23, (1152, 16381)
//              249 / 221, (2048, 1000) 47 / 50, (2048, 16000) 522 / 563
//   dY1        (1152, 1000) 29 / 39, (1152, 2500) 43 / 42, (1152, 16381) 185 /
//              137, (2048, 4000) 127 / 135
// Hidden sizes between, inside a step, fused less library at 4,096 / 8,192 /
// 16,384 / 24,576 tokens:
//   Q, K, V    1,024 -4 / -4 / +18 / +24; 1,280 -24 / -28 / -37 / +14; 1,536 -18 /
//              -8 / -17 / -6; 1,664 -21 / -34 / -17 / -41; 1,792 -17 / +7 / +31 / +42
//   W_up+GELU  1,024 -1 / -7 / +5 / +13; 1,280 -20 / -17 / -16 / -23; 1,536 -16 /
//              -1 / -7 / -5; 1,664 -5 / -3 / -1 / +1; 1,792 -3 / -14 / +5 / -33
//   W_down^T+GELU'  1,024 +5 / +3 / +7 / +18; 1,280 -8 / -28 / +18 / +45; 1,536 -3 /
//              +6 / +8 / +15; 1,664 +5 / 0 / +6 / +37; 1,792 +3 / -12 / +60 / -19
//   dY1        1,024 -6 / -13 / -8 / -20; 1,536 -6 / -13 / -30 / -48; 1,792 +3 / -2 /
//              +18 / -41
constexpr int64_t kProjHidden = 1536;
constexpr int64_t kProjTile = 192;
inline int64_t proj_tiles(int64_t n) { return (n + kProjTile - 1) / kProjTile; }
// (1,024 and smaller powers of two: 192-wide tiles pad them by an eighth or more)
inline bool library_width(const Dims& d) {
  return d.h % 256 == 0 && 10 * kProjTile * proj_tiles(d.h) > 11 * d.h && d.T * d.h > int64_t(12) << 20;
}
inline bool fused_qkv(const Dims& d) {
  return (d.h <= kProjHidden && !library_width(d)) || d.T * d.h <= int64_t(4) << 20;
}
inline bool fused_gelu(const Dims& d) { return d.h <= kProjHidden && d.T >= 512 && !library_width(d); }
inline bool fused_dy1(const Dims& d) { return d.h <= kProjHidden && d.T >= 2048; }
// W_o with its residual and dO (contraction h), W_down with its residual (4 h),
// from 6,144 tokens; below, the library is a little faster.  Where the host's
// enqueueing bounds the step (hidden 256, 6,144 tokens: 73 us forward) all three
// save a library call's 10 to 13 us of it.  Otherwise W_o and dO, if the library's
// 256-wide tiles do not divide the hidden size and the last round of 512 workgroups
// (two per CU) is mostly full.  Fused less library, change of the forward by W_o and
// of the step by dO: 108 sizes within the rule (768 to 1,472 wide, 6,144 to 28,672
// tokens) -1.2 % (worst +2.3, best -5) and -0.3 %; hidden 1,152: 336 tiles (0.66 of
// a round) +7.9 us of 310, 384 (0.75) -4.7 of 385, 768 -16.5 of 710, 1,152 -17 of
// 1,020; multiples of 256: 1,024 +4 to +26, 1,536 -18 to +20.  W_down is the
// library's: +10 to +60 us at most sizes (1,152 wide: 10,240 tokens +5, 12,288 +34,
// 24,576 +10; 1,440: +11 to +62), -25 only around 768 tiles of hidden 1,152.
constexpr int64_t kPlainTokens = 6144;
inline bool enqueue_bound(const Dims& d) { return d.T >= kPlainTokens && d.T * d.h <= int64_t(2) << 20; }
inline bool fused_square(const Dims& d) {
  const int64_t tiles = (d.T + 127) / 128 * proj_tiles(d.h), rounds = (tiles + 511) / 512;
  return enqueue_bound(d) || (d.h <= kProjHidden && d.h % 256 != 0 && d.T >= kPlainTokens && 10 * tiles >= 7 * 512 * rounds);
}

// The weight gradients are the library's at hidden size 4,096, the largest, with
// many tokens: its tiles divide 4,096, 192-wide ones pad each side by 3 %.  One
// launch of all six less six products, change of the step: 4,096 at 2,048 / 8,192 /
// 10,240 / 12,288 / 16,384 / 32,768 tokens -2.0 / +0.1 / -0.9 / +0.6 to +2.3 / +1.4
// to +2.8 / +3.3 %; 2,048 (as much padding) -4.1 / -4.9 / - / -5.7 / -4.8 / -0.9,
// 3,840 -4.3 / -6.6 / - / -4.6 / -4.2 / -4.6.
inline bool library_wgrad(const Dims& d) { return d.h >= 4096 && d.T >= 12288; }

inline char* at(void* base, size_t off) { return static_cast<char*>(base) + off; }

#define DCP_HIP(x)                                                                          \
  do {                                                                                      \
    hipError_t e_ = (x);                                                                    \
    if (e_ != hipSuccess) return fail(DCP_ERR_HIP, "layer kernel: %s", hipGetErrorString(e_)); \
  } while (0)

}  // namespace dcp
