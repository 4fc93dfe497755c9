// 8-bit activation checkpoints: bf16 to codes and scale bytes, the way back, and
// the GELU backward that reads its input from them.  All HBM-bound: a pack reads 2
// and writes 1 + 1/32 bytes an element, an unpack the reverse, the GELU backward
// reads 3 + 1/32 and writes 4.  One 16-byte access of the bf16 side a lane, eight
// elements, so that four lanes hold a group and its largest magnitude takes two lane
// moves.  16,381 x 4,608 in int8: pack 41 us (5.6 TB/s), unpack 33 (7.0: the codes
// come from the last-level cache), GELU backward 88 (6.0), from a bf16 u 103 (5.9); a
// 2 GiB copy 4.9 to 5.0 TB/s.
// 429 x 256: 2.5 us each, the launch.
#include "act8.h"
#include "block_launch.h"

namespace dcp {
namespace {

// Pieces of 8 columns, 4 to a group, `per_row` = 4 ceil(cols / 32) to a row (the
// last ones of a row whose last group is short are idle).  Dense matrices whose
// rows are whole groups are one long row; otherwise piece / per_row comes from a
// 32-bit multiply (pieces stay below 2^31: the launch cuts taller matrices).
struct Pieces {
  uint32_t total, per_row, mul, shift;
  int cols, groups;
  int64_t ld;
};

struct At {
  int64_t wide, dense, group;  // element of the bf16 matrix, of the codes, index of the scale byte
  bool live;
};

template <bool DENSE>
__device__ __forceinline__ At piece_at(const Pieces& d, uint32_t i) {
  if constexpr (DENSE) return At{int64_t(i) * 8, int64_t(i) * 8, int64_t(i >> 2), true};
  const uint32_t row = (__umulhi(i, d.mul) + i) >> d.shift, p = i - row * d.per_row;
  const int c = int(p) * 8;
  return At{int64_t(row) * d.ld + c, int64_t(row) * d.cols + c, int64_t(row) * d.groups + int(p >> 2), c < d.cols};
}

template <int FMT, bool DENSE>
__global__ __launch_bounds__(256) void act8_pack_kernel(ActBatch b, Pieces d) {
  const uint32_t i = blockIdx.x * 256u + threadIdx.x;
  if (i >= d.total) return;  // (total is a multiple of 4: a group's lanes leave together)
  const int m = blockIdx.y;
  const At at = piece_at<DENSE>(d, i);
  bf16x8 v{};
  if (at.live) v = *reinterpret_cast<const bf16x8*>(static_cast<const __bf16*>(b.src[m]) + at.wide);
  const uint32_t byte = scale_byte<FMT>(group_top(top_bits(v)));
  if (at.live) *reinterpret_cast<u32x2*>(static_cast<uint8_t*>(b.dst[m]) + at.dense) = encode8<FMT>(v, byte);
  if ((i & 3) == 0) static_cast<uint8_t*>(b.scales[m])[at.group] = uint8_t(byte);
}

template <int FMT, bool DENSE>
__global__ __launch_bounds__(256) void act8_unpack_kernel(ActBatch b, Pieces d) {
  const uint32_t i = blockIdx.x * 256u + threadIdx.x;
  if (i >= d.total) return;
  const int m = blockIdx.y;
  const At at = piece_at<DENSE>(d, i);
  if (!at.live) return;
  Held8<FMT> h;
  h.load(b.src[m], static_cast<const uint8_t*>(b.scales[m]), at.dense, at.group);
  float x[8];
  h.get(x);
  bf16x8 o;
#pragma unroll
  for (int e = 0; e < 8; ++e) o[e] = __bf16(x[e]);
  *reinterpret_cast<bf16x8*>(static_cast<__bf16*>(b.dst[m]) + at.wide) = o;
}

template <int FMT, bool DENSE>
__global__ __launch_bounds__(256) void act_gelu_bwd_kernel(const void* u, const uint8_t* scales, const __bf16* da,
                                                           __bf16* du, __bf16* a, Pieces d) {
  const uint32_t i = blockIdx.x * 256u + threadIdx.x;
  if (i >= d.total) return;
  const At at = piece_at<DENSE>(d, i);
  if (!at.live) return;
  Held8<FMT> h;
  h.load(u, scales, FMT == DCP_ACT_BF16 ? at.wide : at.dense, at.group);
  const bf16x8 g = *reinterpret_cast<const bf16x8*>(da + at.wide);
  float x[8];
  h.get(x);
  bf16x8 o, ov;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    float act, slope;
    gelu_and_slope(x[e], &act, &slope);
    o[e] = __bf16(float(g[e]) * slope);
    ov[e] = __bf16(act);
  }
  *reinterpret_cast<bf16x8*>(du + at.wide) = o;
  *reinterpret_cast<bf16x8*>(a + at.wide) = ov;
}

// Runs f(first row, rows, Pieces, dense) over slabs of rows with fewer than 2^31 pieces.
template <class F>
hipError_t over_slabs(int64_t rows, int cols, int64_t ld, F f) {
  const uint32_t per_row = uint32_t(act_groups(cols)) * 4;
  const bool dense = ld == cols && cols % kActGroup == 0;
  const int64_t step = ((int64_t(1) << 31) - 1) / per_row;
  for (int64_t r = 0; r < rows; r += step) {
    const int64_t n = rows - r < step ? rows - r : step;
    Pieces d{uint32_t(n * per_row), per_row, 0, 0, cols, int(act_groups(cols)), ld};
    while ((uint64_t(1) << d.shift) < per_row) ++d.shift;
    d.mul = uint32_t(((uint64_t(1) << 32) * ((uint64_t(1) << d.shift) - per_row)) / per_row + 1);
    const hipError_t e = f(r, d, dense);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

inline char* shifted(const void* p, int64_t bytes) { return const_cast<char*>(static_cast<const char*>(p)) + bytes; }

}  // namespace

hipError_t launch_act8_pack(const ActBatch& b, int format, int64_t rows, int cols, int64_t ld, hipStream_t s) {
  return over_slabs(rows, cols, ld, [&](int64_t r, const Pieces& d, bool dense) {
    ActBatch at = b;
    for (int m = 0; m < b.n; ++m) {
      at.src[m] = shifted(b.src[m], 2 * r * ld);
      at.dst[m] = shifted(b.dst[m], r * cols);
      at.scales[m] = shifted(b.scales[m], r * d.groups);
    }
    const dim3 grid((d.total + 255) / 256, unsigned(b.n));
    auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(256), 0, s, at, d); };
    if (format == DCP_ACT_INT8) {
      if (dense) launch(act8_pack_kernel<DCP_ACT_INT8, true>);
      else launch(act8_pack_kernel<DCP_ACT_INT8, false>);
    } else {
      if (dense) launch(act8_pack_kernel<DCP_ACT_E4M3, true>);
      else launch(act8_pack_kernel<DCP_ACT_E4M3, false>);
    }
    return hipGetLastError();
  });
}

hipError_t launch_act8_unpack(const ActBatch& b, int format, int64_t rows, int cols, int64_t ld, hipStream_t s) {
  return over_slabs(rows, cols, ld, [&](int64_t r, const Pieces& d, bool dense) {
    ActBatch at = b;
    for (int m = 0; m < b.n; ++m) {
      at.src[m] = shifted(b.src[m], r * cols);
      at.dst[m] = shifted(b.dst[m], 2 * r * ld);
      at.scales[m] = shifted(b.scales[m], r * d.groups);
    }
    const dim3 grid((d.total + 255) / 256, unsigned(b.n));
    auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(256), 0, s, at, d); };
    if (format == DCP_ACT_INT8) {
      if (dense) launch(act8_unpack_kernel<DCP_ACT_INT8, true>);
      else launch(act8_unpack_kernel<DCP_ACT_INT8, false>);
    } else {
      if (dense) launch(act8_unpack_kernel<DCP_ACT_E4M3, true>);
      else launch(act8_unpack_kernel<DCP_ACT_E4M3, false>);
    }
    return hipGetLastError();
  });
}

hipError_t launch_act_gelu_bwd(const void* u, const void* scales, int format, const void* da, void* du, void* a,
                               int64_t rows, int cols, int64_t ld, hipStream_t s) {
  return over_slabs(rows, cols, ld, [&](int64_t r, const Pieces& d, bool dense) {
    const void* us = shifted(u, format == DCP_ACT_BF16 ? 2 * r * ld : r * cols);
    const uint8_t* sc = format == DCP_ACT_BF16 ? nullptr : reinterpret_cast<uint8_t*>(shifted(scales, r * d.groups));
    auto wide = [&](const void* p) { return reinterpret_cast<__bf16*>(shifted(p, 2 * r * ld)); };
    auto launch = [&](auto kernel) {
      hipLaunchKernelGGL(kernel, dim3((d.total + 255) / 256), dim3(256), 0, s, us, sc, wide(da), wide(du), wide(a), d);
    };
    switch (format) {
      case DCP_ACT_BF16:
        if (dense) launch(act_gelu_bwd_kernel<DCP_ACT_BF16, true>);
        else launch(act_gelu_bwd_kernel<DCP_ACT_BF16, false>);
        break;
      case DCP_ACT_INT8:
        if (dense) launch(act_gelu_bwd_kernel<DCP_ACT_INT8, true>);
        else launch(act_gelu_bwd_kernel<DCP_ACT_INT8, false>);
        break;
      default:
        if (dense) launch(act_gelu_bwd_kernel<DCP_ACT_E4M3, true>);
        else launch(act_gelu_bwd_kernel<DCP_ACT_E4M3, false>);
    }
    return hipGetLastError();
  });
}

}  // namespace dcp
