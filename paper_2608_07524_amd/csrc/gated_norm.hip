// The join of a block's branch f into the residual stream x, with the norm before
// the next block, and its backward.  For row t of sequence s:
//   n = RMSNorm(f; post),  out = alpha x + gate_s o n,  y = RMSNorm(out; pre),
// RMSNorm(z; g) = z o g / sqrt(mean(z^2) + eps); post, gate and pre may each be
// absent.  With f and out kept from the forward (bf16 or 8-bit checkpoints), the
// saved row scales r_f and r_o, fh = f r_f and oh = out r_o, the backward of
// <dout, out> + <dy, y> is
//   G  = dout + r_o (d - oh mean(d oh)),            d = pre o dy,
//   dx = alpha G,
//   df = r_f (e - fh mean(e fh)),                   e = post o gate_s o G,
//   A_s = sum_{t in s} G o fh,   dgate_s = post o A_s,   dpost = sum_s gate_s o A_s,
//   dpre = sum_t dy o oh.
// HBM-bound: every input is read once and every output written once, all of a row
// in registers between; sums, statistics and gradients of the parameters are fp32.
// 131,072 rows of hidden 1,152, eight sequences, int8: join with f's checkpoint 257
// us (5.3 TB/s), with f's and out's, as a block's first join, 281 (5.4); backward 384 + 12
// (4.7 TB/s, and the partial rows), with fp32 dy, as in a block, 450 in all (4.7); a 2 GiB
// copy 4.9 to 5.0 TB/s.  65,536 rows in 1,286 sequences of 1 to 51 tokens: 198 + 12.
// 16,384 rows of hidden 4,096 in bf16: join 98 (5.5), backward 190 + 5 (4.9).  429 rows of
// 256: 3.7; 5.6 + 5.7, chains of memory latencies.
#include <type_traits>

#include "act8.h"
#include "block_launch.h"
#include "tile_shapes.h"

namespace dcp {
namespace {

// A team of TL lanes owns a row, 8 columns (one 16-byte access) a lane: the power
// of two up to 64, or the multiple of 64, that covers hidden / 8.  One piece a lane
// keeps the backward at 128 registers, so that four wavefronts share a SIMD and loads
// are always in flight; with three pieces (one wavefront for hidden 1,152) it took 259,
// one wavefront a SIMD, and twice the time.  Teams take consecutive rows:
// gains, gate and the place in cu_seqlens are fetched once, and the next row is
// loaded before the present one is worked on.  A workgroup is one team of more than
// 128 lanes or 256 lanes of smaller ones (two teams of 192: 12 wavefronts a CU instead
// of 15, 407 -> 421 us for 131,072 rows backward, 333 -> 378 forward).
template <int TL>
struct Team {
  static constexpr int kBlock = TL > 128 ? TL : 256, kTeams = kBlock / TL;
  static constexpr int kSub = TL < 64 ? TL : 64;       // lanes of a team within a wavefront
  static constexpr int kWaves = TL < 64 ? 1 : TL / 64;  // wavefronts a team spans
  // What all lanes of a team have alike is in scalar registers where a wavefront has one team.
  static __device__ __forceinline__ int alike(int v) { return TL < 64 ? v : __builtin_amdgcn_readfirstlane(v); }
};
typedef uint32_t row_t;  // rows < 2^31, and at most a workgroup's more
__device__ __forceinline__ row_t offset_of(const int32_t* cu, int s) { return row_t(max(cu[s], 0)); }
// Rows in use: all, or those of the sequences.
__device__ __forceinline__ row_t rows_of(int64_t rows, const int32_t* cu, int n_seqs) {
  return cu ? min(row_t(rows), offset_of(cu, n_seqs)) : row_t(rows);
}

// Sums of N values over a team.  Teams of several wavefronts meet once, in the half
// of `red` that belongs to this row's parity: the other half's readers are at most
// one barrier behind.
template <int TL, int N>
__device__ __forceinline__ void team_total(float (&v)[N], float* red, int parity) {
#pragma unroll
  for (int n = 0; n < N; ++n) v[n] = lane_total<Team<TL>::kSub>(v[n]);
  if constexpr (Team<TL>::kWaves > 1) {
    constexpr int kWaves = Team<TL>::kBlock / 64;
    const int wave = threadIdx.x >> 6, first = wave / Team<TL>::kWaves * Team<TL>::kWaves;
    float* r = red + parity * kWaves * N;
    if ((threadIdx.x & 63) == 0) {
#pragma unroll
      for (int n = 0; n < N; ++n) r[wave * N + n] = v[n];
    }
    __syncthreads();
#pragma unroll
    for (int n = 0; n < N; ++n) {
      float t = r[first * N + n];
#pragma unroll
      for (int w = 1; w < Team<TL>::kWaves; ++w) t += r[(first + w) * N + n];
      v[n] = t;
    }
  }
}

// The sequence of `row`: the last index s <= n with cu[s] <= row (n: the row lies
// behind the last sequence), by as many probes a step as the team has lanes in the
// wavefront (64: three steps reach 2^18 sequences).  Whatever cu holds, s stays in
// [0, n].
template <int L>
__device__ __forceinline__ int sequence_of(const int32_t* cu, int n, row_t row) {
  const int lane = threadIdx.x & (L - 1), shift = threadIdx.x & 63 & ~(L - 1);
  const uint64_t mask = L == 64 ? ~uint64_t(0) : (uint64_t(1) << (L & 63)) - 1;
  int lo = 0, len = n + 1;
  while (len > 1) {
    const int step = (len + L - 1) / L, at = lane * step;
    const bool below = at < len && offset_of(cu, lo + at) <= row;
    const int c = max(int(__popcll((__ballot(below) >> shift) & mask)) - 1, 0);
    lo += c * step;
    len = min(step, len - c * step);
  }
  return lo;
}

// Follows a team's consecutive rows through cu_seqlens, one offset ahead of them.
template <int TL>
struct Walk {
  const int32_t* cu = nullptr;
  int n = 0, s = 0;
  row_t begin = 0, end = ~row_t(0), end2 = 0;  // rows of sequence s, and the end of the next one
  __device__ __forceinline__ row_t at(int i) const { return row_t(Team<TL>::alike(int(offset_of(cu, i)))); }
  __device__ __forceinline__ void start(const int32_t* c, int n_seqs, row_t row) {
    cu = c;
    n = n_seqs;
    s = Team<TL>::alike(min(sequence_of<Team<TL>::kSub>(c, n_seqs, row), n_seqs - 1));
    begin = at(s);
    end = at(s + 1);
    end2 = at(min(s + 2, n));
  }
  // To the sequence of `row`, which lies behind sequence s; returns how many further.
  __device__ __forceinline__ int step(row_t row) {
    const int from = s;
    while (row >= end && s < n - 1) {
      ++s;
      begin = end;
      end = end2;
      end2 = at(min(s + 2, n));
    }
    return s - from;
  }
};

// 8 values of a bf16 row at column c, 1 where there is none.
__device__ __forceinline__ bf16x8 gain8(const __bf16* g, int c, int h) {
  if (g && c < h) return *reinterpret_cast<const bf16x8*>(g + c);
  bf16x8 one;
#pragma unroll
  for (int e = 0; e < 8; ++e) one[e] = __bf16(1.f);
  return one;
}
// Keeps 8 values as they are, in bf16: without it the compiler converts what a loop does
// not change before the loop and holds twice the registers through it.
__device__ __forceinline__ void stay_packed(bf16x8& v) {
  u32x4 w = __builtin_bit_cast(u32x4, v);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    uint32_t x = w[i];
    asm("" : "+v"(x));
    w[i] = x;
  }
  v = __builtin_bit_cast(bf16x8, w);
}
__device__ __forceinline__ void gains_product(const __bf16* a, const __bf16* b, int c, int h, float (&v)[8]) {
  const bf16x8 x = gain8(a, c, h), y = gain8(b, c, h);
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = float(x[e]) * float(y[e]);
}
__device__ __forceinline__ bf16x8 rounded(const float (&v)[8]) {
  bf16x8 b;
#pragma unroll
  for (int e = 0; e < 8; ++e) b[e] = __bf16(v[e]);
  return b;
}

// v where the mask is all ones, 0 (also for a NaN) where it is zero.
__device__ __forceinline__ float masked(float v, uint32_t mask) { return __uint_as_float(__float_as_uint(v) & mask); }

template <int FMT>
__device__ __forceinline__ void keep8(void* codes, void* scales, bf16x8 v, row_t row, int c, int h, int groups) {
  const uint32_t byte = scale_byte<FMT>(group_top(top_bits(v)));
  if (c < h) *reinterpret_cast<u32x2*>(static_cast<uint8_t*>(codes) + int64_t(row) * h + c) = encode8<FMT>(v, byte);
  if (c < h && (c & 31) == 0) static_cast<uint8_t*>(scales)[int64_t(row) * groups + (c >> 5)] = uint8_t(byte);
}

// KEEP: format of the checkpoints (DCP_ACT_BF16: none).  y and its statistics come
// from out in fp32, the checkpoint of out from out as stored.
template <int TL, int KEEP>
__global__ __launch_bounds__(Team<TL>::kBlock) void gated_norm_fwd_kernel(GatedNormFwd p, int team_rows) {
  using T = Team<TL>;
  __shared__ float red[2][2][T::kBlock / 64];
  const int lane = threadIdx.x % TL, c = 8 * lane, h = p.hidden, groups = (h + kActGroup - 1) / kActGroup;
  const bool mine = c < h;
  const row_t rows = rows_of(p.rows, p.cu, p.n_seqs), block_first = blockIdx.x * row_t(T::kTeams * team_rows);
  const row_t first = block_first + row_t(T::alike(threadIdx.x / TL) * team_rows);
  if (block_first >= rows) return;
  // (teams that meet at barriers all take the first team's turns)
  const row_t lead = T::kWaves > 1 ? block_first : first;
  const int turns = lead < rows ? int(min(rows - lead, row_t(team_rows))) : 0;
  const __bf16 *x = static_cast<const __bf16*>(p.x), *f = static_cast<const __bf16*>(p.f);
  const __bf16 *post = static_cast<const __bf16*>(p.post), *gate = static_cast<const __bf16*>(p.gate);
  bf16x8 xn{}, fn{};
  auto fetch = [&](row_t row) {
    if (mine && row < rows) {
      fn = *reinterpret_cast<const bf16x8*>(f + int64_t(row) * h + c);
      xn = *reinterpret_cast<const bf16x8*>(x + int64_t(row) * h + c);
    }
  };
  fetch(first);
  float branch[8];  // post o gate
  const bf16x8 pre8 = gain8(static_cast<const __bf16*>(p.pre), c, h);
  Walk<TL> walk;
  if (p.cu && first < rows) walk.start(p.cu, p.n_seqs, first);
  gains_product(post, gate ? gate + int64_t(walk.s) * h : nullptr, c, h, branch);
  for (int i = 0; i < turns; ++i) {
    const row_t row = first + row_t(i);
    const bool live = row < rows;
    if (live && row >= walk.end) {
      walk.step(row);
      gains_product(post, gate + int64_t(walk.s) * h, c, h, branch);
    }
    const bf16x8 xv = xn, fv = fn;
    if (i + 1 < turns) fetch(row + 1);
    float fx[8], r[1] = {0.f}, rf = 1.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      fx[e] = float(fv[e]);
      r[0] += fx[e] * fx[e];
    }
    if (p.post) {
      team_total<TL>(r, red[0][0], i & 1);
      rf = rsqrtf(r[0] / float(h) + p.eps);
      if (live && lane == 0) p.rstd_f[row] = rf;
    }
    float o[8];
    r[0] = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      o[e] = p.alpha * float(xv[e]) + branch[e] * (fx[e] * rf);
      r[0] += o[e] * o[e];
    }
    const bf16x8 ov = rounded(o);
    if (live && mine) *reinterpret_cast<bf16x8*>(static_cast<__bf16*>(p.out) + int64_t(row) * h + c) = ov;
    if constexpr (KEEP != DCP_ACT_BF16) {
      if (live && p.keep_f) keep8<KEEP>(p.keep_f, p.keep_f_scales, fv, row, c, h, groups);
      if (live && p.keep_out) keep8<KEEP>(p.keep_out, p.keep_out_scales, ov, row, c, h, groups);
    }
    if (p.pre) {
      team_total<TL>(r, red[1][0], i & 1);
      const float ro = rsqrtf(r[0] / float(h) + p.eps);
      if (live && lane == 0) p.rstd_out[row] = ro;
#pragma unroll
      for (int e = 0; e < 8; ++e) o[e] *= ro * float(pre8[e]);
      if (live && mine) *reinterpret_cast<bf16x8*>(static_cast<__bf16*>(p.y) + int64_t(row) * h + c) = rounded(o);
    }
  }
}

// Backward.  A lane keeps its columns' sums of G o fh and dy o oh over the team's
// rows: one partial row a workgroup for dpost (or A with one gate row) and dpre, and,
// with a gate for each sequence, A_s either straight into dgate (a sequence whose
// rows all lie in one team) or as a partial row of the team: slot 0 for the sequence
// that its first row belongs to, slot 1 for one that starts inside and goes on.  A
// second launch adds the partial rows in a fixed order, so results are bitwise
// reproducible.
//
// The two means of a row need one meeting of the team: with t = dout + r_o d and m =
// mean(d oh), G = t - r_o m oh, so mean(e fh) = mean(b t) - r_o m mean(b oh), b = post
// o gate o fh.
struct BwdShape {
  int lanes, block, teams_of_block, team_rows;
  int64_t blocks, teams;
};
inline int team_lanes(int hidden) {
  const int need = (hidden + 7) / 8;
  if (need > 64) return (need + 63) / 64 * 64;
  int l = 8;
  while (l < need) l *= 2;
  return l;
}
// Wavefronts that share a SIMD: 128 registers each where a team's rows and offsets are in
// scalar registers, more otherwise.  2 to 6 of the 128 spill at 448 and 512 lanes with an
// fp32 dy (bf16 activations: from 384 lanes) and 2 at 512 with a bf16 dy and int8, at no
// cost that shows: 32,768 rows of 4,096, int8, 390 us with fp32 dy and 341 with bf16, 2,048
// wide (no spills) 60,000 rows 373 and 325, all 4.6 to 4.8 TB/s.
constexpr int bwd_waves(int lanes) { return lanes < 64 ? 3 : 4; }
constexpr int kBwdRowsMax = 128, kShortRows = 32;
inline BwdShape bwd_shape(int64_t rows, int hidden, int n_seqs) {
  BwdShape s;
  s.lanes = team_lanes(hidden);
  s.block = s.lanes > 128 ? s.lanes : 256;
  s.teams_of_block = s.block / s.lanes;
  // Rows of a team: the workgroups are one evenly filled round of what fits the chip, or
  // as few as teams of at most kBwdRowsMax rows (which a lane adds one after another)
  // allow.  Long sequences, 131,072 rows of hidden 1,152: 103 / 64 / 52 / 32 / 16 rows
  // 392 / 411 / 401 / 409 / 429 us; 16,384 rows of 4,096: 64 / 32 / 16 / 8 rows 192 / 197
  // / 202 / 208.
  //   Two rounds where sequences have fewer than kShortRows rows on average, if that
  // leaves a team four rows (65,536 rows of 64: three rows a team 35 us, two 44).  A
  // sequence's end costs a team as much as a row, and clips of one frame beside longer ones
  // put many ends into few teams, which a second round evens out.  The host knows no more of
  // that than the average (allocated rows, all sequences, empty ones too).  One round / two:
  //   clips of 1, 16, 32 or 51 rows mixed, average 16 to 20: 131,072 rows of 1,152 503 to
  //     528 / 412 to 476, of 256 129 to 134 / 110 to 134; 32,768 of 4,096, 7: 470 / 413
  //   average 32 to 50, nothing in sum: of 1,152 34 rows 397 / 408, 35 398 / 423, 39 500 /
  //     414, 42 398 / 405, 49 395 / 406, 51 395 / 404; of 2,048 32 rows 183 / 192, 36 206 / 190
  //   lengths uniform from 1 to twice the average, where ends are spread evenly: 2 to 6 %
  //     lost at any average (of 1,152: 16 rows 408 / 420, 32 402 / 414, 64 396 / 406)
  const int64_t round = int64_t(s.teams_of_block) * kNumCU * (4 * bwd_waves(s.lanes) / (s.block / 64));
  const bool shorts = n_seqs > 0 && rows < int64_t(kShortRows) * n_seqs && rows >= 8 * round;
  const int64_t least = (rows + round * kBwdRowsMax - 1) / (round * kBwdRowsMax);
  const int64_t rounds = shorts && least < 2 ? 2 : least > 1 ? least : 1;
  s.team_rows = rows > 0 ? int((rows + round * rounds - 1) / (round * rounds)) : 1;
  const int64_t per_block = int64_t(s.teams_of_block) * s.team_rows;
  s.blocks = (rows + per_block - 1) / per_block;
  s.teams = s.blocks * s.teams_of_block;
  return s;
}

struct BwdParts {
  float *pre, *post;  // [blocks][hidden] each
  float* seg;         // [teams][2][hidden]
  int team_rows;
};

template <int TL, int FMT, bool DY32>
__global__ __launch_bounds__(Team<TL>::kBlock, bwd_waves(TL)) void gated_norm_bwd_kernel(GatedNormBwd p, BwdParts w) {
  using T = Team<TL>;
  __shared__ float red[2][3 * (T::kBlock / 64)];
  __shared__ float sums[T::kTeams][8 * TL];
  const int team = T::alike(threadIdx.x / TL), lane = threadIdx.x % TL, c = 8 * lane;
  const int h = p.hidden, groups = (h + kActGroup - 1) / kActGroup;
  const bool mine = c < h;
  const row_t rows = rows_of(p.rows, p.cu, p.n_seqs), block_first = blockIdx.x * row_t(T::kTeams * w.team_rows);
  const row_t first = block_first + row_t(team * w.team_rows), lead = T::kWaves > 1 ? block_first : first;
  const int turns = lead < rows ? int(min(rows - lead, row_t(w.team_rows))) : 0;
  const bool has_f = p.post != nullptr || p.gate != nullptr;
  // (without post df = gate o G, whatever f holds: 0 fh would be NaN where f is not finite; a
  // branch instead of the mask spills registers from 64 lanes on)
  const uint32_t normed = p.post ? ~0u : 0u;
  const __bf16 *dout = static_cast<const __bf16*>(p.dout);
  const __bf16 *post = static_cast<const __bf16*>(p.post), *gate = static_cast<const __bf16*>(p.gate);

  bf16x8 gn{}, dn{};
  f32x4 dn32[2] = {};
  Held8<FMT> fn{}, on{};
  float rfn = 1.f, ron = 0.f;
  auto fetch = [&](row_t row) {
    if (row >= rows) return;
    if (p.post) rfn = p.rstd_f[row];
    if (p.pre) ron = p.rstd_out[row];
    if (!mine) return;
    const int64_t at = int64_t(row) * h + c, grp = int64_t(row) * groups + (c >> 5);
    if (dout) gn = *reinterpret_cast<const bf16x8*>(dout + at);
    if (p.pre) {
      on.load(p.out, static_cast<const uint8_t*>(p.out_scales), at, grp);
      if constexpr (DY32) {
        dn32[0] = *reinterpret_cast<const f32x4*>(static_cast<const float*>(p.dy) + at);
        dn32[1] = *reinterpret_cast<const f32x4*>(static_cast<const float*>(p.dy) + at + 4);
      } else {
        dn = *reinterpret_cast<const bf16x8*>(static_cast<const __bf16*>(p.dy) + at);
      }
    }
    if (has_f) fn.load(p.f, static_cast<const uint8_t*>(p.f_scales), at, grp);
  };
  fetch(first);
  float acc_pre[8], acc_a[8];  // sums of dy o oh, G o fh
  bf16x8 post8 = gain8(post, c, h), pre8 = gain8(static_cast<const __bf16*>(p.pre), c, h);
  Walk<TL> walk;
  row_t from = first;  // first of the team's rows in the current sequence
  if (p.cu && first < rows) walk.start(p.cu, p.n_seqs, first);
  // the gate of the current sequence, and of the next: a short sequence's end waits for
  // neither offsets nor gates
  bf16x8 gate8 = gain8(gate ? gate + int64_t(walk.s) * h : nullptr, c, h), gate_next{};
  if (p.cu) gate_next = gain8(gate + int64_t(min(walk.s + 1, p.n_seqs - 1)) * h, c, h);
  float* sum = &sums[team][c];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    acc_pre[e] = acc_a[e] = 0.f;
    sum[e] = 0.f;
  }
  // The team's sum of G o fh over rows [from, to) of the current sequence leaves the
  // registers.
  auto flush = [&](row_t to) {
    if (!mine) return;
    const bool starts = walk.begin >= first, whole = starts && to >= min(walk.end, rows);
    float* dst = (whole ? p.dgate + int64_t(walk.s) * h
                        : w.seg + ((int64_t(blockIdx.x) * T::kTeams + team) * 2 + (from > first ? 1 : 0)) * h) + c;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      sum[e] += float(gate8[e]) * acc_a[e];
      float v = acc_a[e];
      if (whole) {
        v *= float(post8[e]);
        if (p.accumulate) v += dst[e];
      }
      dst[e] = v;
      acc_a[e] = 0.f;
    }
  };
  for (int i = 0; i < turns; ++i) {
    const row_t row = first + row_t(i);
    const bool live = row < rows;
    if (live && row >= walk.end) {
      flush(row);
      from = row;
      gate8 = gate_next;
      if (walk.step(row) > 1) gate8 = gain8(gate + int64_t(walk.s) * h, c, h);
      gate_next = gain8(gate + int64_t(min(walk.s + 1, p.n_seqs - 1)) * h, c, h);
    }
    stay_packed(post8);
    stay_packed(pre8);
    stay_packed(gate8);
    float t[8], d[8], oh[8], fh[8];
    const float rf = rfn, ro = ron;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      t[e] = float(gn[e]);
      d[e] = DY32 ? dn32[e >> 2][e & 3] : float(dn[e]);
    }
    on.get_scaled(ro, oh);
    if (FMT == DCP_ACT_INT8 && !p.post) fn.get(fh);
    else fn.get_scaled(rf, fh);
    if (!mine || !live) {
#pragma unroll
      for (int e = 0; e < 8; ++e) t[e] = d[e] = oh[e] = fh[e] = 0.f;
    }
    if (i + 1 < turns) fetch(row + 1);
    float r[3] = {0.f, 0.f, 0.f};
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      acc_pre[e] += d[e] * oh[e];
      d[e] *= float(pre8[e]);
      t[e] += ro * d[e];
      r[0] += d[e] * oh[e];
      const float b = float(post8[e]) * float(gate8[e]) * fh[e];
      r[1] += b * t[e];
      r[2] += b * oh[e];
    }
    if (live && mine && p.y) {
      float y[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] = oh[e] * float(pre8[e]);
      *reinterpret_cast<bf16x8*>(static_cast<__bf16*>(p.y) + int64_t(row) * h + c) = rounded(y);
    }
    team_total<TL>(r, red[0], i & 1);
    const float m = ro * (r[0] / float(h));
    const float mf = p.post ? (r[1] - m * r[2]) / float(h) : 0.f;
    float u[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      t[e] -= m * oh[e];  // G
      acc_a[e] += t[e] * fh[e];
      u[e] = rf * (float(post8[e]) * float(gate8[e]) * t[e] - mf * masked(fh[e], normed));
      t[e] *= p.alpha;
    }
    if (live && mine) {
      if (p.dx) *reinterpret_cast<bf16x8*>(static_cast<__bf16*>(p.dx) + int64_t(row) * h + c) = rounded(t);
      *reinterpret_cast<bf16x8*>(static_cast<__bf16*>(p.df) + int64_t(row) * h + c) = rounded(u);
    }
  }
  if (p.cu) {
    if (first < rows) flush(min(first + row_t(w.team_rows), rows));
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) sum[e] = acc_a[e];
  }
  auto add_teams = [&](float* dst) {
    __syncthreads();
    for (int k = threadIdx.x; k < h; k += T::kBlock) {
      float v = sums[0][k];
#pragma unroll
      for (int j = 1; j < T::kTeams; ++j) v += sums[j][k];
      dst[int64_t(blockIdx.x) * h + k] = v;
    }
    __syncthreads();
  };
  if (has_f) add_teams(w.post);
  if (p.pre) {
#pragma unroll
    for (int e = 0; e < 8; ++e) sum[e] = acc_pre[e];
    add_teams(w.pre);
  }
}

// Second launch, 1024 lanes a workgroup, four kinds of work side by side:
//  - columns: dpre and dpost (and dgate with one gate row) from the workgroups' partial
//    rows, 32 columns by 32 parts;
//  - long: 128 columns of a sequence that goes on for more than kSpan teams behind its
//    first, 32 half-wavefronts along the teams.  Such a sequence contains the first row of
//    some kSpan-th team, and the first of these finds it;
//  - short: one wavefront for each team t and 256 columns, for the sequence, if any,
//    that starts in t and ends at most kSpan teams later;
//  - empty: zeros for the sequences without rows.
// (With a list of the sequences for every 32 columns: 79 us for 1,286 sequences of 1 to
// 51 tokens, hidden 1,152; long ones one after another in 32 columns: 65 us for 32,768
// rows of hidden 4,096 in 42 sequences.)
constexpr int kCols = 32, kParts = 32, kSpan = 32, kLong = 128, kWaves = 16, kWide = 256;
constexpr int kRuns = 8;  // loads in flight along a column (4 along a short sequence's)

struct ReduceShape {
  int chunks, strips, wide, long_blocks, short_blocks, empty_blocks;  // 2 * chunks workgroups, then long_blocks, ...
};
inline ReduceShape reduce_shape(const BwdShape& b, int hidden, int n_seqs) {
  ReduceShape r{(hidden + kCols - 1) / kCols, (hidden + kLong - 1) / kLong, (hidden + kWide - 1) / kWide, 0, 0, 0};
  if (n_seqs == 0) return r;
  if (b.teams > kSpan) r.long_blocks = int((b.teams + kSpan - 1) / kSpan) * r.strips;
  r.short_blocks = int((b.teams * r.wide + kWaves - 1) / kWaves);
  r.empty_blocks = (n_seqs + 1023) / 1024;
  return r;
}

__global__ __launch_bounds__(1024) void gated_norm_reduce_kernel(GatedNormBwd p, BwdParts w, ReduceShape g,
                                                                 int blocks) {
  __shared__ float part_sum[kParts][kCols];
  __shared__ f32x4 long_sum[kParts][kLong / 4];
  const int h = p.hidden, R = w.team_rows, wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  auto put = [&](float* dst, float v) { *dst = p.accumulate ? *dst + v : v; };
  const __bf16 *post = static_cast<const __bf16*>(p.post), *gate = static_cast<const __bf16*>(p.gate);
  int role = blockIdx.x;
  if (role < 2 * g.chunks) {
    const int part = threadIdx.x / kCols, col = threadIdx.x % kCols, c = (role >> 1) * kCols + col;
    const bool pre = (role & 1) == 0;
    if (pre ? !p.dpre : !p.dpost && (p.cu || !p.dgate)) return;
    const float* src = pre ? w.pre : w.post;
    float run[kRuns] = {};
    if (c < h) {
      int b = part;
      for (; b + (kRuns - 1) * kParts < blocks; b += kRuns * kParts)
#pragma unroll
        for (int j = 0; j < kRuns; ++j) run[j] += src[int64_t(b + j * kParts) * h + c];
      for (; b < blocks; b += kParts) run[0] += src[int64_t(b) * h + c];
    }
#pragma unroll
    for (int j = kRuns / 2; j > 0; j /= 2)
#pragma unroll
      for (int i = 0; i < j; ++i) run[i] += run[i + j];
    part_sum[part][col] = run[0];
    __syncthreads();
    if (part > 0 || c >= h) return;
    float t = 0.f;
#pragma unroll
    for (int q = 0; q < kParts; ++q) t += part_sum[q][col];
    if (pre) return put(p.dpre + c, t);
    if (p.dpost) put(p.dpost + c, p.cu || !gate ? t : t * float(gate[c]));
    if (!p.cu && p.dgate) put(p.dgate + c, post ? t * float(post[c]) : t);
    return;
  }
  role -= 2 * g.chunks;
  const int64_t rows = rows_of(p.rows, p.cu, p.n_seqs);
  // Sequence s as first team, last team and the partial row of the first.
  struct Span {
    int64_t t0, t1, head;
  };
  auto span = [&](int s) {
    const int64_t lo = offset_of(p.cu, s), hi = min(int64_t(offset_of(p.cu, s + 1)), rows);
    Span q{lo / R, (hi - 1) / R, 0};
    q.head = 2 * q.t0 + (lo % R != 0 ? 1 : 0);
    return q;
  };
  auto partial = [&](int64_t row, int c) { return *reinterpret_cast<const f32x4*>(w.seg + row * h + c); };
  // Partial rows 2 k, k = k0, k0 + step, ... <= k1.
  auto along = [&](auto in_flight, int64_t k0, int64_t k1, int64_t step, int c) {
    constexpr int kN = decltype(in_flight)::value;
    f32x4 v[kN] = {};
    int64_t k = k0;
    for (; k + (kN - 1) * step <= k1; k += kN * step)
#pragma unroll
      for (int j = 0; j < kN; ++j) v[j] += partial(2 * (k + j * step), c);
    for (; k <= k1; k += step) v[0] += partial(2 * k, c);
#pragma unroll
    for (int j = kN / 2; j > 0; j /= 2)
#pragma unroll
      for (int i = 0; i < j; ++i) v[i] += v[i + j];
    return v[0];
  };
  auto finish = [&](int s, int c, f32x4 v) {
#pragma unroll
    for (int e = 0; e < 4; ++e) put(p.dgate + int64_t(s) * h + c + e, post ? v[e] * float(post[c + e]) : v[e]);
  };
  if (role < g.long_blocks) {
    const int64_t t = int64_t(role / g.strips) * kSpan;
    const int part = threadIdx.x / (kLong / 4), col = threadIdx.x % (kLong / 4), c = role % g.strips * kLong + 4 * col;
    if (t * R >= rows) return;
    const int s = min(sequence_of<64>(p.cu, p.n_seqs, row_t(t * R)), p.n_seqs - 1);
    const Span q = span(s);
    const int64_t from = q.head - q.t0;  // the first team whose first row it contains
    if (q.t1 - q.t0 <= kSpan || t < from || t >= from + kSpan) return;
    long_sum[part][col] =
        c < h ? along(std::integral_constant<int, kRuns>{}, q.t0 + 1 + part, q.t1, kParts, c) : f32x4{};
    __syncthreads();
    if (part > 0 || c >= h) return;
    f32x4 v = partial(q.head, c);
#pragma unroll
    for (int k = 0; k < kParts; ++k) v += long_sum[k][col];
    finish(s, c, v);
    return;
  }
  role -= g.long_blocks;
  if (role < g.short_blocks) {
    const int64_t unit = int64_t(role) * kWaves + wave, t = unit / g.wide, next = (t + 1) * R;
    if (next >= rows) return;  // nothing goes on behind team t
    const int s = min(sequence_of<64>(p.cu, p.n_seqs, row_t(next)), p.n_seqs - 1);
    const Span q = span(s);
    if (q.t0 != t || q.t1 == t || q.t1 - t > kSpan) return;
    const int c = int(unit % g.wide) * kWide + 4 * lane;
    if (c < h) finish(s, c, partial(q.head, c) + along(std::integral_constant<int, 4>{}, t + 1, q.t1, 1, c));
    return;
  }
  role -= g.short_blocks;
  if (p.accumulate) return;
  const int64_t s = int64_t(role) * 1024 + threadIdx.x;
  bool none = false;
  if (s < p.n_seqs) none = min(int64_t(offset_of(p.cu, int(s) + 1)), rows) <= int64_t(offset_of(p.cu, int(s)));
  for (uint64_t left = __ballot(none); left; left &= left - 1) {
    float* dst = p.dgate + (s - lane + __ffsll(static_cast<unsigned long long>(left)) - 1) * h;
    for (int c = lane; c < h; c += 64) dst[c] = 0.f;
  }
}

inline size_t up256(size_t n) { return (n + 255) / 256 * 256; }

// Calls f with the team width of `lanes` as a compile-time constant.
template <class F>
void with_lanes(int lanes, F f) {
  switch (lanes) {
    case 8: return f(std::integral_constant<int, 8>{});
    case 16: return f(std::integral_constant<int, 16>{});
    case 32: return f(std::integral_constant<int, 32>{});
    case 64: return f(std::integral_constant<int, 64>{});
    case 128: return f(std::integral_constant<int, 128>{});
    case 192: return f(std::integral_constant<int, 192>{});
    case 256: return f(std::integral_constant<int, 256>{});
    case 320: return f(std::integral_constant<int, 320>{});
    case 384: return f(std::integral_constant<int, 384>{});
    case 448: return f(std::integral_constant<int, 448>{});
    default: return f(std::integral_constant<int, 512>{});
  }
}

// Rows of a team in the forward, from one on: 131,072 rows of hidden 1,152 at 1 / 2 / 4 /
// 8 / 16 rows 433 / 353 / 334 / 336 / 352 us (with the unpack of f's checkpoint), 16,384
// of 4,096 104 / 96 / 99 / 99 / 99.
constexpr int kFwdRowsMax = 4, kFwdTeams = 4096;

}  // namespace

hipError_t launch_gated_norm_fwd(const GatedNormFwd& p, hipStream_t s) {
  if (p.rows == 0) return hipSuccess;
  const int64_t want = p.rows / kFwdTeams;
  int team_rows = int(want < 1 ? 1 : want > kFwdRowsMax ? kFwdRowsMax : want);
  with_lanes(team_lanes(p.hidden), [&](auto tl) {
    constexpr int TL = decltype(tl)::value;
    auto blocks = [&] {
      const int64_t per_block = int64_t(Team<TL>::kTeams) * team_rows;
      return (p.rows + per_block - 1) / per_block;
    };
    // (a launch holds fewer than 2^32 lanes: the last rows below 2^31 at a width of 64 or less)
    while (blocks() * Team<TL>::kBlock >= int64_t(1) << 32) team_rows *= 2;
    const dim3 grid{unsigned(blocks())}, block{unsigned(Team<TL>::kBlock)};
    if (!p.keep_f && !p.keep_out)
      hipLaunchKernelGGL((gated_norm_fwd_kernel<TL, DCP_ACT_BF16>), grid, block, 0, s, p, team_rows);
    else if (p.format == DCP_ACT_INT8)
      hipLaunchKernelGGL((gated_norm_fwd_kernel<TL, DCP_ACT_INT8>), grid, block, 0, s, p, team_rows);
    else
      hipLaunchKernelGGL((gated_norm_fwd_kernel<TL, DCP_ACT_E4M3>), grid, block, 0, s, p, team_rows);
  });
  return hipGetLastError();
}

size_t gated_norm_bwd_workspace(int64_t rows, int hidden, int n_seqs) {
  const BwdShape b = bwd_shape(rows, hidden, n_seqs);
  return 2 * up256(4 * size_t(b.blocks) * size_t(hidden)) + (n_seqs ? up256(8 * size_t(b.teams) * size_t(hidden)) : 0);
}

hipError_t launch_gated_norm_bwd(const GatedNormBwd& p, void* workspace, hipStream_t s) {
  const BwdShape b = bwd_shape(p.rows, p.hidden, p.cu ? p.n_seqs : 0);
  char* ws = static_cast<char*>(workspace);
  const size_t part = up256(4 * size_t(b.blocks) * size_t(p.hidden));
  const BwdParts w{reinterpret_cast<float*>(ws), reinterpret_cast<float*>(ws + part),
                   reinterpret_cast<float*>(ws + 2 * part), b.team_rows};
  if (b.blocks > 0) {
    with_lanes(b.lanes, [&](auto tl) {
      constexpr int TL = decltype(tl)::value;
      auto launch = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, dim3(unsigned(b.blocks)), dim3(Team<TL>::kBlock), 0, s, p, w);
      };
      if (p.format == DCP_ACT_BF16)
        p.dy_f32 ? launch(gated_norm_bwd_kernel<TL, DCP_ACT_BF16, true>)
                 : launch(gated_norm_bwd_kernel<TL, DCP_ACT_BF16, false>);
      else if (p.format == DCP_ACT_INT8)
        p.dy_f32 ? launch(gated_norm_bwd_kernel<TL, DCP_ACT_INT8, true>)
                 : launch(gated_norm_bwd_kernel<TL, DCP_ACT_INT8, false>);
      else
        p.dy_f32 ? launch(gated_norm_bwd_kernel<TL, DCP_ACT_E4M3, true>)
                 : launch(gated_norm_bwd_kernel<TL, DCP_ACT_E4M3, false>);
    });
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (!p.dpre && !p.dpost && !p.dgate) return hipSuccess;
  const ReduceShape g = reduce_shape(b, p.hidden, p.cu ? p.n_seqs : 0);
  const unsigned grid = unsigned(2 * g.chunks + g.long_blocks + g.short_blocks + g.empty_blocks);
  hipLaunchKernelGGL(gated_norm_reduce_kernel, dim3(grid), dim3(1024), 0, s, p, w, g, int(b.blocks));
  return hipGetLastError();
}

}  // namespace dcp
