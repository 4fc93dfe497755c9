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
#include "act8.h"
#include "block_launch.h"

namespace dcp {
namespace {

// A team of W wavefronts owns a row: lane l of the team has columns 8 l + 512 W c,
// c < NC (the last chunk may be partly idle), so one access is 16 bytes a lane.
// Teams take kFwdRows consecutive rows (so that gains, gate and the place in
// cu_seqlens are fetched once); a workgroup is 4 wavefronts.
constexpr int kFwdRows = 8;

template <int W>
__device__ __forceinline__ float team_total(float v, float* red) {
  v = wave_total(v);
  if constexpr (W > 1) {
    const int wave = threadIdx.x >> 6;
    __syncthreads();  // (the last sum's readers are done)
    red[wave] = v;
    __syncthreads();
    const int first = wave / W * W;
    v = red[first];
#pragma unroll
    for (int w = 1; w < W; ++w) v += red[first + w];
  }
  return v;
}

// The sequence of `row`: the last index s <= n with cu[s] <= row (n: the row lies
// behind the last sequence).  64 probes a step, so three steps reach 2^18
// sequences.  Whatever cu holds, s stays in [0, n].
__device__ __forceinline__ int sequence_of(const int32_t* cu, int n, int64_t row) {
  const int lane = threadIdx.x & 63;
  int lo = 0, len = n + 1;
  while (len > 1) {
    const int step = (len + 63) >> 6, at = lane * step;
    const bool below = at < len && int64_t(cu[lo + at]) <= row;
    const int c = max(int(__popcll(__ballot(below))) - 1, 0);
    lo += c * step;
    len = min(step, len - c * step);
    if (len < 1) len = 1;  // (only if cu is not sorted)
  }
  return min(lo, n);
}

// Follows consecutive rows through cu_seqlens.
struct Walk {
  const int32_t* cu;
  int n, s;
  int64_t end;  // first row behind sequence s
  __device__ __forceinline__ void start(const int32_t* c, int n_seqs, int64_t row) {
    cu = c;
    n = n_seqs;
    s = __builtin_amdgcn_readfirstlane(min(sequence_of(c, n_seqs, row), n_seqs - 1));
    end = cu[s + 1];
  }
  // whether `row` lies in a later sequence than the row before
  __device__ __forceinline__ bool step(int64_t row) {
    if (row < end) return false;
    while (row >= end && s < n - 1) end = cu[++s + 1];
    return true;
  }
};

template <int FMT>
__device__ __forceinline__ void keep8(void* codes, void* scales, bf16x8 v, int64_t row, int c, int h, int groups) {
  const uint32_t byte = scale_byte<FMT>(group_top(top_bits(v)));
  if (c < h) *reinterpret_cast<u32x2*>(static_cast<uint8_t*>(codes) + row * h + c) = encode8<FMT>(v, byte);
  if (c < h && (c & 31) == 0) static_cast<uint8_t*>(scales)[row * groups + (c >> 5)] = uint8_t(byte);
}

// KEEP: format of the checkpoints (DCP_ACT_BF16: none).  y, its statistics and the
// checkpoint of out come from out in fp32 and from out as stored, respectively.
template <int W, int NC, int KEEP>
__global__ __launch_bounds__(256) void gated_norm_fwd_kernel(GatedNormFwd p) {
  __shared__ float red[4];
  const int lane = threadIdx.x % (64 * W), team = threadIdx.x / (64 * W);
  const int h = p.hidden, groups = (h + kActGroup - 1) / kActGroup;
  const int64_t first = (int64_t(blockIdx.x) * (4 / W) + team) * kFwdRows;
  int64_t rows = p.rows;
  if (p.cu) rows = min(rows, int64_t(p.cu[p.n_seqs]));
  if (W == 1 && first >= rows) return;
  const __bf16 *x = static_cast<const __bf16*>(p.x), *f = static_cast<const __bf16*>(p.f);
  const __bf16 *gate = static_cast<const __bf16*>(p.gate);
  bf16x8 post[NC], pre[NC], gt[NC];
  auto row_of = [&](const __bf16* g, bf16x8 (&v)[NC]) {
#pragma unroll
    for (int k = 0; k < NC; ++k) {
      const int c = 8 * lane + 512 * W * k;
      if (c < h && g) {
        v[k] = *reinterpret_cast<const bf16x8*>(g + c);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[k][e] = __bf16(1.f);
      }
    }
  };
  row_of(static_cast<const __bf16*>(p.post), post);
  row_of(static_cast<const __bf16*>(p.pre), pre);
  Walk walk;
  if (p.cu && first < rows) {
    walk.start(p.cu, p.n_seqs, first);
    row_of(gate + int64_t(walk.s) * h, gt);
  } else {
    row_of(gate, gt);
  }
  for (int i = 0; i < kFwdRows; ++i) {
    const int64_t row = first + i;
    const bool live = row < rows;
    if (W == 1 && !live) break;
    if (p.cu && i > 0 && live && walk.step(row)) row_of(gate + int64_t(walk.s) * h, gt);
    bf16x8 xv[NC], fv[NC];
#pragma unroll
    for (int k = 0; k < NC; ++k) {
      const int c = 8 * lane + 512 * W * k;
      xv[k] = fv[k] = bf16x8{};
      if (live && c < h) {
        fv[k] = *reinterpret_cast<const bf16x8*>(f + row * h + c);
        xv[k] = *reinterpret_cast<const bf16x8*>(x + row * h + c);
      }
    }
    float rf = 1.f;
    if (p.post) {
      float ss = 0.f;
#pragma unroll
      for (int k = 0; k < NC; ++k)
#pragma unroll
        for (int e = 0; e < 8; ++e) ss += float(fv[k][e]) * float(fv[k][e]);
      rf = rsqrtf(team_total<W>(ss, red) / float(h) + p.eps);
      if (live && lane == 0) p.rstd_f[row] = rf;
    }
    float o[NC][8], ss = 0.f;
#pragma unroll
    for (int k = 0; k < NC; ++k) {
      const int c = 8 * lane + 512 * W * k;
      bf16x8 ov;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        o[k][e] = p.alpha * float(xv[k][e]) + float(gt[k][e]) * (float(fv[k][e]) * rf * float(post[k][e]));
        ss += o[k][e] * o[k][e];
        ov[e] = __bf16(o[k][e]);
      }
      if (live && c < h) *reinterpret_cast<bf16x8*>(static_cast<__bf16*>(p.out) + row * h + c) = ov;
      if constexpr (KEEP != DCP_ACT_BF16) {
        if (live && p.keep_f) keep8<KEEP>(p.keep_f, p.keep_f_scales, fv[k], row, c, h, groups);
        if (live && p.keep_out) keep8<KEEP>(p.keep_out, p.keep_out_scales, ov, row, c, h, groups);
      }
    }
    if (p.pre) {
      const float ro = rsqrtf(team_total<W>(ss, red) / float(h) + p.eps);
      if (live && lane == 0) p.rstd_out[row] = ro;
#pragma unroll
      for (int k = 0; k < NC; ++k) {
        const int c = 8 * lane + 512 * W * k;
        bf16x8 yv;
#pragma unroll
        for (int e = 0; e < 8; ++e) yv[e] = __bf16(o[k][e] * ro * float(pre[k][e]));
        if (live && c < h) *reinterpret_cast<bf16x8*>(static_cast<__bf16*>(p.y) + row * h + c) = yv;
      }
    }
  }
}

// Backward.  Teams take `team_rows` consecutive rows and keep the column sums of
// G o fh and dy o oh in registers: one partial row a workgroup for dpost (or A with
// one gate row) and dpre, and, with a gate for each sequence, A_s either straight
// into dgate (a sequence whose rows all lie in one team) or as a partial row of the
// team: slot 0 for the sequence that its first row belongs to, slot 1 for one that
// starts inside and goes on.  A second launch adds the partial rows in a fixed
// order, so results are bitwise reproducible.
constexpr int kBwdRowsMin = 4, kBwdRowsMax = 64, kBwdTeams = 4096;

struct BwdShape {
  int team_rows, waves;  // rows of a team, wavefronts of a team
  int64_t teams, blocks;
};
inline int team_waves(int hidden) { return hidden <= 1536 ? 1 : hidden <= 3072 ? 2 : 4; }
inline BwdShape bwd_shape(int64_t rows, int hidden) {
  BwdShape s;
  s.waves = team_waves(hidden);
  const int64_t want = (rows + kBwdTeams / s.waves - 1) / (kBwdTeams / s.waves);
  s.team_rows = int(want < kBwdRowsMin ? kBwdRowsMin : want > kBwdRowsMax ? kBwdRowsMax : want);
  s.teams = (rows + s.team_rows - 1) / s.team_rows;
  s.blocks = (s.teams + 4 / s.waves - 1) / (4 / s.waves);
  s.teams = s.blocks * (4 / s.waves);
  return s;
}

struct BwdParts {
  float *pre, *post;  // [blocks][hidden] each
  float* seg;         // [teams][2][hidden]
  int team_rows;
};

template <int W, int NC, int FMT, bool DY32>
__global__ __launch_bounds__(256) void gated_norm_bwd_kernel(GatedNormBwd p, BwdParts w) {
  __shared__ float red[4];
  extern __shared__ float sums[];  // [4 / W teams][h]
  constexpr int kTeams = 4 / W;
  const int lane = threadIdx.x % (64 * W), team = threadIdx.x / (64 * W);
  const int h = p.hidden, groups = (h + kActGroup - 1) / kActGroup;
  const int64_t first = (int64_t(blockIdx.x) * kTeams + team) * w.team_rows;
  int64_t rows = p.rows;
  if (p.cu) rows = min(rows, int64_t(p.cu[p.n_seqs]));
  const bool has_f = p.post != nullptr || p.gate != nullptr;
  const __bf16 *dout = static_cast<const __bf16*>(p.dout), *gate = static_cast<const __bf16*>(p.gate);
  bf16x8 post[NC], pre[NC], gt[NC];
  float acc_pre[NC][8], acc_a[NC][8];
  auto row_of = [&](const __bf16* g, bf16x8 (&v)[NC]) {
#pragma unroll
    for (int k = 0; k < NC; ++k) {
      const int c = 8 * lane + 512 * W * k;
      if (c < h && g) {
        v[k] = *reinterpret_cast<const bf16x8*>(g + c);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[k][e] = __bf16(1.f);
      }
    }
  };
  row_of(static_cast<const __bf16*>(p.post), post);
  row_of(static_cast<const __bf16*>(p.pre), pre);
#pragma unroll
  for (int k = 0; k < NC; ++k)
#pragma unroll
    for (int e = 0; e < 8; ++e) acc_pre[k][e] = acc_a[k][e] = 0.f;
  float* mine = sums + team * h;
  Walk walk;
  walk.s = 0;
  walk.end = 0;
  int64_t from = first;  // first row of the team's current sequence
  if (p.cu && first < rows) {
    walk.start(p.cu, p.n_seqs, first);
    row_of(gate + int64_t(walk.s) * h, gt);
  } else {
    row_of(p.cu ? nullptr : gate, gt);
  }
#pragma unroll
  for (int k = 0; k < NC; ++k) {
    const int c = 8 * lane + 512 * W * k;
    if (c < h)
#pragma unroll
      for (int e = 0; e < 8; ++e) mine[c + e] = 0.f;
  }
  // The team's sum of G o fh over rows [from, to) of sequence s leaves the registers.
  auto flush = [&](int s, int64_t from_, int64_t to, int64_t seq_end) {
    const bool starts = int64_t(p.cu[s]) >= first, ends = to >= min(seq_end, rows);
    float* dst = starts && ends ? p.dgate + int64_t(s) * h
                                : w.seg + ((int64_t(blockIdx.x) * kTeams + team) * 2 + (from_ > first ? 1 : 0)) * h;
#pragma unroll
    for (int k = 0; k < NC; ++k) {
      const int c = 8 * lane + 512 * W * k;
      if (c < h)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          float v = acc_a[k][e];
          mine[c + e] += float(gt[k][e]) * v;
          if (starts && ends) {
            v *= float(post[k][e]);
            if (p.accumulate) v += dst[c + e];
          }
          dst[c + e] = v;
          acc_a[k][e] = 0.f;
        }
    }
  };
  for (int i = 0; i < w.team_rows; ++i) {
    const int64_t row = first + i;
    const bool live = row < rows;
    if (W == 1 && !live) break;
    if (p.cu && i > 0 && live) {
      const int s = walk.s;
      const int64_t e = walk.end;
      if (walk.step(row)) {
        flush(s, from, row, e);
        from = row;
        row_of(gate + int64_t(walk.s) * h, gt);
      }
    }
    bf16x8 gv[NC];
    float d[NC][8];
    Held8<FMT> fv[NC], ov[NC];
    float rf = 1.f, ro = 0.f;
    if (live && p.post) rf = p.rstd_f[row];
    if (live && p.pre) ro = p.rstd_out[row];
#pragma unroll
    for (int k = 0; k < NC; ++k) {
      const int c = 8 * lane + 512 * W * k;
      gv[k] = bf16x8{};
      fv[k] = ov[k] = Held8<FMT>{};
#pragma unroll
      for (int e = 0; e < 8; ++e) d[k][e] = 0.f;
      if (live && c < h) {
        const int64_t at = row * h + c, grp = row * groups + (c >> 5);
        if (dout) gv[k] = *reinterpret_cast<const bf16x8*>(dout + at);
        if (p.pre) {
          ov[k].load(p.out, static_cast<const uint8_t*>(p.out_scales), at, grp);
          if constexpr (DY32) {
            const f32x4 a = *reinterpret_cast<const f32x4*>(static_cast<const float*>(p.dy) + at);
            const f32x4 b = *reinterpret_cast<const f32x4*>(static_cast<const float*>(p.dy) + at + 4);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              d[k][e] = a[e];
              d[k][e + 4] = b[e];
            }
          } else {
            const bf16x8 a = *reinterpret_cast<const bf16x8*>(static_cast<const __bf16*>(p.dy) + at);
#pragma unroll
            for (int e = 0; e < 8; ++e) d[k][e] = float(a[e]);
          }
        }
        if (has_f) fv[k].load(p.f, static_cast<const uint8_t*>(p.f_scales), at, grp);
      }
    }
    float G[NC][8];
#pragma unroll
    for (int k = 0; k < NC; ++k)
#pragma unroll
      for (int e = 0; e < 8; ++e) G[k][e] = float(gv[k][e]);
    if (p.pre) {
      float dot = 0.f;
      float oh[NC][8];
#pragma unroll
      for (int k = 0; k < NC; ++k) {
        const int c = 8 * lane + 512 * W * k;
        ov[k].get(oh[k]);
        bf16x8 yv;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          oh[k][e] = c < h ? oh[k][e] * ro : 0.f;
          acc_pre[k][e] += d[k][e] * oh[k][e];
          d[k][e] *= float(pre[k][e]);
          dot += d[k][e] * oh[k][e];
          yv[e] = __bf16(oh[k][e] * float(pre[k][e]));
        }
        if (live && p.y && c < h) *reinterpret_cast<bf16x8*>(static_cast<__bf16*>(p.y) + row * h + c) = yv;
      }
      const float mean = team_total<W>(dot, red) / float(h);
#pragma unroll
      for (int k = 0; k < NC; ++k)
#pragma unroll
        for (int e = 0; e < 8; ++e) G[k][e] += ro * (d[k][e] - oh[k][e] * mean);
    }
    if (p.dx) {
#pragma unroll
      for (int k = 0; k < NC; ++k) {
        const int c = 8 * lane + 512 * W * k;
        bf16x8 v;
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = __bf16(p.alpha * G[k][e]);
        if (live && c < h) *reinterpret_cast<bf16x8*>(static_cast<__bf16*>(p.dx) + row * h + c) = v;
      }
    }
    float dot = 0.f;
    float fh[NC][8];
#pragma unroll
    for (int k = 0; k < NC; ++k) {
      const int c = 8 * lane + 512 * W * k;
      fv[k].get(fh[k]);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        fh[k][e] = c < h ? fh[k][e] * rf : 0.f;
        acc_a[k][e] += G[k][e] * fh[k][e];
        G[k][e] *= float(gt[k][e]) * float(post[k][e]);
        dot += G[k][e] * fh[k][e];
      }
    }
    float mean = 0.f;
    if (p.post) mean = team_total<W>(dot, red) / float(h);
#pragma unroll
    for (int k = 0; k < NC; ++k) {
      const int c = 8 * lane + 512 * W * k;
      bf16x8 v;
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = __bf16(rf * (G[k][e] - fh[k][e] * mean));
      if (live && p.df && c < h) *reinterpret_cast<bf16x8*>(static_cast<__bf16*>(p.df) + row * h + c) = v;
    }
  }
  if (p.cu) {
    if (first < rows) flush(walk.s, from, min(first + w.team_rows, rows), walk.end);
  } else {
#pragma unroll
    for (int k = 0; k < NC; ++k) {
      const int c = 8 * lane + 512 * W * k;
      if (c < h)
#pragma unroll
        for (int e = 0; e < 8; ++e) mine[c + e] = acc_a[k][e];
    }
  }
  auto add_teams = [&](float* dst) {
    __syncthreads();
    for (int c = threadIdx.x; c < h; c += 256) {
      float t = sums[c];
#pragma unroll
      for (int j = 1; j < kTeams; ++j) t += sums[j * h + c];
      dst[int64_t(blockIdx.x) * h + c] = t;
    }
    __syncthreads();
  };
  if (has_f) add_teams(w.post);
  if (p.pre) {
    if (!has_f) __syncthreads();
#pragma unroll
    for (int k = 0; k < NC; ++k) {
      const int c = 8 * lane + 512 * W * k;
      if (c < h)
#pragma unroll
        for (int e = 0; e < 8; ++e) mine[c + e] = acc_pre[k][e];
    }
    add_teams(w.pre);
  }
}

// Second launch: 32 columns by 32 half-wavefronts a workgroup.  Role 0 adds the
// workgroups' partial rows of dpre, role 1 those of dpost (and dgate with one gate
// row); the other roles take sequences, `zs` workgroups along them: each lists those
// of its share that no team finished, then short ones (up to 32 teams) go one to a
// half-wavefront, long ones one after another to the whole workgroup.
constexpr int kCols = 32, kParts = 32, kShareMax = 1024, kSeqBlocks = 64;
__global__ __launch_bounds__(kCols* kParts) void gated_norm_reduce_kernel(GatedNormBwd p, BwdParts w, int blocks, int zs,
                                                                          int share) {
  __shared__ float part_sum[kParts][kCols];
  __shared__ int list[kShareMax], count;
  const int h = p.hidden, lane = threadIdx.x % kCols, part = threadIdx.x / kCols;
  const int chunks = (h + kCols - 1) / kCols, role = blockIdx.x / chunks;
  const int c = (blockIdx.x % chunks) * kCols + lane;
  // sum of `n` rows of h floats from `src`, stride `stride` rows, over the workgroup
  auto column = [&](const float* src, int64_t stride, int n) {
    float s4[4] = {0.f, 0.f, 0.f, 0.f};
    if (c < h) {
      int b = part;
      for (; b + 3 * kParts < n; b += 4 * kParts)
#pragma unroll
        for (int j = 0; j < 4; ++j) s4[j] += src[(b + j * kParts) * stride * h + c];
      for (int j = 0; b < n; b += kParts, ++j) s4[j & 3] += src[b * stride * h + c];
    }
    __syncthreads();
    part_sum[part][lane] = (s4[0] + s4[1]) + (s4[2] + s4[3]);
    __syncthreads();
    float t = 0.f;
    if (part == 0) {
#pragma unroll
      for (int q = 0; q < kParts; ++q) t += part_sum[q][lane];
    }
    return t;
  };
  auto put = [&](float* dst, float v) { *dst = p.accumulate ? *dst + v : v; };
  const __bf16 *post = static_cast<const __bf16*>(p.post), *gate = static_cast<const __bf16*>(p.gate);
  if (role == 0) {
    if (!p.dpre) return;
    const float t = column(w.pre, 1, blocks);
    if (part == 0 && c < h) put(p.dpre + c, t);
    return;
  }
  if (role == 1) {
    if (!p.dpost && (p.cu || !p.dgate)) return;
    const float t = column(w.post, 1, blocks);
    if (part == 0 && c < h) {
      if (p.dpost) put(p.dpost + c, p.cu || !gate ? t : t * float(gate[c]));
      if (!p.cu && p.dgate) put(p.dgate + c, post ? t * float(post[c]) : t);
    }
    return;
  }
  const int z = role - 2, R = w.team_rows;
  const int64_t rows = min(p.rows, int64_t(p.cu[p.n_seqs]));
  const float pc = post && c < h ? float(post[c]) : 1.f;
  for (int64_t base = int64_t(z) * share; base < p.n_seqs; base += int64_t(zs) * share) {
    __syncthreads();
    if (threadIdx.x == 0) count = 0;
    __syncthreads();
    const int64_t s = base + threadIdx.x;
    bool listed = false;
    if (int(threadIdx.x) < share && s < p.n_seqs) {
      const int64_t lo = max(int64_t(p.cu[s]), int64_t(0)), hi = min(int64_t(p.cu[s + 1]), rows);
      if (hi <= lo) {
        listed = !p.accumulate;  // no rows: the gradient is zero
      } else {
        listed = lo / R != (hi - 1) / R;
      }
    }
    if (listed) list[atomicAdd(&count, 1)] = int(s);  // (the order does not reach the results)
    __syncthreads();
    const int n = count;
    for (int i = part; i < n; i += kParts) {
      const int q = list[i];
      const int64_t lo = max(int64_t(p.cu[q]), int64_t(0)), hi = min(int64_t(p.cu[q + 1]), rows);
      const int64_t t0 = lo / R, t1 = hi > lo ? (hi - 1) / R : t0 - 1;
      if (t1 - t0 >= kParts || c >= h) continue;
      float v = 0.f;
      for (int64_t t = t0; t <= t1; ++t) v += w.seg[(2 * t + (t == t0 && lo % R != 0 ? 1 : 0)) * h + c];
      put(p.dgate + int64_t(q) * h + c, v * pc);
    }
    for (int i = 0; i < n; ++i) {
      const int q = list[i];
      const int64_t lo = max(int64_t(p.cu[q]), int64_t(0)), hi = min(int64_t(p.cu[q + 1]), rows);
      const int64_t t0 = lo / R, t1 = hi > lo ? (hi - 1) / R : t0 - 1;
      if (t1 - t0 < kParts) continue;
      // the first team's part may lie in slot 1, the others' lie in slot 0
      float v = column(w.seg + (2 * t0 + 2) * h, 2, int(t1 - t0));
      if (part == 0 && c < h) {
        v += w.seg[(2 * t0 + (lo % R != 0 ? 1 : 0)) * h + c];
        put(p.dgate + int64_t(q) * h + c, v * pc);
      }
    }
  }
}

inline size_t up256(size_t n) { return (n + 255) / 256 * 256; }

}  // namespace

hipError_t launch_gated_norm_fwd(const GatedNormFwd& p, hipStream_t s) {
  if (p.rows == 0) return hipSuccess;
  const int waves = team_waves(p.hidden), chunks = (p.hidden + 512 * waves - 1) / (512 * waves);
  const int64_t per_block = int64_t(4 / waves) * kFwdRows;
  const unsigned blocks = unsigned((p.rows + per_block - 1) / per_block);
  auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(blocks), dim3(256), 0, s, p); };
  auto keep = [&](auto bf16, auto int8, auto e4m3) {
    if (!p.keep_f && !p.keep_out) launch(bf16);
    else if (p.format == DCP_ACT_INT8) launch(int8);
    else launch(e4m3);
  };
#define DCP_FWD(W, NC)                                                                            \
  keep(gated_norm_fwd_kernel<W, NC, DCP_ACT_BF16>, gated_norm_fwd_kernel<W, NC, DCP_ACT_INT8>, \
       gated_norm_fwd_kernel<W, NC, DCP_ACT_E4M3>)
  if (waves == 4) DCP_FWD(4, 2);
  else if (waves == 2 && chunks == 3) DCP_FWD(2, 3);
  else if (waves == 2) DCP_FWD(2, 2);
  else if (chunks == 3) DCP_FWD(1, 3);
  else if (chunks == 2) DCP_FWD(1, 2);
  else DCP_FWD(1, 1);
#undef DCP_FWD
  return hipGetLastError();
}

size_t gated_norm_bwd_workspace(int64_t rows, int hidden, int n_seqs) {
  const BwdShape b = bwd_shape(rows, hidden);
  return 2 * up256(4 * size_t(b.blocks) * size_t(hidden)) + (n_seqs ? up256(8 * size_t(b.teams) * size_t(hidden)) : 0);
}

hipError_t launch_gated_norm_bwd(const GatedNormBwd& p, void* workspace, hipStream_t s) {
  const BwdShape b = bwd_shape(p.rows, p.hidden);
  char* ws = static_cast<char*>(workspace);
  const size_t part = up256(4 * size_t(b.blocks) * size_t(p.hidden));
  const BwdParts w{reinterpret_cast<float*>(ws), reinterpret_cast<float*>(ws + part), reinterpret_cast<float*>(ws + 2 * part),
                   b.team_rows};
  const int chunks = (p.hidden + 512 * b.waves - 1) / (512 * b.waves);
  const size_t lds = size_t(4 / b.waves) * p.hidden * sizeof(float);
  auto launch = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3(unsigned(b.blocks)), dim3(256), lds, s, p, w);
  };
  auto pick = [&](auto bf16, auto bf16_32, auto int8, auto int8_32, auto e4m3, auto e4m3_32) {
    if (p.format == DCP_ACT_BF16) p.dy_f32 ? launch(bf16_32) : launch(bf16);
    else if (p.format == DCP_ACT_INT8) p.dy_f32 ? launch(int8_32) : launch(int8);
    else p.dy_f32 ? launch(e4m3_32) : launch(e4m3);
  };
#define DCP_BWD(W, NC)                                                                                              \
  pick(gated_norm_bwd_kernel<W, NC, DCP_ACT_BF16, false>, gated_norm_bwd_kernel<W, NC, DCP_ACT_BF16, true>,       \
       gated_norm_bwd_kernel<W, NC, DCP_ACT_INT8, false>, gated_norm_bwd_kernel<W, NC, DCP_ACT_INT8, true>,       \
       gated_norm_bwd_kernel<W, NC, DCP_ACT_E4M3, false>, gated_norm_bwd_kernel<W, NC, DCP_ACT_E4M3, true>)
  if (b.blocks > 0) {
    if (b.waves == 4) DCP_BWD(4, 2);
    else if (b.waves == 2 && chunks == 3) DCP_BWD(2, 3);
    else if (b.waves == 2) DCP_BWD(2, 2);
    else if (chunks == 3) DCP_BWD(1, 3);
    else if (chunks == 2) DCP_BWD(1, 2);
    else DCP_BWD(1, 1);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
#undef DCP_BWD
  if (!p.dpre && !p.dpost && !p.dgate) return hipSuccess;
  int zs = 0, share = 1;
  if (p.cu) {
    zs = p.n_seqs < kSeqBlocks ? p.n_seqs : kSeqBlocks;
    share = (p.n_seqs + zs - 1) / zs;
    share = share < kShareMax ? share : kShareMax;
  }
  const unsigned cols = unsigned((p.hidden + kCols - 1) / kCols);
  hipLaunchKernelGGL(gated_norm_reduce_kernel, dim3(cols * unsigned(2 + zs)), dim3(kCols * kParts), 0, s, p, w,
                     int(b.blocks), zs, share);
  return hipGetLastError();
}

}  // namespace dcp
