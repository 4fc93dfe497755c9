// C ABI of the transformer block: the layer of layer_api.cpp with gated, normed
// joins, whose kept activations may be 8-bit checkpoints.
//   y1 = RMSNorm(x; norm1), q, k, v = y1 W{q,k,v}, o = attention(q, k, v),
//   f1 = o Wo,       h, y2 = join(x, f1; post1, gate1, norm2),
//   u  = y2 Wup,     a = GELU(u),
//   f2 = a Wdown,    out = join(h, f2; post2, gate2).
// Kept: q, k, v, o, h, u (and f1, f2 where a norm or gate needs them), the LSE and
// the row scales.  y1, y2 and a, which the layer keeps as well, come out of passes
// that the backward makes anyway (a from the activation's, y2 from the join's) or of
// one short one (y1).  The forward writes the checkpoints of f1, h and f2 in the
// joins' own passes, that of u in W_up's (where the kernel of layer_proj.hip forms
// it), and packs q, k and v in one launch; the backward's joins and activation read
// theirs in place, and one launch brings q, k and v back for the attention.
//
// The weight gradients of W_up and W_down multiply y2 and a as formed again: y2 from h as
// held (the forward's comes from h in fp32), a by gelu_and_slope (act8.h; the forward's by
// the gelu of layer_proj.hip or layer.hip: the same function in another order of fp32
// operations).  With a bf16 stash either is within a rounding to bf16, 2^-8 of itself, of
// what the forward multiplied, as far as any bf16 product's operands are known.
//
// o stays in bf16 in every stash.  The backward forms Delta = dO . o, which the sum over
// keys of P (dO . v) has to cancel: o's rounding does not (v's averages out over the
// keys), and the difference, the same for all keys of a query, becomes a part of dQ that
// grows as attention spreads.  Four blocks of random weights, hidden 1,152, sequences of
// 1,024 to 2,048 tokens, relative error of dWq in the last: int8 7.0 % with o in 8 bits,
// 1.7 % with o in bf16; e4m3 22.7 % and 5.2 %.  The stash grows by a tenth.  (v in bf16
// as well: 1.5 and 4.5 %; sequences of 1 to 51 tokens, o / o and v: 2.3 / 1.9 % in int8.)
#include <hip/hip_runtime.h>
#include <rocblas/rocblas.h>

#include <cmath>
#include <cstdint>

#include "block_launch.h"
#include "dcp_internal.h"
#include "layer_internal.h"
#include "layer_launch.h"

namespace dcp {
namespace {

// Where the kept activations are (q, k, v, o, f1, h, f2 [T, hidden], u [T, 4 hidden]:
// bf16, or, all but o, codes with scale bytes), byte offsets.
constexpr int kKept = 8;
enum { kQ, kK, kV, kO, kF1, kH, kF2, kU };
struct Kept {
  size_t data[kKept], scales[kKept], lse, rstd_f1, rstd_h, rstd_f2, total;
};

struct Block {
  Dims d;
  bool branch;  // a norm or a gate on the branches' outputs
  int format;
  int64_t cols(int i) const { return i == kU ? 4 * d.h : d.h; }
};

Kept kept_layout(const Block& b, int format) {
  Kept k{};
  size_t off = 0;
  auto take = [&](size_t bytes) {
    const size_t at = off;
    off += up(bytes);
    return at;
  };
  for (int i = 0; i < kKept; ++i) {
    if ((i == kF1 || i == kF2) && !b.branch) continue;
    const size_t n = size_t(b.d.T) * size_t(b.cols(i));
    const bool wide = format == DCP_ACT_BF16 || i == kO;
    k.data[i] = take(wide ? 2 * n : n);
    if (!wide) k.scales[i] = take(size_t(b.d.T) * size_t(act_groups(b.cols(i))));
  }
  k.lse = take(4 * size_t(b.d.H) * size_t(b.d.T));
  k.rstd_f1 = take(4 * size_t(b.d.T));
  k.rstd_h = take(4 * size_t(b.d.T));
  k.rstd_f2 = take(4 * size_t(b.d.T));
  k.total = off;
  return k;
}

int block_of(const dcp_block_desc* desc, Block* b) {
  if (!desc) return fail(DCP_ERR_INVALID, "block desc is null");
  DCP_TRY(dims_of(desc->layer, &b->d));
  if (desc->stash_format < DCP_ACT_BF16 || desc->stash_format > DCP_ACT_E4M3)
    return fail(DCP_ERR_INVALID, "unknown activation format %d", desc->stash_format);
  if (desc->post_norm & ~1) return fail(DCP_ERR_INVALID, "post_norm is 0 or 1");
  if (desc->gate < DCP_GATE_NONE || desc->gate > DCP_GATE_SEQUENCE)
    return fail(DCP_ERR_INVALID, "unknown gate %d", desc->gate);
  if ((desc->gate == DCP_GATE_SEQUENCE) != (desc->cu_seqlens != nullptr) ||
      reinterpret_cast<uintptr_t>(desc->cu_seqlens) % 4)
    return fail(DCP_ERR_INVALID, "cu_seqlens (device, 4-byte aligned) goes with a gate for each sequence");
  if (!std::isfinite(desc->residual_scale)) return fail(DCP_ERR_INVALID, "residual_scale must be finite");
  b->branch = desc->post_norm || desc->gate != DCP_GATE_NONE;
  b->format = desc->stash_format;
  return DCP_OK;
}

// Workspaces.  `act` holds the activations in bf16: the forward's where the stash does
// not, the backward's when it recomputes or reads q, k and v back from 8 bits.
struct FwdWs {
  size_t attn, act, y1, y2, a, rstd1, total;
};
struct BwdWs {
  size_t attn_f, attn_b, act, y1, y2, a, rstd1, out, da, f32, f2, dh, dx1, f1, dq, dk, dv, partial, join, total;
};

int fwd_ws(const dcp_block_desc* desc, const Block& b, FwdWs* w) {
  size_t na = 0;
  DCP_TRY(dcp_varlen_attn_fwd_workspace_size(desc->layer->attn, &na));
  const size_t Th = size_t(b.d.T) * size_t(b.d.h);
  size_t off = up(kGemmWorkspace);
  auto take = [&](size_t bytes) {
    const size_t at = off;
    off += up(bytes);
    return at;
  };
  w->attn = take(na);
  w->act = take(kept_layout(b, DCP_ACT_BF16).total + 4 * Th);  // (f1 and f2 also where they are not kept)
  w->y1 = take(2 * Th);
  w->y2 = take(2 * Th);
  w->a = take(8 * Th);
  w->rstd1 = take(4 * size_t(b.d.T));
  w->total = off;
  return DCP_OK;
}

int bwd_ws(const dcp_block_desc* desc, const Block& b, BwdWs* w) {
  size_t na = 0, nb = 0;
  DCP_TRY(dcp_varlen_attn_fwd_workspace_size(desc->layer->attn, &na));
  DCP_TRY(dcp_varlen_attn_bwd_workspace_size(desc->layer->attn, &nb));
  const size_t Th = size_t(b.d.T) * size_t(b.d.h);
  size_t off = up(kGemmWorkspace);
  auto take = [&](size_t bytes) {
    const size_t at = off;
    off += up(bytes);
    return at;
  };
  w->attn_f = take(na);
  w->attn_b = take(nb);
  w->act = take(kept_layout(b, DCP_ACT_BF16).total + 4 * Th);
  w->y1 = take(2 * Th);
  w->y2 = take(2 * Th);
  w->a = take(8 * Th);
  w->rstd1 = take(4 * size_t(b.d.T));
  w->out = take(2 * Th);
  w->da = take(8 * Th);   // dA, then dU in place
  w->f32 = take(4 * Th);  // dY2, dO (bf16), dY1
  w->f2 = take(2 * Th);   // gradient of f2
  w->dh = take(2 * Th);
  w->dx1 = take(2 * Th);
  w->f1 = take(2 * Th);  // gradient of f1
  w->dq = take(2 * Th);
  w->dk = take(2 * Th);
  w->dv = take(2 * Th);
  w->partial = take(4 * size_t(rmsnorm_bwd_blocks(b.d.T)) * size_t(b.d.h));
  w->join = take(gated_norm_bwd_workspace(b.d.T, int(b.d.h), desc->cu_seqlens ? desc->layer->attn->n_seqs : 0));
  w->total = off;
  return DCP_OK;
}

// One activation: where it is computed (bf16) and where the stash keeps it.
struct Acts {
  void* bf16[kKept];
  dcp_kept kept[kKept];  // data null: not kept apart from bf16
  float *lse, *rstd_f1, *rstd_h, *rstd_f2;
};

// W_up with GELU (and u's checkpoint) is one kernel of layer_proj.hip at every token
// count.  One kernel less the library's product and the passes behind it, us:
//   W_up, u in 8 bits  (128, 429) -18, (1152, 300) -4, (1152, 1000) -14, (1152, 4096)
//              -23, (1152, 16381) -71, (1024, 16384) -36, (1536, 8192) -37, (1792,
//              8192) +4, (4096, 4096) +47
//   W_up, u in bf16    -16, -3, -13, -9, -20, -18, -11, +20, +72 (the rule is the same, so
//              that the output does not depend on the stash)
inline bool fused_up(const Dims& d) { return d.h <= kProjHidden; }

// W_down^T with GELU' and GELU is one kernel where u is kept in bf16 (8 bits: (1152, 16381)
// +29, (1024, 4096) +20, (1536, 8192) +34) and the layer's rule for W_down^T with GELU'
// takes it, but for multiples of 256 from 1,024 on, which suit the library's tiles: there up
// to 12 M elements of a [T, hidden] matrix, and, where 192-wide tiles pad the width by a tenth
// (1,024), 1 M.  One kernel less the library's product and the pass, us, at 1,000 / 2,048 /
// 4,096 / 8,192 / 12,288 / 16,384 / 24,576 tokens:
//   256   -11 / -10 / -6 / -1 / -5 / -2 / -3        576   -6 / -1 / -4 / -19 / -2 / -11 / -6
//   768   -3 / -3 / -8 / -7 / -2 / +1 / -21         1,152 -0 / -0 / -16 / -8 / -12 / -33 / +3
//   1,408 -4 / -12 / +1 / -14 / -36 / +3 / +12      1,024 +1 / +2 / +8 / +9 / +14 / +15 / +29
//   1,280 -4 / -5 / -7 / -27 / +13 / +21 / +50      1,536 -2 / -5 / -3 / +7 / -27 / +13 / +24
inline bool fused_back(const Dims& d) {
  const bool padded = 10 * kProjTile * proj_tiles(d.h) > 11 * d.h;
  const bool library = d.h % 256 == 0 && d.h >= 1024 && d.T * d.h > int64_t(padded ? 1 : 12) << 20;
  return fused_gelu(d) && !library;
}

// Activations in bf16 at `base`, in kept_layout's places; f1 and f2, where it has
// none, behind them.
Acts acts_in(const Block& b, void* base) {
  const Kept k = kept_layout(b, DCP_ACT_BF16);
  const size_t Th = size_t(b.d.T) * size_t(b.d.h);
  Acts s{};
  for (int i = 0; i < kKept; ++i) s.bf16[i] = at(base, k.data[i]);
  if (!b.branch) {
    s.bf16[kF1] = at(base, k.total);
    s.bf16[kF2] = at(base, k.total + 2 * Th);
  }
  s.lse = reinterpret_cast<float*>(at(base, k.lse));
  s.rstd_f1 = reinterpret_cast<float*>(at(base, k.rstd_f1));
  s.rstd_h = reinterpret_cast<float*>(at(base, k.rstd_h));
  s.rstd_f2 = reinterpret_cast<float*>(at(base, k.rstd_f2));
  return s;
}

// The forward's activations with a stash (or none): bf16 in the stash itself, or, all
// but o, in the workspace with 8-bit checkpoints in the stash.
Acts forward_acts(const Block& b, void* stash, void* act) {
  if (!stash) return acts_in(b, act);
  if (b.format == DCP_ACT_BF16) {
    Acts s = acts_in(b, stash);
    if (!b.branch) {
      const Acts t = acts_in(b, act);
      s.bf16[kF1] = t.bf16[kF1];
      s.bf16[kF2] = t.bf16[kF2];
    }
    return s;
  }
  Acts s = acts_in(b, act);
  const Kept k = kept_layout(b, b.format);
  for (int i = 0; i < kKept; ++i)
    if (i != kO && ((i != kF1 && i != kF2) || b.branch)) s.kept[i] = {at(stash, k.data[i]), at(stash, k.scales[i])};
  s.bf16[kO] = at(stash, k.data[kO]);
  s.lse = reinterpret_cast<float*>(at(stash, k.lse));
  s.rstd_f1 = reinterpret_cast<float*>(at(stash, k.rstd_f1));
  s.rstd_h = reinterpret_cast<float*>(at(stash, k.rstd_h));
  s.rstd_f2 = reinterpret_cast<float*>(at(stash, k.rstd_f2));
  return s;
}

// The gates' offsets, shared by both joins.
int n_gates(const dcp_block_desc* desc) { return desc->cu_seqlens ? desc->layer->attn->n_seqs : 0; }

int forward(const dcp_block_desc* desc, const Block& b, const dcp_block_weights* w, const void* x, void* out,
            const Acts& s, void* y1, void* y2, void* a, float* rstd1, void* attn_ws, size_t attn_ws_bytes,
            rocblas_handle hd, hipStream_t st) {
  const Dims& d = b.d;
  const int64_t T = d.T, h = d.h;
  const dcp_layer_weights& lw = w->layer;
  DCP_HIP(launch_rmsnorm_fwd(x, lw.norm1, y1, rstd1, T, int(h), desc->layer->eps, st));
  if (fused_qkv(d)) {
    const Proj p{{y1, y1, y1}, {lw.wq, lw.wk, lw.wv}, {s.bf16[kQ], s.bf16[kK], s.bf16[kV]}, nullptr, nullptr, T, int(h),
                 int(h), 1, 3, 0};
    DCP_HIP(launch_proj(p, ProjEpilogue::kStore, st));
  } else {
    DCP_TRY(gemm(hd, false, false, T, h, h, y1, lw.wq, 0.f, s.bf16[kQ], s.bf16[kQ], false));
    DCP_TRY(gemm(hd, false, false, T, h, h, y1, lw.wk, 0.f, s.bf16[kK], s.bf16[kK], false));
    DCP_TRY(gemm(hd, false, false, T, h, h, y1, lw.wv, 0.f, s.bf16[kV], s.bf16[kV], false));
  }
  DCP_TRY(dcp_varlen_attn_fwd(desc->layer->attn, s.bf16[kQ], s.bf16[kK], s.bf16[kV], s.bf16[kO], s.lse, attn_ws,
                              attn_ws_bytes, st));
  if (s.kept[kQ].data) {
    ActBatch p{};
    for (p.n = 0; p.n < 3; ++p.n) {
      p.src[p.n] = s.bf16[kQ + p.n];
      p.dst[p.n] = s.kept[kQ + p.n].data;
      p.scales[p.n] = s.kept[kQ + p.n].scales;
    }
    DCP_HIP(launch_act8_pack(p, b.format, T, int(h), h, st));
  }
  DCP_TRY(gemm(hd, false, false, T, h, h, s.bf16[kO], lw.wo, 0.f, s.bf16[kF1], s.bf16[kF1], false));
  GatedNormFwd j{};
  j.x = x;
  j.f = s.bf16[kF1];
  j.post = w->post1;
  j.gate = w->gate1;
  j.pre = lw.norm2;
  j.cu = desc->cu_seqlens;
  j.out = s.bf16[kH];
  j.y = y2;
  j.rstd_f = s.rstd_f1;
  j.rstd_out = s.rstd_h;
  j.keep_f = s.kept[kF1].data;
  j.keep_f_scales = s.kept[kF1].scales;
  j.keep_out = s.kept[kH].data;
  j.keep_out_scales = s.kept[kH].scales;
  j.rows = T;
  j.hidden = int(h);
  j.n_seqs = n_gates(desc);
  j.format = b.format;
  j.alpha = desc->residual_scale;
  j.eps = desc->layer->eps;
  DCP_HIP(launch_gated_norm_fwd(j, st));
  const bool keep_u = s.kept[kU].data != nullptr;
  if (fused_up(d)) {
    const Proj p{{y2}, {lw.w_up}, {keep_u ? s.kept[kU].data : s.bf16[kU]}, nullptr, a, T, int(4 * h), int(h), 1, 1, 0,
                 b.format, s.kept[kU].scales};
    DCP_HIP(launch_proj(p, keep_u ? ProjEpilogue::kGeluKeep : ProjEpilogue::kGelu, st));
  } else {
    DCP_TRY(gemm(hd, false, false, T, 4 * h, h, y2, lw.w_up, 0.f, s.bf16[kU], s.bf16[kU], false));
    DCP_HIP(launch_gelu_fwd(s.bf16[kU], a, T * 4 * h, st));
    if (keep_u) {
      const ActBatch p{{s.bf16[kU]}, {s.kept[kU].data}, {s.kept[kU].scales}, 1};
      DCP_HIP(launch_act8_pack(p, b.format, T, int(4 * h), 4 * h, st));
    }
  }
  DCP_TRY(gemm(hd, false, false, T, h, 4 * h, a, lw.w_down, 0.f, s.bf16[kF2], s.bf16[kF2], false));
  j.x = s.bf16[kH];
  j.f = s.bf16[kF2];
  j.post = w->post2;
  j.gate = w->gate2;
  j.pre = nullptr;
  j.out = out;
  j.y = nullptr;
  j.rstd_f = s.rstd_f2;
  j.rstd_out = nullptr;
  j.keep_f = s.kept[kF2].data;
  j.keep_f_scales = s.kept[kF2].scales;
  j.keep_out = j.keep_out_scales = nullptr;
  DCP_HIP(launch_gated_norm_fwd(j, st));
  return DCP_OK;
}

int check_block_weights(const dcp_block_desc* desc, const dcp_block_weights* w) {
  if (!w) return fail(DCP_ERR_INVALID, "weights are null");
  DCP_TRY(check_weights(&w->layer));
  const bool gate = desc->gate != DCP_GATE_NONE;
  if ((desc->post_norm != 0) != (w->post1 != nullptr) || (desc->post_norm != 0) != (w->post2 != nullptr))
    return fail(DCP_ERR_INVALID, "post1 and post2 go with post_norm");
  if (gate != (w->gate1 != nullptr) || gate != (w->gate2 != nullptr))
    return fail(DCP_ERR_INVALID, "gate1 and gate2 go with gate");
  for (const void* p : {w->post1, w->gate1, w->post2, w->gate2})
    if (reinterpret_cast<uintptr_t>(p) % 16) return fail(DCP_ERR_INVALID, "weights: not 16-byte aligned");
  return DCP_OK;
}

int check_space(const void* ws, size_t bytes, size_t need, const void* stash, const char* what) {
  if (!ws || bytes < need || reinterpret_cast<uintptr_t>(ws) % kAlign)
    return fail(DCP_ERR_WORKSPACE, "block %s workspace needs %zu bytes (256-byte aligned), got %zu", what, need, bytes);
  if (reinterpret_cast<uintptr_t>(stash) % kAlign) return fail(DCP_ERR_INVALID, "stash must be 256-byte aligned");
  return DCP_OK;
}

}  // namespace
}  // namespace dcp

using namespace dcp;

extern "C" int dcp_block_sizes(const dcp_block_desc* desc, size_t* stash_bytes, size_t* fwd_workspace_bytes,
                               size_t* bwd_workspace_bytes) {
  clear_error();
  Block b;
  DCP_TRY(block_of(desc, &b));
  FwdWs f;
  BwdWs g;
  DCP_TRY(fwd_ws(desc, b, &f));
  DCP_TRY(bwd_ws(desc, b, &g));
  if (stash_bytes) *stash_bytes = kept_layout(b, b.format).total;
  if (fwd_workspace_bytes) *fwd_workspace_bytes = f.total;
  if (bwd_workspace_bytes) *bwd_workspace_bytes = g.total;
  return DCP_OK;
}

extern "C" int dcp_block_fwd(const dcp_block_desc* desc, const dcp_block_weights* w, const void* x, void* out,
                             void* stash, void* workspace, size_t workspace_bytes, void* stream) {
  clear_error();
  Block b;
  DCP_TRY(block_of(desc, &b));
  DCP_TRY(check_block_weights(desc, w));
  if (b.d.T == 0) return DCP_OK;
  DCP_TRY(check_ptrs({x, out}, "x and out"));
  FwdWs f;
  DCP_TRY(fwd_ws(desc, b, &f));
  DCP_TRY(check_space(workspace, workspace_bytes, f.total, stash, "forward"));
  hipStream_t st = static_cast<hipStream_t>(stream);
  rocblas_handle hd;
  DCP_TRY(blas(st, workspace, &hd));
  return forward(desc, b, w, x, out, forward_acts(b, stash, at(workspace, f.act)), at(workspace, f.y1),
                 at(workspace, f.y2), at(workspace, f.a), reinterpret_cast<float*>(at(workspace, f.rstd1)),
                 at(workspace, f.attn), f.act - f.attn, hd, st);
}

extern "C" int dcp_block_bwd(const dcp_block_desc* desc, const dcp_block_weights* w, const void* x, const void* dout,
                             void* dx, const dcp_block_grads* g, const void* stash, void* workspace,
                             size_t workspace_bytes, void* stream) {
  clear_error();
  Block b;
  DCP_TRY(block_of(desc, &b));
  DCP_TRY(check_block_weights(desc, w));
  if (b.d.T == 0) return DCP_OK;
  DCP_TRY(check_ptrs({x, dout, dx}, "x, dout and dx"));
  if (!g) return fail(DCP_ERR_INVALID, "grads are null");
  const dcp_layer_grads& lg = g->layer;
  DCP_TRY(check_ptrs({lg.norm1, lg.wq, lg.wk, lg.wv, lg.wo, lg.norm2, lg.w_up, lg.w_down}, "grads"));
  if (w->post1) DCP_TRY(check_ptrs({g->post1, g->post2}, "post grads"));
  if (w->gate1) DCP_TRY(check_ptrs({g->gate1, g->gate2}, "gate grads"));
  if ((w->post1 && (g->post1 == lg.norm2 || (w->gate1 && (g->post1 == g->gate1 || g->post2 == g->gate2)))) ||
      (w->gate1 && g->gate1 == lg.norm2))
    return fail(DCP_ERR_INVALID, "two gradients of one join are one buffer");
  BwdWs v;
  DCP_TRY(bwd_ws(desc, b, &v));
  DCP_TRY(check_space(workspace, workspace_bytes, v.total, stash, "backward"));
  hipStream_t st = static_cast<hipStream_t>(stream);
  rocblas_handle hd;
  DCP_TRY(blas(st, workspace, &hd));
  const Dims& d = b.d;
  const int64_t T = d.T, h = d.h;
  const dcp_layer_weights& lw = w->layer;
  void *y1 = at(workspace, v.y1), *y2 = at(workspace, v.y2), *a = at(workspace, v.a);
  float* rstd1 = reinterpret_cast<float*>(at(workspace, v.rstd1));
  // the activations as kept (8 bits or bf16), and q, k and v in bf16
  Acts s = forward_acts(b, const_cast<void*>(stash), at(workspace, v.act));
  int format = b.format;
  if (!stash) {  // recomputation: the forward again, its output discarded
    DCP_TRY(forward(desc, b, w, x, at(workspace, v.out), s, y1, y2, a, rstd1, at(workspace, v.attn_f),
                    v.attn_b - v.attn_f, hd, st));
    format = DCP_ACT_BF16;
  }
  for (dcp_kept& k : s.kept)
    if (!k.data) k = {s.bf16[&k - s.kept], nullptr};
  if (format != DCP_ACT_BF16) {
    ActBatch p{};
    for (p.n = 0; p.n < 3; ++p.n) {
      p.src[p.n] = s.kept[kQ + p.n].data;
      p.dst[p.n] = s.bf16[kQ + p.n];
      p.scales[p.n] = s.kept[kQ + p.n].scales;
    }
    DCP_HIP(launch_act8_unpack(p, format, T, int(h), h, st));
  }
  // the MLP's join: gradients of f2 and h (which, with nothing on the branch, are dout)
  const void *df2 = dout, *dh = dout;
  GatedNormBwd j{};
  j.cu = desc->cu_seqlens;
  j.rows = T;
  j.hidden = int(h);
  j.n_seqs = n_gates(desc);
  j.format = format;
  j.accumulate = 1;
  j.alpha = desc->residual_scale;
  if (b.branch || desc->residual_scale != 1.f) {
    df2 = at(workspace, v.f2);
    dh = desc->residual_scale != 1.f ? at(workspace, v.dh) : dout;
    j.dout = dout;
    j.f = s.kept[kF2].data;
    j.f_scales = s.kept[kF2].scales;
    j.rstd_f = s.rstd_f2;
    j.post = w->post2;
    j.gate = w->gate2;
    j.dx = dh == dout ? nullptr : at(workspace, v.dh);
    j.df = at(workspace, v.f2);
    j.dpost = g->post2;
    j.dgate = g->gate2;
    if (!w->post2) j.dpost = nullptr;
    if (!w->gate2) j.dgate = nullptr;
    DCP_HIP(launch_gated_norm_bwd(j, at(workspace, v.join), st));
  }
  // MLP: dA = dF2 Wdown^T; dU = dA GELU'(U) in place, A = GELU(U)
  void* da = at(workspace, v.da);
  if (format == DCP_ACT_BF16 && fused_back(d)) {
    const Proj p{{df2}, {lw.w_down}, {da}, s.bf16[kU], a, T, int(4 * h), int(h), 1, 1, 0, format, nullptr};
    DCP_HIP(launch_proj(p, ProjEpilogue::kGeluBack, st));
  } else {
    DCP_TRY(gemm(hd, false, true, T, 4 * h, h, df2, lw.w_down, 0.f, da, da, false));
    DCP_HIP(launch_act_gelu_bwd(s.kept[kU].data, s.kept[kU].scales, format, da, da, a, T, int(4 * h), 4 * h, st));
  }
  // dY2 = dU Wup^T (fp32), then the attention's join: gradients of f1 and x, and Y2
  void* dY2 = at(workspace, v.f32);
  DCP_TRY(gemm(hd, false, true, T, h, 4 * h, da, lw.w_up, 0.f, dY2, dY2, true));
  j.dout = dh;
  j.dy = dY2;
  j.dy_f32 = 1;
  j.f = s.kept[kF1].data;
  j.f_scales = s.kept[kF1].scales;
  j.out = s.kept[kH].data;
  j.out_scales = s.kept[kH].scales;
  j.rstd_f = s.rstd_f1;
  j.rstd_out = s.rstd_h;
  j.post = w->post1;
  j.gate = w->gate1;
  j.pre = lw.norm2;
  j.dx = at(workspace, v.dx1);
  j.df = at(workspace, v.f1);
  j.y = y2;
  j.dpost = w->post1 ? g->post1 : nullptr;
  j.dgate = w->gate1 ? g->gate1 : nullptr;
  j.dpre = lg.norm2;
  DCP_HIP(launch_gated_norm_bwd(j, at(workspace, v.join), st));
  // attention block: dO = dF1 Wo^T; attention backward
  const void* df1 = at(workspace, v.f1);
  void* dO = at(workspace, v.f32);  // (dY2 is done with)
  if (fused_square(d)) {
    const Proj p{{df1}, {lw.wo}, {dO}, nullptr, nullptr, T, int(h), int(h), 1, 1, 0};
    DCP_HIP(launch_proj(p, ProjEpilogue::kStoreT, st));
  } else {
    DCP_TRY(gemm(hd, false, true, T, h, h, df1, lw.wo, 0.f, dO, dO, false));
  }
  void *dq = at(workspace, v.dq), *dk = at(workspace, v.dk), *dv = at(workspace, v.dv);
  DCP_TRY(dcp_varlen_attn_bwd(desc->layer->attn, dO, s.bf16[kO], s.lse, s.bf16[kQ], s.bf16[kK], s.bf16[kV], dq, dk, dv,
                              at(workspace, v.attn_b), v.act - v.attn_b, st));
  // dY1 = dQ Wq^T + dK Wk^T + dV Wv^T (fp32)
  void* dY1 = at(workspace, v.f32);
  if (fused_dy1(d)) {
    const Proj p{{dq, dk, dv}, {lw.wq, lw.wk, lw.wv}, {dY1}, nullptr, nullptr, T, int(h), int(h), 3, 1, 0};
    DCP_HIP(launch_proj(p, ProjEpilogue::kSumF32, st));
  } else {
    DCP_TRY(gemm(hd, false, true, T, h, h, dq, lw.wq, 0.f, dY1, dY1, true));
    DCP_TRY(gemm(hd, false, true, T, h, h, dk, lw.wk, 1.f, dY1, dY1, true));
    DCP_TRY(gemm(hd, false, true, T, h, h, dv, lw.wv, 1.f, dY1, dY1, true));
  }
  // the weight gradients (Y1 formed again, unless the recomputation just did)
  if (stash) DCP_HIP(launch_rmsnorm_fwd(x, lw.norm1, y1, rstd1, T, int(h), desc->layer->eps, st));
  const int hi = int(h);
  const WgradBatch wb{{{a, df2, lg.w_down, 4 * hi, hi, 0},
                       {y2, da, lg.w_up, hi, 4 * hi, 0},
                       {s.bf16[kO], df1, lg.wo, hi, hi, 0},
                       {y1, dq, lg.wq, hi, hi, 0},
                       {y1, dk, lg.wk, hi, hi, 0},
                       {y1, dv, lg.wv, hi, hi, 0}},
                      T, 0, 0};
  if (library_wgrad(d)) {
    for (const WgradProblem& p : wb.p) DCP_TRY(gemm(hd, true, false, p.m, p.n, T, p.a, p.b, 1.f, p.c, p.c, true));
  } else {
    DCP_HIP(launch_wgrad(wb, workspace, kGemmWorkspace, st));
  }
  // dX = dX1 + RMSNorm backward of dY1
  DCP_HIP(launch_rmsnorm_bwd(static_cast<float*>(dY1), x, lw.norm1, rstd1, at(workspace, v.dx1), dx,
                             reinterpret_cast<float*>(at(workspace, v.partial)), lg.norm1, T, int(h), st));
  return DCP_OK;
}
