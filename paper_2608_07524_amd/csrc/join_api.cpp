// C ABI of the 8-bit activation checkpoints and of the gated, normed join:
// argument checks (host only, before any device call) and launches.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>
#include <initializer_list>

#include "api_internal.h"
#include "block_launch.h"
#include "buffers.h"
#include "dcp_internal.h"

namespace dcp {
namespace {

int aligned(std::initializer_list<const void*> ps, uintptr_t to, const char* what) {
  for (const void* p : ps)
    if (!p || reinterpret_cast<uintptr_t>(p) % to)
      return fail(DCP_ERR_INVALID, "%s: null or not %d-byte aligned", what, int(to));
  return DCP_OK;
}

int check_act8(const dcp_act8_desc* d, bool bf16_too) {
  if (!d) return fail(DCP_ERR_INVALID, "activation desc is null");
  if (d->rows < 0 || d->rows >= (int64_t(1) << 31)) return fail(DCP_ERR_INVALID, "rows must lie in [0, 2^31)");
  if (d->cols <= 0) return fail(DCP_ERR_INVALID, "cols must be positive");
  if (d->cols % 8) return fail(DCP_ERR_UNSUPPORTED, "cols %d is not a multiple of 8", d->cols);
  if (d->ld < d->cols || d->ld % 8 || d->ld >= (int64_t(1) << 31))
    return fail(DCP_ERR_INVALID, "ld must be a multiple of 8, at least cols and below 2^31");
  if (d->format != DCP_ACT_INT8 && d->format != DCP_ACT_E4M3 && !(bf16_too && d->format == DCP_ACT_BF16))
    return fail(DCP_ERR_INVALID, "unknown activation format %d", d->format);
  return DCP_OK;
}

int launched(hipError_t e) {
  if (e != hipSuccess) return fail(DCP_ERR_HIP, "launch: %s", hipGetErrorString(e));
  return DCP_OK;
}

int check_join(const dcp_gated_norm_desc* d, const dcp_gated_norm_weights* w) {
  if (!d) return fail(DCP_ERR_INVALID, "join desc is null");
  if (d->rows < 0 || d->rows >= (int64_t(1) << 31)) return fail(DCP_ERR_INVALID, "rows must lie in [0, 2^31)");
  if (d->hidden <= 0) return fail(DCP_ERR_INVALID, "hidden must be positive");
  if (d->hidden % 8 || d->hidden > 4096)
    return fail(DCP_ERR_UNSUPPORTED, "hidden %d is not a multiple of 8 up to 4096", d->hidden);
  if (d->n_seqs < 0 || (d->n_seqs > 0) != (d->cu_seqlens != nullptr))
    return fail(DCP_ERR_INVALID, "n_seqs and cu_seqlens go together");
  if (d->n_seqs > 1 << 30) return fail(DCP_ERR_UNSUPPORTED, "%d sequences: more than 2^30", d->n_seqs);
  if (reinterpret_cast<uintptr_t>(d->cu_seqlens) % 4) return fail(DCP_ERR_INVALID, "cu_seqlens is not 4-byte aligned");
  if (!std::isfinite(d->residual_scale)) return fail(DCP_ERR_INVALID, "residual_scale must be finite");
  if (!(std::isfinite(d->eps) && d->eps >= 0.f)) return fail(DCP_ERR_INVALID, "eps must be finite and >= 0");
  if (d->keep_format < DCP_ACT_BF16 || d->keep_format > DCP_ACT_E4M3)
    return fail(DCP_ERR_INVALID, "unknown activation format %d", d->keep_format);
  if ((d->dy_f32 & ~1) || (d->accumulate & ~1)) return fail(DCP_ERR_INVALID, "dy_f32 and accumulate are 0 or 1");
  if (!w) return DCP_OK;
  for (const void* p : {w->post, w->gate, w->pre})
    if (reinterpret_cast<uintptr_t>(p) % 16) return fail(DCP_ERR_INVALID, "weights: not 16-byte aligned");
  if (d->n_seqs > 0 && !w->gate)
    return fail(DCP_ERR_INVALID, "cu_seqlens is for a gate of each sequence: gate is null");
  return DCP_OK;
}

// Buffers of a call on checkpoints: its bf16 matrices, and a checkpoint's two parts.
Buffer matrix(const dcp_act8_desc* d, const void* p, bool written) {
  const Buffer::Kind kind = written ? Buffer::kActsWritten : Buffer::kActsRead;
  if (d->ld == d->cols) return {p, kind, 2 * size_t(d->rows) * size_t(d->cols)};
  return {p, kind, 2 * size_t(d->cols), d->rows, 2 * size_t(d->ld)};
}
Buffer codes_of(const dcp_act8_desc* d, const void* p, bool written) {
  return {p, written ? Buffer::kWritten : Buffer::kRead, size_t(d->rows) * size_t(d->cols)};
}
Buffer scales_of(const dcp_act8_desc* d, const void* p, bool written) {
  return {p, written ? Buffer::kWritten : Buffer::kRead, size_t(d->rows) * size_t(act_groups(d->cols))};
}

int apart(std::initializer_list<Buffer> all) {
  const Buffer* b = clash(all);
  if (b) return fail(DCP_ERR_INVALID, "the output at %p shares memory with another buffer of the call", b->p);
  return DCP_OK;
}

// Buffers of a join.
struct JoinBuffers {
  const dcp_gated_norm_desc* d;
  size_t rows = size_t(d->rows), h = size_t(d->hidden);
  Buffer read(const void* p) const { return {p, Buffer::kActsRead, 2 * rows * h}; }
  Buffer written(const void* p) const { return {p, Buffer::kActsWritten, 2 * rows * h}; }
  Buffer row_scales(const float* p, bool out) const { return {p, out ? Buffer::kWritten : Buffer::kRead, 4 * rows}; }
  // a kept activation's data and scale bytes
  Buffer data(const dcp_kept* k, bool out) const {
    const void* p = k ? k->data : nullptr;
    if (d->keep_format == DCP_ACT_BF16) return out ? written(p) : read(p);
    return {p, out ? Buffer::kWritten : Buffer::kRead, rows * h};
  }
  Buffer scales(const dcp_kept* k, bool out) const {
    const bool has = k && k->data && d->keep_format != DCP_ACT_BF16;
    return {has ? k->scales : nullptr, out ? Buffer::kWritten : Buffer::kRead, rows * size_t(act_groups(d->hidden))};
  }
  size_t gates() const { return d->n_seqs > 0 ? size_t(d->n_seqs) : 1; }
  Buffer weight(const void* p, size_t n) const { return {p, Buffer::kRead, 2 * n * h}; }
  Buffer grad(const float* p, size_t n) const { return {p, Buffer::kWritten, 4 * n * h}; }
  Buffer offsets() const { return {d->cu_seqlens, Buffer::kRead, 4 * (size_t(d->n_seqs) + 1)}; }
};

// A kept activation as an operand: 16-byte aligned bf16, or codes (8-byte) and bytes.
int check_kept(const dcp_kept* k, int format, const char* what) {
  if (!k) return fail(DCP_ERR_INVALID, "%s is null", what);
  int st = aligned({k->data}, format == DCP_ACT_BF16 ? 16 : 8, what);
  if (st) return st;
  if (format != DCP_ACT_BF16 && !k->scales) return fail(DCP_ERR_INVALID, "%s: scales are null", what);
  return DCP_OK;
}

}  // namespace
}  // namespace dcp

using namespace dcp;

extern "C" int dcp_act8_pack(const dcp_act8_desc* d, const void* x, void* codes, void* scales, void* stream) {
  clear_error();
  DCP_TRY(check_act8(d, false));
  if (d->rows == 0) return DCP_OK;
  DCP_TRY(aligned({x}, 16, "x"));
  DCP_TRY(aligned({codes}, 8, "codes"));
  DCP_TRY(aligned({scales}, 1, "scales"));
  DCP_TRY(apart({matrix(d, x, false), codes_of(d, codes, true), scales_of(d, scales, true)}));
  DCP_TRY(check_device());
  const ActBatch b{{x}, {codes}, {scales}, 1};
  return launched(launch_act8_pack(b, d->format, d->rows, d->cols, d->ld, static_cast<hipStream_t>(stream)));
}

extern "C" int dcp_act8_unpack(const dcp_act8_desc* d, const void* codes, const void* scales, void* x, void* stream) {
  clear_error();
  DCP_TRY(check_act8(d, false));
  if (d->rows == 0) return DCP_OK;
  DCP_TRY(aligned({x}, 16, "x"));
  DCP_TRY(aligned({codes}, 8, "codes"));
  DCP_TRY(aligned({scales}, 1, "scales"));
  DCP_TRY(apart({matrix(d, x, true), codes_of(d, codes, false), scales_of(d, scales, false)}));
  DCP_TRY(check_device());
  const ActBatch b{{codes}, {x}, {const_cast<void*>(scales)}, 1};
  return launched(launch_act8_unpack(b, d->format, d->rows, d->cols, d->ld, static_cast<hipStream_t>(stream)));
}

extern "C" int dcp_act8_gelu_bwd(const dcp_act8_desc* d, const void* codes, const void* scales, const void* da,
                                 void* du, void* a, void* stream) {
  clear_error();
  DCP_TRY(check_act8(d, true));
  if (d->rows == 0) return DCP_OK;
  DCP_TRY(aligned({da, du, a}, 16, "da, du and a"));
  if (du == a) return fail(DCP_ERR_INVALID, "du and a are one buffer");
  const dcp_kept u{const_cast<void*>(codes), const_cast<void*>(scales)};
  DCP_TRY(check_kept(&u, d->format, "u"));
  const bool wide = d->format == DCP_ACT_BF16;
  DCP_TRY(apart({matrix(d, du, true), matrix(d, a, true), matrix(d, da, false),
                 wide ? matrix(d, codes, false) : codes_of(d, codes, false),
                 scales_of(d, wide ? nullptr : scales, false)}));
  DCP_TRY(check_device());
  return launched(launch_act_gelu_bwd(codes, scales, d->format, da, du, a, d->rows, d->cols, d->ld,
                                      static_cast<hipStream_t>(stream)));
}

extern "C" int dcp_gated_norm_fwd(const dcp_gated_norm_desc* d, const dcp_gated_norm_weights* w, const void* x,
                                  const void* f, void* out, void* y, float* rstd_f, float* rstd_out,
                                  const dcp_kept* keep_f, const dcp_kept* keep_out, void* stream) {
  clear_error();
  DCP_TRY(check_join(d, w));
  if (!w) return fail(DCP_ERR_INVALID, "weights are null");
  if (d->rows == 0) return DCP_OK;  // (buffers of no rows may be null)
  if ((w->pre != nullptr) != (y != nullptr) || (w->pre != nullptr) != (rstd_out != nullptr))
    return fail(DCP_ERR_INVALID, "y and rstd_out go with the weight pre");
  if ((w->post != nullptr) != (rstd_f != nullptr)) return fail(DCP_ERR_INVALID, "rstd_f goes with the weight post");
  const bool kf = keep_f && keep_f->data, ko = keep_out && keep_out->data;
  if ((kf || ko) && d->keep_format == DCP_ACT_BF16)
    return fail(DCP_ERR_INVALID, "in bf16 f and out themselves are kept");
  DCP_TRY(aligned({x, f, out}, 16, "x, f and out"));
  if (y) DCP_TRY(aligned({y}, 16, "y"));
  if (y == out) return fail(DCP_ERR_INVALID, "out and y are one buffer");
  if (kf) DCP_TRY(check_kept(keep_f, d->keep_format, "keep_f"));
  if (ko) DCP_TRY(check_kept(keep_out, d->keep_format, "keep_out"));
  const JoinBuffers b{d};
  DCP_TRY(apart({b.written(out), b.written(y), b.row_scales(rstd_f, true), b.row_scales(rstd_out, true),
                 b.data(kf ? keep_f : nullptr, true), b.scales(kf ? keep_f : nullptr, true),
                 b.data(ko ? keep_out : nullptr, true), b.scales(ko ? keep_out : nullptr, true), b.read(x), b.read(f),
                 b.weight(w->post, 1), b.weight(w->gate, b.gates()), b.weight(w->pre, 1), b.offsets()}));
  DCP_TRY(check_device());
  GatedNormFwd p{};
  p.x = x;
  p.f = f;
  p.post = w->post;
  p.gate = w->gate;
  p.pre = w->pre;
  p.cu = d->cu_seqlens;
  p.out = out;
  p.y = y;
  p.rstd_f = rstd_f;
  p.rstd_out = rstd_out;
  if (kf) {
    p.keep_f = keep_f->data;
    p.keep_f_scales = keep_f->scales;
  }
  if (ko) {
    p.keep_out = keep_out->data;
    p.keep_out_scales = keep_out->scales;
  }
  p.rows = d->rows;
  p.hidden = d->hidden;
  p.n_seqs = d->n_seqs;
  p.format = d->keep_format;
  p.alpha = d->residual_scale;
  p.eps = d->eps;
  return launched(launch_gated_norm_fwd(p, static_cast<hipStream_t>(stream)));
}

extern "C" int dcp_gated_norm_bwd_workspace_size(const dcp_gated_norm_desc* d, size_t* bytes) {
  clear_error();
  DCP_TRY(check_join(d, nullptr));
  if (!bytes) return fail(DCP_ERR_INVALID, "bytes is null");
  *bytes = gated_norm_bwd_workspace(d->rows, d->hidden, d->n_seqs);
  return DCP_OK;
}

extern "C" int dcp_gated_norm_bwd(const dcp_gated_norm_desc* d, const dcp_gated_norm_weights* w, const void* dout,
                                  const void* dy, const dcp_kept* f, const dcp_kept* out, const float* rstd_f,
                                  const float* rstd_out, void* dx, void* df, void* y, const dcp_gated_norm_grads* g,
                                  void* workspace, size_t workspace_bytes, void* stream) {
  clear_error();
  DCP_TRY(check_join(d, w));
  if (!w || !g) return fail(DCP_ERR_INVALID, "weights or grads are null");
  const bool need_f = w->post || w->gate;
  if ((w->post != nullptr) != (g->post != nullptr) || (w->gate != nullptr) != (g->gate != nullptr) ||
      (w->pre != nullptr) != (g->pre != nullptr))
    return fail(DCP_ERR_INVALID, "a gradient goes with each weight");
  if ((g->post && (g->post == g->gate || g->post == g->pre)) || (g->gate && g->gate == g->pre))
    return fail(DCP_ERR_INVALID, "two gradients are one buffer");
  for (const float* p : {g->post, g->gate, g->pre})
    if (reinterpret_cast<uintptr_t>(p) % 4) return fail(DCP_ERR_INVALID, "grads: not 4-byte aligned");
  if (d->rows > 0) {  // (buffers of no rows may be null)
    if (!w->pre && (dy || y || !dout))
      return fail(DCP_ERR_INVALID, "without the weight pre dout is needed, dy and y are not");
    DCP_TRY(aligned({df}, 16, "df"));
    for (const void* p : {dout, static_cast<const void*>(dx), static_cast<const void*>(y)})
      if (reinterpret_cast<uintptr_t>(p) % 16) return fail(DCP_ERR_INVALID, "dout, dx or y: not 16-byte aligned");
    if (dx == df || (y && (y == dx || y == df))) return fail(DCP_ERR_INVALID, "two of dx, df and y are one buffer");
    if (w->pre) {
      DCP_TRY(aligned({dy}, 16, "dy"));
      DCP_TRY(check_kept(out, d->keep_format, "out"));
      DCP_TRY(aligned({rstd_out}, 4, "rstd_out"));
    }
    if (need_f) DCP_TRY(check_kept(f, d->keep_format, "f"));
    if (w->post) DCP_TRY(aligned({rstd_f}, 4, "rstd_f"));
  }
  const size_t need = gated_norm_bwd_workspace(d->rows, d->hidden, d->n_seqs);
  if (need > 0 && (!workspace || workspace_bytes < need || reinterpret_cast<uintptr_t>(workspace) % 256))
    return fail(DCP_ERR_WORKSPACE, "join backward workspace needs %zu bytes (256-byte aligned), got %zu", need,
                workspace_bytes);
  const JoinBuffers b{d};
  Buffer dys = b.read(dy);
  if (d->dy_f32) dys = {dy, Buffer::kRead, 4 * b.rows * b.h};
  const dcp_kept *kf = need_f ? f : nullptr, *ko = w->pre ? out : nullptr;
  DCP_TRY(apart({b.written(dx), b.written(df), b.written(y), b.grad(g->post, 1), b.grad(g->gate, b.gates()),
                 b.grad(g->pre, 1), {workspace, Buffer::kWritten, need}, b.read(dout), dys, b.data(kf, false),
                 b.scales(kf, false), b.data(ko, false), b.scales(ko, false),
                 b.row_scales(w->post ? rstd_f : nullptr, false), b.row_scales(w->pre ? rstd_out : nullptr, false),
                 b.weight(w->post, 1), b.weight(w->gate, b.gates()), b.weight(w->pre, 1), b.offsets()}));
  DCP_TRY(check_device());
  GatedNormBwd p{};
  p.dout = dout;
  p.dy = dy;
  if (need_f && f) {
    p.f = f->data;
    p.f_scales = f->scales;
  }
  if (w->pre && out) {
    p.out = out->data;
    p.out_scales = out->scales;
  }
  p.rstd_f = rstd_f;
  p.rstd_out = rstd_out;
  p.post = w->post;
  p.gate = w->gate;
  p.pre = w->pre;
  p.cu = d->cu_seqlens;
  p.dx = dx;
  p.df = df;
  p.y = y;
  p.dpost = g->post;
  p.dgate = g->gate;
  p.dpre = g->pre;
  p.rows = d->rows;
  p.hidden = d->hidden;
  p.n_seqs = d->n_seqs;
  p.format = d->keep_format;
  p.dy_f32 = d->dy_f32;
  p.accumulate = d->accumulate;
  p.alpha = d->residual_scale;
  return launched(launch_gated_norm_bwd(p, workspace, static_cast<hipStream_t>(stream)));
}
