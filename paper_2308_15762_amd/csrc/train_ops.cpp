// C entry points of the operators around the chunks of a training iteration: embedding with a scale, the join between two
// sub-layers, the gradient norm with clipping.  Everything that a kernel assumes of its arguments is checked here.
#include <hip/hip_runtime.h>

#include <cmath>

#include "ends.h"
#include "kernels.h"

using namespace hanayo;

namespace {

#define TRY(expr)           \
  do {                      \
    const int rc_ = (expr); \
    if (rc_) return rc_;    \
  } while (0)

bool off16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) != 0; }
bool off(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a != 0; }

int check_dtype(const char* what, int dtype) {
  if (dtype != HANAYO_FP32 && dtype != HANAYO_BF16) return set_error(HANAYO_EINVAL, "%s: dtype %d", what, dtype);
  return HANAYO_OK;
}

// ------------------------------------------------------------------ embedding

int check_embedding(const char* what, int dtype, float scale, int rows, int hidden, int vocab) {
  TRY(check_dtype(what, dtype));
  if (rows < 0 || hidden < 8 || hidden % 8 || vocab < 1)
    return set_error(HANAYO_EINVAL, "%s: rows %d, hidden %d (a multiple of 8), vocab %d", what, rows, hidden, vocab);
  if (rows > k::kEmbeddingMaxRows || hidden > 65536 || vocab > 1 << 28)
    return set_error(HANAYO_EUNSUPPORTED, "%s: more than %d rows, 65536 columns or 2^28 tokens", what, k::kEmbeddingMaxRows);
  if (!std::isfinite(scale)) return set_error(HANAYO_EINVAL, "%s: scale is not finite", what);
  return HANAYO_OK;
}

// ------------------------------------------------------------------ residual join

int check_residual(const hanayo_residual_desc* d) {
  if (!d) return set_error(HANAYO_EINVAL, "residual: NULL descriptor");
  TRY(check_dtype("residual", d->dtype));
  if (d->rows < 0 || d->hidden < 8 || d->hidden % 8)
    return set_error(HANAYO_EINVAL, "residual: rows %d, hidden %d (a multiple of 8)", d->rows, d->hidden);
  if (d->hidden > k::kResidualMaxHidden || d->rows > 1 << 30)
    return set_error(HANAYO_EUNSUPPORTED, "residual: hidden %d > %d, or more than 2^30 rows", d->hidden, k::kResidualMaxHidden);
  for (int kind : {d->post_norm, d->pre_norm})
    if (kind != HANAYO_NORM_NONE && kind != HANAYO_NORM_LAYER && kind != HANAYO_NORM_RMS)
      return set_error(HANAYO_EINVAL, "residual: norm %d", kind);
  if (d->gate != HANAYO_GATE_NONE && d->gate != HANAYO_GATE_CHANNEL && d->gate != HANAYO_GATE_ELEMENT)
    return set_error(HANAYO_EINVAL, "residual: gate %d", d->gate);
  if (!std::isfinite(d->x_scale) || !std::isfinite(d->branch_scale))
    return set_error(HANAYO_EINVAL, "residual: scales have to be finite");
  if (!(d->eps > 0.f)) return set_error(HANAYO_EINVAL, "residual: eps must be > 0");
  return HANAYO_OK;
}

k::ResidualArgs residual_args(const hanayo_residual_desc* d) {
  k::ResidualArgs a{};
  a.rows = d->rows; a.H = d->hidden; a.post = d->post_norm; a.pre = d->pre_norm; a.gate_kind = d->gate;
  a.x_scale = d->x_scale; a.branch_scale = d->branch_scale; a.eps = d->eps;
  return a;
}

// ------------------------------------------------------------------ gradient norm

int check_grads(const char* what, const hanayo_grad* grads, size_t n, bool outs) {
  if (n && !grads) return set_error(HANAYO_EINVAL, "%s: NULL list", what);
  size_t left = k::kGradMaxElements;
  for (size_t i = 0; i < n; ++i) {
    TRY(check_dtype(what, grads[i].dtype));
    if (!grads[i].count) continue;
    if (!grads[i].grad) return set_error(HANAYO_EINVAL, "%s: tensor %zu is NULL", what, i);
    const size_t size = grads[i].dtype == HANAYO_BF16 ? 2 : 4;
    if (off(grads[i].grad, size) || (outs && off(grads[i].out, size)))
      return set_error(HANAYO_EINVAL, "%s: tensor %zu does not lie on an element's boundary", what, i);
    if (grads[i].count > left) return set_error(HANAYO_EUNSUPPORTED, "%s: more than 2^40 elements", what);
    left -= grads[i].count;
    if (outs && grads[i].out && grads[i].out != grads[i].grad) {
      const uintptr_t in = reinterpret_cast<uintptr_t>(grads[i].grad), out = reinterpret_cast<uintptr_t>(grads[i].out);
      if ((in < out ? out - in : in - out) < grads[i].count * size)
        return set_error(HANAYO_EINVAL, "%s: tensor %zu overlaps its own output", what, i);
    }
  }
  return HANAYO_OK;
}

int check_clip(const char* what, const hanayo_clip* c, k::ClipArgs& out) {
  if (!c || !c->sumsq) return set_error(HANAYO_EINVAL, "%s: NULL clip or sumsq", what);
  if (c->parts < 1 || c->parts > 65536) return set_error(HANAYO_EINVAL, "%s: parts %d", what, c->parts);
  if (!(c->max_norm >= 0.f)) return set_error(HANAYO_EINVAL, "%s: max_norm must be >= 0", what);
  if (off(c->sumsq, 8) || off(c->norm, 4) || off(c->skipped, 4))
    return set_error(HANAYO_EINVAL, "%s: misaligned sumsq, norm or skipped", what);
  out = k::ClipArgs{c->sumsq, c->parts, c->max_norm, c->norm, c->skipped};
  return HANAYO_OK;
}

}  // namespace

extern "C" {

int hanayo_op_embedding_forward(int dtype, const void* table, const int32_t* tokens, float scale, void* out, int rows,
                                int hidden, int vocab, void* hip_stream) {
  TRY(check_embedding("op_embedding_forward", dtype, scale, rows, hidden, vocab));
  if (!table || (rows && (!tokens || !out))) return set_error(HANAYO_EINVAL, "op_embedding_forward: NULL pointer");
  if (off16(table) || off16(out) || off(tokens, 4))
    return set_error(HANAYO_EINVAL, "op_embedding_forward: table and out have to be 16-byte aligned, tokens 4-byte");
  TRY(device_ok());
  return k::embedding_forward(dtype, table, tokens, scale, out, rows, hidden, vocab, static_cast<hipStream_t>(hip_stream));
}

size_t hanayo_op_embedding_workspace_bytes(int rows, int hidden, int vocab) {
  if (check_embedding("op_embedding_workspace_bytes", HANAYO_FP32, 1.f, rows, hidden, vocab)) return 0;
  return k::embedding_workspace_bytes(rows, hidden, vocab);
}

int hanayo_op_embedding_backward(int dtype, const int32_t* tokens, const void* dout, float scale, float* d_table, int rows,
                                 int hidden, int vocab, int accumulate, void* workspace, void* hip_stream) {
  TRY(check_embedding("op_embedding_backward", dtype, scale, rows, hidden, vocab));
  if (!d_table || !workspace || (rows && (!tokens || !dout)))
    return set_error(HANAYO_EINVAL, "op_embedding_backward: NULL pointer");
  if (off16(d_table) || off16(dout) || off16(workspace) || off(tokens, 4))
    return set_error(HANAYO_EINVAL, "op_embedding_backward: dout, d_table and workspace have to be 16-byte aligned, tokens 4-byte");
  TRY(device_ok());
  return k::embedding_backward(dtype, tokens, dout, scale, d_table, rows, hidden, vocab, accumulate != 0, workspace,
                               static_cast<hipStream_t>(hip_stream));
}

int hanayo_op_residual_forward(const hanayo_residual_desc* d, const void* x, const void* branch, const void* gate,
                               const void* post, const void* pre, void* x_out, void* h, float* stats, void* hip_stream) {
  TRY(check_residual(d));
  if (d->rows && (!x || !branch || !x_out || (d->pre_norm && !h) || (d->gate == HANAYO_GATE_ELEMENT && !gate)))
    return set_error(HANAYO_EINVAL, "op_residual_forward: NULL pointer");
  if ((d->gate == HANAYO_GATE_CHANNEL && !gate) || (d->post_norm && !post) || (d->pre_norm && !pre))
    return set_error(HANAYO_EINVAL, "op_residual_forward: the gate or a norm's parameters are missing");
  for (const void* p : {x, branch, gate, post, pre, static_cast<const void*>(x_out), static_cast<const void*>(h), static_cast<const void*>(stats)})
    if (off16(p)) return set_error(HANAYO_EINVAL, "op_residual_forward: pointers have to be 16-byte aligned");
  if (d->rows && (x_out == branch || (d->pre_norm && (h == x_out || h == x || h == branch || h == gate)) ||
                  (gate && x_out == gate)))
    return set_error(HANAYO_EINVAL, "op_residual_forward: an output aliases an operand (only x_out may be x)");
  TRY(device_ok());
  k::ResidualArgs a = residual_args(d);
  a.x = x; a.branch = branch; a.gate = gate; a.w_post = post; a.w_pre = pre; a.x_out = x_out; a.h = h;
  a.stats = reinterpret_cast<float4*>(stats);
  return k::residual_forward(d->dtype, a, static_cast<hipStream_t>(hip_stream));
}

size_t hanayo_op_residual_scratch_bytes(const hanayo_residual_desc* d) {
  return check_residual(d) ? 0 : k::residual_scratch_bytes(d->rows, d->hidden);
}

int hanayo_op_residual_backward(const hanayo_residual_desc* d, const void* x_out, const void* branch, const void* gate,
                                const void* post, const void* pre, const float* stats, const void* dh, const void* dx_out,
                                void* dx, void* dbranch, void* dgate, float* d_post, float* d_pre, int accumulate,
                                void* scratch, void* hip_stream) {
  TRY(check_residual(d));
  if (d->rows && (!branch || !stats || !dx || !dbranch || (d->pre_norm ? !x_out || !dh : !dx_out) ||
                  (d->gate == HANAYO_GATE_ELEMENT && (!gate || !dgate))))
    return set_error(HANAYO_EINVAL, "op_residual_backward: NULL pointer");
  if ((d->gate == HANAYO_GATE_CHANNEL && (!gate || !dgate)) || (d->post_norm && (!post || !d_post)) ||
      (d->pre_norm && (!pre || !d_pre)) || !scratch)
    return set_error(HANAYO_EINVAL, "op_residual_backward: the gate's or a norm's parameters or gradients, or the scratch, are missing");
  for (const void* p : {x_out, branch, gate, post, pre, static_cast<const void*>(stats), dh, dx_out, static_cast<const void*>(dx),
                        static_cast<const void*>(dbranch), static_cast<const void*>(scratch)})
    if (off16(p)) return set_error(HANAYO_EINVAL, "op_residual_backward: pointers have to be 16-byte aligned");
  if (d->gate == HANAYO_GATE_ELEMENT ? off16(dgate) : off(dgate, 4))
    return set_error(HANAYO_EINVAL, "op_residual_backward: dgate is misaligned");
  if (off(d_post, 4) || off(d_pre, 4)) return set_error(HANAYO_EINVAL, "op_residual_backward: d_post or d_pre is misaligned");
  const bool element = d->gate == HANAYO_GATE_ELEMENT;
  if (d->rows) {
    const void* outs[3] = {dx, dbranch, element ? dgate : nullptr};
    for (int i = 0; i < 3; ++i) {
      if (!outs[i]) continue;
      for (const void* in : {x_out, branch, gate, dh, dx_out})
        if (in == outs[i] && !(i == 0 && in == dx_out))
          return set_error(HANAYO_EINVAL, "op_residual_backward: an output aliases an operand (only dx may be dx_out)");
      for (int j = 0; j < i; ++j)
        if (outs[i] == outs[j]) return set_error(HANAYO_EINVAL, "op_residual_backward: two outputs are the same");
    }
  }
  TRY(device_ok());
  k::ResidualArgs a = residual_args(d);
  a.x_out = const_cast<void*>(x_out); a.branch = branch; a.gate = gate; a.w_post = post; a.w_pre = pre;
  a.stats = reinterpret_cast<float4*>(const_cast<float*>(stats));
  a.dh = dh; a.dx_out = dx_out; a.dx = dx; a.dbranch = dbranch; a.dgate = d->gate ? dgate : nullptr;
  a.d_post = d->post_norm ? d_post : nullptr;
  a.d_pre = d->pre_norm ? d_pre : nullptr;
  a.accumulate = accumulate != 0;
  a.scratch = static_cast<float*>(scratch);
  return k::residual_backward(d->dtype, a, static_cast<hipStream_t>(hip_stream));
}

size_t hanayo_op_grad_workspace_bytes(size_t n) { return k::grad_workspace_bytes(n); }

int hanayo_op_grad_sumsq(const hanayo_grad* grads, size_t n, double* sumsq, void* workspace, void* hip_stream) {
  TRY(check_grads("op_grad_sumsq", grads, n, false));
  if (!sumsq || !workspace) return set_error(HANAYO_EINVAL, "op_grad_sumsq: NULL pointer");
  if (off(sumsq, 8) || off(workspace, 8)) return set_error(HANAYO_EINVAL, "op_grad_sumsq: misaligned sumsq or workspace");
  TRY(device_ok());
  return k::grad_sumsq(grads, n, sumsq, static_cast<double*>(workspace), static_cast<hipStream_t>(hip_stream));
}

int hanayo_op_grad_clip(const hanayo_grad* grads, size_t n, const hanayo_clip* clip, void* hip_stream) {
  k::ClipArgs c;
  TRY(check_grads("op_grad_clip", grads, n, true));
  TRY(check_clip("op_grad_clip", clip, c));
  TRY(device_ok());
  return k::grad_clip(grads, n, c, static_cast<hipStream_t>(hip_stream));
}

int hanayo_adam_step_clipped(const hanayo_adam* o, const hanayo_clip* clip, int dtype, void* params, float* master,
                             float* grads, float* m, float* v, size_t count, void* hip_stream) {
  if (!o) return set_error(HANAYO_EINVAL, "adam_step_clipped: NULL argument");
  TRY(check_dtype("adam_step_clipped", dtype));
  k::AdamArgs a = adam_args(o, params, master, grads, m, v, count);
  TRY(check_clip("adam_step_clipped", clip, a.clip));
  TRY(k::adam_check(dtype, a));
  if (off(params, dtype == HANAYO_BF16 ? 8 : 16) || off16(a.master) || off16(grads) || off16(m) || off16(v))
    return set_error(HANAYO_EINVAL, "adam_step_clipped: arrays have to be 16-byte aligned");
  TRY(device_ok());
  return k::adam(dtype, a, static_cast<hipStream_t>(hip_stream));
}

int hanayo_chunk_adam_step_clipped(const hanayo_adam* o, const hanayo_clip* clip, const hanayo_chunk_desc* d, void* weights,
                                   float* master, float* grads, float* m, float* v, void* hip_stream) {
  if (!o) return set_error(HANAYO_EINVAL, "chunk_adam_step_clipped: NULL argument");
  Shape sh;
  TRY(make_shape(d, sh));
  k::ClipArgs c;
  TRY(check_clip("chunk_adam_step_clipped", clip, c));
  if (off16(weights) || off16(master) || off16(grads) || off16(m) || off16(v))
    return set_error(HANAYO_EINVAL, "chunk_adam_step_clipped: arrays have to be 16-byte aligned");
  TRY(device_ok());
  return chunk_adam_step(o, sh, weights, master, grads, m, v, static_cast<hipStream_t>(hip_stream), &c);
}

}  // extern "C"
