// C ABI of a layer's operators: argument checks, then the launches of norm_residual.hip, cross_attention.hip and
// gated_mlp.hip.
#include <algorithm>
#include <initializer_list>

#include "layer.h"

using namespace ravel;

namespace {

// One call's checks; the first that fails is the call's status.
struct Check {
  const char* call;
  ravel_status status = RAVEL_OK;
  bool ok() const { return status == RAVEL_OK; }
  void fail(ravel_status s, const std::string& msg) {
    if (ok()) status = set_error(s, std::string(call) + ": " + msg);
  }
  void valid(bool good, const char* msg) {
    if (!good) fail(RAVEL_E_INVALID, msg);
  }
  void shape(bool good, const char* msg) {
    if (!good) fail(RAVEL_E_SHAPE, msg);
  }
  void dtype(int32_t d) { valid(d == RAVEL_F32 || d == RAVEL_BF16, "dtype must be RAVEL_F32 or RAVEL_BF16"); }
  // a tensor that may be absent
  void aligned(std::initializer_list<const void*> tensors, size_t n = 16) {
    for (const void* p : tensors)
      if ((uintptr_t)p % n) return fail(RAVEL_E_INVALID, "tensors must be " + std::to_string(n) + "-byte aligned");
  }
  void present(std::initializer_list<const void*> tensors) {
    for (const void* p : tensors) valid(p != nullptr, "null pointer");
  }
  // outputs (the first `outs` of the list) that are another's memory
  void apart(std::initializer_list<const void*> tensors, size_t outs) {
    for (size_t i = 0; i < outs; ++i)
      for (size_t j = i + 1; j < tensors.size(); ++j) {
        const void *a = tensors.begin()[i], *b = tensors.begin()[j];
        valid(!a || a != b, "outputs must not share memory with other tensors");
      }
  }
  // Rows of `inner` elements of `elt` bytes.  The stride of a dimension with one index is of no account.
  void rows(int64_t n, int64_t stride, int64_t inner, int elt, bool output) {
    if (n <= 1) return;
    shape(stride >= 0 && stride * elt % 16 == 0, "strides must be multiples of 16 bytes, not negative");
    shape(!output || stride >= inner, "rows of an output must not overlap");
    shape(stride <= (1ll << 60) / n, "strides reach past 64-bit addresses");
  }
  void workspace(const void* ws, int64_t bytes, size_t need) {
    if (!need || !ok()) return;
    if (!ws || bytes < 0 || (size_t)bytes < need) return fail(RAVEL_E_INVALID, "needs a workspace of " + std::to_string(need) + " bytes");
    if ((uintptr_t)ws % 256) fail(RAVEL_E_INVALID, "the workspace must be 256-byte aligned");
  }
  ravel_status launched(hipError_t e) const {
    return e == hipSuccess ? RAVEL_OK : set_error(RAVEL_E_HIP, std::string(call) + ": " + hipGetErrorString(e));
  }
};
constexpr int64_t kBlocks = 1 << 24;  // blocks of 256 threads: below 2^32 of them in a launch
int bytes_of(int32_t dtype) { return dtype == RAVEL_F32 ? 4 : 2; }

// ---------------------------------------------------------------------------
// gated residual and norm
// ---------------------------------------------------------------------------
void norm_sizes(Check& k, const ravel_norm* n) {
  k.valid(n, "null struct");
  if (!k.ok()) return;
  k.dtype(n->stream_dtype);
  k.dtype(n->dtype);
  k.valid(n->stream_dtype != RAVEL_BF16 || n->dtype == RAVEL_BF16, "a bf16 stream needs bf16 blocks");
  k.valid(n->reserved == 0, "reserved must be 0");
  k.shape(n->rows >= 0 && n->rows < 1 << 23, "rows must be in 0..2^23 - 1");  // (times 512 threads below 2^32)
  k.shape(n->width >= 8 && n->width <= 8192 && n->width % 8 == 0, "width must be a multiple of 8 in 8..8192");
  k.shape(n->mods >= 1 && n->mods <= 1 << 30 && n->group >= 1, "mods and group must be >= 1");
}
void norm_inputs(Check& k, const ravel_norm* n) {
  const int S = bytes_of(n->stream_dtype), T = bytes_of(n->dtype);
  k.valid(n->eps > 0.f && n->eps < INFINITY, "eps must be positive and finite");
  k.aligned({n->x, n->f, n->post, n->gate, n->scale, n->shift, n->x_out, n->y});
  k.aligned({n->alpha}, 4);
  k.valid(n->f || n->rows == 0 || (!n->post && !n->alpha && !n->gate), "post, alpha and gate need f");
  k.rows(n->rows, n->f_stride, n->width, T, false);
  for (const auto& m : {std::make_pair(n->gate, n->gate_stride), std::make_pair(n->scale, n->scale_stride)})
    if (m.first) k.rows(n->mods, m.second, n->width, 4, false);
}

ravel_status norm_call(const ravel_norm* n, hipStream_t s) {
  Check k{"ravel_norm_residual"};
  norm_sizes(k, n);
  if (!k.ok()) return k.status;
  norm_inputs(k, n);
  const int S = bytes_of(n->stream_dtype), T = bytes_of(n->dtype);
  if (n->shift) k.rows(n->mods, n->shift_stride, n->width, 4, false);
  k.rows(n->rows, n->x_stride, n->width, S, false);
  if (n->x_out) k.rows(n->rows, n->x_out_stride, n->width, S, true);
  if (n->y) k.rows(n->rows, n->y_stride, n->width, T, true);
  if (n->rows == 0) return k.status;
  k.present({n->x});
  k.valid(n->f ? n->x_out != nullptr : n->x_out == nullptr, "x_out goes with f");
  k.valid(n->y || n->x_out, "nothing to compute");
  k.valid(n->x_out != n->x || n->x_out_stride == n->x_stride || n->rows == 1, "x_out in place of x needs its stride");
  k.apart({n->x_out, n->y, n->f, n->post, n->alpha, n->gate, n->scale, n->shift}, 2);
  k.apart({n->y, n->x}, 1);
  return k.ok() ? k.launched(launch_norm_residual(*n, s)) : k.status;
}

void norm_grad_sizes(Check& k, const ravel_norm* n, const ravel_norm_grad* g) {
  norm_sizes(k, n);
  k.valid(g, "null struct");
  if (!k.ok()) return;
  k.valid((!g->dpost || n->post) && (!g->dalpha || n->alpha) && (!g->dgate || n->gate) && (!g->dscale || n->scale) &&
              (!g->df || n->f || n->rows == 0),
          "a gradient of what is not there");
  const struct {
    const float *d, *of;
    int64_t stride, of_stride;
  } mods[] = {{g->dgate, n->gate, g->dgate_stride, n->gate_stride},
              {g->dscale, n->scale, g->dscale_stride, n->scale_stride},
              {g->dshift, nullptr, g->dshift_stride, 0}};
  for (const auto& m : mods) {
    if (!m.d || n->mods == 1) continue;
    k.shape(!m.of || (m.stride == 0) == (m.of_stride == 0), "a vector has a vector's gradient, rows have rows'");
    if (m.stride) k.rows(n->mods, m.stride, n->width, 4, true);
  }
}

ravel_status norm_grad_call(const ravel_norm* n, const ravel_norm_grad* g, hipStream_t s) {
  Check k{"ravel_norm_residual_grad"};
  norm_grad_sizes(k, n, g);
  if (!k.ok()) return k.status;
  norm_inputs(k, n);
  const int S = bytes_of(n->stream_dtype), T = bytes_of(n->dtype);
  const void* const t = n->f ? n->x_out : n->x;
  k.rows(n->rows, n->f ? n->x_out_stride : n->x_stride, n->width, S, false);
  if (g->dy) k.rows(n->rows, g->dy_stride, n->width, T, false);
  if (g->d_out) k.rows(n->rows, g->d_out_stride, n->width, S, false);
  if (g->dx) k.rows(n->rows, g->dx_stride, n->width, S, true);
  if (g->df) k.rows(n->rows, g->df_stride, n->width, T, true);
  k.aligned({g->dy, g->d_out, g->dx, g->df, g->dpost, g->dgate, g->dscale, g->dshift});
  k.aligned({g->dalpha}, 4);
  if (n->rows > 0) k.present({t});
  k.valid(g->dx != g->d_out || !g->dx || g->dx_stride == g->d_out_stride || n->rows <= 1, "dx in place of d_out needs its stride");
  k.apart({g->dx, g->df, g->dpost, g->dalpha, g->dgate, g->dscale, g->dshift, t, g->dy, n->f, n->post, n->alpha, n->gate, n->scale}, 7);
  k.apart({g->df, g->d_out}, 1);
  const size_t need = k.ok() ? norm_grad_workspace(*n, *g) : 0;
  k.workspace(g->workspace, g->workspace_bytes, need);
  if (!k.ok() || !(g->dx || g->df || g->dpost || g->dalpha || g->dgate || g->dscale || g->dshift)) return k.status;
  return k.launched(launch_norm_residual_grad(*n, *g, s));
}

// ---------------------------------------------------------------------------
// cross attention
// ---------------------------------------------------------------------------
void cross_sizes(Check& k, const ravel_cross* c) {
  k.valid(c, "null struct");
  if (!k.ok()) return;
  k.dtype(c->dtype);
  // (times log2 e it has to stay finite: 0 times infinity is not 0; and so has the logarithm of a row's sum over the scale, from
  // which the gradients' scores start)
  k.valid(c->scale == 0.f || (c->scale >= 0x1p-100f && c->scale <= 0x1p100f), "scale must be 0 or in 2^-100..2^100");
  k.shape(c->batch >= 0 && c->batch <= 65535, "batch must be in 0..65535");
  k.shape(c->head_dim == 32 || c->head_dim == 64 || c->head_dim == 128 || c->head_dim == 256, "head_dim must be 32, 64, 128 or 256");
  k.shape(c->n_kv_heads >= 1 && c->n_q_heads >= 1 && c->n_q_heads <= 256 && c->n_q_heads % c->n_kv_heads == 0,
          "n_q_heads must be a multiple of n_kv_heads, at most 256");
  k.shape(c->rows >= 0 && c->rows <= 1 << 20, "rows must be in 0..2^20");
  k.shape(c->keys >= 0 && c->keys <= 1 << 24, "keys must be in 0..2^24");
  if (!k.ok()) return;
  k.shape((int64_t)c->rows * c->n_q_heads <= 1 << 30, "too many rows times heads");
  if (k.ok()) k.shape(cross_blocks(*c) < kBlocks, "too many rows: a launch holds 2^24 - 1 tiles");
}
// Strides of [batch, n, heads, head_dim].  Kernels address the rows, keys and heads of a tile with 24 by 24 bit products.
void cross_strides(Check& k, const ravel_cross* c, const int64_t* st, int64_t n, int64_t heads, bool output) {
  const int e = bytes_of(c->dtype);
  k.rows(c->batch, st[0], c->head_dim, e, output);
  k.rows(n, st[1], c->head_dim, e, output);
  k.rows(heads, st[2], c->head_dim, e, output);
  if (k.ok()) {
    const int64_t r = n > 1 ? st[1] : 0, h = heads > 1 ? st[2] : 0;
    k.shape(r * e <= 1 << 22 && h * e <= 1 << 22, "strides of rows, keys and heads must be at most 2^22 bytes");
  }
}
void cross_inputs(Check& k, const ravel_cross* c) {
  k.aligned({c->q, c->k, c->v, c->out});
  k.aligned({c->q_len, c->k_len, c->lse}, 4);
  cross_strides(k, c, c->q_stride, c->rows, c->n_q_heads, false);
  cross_strides(k, c, c->k_stride, c->keys, c->n_kv_heads, false);
  cross_strides(k, c, c->v_stride, c->keys, c->n_kv_heads, false);
}

ravel_status cross_call(const ravel_cross* c, hipStream_t s) {
  Check k{"ravel_cross_attention"};
  cross_sizes(k, c);
  if (!k.ok()) return k.status;
  cross_inputs(k, c);
  cross_strides(k, c, c->out_stride, c->rows, c->n_q_heads, true);
  if (!k.ok() || c->batch == 0 || c->rows == 0) return k.status;
  k.present({c->q, c->out});
  if (c->keys > 0) k.present({c->k, c->v});
  k.apart({c->out, c->lse, c->q, c->k, c->v, c->q_len, c->k_len}, 2);
  const size_t need = k.ok() ? cross_workspace(*c) : 0;
  k.workspace(c->workspace, c->workspace_bytes, need);
  return k.ok() ? k.launched(launch_cross_attention(*c, s)) : k.status;
}

void cross_grad_sizes(Check& k, const ravel_cross* c, const ravel_cross_grad* g) {
  cross_sizes(k, c);
  k.valid(g, "null struct");
  if (!k.ok()) return;
  k.valid(!g->dk == !g->dv, "dk and dv go together");
  if (k.ok()) k.shape(cross_grad_blocks(*c, *g) < kBlocks, "too many rows or keys: a launch holds 2^24 - 1 tiles");
}

ravel_status cross_grad_call(const ravel_cross* c, const ravel_cross_grad* g, hipStream_t s) {
  Check k{"ravel_cross_attention_grad"};
  cross_grad_sizes(k, c, g);
  if (!k.ok()) return k.status;
  cross_inputs(k, c);
  cross_strides(k, c, c->out_stride, c->rows, c->n_q_heads, false);
  cross_strides(k, c, g->dout_stride, c->rows, c->n_q_heads, false);
  if (g->dq) cross_strides(k, c, g->dq_stride, c->rows, c->n_q_heads, true);
  if (g->dk) {
    cross_strides(k, c, g->dk_stride, c->keys, c->n_kv_heads, true);
    cross_strides(k, c, g->dv_stride, c->keys, c->n_kv_heads, true);
  }
  k.aligned({g->dout, g->dq, g->dk, g->dv});
  if (!k.ok() || c->batch == 0 || (!g->dq && !g->dk)) return k.status;
  if (c->rows > 0) k.present({c->q, c->out, c->lse, g->dout});
  if (c->keys > 0) k.present({c->k, c->v});
  k.apart({g->dq, g->dk, g->dv, c->q, c->k, c->v, c->out, c->lse, g->dout, c->q_len, c->k_len}, 3);
  const size_t need = k.ok() ? cross_grad_workspace(*c, *g) : 0;
  k.workspace(g->workspace, g->workspace_bytes, need);
  return k.ok() ? k.launched(launch_cross_attention_grad(*c, *g, s)) : k.status;
}

// ---------------------------------------------------------------------------
// gated MLP
// ---------------------------------------------------------------------------
void mlp_sizes(Check& k, const ravel_mlp* m) {
  k.valid(m, "null struct");
  if (!k.ok()) return;
  k.dtype(m->dtype);
  const int32_t kind = m->act & ~RAVEL_GATE_F32;
  k.valid(kind == RAVEL_GELU_TANH || kind == RAVEL_SILU, "act must be RAVEL_GELU_TANH or RAVEL_SILU, with or without RAVEL_GATE_F32");
  k.valid(m->reserved == 0, "reserved must be 0");
  k.shape(m->rows >= 0 && m->rows <= 1 << 28, "rows must be in 0..2^28");
  k.shape(m->width >= 8 && m->width <= 1 << 18 && m->width % 8 == 0, "width must be a multiple of 8 in 8..2^18");
  k.shape(m->hidden >= 8 && m->hidden <= 1 << 18 && m->hidden % 8 == 0, "hidden must be a multiple of 8 in 8..2^18");
}
// kernels address the rows of a tile with 24 by 24 bit products
void mlp_rows(Check& k, int64_t n, int64_t stride, int64_t inner, int elt, bool output) {
  k.rows(n, stride, inner, elt, output);
  if (n > 1) k.shape(stride * elt <= 1 << 22, "strides must be at most 2^22 bytes");
}
int gate_bytes(const ravel_mlp* m) { return m->act & RAVEL_GATE_F32 ? 4 : bytes_of(m->dtype); }
void mlp_inputs(Check& k, const ravel_mlp* m) {
  const int e = bytes_of(m->dtype);
  k.aligned({m->x, m->wg, m->wu, m->h, m->gate, m->up});
  mlp_rows(k, m->rows, m->x_stride, m->width, e, false);
  mlp_rows(k, m->hidden, m->w_stride, m->width, e, false);
}

ravel_status mlp_call(const ravel_mlp* m, hipStream_t s) {
  Check k{"ravel_gated_mlp"};
  mlp_sizes(k, m);
  if (!k.ok()) return k.status;
  mlp_inputs(k, m);
  const int e = bytes_of(m->dtype);
  mlp_rows(k, m->rows, m->h_stride, m->hidden, e, true);
  k.valid(!m->gate == !m->up, "gate and up go together");
  if (m->gate) mlp_rows(k, m->rows, m->gate_stride, m->hidden, gate_bytes(m), true);
  if (!k.ok() || m->rows == 0) return k.status;
  k.present({m->x, m->wg, m->wu, m->h});
  k.apart({m->h, m->gate, m->up, m->x, m->wg, m->wu}, 3);
  const size_t need = k.ok() ? mlp_workspace(*m) : 0;
  k.workspace(m->workspace, m->workspace_bytes, need);
  return k.ok() ? k.launched(launch_gated_mlp(*m, s)) : k.status;
}

void mlp_grad_sizes(Check& k, const ravel_mlp* m, const ravel_mlp_grad* g) {
  mlp_sizes(k, m);
  k.valid(g, "null struct");
  if (!k.ok()) return;
  k.valid(g->reserved == 0, "reserved must be 0");
  k.valid(g->weight_dtype == m->dtype || g->weight_dtype == RAVEL_F32, "weight_dtype must be dtype or RAVEL_F32");
  k.valid(!g->dwg == !g->dwu, "dwg and dwu go together");
}

ravel_status mlp_grad_call(const ravel_mlp* m, const ravel_mlp_grad* g, hipStream_t s) {
  Check k{"ravel_gated_mlp_grad"};
  mlp_grad_sizes(k, m, g);
  if (!k.ok()) return k.status;
  mlp_inputs(k, m);
  const int e = bytes_of(m->dtype);
  mlp_rows(k, m->rows, m->gate_stride, m->hidden, gate_bytes(m), false);
  mlp_rows(k, m->rows, g->dh_stride, m->hidden, e, false);
  if (g->dx) mlp_rows(k, m->rows, g->dx_stride, m->width, e, true);
  if (g->dwg) mlp_rows(k, m->hidden, g->dw_stride, m->width, bytes_of(g->weight_dtype), true);
  k.aligned({g->dh, g->dx, g->dwg, g->dwu});
  if (!k.ok() || (!g->dx && !g->dwg)) return k.status;
  if (m->rows > 0) {
    k.present({m->gate, m->up, g->dh});
    if (g->dx) k.present({m->wg, m->wu});
    if (g->dwg) k.present({m->x});
  }
  k.apart({g->dx, g->dwg, g->dwu, m->x, m->wg, m->wu, m->gate, m->up, g->dh}, 3);
  const size_t need = k.ok() ? mlp_grad_workspace(*m, *g) : 0;
  k.workspace(g->workspace, g->workspace_bytes, need);
  return k.ok() ? k.launched(launch_gated_mlp_grad(*m, *g, s)) : k.status;
}

// no exception (a message that cannot be allocated, say) leaves the library
template <typename F>
ravel_status guarded(F f) noexcept {
  try {
    return f();
  } catch (...) {
    return RAVEL_E_NOMEM;
  }
}

}  // namespace

extern "C" {

ravel_status ravel_norm_residual(const ravel_norm* n, void* stream) {
  return guarded([&] { return norm_call(n, (hipStream_t)stream); });
}
ravel_status ravel_norm_residual_grad_workspace(const ravel_norm* n, const ravel_norm_grad* g, int64_t* bytes) {
  return guarded([&] {
    Check k{"ravel_norm_residual_grad_workspace"};
    norm_grad_sizes(k, n, g);
    k.present({bytes});
    if (k.ok()) *bytes = (int64_t)norm_grad_workspace(*n, *g);
    return k.status;
  });
}
ravel_status ravel_norm_residual_grad(const ravel_norm* n, const ravel_norm_grad* g, void* stream) {
  return guarded([&] { return norm_grad_call(n, g, (hipStream_t)stream); });
}

ravel_status ravel_cross_attention_workspace(const ravel_cross* c, int64_t* bytes) {
  return guarded([&] {
    Check k{"ravel_cross_attention_workspace"};
    cross_sizes(k, c);
    k.present({bytes});
    if (k.ok()) *bytes = c->batch && c->rows ? (int64_t)cross_workspace(*c) : 0;
    return k.status;
  });
}
ravel_status ravel_cross_attention(const ravel_cross* c, void* stream) {
  return guarded([&] { return cross_call(c, (hipStream_t)stream); });
}
ravel_status ravel_cross_attention_grad_workspace(const ravel_cross* c, const ravel_cross_grad* g, int64_t* bytes) {
  return guarded([&] {
    Check k{"ravel_cross_attention_grad_workspace"};
    cross_grad_sizes(k, c, g);
    k.present({bytes});
    if (k.ok()) *bytes = c->batch ? (int64_t)cross_grad_workspace(*c, *g) : 0;
    return k.status;
  });
}
ravel_status ravel_cross_attention_grad(const ravel_cross* c, const ravel_cross_grad* g, void* stream) {
  return guarded([&] { return cross_grad_call(c, g, (hipStream_t)stream); });
}

ravel_status ravel_gated_mlp_workspace(const ravel_mlp* m, int64_t* bytes) {
  return guarded([&] {
    Check k{"ravel_gated_mlp_workspace"};
    mlp_sizes(k, m);
    k.present({bytes});
    if (k.ok()) *bytes = (int64_t)mlp_workspace(*m);
    return k.status;
  });
}
ravel_status ravel_gated_mlp(const ravel_mlp* m, void* stream) {
  return guarded([&] { return mlp_call(m, (hipStream_t)stream); });
}
ravel_status ravel_gated_mlp_grad_workspace(const ravel_mlp* m, const ravel_mlp_grad* g, int64_t* bytes) {
  return guarded([&] {
    Check k{"ravel_gated_mlp_grad_workspace"};
    mlp_grad_sizes(k, m, g);
    k.present({bytes});
    if (k.ok()) *bytes = (int64_t)mlp_grad_workspace(*m, *g);
    return k.status;
  });
}
ravel_status ravel_gated_mlp_grad(const ravel_mlp* m, const ravel_mlp_grad* g, void* stream) {
  return guarded([&] { return mlp_grad_call(m, g, (hipStream_t)stream); });
}

}  // extern "C"
