// Gated residual and norm, t = x + alpha gate F, y = t / rms(t) (1 + scale) + shift, and its gradients.
//
// A row's statistics need the whole row, its values are used once: every row is read once, into registers, by
// 64 to 512 threads of 4-element pieces, so a call moves the bytes that it has to and is bound by HBM: 6400 x 2048 of a 32-bit
// stream with normed bf16 blocks 32.4 us (4.9 TB/s), its gradients 53.4 (4.4) and 4.9 for the workers' sums; 3200 x 1024 with a
// modulation row each, 13.8 and 24.
// Gradients of what rows share are sums over rows: a worker (the threads of one row) takes a run of the rows
// that share a modulation row, keeps the sums of its columns in registers, and writes them once; where several
// workers share one, a second launch adds their sums in order.
#include "layer.h"

namespace ravel {
namespace {

RAVEL_DEV f32x4_t load4(const float* p) { return *(const f32x4_t*)p; }
RAVEL_DEV f32x4_t load4(const bf16_t* p) {
  const u32x2_t w = *(const u32x2_t*)p;
  return f32x4_t{__uint_as_float(w[0] << 16), __uint_as_float(w[0] & 0xFFFF0000u), __uint_as_float(w[1] << 16),
                 __uint_as_float(w[1] & 0xFFFF0000u)};
}
RAVEL_DEV void store4(float* p, f32x4_t v) { *(f32x4_t*)p = v; }
RAVEL_DEV void store4(bf16_t* p, f32x4_t v) { *(u32x2_t*)p = u32x2_t{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])}; }
RAVEL_DEV f32x4_t rounded(f32x4_t v, const float*) { return v; }
RAVEL_DEV f32x4_t rounded(f32x4_t v, const bf16_t*) {
  u32x2_t w{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
  return load4((const bf16_t*)&w);
}
RAVEL_DEV f32x4_t all4(float v) { return f32x4_t{v, v, v, v}; }
RAVEL_DEV float sum4(f32x4_t v) { return (v[0] + v[1]) + (v[2] + v[3]); }

// Sum over the wave's lanes without LDS: rotations inside its rows of 16, then the rows.
template <int ROTATE>
RAVEL_DEV float plus_rotated(float v) {
  return v + __uint_as_float(__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), 0x120 + ROTATE, 0xf, 0xf, true));
}
RAVEL_DEV float lanes_sum(float v) {
  v = plus_rotated<8>(v);
  v = plus_rotated<4>(v);
  v = plus_rotated<2>(v);
  v = plus_rotated<1>(v);
  auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// Sums over the TPR threads of a row.  `slot` alternates between consecutive calls (0, 1, 0, ...), so that one
// barrier a call is enough.
template <int TPR, int N>
RAVEL_DEV void row_sum(float (&v)[N], float (*part)[TPR / 64][4], int slot) {
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = lanes_sum(v[i]);
  if constexpr (TPR > 64) {
    const int wave = threadIdx.x >> 6;
    if ((threadIdx.x & 63) == 0)
#pragma unroll
      for (int i = 0; i < N; ++i) part[slot][wave][i] = v[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
      v[i] = part[slot][0][i];
#pragma unroll
      for (int w = 1; w < TPR / 64; ++w) v[i] += part[slot][w][i];
    }
  }
}

// x + (alpha gate) F, each operation rounded by itself: the bits that the formula gives one operation at a time.  (Contracted
// it would round once less, and now and then a bf16 stream the other way: half a step of n in the modulation's gradients.)
RAVEL_DEV f32x4_t add_block(f32x4_t x, float alpha, f32x4_t gate, f32x4_t f) {
#pragma clang fp contract(off)
  return x + alpha * gate * f;
}

template <int TPR>
constexpr int rows_per_block() {
  return TPR == 64 ? 4 : 1;
}

template <typename S, typename T, int TPR, int NC>
__global__ __launch_bounds__(TPR * rows_per_block<TPR>()) void norm_residual_kernel(ravel_norm a) {
  __shared__ float part[2][TPR / 64][4];
  const int lane = threadIdx.x % TPR;
  const int row = blockIdx.x * rows_per_block<TPR>() + threadIdx.x / TPR;
  if (row >= a.rows) return;  // a whole wave; blocks of one row have none
  const size_t mod = (row / a.group) % a.mods;
  f32x4_t t[NC], f[NC], gate[NC], scale[NC], shift[NC];
  // every load of the row is issued before the first sum
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    const int col = (c * TPR + lane) * 4;
    t[c] = f[c] = shift[c] = all4(0.f);
    gate[c] = scale[c] = all4(1.f);
    if (col < a.width) {
      t[c] = load4((const S*)a.x + row * a.x_stride + col);
      if (a.f) f[c] = load4((const T*)a.f + row * a.f_stride + col);
      if (a.f && a.gate) gate[c] = load4(a.gate + mod * a.gate_stride + col);
      if (a.scale) scale[c] = load4(a.scale + mod * a.scale_stride + col) + 1.f;
      if (a.shift) shift[c] = load4(a.shift + mod * a.shift_stride + col);
    }
  }
  float v[1];
  if (a.f) {
    const float alpha = a.alpha ? *a.alpha : 1.f;
    float rf = 1.f;
    if (a.post) {
      v[0] = 0.f;
#pragma unroll
      for (int c = 0; c < NC; ++c) v[0] += sum4(f[c] * f[c]);
      row_sum<TPR>(v, part, 0);
      rf = 1.f / sqrtf(v[0] / a.width + a.eps);
    }
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      const int col = (c * TPR + lane) * 4;
      if (col >= a.width) continue;
      if (a.post) f[c] = f[c] * rf * (load4(a.post + col) + 1.f);
      t[c] = rounded(add_block(t[c], alpha, gate[c], f[c]), (const S*)nullptr);
      if (a.x_out) store4((S*)a.x_out + row * a.x_out_stride + col, t[c]);
    }
  }
  if (!a.y) return;
  v[0] = 0.f;
#pragma unroll
  for (int c = 0; c < NC; ++c) v[0] += sum4(t[c] * t[c]);
  row_sum<TPR>(v, part, 1);
  const float r = 1.f / sqrtf(v[0] / a.width + a.eps);
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    const int col = (c * TPR + lane) * 4;
    if (col < a.width) store4((T*)a.y + row * a.y_stride + col, t[c] * r * scale[c] + shift[c]);
  }
}

// How the rows are dealt out.  Row i of modulation row m (i < count) is row (i / group) * group * mods + m * group +
// i % group where that is below rows.  Worker k takes modulation rows k, k + workers, ... whole (segs 1), or rows s, s +
// segs, ... of row m (k = m segs + s): at any time all workers are at neighbouring rows.  (Runs of rows a worker, spread
// over the whole tensors, took 76 us instead of 69 for 6400 x 2048.)
struct GradPlan {
  int mods, group, count, segs, workers;
  // where the sums go: to their place (one worker), or to the workspace, to be added
  bool mod_part, all_part;
  bool all[3];  // gate, scale, shift: summed over all rows
  float *gate, *scale, *shift, *post, *alpha;  // the sums of a modulation row (stride), or of a worker
  long long gate_stride, scale_stride, shift_stride;
  float* partial[5];  // the workspace's sums of dgate, dscale, dshift, dpost, dalpha; null: none
  size_t bytes;
};

GradPlan grad_plan(const ravel_norm& n, const ravel_norm_grad& g) {
  GradPlan p{};
  float* const out[3] = {g.dgate, g.dscale, g.dshift};
  const int64_t stride[3] = {g.dgate_stride, g.dscale_stride, g.dshift_stride};
  bool any_mod = false, any_all = g.dpost || g.dalpha;
  for (int i = 0; i < 3; ++i) {
    p.all[i] = out[i] && (stride[i] == 0 || n.mods == 1);
    any_all |= p.all[i];
    any_mod |= out[i] && !p.all[i];
  }
  // The modulations that are read may have several rows where no gradient does: every worker then takes any rows.
  p.mods = any_mod ? n.mods : 1;
  p.group = any_mod ? (n.group < n.rows ? n.group : n.rows) : n.rows;
  if (p.group < 1) p.group = 1;
  const long long cycle = (long long)p.group * p.mods, rest = n.rows % cycle;
  p.count = (int)(n.rows / cycle * p.group + (rest < p.group ? rest : p.group));
  // At least 4 rows a worker, so that its sums are few beside its rows, and no more workers than run at once (two waves a
  // SIMD): 914 of 256 threads, where 512 fit, took 96 us for 6400 x 2048, 512 took 90.
  const int most = n.width <= 256 ? 4096 : n.width <= 512 ? 2048 : n.width <= 1024 ? 1024 : n.width <= 2048 ? 512 : 256;
  const int rows = n.rows > p.mods ? n.rows : p.mods;
  int want = (rows + 3) / 4;
  want = want < 1 ? 1 : want > most ? most : want;
  p.segs = want / p.mods < p.count ? want / p.mods : p.count;
  if (p.segs < 1) p.segs = 1;
  p.workers = p.mods >= want ? want : p.mods * p.segs;
  p.mod_part = any_mod && p.segs > 1;
  p.all_part = any_all && p.workers > 1;
  float* const dst[5] = {g.dgate, g.dscale, g.dshift, g.dpost, g.dalpha};
  float* at[5];
  long long st[5];
  float* ws = (float*)g.workspace;
  size_t used = 0;
  for (int i = 0; i < 5; ++i) {
    const bool all = i >= 3 || p.all[i];
    const size_t w = i == 4 ? 1 : n.width;
    at[i] = dst[i];
    st[i] = all ? 0 : stride[i];
    if (dst[i] && (all ? p.all_part : p.mod_part)) {
      p.partial[i] = at[i] = ws + used;
      st[i] = w;
      used += ((size_t)p.workers * w + 63) / 64 * 64;
    }
  }
  p.gate = at[0], p.scale = at[1], p.shift = at[2], p.post = at[3], p.alpha = at[4];
  p.gate_stride = st[0], p.scale_stride = st[1], p.shift_stride = st[2];
  p.bytes = used * 4;
  return p;
}

// A row of a tensor as a buffer: what lies behind its width, or the whole of an absent row, reads as 0 and is not stored.
struct RowBuffer {
  __amdgpu_buffer_rsrc_t r;
  RAVEL_DEV RowBuffer(const void* p, long long stride, long long row, int width, int elt, bool there) {
    r = __builtin_amdgcn_make_buffer_rsrc((char*)const_cast<void*>(p) + row * stride * elt, (short)0, p && there ? width * elt : 0,
                                          0x00020000);
  }
  template <typename T> RAVEL_DEV f32x4_t load(int col) const {
    if constexpr (sizeof(T) == 4) return __builtin_bit_cast(f32x4_t, __builtin_amdgcn_raw_buffer_load_b128(r, col * 4, 0, 0));
    const u32x2_t w = __builtin_bit_cast(u32x2_t, __builtin_amdgcn_raw_buffer_load_b64(r, col * 2, 0, 0));
    return f32x4_t{__uint_as_float(w[0] << 16), __uint_as_float(w[0] & 0xFFFF0000u), __uint_as_float(w[1] << 16),
                   __uint_as_float(w[1] & 0xFFFF0000u)};
  }
  template <typename T> RAVEL_DEV void store(int col, f32x4_t v) const {
    if constexpr (sizeof(T) == 4) {
      __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4_t, v), r, col * 4, 0, 0);
    } else {
      __builtin_amdgcn_raw_buffer_store_b64(u32x2_t{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])}, r, col * 2, 0, 0);
    }
  }
};

// dn = dy (1 + scale); dt = d_out + r (dn - n mean(dn n)) with n = t r; dF = alpha gate dt; and through the block
// output's own norm, m = f rf, dm = dF (1 + post): df = rf (dm - m mean(dm m)).  The sums of t^2, dn t and f^2 are
// formed together; the last one needs dt and comes second.
//
// All loads of a row are issued a row ahead (beyond 4096 elements, where registers do not hold two rows, at its start).
// Loads and stores are waited for in the order of their issue, and the compiler waits for as many as are certain to have
// been issued: a row therefore has no branch, only buffers of no length for what is not there (with branches around its
// stores every row waited for the one before to be stored: 69 us instead of 53 for 6400 x 2048, which is 4.4 TB/s).
template <typename S, typename T, int TPR, int NC>
__global__ __launch_bounds__(TPR * rows_per_block<TPR>()) void norm_residual_grad_kernel(ravel_norm a, ravel_norm_grad g,
                                                                                      GradPlan p) {
  __shared__ float part[2][TPR / 64][4];
  const int lane = threadIdx.x % TPR;
  const int worker = __builtin_amdgcn_readfirstlane(blockIdx.x * rows_per_block<TPR>() + threadIdx.x / TPR);
  if (worker >= p.workers) return;  // a whole wave; blocks of one worker have none
  const int m_step = p.segs > 1 ? p.mods : p.workers, i_beg = worker % p.segs;
  const long long cycle = (long long)p.group * p.mods;
  const void* const t_in = a.f ? a.x_out : a.x;
  const long long t_stride = a.f ? a.x_out_stride : a.x_stride;
  const float alpha = a.f && a.alpha ? *a.alpha : 1.f, inv = 1.f / a.width;
  const bool want_f = a.f && (g.df || g.dpost || g.dgate || g.dalpha), second = a.post && g.df;
  const float post_of = a.post ? 1.f : 0.f, gate_of = a.gate ? 0.f : 1.f;

  f32x4_t s_gate[NC], s_scale[NC], s_shift[NC], s_post[NC], post1[NC];
  float s_alpha = 0.f;
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    s_gate[c] = s_scale[c] = s_shift[c] = s_post[c] = all4(0.f);
    post1[c] = RowBuffer(a.post, 0, 0, a.width, 4, true).load<float>((c * TPR + lane) * 4) + 1.f;
  }
  struct Row {
    f32x4_t t[NC], dy[NC], dt[NC], f[NC], gate[NC], scale[NC];
  } next;
  const auto row_of = [&](int m, int i) { return i / p.group * cycle + (long long)m * p.group + i % p.group; };
  const auto fetch = [&](int m, int i) {
    const long long row = m < p.mods && i < p.count ? row_of(m, i) : a.rows;
    const long long mod = (row / a.group) % a.mods;
    const bool in = row < a.rows;
    const RowBuffer t(t_in, t_stride, row, a.width, sizeof(S), in), dy(g.dy, g.dy_stride, row, a.width, sizeof(T), in),
        dt(g.d_out, g.d_out_stride, row, a.width, sizeof(S), in), f(a.f, a.f_stride, row, a.width, sizeof(T), in && want_f),
        gate(a.gate, a.gate_stride, mod, a.width, 4, in && want_f), scale(a.scale, a.scale_stride, mod, a.width, 4, in);
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      const int col = (c * TPR + lane) * 4;
      next.t[c] = t.template load<S>(col);
      next.dy[c] = dy.template load<T>(col);
      next.dt[c] = dt.template load<S>(col);
      next.f[c] = f.template load<T>(col);
      next.gate[c] = gate.template load<float>(col);
      next.scale[c] = scale.template load<float>(col);
    }
  };
  // a modulation row's sum to its place, and from 0 on again; nothing where it is summed over all rows
  const auto flush = [&](float* to, long long stride, int at, bool now, f32x4_t(&s)[NC]) {
    const RowBuffer out(to, stride, at, a.width, 4, now);
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      out.template store<float>((c * TPR + lane) * 4, s[c]);
#pragma unroll
      for (int e = 0; e < 4; ++e) s[c][e] = now ? 0.f : s[c][e];
    }
  };

  constexpr bool AHEAD = NC < 4;
  int m = worker / p.segs, i = i_beg;
  if constexpr (AHEAD) fetch(m, i);
  while (m < p.mods) {
    if constexpr (!AHEAD) fetch(m, i);
    const long long row = i < p.count ? row_of(m, i) : a.rows;
    const bool in = row < a.rows;
    const int i_next = i + p.segs;
    const bool last = i_next >= p.count;
    f32x4_t t[NC], dn[NC], dt[NC], f[NC], gate[NC], dy[NC], dm[NC];
    float v[3] = {0.f, 0.f, 0.f};
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      t[c] = next.t[c], dy[c] = next.dy[c], dt[c] = next.dt[c], f[c] = next.f[c], gate[c] = next.gate[c] + gate_of;
      dn[c] = dy[c] * (next.scale[c] + 1.f);
    }
    if constexpr (AHEAD) fetch(last ? m + m_step : m, last ? i_beg : i_next);
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      v[0] += sum4(t[c] * t[c]);
      v[1] += sum4(dn[c] * t[c]);
      v[2] += sum4(f[c] * f[c]);
    }
    row_sum<TPR>(v, part, 0);
    const float r = 1.f / sqrtf(v[0] * inv + a.eps), k = r * (r * (v[1] * inv));  // (r r may overflow)
    const float rf = post_of != 0.f ? 1.f / sqrtf(v[2] * inv + a.eps) : 1.f;
    const RowBuffer dx(g.dx, g.dx_stride, row, a.width, sizeof(S), in), df(g.df, g.df_stride, row, a.width, sizeof(T), in);
    float u[1] = {0.f};
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      dt[c] += r * (dn[c] - k * t[c]);
      dx.template store<S>((c * TPR + lane) * 4, dt[c]);
      s_scale[c] += dy[c] * (t[c] * r);
      s_shift[c] += dy[c];
      f[c] *= rf;                                // m
      const f32x4_t d = dt[c] * f[c] * post1[c];  // dt F
      s_gate[c] += alpha * d;
      s_alpha += sum4(d * gate[c]);
      dm[c] = alpha * gate[c] * dt[c];  // dF
      s_post[c] += dm[c] * f[c];
      dm[c] *= post1[c];
      u[0] += sum4(dm[c] * f[c]);
    }
    row_sum<TPR>(u, part, 1);
    const float back = second ? u[0] * inv : 0.f;
#pragma unroll
    for (int c = 0; c < NC; ++c) df.template store<T>((c * TPR + lane) * 4, rf * (dm[c] - back * f[c]));
    const int at = p.mod_part ? worker : m;
    flush(p.gate, p.gate_stride, at, last && !p.all[0], s_gate);
    flush(p.scale, p.scale_stride, at, last && !p.all[1], s_scale);
    flush(p.shift, p.shift_stride, at, last && !p.all[2], s_shift);
    m = last ? m + m_step : m;
    i = last ? i_beg : i_next;
  }
  flush(p.gate, p.gate_stride, worker, p.all[0], s_gate);
  flush(p.scale, p.scale_stride, worker, p.all[1], s_scale);
  flush(p.shift, p.shift_stride, worker, p.all[2], s_shift);
  flush(p.post, a.width, worker, true, s_post);
  float v[1] = {s_alpha};
  row_sum<TPR>(v, part, 0);
  if (p.alpha && lane == 0) p.alpha[worker] = v[0];
}

// Sums of the workers: row m of a task is the sum of partial rows m n .. m n + n - 1, each slice's in order, then the
// slices'.
struct SumTask {
  const float* src;
  float* dst;
  long long stride;
  int rows, n, width;
};
struct SumTasks {
  SumTask t[5];
};
__global__ __launch_bounds__(256) void norm_sum_kernel(SumTasks tasks) {
  const SumTask t = tasks.t[blockIdx.z];
  const int m = blockIdx.y;
  if (m >= t.rows) return;
  __shared__ f32x4_t part[64][4];
  if (t.width == 1) {
    if (blockIdx.x) return;
    float s = 0.f;
    for (int i = threadIdx.x; i < t.n; i += 256) s += t.src[i];
    float* const f = (float*)part;
    f[threadIdx.x] = s;
    __syncthreads();
    if (threadIdx.x < 64) {
      s = lanes_sum(f[threadIdx.x] + f[threadIdx.x + 64] + f[threadIdx.x + 128] + f[threadIdx.x + 192]);
      if (threadIdx.x == 0) t.dst[0] = s;
    }
    return;
  }
  const int quad = threadIdx.x & 3, slice = threadIdx.x >> 2, col = blockIdx.x * 16 + quad * 4;
  f32x4_t s = all4(0.f);
  if (col < t.width) {
    const float* const p = t.src + (size_t)m * t.n * t.width + col;
#pragma unroll 4
    for (int i = slice; i < t.n; i += 64) s += load4(p + (size_t)i * t.width);
  }
  part[slice][quad] = s;
  __syncthreads();
  if (threadIdx.x >= 32) return;
  s = part[slice][quad];  // eight slices of eight
#pragma unroll
  for (int i = 1; i < 8; ++i) s += part[slice + 8 * i][quad];
  part[slice][quad] = s;
  __builtin_amdgcn_wave_barrier();
  if (slice == 0 && col < t.width) {
#pragma unroll
    for (int i = 1; i < 8; ++i) s += part[i][quad];
    store4(t.dst + m * t.stride + col, s);
  }
}

template <typename S, typename T, int TPR, int NC>
void launch_forward(const ravel_norm& n, hipStream_t s) {
  constexpr int R = rows_per_block<TPR>();
  norm_residual_kernel<S, T, TPR, NC><<<(n.rows + R - 1) / R, TPR * R, 0, s>>>(n);
}
template <typename S, typename T, int TPR, int NC>
void launch_rows(const ravel_norm& n, const ravel_norm_grad* g, const GradPlan& p, hipStream_t s) {
  constexpr int R = rows_per_block<TPR>();
  if (g)
    norm_residual_grad_kernel<S, T, TPR, NC><<<(p.workers + R - 1) / R, TPR * R, 0, s>>>(n, *g, p);
  else
    launch_forward<S, T, TPR, NC>(n, s);
}
template <typename S, typename T>
void launch_width(const ravel_norm& n, const ravel_norm_grad* g, const GradPlan& p, hipStream_t s) {
  if (n.width <= 256) launch_rows<S, T, 64, 1>(n, g, p, s);
  else if (n.width <= 512) launch_rows<S, T, 64, 2>(n, g, p, s);
  else if (n.width <= 1024 && !g && n.rows >= 1024) launch_forward<S, T, 64, 4>(n, s);
  else if (n.width <= 1024) launch_rows<S, T, 128, 2>(n, g, p, s);
  else if (n.width <= 2048) launch_rows<S, T, 256, 2>(n, g, p, s);
  else if (n.width <= 4096) launch_rows<S, T, 512, 2>(n, g, p, s);
  else launch_rows<S, T, 512, 4>(n, g, p, s);
}
void launch_types(const ravel_norm& n, const ravel_norm_grad* g, const GradPlan& p, hipStream_t s) {
  if (n.stream_dtype == RAVEL_BF16) launch_width<bf16_t, bf16_t>(n, g, p, s);
  else if (n.dtype == RAVEL_BF16) launch_width<float, bf16_t>(n, g, p, s);
  else launch_width<float, float>(n, g, p, s);
}

}  // namespace

hipError_t launch_norm_residual(const ravel_norm& n, hipStream_t s) {
  if (n.rows == 0) return hipSuccess;
  launch_types(n, nullptr, GradPlan{}, s);
  return hipGetLastError();
}

size_t norm_grad_workspace(const ravel_norm& n, const ravel_norm_grad& g) { return grad_plan(n, g).bytes; }

hipError_t launch_norm_residual_grad(const ravel_norm& n, const ravel_norm_grad& g, hipStream_t s) {
  const GradPlan p = grad_plan(n, g);
  launch_types(n, &g, p, s);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || (!p.mod_part && !p.all_part)) return e;
  SumTasks tasks;
  float* const dst[5] = {g.dgate, g.dscale, g.dshift, g.dpost, g.dalpha};
  const int64_t stride[3] = {g.dgate_stride, g.dscale_stride, g.dshift_stride};
  int count = 0, rows = 1;
  for (int i = 0; i < 5; ++i) {
    if (!p.partial[i]) continue;
    const bool all = i >= 3 || p.all[i];
    SumTask& t = tasks.t[count++];
    t = {p.partial[i], dst[i], all ? 0 : stride[i], all ? 1 : p.mods, all ? p.workers : p.segs, i == 4 ? 1 : n.width};
    if (t.rows > rows) rows = t.rows;
  }
  norm_sum_kernel<<<dim3((n.width + 15) / 16, rows, count), 256, 0, s>>>(tasks);
  return hipGetLastError();
}

}  // namespace ravel
