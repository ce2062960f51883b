// Gated residual and norm, t = x + alpha gate F, y = t / rms(t) (1 + scale) + shift, and its gradients.
//
// A row's statistics need the whole row, its values are used once: every row is read once, into registers, by
// 64, 256 or 512 threads of 4-element pieces, so a call moves the bytes that it has to and is bound by HBM.
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

// Sums over the TPR threads of a row.  `slot` alternates between consecutive calls (0, 1, 0, ...), so that one
// barrier a call is enough.
template <int TPR, int N>
RAVEL_DEV void row_sum(float (&v)[N], float (*part)[TPR / 64][4], int slot) {
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = wave_sum(v[i]);
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
      t[c] = rounded(t[c] + alpha * gate[c] * f[c], (const S*)nullptr);
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
// i % group where that is below rows.  A worker takes `per` modulation rows whole (segs 1), or rows [s seg, (s + 1) seg)
// of one.
struct GradPlan {
  int mods, group, count, per, segs, seg, workers;
  // where the sums go: to their place (one worker), or to the workspace, to be added
  bool mod_part, all_part;
  bool all[3];  // gate, scale, shift: summed over all rows
  float *gate, *scale, *shift, *post, *alpha;  // the sums of a modulation row (stride), or of a worker
  long long gate_stride, scale_stride, shift_stride;
  float* partial[5];  // the workspace's sums of dgate, dscale, dshift, dpost, dalpha; null: none
  size_t bytes;
};

int threads_per_row(int width) { return width <= 1024 ? 64 : width <= 4096 ? 256 : 512; }

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
  // At least 4 rows a worker, so that its sums are few beside its rows; 8 waves a CU keep enough loads in flight.
  const int most = n.width <= 1024 ? 2048 : n.width <= 4096 ? 768 : 512;
  const int rows = n.rows > p.mods ? n.rows : p.mods;
  int want = (rows + 3) / 4;
  want = want < 1 ? 1 : want > most ? most : want;
  if (p.mods >= want) {
    p.per = (p.mods + want - 1) / want;
    p.segs = 1;
    p.seg = p.count;
    p.workers = (p.mods + p.per - 1) / p.per;
  } else {
    p.per = 1;
    const int segs = want / p.mods;
    p.seg = (p.count + segs - 1) / segs;
    if (p.seg < 1) p.seg = 1;
    p.segs = (p.count + p.seg - 1) / p.seg;
    if (p.segs < 1) p.segs = 1;
    p.workers = p.mods * p.segs;
  }
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

// dn = dy (1 + scale); dt = d_out + r (dn - n mean(dn n)) with n = t r; dF = alpha gate dt; and through the block
// output's own norm, m = f rf, dm = dF (1 + post): df = rf (dm - m mean(dm m)).  The sums of t^2, dn t and f^2 are
// formed together; the last one needs dt and comes second.
template <typename S, typename T, int TPR, int NC>
__global__ __launch_bounds__(TPR * rows_per_block<TPR>()) void norm_residual_grad_kernel(ravel_norm a, ravel_norm_grad g,
                                                                                      GradPlan p) {
  __shared__ float part[2][TPR / 64][4];
  const int lane = threadIdx.x % TPR;
  const int worker = blockIdx.x * rows_per_block<TPR>() + threadIdx.x / TPR;
  if (worker >= p.workers) return;  // a whole wave; blocks of one worker have none
  const int m_beg = p.segs > 1 ? worker / p.segs : worker * p.per;
  const int m_end = min(p.mods, p.segs > 1 ? m_beg + 1 : m_beg + p.per);
  const int i_beg = p.segs > 1 ? worker % p.segs * p.seg : 0, i_end = min(p.count, i_beg + p.seg);
  const long long cycle = (long long)p.group * p.mods;
  const S* const t_in = (const S*)(a.f ? a.x_out : a.x);
  const long long t_stride = a.f ? a.x_out_stride : a.x_stride;
  const float alpha = a.f && a.alpha ? *a.alpha : 1.f, inv = 1.f / a.width;
  const bool want_f = a.f && (g.df || g.dpost || g.dgate || g.dalpha);

  f32x4_t s_gate[NC], s_scale[NC], s_shift[NC], s_post[NC];
  float s_alpha = 0.f;
#pragma unroll
  for (int c = 0; c < NC; ++c) s_gate[c] = s_scale[c] = s_shift[c] = s_post[c] = all4(0.f);
  // one of the three sums to its place, and from 0 on again
  const auto flush = [&](float* to, long long stride, size_t at, f32x4_t(&s)[NC]) {
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      const int col = (c * TPR + lane) * 4;
      if (to && col < a.width) store4(to + at * stride + col, s[c]);
      s[c] = all4(0.f);
    }
  };

  for (int m = m_beg; m < m_end; ++m) {
    for (int i = i_beg; i < i_end; ++i) {
      const long long row = i / p.group * cycle + (long long)m * p.group + i % p.group;
      if (row >= a.rows) break;
      const size_t mod = (row / a.group) % a.mods;
      f32x4_t t[NC], dn[NC], dt[NC], f[NC], gate[NC];
      float v[3] = {0.f, 0.f, 0.f};
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        const int col = (c * TPR + lane) * 4;
        t[c] = dn[c] = dt[c] = f[c] = all4(0.f);
        gate[c] = all4(1.f);
        if (col < a.width) {
          t[c] = load4(t_in + row * t_stride + col);
          if (g.dy) dn[c] = load4((const T*)g.dy + row * g.dy_stride + col);
          if (g.d_out) dt[c] = load4((const S*)g.d_out + row * g.d_out_stride + col);
          if (want_f) f[c] = load4((const T*)a.f + row * a.f_stride + col);
          if (want_f && a.gate) gate[c] = load4(a.gate + mod * a.gate_stride + col);
        }
      }
      f32x4_t dy[NC];
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        const int col = (c * TPR + lane) * 4;
        dy[c] = dn[c];
        if (a.scale && col < a.width) dn[c] = dn[c] * (load4(a.scale + mod * a.scale_stride + col) + 1.f);
        v[0] += sum4(t[c] * t[c]);
        v[1] += sum4(dn[c] * t[c]);
        v[2] += sum4(f[c] * f[c]);
      }
      row_sum<TPR>(v, part, 0);
      const float r = 1.f / sqrtf(v[0] * inv + a.eps), k = r * r * (v[1] * inv);
      const float rf = a.post ? 1.f / sqrtf(v[2] * inv + a.eps) : 1.f;
      float u[1] = {0.f};
      f32x4_t dm[NC];
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        const int col = (c * TPR + lane) * 4;
        const bool in = col < a.width;
        dt[c] += r * (dn[c] - k * t[c]);
        if (in && g.dx) store4((S*)g.dx + row * g.dx_stride + col, dt[c]);
        s_scale[c] += dy[c] * (t[c] * r);
        s_shift[c] += dy[c];
        if (want_f) {
          f[c] *= rf;  // m
          const f32x4_t post1 = a.post && in ? load4(a.post + col) + 1.f : all4(1.f);
          const f32x4_t d = dt[c] * f[c] * post1;  // dt F
          s_gate[c] += alpha * d;
          s_alpha += sum4(d * gate[c]);
          dm[c] = alpha * gate[c] * dt[c];  // dF
          s_post[c] += dm[c] * f[c];
          dm[c] *= post1;
          u[0] += sum4(dm[c] * f[c]);
        }
      }
      if (a.post && g.df) row_sum<TPR>(u, part, 1);
      if (g.df)
#pragma unroll
        for (int c = 0; c < NC; ++c) {
          const int col = (c * TPR + lane) * 4;
          if (col >= a.width) continue;
          const f32x4_t d = a.post ? rf * (dm[c] - (u[0] * inv) * f[c]) : dm[c];
          store4((T*)g.df + row * g.df_stride + col, d);
        }
      if constexpr (TPR > 64)
        if (!(a.post && g.df)) __syncthreads();  // the next row's first sum uses slot 0 again
    }
    const size_t at = p.mod_part ? worker : m;
    if (!p.all[0]) flush(p.gate, p.gate_stride, at, s_gate);
    if (!p.all[1]) flush(p.scale, p.scale_stride, at, s_scale);
    if (!p.all[2]) flush(p.shift, p.shift_stride, at, s_shift);
  }
  if (p.all[0]) flush(p.gate, p.gate_stride, worker, s_gate);
  if (p.all[1]) flush(p.scale, p.scale_stride, worker, s_scale);
  if (p.all[2]) flush(p.shift, p.shift_stride, worker, s_shift);
  flush(p.post, a.width, worker, s_post);
  if (p.alpha) {
    float v[1] = {s_alpha};
    row_sum<TPR>(v, part, 0);  // the last sum, if any, was slot 1's or has a barrier behind it
    if (lane == 0) p.alpha[worker] = v[0];
  }
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
  __shared__ f32x4_t part[16][16];
  const int quad = threadIdx.x & 15, slice = threadIdx.x >> 4;
  if (t.width == 1) {
    if (blockIdx.x) return;
    float s = 0.f;
    for (int i = threadIdx.x; i < t.n; i += 256) s += t.src[i];
    float* const f = (float*)part;
    f[threadIdx.x] = s;
    __syncthreads();
    if (threadIdx.x < 64) {
      s = wave_sum(f[threadIdx.x] + f[threadIdx.x + 64] + f[threadIdx.x + 128] + f[threadIdx.x + 192]);
      if (threadIdx.x == 0) t.dst[0] = s;
    }
    return;
  }
  const int col = blockIdx.x * 64 + quad * 4;
  f32x4_t s = all4(0.f);
  if (col < t.width)
    for (int i = slice; i < t.n; i += 16) s += load4(t.src + ((size_t)m * t.n + i) * t.width + col);
  part[slice][quad] = s;
  __syncthreads();
  if (slice == 0 && col < t.width) {
#pragma unroll
    for (int i = 1; i < 16; ++i) s += part[i][quad];
    store4(t.dst + m * t.stride + col, s);
  }
}

template <typename S, typename T, int TPR, int NC>
void launch_rows(const ravel_norm& n, const ravel_norm_grad* g, const GradPlan& p, hipStream_t s) {
  constexpr int R = rows_per_block<TPR>();
  if (g)
    norm_residual_grad_kernel<S, T, TPR, NC><<<(p.workers + R - 1) / R, TPR * R, 0, s>>>(n, *g, p);
  else
    norm_residual_kernel<S, T, TPR, NC><<<(n.rows + R - 1) / R, TPR * R, 0, s>>>(n);
}
template <typename S, typename T>
void launch_width(const ravel_norm& n, const ravel_norm_grad* g, const GradPlan& p, hipStream_t s) {
  if (n.width <= 256) launch_rows<S, T, 64, 1>(n, g, p, s);
  else if (n.width <= 512) launch_rows<S, T, 64, 2>(n, g, p, s);
  else if (n.width <= 1024) launch_rows<S, T, 64, 4>(n, g, p, s);
  else if (n.width <= 2048) launch_rows<S, T, 256, 2>(n, g, p, s);
  else if (n.width <= 4096) launch_rows<S, T, 256, 4>(n, g, p, s);
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
  norm_sum_kernel<<<dim3((n.width + 63) / 64, rows, count), 256, 0, s>>>(tasks);
  return hipGetLastError();
}

}  // namespace ravel
