// Cross attention, out = softmax(scale q k^T) v over k_len keys, and its gradients.
//
// No row masks another's keys, so the query heads of a KV head are one row space: row r of (batch row, KV head) is
// query row r / G of its G heads' head r % G, and every key and value tile is used by all of them.
//
// Rows are the columns of every result: s^T = K q^T leaves each lane 4 keys of one row, which is the operand of
// o^T = V^T p^T as it stands (lds_tile.h), with V's fragments read along columns.  Probabilities never leave
// registers, a row's maximum is one lane's business and two exchanges, and the running maximum and sum take one pass.
//
// The gradients are two passes over the same tiles, each writing what it owns, so that nothing is added by atomics:
// rows against all keys (dq; also each row's D = sum dout out), then keys against all rows (dk, dv).  That forms
// s and dout v^T twice, 7 products for 5.
//
// What bounds it with many rows: LDS.  Each of the four waves reads the fragments of a tile's 64 keys, and with the next
// tile's fill that takes 1.2 to 1.4 times as long as the products; exponentials come in between, and two waves a SIMD, all
// that the sums leave registers for, cover each other in part: matrix instructions are busy 45 % of the time in the forward, 50 %
// for dq, 54 % for dk and dv.  16 x 800 rows of 16 heads over 2048 keys of 4 heads, 128 dims: forward 250 us (860 TFLOP/s), dq 341
// (945), dk and dv 384 (1118); with lengths of 512 to 2048 and one of 0, 144, 202 and 346.  The last does not shrink as the
// keys do: its 1024 blocks of 128 keys are equally long, some 630 of them live, which is two rounds of 512, the second a quarter full.
//
// What a bf16 call rounds: probabilities before p v and p^T dout, the scores' gradients before ds k and ds^T q (operands of
// bf16 matrix instructions; 2.3e-3 off 64 bits with the results' own rounding, which alone makes 1.7e-3), and D takes out as the
// forward has rounded it: exact sums would need the keys once more.  That is little where many keys share the weight, and
// most of the error where one key has it all (a mean largest probability of 0.89: 5.9e-3).  Calls in 32 bits round nothing between.
#include <algorithm>

#include "layer.h"
#include "lds_tile.h"

namespace ravel {
namespace {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f, kLazy = 8.f;

// Whether the gradients' scores start from -lse / scale, which saves an addition a probability (dk, dv of 16 x 800 rows
// over 2048 keys: 422 us from 451) but rounds every partial sum at the size of lse / scale: under bf16's rounding of the
// probabilities nothing, in 32 bits 2.6 times the error.
template <typename T> constexpr bool kStart = sizeof(T) == 2;

struct CrossArgs {
  ravel_cross c;
  ravel_cross_grad g;
  int G, tiles, splits;  // query heads of a KV head; tiles of what the blocks own; ranges of what they walk
  int padded;            // rows of stat per (batch row, KV head): whole tiles of the pass that writes it
  float* part;           // partial results [split][batch][KV head][row or key][head_dim], or null
  float* part_ml;        // forward: [split][batch][KV head][row][2], maximum (log2 units) and sum
  float* stat;           // gradients: [2][batch][KV head][padded]: -lse / scale (f32: -lse log2 e) and -D
  float* part2;          // dv's partials
};

RAVEL_DEV int live_len(const int* len, int b, int most) { return len ? min(max(len[b], 0), most) : most; }

template <typename T> RAVEL_DEV void store_row4(T* p, f32x4_t v);
template <> RAVEL_DEV void store_row4<float>(float* p, f32x4_t v) { *(f32x4_t*)p = v; }
template <> RAVEL_DEV void store_row4<bf16_t>(bf16_t* p, f32x4_t v) {
  *(u32x2_t*)p = u32x2_t{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
}
// 32 columns of row l16, two blocks (all lanes of a row take part)
RAVEL_DEV void store_blocks(float* row, int lane, f32x4_t v, f32x4_t w) {
  store_row4(row + (lane >> 4) * 4, v);
  store_row4(row + 16 + (lane >> 4) * 4, w);
}
RAVEL_DEV void store_blocks(bf16_t* row, int lane, f32x4_t v, f32x4_t w) { *(u32x4_t*)(row + joined_column(lane)) = join_blocks(v, w); }
RAVEL_DEV float dot16(f32x4_t a, f32x4_t b) { return (a[0] * b[0] + a[1] * b[1]) + (a[2] * b[2] + a[3] * b[3]); }
RAVEL_DEV float dot16(bf16x8_t a, bf16x8_t b) {
  const u32x4_t x = __builtin_bit_cast(u32x4_t, a), y = __builtin_bit_cast(u32x4_t, b);
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    s += __uint_as_float(x[i] << 16) * __uint_as_float(y[i] << 16) +
         __uint_as_float(x[i] & 0xFFFF0000u) * __uint_as_float(y[i] & 0xFFFF0000u);
  return s;
}

// A value of the four lanes that hold a column's parts (lanes l16 + 16 g), combined.
RAVEL_DEV float column_max(float x) {
  auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
  r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
RAVEL_DEV float column_sum(float x) {
  auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// A block's tile, range, KV head and batch row.  Neighbouring blocks, which run on different XCDs, take the tiles of one
// head: lengths differ from batch row to batch row, and where every XCD had heads of its own (their keys in one L2) the one
// with the longest rows ended last, 203 us instead of 149 for 16 batch rows of up to 2048 keys.  Tiles are
// turned by the head, so that those behind a length do not all fall to one XCD either.
struct Work {
  int tile, h, b, split;
};
RAVEL_DEV Work work_of(const CrossArgs& a) {
  const unsigned id = blockIdx.x, head = id / (a.tiles * a.splits), in = id - head * (a.tiles * a.splits);
  Work w;
  w.split = in / a.tiles;
  w.tile = (in - w.split * a.tiles + head) % a.tiles;
  w.h = head % a.c.n_kv_heads, w.b = head / a.c.n_kv_heads;
  return w;
}

// K and V tiles (or q and dout): sizes and what a wave loads.
template <typename T, int HD, int ROWS>
struct Tiles {
  static constexpr int RB = HD * sizeof(T), BYTES = ROWS * RB, SEGS = (BYTES + 4095) / 4096;  // segments per wave
};

// Keys [first, first + TK) of one head into a tile; keys from `end` on are zeros (by their index: their memory may be a live key's).
template <typename T, int HD, int TK>
RAVEL_DEV void load_keys(const Segments<T, HD * sizeof(T)>& at, const T* head, int stride, int first, int end, char* tile, int wave) {
  typedef Tiles<T, HD, TK> Z;
  const unsigned step = (unsigned)stride * (unsigned)sizeof(T), row = __umul24(at.row, step);
  const rsrc_t from = buffer_from((const char*)head + (int64_t)first * (int)step);
#pragma unroll
  for (int i = 0; i < Z::SEGS; ++i) {
    const int seg = wave * Z::SEGS + i;
    if (Z::BYTES % 4096 && seg * 1024 >= Z::BYTES) break;
    load_segment(from, tile, seg, seg * at.ROWS + at.row < end - first ? row + at.byte_of(seg) + seg * at.ROWS * step : kOutside);
  }
}
// Rows [first, first + TR) of a (batch row, KV head)'s row space; rows from `end` on are zeros, or with REPEAT the last row
// (there is one) again.  head: row 0 of the first query head.  Quotients by G through its reciprocal `inv` = ceil(2^23 / G), exact
// for what is below 2^23 / G.
struct RowSpace {
  int G, inv;
};
template <typename T, int HD, int TR, bool REPEAT = false>
RAVEL_DEV void load_rows(const Segments<T, HD * sizeof(T)>& at, const T* head, int64_t row_stride, int head_stride, RowSpace sp, int first,
                         int end, char* tile, int wave) {
  typedef Tiles<T, HD, TR> Z;
  const int i0 = first / sp.G, rest = first - i0 * sp.G, last = end - 1 - first;
  const rsrc_t from = buffer_from(head + i0 * row_stride);
#pragma unroll
  for (int i = 0; i < Z::SEGS; ++i) {
    const int seg = wave * Z::SEGS + i, r = seg * at.ROWS + at.row;
    if (Z::BYTES % 4096 && seg * 1024 >= Z::BYTES) break;
    const unsigned x = rest + (REPEAT ? min(r, last) : r), q = __umul24(x, sp.inv) >> 23, g = x - __umul24(q, sp.G);
    const unsigned off = __umul24(q, (unsigned)row_stride * (unsigned)sizeof(T)) + __umul24(g, head_stride * (unsigned)sizeof(T));
    load_segment(from, tile, seg, REPEAT || r <= last ? off + at.byte_of(seg) : kOutside);
  }
}

// ---------------------------------------------------------------------------
// forward
// ---------------------------------------------------------------------------
// Four waves: KW of them share 16 MI rows and split a tile's keys between them (few rows), 4 / KW groups of rows.  Few rows
// are bound by HBM: 64 batch rows of one row over up to 4096 keys, 64 us and 6 to join the ranges, 5.2 TB/s, where a bare read of
// 320 MB has 6.5.
template <typename T, int HD, int MI, int KW, int TK>
__global__ __launch_bounds__(256, (4 * Tiles<T, HD, TK>::BYTES <= 65536 ? 2 : 1)) void cross_kernel(CrossArgs a) {
  typedef Tiles<T, HD, TK> Z;
  typedef Mat<T> M;
  typedef typename M::frag frag;
  constexpr int RB = Z::RB, STEPS = RB / 64, DF = HD / 16, TKW = TK / KW, NF = TKW / 16, NP = TKW / M::CK;
  static_assert(TKW % M::CK == 0, "whole contraction steps");
  constexpr int JOIN = KW > 1 ? 16 * MI * (HD + 2) * 4 : 0;  // bytes of a wave's results
  static_assert(JOIN <= Z::BYTES, "a wave's results in a tile");
  // Four arrays: reads along columns of one buffer wait for the loads in flight into another unless the compiler sees
  // that they are apart.
  __shared__ __attribute__((aligned(1024))) char k0[Z::BYTES], v0[Z::BYTES], k1[Z::BYTES], v1[Z::BYTES];

  const int lane = threadIdx.x & 63, wave = wave_index(), l16 = lane & 15, grp = lane >> 4;
  const int wk = wave % KW, wr = wave / KW;
  const ravel_cross& c = a.c;
  const Work w = work_of(a);
  const int live = live_len(c.q_len, w.b, c.rows) * a.G, all = c.rows * a.G;
  const int klen = live_len(c.k_len, w.b, c.keys);
  const int first = w.tile * (16 * MI * (4 / KW)), row0 = first + wr * 16 * MI;  // the block's rows, this wave's
  const int ktiles = first < live ? (klen + TK - 1) / TK : 0, per = (ktiles + a.splits - 1) / a.splits;
  const int t0 = min(ktiles, w.split * per), t1 = min(ktiles, t0 + per);

  const T* const q = (const T*)c.q + w.b * c.q_stride[0] + (int64_t)w.h * a.G * c.q_stride[2];
  const T* const k = (const T*)c.k + w.b * c.k_stride[0] + w.h * c.k_stride[2];
  const T* const v = (const T*)c.v + w.b * c.v_stride[0] + w.h * c.v_stride[2];
  const Segments<T, RB> seg0(lane);
  const auto issue = [&](int t, char* kt, char* vt) {
    const auto seg = seg0.fresh();
    load_keys<T, HD, TK>(seg, k, (int)c.k_stride[1], t * TK, klen, kt, wave);
    load_keys<T, HD, TK>(seg, v, (int)c.v_stride[1], t * TK, klen, vt, wave);
  };
  if (t0 < t1) issue(t0, k0, v0);

  frag qf[MI][STEPS];
#pragma unroll
  for (int i = 0; i < MI; ++i) {
    const int r = row0 + i * 16 + l16, qr = r / a.G;
    const T* const p = q + qr * c.q_stride[1] + (r - qr * a.G) * c.q_stride[2];
#pragma unroll
    for (int s = 0; s < STEPS; ++s) qf[i][s] = r < live && c.scale > 0.f ? *(const frag*)(p + (s * 4 + grp) * (16 / sizeof(T))) : frag{};
  }
  const float cs = c.scale > 0.f ? c.scale * kLog2e : 1.f;  // (a scale of 0: rows of zeros, so that -infinity stays)
  f32x4_t o[MI][DF];
  float m[MI], l[MI];
#pragma unroll
  for (int i = 0; i < MI; ++i) {
    m[i] = -INFINITY, l[i] = 0.f;
#pragma unroll
    for (int d = 0; d < DF; ++d) o[i][d] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  }
  const TileLane<T, RB> at0(lane);

  // Keys that do not exist start from -infinity: the last tile's, whose rows are zeros.  (A select behind the products,
  // under a branch, read them too early: the compiler leaves out wait states where a branch skips a few instructions
  // between matrix instructions and their results' use.)
  f32x4_t start[NF];
#pragma unroll
  for (int f = 0; f < NF; ++f) start[f] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  const auto step = [&](int t, const char* kc, const char* vc, char* kn, char* vn) {
    tile_barrier<0>();
    if (t + 1 < t1) issue(t + 1, kn, vn);
    if (row0 >= live) return;  // (a wave without rows, or without keys in this tile, has loaded its part)
    if (KW > 1 && t * TK + wk * TKW >= klen) return;
    lds_char_t* const kt = (lds_char_t*)kc + wk * TKW * RB;
    lds_char_t* const vt = (lds_char_t*)vc + wk * TKW * RB;
    if (t == ktiles - 1) {
      const int left = klen - t * TK - wk * TKW - grp * 4;
#pragma unroll
      for (int f = 0; f < NF; ++f)
#pragma unroll
        for (int r = 0; r < 4; ++r) start[f][r] = f * 16 + r < left ? 0.f : -INFINITY;
    }
    auto at = at0.fresh();
    f32x4_t s[MI][NF];
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
      for (int f = 0; f < NF; ++f) s[i][f] = start[f];
#pragma unroll
    for (int f = 0; f < NF; ++f)
#pragma unroll
      for (int st = 0; st < STEPS; ++st) {
        const frag kf = at.along_row(kt, f, st);
#pragma unroll
        for (int i = 0; i < MI; ++i) s[i][f] = M::mma(kf, qf[i][st], s[i][f]);
      }
    frag pf[MI][NP];
#pragma unroll
    for (int i = 0; i < MI; ++i) {
      float top = -INFINITY;
#pragma unroll
      for (int f = 0; f < NF; ++f)
#pragma unroll
        for (int r = 0; r < 4; ++r) top = fmaxf(top, s[i][f][r]);
      top = column_max(top) * cs;
      // The reference moves only where the maximum is past it by kLazy (log2 units): probabilities stay below 2^kLazy,
      // and what was summed is scaled rarely.
      if (__any(top > m[i] + kLazy)) {
        const float to = fmaxf(m[i], top), fall = __builtin_amdgcn_exp2f(m[i] - (to == -INFINITY ? 0.f : to));
        l[i] *= fall;
#pragma unroll
        for (int d = 0; d < DF; ++d) o[i][d] *= fall;
        m[i] = to;
      }
      const float ref = m[i] == -INFINITY ? 0.f : m[i];
#pragma unroll
      for (int f = 0; f < NF; ++f)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          s[i][f][r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i][f][r], cs, -ref));
          l[i] += s[i][f][r];
        }
#pragma unroll
      for (int p = 0; p < NP; ++p) pf[i][p] = M::operand(&s[i][p * (NF / NP)]);
    }
    at = at0.fresh();
#pragma unroll
    for (int d = 0; d < DF; ++d)
#pragma unroll
      for (int p = 0; p < NP; ++p) {
        const frag vf = at.along_col(vt, p, d);
#pragma unroll
        for (int i = 0; i < MI; ++i) o[i][d] = M::mma(vf, pf[i][p], o[i][d]);
      }
  };
  for (int t = t0; t < t1; t += 2) {
    step(t, k0, v0, k1, v1);
    if (t + 1 < t1) step(t + 1, k1, v1, k0, v0);
  }
  results_ready(o);
#pragma unroll
  for (int i = 0; i < MI; ++i) l[i] = column_sum(l[i]);
  if constexpr (KW > 1) {  // the waves that share rows: wave wk = 0 takes their sum
    __syncthreads();
    const auto results = [&](int w) { return (float*)(w == 0 ? k0 : w == 1 ? v0 : w == 2 ? k1 : v1); };
    float* const mine = results(wave);
#pragma unroll
    for (int i = 0; i < MI; ++i) {
      float* const p = mine + (i * 16 + l16) * (HD + 2);
      if (wk > 0) {
#pragma unroll
        for (int d = 0; d < DF; ++d)
#pragma unroll
          for (int r = 0; r < 4; ++r) p[d * 16 + grp * 4 + r] = o[i][d][r];
        if (grp == 0) p[HD] = m[i], p[HD + 1] = l[i];
      }
    }
    __syncthreads();
    if (wk > 0) return;
#pragma unroll
    for (int j = 1; j < KW; ++j)
#pragma unroll
      for (int i = 0; i < MI; ++i) {
        const float* const p = results(wave + j) + (i * 16 + l16) * (HD + 2);
        const float mj = p[HD], top = fmaxf(m[i], mj), ref = top == -INFINITY ? 0.f : top;
        const float fa = __builtin_amdgcn_exp2f(m[i] - ref), fb = __builtin_amdgcn_exp2f(mj - ref);
        m[i] = top;
        l[i] = l[i] * fa + p[HD + 1] * fb;
#pragma unroll
        for (int d = 0; d < DF; ++d)
#pragma unroll
          for (int r = 0; r < 4; ++r) o[i][d][r] = o[i][d][r] * fa + p[d * 16 + grp * 4 + r] * fb;
      }
  }
#pragma unroll
  for (int i = 0; i < MI; ++i) {
    const int r = row0 + i * 16 + l16;
    if (r >= all) continue;
    if (a.part) {
      const size_t at = (((size_t)w.split * c.batch + w.b) * c.n_kv_heads + w.h) * all + r;
#pragma unroll
      for (int d = 0; d < DF; ++d) *(f32x4_t*)(a.part + at * HD + d * 16 + grp * 4) = o[i][d];
      if (grp == 0) a.part_ml[at * 2] = m[i], a.part_ml[at * 2 + 1] = l[i];
      continue;
    }
    const int qr = r / a.G, g = r - qr * a.G;
    const bool any = r < live && klen > 0;
    const float f = any ? 1.f / l[i] : 0.f;
    const f32x4_t zero = {0.f, 0.f, 0.f, 0.f};
    T* const out = (T*)c.out + w.b * c.out_stride[0] + qr * c.out_stride[1] + (int64_t)(w.h * a.G + g) * c.out_stride[2];
#pragma unroll
    for (int d = 0; d < DF; d += 2) store_blocks(out + d * 16, lane, any ? o[i][d] * f : zero, any ? o[i][d + 1] * f : zero);
    if (c.lse && grp == 0)
      c.lse[((size_t)w.b * c.n_q_heads + w.h * a.G + g) * c.rows + qr] = any ? m[i] * kLn2 + logf(l[i]) : -INFINITY;
  }
}

// Key ranges joined: a thread takes 4 dims of a row.
template <typename T>
__global__ __launch_bounds__(256) void cross_join_kernel(CrossArgs a) {
  const ravel_cross& c = a.c;
  const int hd4 = c.head_dim / 4, all = c.rows * a.G;
  const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x, n = (int64_t)c.batch * c.n_kv_heads * all;
  if (id >= n * hd4) return;
  const int64_t at = id / hd4;
  const int d = (int)(id - at * hd4) * 4, r = (int)(at % all), h = (int)(at / all % c.n_kv_heads);
  const int b = (int)(at / all / c.n_kv_heads);
  const int qr = r / a.G, g = r - qr * a.G;
  const bool any = r < live_len(c.q_len, b, c.rows) * a.G && live_len(c.k_len, b, c.keys) > 0;
  float m = -INFINITY, l = 0.f;
  f32x4_t o = {0.f, 0.f, 0.f, 0.f};
  if (any) {
    for (int s = 0; s < a.splits; ++s) m = fmaxf(m, a.part_ml[(s * n + at) * 2]);
    const float ref = m == -INFINITY ? 0.f : m;
    for (int s = 0; s < a.splits; ++s) {
      const float f = __builtin_amdgcn_exp2f(a.part_ml[(s * n + at) * 2] - ref);
      l += f * a.part_ml[(s * n + at) * 2 + 1];
      o += f * *(const f32x4_t*)(a.part + (s * n + at) * c.head_dim + d);
    }
    o *= 1.f / l;
  }
  store_row4<T>((T*)c.out + b * c.out_stride[0] + qr * c.out_stride[1] + (int64_t)(h * a.G + g) * c.out_stride[2] + d, o);
  if (c.lse && d == 0) c.lse[((size_t)b * c.n_q_heads + h * a.G + g) * c.rows + qr] = any ? m * kLn2 + logf(l) : -INFINITY;
}

// ---------------------------------------------------------------------------
// dq (and D): KW waves share 16 MI rows and split a tile's keys between them, the block walks the keys
// ---------------------------------------------------------------------------
template <typename T, int HD, int MI, int KW, int TK>
__global__ __launch_bounds__(256, (4 * Tiles<T, HD, TK>::BYTES <= 65536 ? 2 : 1)) void cross_dq_kernel(CrossArgs a) {
  typedef Tiles<T, HD, TK> Z;
  typedef Mat<T> M;
  typedef typename M::frag frag;
  constexpr int RB = Z::RB, STEPS = RB / 64, DF = HD / 16, TKW = TK / KW, NP = TKW / M::CK, FP = M::CK / 16;
  static_assert(TKW % M::CK == 0 && (KW == 1 || 16 * MI * HD * 4 <= Z::BYTES), "whole contraction steps, a wave's sums in a tile");
  __shared__ __attribute__((aligned(1024))) char k0[Z::BYTES], v0[Z::BYTES], k1[Z::BYTES], v1[Z::BYTES];

  const int lane = threadIdx.x & 63, wave = wave_index(), l16 = lane & 15, grp = lane >> 4;
  const int wk = wave % KW, wr = wave / KW;
  const ravel_cross& c = a.c;
  const ravel_cross_grad& g = a.g;
  const Work w = work_of(a);
  const int live = live_len(c.q_len, w.b, c.rows) * a.G, all = c.rows * a.G;
  const int klen = live_len(c.k_len, w.b, c.keys);
  const int first = w.tile * (16 * MI * (4 / KW)), row0 = first + wr * 16 * MI;
  const int ktiles = g.dq && first < live ? (klen + TK - 1) / TK : 0, per = (ktiles + a.splits - 1) / a.splits;
  const int t0 = min(ktiles, w.split * per), t1 = min(ktiles, t0 + per);

  const T* const k = (const T*)c.k + w.b * c.k_stride[0] + w.h * c.k_stride[2];
  const T* const v = (const T*)c.v + w.b * c.v_stride[0] + w.h * c.v_stride[2];
  const Segments<T, RB> seg0(lane);
  const auto issue = [&](int t, char* kt, char* vt) {
    const auto seg = seg0.fresh();
    load_keys<T, HD, TK>(seg, k, (int)c.k_stride[1], t * TK, klen, kt, wave);
    load_keys<T, HD, TK>(seg, v, (int)c.v_stride[1], t * TK, klen, vt, wave);
  };
  if (t0 < t1) issue(t0, k0, v0);

  frag qf[MI][STEPS], of[MI][STEPS];  // of: dout
  const float cs = c.scale > 0.f ? c.scale * kLog2e : 1.f;
  float lse[MI], D[MI];  // negative; what the sums start from, so that p = exp2(cs s) and ds = p dp, but see kStart
#pragma unroll
  for (int i = 0; i < MI; ++i) {
    const int r = row0 + i * 16 + l16, qr = r / a.G, gh = w.h * a.G + r - qr * a.G;
    const bool in = r < live;
    const T* const pq = (const T*)c.q + w.b * c.q_stride[0] + qr * c.q_stride[1] + gh * c.q_stride[2];
    const T* const po = (const T*)c.out + w.b * c.out_stride[0] + qr * c.out_stride[1] + gh * c.out_stride[2];
    const T* const pd = (const T*)g.dout + w.b * g.dout_stride[0] + qr * g.dout_stride[1] + gh * g.dout_stride[2];
    D[i] = 0.f;
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
      const int e = (s * 4 + grp) * (16 / sizeof(T));
      qf[i][s] = in && c.scale > 0.f ? *(const frag*)(pq + e) : frag{};
      of[i][s] = in ? *(const frag*)(pd + e) : frag{};
      D[i] += dot16(of[i][s], in ? *(const frag*)(po + e) : frag{});
    }
    D[i] = -column_sum(D[i]);
    lse[i] = in ? -(c.lse[((size_t)w.b * c.n_q_heads + gh) * c.rows + qr] * kLog2e / (kStart<T> ? cs : 1.f)) : -INFINITY;
    if (a.stat && grp == 0 && wk == 0 && w.split == 0) {
      float* const p = a.stat + ((size_t)w.b * c.n_kv_heads + w.h) * a.padded + r;
      p[0] = lse[i];
      p[(size_t)c.batch * c.n_kv_heads * a.padded] = D[i];
    }
  }
  if (!g.dq) return;
  f32x4_t dq[MI][DF];
#pragma unroll
  for (int i = 0; i < MI; ++i)
#pragma unroll
    for (int d = 0; d < DF; ++d) dq[i][d] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  const TileLane<T, RB> at0(lane);

  f32x4_t start[TKW / 16];  // as in the forward: keys that do not exist
#pragma unroll
  for (int f = 0; f < TKW / 16; ++f) start[f] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  const auto step = [&](int t, const char* kc, const char* vc, char* kn, char* vn) {
    tile_barrier<0>();
    if (t + 1 < t1) issue(t + 1, kn, vn);
    if (row0 >= live) return;  // (a wave without rows, or without keys in this tile, has loaded its part)
    if (KW > 1 && t * TK + wk * TKW >= klen) return;
    lds_char_t* const kt = (lds_char_t*)kc + wk * TKW * RB;
    lds_char_t* const vt = (lds_char_t*)vc + wk * TKW * RB;
    if (t == ktiles - 1) {
      const int left = klen - t * TK - wk * TKW - grp * 4;
#pragma unroll
      for (int f = 0; f < TKW / 16; ++f)
#pragma unroll
        for (int r = 0; r < 4; ++r) start[f][r] = f * 16 + r < left ? 0.f : -INFINITY;
    }
#pragma unroll
    for (int p = 0; p < NP; ++p) {
      const auto at = at0.fresh();
      f32x4_t s[MI][FP], dp[MI][FP];
#pragma unroll
      for (int f = 0; f < FP; ++f) {
#pragma unroll
        for (int i = 0; i < MI; ++i) s[i][f] = kStart<T> ? start[p * FP + f] + lse[i] : start[p * FP + f], dp[i][f] = f32x4_t{D[i], D[i], D[i], D[i]};
#pragma unroll
        for (int st = 0; st < STEPS; ++st) {
          const frag kf = at.along_row(kt, p * FP + f, st), vf = at.along_row(vt, p * FP + f, st);
#pragma unroll
          for (int i = 0; i < MI; ++i) {
            s[i][f] = M::mma(kf, qf[i][st], s[i][f]);
            dp[i][f] = M::mma(vf, of[i][st], dp[i][f]);
          }
        }
      }
      frag ds[MI];
#pragma unroll
      for (int i = 0; i < MI; ++i) {
#pragma unroll
        for (int f = 0; f < FP; ++f)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            s[i][f][r] = __builtin_amdgcn_exp2f(kStart<T> ? s[i][f][r] * cs : __builtin_fmaf(s[i][f][r], cs, lse[i])) * dp[i][f][r];
          }
        ds[i] = M::operand(s[i]);
      }
#pragma unroll
      for (int d = 0; d < DF; ++d) {
        const frag kf = at.along_col(kt, p, d);
#pragma unroll
        for (int i = 0; i < MI; ++i) dq[i][d] = M::mma(kf, ds[i], dq[i][d]);
      }
    }
  };
  for (int t = t0; t < t1; t += 2) {
    step(t, k0, v0, k1, v1);
    if (t + 1 < t1) step(t + 1, k1, v1, k0, v0);
  }
  results_ready(dq);
  if constexpr (KW > 1) {  // the waves that share rows: wave wk = 0 takes their sum
    const auto sums = [&](int w) { return (float*)(w == 0 ? k0 : w == 1 ? v0 : w == 2 ? k1 : v1); };
    __syncthreads();
    if (wk > 0)
#pragma unroll
      for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int d = 0; d < DF; ++d) *(f32x4_t*)(sums(wave) + (i * DF + d) * 256 + lane * 4) = dq[i][d];
    __syncthreads();
    if (wk > 0) return;
#pragma unroll
    for (int j = 1; j < KW; ++j)
#pragma unroll
      for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int d = 0; d < DF; ++d) dq[i][d] += *(const f32x4_t*)(sums(wave + j) + (i * DF + d) * 256 + lane * 4);
  }
#pragma unroll
  for (int i = 0; i < MI; ++i) {
    const int r = row0 + i * 16 + l16;
    if (r >= all) continue;
    if (a.part) {
      const size_t to = (((size_t)w.split * c.batch + w.b) * c.n_kv_heads + w.h) * all + r;
#pragma unroll
      for (int d = 0; d < DF; ++d) *(f32x4_t*)(a.part + to * HD + d * 16 + grp * 4) = dq[i][d];
      continue;
    }
    const int qr = r / a.G, gh = w.h * a.G + r - qr * a.G;
    const f32x4_t zero = {0.f, 0.f, 0.f, 0.f};
    T* const to = (T*)g.dq + w.b * g.dq_stride[0] + qr * g.dq_stride[1] + gh * g.dq_stride[2];
#pragma unroll
    for (int d = 0; d < DF; d += 2)
      store_blocks(to + d * 16, lane, r < live ? dq[i][d] * c.scale : zero, r < live ? dq[i][d + 1] * c.scale : zero);
  }
}

// ---------------------------------------------------------------------------
// dk, dv: RW waves share 16 KI keys and split a tile's rows between them, the block walks the rows
// ---------------------------------------------------------------------------
template <typename T, int HD, int KI, int RW, int TR>
__global__ __launch_bounds__(256, (4 * Tiles<T, HD, TR>::BYTES <= 65536 && Tiles<T, HD, TR>::RB < 1024 ? 2 : 1)) void cross_dkv_kernel(CrossArgs a) {
  typedef Tiles<T, HD, TR> Z;
  typedef Mat<T> M;
  typedef typename M::frag frag;
  constexpr int RB = Z::RB, STEPS = RB / 64, DF = HD / 16, TRW = TR / RW, NP = TRW / M::CK, FP = M::CK / 16;
  static_assert(TRW % M::CK == 0, "whole contraction steps");
  static_assert(RW == 1 || 16 * KI * HD * 4 <= Z::BYTES, "a wave's sums in a tile");
  constexpr int TS = TR < 64 ? 64 : TR;  // a tile's lse and D, 64 a load
  __shared__ __attribute__((aligned(1024))) char q0[Z::BYTES], o0[Z::BYTES], q1[Z::BYTES], o1[Z::BYTES];  // o: dout
  __shared__ __attribute__((aligned(1024))) float s0[2 * TS], s1[2 * TS];

  const int lane = threadIdx.x & 63, wave = wave_index(), l16 = lane & 15, grp = lane >> 4;
  const int wr = wave % RW, wk = wave / RW;
  const ravel_cross& c = a.c;
  const ravel_cross_grad& g = a.g;
  const Work w = work_of(a);
  const int live = live_len(c.q_len, w.b, c.rows) * a.G;
  const int klen = live_len(c.k_len, w.b, c.keys);
  const int first = w.tile * (16 * KI * (4 / RW)), key0 = first + wk * 16 * KI;
  const int rtiles = first < klen ? (live + TR - 1) / TR : 0, per = (rtiles + a.splits - 1) / a.splits;
  const int t0 = min(rtiles, w.split * per), t1 = min(rtiles, t0 + per);

  const T* const q = (const T*)c.q + w.b * c.q_stride[0] + (int64_t)w.h * a.G * c.q_stride[2];
  const T* const dout = (const T*)g.dout + w.b * g.dout_stride[0] + (int64_t)w.h * a.G * g.dout_stride[2];
  const float* const stat = a.stat + ((size_t)w.b * c.n_kv_heads + w.h) * a.padded;
  const size_t apart = (size_t)c.batch * c.n_kv_heads * a.padded;  // from lse to D
  const RowSpace space{a.G, ((1 << 23) + a.G - 1) / a.G};
  const Segments<T, RB> seg0(lane);
  // Rows that do not exist take part as the last one again, with zeros for dout and D: their gradients are 0 times what the last
  // row has (as rows of zeros they would make an infinite key's score 0 times infinity).
  const auto issue = [&](int t, char* qt, char* ot, float* st) {
    const auto seg = seg0.fresh();
    if (wave < 2) {  // one of lse and D (through LDS: loads into registers would wait for the tiles issued before them)
      const rsrc_t from = buffer_from(stat + wave * apart + t * TR);
      const int last = live - t * TR - 1;
      const unsigned behind = wave == 0 ? last * 4u : kOutside;
#pragma unroll
      for (int i = 0; i < TS / 64; ++i)
        __builtin_amdgcn_raw_ptr_buffer_load_lds(from, (lds_dst_t*)(st + wave * TS + i * 64), 4,
                                                 (int)(i * 64 + lane <= last ? (i * 64 + lane) * 4u : behind), 0, 0, 0);
    }
    load_rows<T, HD, TR, true>(seg, q, c.q_stride[1], (int)c.q_stride[2], space, t * TR, live, qt, wave);
    load_rows<T, HD, TR>(seg, dout, g.dout_stride[1], (int)g.dout_stride[2], space, t * TR, live, ot, wave);
  };
  if (t0 < t1) issue(t0, q0, o0, s0);

  frag kf[KI][STEPS], vf[KI][STEPS];
#pragma unroll
  for (int i = 0; i < KI; ++i) {
    const int key = key0 + i * 16 + l16;
    const T* const pk = (const T*)c.k + w.b * c.k_stride[0] + key * c.k_stride[1] + w.h * c.k_stride[2];
    const T* const pv = (const T*)c.v + w.b * c.v_stride[0] + key * c.v_stride[1] + w.h * c.v_stride[2];
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
      const int e = (s * 4 + grp) * (16 / sizeof(T));
      kf[i][s] = key < klen && c.scale > 0.f ? *(const frag*)(pk + e) : frag{};
      vf[i][s] = key < klen ? *(const frag*)(pv + e) : frag{};
    }
  }
  const float cs = c.scale > 0.f ? c.scale * kLog2e : 1.f;
  f32x4_t dk[KI][DF], dv[KI][DF];
#pragma unroll
  for (int i = 0; i < KI; ++i)
#pragma unroll
    for (int d = 0; d < DF; ++d) dk[i][d] = dv[i][d] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  const TileLane<T, RB> at0(lane);

  const auto step = [&](int t, const char* qc, const char* oc, const float* sc, char* qn, char* on, float* sn) {
    tile_barrier<0>();
    if (t + 1 < t1) issue(t + 1, qn, on, sn);
    RAVEL_LDS const float* const st = (RAVEL_LDS const float*)sc + wr * TRW + grp * 4;
    if (key0 >= klen || (RW > 1 && t * TR + wr * TRW >= live)) return;  // nothing for this wave
    lds_char_t* const qt = (lds_char_t*)qc + wr * TRW * RB;
    lds_char_t* const ot = (lds_char_t*)oc + wr * TRW * RB;
#pragma unroll
    for (int p = 0; p < NP; ++p) {
      if (sizeof(T) == 4 && p > 0 && t * TR + wr * TRW + p * M::CK >= live) break;  // (32-bit products take long: 71 rows over 2499 keys 193 us from 219, with the forward and dq)
      const auto at = at0.fresh();
      f32x4_t s[KI][FP], dp[KI][FP], lse[FP];
#pragma unroll
      for (int f = 0; f < FP; ++f) {
        const f32x4_t s0 = *(RAVEL_LDS const f32x4_t*)(st + (p * FP + f) * 16), dp0 = *(RAVEL_LDS const f32x4_t*)(st + TS + (p * FP + f) * 16);
#pragma unroll
        for (int i = 0; i < KI; ++i) s[i][f] = kStart<T> ? s0 : f32x4_t{0.f, 0.f, 0.f, 0.f}, dp[i][f] = dp0;
        if (!kStart<T>) lse[f] = s0;
#pragma unroll
        for (int x = 0; x < STEPS; ++x) {
          const frag qf = at.along_row(qt, p * FP + f, x), of = at.along_row(ot, p * FP + f, x);
#pragma unroll
          for (int i = 0; i < KI; ++i) {
            s[i][f] = M::mma(qf, kf[i][x], s[i][f]);
            dp[i][f] = M::mma(of, vf[i][x], dp[i][f]);
          }
        }
      }
      frag pf[KI], ds[KI];
#pragma unroll
      for (int i = 0; i < KI; ++i) {
#pragma unroll
        for (int f = 0; f < FP; ++f)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            s[i][f][r] = __builtin_amdgcn_exp2f(kStart<T> ? s[i][f][r] * cs : __builtin_fmaf(s[i][f][r], cs, lse[f][r]));
            dp[i][f][r] *= s[i][f][r];
          }
        pf[i] = M::operand(s[i]);
        ds[i] = M::operand(dp[i]);
      }
#pragma unroll
      for (int d = 0; d < DF; ++d) {
        const frag of = at.along_col(ot, p, d), qf = at.along_col(qt, p, d);
#pragma unroll
        for (int i = 0; i < KI; ++i) {
          dv[i][d] = M::mma(of, pf[i], dv[i][d]);
          dk[i][d] = M::mma(qf, ds[i], dk[i][d]);
        }
      }
    }
  };
  for (int t = t0; t < t1; t += 2) {
    step(t, q0, o0, s0, q1, o1, s1);
    if (t + 1 < t1) step(t + 1, q1, o1, s1, q0, o0, s0);
  }
  results_ready(dk);
  results_ready(dv);
  if constexpr (RW > 1) {  // the waves that share keys: wave wr = 0 takes their sum, dv first, then dk
    const auto sums = [&](int w) { return (float*)(w == 0 ? q0 : w == 1 ? o0 : w == 2 ? q1 : o1); };
    float* const mine = sums(wave);
#pragma unroll
    for (int which = 0; which < 2; ++which) {
      f32x4_t(&x)[KI][DF] = which ? dk : dv;
      __syncthreads();
      if (wr > 0)
#pragma unroll
        for (int i = 0; i < KI; ++i)
#pragma unroll
          for (int d = 0; d < DF; ++d) *(f32x4_t*)(mine + (i * DF + d) * 256 + lane * 4) = x[i][d];
      __syncthreads();
      if (wr == 0)
#pragma unroll
        for (int j = 1; j < RW; ++j)
#pragma unroll
          for (int i = 0; i < KI; ++i)
#pragma unroll
            for (int d = 0; d < DF; ++d) x[i][d] += *(const f32x4_t*)(sums(wave + j) + (i * DF + d) * 256 + lane * 4);
    }
    if (wr > 0) return;
  }
#pragma unroll
  for (int i = 0; i < KI; ++i) {
    const int key = key0 + i * 16 + l16;
    if (key >= c.keys) continue;
    if (a.part) {
      const size_t to = (((size_t)w.split * c.batch + w.b) * c.n_kv_heads + w.h) * c.keys + key;
#pragma unroll
      for (int d = 0; d < DF; ++d) {
        *(f32x4_t*)(a.part + to * HD + d * 16 + grp * 4) = dk[i][d];
        *(f32x4_t*)(a.part2 + to * HD + d * 16 + grp * 4) = dv[i][d];
      }
      continue;
    }
    T* const pk = (T*)g.dk + w.b * g.dk_stride[0] + key * g.dk_stride[1] + w.h * g.dk_stride[2];
    T* const pv = (T*)g.dv + w.b * g.dv_stride[0] + key * g.dv_stride[1] + w.h * g.dv_stride[2];
    const f32x4_t zero = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int d = 0; d < DF; d += 2) {
      store_blocks(pk + d * 16, lane, key < klen ? dk[i][d] * c.scale : zero, key < klen ? dk[i][d + 1] * c.scale : zero);
      store_blocks(pv + d * 16, lane, key < klen ? dv[i][d] : zero, key < klen ? dv[i][d + 1] : zero);
    }
  }
}

// ---------------------------------------------------------------------------
// all gradients where there are at most 16 KF keys: one pass over the rows
// ---------------------------------------------------------------------------
// Every row tile sees all keys, so its scores serve dq and, through LDS (the contraction over rows needs them as columns),
// its share of dk and dv as well: q and dout are read once, not by two passes (with 16 keys of 256 dims 64 x 400 rows
// take 17 us, 3.3 TB/s with the ranges' sums, and 4.6 to add these, instead of 37 and 4.6; a block's chain of load,
// products, exchange and products, two tiles long, bounds it).  A wave takes 16 rows, or where a tile has fewer than 64 a part of their dims;
// for dk and dv the dims are dealt out to the waves.
template <typename T, int HD, int KF, int TR>
__global__ __launch_bounds__(256) void cross_few_keys_grad_kernel(CrossArgs a) {
  typedef Tiles<T, HD, TR> Z;
  typedef Tiles<T, HD, 32> ZK;
  typedef Mat<T> M;
  typedef typename M::frag frag;
  constexpr int E = sizeof(T), RB = Z::RB, STEPS = RB / 64, DF = HD / 16, NK = 32 / M::CK, FP = M::CK / 16;
  constexpr int RF = TR / 16, DW = 4 / RF, DQ = DF / DW < 1 ? 1 : DF / DW, DKV = (DF + 3) / 4;
  static_assert(DQ == 1 || DQ % 2 == 0, "blocks of dq stored in pairs");
  constexpr int PB = 32 * E;  // bytes of a row of probabilities
  __shared__ __attribute__((aligned(1024))) char kt[ZK::BYTES], vt[ZK::BYTES], qt[Z::BYTES], ot[Z::BYTES], pt[TR * PB], st[TR * PB];

  const int lane = threadIdx.x & 63, wave = wave_index(), l16 = lane & 15, grp = lane >> 4;
  const int rf = wave % RF, dw = wave / RF;
  const ravel_cross& c = a.c;
  const ravel_cross_grad& g = a.g;
  const Work w = work_of(a);
  const int klen = live_len(c.k_len, w.b, c.keys), all = c.rows * a.G;
  const int live = klen > 0 ? live_len(c.q_len, w.b, c.rows) * a.G : 0;
  const int rtiles = (all + TR - 1) / TR, per = (rtiles + a.splits - 1) / a.splits;
  const int t0 = min(rtiles, w.split * per), t1 = min(rtiles, t0 + per);

  const T* const k = (const T*)c.k + w.b * c.k_stride[0] + w.h * c.k_stride[2];
  const T* const v = (const T*)c.v + w.b * c.v_stride[0] + w.h * c.v_stride[2];
  const T* const q = (const T*)c.q + w.b * c.q_stride[0] + (int64_t)w.h * a.G * c.q_stride[2];
  const T* const dout = (const T*)g.dout + w.b * g.dout_stride[0] + (int64_t)w.h * a.G * g.dout_stride[2];
  const RowSpace space{a.G, ((1 << 23) + a.G - 1) / a.G};
  const Segments<T, RB> seg(lane);
  load_keys<T, HD, 32>(seg, k, (int)c.k_stride[1], 0, klen, kt, wave);
  load_keys<T, HD, 32>(seg, v, (int)c.v_stride[1], 0, klen, vt, wave);
  const TileLane<T, RB> at0(lane);
  const TileLane<T, PB> ap0(lane);
  const float cs = c.scale > 0.f ? c.scale * kLog2e : 1.f;
  f32x4_t start[KF];  // keys that do not exist
#pragma unroll
  for (int f = 0; f < KF; ++f)
#pragma unroll
    for (int r = 0; r < 4; ++r) start[f][r] = f * 16 + grp * 4 + r < klen ? 0.f : -INFINITY;
  f32x4_t dk[DKV][KF], dv[DKV][KF];
#pragma unroll
  for (int d = 0; d < DKV; ++d)
#pragma unroll
    for (int f = 0; f < KF; ++f) dk[d][f] = dv[d][f] = f32x4_t{0.f, 0.f, 0.f, 0.f};

  for (int t = t0; t < t1; ++t) {
    load_rows<T, HD, TR>(seg, q, c.q_stride[1], (int)c.q_stride[2], space, t * TR, live, qt, wave);
    load_rows<T, HD, TR>(seg, dout, g.dout_stride[1], (int)g.dout_stride[2], space, t * TR, live, ot, wave);
    const int r = t * TR + rf * 16 + l16, qr = r / a.G, gh = w.h * a.G + r - qr * a.G;
    const bool in = r < live;
    const float lse = in ? c.lse[((size_t)w.b * c.n_q_heads + gh) * c.rows + qr] * kLog2e : 0.f;
    tile_barrier<0>();
    const auto at = at0.fresh();
    f32x4_t s[2], dp[2];
#pragma unroll
    for (int f = 0; f < 2; ++f) s[f] = dp[f] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int f = 0; f < KF; ++f) s[f] = start[f];
#pragma unroll
    for (int x = 0; x < STEPS; ++x) {
      frag qf = at.along_row((lds_char_t*)qt, rf, x);
      const frag of = at.along_row((lds_char_t*)ot, rf, x);
      if (!(c.scale > 0.f)) qf = frag{};
#pragma unroll
      for (int f = 0; f < KF; ++f) {
        s[f] = M::mma(at.along_row((lds_char_t*)kt, f, x), qf, s[f]);
        dp[f] = M::mma(at.along_row((lds_char_t*)vt, f, x), of, dp[f]);
      }
    }
    // D = sum p dout v^T, which is dout out before out was rounded.  Rows that do not exist are selected away: their zeros times
    // an infinite key or value are not 0.
    float D = 0.f;
#pragma unroll
    for (int f = 0; f < KF; ++f)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        s[f][i] = in ? __builtin_amdgcn_exp2f(__builtin_fmaf(s[f][i], cs, -lse)) : 0.f;
        D += s[f][i] * dp[f][i];
      }
    D = column_sum(D);
#pragma unroll
    for (int f = 0; f < KF; ++f)
#pragma unroll
      for (int i = 0; i < 4; ++i) dp[f][i] = in ? s[f][i] * (dp[f][i] - D) : 0.f;
    if (dw == 0) {  // columns 16 f + 4 grp .. + 3 of the row's probabilities and their gradients
      const int row = rf * 16 + l16;
#pragma unroll
      for (int f = 0; f < 2; ++f) {
        const int byte = (f * 16 + grp * 4) * E, to = row * PB + ((byte & ~15) ^ (swizzle<T, PB>(row) << 4)) + (byte & 15);
        store_row4<T>((T*)(pt + to), s[f]);
        store_row4<T>((T*)(st + to), dp[f]);
      }
    }
    if (g.dq) {  // (every lane's fragments take part, also those of rows that do not exist)
      T* const to = (T*)g.dq + w.b * g.dq_stride[0] + qr * g.dq_stride[1] + gh * g.dq_stride[2];
      const auto product = [&](int df) {
        f32x4_t dq = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int j = 0; j < NK; ++j)
          if (j * FP < KF) dq = M::mma(at.along_col((lds_char_t*)kt, j, df), M::operand(&dp[j * FP]), dq);
        return in ? dq * c.scale : f32x4_t{0.f, 0.f, 0.f, 0.f};
      };
#pragma unroll
      for (int d = 0; d < DQ; d += 2) {
        const int df = dw * DQ + d;
        if (df >= DF) continue;
        if constexpr (DQ % 2 == 0) {
          const f32x4_t x = product(df), y = product(df + 1);
          if (r < all) store_blocks(to + df * 16, lane, x, y);
        } else {
          const f32x4_t x = product(df);
          if (r < all) store_row4<T>(to + df * 16 + grp * 4, x);
        }
      }
    }
    __syncthreads();
    if (g.dk)
#pragma unroll
      for (int j = 0; j < TR / M::CK; ++j) {
        const auto ap = ap0.fresh();
        frag pf[KF], sf[KF];
#pragma unroll
        for (int f = 0; f < KF; ++f) {
          pf[f] = ap.along_col((lds_char_t*)pt, j, f);
          sf[f] = ap.along_col((lds_char_t*)st, j, f);
        }
#pragma unroll
        for (int d = 0; d < DKV; ++d) {
          const int df = wave + d * 4;
          if (df >= DF) continue;
          const frag qc = at.along_col((lds_char_t*)qt, j, df), oc = at.along_col((lds_char_t*)ot, j, df);
#pragma unroll
          for (int f = 0; f < KF; ++f) {
            dv[d][f] = M::mma(oc, pf[f], dv[d][f]);
            dk[d][f] = M::mma(qc, sf[f], dk[d][f]);
          }
        }
      }
    __syncthreads();
  }
  if (!g.dk) return;
  results_ready(dk);
  results_ready(dv);
#pragma unroll
  for (int f = 0; f < KF; ++f) {
    const int key = f * 16 + l16;
    if (key >= c.keys) continue;
    const f32x4_t zero = {0.f, 0.f, 0.f, 0.f};
    const size_t to = (((size_t)w.split * c.batch + w.b) * c.n_kv_heads + w.h) * c.keys + key;
    T* const pk = (T*)g.dk + w.b * g.dk_stride[0] + key * g.dk_stride[1] + w.h * g.dk_stride[2];
    T* const pv = (T*)g.dv + w.b * g.dv_stride[0] + key * g.dv_stride[1] + w.h * g.dv_stride[2];
#pragma unroll
    for (int d = 0; d < DKV; ++d) {
      const int df = wave + d * 4, e = df * 16 + grp * 4;
      if (df >= DF) continue;
      if (a.part) {
        *(f32x4_t*)(a.part + to * HD + e) = dk[d][f];
        *(f32x4_t*)(a.part2 + to * HD + e) = dv[d][f];
      } else {
        store_row4<T>(pk + e, key < klen ? dk[d][f] * c.scale : zero);
        store_row4<T>(pv + e, key < klen ? dv[d][f] : zero);
      }
    }
  }
}

// Partial sums of ranges added in order: to (b, i, h, d) of a tensor whose index i takes the G heads of a KV head (dq) or
// is a key (dk, dv: G = 1).
struct SumArgs {
  const float* part;
  void* to;
  int64_t stride[3];
  int splits, batch, heads, n, G, hd;  // n = indices of a (batch row, KV head) in part
  const int* len;
  int most;
  float scale;
};
template <typename T>
__global__ __launch_bounds__(256) void cross_sum_kernel(SumArgs x0, SumArgs x1) {
  const SumArgs a = blockIdx.y ? x1 : x0;
  const int hd4 = a.hd / 4;
  const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x, n = (int64_t)a.batch * a.heads * a.n;
  if (id >= n * hd4) return;
  const int64_t at = id / hd4;
  const int d = (int)(id - at * hd4) * 4, i = (int)(at % a.n), h = (int)(at / a.n % a.heads), b = (int)(at / a.n / a.heads);
  f32x4_t s = {0.f, 0.f, 0.f, 0.f};
  const int qr = i / a.G, g = i - qr * a.G;
  if (qr < live_len(a.len, b, a.most)) {
    for (int j = 0; j < a.splits; ++j) s += *(const f32x4_t*)(a.part + (j * n + at) * a.hd + d);
    s *= a.scale;
  }
  store_row4<T>((T*)a.to + b * a.stride[0] + qr * a.stride[1] + (int64_t)(h * a.G + g) * a.stride[2] + d, s);
}

// ---------------------------------------------------------------------------
// plans
// ---------------------------------------------------------------------------
// Tile heights, the rows (or keys) of a wave in 16s, and how many waves of a block share theirs.
template <typename T, int HD>
struct Shape {
  static constexpr int RB = HD * sizeof(T);
  // many rows or keys a block: 64 MI rows in the forward, 64 BI in the gradients (64 where a row is too long for the
  // registers of 128), over tiles of 16 KB, 64 keys at most
  static constexpr int MI = RB >= 512 ? 1 : 2, BI = RB >= 512 ? 1 : 2, TK = RB >= 256 ? 16384 / RB : 64;
  // few: waves share rows and split tiles of up to 16 KB, of which each takes one contraction step at least
  static constexpr int TF = RB >= 128 ? 16384 / RB : 128, KW = TF / Mat<T>::CK < 4 ? TF / Mat<T>::CK : 4;
  // few keys in the gradients: the same over rows, tiles of up to 32 KB
  static constexpr int TR = RB >= 256 ? 32768 / RB : 128, RW = TR / Mat<T>::CK < 4 ? TR / Mat<T>::CK : 4;
  // up to 32 keys: rows of a tile
  static constexpr int TS = RB >= 1024 ? 16 : RB >= 512 ? 32 : 64;
};
constexpr int kFill = 512;  // blocks that fill the chip, two a CU

// Ranges of `tiles` tiles, at least `least` tiles each, for `blocks` blocks to become `fill`.
int ranges(int64_t blocks, int tiles, int least, int fill) {
  int64_t s = fill / (blocks < 1 ? 1 : blocks);
  if (s > tiles / least) s = tiles / least;
  return s < 1 ? 1 : (int)(s > 64 ? 64 : s);
}

struct Plan {
  bool few;
  int tiles, splits;
  size_t bytes;
};
size_t round256(size_t n) { return (n + 255) / 256 * 256; }

template <typename T, int HD>
Plan plan_forward(const ravel_cross& c) {
  typedef Shape<T, HD> S;
  const int all = c.rows * (c.n_q_heads / c.n_kv_heads);
  const int64_t heads = (int64_t)c.batch * c.n_kv_heads;
  Plan p;
  // Waves that share rows read a tile's keys once instead of four times, and finish small calls sooner.
  p.few = all <= 32 || heads * ((all + 64 * S::MI - 1) / (64 * S::MI)) < kFill / 2;
  const int per = p.few ? 16 * (4 / S::KW) : 64 * S::MI, tk = p.few ? S::TF : S::TK;
  p.tiles = (all + per - 1) / per;
  p.splits = ranges(heads * p.tiles, (c.keys + tk - 1) / tk, 4, p.few ? 3 * kFill : kFill);
  p.bytes = p.splits > 1 ? round256((size_t)p.splits * heads * all * (HD + 2) * 4) : 0;
  return p;
}

template <typename T, int HD>
hipError_t forward(const ravel_cross& c, hipStream_t s) {
  typedef Shape<T, HD> S;
  const Plan p = plan_forward<T, HD>(c);
  CrossArgs a{};
  a.c = c;
  a.G = c.n_q_heads / c.n_kv_heads;
  a.tiles = p.tiles;
  a.splits = p.splits;
  const int64_t heads = (int64_t)c.batch * c.n_kv_heads, all = (int64_t)c.rows * a.G;
  if (p.splits > 1) {
    a.part = (float*)c.workspace;
    a.part_ml = a.part + p.splits * heads * all * HD;
  }
  const dim3 grid((unsigned)(heads * p.tiles * p.splits));
  if (p.few)
    cross_kernel<T, HD, 1, S::KW, S::TF><<<grid, 256, 0, s>>>(a);
  else
    cross_kernel<T, HD, S::MI, 1, S::TK><<<grid, 256, 0, s>>>(a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.splits == 1) return e;
  cross_join_kernel<T><<<(unsigned)((heads * all * (HD / 4) + 255) / 256), 256, 0, s>>>(a);
  return hipGetLastError();
}

struct GradPlan {
  int qtiles, qsplits, ktiles, ksplits, padded;
  bool few_rows, few_keys, one_pass, half;
  size_t stat, part;
};
template <typename T, int HD>
GradPlan plan_grad(const ravel_cross& c, const ravel_cross_grad& g) {
  typedef Shape<T, HD> S;
  const int all = c.rows * (c.n_q_heads / c.n_kv_heads);
  const int64_t heads = (int64_t)c.batch * c.n_kv_heads;
  GradPlan p{};
  if (c.keys > 0 && c.keys <= 32) {
    p.one_pass = true;
    p.ksplits = ranges(heads, (all + S::TS - 1) / S::TS, 1, kFill);
    p.part = g.dk && p.ksplits > 1 ? round256((size_t)p.ksplits * heads * c.keys * HD * 4 * 2) : 0;
    return p;
  }
  p.few_rows = all <= 32 || heads * ((all + 64 * S::BI - 1) / (64 * S::BI)) < kFill / 2;
  const int per = p.few_rows ? 16 * (4 / S::KW) : 64 * S::BI, tk = p.few_rows ? S::TF : S::TK;
  p.qtiles = (all + per - 1) / per;
  p.padded = p.qtiles * per;
  p.qsplits = g.dq ? ranges(heads * p.qtiles, (c.keys + tk - 1) / tk, 4, p.few_rows ? 3 * kFill : kFill) : 1;
  if (p.qsplits > 1) p.part = (size_t)p.qsplits * heads * all * HD * 4;
  if (g.dk) {
    p.few_keys = c.keys <= 64;
    // blocks of half as many keys where they do not fill the CUs (4 heads of 32 dims in 32 bits, 4 x 601 rows over 72 keys, all
    // gradients: 40 us from 49; elsewhere within 2 %)
    p.half = S::BI == 2 && !p.few_keys && heads * ((c.keys + 127) / 128) < kFill / 2;
    const int kper = p.few_keys ? 16 * (4 / S::RW) : p.half ? 64 : 64 * S::BI, tr = p.few_keys ? S::TR : S::TK;
    p.ktiles = (c.keys + kper - 1) / kper;
    p.ksplits = ranges(heads * p.ktiles, (all + tr - 1) / tr, p.few_keys ? 1 : 4, kFill);
    p.stat = round256((size_t)heads * p.padded * 2 * 4);
    if (p.ksplits > 1) {
      const size_t n = (size_t)p.ksplits * heads * c.keys * HD * 4 * 2;
      if (n > p.part) p.part = n;
    }
  }
  p.part = round256(p.part);
  return p;
}

// dk and dv from the ranges' sums
template <typename T>
hipError_t sum_keys(const CrossArgs& a, hipStream_t s) {
  const ravel_cross& c = a.c;
  const ravel_cross_grad& g = a.g;
  SumArgs x{a.part, g.dk, {g.dk_stride[0], g.dk_stride[1], g.dk_stride[2]}, a.splits, c.batch, c.n_kv_heads, c.keys, 1, c.head_dim,
            c.k_len, c.keys, c.scale};
  SumArgs y = x;
  y.part = a.part2;
  y.to = g.dv;
  for (int i = 0; i < 3; ++i) y.stride[i] = g.dv_stride[i];
  y.scale = 1.f;
  const int64_t n = (int64_t)c.batch * c.n_kv_heads * c.keys * (c.head_dim / 4);
  cross_sum_kernel<T><<<dim3((unsigned)((n + 255) / 256), 2), 256, 0, s>>>(x, y);
  return hipGetLastError();
}

template <typename T, int HD>
hipError_t gradients(const ravel_cross& c, const ravel_cross_grad& g, hipStream_t s) {
  typedef Shape<T, HD> S;
  const GradPlan p = plan_grad<T, HD>(c, g);
  CrossArgs a{};
  a.c = c;
  a.g = g;
  a.G = c.n_q_heads / c.n_kv_heads;
  a.padded = p.padded;
  a.stat = p.stat ? (float*)g.workspace : nullptr;
  float* const part = (float*)((char*)g.workspace + p.stat);
  const int64_t heads = (int64_t)c.batch * c.n_kv_heads, all = (int64_t)c.rows * a.G;
  hipError_t e;
  if (p.one_pass) {
    a.tiles = 1;
    a.splits = p.ksplits;
    a.part = p.ksplits > 1 ? part : nullptr;
    a.part2 = part + (size_t)p.ksplits * heads * c.keys * HD;
    const dim3 grid((unsigned)(heads * a.splits));
    if (c.keys <= 16)
      cross_few_keys_grad_kernel<T, HD, 1, S::TS><<<grid, 256, 0, s>>>(a);
    else
      cross_few_keys_grad_kernel<T, HD, 2, S::TS><<<grid, 256, 0, s>>>(a);
    if ((e = hipGetLastError()) != hipSuccess || !g.dk || p.ksplits == 1) return e;
    return sum_keys<T>(a, s);
  }
  if (all > 0) {
    a.tiles = p.qtiles;
    a.splits = p.qsplits;
    a.part = p.qsplits > 1 ? part : nullptr;
    const dim3 grid((unsigned)(heads * a.tiles * a.splits));
    if (p.few_rows)
      cross_dq_kernel<T, HD, 1, S::KW, S::TF><<<grid, 256, 0, s>>>(a);
    else
      cross_dq_kernel<T, HD, S::BI, 1, S::TK><<<grid, 256, 0, s>>>(a);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    if (a.part) {
      const SumArgs x{part, g.dq, {g.dq_stride[0], g.dq_stride[1], g.dq_stride[2]}, p.qsplits, c.batch, c.n_kv_heads,
                      (int)all, a.G, HD, c.q_len, c.rows, c.scale};
      cross_sum_kernel<T><<<dim3((unsigned)((heads * all * (HD / 4) + 255) / 256), 1), 256, 0, s>>>(x, x);
      if ((e = hipGetLastError()) != hipSuccess) return e;
    }
  }
  if (!g.dk || c.keys == 0) return hipSuccess;
  a.tiles = p.ktiles;
  a.splits = p.ksplits;
  a.part = p.ksplits > 1 ? part : nullptr;
  a.part2 = part + (size_t)p.ksplits * heads * c.keys * HD;
  const dim3 grid((unsigned)(heads * a.tiles * a.splits));
  if (p.few_keys)
    cross_dkv_kernel<T, HD, 1, S::RW, S::TR><<<grid, 256, 0, s>>>(a);
  else if (p.half)
    cross_dkv_kernel<T, HD, 1, 1, S::TK><<<grid, 256, 0, s>>>(a);
  else
    cross_dkv_kernel<T, HD, S::BI, 1, S::TK><<<grid, 256, 0, s>>>(a);
  if ((e = hipGetLastError()) != hipSuccess || !a.part) return e;
  return sum_keys<T>(a, s);
}

template <typename F>
auto by_shape(const ravel_cross& c, F f) {
  const auto dims = [&](auto t) {
    switch (c.head_dim) {
      case 32: return f(t, std::integral_constant<int, 32>());
      case 64: return f(t, std::integral_constant<int, 64>());
      case 128: return f(t, std::integral_constant<int, 128>());
      default: return f(t, std::integral_constant<int, 256>());
    }
  };
  return c.dtype == RAVEL_F32 ? dims(float()) : dims(bf16_t());
}

}  // namespace

int64_t cross_blocks(const ravel_cross& c) {
  const int64_t heads = (int64_t)c.batch * c.n_kv_heads;
  return by_shape(c, [&](auto t, auto hd) {
    const Plan p = plan_forward<decltype(t), hd.value>(c);
    return heads * p.tiles * p.splits;
  });
}
int64_t cross_grad_blocks(const ravel_cross& c, const ravel_cross_grad& g) {
  const int64_t heads = (int64_t)c.batch * c.n_kv_heads;
  return by_shape(c, [&](auto t, auto hd) {
    const GradPlan p = plan_grad<decltype(t), hd.value>(c, g);
    return heads * std::max((int64_t)p.qtiles * p.qsplits, (int64_t)(p.one_pass ? 1 : p.ktiles) * p.ksplits);
  });
}
size_t cross_workspace(const ravel_cross& c) {
  return by_shape(c, [&](auto t, auto hd) { return plan_forward<decltype(t), hd.value>(c).bytes; });
}
hipError_t launch_cross_attention(const ravel_cross& c, hipStream_t s) {
  if (c.batch == 0 || c.rows == 0) return hipSuccess;
  return by_shape(c, [&](auto t, auto hd) { return forward<decltype(t), hd.value>(c, s); });
}
size_t cross_grad_workspace(const ravel_cross& c, const ravel_cross_grad& g) {
  return by_shape(c, [&](auto t, auto hd) {
    const GradPlan p = plan_grad<decltype(t), hd.value>(c, g);
    return p.stat + p.part;
  });
}
hipError_t launch_cross_attention_grad(const ravel_cross& c, const ravel_cross_grad& g, hipStream_t s) {
  if (c.batch == 0) return hipSuccess;
  return by_shape(c, [&](auto t, auto hd) { return gradients<decltype(t), hd.value>(c, g, s); });
}

}  // namespace ravel
