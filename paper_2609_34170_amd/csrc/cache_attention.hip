// Attention over the 8-bit key/value cache and the call's own keys and values
// (bidirectional, grouped-query heads), and the accumulated weights of its tokens.
//
// The G = nq / nkv query heads that share a kv head are flattened with the rows of the
// call into one row space (row = h * rows + i, R = G * rows).  Scores are computed
// transposed, S^T = K Q^T: a lane owns one row and four keys of each 16, its softmax
// statistics stay in registers, and P^T is the second product's B operand as it stands.
//
// Codes are exact as bf16, so both products run on the bf16 matrix instruction with 32-bit
// sums; the scales (one per at least 16 keys: uniform over a 16-key tile) multiply the
// scores and the probabilities.  32-bit queries, own keys and values and probabilities are
// split in three bf16 numbers of 8 significand bits each, which hold them exactly; products
// of the order 2^-24 and below are left out.
#include <algorithm>

#include "cache.h"

namespace ravel {

namespace {

constexpr float kLog2e = 1.4426950408889634f;
// The running maximum of a row moves when a tile raises it by more than this (log2 units):
// between moves the probabilities stay below 2^8 and nothing is rescaled.
constexpr float kLazy = 8.f;
// Waves of a block of few rows: as many as its registers take (8 of 256 dims instead of 4 and
// key ranges to match: 400 rows over 866 keys 20 -> 15 us for 2 sequences, 30 -> 17 for 8; 16 heads
// of 64 dims over 256 keys 7.1 -> 4.8, one launch instead of two).
constexpr int few_row_waves(int hd, bool f32, int rt = 1) {
  return hd <= 64 ? 16 : hd == 256 && (f32 || rt == 2) ? 4 : 8;
}

RAVEL_DEV f32x4_t mfma_bf16(bf16x8_t a, bf16x8_t b, f32x4_t c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
RAVEL_DEV uint32_t codes2(uint32_t w, bool hi) {  // two of four codes as bf16
  return __builtin_bit_cast(uint32_t, hi ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.f, true)
                                         : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.f, false));
}
RAVEL_DEV bf16x8_t codes8(uint32_t w0, uint32_t w1) {
  return __builtin_bit_cast(bf16x8_t, (u32x4_t{codes2(w0, false), codes2(w0, true), codes2(w1, false), codes2(w1, true)}));
}
// 8 values as NP bf16 planes: one, rounded; or three, cut off after 8 significand bits each
template <int NP>
RAVEL_DEV void planes(const float (&x)[8], bf16x8_t (&p)[NP]) {
  if constexpr (NP == 1) {
    p[0] = __builtin_bit_cast(bf16x8_t, (u32x4_t{pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]),
                                                 pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7])}));
  } else {
    float r[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) r[i] = x[i];
#pragma unroll
    for (int n = 0; n < NP; ++n) {
      u32x4_t w;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t a = __float_as_uint(r[2 * i]), b = __float_as_uint(r[2 * i + 1]);
        w[i] = __builtin_amdgcn_perm(b, a, 0x07060302u);
        r[2 * i] -= __uint_as_float(a & 0xFFFF0000u);
        r[2 * i + 1] -= __uint_as_float(b & 0xFFFF0000u);
      }
      p[n] = __builtin_bit_cast(bf16x8_t, w);
    }
  }
}
// 8 consecutive elements of the model's type as planes
template <bool F32, int NP>
RAVEL_DEV void load8(const void* base, long long at, bf16x8_t (&p)[NP]) {
  if constexpr (F32) {
    const f32x4_t lo = *(const f32x4_t*)((const float*)base + at), hi = *(const f32x4_t*)((const float*)base + at + 4);
    const float x[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
    planes<NP>(x, p);
  } else {
    p[0] = *(const bf16x8_t*)((const bf16_t*)base + at);
  }
}

// Blocks are dealt out to the 8 XCDs in turn; this numbering gives each XCD a run of
// consecutive ones, so that those which read the same keys share an L2.
RAVEL_DEV int xcd_block() {
  const int n = gridDim.x, x = blockIdx.x & 7;
  return x * (n >> 3) + min(x, n & 7) + (blockIdx.x >> 3);
}

// a buffer of `bytes` readable bytes from p on (uniform)
RAVEL_DEV __amdgpu_buffer_rsrc_t buffer_of(const void* p, int bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, bytes, 0x00027000);
}

// Partial results of a key range: [split][batch][kv head][row]
struct Part {
  float* o;   // [..][hd], unnormalised
  float* ml;  // [..][2]: maximum (log2 units), sum
  float* lse;  // [batch][kv head][row]: log2 of the softmax's denominator (track)
  int nsplit;
};

// raw codes of a wave's 32-key tile: keys as the A operand's rows, 16 (HD 32: 8) dims a
// load; values 8 keys x HD / 16 consecutive dims a lane
template <int HD>
struct Raw {
  static constexpr int KC = HD >= 64 ? HD / 64 : 1;
  static constexpr int VW = HD >= 64 ? HD / 64 : 1;
  u32x4_t k[2][KC];
  uint32_t v[8][VW];
};

template <int HD>
RAVEL_DEV void load_raw(Raw<HD>& r, const uint8_t* k, const uint8_t* v, int key0, int last, int l16, int grp) {
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    const uint8_t* p = k + (long long)min(key0 + 16 * u + l16, last) * HD;
    if constexpr (HD == 32) {
      const u32x2_t w = *(const u32x2_t*)(p + grp * 8);
      r.k[u][0] = u32x4_t{w[0], w[1], 0, 0};
    } else {
#pragma unroll
      for (int c = 0; c < HD / 64; ++c) r.k[u][c] = *(const u32x4_t*)(p + c * 64 + grp * 16);
    }
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const uint8_t* p = v + (long long)min(key0 + 16 * (j >> 2) + 4 * grp + (j & 3), last) * HD + l16 * (HD / 16);
    if constexpr (HD == 32) r.v[j][0] = *(const uint16_t*)p;
    if constexpr (HD == 64) r.v[j][0] = *(const uint32_t*)p;
    if constexpr (HD == 128) {
      const u32x2_t w = *(const u32x2_t*)p;
      r.v[j][0] = w[0];
      r.v[j][1] = w[1];
    }
    if constexpr (HD == 256) {
      const u32x4_t w = *(const u32x4_t*)p;
#pragma unroll
      for (int i = 0; i < 4; ++i) r.v[j][i] = w[i];
    }
  }
}

// dims of the query and key operands' k-step ks, group grp: 8 consecutive from here
template <int HD>
RAVEL_DEV int kdim(int ks, int grp) {
  return HD == 32 ? grp * 8 : (ks >> 1) * 64 + grp * 16 + (ks & 1) * 8;
}

template <int HD>
RAVEL_DEV bf16x8_t key_operand(const Raw<HD>& r, int u, int ks) {
  const u32x4_t w = r.k[u][HD == 32 ? 0 : ks >> 1];
  return (ks & 1) ? codes8(w[2], w[3]) : codes8(w[0], w[1]);
}

// byte b of eight words
RAVEL_DEV bf16x8_t byte8(const uint32_t (&w)[8], int b) {
  const uint32_t s2 = b == 0 ? 0x0c0c0400u : b == 1 ? 0x0c0c0501u : b == 2 ? 0x0c0c0602u : 0x0c0c0703u;
  const uint32_t a = __builtin_amdgcn_perm(w[1], w[0], s2), c = __builtin_amdgcn_perm(w[3], w[2], s2);
  const uint32_t d = __builtin_amdgcn_perm(w[5], w[4], s2), e = __builtin_amdgcn_perm(w[7], w[6], s2);
  return __builtin_bit_cast(bf16x8_t, (u32x4_t{codes2(a, false), codes2(c, false), codes2(d, false), codes2(e, false)}));
}

// Few rows: a block owns 16 RT rows of a (batch row, kv head) and a range of its keys; its waves
// take the range's tiles of 32 in turn and are joined at the end.  Nothing but the joining goes
// through LDS: a wave loads its own keys as the first product's operand lies, and values 8 keys x
// HD / 16 dims a lane, transposed by byte permutes (whole rows either way).
// Turning codes into operands binds where the codes are at hand: 32 rows share it.
template <int HD, bool F32, int RT, int NW = few_row_waves(HD, F32, RT)>
__global__ __launch_bounds__(NW * 64) void cache_attn_kernel(CacheAttnArgs a, Part part, int chunks) {
  constexpr int KS = HD / 32, NT = HD / 16, NP = F32 ? 3 : 1;
  __shared__ __attribute__((aligned(16))) float so[NW][16 * RT][HD + 4];
  __shared__ float sml[NW][16 * RT][2];
  const CacheView& c = a.c;
  const int split = blockIdx.x % part.nsplit, chunk = blockIdx.x / part.nsplit % chunks;
  const int bg = blockIdx.x / (part.nsplit * chunks), g = bg % c.nkv, b = bg / c.nkv;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l16 = lane & 15, grp = lane >> 4;
  const int G = a.nq / c.nkv, R = G * a.rows;
  const int id = cache_seq(c, a.seq, b), n = id < 0 ? 0 : cache_len(c, id), S = id < 0 ? 0 : a.n_self;
  const int ct = (n + 31) >> 5, tiles = ct + ((S + 31) >> 5);
  const int t0 = tiles * split / part.nsplit, t1 = tiles * (split + 1) / part.nsplit;  // (at most 64 splits)
  const long long head = (long long)max(id, 0) * c.nkv + g;
  const uint8_t *kc = c.k + head * c.cap * HD, *vc = c.v + head * c.cap * HD;
  const float *ksc = c.ks + head * c.nblk, *vsc = c.vs + head * c.nblk;

  bf16x8_t q[RT][KS][NP];
  f32x4_t o[RT][NT];
  float m[RT], l[RT];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const int r = min(chunk * 16 * RT + rt * 16 + l16, R - 1);  // rows past the group are computed and never stored
    const long long at = b * a.qb + r % a.rows * a.qr + (g * G + r / a.rows) * a.qh;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) load8<F32>(a.q, at + kdim<HD>(ks, grp), q[rt][ks]);
#pragma unroll
    for (int t = 0; t < NT; ++t) o[rt][t] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    m[rt] = -INFINITY;
    l[rt] = 0.f;
  }
  const float sl2 = a.scale * kLog2e;

  // x: this lane's scores (log2 units, -inf where masked) of keys 16 u + 4 grp + r; leaves
  // the probabilities times vs[u] in pl, the operand planes
  const auto softmax = [&](int rt, float (&x)[8], const float (&vs)[2], bf16x8_t (&pl)[NP]) {
    float mx = x[0];
#pragma unroll
    for (int i = 1; i < 8; ++i) mx = fmaxf(mx, x[i]);
    if (__any(mx > m[rt] + kLazy)) {
      mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
      mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
      const float mnew = mx > m[rt] + kLazy ? mx : m[rt];
      const float corr = m[rt] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m[rt] - mnew);
      m[rt] = mnew;
      l[rt] *= corr;
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) o[rt][t][r] *= corr;
    }
    const float mref = m[rt] == -INFINITY ? 0.f : m[rt];
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = __builtin_amdgcn_exp2f(x[i] - mref);
    l[rt] += ((x[0] + x[1]) + (x[2] + x[3])) + ((x[4] + x[5]) + (x[6] + x[7]));
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] *= vs[i >> 2];
    planes<NP>(x, pl);
  };

  // cached tokens
  const int c1 = min(t1, ct);
  Raw<HD> nxt;
  if (t0 + wave < c1) load_raw(nxt, kc, vc, (t0 + wave) * 32, n - 1, l16, grp);
  for (int t = t0 + wave; t < c1; t += NW) {
    const Raw<HD> cur = nxt;
    if (t + NW < c1) load_raw(nxt, kc, vc, (t + NW) * 32, n - 1, l16, grp);
    const int key0 = t * 32;
    const int blk0 = key0 >> c.shift, blk1 = min(key0 + 16, n - 1) >> c.shift;
    const float k2[2] = {ksc[blk0] * sl2, ksc[blk1] * sl2}, vs[2] = {vsc[blk0], vsc[blk1]};
    float x[RT][8];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      f32x4_t s[RT];
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) s[rt] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        const bf16x8_t kf = key_operand<HD>(cur, u, ks);
#pragma unroll
        for (int rt = 0; rt < RT; ++rt)
#pragma unroll
          for (int p = NP - 1; p >= 0; --p) s[rt] = mfma_bf16(kf, q[rt][ks][p], s[rt]);
      }
#pragma unroll
      for (int rt = 0; rt < RT; ++rt)
#pragma unroll
        for (int r = 0; r < 4; ++r) x[rt][4 * u + r] = key0 + 16 * u + 4 * grp + r < n ? s[rt][r] * k2[u] : -INFINITY;
    }
    bf16x8_t pl[RT][NP];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) softmax(rt, x[rt], vs, pl[rt]);
#pragma unroll
    for (int i = 0; i < NT; ++i) {  // dim tile i: dims l16 * NT + i
      uint32_t w[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) w[j] = cur.v[j][i >> 2];
      const bf16x8_t vf = byte8(w, i & 3);
#pragma unroll
      for (int rt = 0; rt < RT; ++rt)
#pragma unroll
        for (int p = NP - 1; p >= 0; --p) o[rt][i] = mfma_bf16(vf, pl[rt][p], o[rt][i]);
    }
  }
  // the call's own tokens
  for (int t = max(t0 + wave, ct + ((t0 + wave - ct) & (NW - 1))); t < t1; t += NW) {
    const int key0 = (t - ct) * 32;
    float x[RT][8];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const long long at = b * a.sb + (long long)min(key0 + 16 * u + l16, S - 1) * a.st + g * a.sh;
      f32x4_t s[RT];
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) s[rt] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        bf16x8_t kf[NP];
        load8<F32>(a.sk, at + kdim<HD>(ks, grp), kf);
#pragma unroll
        for (int rt = 0; rt < RT; ++rt)
#pragma unroll
          for (int i = NP - 1; i >= 0; --i)
#pragma unroll
            for (int p = NP - 1 - i; p >= 0; --p) s[rt] = mfma_bf16(kf[i], q[rt][ks][p], s[rt]);
      }
#pragma unroll
      for (int rt = 0; rt < RT; ++rt)
#pragma unroll
        for (int r = 0; r < 4; ++r) x[rt][4 * u + r] = key0 + 16 * u + 4 * grp + r < S ? s[rt][r] * sl2 : -INFINITY;
    }
    bf16x8_t pl[RT][NP];
    const float one[2] = {1.f, 1.f};
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) softmax(rt, x[rt], one, pl[rt]);
    long long va[8];
#pragma unroll
    for (int j = 0; j < 8; ++j)
      va[j] = b * a.sb + (long long)min(key0 + 16 * (j >> 2) + 4 * grp + (j & 3), S - 1) * a.st + g * a.sh + l16 * NT;
#pragma unroll
    for (int i = 0; i < NT; ++i) {
      bf16x8_t vf[NP];
      float y[8];
#pragma unroll
      for (int j = 0; j < 8; ++j)
        y[j] = F32 ? ((const float*)a.sv)[va[j] + i] : bf16_to_f32(((const bf16_t*)a.sv)[va[j] + i]);
      planes<NP>(y, vf);
#pragma unroll
      for (int rt = 0; rt < RT; ++rt)
#pragma unroll
        for (int k = NP - 1; k >= 0; --k)
#pragma unroll
          for (int p = NP - 1 - k; p >= 0; --p) o[rt][i] = mfma_bf16(vf[k], pl[rt][p], o[rt][i]);
    }
  }

  // join the waves: o[t][r] is dim (4 grp + r) NT + t of row l16
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    l[rt] += __shfl_xor(l[rt], 16, 64);
    l[rt] += __shfl_xor(l[rt], 32, 64);
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int t = 0; t < NT; ++t) so[wave][16 * rt + l16][(4 * grp + r) * NT + t] = o[rt][t][r];
    if (grp == 0) {
      sml[wave][16 * rt + l16][0] = m[rt];
      sml[wave][16 * rt + l16][1] = l[rt];
    }
  }
  __syncthreads();
  constexpr int Q4 = HD / 4;
  for (int i = tid; i < 16 * RT * Q4; i += NW * 64) {
    const int r = i / Q4, d = i % Q4 * 4, rr = chunk * 16 * RT + r;
    if (rr >= R) break;
    float mm = sml[0][r][0];
#pragma unroll
    for (int w = 1; w < NW; ++w) mm = fmaxf(mm, sml[w][r][0]);
    const float mref = mm == -INFINITY ? 0.f : mm;
    float num[4] = {0.f, 0.f, 0.f, 0.f}, den = 0.f;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      const float wt = __builtin_amdgcn_exp2f(sml[w][r][0] - mref);  // a wave without keys: 0
      den += wt * sml[w][r][1];
      const f32x4_t v = *(const f32x4_t*)&so[w][r][d];
#pragma unroll
      for (int k = 0; k < 4; ++k) num[k] += wt * v[k];
    }
    if (part.nsplit > 1) {
      const long long pr = (((long long)split * a.batch + b) * c.nkv + g) * R + rr;
      *(f32x4_t*)(part.o + pr * HD + d) = f32x4_t{num[0], num[1], num[2], num[3]};
      if (d == 0) {
        part.ml[pr * 2] = mm;
        part.ml[pr * 2 + 1] = den;
      }
      continue;
    }
    const float inv = den == 0.f ? 0.f : 1.f / den;  // a row that sees nothing: 0
    if (part.lse && d == 0) part.lse[((long long)b * c.nkv + g) * R + rr] = den == 0.f ? INFINITY : mref + log2f(den);
    const long long at = b * a.ob + rr % a.rows * a.orow + (g * G + rr / a.rows) * a.oh + d;
    if constexpr (F32)
      *(f32x4_t*)((float*)a.out + at) = f32x4_t{num[0] * inv, num[1] * inv, num[2] * inv, num[3] * inv};
    else
      *(u32x2_t*)((bf16_t*)a.out + at) = u32x2_t{pack_bf16x2(num[0] * inv, num[1] * inv), pack_bf16x2(num[2] * inv, num[3] * inv)};
  }
}

// ---------------------------------------------------------------------------
// Many rows: a block of 8 waves owns 128 rows of a (batch row, kv head) and walks stages of 64 (256
// dims) or 128 keys; wave (rg, kh) takes the 32 rows of group rg over the half kh of every stage, and the two
// waves of a group are joined at the end: of a SIMD's two waves one's exponentials overlap the
// other's matrix instructions.  (Not tried: one wave a SIMD with 64 rows and its outputs in
// accumulation registers, which would halve the fragments' LDS reads.)  On the 32 x 32 matrix
// instruction a lane owns one row of S^T and O^T, and 16 of each 32 keys (the other 16 the lane
// 32 further on).
//
// Codes become bf16, scale included, on the way into LDS, where they lie as the call's own
// tokens do (converted on the way into the products the four row groups would each repeat it, and
// vector instructions bind as it is: matrix and vector instructions of a SIMD hardly overlap).
// 16-byte chunks are XOR-swizzled by row, so that a fragment's rows fall on distinct
// banks.  Values are read transposed: 16 lanes fetch 4 keys x 16 dims and each receives one
// dim's 4 keys.  The next stage's codes are on their way into registers while one is computed on,
// by buffer loads, which leave the addresses to scalar registers and give 0 past the last token.
// One barrier a stage.
//
// 64 sequences of 400 rows of 256 dims over 866 keys (22.7 GFLOP) take 37 us, 0.62 PFLOP/s.  Of a
// stage's 2.1 us the matrix instructions take 0.96 and the LDS traffic (K and V once a row group,
// 2 HD bytes a key and wave) 1.1, one after the other more than beside each other; start and end of a
// block take 6.  400 rows are 13 groups of 32: three of the fourth block's four are idle.
// ---------------------------------------------------------------------------
typedef __attribute__((__vector_size__(16 * sizeof(float)))) float f32x16_t;
typedef __attribute__((__vector_size__(4 * sizeof(short)))) short s16x4_t;

RAVEL_DEV uint32_t scaled2(uint32_t w, float s, bool hi) {
  return __builtin_bit_cast(uint32_t, hi ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, s, true)
                                         : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, s, false));
}
RAVEL_DEV bf16x8_t scaled8(uint32_t w0, uint32_t w1, float s) {
  return __builtin_bit_cast(bf16x8_t, (u32x4_t{scaled2(w0, s, false), scaled2(w0, s, true), scaled2(w1, s, false),
                                               scaled2(w1, s, true)}));
}
RAVEL_DEV f32x16_t mfma32(bf16x8_t a, bf16x8_t b, f32x16_t c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
typedef __attribute__((address_space(3))) char lds_char;
RAVEL_DEV lds_char* lds_ptr(void* p) { return (lds_char*)p; }
// order of a wave's own accesses to LDS, lane to lane
RAVEL_DEV void wave_lds_order() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}
RAVEL_DEV float half_max(float x) {  // over a lane and the one 32 further on
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
RAVEL_DEV float half_sum(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

template <int HD>
__global__ __launch_bounds__(512, 2) void cache_attn_tile_kernel(CacheAttnArgs a, Part part, int chunks) {
  // rows of a block, 32-key tiles of a wave in a stage (256 dims: LDS holds one for each), keys of a stage
  constexpr int RB = 128, NT = HD == 256 ? 1 : 2, SK = 64 * NT;
  constexpr int KS = HD / 16, DT = HD / 32;
  constexpr int CH = HD / 16;                     // 16-byte chunks of a token's codes
  constexpr int CB = SK * HD;                     // bytes of a stage's codes (keys or values)
  constexpr int NL = CB >= 8192 ? CB / 8192 : 1;  // 16-byte loads per thread
  constexpr int CH2 = HD / 8;                     // the same of bf16 rows, as they lie in LDS
  constexpr int TB = SK * 2 * HD;
  constexpr int NL2 = TB >= 8192 ? TB / 8192 : 1;
  constexpr int RP = CH2 >= 16 ? 1 : 16 / CH2;    // tokens per 256 bytes (all banks)
  constexpr int XK = (CH2 < 16 ? CH2 : 16) - 1;   // swizzle masks: keys' fragments take 16 rows' same chunk,
  constexpr int XV = (CH2 < 16 ? CH2 : 16) / 4 - 1;  // values' four rows' same four chunks
  // two buffers of keys and values; at the end half of each wave's accumulators, then its output rows
  __shared__ __attribute__((aligned(1024))) char buf[4 * TB];
  __shared__ float ml_s[2][RB][2];
  // at 256 dims the last QL query fragments live in LDS: with all of them in registers some
  // spill, and a reload waits for every load of the next stage
  constexpr int QL = HD == 256 ? 7 : 0;
  __shared__ __attribute__((aligned(16))) char q_s[QL ? 4 * QL * 1024 : 16];

  const CacheView& c = a.c;
  const int bid = xcd_block();
  const int chunk = bid % chunks, split = bid / chunks % part.nsplit;
  const int bg = bid / (part.nsplit * chunks), g = bg % c.nkv, b = bg / c.nkv;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int rg = wave >> 1, kh = wave & 1;
  const int l32 = lane & 31, h = lane >> 5;
  const int G = a.nq / c.nkv, R = G * a.rows, row0 = chunk * RB + rg * 32, row = row0 + l32;
  const bool idle = row0 >= R;  // a group without rows: stages keys, and no more
  const int id = __builtin_amdgcn_readfirstlane(cache_seq(c, a.seq, b));
  const int n = __builtin_amdgcn_readfirstlane(id < 0 ? 0 : cache_len(c, id)), S = id < 0 ? 0 : a.n_self;
  const int st = (S + SK - 1) / SK, tiles = st + (n + SK - 1) / SK;
  const int t0 = tiles * split / part.nsplit, t1 = tiles * (split + 1) / part.nsplit;  // (at most 64 splits)
  const int c0 = max(t0 - st, 0), c1 = t1 - st;  // stages of cached tokens
  const long long head = (long long)max(id, 0) * c.nkv + g;
  const uint8_t *kc = c.k + head * c.cap * HD, *vc = c.v + head * c.cap * HD;
  const float *ksc = c.ks + head * c.nblk, *vsc = c.vs + head * c.nblk;

  // codes on their way to LDS, with the scales of their tokens (a stage starts on a scale block's
  // border or, stages of 64 with 128 tokens to a scale, halfway)
  u32x4_t kl[NL], vl[NL];
  float kscale[NL], vscale[NL];
  const int cn = max(n - c0 * SK, 0), sblk = (c0 * SK) >> c.shift;
  // (a key range holds less than 2^31 bytes)
  const auto rk = buffer_of(kc + (long long)c0 * SK * HD, min(cn, (c1 - c0) * SK) * HD);
  const auto rv = buffer_of(vc + (long long)c0 * SK * HD, min(cn, (c1 - c0) * SK) * HD);
  // (blocks behind the last token give a scale of 0: what lies there need not be a number)
  const int sbytes = max(((n - 1) >> c.shift) + 1 - sblk, 0) * 4;
  const auto rks = buffer_of(ksc + sblk, sbytes), rvs = buffer_of(vsc + sblk, sbytes);
  // a thread's loads lie 8 KB apart: LR tokens, whole scale blocks or inside one
  constexpr int LR = 512 / CH;
  const int voff = CB < 8192 && tid >= CB / 16 ? 0x7FFFFFF0 : tid * 16;  // (past the end: nothing is read)
  const int soff = (tid / CH >> c.shift) * 4;
  const auto load = [&](int t) {
    const int at = (t - c0) * CB, sat = (((t * SK) >> c.shift) - sblk) * 4;
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      kl[i] = __builtin_amdgcn_raw_buffer_load_b128(rk, voff, at + i * 8192, 0);
      vl[i] = __builtin_amdgcn_raw_buffer_load_b128(rv, voff, at + i * 8192, 0);
      kscale[i] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(rks, soff, sat + (i * LR >> c.shift) * 4, 0));
      vscale[i] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(rvs, soff, sat + (i * LR >> c.shift) * 4, 0));
    }
  };
  // chunk ch of row r in LDS
  const auto k_at = [](int r, int ch) { return r * 2 * HD + ((ch ^ ((r / RP) & XK)) << 4); };
  const auto v_at = [](int r, int ch) { return TB + r * 2 * HD + ((ch ^ ((r / RP) & XV) << 2) << 4); };
  // own tokens of stage t, through registers into LDS
  const auto load_own = [&](int t, u32x4_t (&ok)[NL2], u32x4_t (&ov)[NL2]) {
#pragma unroll
    for (int i = 0; i < NL2; ++i) {
      const int p = tid + i * 512, r = p / CH2, ch = p % CH2;
      if (TB < 8192 && p >= TB / 16) break;
      const long long at = b * a.sb + (long long)min(t * SK + r, S - 1) * a.st + g * a.sh + ch * 8;
      ok[i] = *(const u32x4_t*)((const bf16_t*)a.sk + at);
      ov[i] = *(const u32x4_t*)((const bf16_t*)a.sv + at);
    }
  };
  const auto store_own = [&](int t, const u32x4_t (&ok)[NL2], const u32x4_t (&ov)[NL2]) {
#pragma unroll
    for (int i = 0; i < NL2; ++i) {
      const int p = tid + i * 512, r = p / CH2, ch = p % CH2;
      if (TB < 8192 && p >= TB / 16) break;
      *(u32x4_t*)(buf + (t & 1) * 2 * TB + k_at(r, ch)) = ok[i];
      *(u32x4_t*)(buf + (t & 1) * 2 * TB + v_at(r, ch)) = ov[i];
    }
  };
  // the first stage's loads are all on their way before the first is waited for
  u32x4_t ok0[NL2], ov0[NL2];
  if (t0 < st) load_own(t0, ok0, ov0);
  if (c0 < c1 && t0 >= st) load(c0);

  bf16x8_t q[KS - QL], qx[KS];
  {
    const int r = min(row, R - 1);  // rows past the group are computed and never stored
    const bf16_t* qr = (const bf16_t*)a.q + b * a.qb + r % a.rows * a.qr + (g * G + r / a.rows) * a.qh + h * 16;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) qx[ks] = *(const bf16x8_t*)(qr + (ks >> 1) * 32 + (ks & 1) * 8);
    __builtin_amdgcn_sched_barrier(0);
    if (t0 < st) store_own(t0, ok0, ov0);
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      const bf16x8_t x = qx[ks];
      if (ks < KS - QL)
        q[ks] = x;
      else if (kh == 0)
        *(bf16x8_t*)(q_s + (rg * QL + ks - (KS - QL)) * 1024 + lane * 16) = x;
    }
  }
  f32x16_t o[DT];
#pragma unroll
  for (int d = 0; d < DT; ++d)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[d][r] = 0.f;
  float m = -INFINITY, l = 0.f;
  // masked scores are -inf before the scale multiplies them: a scale of 0 is the smallest positive number
  // here (-inf * 0 is NaN), which still rounds every finite score to 2^-21 and less
  const float sl2 = fmaxf(a.scale * kLog2e, 0x1p-149f);

  // LDS addresses of this lane's first fragments; the others' differ in bits that the swizzle
  // leaves alone or only flips
  const int ka0 = k_at(kh * 32 * NT + l32, h * 2);
  const int va0 = v_at(kh * 32 * NT + 4 * h + ((lane & 15) >> 2), ((lane >> 4) & 1) * 2 + ((lane & 3) >> 1)) + (lane & 1) * 8;

  const auto store = [&](int t) {  // the stage in registers, converted, into LDS
    char* const kb = buf + (t & 1) * 2 * TB;
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      const int p = tid + i * 512, r = p / CH, ch = p % CH * 2;
      if (CB < 8192 && p >= CB / 16) break;
      const int ka = k_at(r, ch), va = v_at(r, ch);
      *(bf16x8_t*)(kb + ka) = scaled8(kl[i][0], kl[i][1], kscale[i]);
      *(bf16x8_t*)(kb + (ka ^ 16)) = scaled8(kl[i][2], kl[i][3], kscale[i]);
      *(bf16x8_t*)(kb + va) = scaled8(vl[i][0], vl[i][1], vscale[i]);
      *(bf16x8_t*)(kb + (va ^ 16)) = scaled8(vl[i][2], vl[i][3], vscale[i]);
    }
  };
  const auto fetch = [&](int t) {
    if (t >= st && t < t1) load(t - st);
  };
  if (t0 >= st && t0 < t1) store(t0);
  // Of a SIMD's two waves one writes the next stage before it computes on this one, the other after,
  // and matrix instructions go first: so one's conversions and exponentials fall into the
  // other's products (256 / 128 dims 43.6 / 45.0 -> 41.2 / 41.9 us; 64 dims 17.1 and 18.4: not there).
  constexpr bool kStagger = HD >= 128;
  const bool early = kStagger && wave >= 4;
  const auto first = [&](bool on) {
    if constexpr (kStagger) {
      if (on)
        __builtin_amdgcn_s_setprio(1);
      else
        __builtin_amdgcn_s_setprio(0);
    }
  };
  if (early) fetch(t0 + 1);
  for (int t = t0; t < t1; ++t) {
    char* const kb = buf + (t & 1) * 2 * TB;
    // keys of this wave's part that are there; without any the probabilities are 0
    const int left = (t < st ? S - t * SK : n - (t - st) * SK) - kh * 32 * NT;
    __syncthreads();
    if (t + 1 < min(st, t1)) {
      load_own(t + 1, ok0, ov0);
      store_own(t + 1, ok0, ov0);
    } else if (early && t + 1 < t1) {
      store(t + 1);
    }
    fetch(early ? t + 2 : t + 1);
    // Fragments are read ahead, and the steps keep their order: with two tiles the exponentials of
    // the first lie between the matrix instructions of the second's scores, those of the
    // second between the first's of the second product.
    int ka = ka0, va = va0;
    asm volatile("" : "+v"(ka), "+v"(va));  // the addresses of the fragments are formed here, not kept
    const auto read_k = [&](int j) {  // step j: tile j / KS, dims j % KS
      const int ks = j % KS;
      return *(const bf16x8_t*)(kb + (ka ^ ((ks >> 1) << 6 | (ks & 1) << 4)) + j / KS * 64 * HD);
    };
    const auto read_v = [&](int j) {  // step j: 16 keys j / DT, dims j % DT
      u32x2_t w[2];
#pragma unroll
      for (int k = 0; k < 2; ++k)
        w[k] = __builtin_bit_cast(u32x2_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                                               (__attribute__((address_space(3))) s16x4_t*)(lds_ptr(kb) + (va ^ (j % DT << 6)) +
                                                                                            (16 * (j / DT) + 8 * k) * 2 * HD)));
      return __builtin_bit_cast(bf16x8_t, (u32x4_t{w[0][0], w[0][1], w[1][0], w[1][1]}));
    };
    constexpr int PK = HD == 256 ? 2 : KS < 4 ? KS : 4, PV = HD == 256 ? 2 : 2 * DT < 4 ? 2 * DT : 4;
    bf16x8_t kf[PK], vf[PV], ql[2];
    f32x16_t s[NT];
    float x[16];
    uint32_t pw[NT][8];  // probabilities: each tile's two B operands of the second product
    float mref = 0.f;
    // s[u][r] is key 32 u + 8 (r / 4) + 4 h + r % 4: masked, and the running maximum moved where it has to
    const auto maximum = [&](int u) {
#pragma unroll
      for (int r = 0; r < 16; ++r) x[r] = s[u][r];
      if (left < 32 * (u + 1)) {
        const int mine = left - 32 * u - 4 * h;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          float y = 8 * (r >> 2) + (r & 3) < mine ? x[r] : -INFINITY;
          asm volatile("" : "+v"(y));  // stays in its branch
          x[r] = y;
        }
      }
      float mx = x[0];
#pragma unroll
      for (int r = 1; r < 16; ++r) mx = fmaxf(mx, x[r]);
      mx = half_max(mx) * sl2;
      if (__any(mx > m + kLazy)) {
        const float mnew = mx > m + kLazy ? mx : m;
        const float corr = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - mnew);
        m = mnew;
        l *= corr;
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
          for (int r = 0; r < 16; ++r) o[d][r] *= corr;
        if (u == 1) {  // the first tile's are not in the sums yet (and rounded a second time here)
#pragma unroll
          for (int i = 0; i < 8; ++i)
            pw[0][i] = pack_bf16x2(__uint_as_float(pw[0][i] << 16) * corr, __uint_as_float(pw[0][i] & 0xFFFF0000u) * corr);
        }
      }
      mref = m == -INFINITY ? 0.f : m;
    };
    const auto exponentials = [&](int u, int e0, int e1) {
#pragma unroll
      for (int e = e0; e < e1; ++e) {
        x[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[e], sl2, -mref));
        if (e & 1) {
          l += x[e - 1] + x[e];
          pw[u][e >> 1] = pack_bf16x2(x[e - 1], x[e]);
        }
      }
    };
    const auto scores = [&](int u) {
#pragma unroll
      for (int r = 0; r < 16; ++r) s[u][r] = 0.f;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        const int j = u * KS + ks;
        if (ks + 1 >= KS - QL && ks + 1 < KS) ql[(ks + 1) & 1] = *(const bf16x8_t*)(q_s + (rg * QL + ks + 1 - (KS - QL)) * 1024 + lane * 16);
        if (u == 1) exponentials(0, ks * 16 / KS, (ks + 1) * 16 / KS);
        __builtin_amdgcn_sched_barrier(0);
        if (ks < KS - QL)
          s[u] = mfma32(kf[j % PK], q[ks], s[u]);
        else
          s[u] = mfma32(kf[j % PK], ql[ks & 1], s[u]);
        if (j + PK < NT * KS) kf[j % PK] = read_k(j + PK);
      }
    };
    const auto outputs = [&](int u) {
#pragma unroll
      for (int i = 0; i < 2 * DT; ++i) {
        const int j = u * 2 * DT + i;
        if (u == 0 && NT == 2) exponentials(1, i * 8 / DT, (i + 1) * 8 / DT);
        __builtin_amdgcn_sched_barrier(0);
        const uint32_t* w = &pw[u][i / DT * 4];
        o[i % DT] = mfma32(vf[j % PV], __builtin_bit_cast(bf16x8_t, (u32x4_t{w[0], w[1], w[2], w[3]})), o[i % DT]);
        if (j + PV < NT * 2 * DT) vf[j % PV] = read_v(j + PV);
      }
    };
#pragma unroll
    for (int j = 0; j < PK; ++j) kf[j] = read_k(j);
    first(true);
    scores(0);
    first(false);
    if constexpr (NT == 2) {
      maximum(0);
      first(true);
      scores(1);
      first(false);
    }
    if constexpr (NT == 2) {
#pragma unroll
      for (int j = 0; j < PV; ++j) vf[j] = read_v(j);
      __builtin_amdgcn_sched_barrier(0);
      maximum(1);
      first(true);
      outputs(0);
      outputs(1);
      first(false);
    } else {
      maximum(0);
      exponentials(0, 0, 16);
#pragma unroll
      for (int j = 0; j < PV; ++j) vf[j] = read_v(j);
      first(true);
      outputs(0);
      first(false);
    }
    if (!early && t + 1 >= st && t + 1 < t1) store(t + 1);
  }

  // The two waves of a row group hold the same dims of the same rows in the same lanes: each gives
  // the other one half of its accumulators and finishes the other half.
  l = half_sum(l);
  __syncthreads();  // the buffers are free
  constexpr int HR = DT * 8;  // accumulators of half the dims
  const auto acc = [&](int r) -> f32x4_t {
    return f32x4_t{o[r / 16][r % 16], o[r / 16][r % 16 + 1], o[r / 16][r % 16 + 2], o[r / 16][r % 16 + 3]};
  };
  if (h == 0) {
    ml_s[kh][rg * 32 + l32][0] = m;
    ml_s[kh][rg * 32 + l32][1] = l;
  }
  char* give = buf + wave * HR * 256 + lane * 16;
#pragma unroll
  for (int r = 0; r < HR; r += 4) *(f32x4_t*)(give + r * 256) = kh ? acc(r) : acc(HR + r);
  __syncthreads();
  if (idle) return;
  const float m1 = ml_s[kh ^ 1][rg * 32 + l32][0], l1 = ml_s[kh ^ 1][rg * 32 + l32][1], mm = fmaxf(m, m1);
  const float ref = mm == -INFINITY ? 0.f : mm;
  const float w0 = __builtin_amdgcn_exp2f(m - ref), w1 = __builtin_amdgcn_exp2f(m1 - ref), den = w0 * l + w1 * l1;
  char* const ob = buf + (wave ^ 1) * HR * 256;  // what the other gave: read by this wave only
  f32x4_t y[HR / 4];  // y[r]: dim HD / 2 * kh + 8 r + 4 h + ...
#pragma unroll
  for (int r = 0; r < HR; r += 4) y[r / 4] = (kh ? acc(HR + r) : acc(r)) * w0 + *(const f32x4_t*)(ob + lane * 16 + r * 256) * w1;
  if (part.nsplit > 1) {
    if (row >= R) return;
    const long long pr = (((long long)split * a.batch + b) * c.nkv + g) * R + row;
#pragma unroll
    for (int r = 0; r < HR / 4; ++r) *(f32x4_t*)(part.o + pr * HD + HD / 2 * kh + 8 * r + 4 * h) = y[r];
    if (lane < 32 && kh == 0) {
      part.ml[pr * 2] = mm;
      part.ml[pr * 2 + 1] = den;
    }
    return;
  }
  const float inv = den == 0.f ? 0.f : 1.f / den;  // a row that sees nothing: 0
  if (part.lse && lane < 32 && kh == 0 && row < R)
    part.lse[((long long)b * c.nkv + g) * R + row] = den == 0.f ? INFINITY : mm + log2f(den);
  // through LDS (the wave's own part), so that half rows are written whole: 8-byte pieces XOR-swizzled by row
  constexpr int PX = (HD / 8 < 32 ? HD / 8 : 32) - 1;
#pragma unroll
  for (int r = 0; r < HR / 4; ++r)
    *(u32x2_t*)(ob + l32 * HD + (((2 * r + h) ^ (l32 * 2 & PX)) << 3)) =
        u32x2_t{pack_bf16x2(y[r][0] * inv, y[r][1] * inv), pack_bf16x2(y[r][2] * inv, y[r][3] * inv)};
  wave_lds_order();
  constexpr int RS = 1024 / HD;  // rows a store
  int r = lane / (HD / 16), ix = (row0 + r) % a.rows, hx = (row0 + r) / a.rows;
  const int xc = lane % (HD / 16);
#pragma unroll 4
  for (int i = 0; i < 32 / RS; ++i) {
    const u32x4_t w = *(const u32x4_t*)(ob + r * HD + (((2 * xc) ^ (r * 2 & PX)) << 3));
    if (row0 + r < R) *(u32x4_t*)((bf16_t*)a.out + b * a.ob + ix * a.orow + (g * G + hx) * a.oh + HD / 2 * kh + xc * 8) = w;
    r += RS;
    ix += RS;
    while (ix >= a.rows) {
      ix -= a.rows;
      ++hx;
    }
  }
}

// The key ranges joined in range order, four dims a thread, eight ranges' loads in flight (one
// after the other, 64 ranges are 64 round trips to memory: 18 us).
template <bool F32>
__global__ __launch_bounds__(64) void cache_join_kernel(CacheAttnArgs a, Part part) {
  const CacheView& c = a.c;
  const int G = a.nq / c.nkv, R = G * a.rows, Q4 = c.hd / 4;
  const long long rows = (long long)a.batch * c.nkv * R, i = (long long)blockIdx.x * 64 + threadIdx.x;
  if (i >= rows * Q4) return;
  const long long pr = i / Q4;
  const int d = (int)(i % Q4) * 4, rr = (int)(pr % R), g = (int)(pr / R % c.nkv), b = (int)(pr / R / c.nkv);
  float m = -INFINITY, den = 0.f;
  f32x4_t num = {0.f, 0.f, 0.f, 0.f};
  for (int s0 = 0; s0 < part.nsplit; s0 += 8) {
    float2 ml[8];
    f32x4_t v[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const long long at = (long long)min(s0 + k, part.nsplit - 1) * rows + pr;
      ml[k] = *(const float2*)(part.ml + at * 2);
      v[k] = *(const f32x4_t*)(part.o + at * c.hd + d);
    }
    __builtin_amdgcn_sched_barrier(0);  // without it the compiler sinks the loads to their uses
    float mx = m;
#pragma unroll
    for (int k = 0; k < 8; ++k) mx = fmaxf(mx, ml[k].x);
    const float ref = mx == -INFINITY ? 0.f : mx, corr = __builtin_amdgcn_exp2f(m - ref);
    m = mx;
    den *= corr;
#pragma unroll
    for (int j = 0; j < 4; ++j) num[j] *= corr;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const float wt = s0 + k < part.nsplit ? __builtin_amdgcn_exp2f(ml[k].x - ref) : 0.f;
      den += wt * ml[k].y;
#pragma unroll
      for (int j = 0; j < 4; ++j) num[j] += wt * v[k][j];
    }
  }
  const float inv = den == 0.f ? 0.f : 1.f / den;
  if (part.lse && d == 0) part.lse[pr] = den == 0.f ? INFINITY : m + log2f(den);
  const long long at = b * a.ob + rr % a.rows * a.orow + (g * G + rr / a.rows) * a.oh + d;
  if constexpr (F32)
    *(f32x4_t*)((float*)a.out + at) = f32x4_t{num[0] * inv, num[1] * inv, num[2] * inv, num[3] * inv};
  else
    *(u32x2_t*)((bf16_t*)a.out + at) = u32x2_t{pack_bf16x2(num[0] * inv, num[1] * inv), pack_bf16x2(num[2] * inv, num[3] * inv)};
}

// Accumulated weights: rw waves own 64 keys of a (sequence, kv head), form their scores with
// every row once more, 32 rows at a time in turn, and add 2^(score - lse).  Rows are the first
// operand's here: a lane owns a key of each of two tiles and adds over its registers.
// Batch rows that name one sequence are added in row order by the first of them, so that the
// sums have one order.  One wave, or all four of the block where there would be too few (they
// read the same keys: one row of each of 16 heads over 8000 keys 7.5 us with one, 28 with more;
// 400 rows of 256 dims over 816 keys 13 us with four, 37 with one).
//
// Keys and rows come in whole lines and go through LDS: fragment by fragment from memory each load
// touches 32 lines, and the rows, read once for every 64 keys, bind on that (400 rows of 128 dims over 64
// heads of 2048 keys 44 us so, 25 through LDS; of 256 dims over 64 x 816 keys 40 and 30).
constexpr int WW = 4;  // waves of a block of keys
template <int HD, bool F32>
__global__ __launch_bounds__(WW * 64, 2) void cache_weight_kernel(CacheAttnArgs a, const float* lse, int rw) {
  constexpr int KS = HD / 16, NP = F32 ? 3 : 1;
  constexpr int CK = HD / 16, CQ = HD / 8;  // 16-byte chunks of a key, of a bf16 row
  constexpr int RS = 64 / CQ;               // rows of a load
  constexpr bool kAhead = HD < 256;         // the next rows' loads in flight: 256 dims' do not fit the registers
  __shared__ float sum_s[WW][64];
  __shared__ float ls_s[WW][32];
  __shared__ __attribute__((aligned(128))) char stage_s[WW][64 * HD];  // a wave's keys, then 32 rows
  const CacheView& c = a.c;
  const int bid = xcd_block(), bk = 64 * WW / rw, nkt = (c.cap + bk - 1) / bk;  // keys of a block
  const int g = bid / nkt % c.nkv, b0 = bid / nkt / c.nkv;
  const int id = __builtin_amdgcn_readfirstlane(cache_seq(c, a.seq, b0));
  if (id < 0 || cache_seq_before(c, a.seq, b0, id)) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l32 = lane & 31, h = lane >> 5;
  const int n = cache_len(c, id), key0 = bid % nkt * bk + wave / rw * 64, sub = wave % rw;
  const int G = a.nq / c.nkv, R = G * a.rows;
  const long long head = (long long)id * c.nkv + g;
  char* const sw = stage_s[wave];
  // chunk ch of row r of C chunks: 8 neighbouring rows' same chunk fall on all banks
  const auto at = [](int C, int r, int ch) {
    return (r * C + (ch ^ (C < 8 ? r / (8 / C) & (C - 1) : r & 7))) * 16;
  };
  float acc[2] = {0.f, 0.f};
  if (key0 < n && sub * 32 < R) {
    u32x4_t raw[CK];
#pragma unroll
    for (int i = 0; i < CK; ++i) {
      const int p = i * 64 + lane;
      raw[i] = *(const u32x4_t*)(c.k + (head * c.cap + min(key0 + p / CK, n - 1)) * HD + p % CK * 16);
    }
    float sc[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) sc[u] = c.ks[head * c.nblk + (min(key0 + 32 * u + l32, n - 1) >> c.shift)];
    // bf16 rows r0 to r0 + 31 and their sums, on their way into registers (rows past the group: row 0,
    // with a sum that makes their weights 0)
    u32x4_t qraw[CK];
    float lraw;
    // A step of some rows is di further on in rows and dh in heads, or one head more and a.rows back.
    const long long wrap = a.qh - a.rows * a.qr, step = RS % a.rows * a.qr + RS / a.rows * a.qh;
    const int skip = (rw - 1) * 32;
    const long long leap = skip % a.rows * a.qr + skip / a.rows * a.qh;
    const int r_first = sub * 32 + lane / CQ, i_first = r_first % a.rows;
    const long long off_first = i_first * a.qr + r_first / a.rows * a.qh;
    int qrow, qi;
    long long off;
    const auto move = [&](int rows, int i, long long by) {
      qrow += rows;
      qi += i;
      off += by;
      if (qi >= a.rows) {
        qi -= a.rows;
        off += wrap;
      }
    };
    const auto fetch = [&](int b, int r0) {
      if constexpr (!F32) {
        const bf16_t* q = (const bf16_t*)a.q + b * a.qb + g * G * a.qh + lane % CQ * 8;
        if (r0 == sub * 32) {
          qrow = r_first;
          qi = i_first;
          off = off_first;
        } else {
          move(skip, skip % a.rows, leap);
        }
#pragma unroll
        for (int i = 0; i < CK; ++i) {
          qraw[i] = *(const u32x4_t*)(q + (qrow < R ? off : 0));
          move(RS, RS % a.rows, step);
        }
        lraw = r0 + l32 < R ? lse[((long long)b * c.nkv + g) * R + r0 + l32] : INFINITY;
      }
    };
    if (kAhead) fetch(b0, sub * 32);
#pragma unroll
    for (int i = 0; i < CK; ++i) *(u32x4_t*)(sw + at(CK, (i * 64 + lane) / CK, (i * 64 + lane) % CK)) = raw[i];
    wave_lds_order();
    bf16x8_t kf[2][KS];
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int j = 0; j < KS / 2; ++j) {
        const u32x4_t w = *(const u32x4_t*)(sw + at(CK, 32 * u + l32, 2 * j + h));
        kf[u][2 * j] = scaled8(w[0], w[1], sc[u]);
        kf[u][2 * j + 1] = scaled8(w[2], w[3], sc[u]);
      }
    const float sl2 = a.scale * kLog2e;
    // the rows that name this sequence, found 64 at a time; only b0 where all rows differ
    const int b1 = !a.seq.idx || a.seq.row ? b0 + 1 : a.batch;
    for (int bw = b0; bw < b1; bw += 64) {
      unsigned long long same = __ballot(bw + lane < b1 && cache_seq(c, a.seq, bw + lane) == id);
      for (; same; same &= same - 1) {
        const int b = bw + __builtin_ctzll(same);
        const float* lr = lse + ((long long)b * c.nkv + g) * R;
        if (kAhead && b != b0) fetch(b, sub * 32);
        for (int r0 = sub * 32; r0 < R; r0 += rw * 32) {
          f32x4_t ls[4];
          if constexpr (F32) {
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              const int rr = r0 + 8 * (i >> 2) + 4 * h + (i & 3);
              ls[i >> 2][i & 3] = rr < R ? lr[min(rr, R - 1)] : INFINITY;
            }
          } else {
            wave_lds_order();
            if (!kAhead) fetch(b, r0);
#pragma unroll
            for (int i = 0; i < CK; ++i) *(u32x4_t*)(sw + at(CQ, (i * 64 + lane) / CQ, (i * 64 + lane) % CQ)) = qraw[i];
            ls_s[wave][l32] = lraw;
            wave_lds_order();
            if (kAhead && r0 + rw * 32 < R) fetch(b, r0 + rw * 32);
#pragma unroll
            for (int i = 0; i < 4; ++i) ls[i] = *(const f32x4_t*)&ls_s[wave][8 * i + 4 * h];
          }
          f32x16_t s[2];
#pragma unroll
          for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int i = 0; i < 16; ++i) s[u][i] = 0.f;
          // 32 bits: planes are made fragment by fragment
          const int r = min(r0 + l32, R - 1);
          const long long q0 = F32 ? b * a.qb + r % a.rows * a.qr + (g * G + r / a.rows) * a.qh + h * 16 : 0;
#pragma unroll
          for (int ks = 0; ks < KS; ++ks) {
            bf16x8_t q[NP];
            if constexpr (F32)
              load8<true>(a.q, q0 + (ks >> 1) * 32 + (ks & 1) * 8, q);
            else
              q[0] = *(const bf16x8_t*)(sw + at(CQ, l32, (ks >> 1) * 4 + h * 2 + (ks & 1)));
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
              for (int p = NP - 1; p >= 0; --p) s[u] = mfma32(q[p], kf[u][ks], s[u]);
          }
#pragma unroll
          for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[u] += __builtin_amdgcn_exp2f(__builtin_fmaf(s[u][i], sl2, -ls[i >> 2][i & 3]));
        }
      }
    }
  }
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    acc[u] = half_sum(acc[u]);
    if (h == 0) sum_s[wave][u * 32 + l32] = acc[u];
  }
  __syncthreads();
  const int key = key0 + lane;
  if (sub == 0 && key < n) {
    float v = sum_s[wave][lane];
    for (int w = 1; w < rw; ++w) v += sum_s[wave + w][lane];
    c.weight[head * c.cap + key] += v;
  }
}

struct Plan {
  bool tile;
  int rt;  // few rows: 16 rt rows of a block
  int chunks, nsplit;
  size_t o_off, ml_off, lse_off, bytes;
};
size_t up256(size_t x) { return (x + 255) / 256 * 256; }

Plan plan_of(const CacheAttnArgs& a) {
  Plan p;
  const long long R = (long long)(a.nq / a.c.nkv) * a.rows, heads = (long long)a.batch * a.c.nkv;
  // All by the capacity: the host does not know the lengths, and a long cache of short contents is
  // planned as if it were full.
  // Rows of a block, by how often its blocks fill the 256 CUs (one of them a CU): 32 rows take 1.4 times
  // as long as 16 and half the blocks, 128 some 1.8 times as long as 32, and their start and the sum
  // of their key ranges cost 9 us and more.  us with 16 / 32 / 128 rows:
  //   400 rows of 256 dims over 866 keys, 8 sequences 17 / 24 / 31, 16 32 / 25 / 33, 24 47 / 47 / 38
  //   400 rows of 128 dims over 2148 keys, 8 heads 17 / 21 / 23, 16 33 / 23 / 27, 24 48 / 41 / 34
  //   64 rows of 64 dims over 320 keys, 128 heads 9.4 / 7.3 / 13, 256 18 / 12 / 9
  //   128 heads of 128 dims over 4096 keys, 32 rows 41 / 30 / 47, 64 77 / 44 / 48
  //   512 heads of 128 dims over 1024 keys, 32 rows 47 / 30 / 45, 33 66 / 54 / 45
  //   16 heads of 128 dims over 8192 keys, 64 rows 22 / 19 / 21, 128 33 / 26 / 24
  const long long b16 = (R + 15) / 16 * heads, b32 = (R + 31) / 32 * heads, keys_all = (long long)a.c.cap + a.n_self;
  p.tile = !a.f32 && R > 32 && (b32 > 256 || (R >= 96 && b32 * keys_all >= 500000));
  p.rt = !a.f32 && R > 16 && (5 * ((b16 + 255) / 256) > 7 * ((b32 + 255) / 256) || (b16 > 128 && keys_all >= 4096)) ? 2 : 1;
  const int rows = p.tile ? 128 : 16 * p.rt;
  p.chunks = (int)((R + rows - 1) / rows);
  const long long blocks = p.chunks * heads;
  // Key ranges up to one block a CU.  128 rows: a stage at least.  16 rows: a tile a wave, but no
  // ranges where a block has two for each of its waves (16 heads of 128 dims over 512 keys 7.3
  // us so, 9.2 with two ranges; over 1024 11.0 and 9.3).
  const int w = few_row_waves(a.c.hd, a.f32, p.rt), keys = !p.tile ? 32 * w : a.c.hd < 256 ? 128 : 64;
  long long steps = (a.c.cap + keys - 1) / keys + (a.n_self + keys - 1) / keys;
  if (!p.tile) {
    const long long tiles = (a.c.cap + 31) / 32 + (a.n_self + 31) / 32;
    steps = tiles <= 2 * w ? 1 : (tiles + w - 1) / w;
  }
  p.nsplit = (int)std::max(1ll, std::min({256 / std::max(blocks, 1ll), steps, 64ll}));
  if (p.tile) p.nsplit = std::max(p.nsplit, (int)(((long long)a.c.cap * a.c.hd >> 30) + 1));  // 32-bit offsets in a range
  p.o_off = 0;
  p.ml_off = p.nsplit > 1 ? up256((size_t)p.nsplit * heads * R * a.c.hd * 4) : 0;
  p.lse_off = p.ml_off + (p.nsplit > 1 ? up256((size_t)p.nsplit * heads * R * 8) : 0);
  p.bytes = p.lse_off + (a.track ? up256((size_t)heads * R * 4) : 0);
  return p;
}

template <int HD, bool F32>
hipError_t launch_hd(const CacheAttnArgs& a, hipStream_t s, int launches) {
  const Plan p = plan_of(a);
  const long long heads = (long long)a.batch * a.c.nkv, R = (long long)(a.nq / a.c.nkv) * a.rows;
  char* ws = (char*)a.ws;
  const Part part{(float*)(ws + p.o_off), (float*)(ws + p.ml_off), a.track ? (float*)(ws + p.lse_off) : nullptr, p.nsplit};
  const long long blocks = p.chunks * heads * p.nsplit, joins = (heads * R * (HD / 4) + 63) / 64;
  if (blocks > 0x7FFFFFFF || joins > 0x7FFFFFFF || (a.track && heads * ((a.c.cap + 63) / 64) > 0x7FFFFFFF)) return hipErrorInvalidValue;
  if (launches & CACHE_ATTEND) {
    if constexpr (!F32) {
      if (p.tile) hipLaunchKernelGGL((cache_attn_tile_kernel<HD>), dim3((unsigned)blocks), dim3(512), 0, s, a, part, p.chunks);
    }
    if constexpr (!F32) {
      if (!p.tile && p.rt == 2)
        hipLaunchKernelGGL((cache_attn_kernel<HD, F32, 2>), dim3((unsigned)blocks), dim3(few_row_waves(HD, F32, 2) * 64), 0, s, a,
                           part, p.chunks);
    }
    if (!p.tile && p.rt == 1)
      hipLaunchKernelGGL((cache_attn_kernel<HD, F32, 1>), dim3((unsigned)blocks), dim3(few_row_waves(HD, F32) * 64), 0, s, a, part,
                         p.chunks);
  }
  if ((launches & CACHE_JOIN) && p.nsplit > 1)
    hipLaunchKernelGGL(cache_join_kernel<F32>, dim3((unsigned)joins), dim3(64), 0, s, a, part);
  if ((launches & CACHE_WEIGHTS) && a.track) {
    // one wave where its rows are few, or its keys alone give every SIMD a wave
    const int rw = R <= 32 || heads * ((a.c.cap + 63) / 64) >= 1024 ? 1 : WW, bk = 64 * WW / rw;
    hipLaunchKernelGGL((cache_weight_kernel<HD, F32>), dim3((unsigned)(heads * ((a.c.cap + bk - 1) / bk))), dim3(WW * 64), 0, s, a,
                       part.lse, rw);
  }
  return hipGetLastError();
}

}  // namespace

size_t cache_attn_workspace(const CacheAttnArgs& a) { return a.batch == 0 ? 0 : plan_of(a).bytes; }

int cache_attn_ranges(const CacheAttnArgs& a) { return a.batch == 0 ? 1 : plan_of(a).nsplit; }

hipError_t launch_cache_attention(const CacheAttnArgs& a, hipStream_t s, int launches) {
  if (a.batch == 0) return hipSuccess;
  switch (a.c.hd) {
    case 32: return a.f32 ? launch_hd<32, true>(a, s, launches) : launch_hd<32, false>(a, s, launches);
    case 64: return a.f32 ? launch_hd<64, true>(a, s, launches) : launch_hd<64, false>(a, s, launches);
    case 128: return a.f32 ? launch_hd<128, true>(a, s, launches) : launch_hd<128, false>(a, s, launches);
    case 256: return a.f32 ? launch_hd<256, true>(a, s, launches) : launch_hd<256, false>(a, s, launches);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace ravel
