// Writing and shortening the 8-bit key/value cache.
//
// A block of tokens of one (sequence, kv head) holds x as rne_e4m3(x / s), s a power of
// two: e4m3 is a floating-point format, so a power of two costs its values no relative
// precision, the division and every product with s are exact, and a token that moves to a
// block of another scale only changes its exponent (what falls below e4m3's smallest
// normal number is rounded again).
#include <algorithm>

#include "cache.h"

namespace ravel {

namespace {

constexpr float kCodeMax = 448.f;
constexpr int kMinExp = -100;  // scales from 2^-100 on: their reciprocals and products stay normal numbers

// The smallest power of two s >= 2^kMinExp with amax / s <= 448 = 1.75 * 2^8 (bits of a
// finite amax >= 0): its exponent is amax's less 8, one more where the significand is over 1.75.
RAVEL_DEV float scale_for(uint32_t amax_bits) {
  const int e = (int)((amax_bits + 0x1FFFFFu) >> 23) - 127 - 8;
  return __uint_as_float((uint32_t)(max(e, kMinExp) + 127) << 23);
}
RAVEL_DEV float reciprocal(float s) { return __uint_as_float((254u << 23) - __float_as_uint(s)); }  // of a power of two

// infinities saturate, NaN stays (the plain min / max would drop it)
RAVEL_DEV float clamp_code(float x) { return x != x ? x : __builtin_amdgcn_fmed3f(x, -kCodeMax, kCodeMax); }
RAVEL_DEV uint32_t to_codes(float a, float b, float c, float d) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(clamp_code(a), clamp_code(b), 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(clamp_code(c), clamp_code(d), w, true);
}
// four codes times a power of two r <= 1, rounded again
RAVEL_DEV uint32_t rescale4(uint32_t w, float r) {
  const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
  int q = __builtin_amdgcn_cvt_pk_fp8_f32(lo[0] * r, lo[1] * r, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(hi[0] * r, hi[1] * r, q, true);
}
RAVEL_DEV u32x4_t rescale16(u32x4_t w, float r) {
  return u32x4_t{rescale4(w[0], r), rescale4(w[1], r), rescale4(w[2], r), rescale4(w[3], r)};
}

RAVEL_DEV uint32_t finite_abs(float x) {
  const uint32_t a = __float_as_uint(x) & 0x7FFFFFFFu;
  return a < 0x7F800000u ? a : 0u;
}
RAVEL_DEV uint32_t block_max(uint32_t v, uint32_t* lds) {  // over the block; every thread calls
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) v = max(v, (uint32_t)__shfl_xor((int)v, off, 64));
  if (blockDim.x == 64) return v;
  __syncthreads();
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
  __syncthreads();
  v = lds[0];
  for (int i = 1; i < (int)blockDim.x / 64; ++i) v = max(v, lds[i]);
  return v;
}

// 16 elements, as they lie in memory
template <typename T>
struct Unit {
  u32x4_t w[sizeof(T)];  // 2 bytes an element: 2 x 16 bytes; 4: 4 x 16
  RAVEL_DEV void load(const T* p) {
#pragma unroll
    for (int i = 0; i < (int)sizeof(T); ++i) w[i] = *(const u32x4_t*)(p + i * (16 / sizeof(T)));
  }
  RAVEL_DEV float operator[](int i) const {
    if constexpr (sizeof(T) == 4) return __uint_as_float(w[i / 4][i % 4]);
    const uint32_t x = w[i / 8][i % 8 / 2];
    return __uint_as_float(i % 2 ? x & 0xFFFF0000u : x << 16);
  }
};

// ---------------------------------------------------------------------------
// Append: one block per (scale block that the row's tokens touch, kv head, K or V of a batch row).
// The tokens are read once: their NU units a thread (of TH threads) wait in registers for the
// scale that all of them together give.  Memory binds: 7.4 us for a context of 18 x 816 tokens of
// 256 dims, 117 for 96 x 1250 tokens of 4 x 128 in 32 bits, 5.2 TB/s (read again from the cache
// instead: 9.0 and 135).
// ---------------------------------------------------------------------------
template <typename T, int NU, int TH>
__global__ __launch_bounds__(TH) void cache_append_kernel(CacheAppendArgs a) {
  __shared__ uint32_t red[4];
  const CacheView& c = a.c;
  const int h = blockIdx.y, b = blockIdx.z >> 1;
  const bool is_v = blockIdx.z & 1;
  const int id = cache_seq(c, a.seq, b);
  if (id < 0 || cache_seq_before(c, a.seq, b, id)) return;
  const int pos = a.pos ? a.pos[b] : cache_len(c, id);
  if (pos < 0 || pos > c.cap) return;
  const int cnt = min(a.count ? min(max(a.count[b], 0), a.n) : a.n, c.cap - pos);
  // without pos, every block of the row reads the length: a launch of its own moves it afterwards
  if (a.pos && blockIdx.x == 0 && h == 0 && !is_v && threadIdx.x == 0) c.len[id] = pos + cnt;
  const int blk = (pos >> c.shift) + blockIdx.x, b0 = blk << c.shift;
  const int lo = max(pos, b0), hi = min(pos + cnt, b0 + (1 << c.shift));
  if (lo >= hi) return;

  const int us = c.hd == 32 ? 1 : c.hd == 64 ? 2 : c.hd == 128 ? 3 : 4;  // log2 of the units of a row
  const int units = (hi - lo) << us;
  const T* src = (const T*)(is_v ? a.v : a.k) + (long long)b * a.sb + h * a.sh + (long long)(lo - pos) * a.st;
  Unit<T> x[NU];
#pragma unroll
  for (int k = 0; k < NU; ++k) {
    const int i = min((int)threadIdx.x + k * TH, units - 1);  // (past the end: the last one again)
    x[k].load(src + (long long)(i >> us) * a.st + (i & ((1 << us) - 1)) * 16);
  }
  uint32_t amax = 0;
#pragma unroll
  for (int k = 0; k < NU; ++k)
#pragma unroll
    for (int j = 0; j < 16; ++j) amax = max(amax, finite_abs(x[k][j]));
  float s = scale_for(block_max(amax, red));
  const long long head = (long long)id * c.nkv + h;
  float* sc = (is_v ? c.vs : c.ks) + head * c.nblk + blk;
  uint8_t* dst = (is_v ? c.v : c.k) + (head * c.cap + b0) * c.hd;
  if (lo > b0) {  // older tokens share the block
    const float s0 = *sc;
    if (s > s0) {
      const float r = s0 * reciprocal(s);
      for (int i = threadIdx.x; i < (lo - b0) << us; i += TH) {
        u32x4_t* p = (u32x4_t*)(dst + (size_t)i * 16);
        *p = rescale16(*p, r);
      }
    } else {
      s = s0;
    }
    __syncthreads();  // every thread has read the old scale
  }
  const float inv = reciprocal(s);
  dst += (size_t)(lo - b0) * c.hd;
#pragma unroll
  for (int k = 0; k < NU; ++k) {
    const int i = threadIdx.x + k * TH;
    if (i >= units) break;
    u32x4_t w;
#pragma unroll
    for (int j = 0; j < 4; ++j)
      w[j] = to_codes(x[k][4 * j] * inv, x[k][4 * j + 1] * inv, x[k][4 * j + 2] * inv, x[k][4 * j + 3] * inv);
    *(u32x4_t*)(dst + (size_t)i * 16) = w;
  }
  if (threadIdx.x == 0) *sc = s;
  if (c.weight && !is_v)
    for (int t = lo + threadIdx.x; t < hi; t += TH) c.weight[head * c.cap + t] = 0.f;
}

__global__ __launch_bounds__(64) void cache_append_len_kernel(CacheAppendArgs a) {
  const int b = blockIdx.x;
  const int id = cache_seq(a.c, a.seq, b);
  if (id < 0 || cache_seq_before(a.c, a.seq, b, id) || threadIdx.x) return;
  const int pos = cache_len(a.c, id);
  a.c.len[id] = pos + min(a.count ? min(max(a.count[b], 0), a.n) : a.n, a.c.cap - pos);
}

}  // namespace

template <typename T>
static void append(const CacheAppendArgs& a, hipStream_t s) {
  const int block = 1 << a.c.shift;
  const int wb = std::max(1, std::min(a.c.nblk, (a.n + block - 2) / block + 1));
  const int units = std::min(a.n, block) * (a.c.hd / 16);
  const dim3 grid(wb, a.c.nkv, a.batch * 2);
  const auto kernel = units <= 64    ? cache_append_kernel<T, 1, 64>
                      : units <= 256 ? cache_append_kernel<T, 1, 256>
                      : units <= 512 ? cache_append_kernel<T, 2, 256>
                      : units <= 1024 ? cache_append_kernel<T, 4, 256>
                                      : cache_append_kernel<T, 8, 256>;
  hipLaunchKernelGGL(kernel, grid, dim3(units <= 64 ? 64 : 256), 0, s, a);
}

hipError_t launch_cache_append(const CacheAppendArgs& a, hipStream_t s) {
  if (a.batch == 0) return hipSuccess;
  if (a.f32)
    append<float>(a, s);
  else
    append<bf16_t>(a, s);
  if (!a.pos) hipLaunchKernelGGL(cache_append_len_kernel, dim3(a.batch), dim3(64), 0, s, a);
  return hipGetLastError();
}

// ---------------------------------------------------------------------------
// Eviction: a selection per (batch row, kv head), then the moves.
//
// The kept tokens of index < keep stay where they are, the others fill the holes in
// ascending order (attention does not depend on the order of the tokens): in place, no
// source is ever a destination, and only the arrivals move.
// ---------------------------------------------------------------------------
namespace {

struct EvictInfo {
  int m, pad;             // tokens after the call
  float ks_edge, vs_edge;  // scales of the block that holds position keep, as they were
};

// order of weights as unsigned numbers: NaN below everything, -0 = 0
RAVEL_DEV uint32_t weight_key(float w) {
  if (w != w) return 0;
  const uint32_t u = __float_as_uint(w + 0.f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

constexpr int kSelThreads = 1024, kSelWaves = kSelThreads / 64;

RAVEL_DEV int block_scan(int v, int* lds, int& total) {  // exclusive; every thread calls
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int x = v;
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) {
    const int y = __shfl_up(x, off, 64);
    if (lane >= off) x += y;
  }
  __syncthreads();
  if (lane == 63) lds[wave] = x;
  __syncthreads();
  int base = 0;
  total = 0;
#pragma unroll
  for (int i = 0; i < kSelWaves; ++i) {
    if (i < wave) base += lds[i];
    total += lds[i];
  }
  return base + x - v;
}

// The keep-th largest weight is found 11, 11 and 10 bits of its key at a time, by a histogram of
// the keys that share the bits found so far; then the kept tokens are the keys above it and
// the first of those equal to it.  A thread holds KPT consecutive tokens' keys in registers (where
// that is not all of them, 1024 KPT at a time), so that ranks in token order take two scans over
// the threads' counts.  One workgroup for all of a (sequence, head): its vector instructions bind
// (16384 tokens: 18 us; 47 with a scan for every 1024 of them and a pass over memory for every digit).
template <int KPT>
__global__ __launch_bounds__(kSelThreads) void cache_select_kernel(CacheEvictArgs a, EvictInfo* info, int* holes) {
  constexpr int CHUNK = kSelThreads * KPT;
  __shared__ unsigned hist[2048];
  __shared__ int scan[kSelWaves];
  __shared__ unsigned digit_s, above_s;
  const CacheView& c = a.src;
  const int h = blockIdx.x, b = blockIdx.y, tid = threadIdx.x;
  const int id = cache_seq(c, a.seq, b);
  const long long out = ((long long)b * c.nkv + h) * a.keep;
  int* kept = a.kept + out;
  EvictInfo* inf = info + (long long)b * c.nkv + h;
  const bool in_place = a.dst.k == c.k;
  // (a sequence named again: its first row does the work)
  const bool dup = id >= 0 && (in_place ? cache_seq_before(c, a.seq, b, id)
                                        : cache_seq_before(a.dst, a.dst_seq, b, cache_seq(a.dst, a.dst_seq, b)));
  if (id < 0 || dup || (!in_place && cache_seq(a.dst, a.dst_seq, b) < 0)) {
    for (int i = tid; i < a.keep; i += kSelThreads) kept[i] = -1;
    if (tid == 0) inf->m = -1;
    return;
  }
  const int n = cache_len(c, id), keep = a.keep;
  const long long head = (long long)id * c.nkv + h;
  if (tid == 0) {
    inf->m = min(n, keep);
    const int edge = min(keep >> c.shift, c.nblk - 1);
    inf->ks_edge = c.ks[head * c.nblk + edge];
    inf->vs_edge = c.vs[head * c.nblk + edge];
  }
  if (n <= keep) {
    for (int i = tid; i < keep; i += kSelThreads) kept[i] = i < n ? i : -1;
    return;
  }
  const float* w = c.weight + head * c.cap;
  uint32_t k[KPT];
  const auto load = [&](int base) {  // 0 past the end, as NaN has
    const int i0 = base + tid * KPT;
    float x[KPT];
    if (i0 + KPT <= n) {
      typedef float __attribute__((ext_vector_type(KPT), aligned(4))) vec_t;
      const vec_t v = *(const vec_t*)(w + i0);
#pragma unroll
      for (int j = 0; j < KPT; ++j) x[j] = v[j];
    } else {
#pragma unroll
      for (int j = 0; j < KPT; ++j) x[j] = i0 + j < n ? w[i0 + j] : __uint_as_float(0x7FC00000u);
    }
#pragma unroll
    for (int j = 0; j < KPT; ++j) k[j] = i0 + j < a.first ? 0xFFFFFFFFu : weight_key(x[j]);
  };
  load(0);
  const bool one = n <= CHUNK;

  // `want`: the rank looked for among the keys that share the bits of prefix
  uint32_t prefix = 0;
  unsigned want = keep;
#pragma unroll
  for (int round = 0; round < 3; ++round) {
    const int sh = round == 0 ? 21 : round == 1 ? 10 : 0, bits = round == 2 ? 10 : 11;
    hist[tid] = 0;
    hist[tid + 1024] = 0;
    __syncthreads();
    for (int base = 0; base < n; base += CHUNK) {
      if (!one) load(base);
      const int mine = n - base - tid * KPT;
#pragma unroll
      for (int j = 0; j < KPT; ++j)
        if (j < mine && (round == 0 || k[j] >> (sh + bits) == prefix >> (sh + bits)))
          atomicAdd(&hist[(k[j] >> sh) & ((1u << bits) - 1)], 1u);
    }
    __syncthreads();
    // two digits a thread, from the largest down
    const unsigned v0 = hist[2047 - 2 * tid], v1 = hist[2046 - 2 * tid];
    int total;
    const unsigned before = block_scan((int)(v0 + v1), scan, total);
    if (before < want && want <= before + v0) {
      digit_s = 2047 - 2 * tid;
      above_s = before;
    } else if (before + v0 < want && want <= before + v0 + v1) {
      digit_s = 2046 - 2 * tid;
      above_s = before + v0;
    }
    __syncthreads();
    prefix |= digit_s << sh;
    want -= above_s;
  }

  int* hole = holes + out;
  int eq_base = 0, hole_base = 0, arr_base = 0;
  for (int base = 0; base < n; base += CHUNK) {
    if (!one) load(base);
    const int i0 = base + tid * KPT;
    // a thread's tokens as bits: there, equal to the threshold, below keep
    const unsigned all = (1u << min(max(n - i0, 0), KPT)) - 1, low = (1u << min(max(keep - i0, 0), KPT)) - 1;
    unsigned over = 0, eq = 0;
#pragma unroll
    for (int j = 0; j < KPT; ++j) {
      over |= k[j] > prefix ? 1u << j : 0u;
      eq |= k[j] == prefix ? 1u << j : 0u;
    }
    eq &= all;
    int total;
    // the first `want` of the equal ones, in token order, stay
    int left = (int)want - eq_base - block_scan(__popc(eq), scan, total);
    eq_base += total;
    unsigned stays = over & all;
#pragma unroll
    for (int j = 0; j < KPT; ++j)
      if (eq >> j & 1 && left-- > 0) stays |= 1u << j;
    // ranks of the holes below keep and of the arrivals from keep on (at most 16384 of either)
    const unsigned gone = all & low & ~stays, come = stays & ~low;
    const int rank = block_scan(__popc(gone) | __popc(come) << 16, scan, total);
    int hr = hole_base + (rank & 0xFFFF), ar = arr_base + (int)((unsigned)rank >> 16);
#pragma unroll
    for (int j = 0; j < KPT; ++j) {
      if (stays & low & 1u << j) kept[i0 + j] = i0 + j;
      if (gone >> j & 1) hole[hr++] = i0 + j;
    }
    __syncthreads();  // the holes are there
#pragma unroll
    for (int j = 0; j < KPT; ++j)
      if (come >> j & 1) kept[hole[ar++]] = i0 + j;
    hole_base += total & 0xFFFF;
    arr_base += (int)((unsigned)total >> 16);
  }
}

__global__ __launch_bounds__(256) void cache_move_kernel(CacheEvictArgs a, const EvictInfo* info) {
  __shared__ int from[128];
  __shared__ float ts[128];
  __shared__ uint32_t red[4];
  const CacheView &c = a.src, &d = a.dst;
  const int h = blockIdx.y, b = blockIdx.z >> 1, tid = threadIdx.x;
  const bool is_v = blockIdx.z & 1, in_place = d.k == c.k;
  const EvictInfo inf = info[(long long)b * c.nkv + h];
  if (inf.m < 0) return;
  const int id = cache_seq(c, a.seq, b), to = in_place ? id : cache_seq(d, a.dst_seq, b);
  if (blockIdx.x == 0 && h == 0 && !is_v && tid == 0) d.len[to] = inf.m;
  const int b0 = blockIdx.x << c.shift, m = min(inf.m - b0, 1 << c.shift);
  if (m <= 0) return;
  const long long sh = (long long)id * c.nkv + h, dh = (long long)to * d.nkv + h;
  const float* ss = (is_v ? c.vs : c.ks) + sh * c.nblk;
  float* ds = (is_v ? d.vs : d.ks) + dh * d.nblk + blockIdx.x;
  uint32_t mine = 0;
  if (tid < m) {
    const int f = a.kept[((long long)b * c.nkv + h) * a.keep + b0 + tid];
    from[tid] = f;
    // the block that holds position keep may be another workgroup's to rescale
    const bool edge = in_place && f >= a.keep && (f >> c.shift) == (a.keep >> c.shift);
    const float s = edge ? (is_v ? inf.vs_edge : inf.ks_edge) : ss[f >> c.shift];
    ts[tid] = s;
    mine = __float_as_uint(s);
  }
  const uint32_t top = block_max(mine, red);
  __syncthreads();
  const float inv = reciprocal(__uint_as_float(top));
  const uint8_t* src = (is_v ? c.v : c.k) + sh * c.cap * c.hd;
  uint8_t* dst = (is_v ? d.v : d.k) + (dh * d.cap + b0) * d.hd;
  const int upr = c.hd >> 4;
  for (int i = tid; i < m * upr; i += 256) {
    const int j = i / upr, f = from[j];
    const float r = ts[j] * inv;
    if (in_place && f == b0 + j && r == 1.f) continue;
    u32x4_t w = *(const u32x4_t*)(src + (long long)f * c.hd + (i % upr) * 16);
    if (r != 1.f) w = rescale16(w, r);
    *(u32x4_t*)(dst + (size_t)i * 16) = w;
  }
  if (tid == 0) *ds = __uint_as_float(top);
  if (!is_v && d.weight && tid < m) d.weight[dh * d.cap + b0 + tid] = c.weight[sh * c.cap + from[tid]];
}

}  // namespace

static size_t evict_info_bytes(int batch, int nkv) { return ((size_t)batch * nkv * sizeof(EvictInfo) + 255) / 256 * 256; }

size_t cache_evict_workspace(int batch, int nkv, int keep) {
  return evict_info_bytes(batch, nkv) + (size_t)batch * nkv * keep * 4;
}

hipError_t launch_cache_evict(const CacheEvictArgs& a, hipStream_t s) {
  if (a.batch == 0) return hipSuccess;
  EvictInfo* info = (EvictInfo*)a.ws;
  int* holes = (int*)((char*)a.ws + evict_info_bytes(a.batch, a.src.nkv));
  const auto select = a.src.cap <= kSelThreads ? cache_select_kernel<1> : a.src.cap <= 4 * kSelThreads ? cache_select_kernel<4>
                                                                                                       : cache_select_kernel<16>;
  hipLaunchKernelGGL(select, dim3(a.src.nkv, a.batch), dim3(kSelThreads), 0, s, a, info, holes);
  const int block = 1 << a.src.shift, nb = (std::min(a.keep, a.src.cap) + block - 1) / block;
  hipLaunchKernelGGL(cache_move_kernel, dim3(nb, a.src.nkv, a.batch * 2), dim3(256), 0, s, a, info);
  return hipGetLastError();
}

}  // namespace ravel
