// The 8-bit key/value cache (internal; the C ABI is in ravel.h): e4m3 codes
// [sequence][kv head][capacity][hd] for keys and values, a power-of-two scale per
// (sequence, kv head, block of tokens) for each, the sequences' lengths, and
// optionally an accumulated attention weight per (sequence, kv head, token).
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include <string>

#include "common.h"
#include "ravel.h"

namespace ravel {

ravel_status set_error(ravel_status s, const std::string& msg);  // the calling thread's last error

struct CacheView {
  uint8_t *k, *v;
  float *ks, *vs;  // [n_seq][nkv][nblk]
  int* len;        // [n_seq]
  float* weight;   // [n_seq][nkv][cap] or null
  int n_seq, nkv, hd, cap;
  int shift, nblk;  // tokens per scale block = 1 << shift; blocks per (sequence, head)
};

// Batch row b's sequence: idx[b / div] * mul + b * row + add (idx null: the first term is 0).
// Rows whose sequence falls outside the cache take no part in a call.  With row != 0 the rows
// name distinct sequences.
struct SeqMap {
  const int* idx;
  int div, mul, row, add;
};

struct CacheAppendArgs {
  CacheView c;
  SeqMap seq;
  int batch, n;
  const int* pos;    // [batch] first position, or null: at len
  const int* count;  // [batch] tokens of a row (clamped to 0..n), or null: n
  const void *k, *v;  // element (b, t, h, d) at b * sb + t * st + h * sh + d
  long long sb, st, sh;
  bool f32;
};
hipError_t launch_cache_append(const CacheAppendArgs& a, hipStream_t s);

struct CacheAttnArgs {
  CacheView c;
  SeqMap seq;
  int batch, nq, rows, n_self;
  const void* q;  // (b, i, h, d) at b * qb + i * qr + h * qh + d
  long long qb, qr, qh;
  const void *sk, *sv;  // (b, t, h, d) at b * sb + t * st + h * sh + d
  long long sb, st, sh;
  void* out;  // (b, i, h, d) at b * ob + i * orow + h * oh + d
  long long ob, orow, oh;
  float scale;
  bool f32, track;
  void* ws;  // cache_attn_workspace() bytes, 16-byte aligned
};
size_t cache_attn_workspace(const CacheAttnArgs& a);  // c.nkv, hd, cap and the sizes of the call are read
int cache_attn_ranges(const CacheAttnArgs& a);            // key ranges, joined by a launch of their own where there are several
// A call's launches: the attention, the join of its key ranges (if there are several), the weights (track).
enum { CACHE_ATTEND = 1, CACHE_JOIN = 2, CACHE_WEIGHTS = 4, CACHE_ALL = 7 };
hipError_t launch_cache_attention(const CacheAttnArgs& a, hipStream_t s, int launches = CACHE_ALL);

struct CacheEvictArgs {
  CacheView src, dst;  // dst the same as src: in place
  SeqMap seq, dst_seq;
  int batch, keep, first;
  int* kept;  // [batch][nkv][keep]
  void* ws;   // cache_evict_workspace() bytes
};
size_t cache_evict_workspace(int batch, int nkv, int keep);
hipError_t launch_cache_evict(const CacheEvictArgs& a, hipStream_t s);

#ifdef __HIPCC__
RAVEL_DEV int cache_seq(const CacheView& c, const SeqMap& m, int b) {  // negative: none
  const long long id = (m.idx ? (long long)m.idx[m.div == 1 ? b : b / m.div] * m.mul : 0) + (long long)b * m.row + m.add;
  return id >= 0 && id < c.n_seq ? (int)id : -1;
}
RAVEL_DEV int cache_len(const CacheView& c, int id) { return min(max(c.len[id], 0), c.cap); }
// Whether a row before b names the same sequence (uniform over the block; every thread calls).
RAVEL_DEV bool cache_seq_before(const CacheView& c, const SeqMap& m, int b, int id) {
  if (!m.idx || m.row) return false;
  bool hit = false;
  for (int i = threadIdx.x; i < b; i += blockDim.x) hit |= cache_seq(c, m, i) == id;
  return __syncthreads_or(hit) != 0;
}
#endif

}  // namespace ravel
