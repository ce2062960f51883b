// C ABI of the 8-bit key/value cache: argument checks, then the launches of cache.hip and
// cache_attention.hip.
#include <algorithm>
#include <array>

#include "cache.h"

using namespace ravel;

namespace {

ravel_status bad(const char* call, const std::string& msg) { return set_error(RAVEL_E_INVALID, std::string(call) + ": " + msg); }
ravel_status bad_shape(const char* call, const std::string& msg) { return set_error(RAVEL_E_SHAPE, std::string(call) + ": " + msg); }
bool aligned(const void* p, size_t n) { return (uintptr_t)p % n == 0; }

bool overlap(const void* a, size_t na, const void* b, size_t nb) {
  return a && b && (uintptr_t)a < (uintptr_t)b + nb && (uintptr_t)b < (uintptr_t)a + na;
}

struct Piece {
  const void* p;
  size_t bytes;
};
bool overlap(const Piece& a, const Piece& b) { return overlap(a.p, a.bytes, b.p, b.bytes); }
std::array<Piece, 6> pieces(const ravel_cache* x) {  // a cache's memory
  const size_t heads = (size_t)x->n_seq * x->n_kv_heads, tokens = heads * x->capacity;
  const size_t scales = heads * ((x->capacity + x->block - 1) / x->block) * 4;
  return {{{x->k, tokens * x->head_dim}, {x->v, tokens * x->head_dim}, {x->k_scale, scales},
           {x->v_scale, scales}, {x->len, (size_t)x->n_seq * 4}, {x->weight, tokens * 4}}};
}

#define CACHE_TRY(expr)              \
  do {                               \
    const ravel_status s_ = (expr);  \
    if (s_ != RAVEL_OK) return s_;   \
  } while (0)

ravel_status check_sizes(const char* call, const ravel_cache* c) {
  if (!c) return bad(call, "null cache");
  if (c->n_seq < 1 || c->n_kv_heads < 1 || c->n_kv_heads > 65535) return bad_shape(call, "n_seq and n_kv_heads must be >= 1");
  if (c->head_dim != 32 && c->head_dim != 64 && c->head_dim != 128 && c->head_dim != 256)
    return bad_shape(call, "head_dim must be 32, 64, 128 or 256");
  if (c->capacity < 1 || c->capacity > 1 << 24) return bad_shape(call, "capacity must be in 1..2^24");
  if (c->block != 16 && c->block != 32 && c->block != 64 && c->block != 128)
    return bad(call, "block must be 16, 32, 64 or 128");
  if (c->reserved) return bad(call, "reserved must be 0");
  return RAVEL_OK;
}

ravel_status check_cache(const char* call, const ravel_cache* c) {
  CACHE_TRY(check_sizes(call, c));
  if (!c->k || !c->v || !c->k_scale || !c->v_scale || !c->len) return bad(call, "null cache tensor");
  if (!aligned(c->k, 16) || !aligned(c->v, 16)) return bad(call, "k and v must be 16-byte aligned");
  if (!aligned(c->k_scale, 4) || !aligned(c->v_scale, 4) || !aligned(c->len, 4) || !aligned(c->weight, 4))
    return bad(call, "scales, len and weight must be 4-byte aligned");
  return RAVEL_OK;
}

ravel_status check_batch(const char* call, int32_t batch, const int32_t* seq) {
  if (batch < 0 || batch > 32767) return bad_shape(call, "batch must be in 0..32767");
  if (!aligned(seq, 4)) return bad(call, "indices must be 4-byte aligned");
  return RAVEL_OK;
}

ravel_status check_dtype(const char* call, int32_t dtype) {
  return dtype == RAVEL_F32 || dtype == RAVEL_BF16 ? RAVEL_OK : bad(call, "dtype must be RAVEL_F32 or RAVEL_BF16");
}

// vectors of 16 bytes wherever an index and a head lead; (stride, extent) of each dimension
struct Dim {
  int64_t stride, extent;
};
ravel_status check_strides(const char* call, int32_t dtype, std::initializer_list<Dim> dims) {
  const int64_t v = dtype == RAVEL_F32 ? 4 : 8;
  for (const Dim& d : dims) {
    if (d.stride < 0 || d.stride % v) return bad_shape(call, "strides must be multiples of 16 bytes, not negative");
    // the sum of three such offsets, in bytes, stays within 64 bits
    if (d.stride > (1ll << 59) / std::max<int64_t>(d.extent, 1)) return bad_shape(call, "strides reach past 64-bit addresses");
  }
  return RAVEL_OK;
}

CacheView view(const ravel_cache* c) {
  CacheView v;
  v.k = (uint8_t*)c->k;
  v.v = (uint8_t*)c->v;
  v.ks = c->k_scale;
  v.vs = c->v_scale;
  v.len = c->len;
  v.weight = c->weight;
  v.n_seq = c->n_seq;
  v.nkv = c->n_kv_heads;
  v.hd = c->head_dim;
  v.cap = c->capacity;
  v.shift = c->block == 16 ? 4 : c->block == 32 ? 5 : c->block == 64 ? 6 : 7;
  v.nblk = (c->capacity + c->block - 1) / c->block;
  return v;
}

SeqMap seq_map(const int32_t* seq) { return seq ? SeqMap{seq, 1, 1, 0, 0} : SeqMap{nullptr, 1, 0, 1, 0}; }

ravel_status launched(const char* call, hipError_t e) {
  return e == hipSuccess ? RAVEL_OK : set_error(RAVEL_E_HIP, std::string(call) + ": " + hipGetErrorString(e));
}

ravel_status check_query_sizes(const char* call, const ravel_cache* c, const ravel_cache_query* q) {
  CACHE_TRY(check_sizes(call, c));
  if (!q) return bad(call, "null query");
  CACHE_TRY(check_dtype(call, q->dtype));
  CACHE_TRY(check_batch(call, q->batch, nullptr));
  if (q->reserved) return bad(call, "reserved must be 0");
  // (times log2 e and a block's scale it has to stay finite: 0 times infinity is not 0)
  if (!(q->scale >= 0.f && q->scale <= 0x1p100f)) return bad(call, "scale must be in 0..2^100");
  if (q->n_q_heads < 1 || q->n_q_heads % c->n_kv_heads) return bad_shape(call, "n_q_heads must be a multiple of n_kv_heads");
  if (q->rows < 1 || q->rows > 1 << 20) return bad_shape(call, "rows must be in 1..2^20");
  if (q->n_self < 0 || q->n_self > 1 << 20) return bad_shape(call, "n_self must be in 0..2^20");
  if ((int64_t)(q->n_q_heads / c->n_kv_heads) * q->rows > INT32_MAX / 2) return bad_shape(call, "too many rows times heads");
  return RAVEL_OK;
}

CacheAttnArgs attn_args(const ravel_cache* c, const ravel_cache_query* q) {
  CacheAttnArgs a;
  a.c = view(c);
  a.seq = seq_map(q->seq);
  a.batch = q->batch;
  a.nq = q->n_q_heads;
  a.rows = q->rows;
  a.n_self = q->n_self;
  a.q = q->q;
  a.qb = q->q_stride[0], a.qr = q->q_stride[1], a.qh = q->q_stride[2];
  a.sk = q->self_k;
  a.sv = q->self_v;
  a.sb = q->self_stride[0], a.st = q->self_stride[1], a.sh = q->self_stride[2];
  a.out = q->out;
  a.ob = q->out_stride[0], a.orow = q->out_stride[1], a.oh = q->out_stride[2];
  a.scale = q->scale;
  a.f32 = q->dtype == RAVEL_F32;
  a.track = q->track != 0;
  a.ws = q->workspace;
  return a;
}

}  // namespace

extern "C" {

ravel_status ravel_cache_append(const ravel_cache* c, int32_t batch, const int32_t* seq, const int32_t* pos,
                                const int32_t* count, int32_t n, int32_t dtype, const void* k, const void* v,
                                int64_t batch_stride, int64_t token_stride, int64_t head_stride, void* stream) {
  const char* me = "ravel_cache_append";
  CACHE_TRY(check_cache(me, c));
  CACHE_TRY(check_batch(me, batch, seq));
  CACHE_TRY(check_dtype(me, dtype));
  if (n < 0 || n > c->capacity) return bad_shape(me, "n must be in 0..capacity");
  CACHE_TRY(check_strides(me, dtype, {{batch_stride, batch}, {token_stride, n}, {head_stride, c->n_kv_heads}}));
  if (!aligned(pos, 4) || !aligned(count, 4)) return bad(me, "pos and count must be 4-byte aligned");
  if (n > 0 && batch > 0 && (!k || !v)) return bad(me, "null keys or values");
  if (!aligned(k, 16) || !aligned(v, 16)) return bad(me, "keys and values must be 16-byte aligned");
  // the call moves the lengths while other rows still read theirs
  const size_t nl = (size_t)c->n_seq * 4, ni = (size_t)batch * 4;
  if (overlap(seq, ni, c->len, nl) || overlap(count, ni, c->len, nl) || (pos != c->len && overlap(pos, ni, c->len, nl)))
    return bad(me, "seq, pos and count must not lie in the cache's len");
  CacheAppendArgs a;
  a.c = view(c);
  a.seq = seq_map(seq);
  a.batch = batch;
  a.n = n;
  a.pos = pos == c->len ? nullptr : pos;
  a.count = count;
  a.k = k;
  a.v = v;
  a.sb = batch_stride;
  a.st = token_stride;
  a.sh = head_stride;
  a.f32 = dtype == RAVEL_F32;
  return launched(me, launch_cache_append(a, (hipStream_t)stream));
}

ravel_status ravel_cache_attention_workspace(const ravel_cache* c, const ravel_cache_query* q, int64_t* bytes) {
  const char* me = "ravel_cache_attention_workspace";
  CACHE_TRY(check_query_sizes(me, c, q));
  if (!bytes) return bad(me, "null result");
  *bytes = (int64_t)cache_attn_workspace(attn_args(c, q));
  return RAVEL_OK;
}

ravel_status ravel_cache_attention(const ravel_cache* c, const ravel_cache_query* q, void* stream) {
  const char* me = "ravel_cache_attention";
  CACHE_TRY(check_cache(me, c));
  CACHE_TRY(check_query_sizes(me, c, q));
  CACHE_TRY(check_batch(me, q->batch, q->seq));
  if (q->batch == 0) return RAVEL_OK;
  if (!q->q || !q->out) return bad(me, "null queries or out");
  if (q->n_self > 0 && (!q->self_k || !q->self_v)) return bad(me, "null own keys or values");
  for (const void* p : {q->q, q->self_k, q->self_v, (const void*)q->out})
    if (!aligned(p, 16)) return bad(me, "q, self_k, self_v and out must be 16-byte aligned");
  for (const int64_t* st : {q->q_stride, q->out_stride})
    CACHE_TRY(check_strides(me, q->dtype, {{st[0], q->batch}, {st[1], q->rows}, {st[2], q->n_q_heads}}));
  const int64_t* ss = q->self_stride;
  CACHE_TRY(check_strides(me, q->dtype, {{ss[0], q->batch}, {ss[1], q->n_self}, {ss[2], c->n_kv_heads}}));
  if (q->track && !c->weight) return bad(me, "track needs a cache with weights");
  const CacheAttnArgs a = attn_args(c, q);
  const size_t need = cache_attn_workspace(a);
  if (need > 0 && (!q->workspace || q->workspace_bytes < 0 || (size_t)q->workspace_bytes < need))
    return bad(me, "needs a workspace of " + std::to_string(need) + " bytes");
  if (need > 0 && !aligned(q->workspace, 256)) return bad(me, "the workspace must be 256-byte aligned");
  if (q->out == q->q) return bad(me, "out must not be the queries' memory");
  return launched(me, launch_cache_attention(a, (hipStream_t)stream));
}

ravel_status ravel_cache_evict_workspace(const ravel_cache* c, int32_t batch, int32_t keep, int64_t* bytes) {
  const char* me = "ravel_cache_evict_workspace";
  CACHE_TRY(check_sizes(me, c));
  CACHE_TRY(check_batch(me, batch, nullptr));
  if (keep < 1 || keep > 1 << 24) return bad_shape(me, "keep must be in 1..2^24");
  if (!bytes) return bad(me, "null result");
  *bytes = (int64_t)cache_evict_workspace(batch, c->n_kv_heads, keep);
  return RAVEL_OK;
}

ravel_status ravel_cache_evict(const ravel_cache* c, int32_t batch, const int32_t* seq, int32_t keep, int32_t first,
                               const ravel_cache* into, const int32_t* into_seq, int32_t* kept, void* workspace,
                               int64_t workspace_bytes, void* stream) {
  const char* me = "ravel_cache_evict";
  CACHE_TRY(check_cache(me, c));
  CACHE_TRY(check_batch(me, batch, seq));
  if (!c->weight) return bad(me, "the cache has no accumulated weights");
  if (keep < 1 || keep > 1 << 24) return bad_shape(me, "keep must be in 1..2^24");
  if (first < 0 || first > keep) return bad_shape(me, "first must be in 0..keep");
  if (into) {
    CACHE_TRY(check_cache(me, into));
    CACHE_TRY(check_batch(me, batch, into_seq));
    if (into->n_kv_heads != c->n_kv_heads || into->head_dim != c->head_dim || into->block != c->block)
      return bad_shape(me, "both caches must have the same KV heads, head_dim and block");
    if (into->capacity < (keep < c->capacity ? keep : c->capacity)) return bad_shape(me, "the destination holds fewer than keep tokens");
    for (const Piece& p : pieces(c))
      for (const Piece& q : pieces(into))
        if (overlap(p, q)) return bad(me, "the caches share memory");
  } else if (into_seq) {
    return bad(me, "into_seq without a destination");
  }
  if (batch == 0) return RAVEL_OK;
  if (!kept || !aligned(kept, 4)) return bad(me, "kept must be a 4-byte aligned tensor");
  const size_t need = cache_evict_workspace(batch, c->n_kv_heads, keep);
  if (!workspace || workspace_bytes < 0 || (size_t)workspace_bytes < need)
    return bad(me, "needs a workspace of " + std::to_string(need) + " bytes");
  if (!aligned(workspace, 256)) return bad(me, "the workspace must be 256-byte aligned");
  // The selection writes kept and the workspace, the moves read both back; the moves write the
  // destination while other blocks still read their indices and the first cache.
  const size_t ni = (size_t)batch * 4;
  const Piece ids{seq, ni}, into_ids{into_seq, ni}, ks{kept, (size_t)batch * c->n_kv_heads * keep * 4}, ws{workspace, need};
  if (overlap(ks, ws)) return bad(me, "kept must not lie in the workspace");
  if (overlap(ids, ks) || overlap(ids, ws) || overlap(into_ids, ks) || overlap(into_ids, ws))
    return bad(me, "seq and into_seq must not lie in kept or the workspace");
  for (const ravel_cache* x : {c, into ? into : c})
    for (const Piece& p : pieces(x)) {
      if (overlap(ks, p)) return bad(me, "kept must not lie in a cache");
      if (overlap(ws, p)) return bad(me, "the workspace must not lie in a cache");
      if (x == (into ? into : c) && (overlap(ids, p) || overlap(into_ids, p)))
        return bad(me, "seq and into_seq must not lie in the cache that is written");
    }
  CacheEvictArgs a;
  a.src = view(c);
  a.dst = view(into ? into : c);
  a.seq = seq_map(seq);
  a.dst_seq = into ? seq_map(into_seq) : a.seq;
  a.batch = batch;
  a.keep = keep;
  a.first = first;
  a.kept = kept;
  a.ws = workspace;
  return launched(me, launch_cache_evict(a, (hipStream_t)stream));
}

}  // extern "C"
