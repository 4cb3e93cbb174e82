// extern "C" entry points of the paged 4-bit cache and of the page plan: argument checks and launches, as in api.hip.
#include "cache4_common.h"

namespace ha {

static int log2_page(int page) {
  for (int k = 4; k <= 8; ++k)
    if (page == 1 << k) return k;
  return -1;
}

static int cache_geometry(const ha_cache4* sh, CacheGeometry* c) {
  if (!sh) return HA_ERR_NULL;
  c->log_page = log2_page(sh->page);
  if (c->log_page < 0 || (sh->d != 64 && sh->d != 128)) return HA_ERR_SHAPE;
  if (sh->n_pages < 0 || sh->Hk < 1 || sh->Hk > 1024 || (int64_t)sh->n_pages * sh->page > 0x7fffffffll) return HA_ERR_SHAPE;
  c->n_pages = sh->n_pages;
  c->page = sh->page;
  c->Hk = sh->Hk;
  c->d = sh->d;
  return HA_OK;
}

static int rows_call(const void* K, const void* V, const int32_t* slots, const void* cache, const ha_cache4* shape, int32_t rows, int32_t dtype,
                     const ha_strides* kv, void* stream, bool write) {
  CacheRowsArgs a{};
  int rc = cache_geometry(shape, &a.c);
  if (rc != HA_OK) return rc;
  if (dtype != HA_BF16 && dtype != HA_FP32) return HA_ERR_DTYPE;
  if (rows < 0 || rows > (1 << 26) || (int64_t)rows * shape->Hk > (1ll << 26)) return HA_ERR_SHAPE;
  rc = row_strides(kv, rows, shape->Hk, shape->d, dtype, !write, &a.k);
  if (rc == HA_OK) rc = row_strides(kv ? kv + 1 : nullptr, rows, shape->Hk, shape->d, dtype, !write, &a.v);
  if (rc != HA_OK) return rc;
  if (rows == 0 || (write && shape->n_pages == 0)) return HA_OK;
  if (!K || !V || !slots || (!cache && shape->n_pages > 0)) return HA_ERR_NULL;
  if (any_misaligned16(K, V, cache) || any_misaligned4(slots)) return HA_ERR_ALIGN;
  a.K = const_cast<void*>(K);
  a.V = const_cast<void*>(V);
  a.slots = slots;
  a.cache = reinterpret_cast<unsigned char*>(const_cast<void*>(cache));
  a.rows = rows;
  return write ? launch_cache4_write(a, dtype, (hipStream_t)stream) : launch_cache4_read(a, dtype, (hipStream_t)stream);
}

// Fills all of *a but the pointers and strides.
static int attn_geometry(const ha_cache4* shape, const ha_cache4_query* q, CacheAttnArgs* a) {
  const int rc = cache_geometry(shape, &a->c);
  if (rc != HA_OK) return rc;
  if (!q) return HA_ERR_NULL;
  if (q->dtype != HA_BF16 && q->dtype != HA_FP32) return HA_ERR_DTYPE;
  if (q->n_seq < 0 || q->n_seq > (1 << 16) || q->q_len < 1 || q->q_len > 64 || q->max_blocks < 0) return HA_ERR_SHAPE;
  if (q->Hq < 1 || q->Hq % shape->Hk != 0 || (int64_t)q->Hq * q->q_len > (1 << 15)) return HA_ERR_SHAPE;
  if ((int64_t)q->n_seq * q->q_len * q->Hq > (1 << 22)) return HA_ERR_SHAPE;
  if ((int64_t)q->n_seq * q->max_blocks > (1ll << 30) || (int64_t)q->max_blocks * shape->page > 0x7fffffffll - 256) return HA_ERR_SHAPE;
  if ((int64_t)q->n_seq * q->max_blocks * shape->page > (1ll << 36)) return HA_ERR_SHAPE;  // (units of 64 tokens are counted in 32 bits)
  a->n_seq = q->n_seq;
  a->q_len = q->q_len;
  a->Hq = q->Hq;
  a->max_blocks = q->max_blocks;
  a->group = q->Hq / shape->Hk;
  a->rows = q->q_len * a->group;
  a->tiles = (a->rows + 15) / 16;
  a->parts = cache4_parts(shape->Hk, a->tiles);
  return HA_OK;
}

struct AttnSpace {
  size_t part_o, part_ml, total;
};
static AttnSpace attn_space(const CacheAttnArgs& a) {
  auto align = [](size_t x) { return (x + 255) & ~(size_t)255; };
  const size_t slots = (size_t)a.c.Hk * a.tiles * ((size_t)a.parts + a.n_seq) * 16;
  AttnSpace s;
  s.part_o = align((size_t)a.n_seq * 8);
  s.part_ml = s.part_o + align(slots * a.c.d * 4);
  s.total = s.part_ml + align(slots * 8);
  return s;
}

// Fills all of *a but the pointers and strides.
static int chunk_geometry(const ha_cache4* shape, const ha_cache4_chunk* q, CacheChunkArgs* a) {
  const int rc = cache_geometry(shape, &a->c);
  if (rc != HA_OK) return rc;
  if (!q) return HA_ERR_NULL;
  if (q->dtype != HA_BF16 && q->dtype != HA_FP32) return HA_ERR_DTYPE;
  if (q->n_seq < 0 || q->n_seq > (1 << 16) || q->rows < 0 || q->rows > (1 << 22) || q->max_blocks < 0) return HA_ERR_SHAPE;
  if (q->Hq < 1 || q->Hq > 1024 || q->Hq % shape->Hk != 0) return HA_ERR_SHAPE;
  if ((int64_t)q->rows * q->Hq > (1 << 26) || (int64_t)q->n_seq * q->Hq > (1 << 22)) return HA_ERR_SHAPE;
  if ((int64_t)q->n_seq * q->max_blocks > (1ll << 30) || (int64_t)q->max_blocks * shape->page > 0x7fffffffll - 256) return HA_ERR_SHAPE;
  if ((int64_t)q->n_seq * q->max_blocks * shape->page > (1ll << 36)) return HA_ERR_SHAPE;  // (units of 64 tokens are counted in 32 bits)
  a->n_seq = q->n_seq;
  a->rows = q->rows;
  a->Hq = q->Hq;
  a->max_blocks = q->max_blocks;
  a->group = q->Hq / shape->Hk;
  return HA_OK;
}

// Sets how the work is split, and both kinds' places in the workspace.
static size_t chunk_space(CacheChunkArgs* a, CacheAttnArgs* n, void* workspace) {
  cache4_chunk_split(a, n);
  unsigned char* const base = reinterpret_cast<unsigned char*>(workspace);
  size_t at = 0;
  auto take = [&](size_t bytes) {
    unsigned char* p = base + at;
    at += (bytes + 255) & ~(size_t)255;
    return p;
  };
  const size_t rows = 2 * (size_t)a->parts * kChunkRows;
  a->joins = reinterpret_cast<int32_t*>(take((size_t)a->parts * 32));
  a->part_o = reinterpret_cast<float*>(take(rows * a->c.d * 4));
  a->part_ml = reinterpret_cast<float*>(take(rows * 8));
  if (a->narrow && a->parts > 0) {
    const size_t slots = (size_t)a->c.Hk * n->parts * 2 * kNarrowRows;
    n->span = reinterpret_cast<int32_t*>(take((size_t)a->n_seq * 8));
    n->part_o = reinterpret_cast<float*>(take(slots * a->c.d * 4));
    n->part_ml = reinterpret_cast<float*>(take(slots * 8));
  }
  return at;
}

}  // namespace ha

using namespace ha;

extern "C" {

size_t ha_cache4_bytes(const ha_cache4* cache) {
  CacheGeometry c;
  return cache_geometry(cache, &c) == HA_OK ? (size_t)c.n_pages * c.Hk * c.block_bytes() : 0;
}

int ha_cache4_write(const void* K, const void* V, const int32_t* slots, void* cache, const ha_cache4* shape, int32_t rows, int32_t dtype,
                    const ha_strides* kv, void* stream) {
  return rows_call(K, V, slots, cache, shape, rows, dtype, kv, stream, true);
}

int ha_cache4_read(const void* cache, const int32_t* slots, void* K, void* V, const ha_cache4* shape, int32_t rows, int32_t dtype,
                   const ha_strides* kv, void* stream) {
  return rows_call(K, V, slots, cache, shape, rows, dtype, kv, stream, false);
}

size_t ha_cache4_attn_workspace_bytes(const ha_cache4* shape, const ha_cache4_query* query) {
  CacheAttnArgs a{};
  return attn_geometry(shape, query, &a) == HA_OK ? attn_space(a).total : 0;
}

int ha_cache4_attn_form(const ha_cache4* shape, const ha_cache4_query* query, int32_t* whole_waves, int32_t* past_caches) {
  if (!whole_waves || !past_caches) return HA_ERR_NULL;
  CacheAttnArgs a{};
  const int rc = attn_geometry(shape, query, &a);
  if (rc != HA_OK) return rc;
  if (a.c.n_pages == 0) a.max_blocks = 0;
  *whole_waves = cache4_whole(a);
  *past_caches = *whole_waves == 0 && cache4_once(a);
  return HA_OK;
}

int ha_cache4_attn(const void* Q, const void* cache, const int32_t* block_table, const int32_t* lens, void* out, float* lse,
                   const ha_cache4* shape, const ha_cache4_query* query, const ha_strides* qo, void* workspace, size_t workspace_bytes,
                   void* stream) {
  CacheAttnArgs a{};
  int rc = attn_geometry(shape, query, &a);
  if (rc != HA_OK) return rc;
  const int64_t rows = (int64_t)a.n_seq * a.q_len;
  rc = row_strides(qo, rows, a.Hq, a.c.d, query->dtype, false, &a.q);
  if (rc == HA_OK) rc = row_strides(qo ? qo + 1 : nullptr, rows, a.Hq, a.c.d, query->dtype, true, &a.o);
  if (rc != HA_OK) return rc;
  if (a.n_seq == 0) return HA_OK;
  if (!Q || !lens || !out || !lse || !workspace || (!cache && a.c.n_pages > 0) || (!block_table && a.max_blocks > 0)) return HA_ERR_NULL;
  if (any_misaligned16(Q, cache, out) || any_misaligned4(block_table, lens, lse)) return HA_ERR_ALIGN;
  const AttnSpace sp = attn_space(a);
  if (workspace_bytes < sp.total || ((uintptr_t)workspace & 255) != 0) return HA_ERR_WORKSPACE;
  if (a.c.n_pages == 0) a.max_blocks = 0;  // (no page is there: every sequence counts as empty)
  a.Q = Q;
  a.cache = reinterpret_cast<const unsigned char*>(cache);
  a.table = block_table;
  a.lens = lens;
  a.out = out;
  a.lse = lse;
  unsigned char* w = reinterpret_cast<unsigned char*>(workspace);
  a.span = reinterpret_cast<int32_t*>(w);
  a.part_o = reinterpret_cast<float*>(w + sp.part_o);
  a.part_ml = reinterpret_cast<float*>(w + sp.part_ml);
  return launch_cache4_attn(a, query->dtype, (hipStream_t)stream);
}

size_t ha_cache4_attn_chunk_workspace_bytes(const ha_cache4* shape, const ha_cache4_chunk* chunk) {
  CacheChunkArgs a{};
  CacheAttnArgs narrow{};
  return chunk_geometry(shape, chunk, &a) == HA_OK ? chunk_space(&a, &narrow, nullptr) : 0;
}

int ha_cache4_attn_chunk(const void* Q, const void* cache, const int32_t* cu_seqlens, const int32_t* block_table, const int32_t* lens, void* out,
                         float* lse, const ha_cache4* shape, const ha_cache4_chunk* chunk, const ha_strides* qo, void* workspace,
                         size_t workspace_bytes, void* stream) {
  CacheChunkArgs a{};
  CacheAttnArgs n{};
  int rc = chunk_geometry(shape, chunk, &a);
  if (rc != HA_OK) return rc;
  rc = row_strides(qo, a.rows, a.Hq, a.c.d, chunk->dtype, false, &a.q);
  if (rc == HA_OK) rc = row_strides(qo ? qo + 1 : nullptr, a.rows, a.Hq, a.c.d, chunk->dtype, true, &a.o);
  if (rc != HA_OK) return rc;
  if (a.n_seq == 0 || a.rows == 0) return HA_OK;
  const size_t space = chunk_space(&a, &n, workspace);
  if (!Q || !cu_seqlens || !lens || !out || !lse || (space > 0 && !workspace) || (!cache && a.c.n_pages > 0) || (!block_table && a.max_blocks > 0))
    return HA_ERR_NULL;
  if (any_misaligned16(Q, cache, out) || any_misaligned4(cu_seqlens, block_table, lens, lse)) return HA_ERR_ALIGN;
  if (workspace_bytes < space || ((uintptr_t)workspace & 255) != 0) return HA_ERR_WORKSPACE;
  if (a.c.n_pages == 0) a.max_blocks = 0;  // (no page is there: every sequence counts as empty)
  a.Q = Q;
  a.cache = reinterpret_cast<const unsigned char*>(cache);
  a.cu = cu_seqlens;
  a.table = block_table;
  a.lens = lens;
  a.out = out;
  a.lse = lse;
  n.Q = Q;
  n.cache = a.cache;
  n.table = block_table;
  n.lens = lens;
  n.out = out;
  n.lse = lse;
  n.c = a.c;
  n.q = a.q;
  n.o = a.o;
  n.n_seq = a.n_seq;
  n.Hq = a.Hq;
  n.max_blocks = a.max_blocks;
  n.group = a.group;
  n.rows = kNarrowRows;
  n.tiles = 1;
  n.cu = cu_seqlens;
  n.rows_all = a.rows;
  return launch_cache4_chunk(a, n, chunk->dtype, (hipStream_t)stream);
}

static size_t weights_space(const CacheChunkArgs& a, size_t* sums) {
  auto align = [](size_t x) { return (x + 255) & ~(size_t)255; };
  *sums = align((size_t)a.parts * 16);
  return *sums + align(2 * (size_t)a.parts * kWeightsTokens * 4);
}

size_t ha_cache4_weights_workspace_bytes(const ha_cache4* shape, const ha_cache4_chunk* chunk) {
  CacheChunkArgs a{};
  if (chunk_geometry(shape, chunk, &a) != HA_OK) return 0;
  cache4_weights_split(&a);
  size_t sums;
  return weights_space(a, &sums);
}

int ha_cache4_weights(const void* Q, const void* cache, const int32_t* cu_seqlens, const int32_t* block_table, const int32_t* lens, const float* lse,
                      float* weights, const ha_cache4* shape, const ha_cache4_chunk* chunk, int32_t fresh, const ha_strides* q, void* workspace,
                      size_t workspace_bytes, void* stream) {
  CacheChunkArgs a{};
  int rc = chunk_geometry(shape, chunk, &a);
  if (rc != HA_OK) return rc;
  rc = row_strides(q, a.rows, a.Hq, a.c.d, chunk->dtype, false, &a.q);
  if (rc != HA_OK) return rc;
  if (a.n_seq == 0 || a.c.n_pages == 0 || a.max_blocks == 0 || (a.rows == 0 && !fresh)) return HA_OK;
  cache4_weights_split(&a);
  size_t sums;
  const size_t total = weights_space(a, &sums);
  if ((a.rows > 0 && (!Q || !lse)) || !cache || !cu_seqlens || !block_table || !lens || !weights || (total > 0 && !workspace)) return HA_ERR_NULL;
  if (any_misaligned16(Q, cache, weights) || any_misaligned4(cu_seqlens, block_table, lens, lse)) return HA_ERR_ALIGN;
  if (workspace_bytes < total || ((uintptr_t)workspace & 255) != 0) return HA_ERR_WORKSPACE;
  a.Q = Q;
  a.cache = reinterpret_cast<const unsigned char*>(cache);
  a.cu = cu_seqlens;
  a.table = block_table;
  a.lens = lens;
  a.lse = const_cast<float*>(lse);
  a.weights = weights;
  a.fresh = fresh != 0;
  a.joins = reinterpret_cast<int32_t*>(workspace);
  a.part_o = reinterpret_cast<float*>(reinterpret_cast<unsigned char*>(workspace) + sums);
  return launch_cache4_weights(a, chunk->dtype, (hipStream_t)stream);
}

// Fills all of *a but the pointers.
static int evict_geometry(const ha_cache4* shape, const ha_cache4_eviction* e, CacheEvictArgs* a) {
  const int rc = cache_geometry(shape, &a->c);
  if (rc != HA_OK) return rc;
  if (!e) return HA_ERR_NULL;
  if (e->n_seq < 0 || e->n_seq > kEvictSeqs || e->max_blocks < 0 || e->recent < 0) return HA_ERR_SHAPE;
  if ((int64_t)e->n_seq * shape->Hk > (1 << 20) || (int64_t)e->n_seq * e->max_blocks > (1ll << 30)) return HA_ERR_SHAPE;
  if ((int64_t)e->max_blocks * shape->page > (1ll << 30)) return HA_ERR_SHAPE;
  a->n_seq = e->n_seq;
  a->max_blocks = e->max_blocks;
  a->recent = e->recent;
  a->moves_most = (int64_t)e->max_blocks * shape->page / 2;  // the places that come free are as many as the tokens that fill them, and neither count twice
  return HA_OK;
}

static size_t evict_space(const CacheEvictArgs& a, size_t* moves) {
  auto align = [](size_t x) { return (x + 255) & ~(size_t)255; };
  const size_t heads = (size_t)a.n_seq * a.c.Hk;
  *moves = align(heads * 8);
  return heads == 0 ? 0 : *moves + align(heads * (size_t)a.moves_most * 8);
}

size_t ha_cache4_evict_workspace_bytes(const ha_cache4* shape, const ha_cache4_eviction* evict) {
  CacheEvictArgs a{};
  size_t moves;
  return evict_geometry(shape, evict, &a) == HA_OK ? evict_space(a, &moves) : 0;
}

int ha_cache4_evict(void* cache, const float* weights, float* weights_out, const int32_t* block_table, const int32_t* lens, const int32_t* keep,
                    int32_t* free_pages, const int32_t* free_count, int32_t* lens_out, int32_t* free_count_out, const ha_cache4* shape,
                    const ha_cache4_eviction* evict, void* workspace, size_t workspace_bytes, void* stream) {
  CacheEvictArgs a{};
  const int rc = evict_geometry(shape, evict, &a);
  if (rc != HA_OK) return rc;
  size_t moves;
  const size_t total = evict_space(a, &moves);
  if (!free_count || !free_count_out || (total > 0 && !workspace)) return HA_ERR_NULL;
  if (a.c.n_pages > 0 && (!cache || !weights || !weights_out || !free_pages)) return HA_ERR_NULL;
  if (a.n_seq > 0 && (!lens || !keep || !lens_out || (a.max_blocks > 0 && !block_table))) return HA_ERR_NULL;
  if (any_misaligned16(cache, weights, weights_out)) return HA_ERR_ALIGN;
  if (any_misaligned4(block_table, lens, keep, free_pages) || any_misaligned4(free_count, lens_out, free_count_out)) return HA_ERR_ALIGN;
  auto apart = [](const int32_t* x, int32_t nx, const int32_t* y, int32_t ny) { return (uintptr_t)x >= (uintptr_t)(y + ny) || (uintptr_t)y >= (uintptr_t)(x + nx); };
  const int32_t n = a.n_seq;  // (one workgroup writes these numbers while others, or other threads of it, read)
  if (!apart(lens_out, n, lens, n) || !apart(lens_out, n, keep, n) || !apart(lens_out, n, free_count, 1)) return HA_ERR_SHAPE;
  if (!apart(free_count_out, 1, lens, n) || !apart(free_count_out, 1, keep, n) || !apart(free_count_out, 1, lens_out, n) || free_count == free_count_out) return HA_ERR_SHAPE;
  if (workspace_bytes < total || ((uintptr_t)workspace & 255) != 0) return HA_ERR_WORKSPACE;
  a.cache = reinterpret_cast<unsigned char*>(cache);
  a.weights = weights;
  a.weights_out = weights_out;
  a.table = block_table;
  a.lens = lens;
  a.keep = keep;
  a.free_pages = free_pages;
  a.free_count = free_count;
  a.lens_out = lens_out;
  a.free_count_out = free_count_out;
  a.counts = reinterpret_cast<int2*>(workspace);
  a.moves = reinterpret_cast<int2*>(reinterpret_cast<unsigned char*>(workspace) + moves);
  return launch_cache4_evict(a, (hipStream_t)stream);
}

int ha_page_plan(const int32_t* lens, const int32_t* add, int32_t* block_table, int32_t* free_pages, const int32_t* free_count,
                 int32_t* lens_out, int32_t* cu_seqlens, int32_t* slots, int32_t* free_count_out, const ha_page_plan_shape* sh,
                 void* stream) {
  if (!sh) return HA_ERR_NULL;
  PagePlanArgs a{};
  a.log_page = log2_page(sh->page);
  if (a.log_page < 0 || sh->n_seq < 0 || sh->n_seq > 8192 || sh->rows < 0 || sh->rows > (1 << 26)) return HA_ERR_SHAPE;
  if (sh->max_blocks < 0 || (int64_t)sh->n_seq * sh->max_blocks > (1ll << 30) || (int64_t)sh->max_blocks * sh->page > 0x7fffffffll - 256)
    return HA_ERR_SHAPE;
  if (sh->n_pages < 0 || (int64_t)sh->n_pages * sh->page > 0x7fffffffll) return HA_ERR_SHAPE;
  if (!cu_seqlens || !free_count || !free_count_out || (sh->rows > 0 && !slots) || (sh->n_pages > 0 && !free_pages)) return HA_ERR_NULL;
  if (sh->n_seq > 0 && (!lens || !add || !lens_out || (sh->max_blocks > 0 && !block_table))) return HA_ERR_NULL;
  if (any_misaligned4(lens, add, block_table, free_pages, free_count, lens_out) || any_misaligned4(cu_seqlens, slots, free_count_out)) return HA_ERR_ALIGN;
  if (free_count == free_count_out || (sh->n_seq > 0 && lens == lens_out)) return HA_ERR_SHAPE;  // (read by workgroups that others write ahead of)
  a.lens = lens;
  a.add = add;
  a.table = block_table;
  a.free_pages = free_pages;
  a.free_count = free_count;
  a.lens_out = lens_out;
  a.cu = cu_seqlens;
  a.slots = slots;
  a.free_count_out = free_count_out;
  a.n_seq = sh->n_seq;
  a.max_blocks = sh->max_blocks;
  a.page = sh->page;
  a.n_pages = sh->n_pages;
  a.rows = sh->rows;
  return launch_page_plan(a, (hipStream_t)stream);
}

}  // extern "C"
