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
