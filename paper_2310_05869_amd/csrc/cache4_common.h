// The paged 4-bit cache (include/hyperattn.h has its format): addresses of a page's parts and the launchers of its kernels.
//
// Why the codes lie as they do: the attention kernel takes 16 tokens at a time in operands of v_mfma_f32_16x16x32_bf16, whose lane (l % 16,
// l / 16) holds eight contraction elements of one row.
//   scores   contraction over channels: row = token l % 16, elements = channels 8 (l / 16) ... + 7 of a group of 32.  K's words are ordered by l / 16
//            first, so that a lane's d / 32 words, one per group, are one piece of 8 or 16 bytes, and a wave's load is whole lines.
//   P V      contraction over tokens: row = channel, elements = tokens 4 (l / 16) ... + 3 of two runs of 16 tokens.  Four tokens' words of the same
//            channels lie together, so that a lane has its four tokens in one piece of 16 bytes, and a token still owns whole words: rows
//            can be written one by one.
#pragma once

#include "ha_common.h"

namespace ha {

constexpr int kCacheGroup = 32;   // channels of a scale
constexpr int kLeastScale = 2, kLargestScale = 252;

struct CacheGeometry {
  int32_t n_pages, page, log_page, Hk, d;
  __host__ __device__ int token_bytes() const { return d + d / 16; }
  __host__ __device__ int64_t block_bytes() const { return (int64_t)page * token_bytes(); }  // of a page and head
  __host__ __device__ int v_at() const { return page * (d / 2); }
  __host__ __device__ int k_scale_at() const { return page * d; }
  __host__ __device__ int v_scale_at() const { return page * (d + d / kCacheGroup); }
};

struct CacheRowsArgs {
  const int32_t* slots;
  void* K;
  void* V;
  unsigned char* cache;
  CacheGeometry c;
  RowStrides k, v;
  int32_t rows;
};
int launch_cache4_write(const CacheRowsArgs& a, int dtype, hipStream_t st);
int launch_cache4_read(const CacheRowsArgs& a, int dtype, hipStream_t st);

struct CacheAttnArgs {
  const void* Q;
  const unsigned char* cache;
  const int32_t* table;
  const int32_t* lens;
  void* out;
  float* lse;
  CacheGeometry c;
  RowStrides q, o;
  int32_t n_seq, q_len, Hq, max_blocks;
  int32_t group, rows, tiles;  // query heads per key head, query rows per (sequence, key head), tiles of 16 of those
  int32_t parts;               // workgroups that share a key head's tokens
  // workspace: first and last workgroup of a sequence; per key head, tile of rows, and part: 16 rows of sums, their references and row sums
  int32_t* span;               // [n_seq][2]
  float* part_o;
  float* part_ml;
};
int launch_cache4_attn(const CacheAttnArgs& a, int dtype, hipStream_t st);
int cache4_parts(int Hk, int tiles);
int cache4_whole(const CacheAttnArgs& a);   // waves of a workgroup that takes a whole sequence, 0: tokens are shared out
bool cache4_once(const CacheAttnArgs& a);   // of shared-out tokens: codes are read past the caches

struct PagePlanArgs {
  const int32_t* lens;
  const int32_t* add;
  int32_t* table;
  int32_t* free_pages;
  const int32_t* free_count;
  int32_t* lens_out;
  int32_t* cu;
  int32_t* slots;
  int32_t* free_count_out;
  int32_t n_seq, max_blocks, page, log_page, n_pages, rows;
  int32_t slot_wgs;  // set by the launcher
};
int launch_page_plan(const PagePlanArgs& a, hipStream_t st);

}  // namespace ha
