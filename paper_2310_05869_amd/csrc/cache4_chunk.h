// Chunks of new tokens over the paged 4-bit cache: how work is found from lengths that only the device knows.  Shared by attention (cache4_chunk.hip) and by
// the sums of attention weights (cache4_weights.hip).
//
// Sequence s brings n_s new tokens, rows cu[s] ... cu[s + 1] - 1 of Q, the last of the lens[s] that the cache holds of it.  The query heads of a key head
// read the same keys, so a tile of query rows holds all of them for some tokens: row r is token r / sub_group of the tile, head r % sub_group.  A key head with
// more query heads than a tile has rows counts as several ("heads" below: key heads times these runs).
#pragma once

#include "attn_common.h"
#include "cache4_common.h"

namespace ha {

struct ChunkSeq {
  int start, n;   // rows
  int len, held;  // tokens in the cache, those before the new ones (negative: more rows than tokens; the first rows see nothing)
};

__device__ inline ChunkSeq chunk_seq(const CacheChunkArgs& a, int s) {
  ChunkSeq q;
  q.start = min(max(a.cu[s], 0), a.rows);
  q.n = max(min(max(a.cu[s + 1], 0), a.rows) - q.start, 0);
  q.len = min(max(a.lens[s], 0), a.max_blocks << a.c.log_page);
  q.held = q.len - q.n;
  return q;
}

__device__ inline ChunkSeq uniform_seq(ChunkSeq q) {
  q.start = __builtin_amdgcn_readfirstlane(q.start);
  q.n = __builtin_amdgcn_readfirstlane(q.n);
  q.len = __builtin_amdgcn_readfirstlane(q.len);
  q.held = __builtin_amdgcn_readfirstlane(q.held);
  return q;
}

__device__ inline int64_t uniform64(int64_t x) {
  const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)x), hi = __builtin_amdgcn_readfirstlane((uint32_t)(x >> 32));
  return (int64_t)((uint64_t)hi << 32 | lo);
}

// Attention: the line before tile t of a key head whose sequence held `held` tokens before its new ones, `tile_tokens` of these a tile and `tile_cost` for its start and end.
__host__ __device__ constexpr int64_t chunk_upto(int held, int tile_tokens, int64_t t, int tile_cost) {
  return t * ((int64_t)(held > 0 ? held : 0) + tile_cost) + tile_tokens * (t * (t + 1) / 2);
}

// Scale i of a token's, as the conversions take it
__device__ inline float scale_of(uint32_t bytes, int i) { return __uint_as_float(i < 3 ? bytes << (23 - 8 * i) : bytes >> 1); }  // (the exponent alone counts)

// Where run p of `parts` begins on a line.  (Rounded down from a product in double, by every workgroup alike; a division of 64 bits takes a microsecond.)
__device__ inline int64_t run_begin(int64_t total, int parts, int p) { return p >= parts ? total : (int64_t)((double)total * ((double)p / (double)parts)); }

// x / y, rounded down, for x of less than 2^62 and quotients of less than 2^31
__device__ inline int whole_part(int64_t x, int64_t y) {
  int64_t n = (int64_t)((double)x / (double)y);
  while (n * y > x) --n;
  while ((n + 1) * y <= x) ++n;
  return (int)n;
}

// The run of `parts` that place x lies in
__device__ inline int run_of(int64_t total, int parts, int64_t x) {
  int p = min((int)((double)x / (double)total * parts), parts - 1);
  while (p > 0 && run_begin(total, parts, p) > x) --p;
  while (run_begin(total, parts, p + 1) <= x) ++p;
  return p;
}

// All sequences' work as one line: sequence s takes cost(s) >= 0 of it.  A lane sums a run of sequences; the sum is the same for all lanes, *before: what
// precedes the lane's run.  Row starts that decrease can give the same rows to many sequences: with more rows in all than there are, there is no work.
template <class Cost>
__device__ inline int64_t chunk_line(const CacheChunkArgs& a, int lane, int64_t* before, Cost&& cost) {
  const int each = (a.n_seq + 63) / 64, s0 = min(a.n_seq, lane * each), s1 = min(a.n_seq, s0 + each);
  int64_t sum = 0;
  float rows = 0.f;  // (exact up to 2^24, rows are at most 2^22)
  for (int s = s0; s < s1; ++s) {
    sum += cost(s);
    rows += (float)chunk_seq(a, s).n;
  }
  int64_t inc = sum;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int64_t up = __shfl_up((long long)inc, o);
    if (lane >= o) inc += up;
    rows += __shfl_xor(rows, o);
  }
  *before = inc - sum;
  return __any(rows > (float)a.rows) ? 0 : uniform64(__shfl((long long)inc, 63));
}

// The sequence at place u of the line (0 <= u < its length), and where it begins
template <class Cost>
__device__ inline int chunk_place(int n_seq, int64_t before, int64_t u, int64_t* first, Cost&& cost) {
  const int each = (n_seq + 63) / 64;
  const unsigned long long le = __ballot(before <= u);  // (runs without work begin where the next one does)
  const int run = 63 - __builtin_clzll(le);
  int64_t at = uniform64(__shfl((long long)before, run));
  int s = min(run * each, n_seq - 1);
  for (; s < n_seq - 1; ++s) {
    const int64_t n = uniform64(cost(s));
    if (u < at + n) break;
    at += n;
  }
  *first = at;
  return __builtin_amdgcn_readfirstlane(s);
}

}  // namespace ha
