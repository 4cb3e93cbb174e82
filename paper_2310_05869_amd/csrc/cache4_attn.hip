// Launches of attention over each sequence's last tokens (cache4_attn.h) and their rules.
#include "cache4_attn.h"

namespace ha {

template <int D, int SPLIT, int NW, bool WHOLE, bool ONCE, bool MULTI>
__global__ __launch_bounds__(64 * NW, SPLIT == 1 && NW == 4 ? 3 : 2) void cache4_attn_kernel(CacheAttnArgs a) {
  __shared__ CacheAttnLds<D, NW> lds;
  cache4_attn_run<D, SPLIT, NW, WHOLE, ONCE, MULTI, false>(a, lds, blockIdx.x, blockIdx.y);
}

template <int D, int SPLIT>
__global__ __launch_bounds__(kJoinThreads) void cache4_join_kernel(CacheAttnArgs a) {
  __shared__ CacheJoinLds<D, SPLIT> lds;
  cache4_join_run<D, SPLIT, false>(a, lds, blockIdx.x, blockIdx.y, (int64_t)(gridDim.x * gridDim.y));
}

// Tables of few tokens: a workgroup takes a whole sequence, and there is no second launch; of eight waves (which fill a CU) where there are few, else of four.
// Up to 2048 tokens from 64 workgroups on.  Shared out -> whole (MI355X, us; [workgroups]): one sequence of 777 tokens, 4 key heads, d = 64 [4] 11.2 -> 8.6; 8 of
// 1024 [64] 11.1 -> 9.0; tables of 2048: 32 sequences, 8 key heads, d = 128 [256] 21.4 -> 16.0, but one [8] 11.2 -> 12.4; 60 of 2048, d = 64, fp32 [480] 39.8 -> 26.2;
// 256 of up to 2048 [2048] 34.4 -> 38.8.  Eight waves -> four: 200 of up to 500, four queries each [1600] 28.7 -> 16.1; 32 of 2048 [256] 16.0 -> 18.8
int cache4_whole(const CacheAttnArgs& a) {
  const int64_t tokens = (int64_t)a.max_blocks * a.c.page, wgs = (int64_t)a.n_seq * a.c.Hk * a.tiles;
  if (tokens > 1024 && (tokens > 2048 || wgs < 64 || wgs > 512)) return 0;
  return wgs > 256 ? 4 : 8;
}

// Codes that are read once are read past the caches where the table has room for more of them than the last cache holds.  Between two calls over the same pages a program's
// other layers read theirs, so codes come from memory; without the detour through the caches they come sooner, however many of the table's entries are used (tables
// of 131072 tokens, states of 79 to 307 MB in turn: 64 sequences of up to 2000 29.5 -> 26.9 us, 16 of up to 16384 38.9 -> 35.2, 64 of up to 8000 62.2 +-0.6; of up to 32768: 256 of
// up to 1000 49.0 -> 45.3; 64 of up to 16384, three queries each 44.6 -> 42.2; 4 of 131072 114 -> 103).  The price is paid where one call's codes, up to 160 MB, are still
// there for the next: the same, same state: 26.7 -> 28.0, 34.3 -> 37.2, 41.4 -> 45.3, 39.8 -> 42.0; a small program, whose table has no room for more, goes without.
bool cache4_once(const CacheAttnArgs& a) {
  return a.tiles == 1 && (int64_t)a.n_seq * a.max_blocks * a.c.Hk * a.c.block_bytes() > (256ll << 20);
}

// Workgroups that share a key head's tokens
int cache4_parts(int Hk, int tiles) {
  const int heads = Hk * tiles;
  return heads >= kMostParts ? 1 : kMostParts / heads;
}

template <int D, int SPLIT, bool MULTI>
static int launch_attn_form(const CacheAttnArgs& a, hipStream_t st) {
  if (const int waves = cache4_whole(a)) {
    const dim3 grid((unsigned)a.n_seq, (unsigned)(a.c.Hk * a.tiles));
    if (waves == 8) hipLaunchKernelGGL((cache4_attn_kernel<D, SPLIT, 8, true, false, MULTI>), grid, dim3(512), 0, st, a);
    else hipLaunchKernelGGL((cache4_attn_kernel<D, SPLIT, 4, true, false, MULTI>), grid, dim3(256), 0, st, a);
    return check_launch();
  }
  const dim3 grid((unsigned)a.parts, (unsigned)(a.c.Hk * a.tiles));
  if (cache4_once(a)) hipLaunchKernelGGL((cache4_attn_kernel<D, SPLIT, 4, false, true, MULTI>), grid, dim3(256), 0, st, a);
  else hipLaunchKernelGGL((cache4_attn_kernel<D, SPLIT, 4, false, false, MULTI>), grid, dim3(256), 0, st, a);
  const int rc = check_launch();
  if (rc != HA_OK) return rc;
  hipLaunchKernelGGL((cache4_join_kernel<D, SPLIT>), dim3((unsigned)a.n_seq, (unsigned)(a.Hq * a.q_len)), dim3(kJoinThreads), 0, st, a);
  return check_launch();
}

template <int D, int SPLIT>
static int launch_attn_q(const CacheAttnArgs& a, hipStream_t st) {
  return a.q_len > 1 ? launch_attn_form<D, SPLIT, true>(a, st) : launch_attn_form<D, SPLIT, false>(a, st);
}

int launch_cache4_attn(const CacheAttnArgs& a, int dtype, hipStream_t st) {
  if (a.c.d == 128) return dtype == HA_BF16 ? launch_attn_q<128, 1>(a, st) : launch_attn_q<128, 3>(a, st);
  return dtype == HA_BF16 ? launch_attn_q<64, 1>(a, st) : launch_attn_q<64, 3>(a, st);
}

}  // namespace ha
