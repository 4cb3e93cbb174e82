// Eviction from the 4-bit cache by accumulated attention weight (ha_cache4_evict): a sequence longer than its budget keeps its last tokens and, for every key
// head, those of most weight among the others.
//
// Of n tokens k stay, r of them the last ones; the other k - r are the largest of n - r.  Kept tokens among the first k - r places stay where they are, the others move
// into the places that come free there, first to first: in a steady state a step moves as many rows as it lets go, where closing up would move nearly all.
// Then the last r follow, in order.  Three launches:
//   select   a workgroup per sequence and key head finds the (k - r)-th largest weight by three histograms of 11, 11 and 10 bits of the weights' bits, made so that they
//            order as numbers do, then who moves where from prefix sums: with c(p) tokens kept before place p, a free place p is the (p - c(p))-th, a kept token the
//            (c(p) - c(k - r))-th that moves.  A wave has a run of places of its own, so that only 16 numbers cross the waves.
//   move     rows of these lists, D / 8 lanes a row
//   last     the last r rows, whose places may overlap: read, a barrier, written, some hundred at a time; lengths and free pages
// Bound by latency: the weights that are chosen from are 4 bytes a token and head beside 136 of its rows.
#include <type_traits>

#include "cache4_common.h"

namespace ha {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kBins = 2048;
constexpr int kMoveThreads = 256, kLastThreads = 1024;

struct EvictSeq {
  int n, k, r;  // tokens, those that stay, the last ones among these
};
__device__ inline EvictSeq evict_seq(const CacheEvictArgs& a, int s) {
  EvictSeq q;
  q.n = min(max(a.lens[s], 0), a.max_blocks << a.c.log_page);
  const int keep = a.keep[s];
  q.k = keep < 0 ? q.n : min(keep, q.n);
  q.r = min(a.recent, q.k);
  return q;
}

// Bits that order as the numbers do; NaN below all of them, -0 as 0.  0 stands for no token.
__device__ inline uint32_t order_of(float x) {
  const uint32_t u = __float_as_uint(x);
  if (x != x) return 1u;
  if (x == 0.f) return 0x80000000u;
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// Sum of the values of the threads before (exclusive) and of all; one barrier before the scratch may be written again is the caller's
template <int NT>
__device__ inline uint32_t block_scan(uint32_t x, uint32_t* all, uint32_t* scratch) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  uint32_t inc = x;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const uint32_t up = __shfl_up(inc, o);
    if (lane >= o) inc += up;
  }
  if (lane == 63) scratch[wave] = inc;
  __syncthreads();
  uint32_t before = 0, total = 0;
#pragma unroll
  for (int w = 0; w < NT / 64; ++w) {
    const uint32_t n = scratch[w];
    if (w < wave) before += n;
    total += n;
  }
  *all = total;
  return before + inc - x;
}

template <int NT>
struct SelectLds {
  uint32_t hist[kBins];
  uint32_t scratch[NT / 64];
  uint32_t gt[NT / 64], eq[NT / 64];  // kept for certain, and equal to the limit, of every wave's places
  uint32_t gt_head, eq_head;          // among the first k - r places
  uint32_t bin, want;
};

// HELD: the weights are few enough to stay in registers, eight pieces of four a thread
template <int NT, bool HELD>
__device__ inline void select_moves(const CacheEvictArgs& a, const EvictSeq& q, int s, int kv, SelectLds<NT>& lds) {
  constexpr int NW = NT / 64, PIECES = 8;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int from = q.n - q.r, stay = q.k - q.r;  // places that are chosen from, and how many of them
  const int32_t* blocks = a.table + (int64_t)s * a.max_blocks;
  const int per = (from + NW * 256 - 1) / (NW * 256);  // pieces of 256 places a wave
  const int place0 = wave * per * 256 + lane * 4;
  auto fetch = [&](int i) {
    const int p = place0 + i * 256;
    u32x4 key = {0, 0, 0, 0};
    if (i < per && p < from) {
      const int page = blocks[p >> a.c.log_page];
      const bool there = (unsigned)page < (unsigned)a.c.n_pages;
      f32x4 x = {0.f, 0.f, 0.f, 0.f};
      if (there) x = *reinterpret_cast<const f32x4*>(a.weights + ((int64_t)page * a.c.Hk + kv) * a.c.page + (p & (a.c.page - 1)));
#pragma unroll
      for (int e = 0; e < 4; ++e) key[e] = p + e >= from ? 0u : there ? order_of(x[e]) : 1u;
    }
    return key;
  };
  u32x4 held[HELD ? PIECES : 1];
  if constexpr (HELD) {
#pragma unroll
    for (int i = 0; i < PIECES; ++i) held[i] = fetch(i);
  }
  auto all_keys = [&](auto&& f) {  // f(piece, its keys)
    if constexpr (HELD) {
#pragma unroll
      for (int i = 0; i < PIECES; ++i)
        if (i < per) f(i, held[i]);
    } else {
      for (int i = 0; i < per; ++i) f(i, fetch(i));
    }
  };

  uint32_t prefix = 0, want = stay;
#pragma unroll
  for (int pass = 0; pass < 3; ++pass) {
    const int bits = pass == 2 ? 10 : 11, shift = pass == 0 ? 21 : pass == 1 ? 10 : 0;
    for (int i = threadIdx.x; i < kBins; i += NT) lds.hist[i] = 0;
    __syncthreads();
    all_keys([&](int, const u32x4& key) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const bool in = key[e] != 0 && (pass == 0 || key[e] >> (shift + bits) == prefix);
        const uint32_t bin = (key[e] >> shift) & ((1u << bits) - 1);
        // (weights that are all alike, zeros say, would queue for one counter: the first lane's bin is counted for all that have it)
        const unsigned long long some = __ballot(in);
        if (some == 0) continue;
        const int lead = __builtin_ctzll(some);
        const uint32_t first = __builtin_amdgcn_readlane(bin, lead);
        const unsigned long long same = __ballot(in && bin == first);
        if (lane == lead) atomicAdd(&lds.hist[first], (uint32_t)__popcll(same));
        else if (in && bin != first) atomicAdd(&lds.hist[bin], 1u);
      }
    });
    __syncthreads();
    constexpr int EACH = kBins / NT;
    uint32_t mine = 0, total;
#pragma unroll
    for (int j = 0; j < EACH; ++j) mine += lds.hist[kBins - 1 - (threadIdx.x * EACH + j)];  // from the largest down
    uint32_t above = block_scan<NT>(mine, &total, lds.scratch);
    if (above < want && want <= above + mine) {
      for (int j = 0; j < EACH; ++j) {
        const int bin = kBins - 1 - (threadIdx.x * EACH + j);
        const uint32_t here = lds.hist[bin];
        if (want <= above + here) {
          lds.bin = bin;
          lds.want = want - above;
          break;
        }
        above += here;
      }
    }
    __syncthreads();
    prefix = prefix << bits | lds.bin;
    want = lds.want;
  }

  // prefix: the last one that is kept; of those equal to it, the first `want`
  uint32_t gt = 0, eq = 0, gt_head = 0, eq_head = 0;
  all_keys([&](int i, const u32x4& key) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const bool head = place0 + i * 256 + e < stay;
      const unsigned long long g = __ballot(key[e] > prefix), q2 = __ballot(key[e] == prefix), h = __ballot(head);
      gt += __popcll(g);
      eq += __popcll(q2);
      gt_head += __popcll(g & h);
      eq_head += __popcll(q2 & h);
    }
  });
  if (threadIdx.x == 0) lds.gt_head = lds.eq_head = 0;
  if (lane == 0) {
    lds.gt[wave] = gt;
    lds.eq[wave] = eq;
  }
  __syncthreads();
  if (lane == 0) {
    atomicAdd(&lds.gt_head, gt_head);
    atomicAdd(&lds.eq_head, eq_head);
  }
  __syncthreads();
  const uint32_t kept_head = lds.gt_head + min(lds.eq_head, want);  // kept among the first k - r places
  uint32_t gt_before = 0, eq_before = 0;
  for (int w = 0; w < wave; ++w) {
    gt_before += lds.gt[w];
    eq_before += lds.eq[w];
  }
  int2* moves = a.moves + ((int64_t)s * a.c.Hk + kv) * a.moves_most;
  all_keys([&](int i, const u32x4& key) {
    uint32_t here = 0;  // kept for certain in the upper half, equal in the lower
#pragma unroll
    for (int e = 0; e < 4; ++e) here += key[e] > prefix ? 0x10000u : key[e] == prefix ? 1u : 0u;
    uint32_t inc = here;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const uint32_t up = __shfl_up(inc, o);
      if (lane >= o) inc += up;
    }
    uint32_t g = gt_before + ((inc - here) >> 16), t = eq_before + ((inc - here) & 0xffffu);
    const uint32_t both = __builtin_amdgcn_readlane(inc, 63);
    gt_before += both >> 16;
    eq_before += both & 0xffffu;
    const int p = place0 + i * 256;
    const int page = p < from ? blocks[p >> a.c.log_page] : -1;
    const int slot = (unsigned)page < (unsigned)a.c.n_pages ? (page << a.c.log_page) + (p & (a.c.page - 1)) : -4;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const bool more = key[e] > prefix, same = key[e] == prefix, kept = more || (same && t < want);
      const uint32_t rank = g + min(t, want);  // kept before
      if (kept && p + e >= stay) moves[rank - kept_head].x = slot + e;
      if (!kept && p + e < stay) moves[p + e - rank].y = slot + e;
      g += more;
      t += same;
    }
  });
  if (threadIdx.x == 0) a.counts[s * a.c.Hk + kv] = stay - (int)kept_head;
}

template <int NT>
__global__ __launch_bounds__(NT) void cache4_select_kernel(CacheEvictArgs a) {
  __shared__ SelectLds<NT> lds;
  const int s = blockIdx.x / a.c.Hk, kv = blockIdx.x - s * a.c.Hk;
  const EvictSeq q = evict_seq(a, s);
  if (q.k == q.n || q.k == q.r) {
    if (threadIdx.x == 0) a.counts[blockIdx.x] = 0;
    return;
  }
  if (q.n - q.r <= NT * 32) select_moves<NT, true>(a, q, s, kv, lds);
  else select_moves<NT, false>(a, q, s, kv, lds);
}

// A row's share of a lane: lane j of D / 8 has word j of K and of V; the first three also K's scales, V's and the weight
template <int D>
struct RowPiece {
  uint32_t k, v, more;
};
template <int D>
__device__ inline RowPiece<D> load_piece(const CacheEvictArgs& a, int kv, int slot, int j) {
  const int64_t head = (int64_t)(slot >> a.c.log_page) * a.c.Hk + kv;
  const int t = slot & (a.c.page - 1);
  const unsigned char* b = a.cache + head * a.c.block_bytes();
  RowPiece<D> x;
  x.k = *reinterpret_cast<const uint32_t*>(b + t * (D / 2) + 4 * j);
  x.v = *reinterpret_cast<const uint32_t*>(b + a.c.v_at() + (t >> 2) * (D * 2) + j * 16 + (t & 3) * 4);
  x.more = 0;
  using Scales = std::conditional_t<D == 128, uint32_t, uint16_t>;
  if (j < 2) x.more = *reinterpret_cast<const Scales*>(b + (j == 0 ? a.c.k_scale_at() : a.c.v_scale_at()) + t * (D / kCacheGroup));
  else if (j == 2) x.more = __float_as_uint(a.weights[head * a.c.page + t]);
  return x;
}
template <int D>
__device__ inline void store_piece(const CacheEvictArgs& a, int kv, int slot, int j, const RowPiece<D>& x) {
  const int64_t head = (int64_t)(slot >> a.c.log_page) * a.c.Hk + kv;
  const int t = slot & (a.c.page - 1);
  unsigned char* b = a.cache + head * a.c.block_bytes();
  *reinterpret_cast<uint32_t*>(b + t * (D / 2) + 4 * j) = x.k;
  *reinterpret_cast<uint32_t*>(b + a.c.v_at() + (t >> 2) * (D * 2) + j * 16 + (t & 3) * 4) = x.v;
  using Scales = std::conditional_t<D == 128, uint32_t, uint16_t>;
  if (j < 2) *reinterpret_cast<Scales*>(b + (j == 0 ? a.c.k_scale_at() : a.c.v_scale_at()) + t * (D / kCacheGroup)) = (Scales)x.more;
  else if (j == 2) a.weights_out[head * a.c.page + t] = __uint_as_float(x.more);
}

template <int D>
__global__ __launch_bounds__(kMoveThreads) void cache4_move_kernel(CacheEvictArgs a) {
  constexpr int LPR = D / 8, ROWS = kMoveThreads / LPR, AHEAD = 4;
  const int count = a.counts[blockIdx.x], kv = blockIdx.x % a.c.Hk, j = threadIdx.x % LPR;
  const int2* moves = a.moves + (int64_t)blockIdx.x * a.moves_most;
  for (int i0 = blockIdx.y * ROWS * AHEAD + threadIdx.x / LPR; i0 < count; i0 += gridDim.y * ROWS * AHEAD) {
    int2 m[AHEAD];
    RowPiece<D> x[AHEAD];
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      const int i = i0 + u * ROWS;
      m[u] = i < count ? moves[i] : int2{-1, -1};
      if (m[u].x >= 0) x[u] = load_piece<D>(a, kv, m[u].x, j);
    }
#pragma unroll
    for (int u = 0; u < AHEAD; ++u)
      if (m[u].x >= 0 && m[u].y >= 0) store_piece<D>(a, kv, m[u].y, j, x[u]);
  }
}

template <int D>
__global__ __launch_bounds__(kLastThreads) void cache4_last_kernel(CacheEvictArgs a) {
  constexpr int LPR = D / 8, ROWS = kLastThreads / LPR, AHEAD = 4;
  extern __shared__ uint32_t upto[];  // pages that sequences before give back
  __shared__ uint32_t scratch[kLastThreads / 64];
  if ((int)blockIdx.x < a.n_seq * a.c.Hk) {
    const int s = blockIdx.x / a.c.Hk, kv = blockIdx.x - s * a.c.Hk, j = threadIdx.x % LPR;
    const EvictSeq q = evict_seq(a, s);
    if (q.k == q.n) return;
    const int32_t* blocks = a.table + (int64_t)s * a.max_blocks;
    auto slot_of = [&](int p) {
      const int page = blocks[p >> a.c.log_page];
      return (unsigned)page < (unsigned)a.c.n_pages ? (page << a.c.log_page) + (p & (a.c.page - 1)) : -1;
    };
    // rows that lie apart from their places are shared among workgroups; else one takes them in order: what it writes lies before what is still to be read
    const bool apart = q.n - q.k >= q.r;
    if (!apart && blockIdx.y > 0) return;
    for (int i0 = apart ? blockIdx.y * ROWS * AHEAD : 0; i0 < q.r; i0 += (apart ? gridDim.y : 1) * ROWS * AHEAD) {
      int to[AHEAD];
      RowPiece<D> x[AHEAD];
#pragma unroll
      for (int u = 0; u < AHEAD; ++u) {
        const int i = i0 + u * ROWS + threadIdx.x / LPR;
        to[u] = -1;
        x[u] = RowPiece<D>{0, 0, 0};
        if (i < q.r) {
          const int at = slot_of(q.n - q.r + i);
          if (at >= 0) {
            to[u] = slot_of(q.k - q.r + i);
            x[u] = load_piece<D>(a, kv, at, j);
          }
        }
      }
#pragma unroll
      for (int u = 0; u < AHEAD; ++u) asm volatile("" : "+v"(x[u].k), "+v"(x[u].v), "+v"(x[u].more));  // (all of them are here before the barrier)
      __syncthreads();
#pragma unroll
      for (int u = 0; u < AHEAD; ++u)
        if (to[u] >= 0) store_piece<D>(a, kv, to[u], j, x[u]);
    }
    return;
  }
  if (blockIdx.y > 0) return;
  // ---- lengths, and the pages that come free, on top of the stack in order ----
  auto pages_of = [&](int tokens) { return (int)(((int64_t)tokens + a.c.page - 1) >> a.c.log_page); };
  const int count = min(max(*a.free_count, 0), a.c.n_pages);
  const int each = (a.n_seq + kLastThreads - 1) / kLastThreads, s0 = min(a.n_seq, (int)threadIdx.x * each), s1 = min(a.n_seq, s0 + each);
  uint32_t mine = 0, all;
  for (int s = s0; s < s1; ++s) {
    const EvictSeq q = evict_seq(a, s);
    a.lens_out[s] = q.k;
    upto[s] = mine;
    mine += pages_of(q.n) - pages_of(q.k);
  }
  const uint32_t before = block_scan<kLastThreads>(mine, &all, scratch);
  for (int s = s0; s < s1; ++s) upto[s] += before;
  __syncthreads();
  if (threadIdx.x == 0) *a.free_count_out = (int)min((int64_t)count + all, (int64_t)a.c.n_pages);
  for (int s = threadIdx.x >> 6; s < a.n_seq; s += kLastThreads / 64) {
    const EvictSeq q = evict_seq(a, s);
    const int left = pages_of(q.k), freed = pages_of(q.n) - left;
    for (int i = threadIdx.x & 63; i < freed; i += 64) {
      const int64_t at = (int64_t)count + upto[s] + i;
      if (at < a.c.n_pages) a.free_pages[at] = a.table[(int64_t)s * a.max_blocks + left + i];
    }
  }
}

template <int D>
static int launch_evict_d(const CacheEvictArgs& a, hipStream_t st) {
  const int64_t tokens = (int64_t)a.max_blocks << a.c.log_page;
  const int heads = a.n_seq * a.c.Hk;
  if (heads > 0 && tokens > 0) {
    if (tokens <= 256 * 32) hipLaunchKernelGGL(cache4_select_kernel<256>, dim3(heads), dim3(256), 0, st, a);
    else hipLaunchKernelGGL(cache4_select_kernel<1024>, dim3(heads), dim3(1024), 0, st, a);
    int rc = check_launch();
    if (rc != HA_OK) return rc;
    constexpr int64_t per = 4 * kMoveThreads / (D / 8);
    const int64_t most = (a.moves_most + per - 1) / per, fill = 2048 / heads + 1;
    hipLaunchKernelGGL(cache4_move_kernel<D>, dim3(heads, (unsigned)(most < fill ? most : fill)), dim3(kMoveThreads), 0, st, a);
    rc = check_launch();
    if (rc != HA_OK) return rc;
  }
  constexpr int64_t per = 4 * kLastThreads / (D / 8);
  const int64_t most = ((int64_t)a.recent + per - 1) / per + 1, fill = 512 / (heads + 1) + 1;
  const size_t lds = ((size_t)a.n_seq * 4 + 15) & ~(size_t)15;
  hipLaunchKernelGGL(cache4_last_kernel<D>, dim3(heads + 1, (unsigned)(most < fill ? most : fill)), dim3(kLastThreads), lds, st, a);
  return check_launch();
}

int launch_cache4_evict(const CacheEvictArgs& a, hipStream_t st) { return a.c.d == 128 ? launch_evict_d<128>(a, st) : launch_evict_d<64>(a, st); }

}  // namespace ha
