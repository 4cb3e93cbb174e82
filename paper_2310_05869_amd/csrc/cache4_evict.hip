// Eviction from the 4-bit cache by accumulated attention weight (ha_cache4_evict): a sequence longer than its budget keeps its last tokens and, for every key
// head, those of most weight among the others.
//
// Of n tokens k stay, r of them the last ones; the other k - r are the largest of n - r.  Kept tokens among the first k - r places stay where they are, the others move
// into the places that come free there, first to first: in a steady state a step moves as many rows as it lets go, where closing up would move nearly all.
// Then the last r follow, in order.
//   select   a workgroup per sequence and key head finds the (k - r)-th largest weight by histograms of 11, 11 and 10 bits of the weights' bits, made so that they
//            order as numbers do (as soon as no more than 256 are left to choose from, their ranks are counted instead), then who moves where from prefix sums: with c(p)
//            tokens kept before place p, a free place p is the (p - c(p))-th, a kept token the (c(p) - c(k - r))-th that moves.  A wave has a run of places of its own,
//            so that only 16 numbers cross the waves.
//   move     rows of these lists, D / 8 lanes a row
//   last     the last r rows, whose places may overlap: read, a barrier, written, some hundred at a time
// One launch, in which the workgroup that chose moves the rows too, where the sequences and key heads fill the chip or are short.  Else a second launch, so that the rows of few heads
// are moved by all of it: few last rows by the first workgroup of their head, after the rows that lie in their places; many in a third.  Lengths and free pages: a workgroup beside those that choose.
#include <type_traits>

#include "cache4_common.h"

namespace ha {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kBins = 2048;
constexpr int kMoveThreads = 256, kLastThreads = 1024;
// Sequences and key heads that fill the chip: a workgroup moves its own rows.  (Launches apart / one: 64 of them, 3800 rows each, 70 / 101 us; 8 key heads, 4096 of 8192 with 128 last ones, 31, 48 and
// 64 sequences 68 / 72, 121 / 131, 178 / 177; 4096 of 4160, 16, 28 and 64 sequences 15.4 / 12.3, 16.7 / 13.5, 24.4 / 20.7: which of both kinds it will be the host does not know.  Tables of up
// to 2048 tokens are one launch too: 4 heads, 900 of 1900 14.9 / 14.0 us, 400 of 900 15.0 / 12.3, but 1900 of 3900 15.3 / 23.8.)
constexpr int kManyHeads = 256;
// Last rows that move in the launch of the others (8 sequences that keep 4096 of 32768, in a launch of their own / in it: 128 last ones 52 / 47 us, 256 53.5 / 48.6, 512 56.6 / 55.4, 1024 55.3 / 68)
constexpr int kFewLast = 512;
constexpr int kAhead = 8;  // rows that a lane has in flight
constexpr int kSmall = 512;  // threads of a workgroup that chooses from up to 32 times as many places

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

// Sum of the lanes up to this one
__device__ inline uint32_t wave_scan(uint32_t x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, true);  // row_shr:1, 2, 4, 8
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, true);  // row_bcast:15 into rows 1 and 3
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, true);  // row_bcast:31 into rows 2 and 3
  return x;
}

// Sum of the values of the threads before (exclusive) and of all; one barrier before the scratch may be written again is the caller's
template <int NT>
__device__ inline uint32_t block_scan(uint32_t x, uint32_t* all, uint32_t* scratch) {
  const int wave = threadIdx.x >> 6;
  const uint32_t inc = wave_scan(x);
  if ((threadIdx.x & 63) == 63) scratch[wave] = inc;
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

constexpr int kRanked = 256;  // numbers whose ranks are counted
constexpr int kCopies = 4;
template <int NT>
struct SelectLds {
  uint32_t hist[kCopies][kBins];  // by lane, for the first pass: weights of like size queue for their counters less
  alignas(16) uint32_t left[kRanked];
  uint32_t n_left;
  uint32_t scratch[NT / 64];
  uint32_t gt[NT / 64], eq[NT / 64];  // kept for certain, and equal to the limit, of every wave's places
  uint32_t gaps, near;
  uint32_t bin, want, here;
};

// Writes the list of rows that change places and returns how many they are, and how many of them (the first) lie where the last rows go.  HELD: the weights are few enough to stay in registers, so many pieces of four a thread (0: they are not)
template <int NT, int HELD>
__device__ __forceinline__ int2 select_moves(const CacheEvictArgs& a, const EvictSeq& q, int s, int kv, SelectLds<NT>& lds) {
  constexpr int NW = NT / 64, PIECES = HELD > 0 ? HELD : 8;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int from = q.n - q.r, stay = q.k - q.r;  // places that are chosen from, and how many of them
  const int32_t* blocks = a.table + (int64_t)s * a.max_blocks;
  const int per = (from + NW * 256 - 1) / (NW * 256);  // pieces of 256 places a wave
  const int place0 = wave * per * 256 + lane * 4;
  // (Page numbers of all pieces first, then all weights, then what they are made into: with a piece after the other, each waits for two loads by itself.)
  auto page_at = [&](int i) { return blocks[min(place0 + i * 256, from - 1) >> a.c.log_page]; };
  auto weights_at = [&](int i, int page) {
    const int p = min(place0 + i * 256, (from - 1) & ~3);
    f32x4 x = {0.f, 0.f, 0.f, 0.f};
    if (a.c.n_pages > 0) x = *reinterpret_cast<const f32x4*>(a.weights + ((int64_t)((unsigned)page < (unsigned)a.c.n_pages ? page : 0) * a.c.Hk + kv) * a.c.page + (p & (a.c.page - 1)));
    return x;
  };
  auto key_of = [&](int i, int page, const f32x4& x) {
    const int p = place0 + i * 256;
    const bool there = (unsigned)page < (unsigned)a.c.n_pages;
    const u32x4 u = {__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3])};
    // (mostly, a wave has a whole piece of numbers that are not negative: vector issue binds here.  With this and the counting without ties below, 8 sequences that keep 4096 of
    // 32768 63.4 us instead of 67.5)
    if (!__any(i >= per || p + 3 >= from || !there || max(max(u[0], u[1]), max(u[2], u[3])) > 0x7f800000u)) return u | 0x80000000u;
    u32x4 key;
#pragma unroll
    for (int e = 0; e < 4; ++e) key[e] = i >= per || p + e >= from ? 0u : there ? order_of(x[e]) : 1u;
    return key;
  };
  u32x4 held[PIECES];
  int held_page[PIECES];
  if constexpr (HELD > 0) {
#pragma unroll
    for (int i = 0; i < PIECES; ++i) held_page[i] = page_at(i);
    f32x4 x[PIECES];
#pragma unroll
    for (int i = 0; i < PIECES; ++i) x[i] = weights_at(i, held_page[i]);
#pragma unroll
    for (int i = 0; i < PIECES; ++i) held[i] = key_of(i, held_page[i], x[i]);
  }
  auto all_keys = [&](auto&& f) {  // f(piece, its keys, their page)
    if constexpr (HELD > 0) {
#pragma unroll
      for (int i = 0; i < PIECES; ++i)
        if (i < per) f(i, held[i], held_page[i]);
    } else {
      for (int i0 = 0; i0 < per; i0 += PIECES) {
        int page[PIECES];
        f32x4 x[PIECES];
#pragma unroll
        for (int i = 0; i < PIECES; ++i) page[i] = page_at(i0 + i);
#pragma unroll
        for (int i = 0; i < PIECES; ++i) x[i] = weights_at(i0 + i, page[i]);
#pragma unroll
        for (int i = 0; i < PIECES; ++i)
          if (i0 + i < per) f(i0 + i, key_of(i0 + i, page[i], x[i]), page[i]);
      }
    }
  };

  uint32_t prefix = 0, want = stay;
  for (int i = threadIdx.x; i < kCopies * kBins; i += NT) lds.hist[0][i] = 0;
  if (threadIdx.x < kRanked) lds.left[threadIdx.x] = 0;
  if (threadIdx.x == 0) lds.n_left = lds.gaps = lds.near = 0;
  __syncthreads();
#pragma unroll
  for (int pass = 0; pass < 3; ++pass) {
    const int bits = pass == 2 ? 10 : 11, shift = pass == 0 ? 21 : pass == 1 ? 10 : 0;
    uint32_t* const hist = pass == 0 ? lds.hist[lane % kCopies] : lds.hist[0];
    if (pass > 0) {
      for (int i = threadIdx.x; i < kBins; i += NT) hist[i] = 0;
      __syncthreads();
    }
    all_keys([&](int, const u32x4& key, int) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const bool in = key[e] != 0 && (pass == 0 || key[e] >> (shift + bits) == prefix);
        const uint32_t bin = (key[e] >> shift) & ((1u << bits) - 1);
        const unsigned long long some = __ballot(in);
        if (some == 0) continue;
        // (weights that are all alike, zeros say, would queue for one counter)
        const uint32_t one = __builtin_amdgcn_readlane(bin, __builtin_ctzll(some));
        if (__ballot(in && bin != one) == 0) {
          if (lane == 0) atomicAdd(&hist[one], (uint32_t)__popcll(some));
        } else if (in) {
          atomicAdd(&hist[bin], 1u);
        }
      }
    });
    __syncthreads();
    constexpr int EACH = kBins / NT;
    uint32_t mine = 0, total;
    auto in_bin = [&](int bin) {
      uint32_t n = lds.hist[0][bin];
      if (pass == 0)
#pragma unroll
        for (int c = 1; c < kCopies; ++c) n += lds.hist[c][bin];
      return n;
    };
#pragma unroll
    for (int j = 0; j < EACH; ++j) mine += in_bin(kBins - 1 - (threadIdx.x * EACH + j));  // from the largest down
    uint32_t above = block_scan<NT>(mine, &total, lds.scratch);
    if (above < want && want <= above + mine) {
      for (int j = 0; j < EACH; ++j) {
        const int bin = kBins - 1 - (threadIdx.x * EACH + j);
        const uint32_t here = in_bin(bin);
        if (want <= above + here) {
          lds.bin = bin;
          lds.want = want - above;
          lds.here = here;
          break;
        }
        above += here;
      }
    }
    __syncthreads();
    prefix = prefix << bits | lds.bin;
    want = lds.want;
    if (pass < 2 && lds.here <= kRanked) {
      const int m = lds.here;
      all_keys([&](int, const u32x4& key, int) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (key[e] != 0 && key[e] >> shift == prefix) {
            const uint32_t at = atomicAdd(&lds.n_left, 1u);
            if (at < kRanked) lds.left[at] = key[e];
          }
      });
      __syncthreads();
      if ((int)threadIdx.x < m) {
        const uint32_t my = lds.left[threadIdx.x];
        uint32_t more = 0, same = 0;
#pragma unroll 4
        for (int i = 0; i < m; i += 4) {  // (zeros behind the last count for nothing)
          const u32x4 x = *reinterpret_cast<const u32x4*>(&lds.left[i]);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            more += x[e] > my;
            same += x[e] == my;
          }
        }
        if (more < want && want <= more + same) {  // (all that are equal to it write the same)
          lds.bin = my;
          lds.want = want - more;
          lds.here = same;
        }
      }
      __syncthreads();
      prefix = lds.bin;
      want = lds.want;
      break;
    }
  }

  // prefix: the last one that is kept; of those equal to it, the first `want`.  Whether these are all of them decides for most calls how much there is to count.
  const bool ties = want < lds.here;
  uint32_t gt = 0, eq = 0;
  if (ties) {
    all_keys([&](int, const u32x4& key, int) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        gt += key[e] > prefix;
        eq += key[e] == prefix;
      }
    });
  } else {
    all_keys([&](int, const u32x4& key, int) {
#pragma unroll
      for (int e = 0; e < 4; ++e) gt += key[e] >= prefix;
    });
  }
  gt = wave_scan(gt);
  eq = wave_scan(eq);
  if (lane == 63) {
    lds.gt[wave] = gt;
    lds.eq[wave] = eq;
  }
  __syncthreads();
  uint32_t gt_before = 0, eq_before = 0;
  for (int w = 0; w < wave; ++w) {
    gt_before += lds.gt[w];
    eq_before += lds.eq[w];
  }
  // (Weights that change from pass to pass, of pages that sequences share against the rule, may give any order, but no place outside the list.)
  int32_t* moves = reinterpret_cast<int32_t*>(a.moves + ((int64_t)s * a.c.Hk + kv) * a.moves_most);
  const uint32_t most = (uint32_t)a.moves_most;
  int gaps = 0, near = 0;
  // (how many stay is not known yet, so rows that move are counted from the last one)
  auto list = [&](bool kept, uint32_t rank, int p, int slot) {
    const bool behind = p >= stay;
    const uint32_t at = behind ? stay - 1 - rank : p - rank;
    if (kept == behind && at < most) moves[2 * (int64_t)at + !behind] = slot;
    gaps += __popcll(__ballot(!kept && !behind));
    near += __popcll(__ballot(kept && behind && p < q.k));
  };
  auto slot_at = [&](int page, int p) { return (unsigned)page < (unsigned)a.c.n_pages ? (page << a.c.log_page) + (p & (a.c.page - 1)) : -4; };
  if (ties) {
    all_keys([&](int i, const u32x4& key, int page) {
      uint32_t here = 0;  // kept for certain in the upper half, equal in the lower
#pragma unroll
      for (int e = 0; e < 4; ++e) here += key[e] > prefix ? 0x10000u : key[e] == prefix ? 1u : 0u;
      const uint32_t inc = wave_scan(here);
      uint32_t g = gt_before + ((inc - here) >> 16), t = eq_before + ((inc - here) & 0xffffu);
      const uint32_t both = __builtin_amdgcn_readlane(inc, 63);
      gt_before += both >> 16;
      eq_before += both & 0xffffu;
      const int p = place0 + i * 256, slot = slot_at(page, p);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const bool more = key[e] > prefix, same = key[e] == prefix;
        list(more || (same && t < want), g + min(t, want), p + e, slot + e);
        g += more;
        t += same;
      }
    });
  } else {
    all_keys([&](int i, const u32x4& key, int page) {
      uint32_t here = 0;
#pragma unroll
      for (int e = 0; e < 4; ++e) here += key[e] >= prefix;
      const uint32_t inc = wave_scan(here);
      uint32_t g = gt_before + inc - here;
      gt_before += __builtin_amdgcn_readlane(inc, 63);
      const int p = place0 + i * 256, slot = slot_at(page, p);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const bool kept = key[e] >= prefix;
        list(kept, g, p + e, slot + e);
        g += kept;
      }
    });
  }
  if (lane == 0) {
    atomicAdd(&lds.gaps, (uint32_t)gaps);
    atomicAdd(&lds.near, (uint32_t)near);
  }
  __syncthreads();
  const uint32_t all = min(lds.gaps, most);
  return int2{(int)all, (int)min(lds.near, all)};
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

// Rows begin ... end - 1 of the list's `count`, by workgroup `part` of `parts`: places that come free from the first on, rows that move from the last
template <int D, int NT>
__device__ inline void move_rows(const CacheEvictArgs& a, int head, int count, int begin, int end, int part, int parts) {
  constexpr int LPR = D / 8, ROWS = NT / LPR, AHEAD = kAhead;
  const int kv = head % a.c.Hk, j = threadIdx.x % LPR;
  const int2* moves = a.moves + (int64_t)head * a.moves_most;
  const uint32_t slots = (uint32_t)a.c.n_pages << a.c.log_page;  // (an entry that no pass wrote, see above, may be anything)
  for (int i0 = begin + part * ROWS * AHEAD + threadIdx.x / LPR; i0 < end; i0 += parts * ROWS * AHEAD) {
    int2 m[AHEAD];
    RowPiece<D> x[AHEAD];
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      const int i = i0 + u * ROWS;
      m[u] = i < end ? int2{moves[count - 1 - i].x, moves[i].y} : int2{-1, -1};
    }
#pragma unroll
    for (int u = 0; u < AHEAD; ++u)
      if ((uint32_t)m[u].x < slots) x[u] = load_piece<D>(a, kv, m[u].x, j);
#pragma unroll
    for (int u = 0; u < AHEAD; ++u)
      if ((uint32_t)m[u].x < slots && (uint32_t)m[u].y < slots) store_piece<D>(a, kv, m[u].y, j, x[u]);
  }
}

// The last rows.  Those that lie apart from their places are shared among workgroups; else one takes them in order: what it writes lies before what is still to be read.
template <int D, int NT>
__device__ inline void move_last(const CacheEvictArgs& a, const EvictSeq& q, int s, int kv, int part, int parts) {
  constexpr int LPR = D / 8, ROWS = NT / LPR, AHEAD = kAhead;
  const int j = threadIdx.x % LPR;
  const int32_t* blocks = a.table + (int64_t)s * a.max_blocks;
  auto slot_of = [&](int p) {
    const int page = blocks[p >> a.c.log_page];
    return (unsigned)page < (unsigned)a.c.n_pages ? (page << a.c.log_page) + (p & (a.c.page - 1)) : -1;
  };
  const bool apart = q.n - q.k >= q.r;
  if (!apart && part > 0) return;
  for (int i0 = apart ? part * ROWS * AHEAD : 0; i0 < q.r; i0 += (apart ? parts : 1) * ROWS * AHEAD) {
    int at[AHEAD], to[AHEAD];
    RowPiece<D> x[AHEAD];
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      const int i = i0 + u * ROWS + threadIdx.x / LPR;
      at[u] = i < q.r ? slot_of(q.n - q.r + i) : -1;
      to[u] = i < q.r ? slot_of(q.k - q.r + i) : -1;
    }
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      x[u] = RowPiece<D>{0, 0, 0};
      if (at[u] >= 0) x[u] = load_piece<D>(a, kv, at[u], j);
    }
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) asm volatile("" : "+v"(x[u].k), "+v"(x[u].v), "+v"(x[u].more));  // (all of them are here before the barrier)
    __syncthreads();
#pragma unroll
    for (int u = 0; u < AHEAD; ++u)
      if (at[u] >= 0 && to[u] >= 0) store_piece<D>(a, kv, to[u], j, x[u]);
  }
}

// Lengths, and the pages that come free, on top of the stack in order.  upto: n_seq words.  (The histograms', which this workgroup has no other use for: with room of its own behind
// them in every workgroup's LDS, 8192 sequences of up to 40 tokens, two key heads, 257 -> 250 us, of up to 500, eight, 1439 -> 1420.)
template <int NT>
__device__ inline void free_pages(const CacheEvictArgs& a, uint32_t* upto, uint32_t* scratch) {
  auto pages_of = [&](int tokens) { return (int)(((int64_t)tokens + a.c.page - 1) >> a.c.log_page); };
  const int count = min(max(*a.free_count, 0), a.c.n_pages);
  const int each = (a.n_seq + NT - 1) / NT, s0 = min(a.n_seq, (int)threadIdx.x * each), s1 = min(a.n_seq, s0 + each);
  uint32_t mine = 0, all;
  for (int s = s0; s < s1; ++s) {
    const EvictSeq q = evict_seq(a, s);
    a.lens_out[s] = q.k;
    upto[s] = mine;
    mine += pages_of(q.n) - pages_of(q.k);
  }
  const uint32_t before = block_scan<NT>(mine, &all, scratch);
  for (int s = s0; s < s1; ++s) upto[s] += before;
  __syncthreads();
  if (threadIdx.x == 0) *a.free_count_out = (int)min((int64_t)count + all, (int64_t)a.c.n_pages);
  for (int s = threadIdx.x >> 6; s < a.n_seq; s += NT / 64) {
    const EvictSeq q = evict_seq(a, s);
    const int left = pages_of(q.k), freed = pages_of(q.n) - left;
    for (int i = threadIdx.x & 63; i < freed; i += 64) {
      const int64_t at = (int64_t)count + upto[s] + i;
      if (at < a.c.n_pages) a.free_pages[at] = a.table[(int64_t)s * a.max_blocks + left + i];
    }
  }
}

// The first workgroup has lengths and pages, each of the others a sequence and key head.  ALL: it moves the rows too.
template <int D, int NT, bool ALL>
__global__ __launch_bounds__(NT) void cache4_select_kernel(CacheEvictArgs a) {
  __shared__ SelectLds<NT> lds;
  if (blockIdx.x == 0) {
    static_assert(kCopies * kBins >= kEvictSeqs);
    free_pages<NT>(a, &lds.hist[0][0], lds.scratch);
    return;
  }
  const int head = blockIdx.x - 1, s = head / a.c.Hk, kv = head - s * a.c.Hk;
  const EvictSeq q = evict_seq(a, s);
  int2 count = {0, 0};
  if (q.k < q.n && q.r < q.k) {  // (two pieces instead of eight: 3 sequences of up to 500 8.6 us, not 9.2; 64 that keep 4096 of 4160 23.1, not 23.8)
    const int from = q.n - q.r;
    count = from <= NT * 8 ? select_moves<NT, 2>(a, q, s, kv, lds) : from <= NT * 32 ? select_moves<NT, 8>(a, q, s, kv, lds) : select_moves<NT, 0>(a, q, s, kv, lds);
  }
  if constexpr (ALL) {
    if (q.k == q.n) return;
    __syncthreads();  // (the list is written, by all waves)
    move_rows<D, NT>(a, head, count.x, 0, count.x, 0, 1);
    __syncthreads();  // (rows have been read that the last ones are written over)
    move_last<D, NT>(a, q, s, kv, 0, 1);
  } else {
    if (threadIdx.x == 0) a.counts[head] = count;
  }
}

// LAST: the first workgroup of a sequence and key head takes its last rows, after those that lie in their places
template <int D, bool LAST>
__global__ __launch_bounds__(kMoveThreads) void cache4_move_kernel(CacheEvictArgs a) {
  const int head = blockIdx.x;
  const int2 count = a.counts[head];
  if constexpr (LAST) {
    if (blockIdx.y > 0) {
      move_rows<D, kMoveThreads>(a, head, count.x, count.y, count.x, blockIdx.y - 1, gridDim.y - 1);
      return;
    }
    const int s = head / a.c.Hk, kv = head - s * a.c.Hk;
    const EvictSeq q = evict_seq(a, s);
    if (q.k == q.n) return;
    move_rows<D, kMoveThreads>(a, head, count.x, 0, count.y, 0, 1);
    __syncthreads();  // (these have been read)
    move_last<D, kMoveThreads>(a, q, s, kv, 0, 1);
  } else {
    move_rows<D, kMoveThreads>(a, head, count.x, 0, count.x, blockIdx.y, gridDim.y);
  }
}

template <int D>
__global__ __launch_bounds__(kLastThreads) void cache4_last_kernel(CacheEvictArgs a) {
  const int s = blockIdx.x / a.c.Hk, kv = blockIdx.x - s * a.c.Hk;
  const EvictSeq q = evict_seq(a, s);
  if (q.k < q.n) move_last<D, kLastThreads>(a, q, s, kv, blockIdx.y, gridDim.y);
}

template <int D, int NT, bool ALL>
static int launch_select(const CacheEvictArgs& a, hipStream_t st) {
  hipLaunchKernelGGL((cache4_select_kernel<D, NT, ALL>), dim3((unsigned)(a.n_seq * a.c.Hk + 1)), dim3(NT), 0, st, a);
  return check_launch();
}

template <int D>
static int launch_evict_d(const CacheEvictArgs& a, hipStream_t st) {
  const int64_t tokens = (int64_t)a.max_blocks << a.c.log_page;
  const int heads = a.n_seq * a.c.Hk;
  if (tokens <= 2048 || heads >= kManyHeads || heads == 0) return tokens <= kSmall * 32 ? launch_select<D, kSmall, true>(a, st) : launch_select<D, 1024, true>(a, st);
  int rc = tokens <= kSmall * 32 ? launch_select<D, kSmall, false>(a, st) : launch_select<D, 1024, false>(a, st);
  if (rc != HA_OK) return rc;
  constexpr int64_t per = kAhead * kMoveThreads / (D / 8), per_last = kAhead * kLastThreads / (D / 8);
  const int64_t most = (a.moves_most + per - 1) / per, fill = 2048 / heads + 1;
  const unsigned parts = (unsigned)(most < fill ? most : fill);
  if (a.recent > 0 && a.recent <= kFewLast) {
    hipLaunchKernelGGL((cache4_move_kernel<D, true>), dim3(heads, 1 + parts), dim3(kMoveThreads), 0, st, a);
    return check_launch();
  }
  hipLaunchKernelGGL((cache4_move_kernel<D, false>), dim3(heads, parts), dim3(kMoveThreads), 0, st, a);
  rc = check_launch();
  if (rc != HA_OK || a.recent == 0) return rc;
  const int64_t most_last = ((int64_t)a.recent + per_last - 1) / per_last, fill_last = 512 / heads + 1;
  hipLaunchKernelGGL(cache4_last_kernel<D>, dim3(heads, (unsigned)(most_last < fill_last ? most_last : fill_last)), dim3(kLastThreads), 0, st, a);
  return check_launch();
}

int launch_cache4_evict(const CacheEvictArgs& a, hipStream_t st) { return a.c.d == 128 ? launch_evict_d<128>(a, st) : launch_evict_d<64>(a, st); }

}  // namespace ha
