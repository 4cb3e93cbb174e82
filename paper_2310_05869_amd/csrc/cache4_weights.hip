// What attention weight the tokens of the 4-bit cache got from new queries (ha_cache4_weights): w[t] += sum over the rows that see token t, and the query heads of
// its key head, of exp(<q, k_t> - lse).
//
// A second pass over K alone, after attention has found lse: nothing is rounded, and no sum depends on the order of workgroups, which sums added up beside P V by
// all workgroups of a head would.  A wave keeps the K of 64 tokens as operands in registers, made from codes once, and rows of Q pass by, 64 a
// step, in LDS for the four waves of a workgroup: S^T = K Q^T by v_mfma_f32_32x32x16_bf16, 16 registers of 16 tokens for one row a lane, so a
// row's lse is one register, and the sums stay apart by lane until the last step, when 31 exchanges add up 32 registers over 32 lanes.
// Per 64 tokens and 32 rows of d = 128: 16 products (512 cycles) and 32 times a multiply-add, an exponential and an addition (some 450).
//
// Split: tiles of 256 tokens of all sequences and key heads are one line, a tile's length in it the steps of rows that see it; cut into equal runs like the
// tiles of attention.  Sums of tiles that a cut divides are added up, in order, by a second launch.
#include "cache4_chunk.h"

namespace ha {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kWWaves = 4;
constexpr int kWTokens = kWeightsTokens;
static_assert(kWTokens == 64 * kWWaves);
constexpr int kWRows = 64;              // of a step
constexpr int kWTileCost = 2;           // what a tile's start and end cost, in steps

template <int D, int SPLIT>
struct WeightsLds {
  static constexpr int STR = (D + 8) * 2;  // bytes per row (+16: conflict-free 16-byte row reads)
  static constexpr int PART = kWRows * STR;
  static constexpr int BUF = SPLIT * PART + kWRows * 4;  // rows in parts, and what their exponents start from
};

// A tile's place in the line.  Tile k of a sequence holds tokens 256 k ... + 255; rows are its new tokens' query heads, in steps of 64 from row 0.  The first
// token that sees the tile is max(0, 256 k - held), and 256 group is a multiple of 64, so that the steps of a tile fall linearly from the first that lies in the new tokens on.
struct WeightsSeq {
  ChunkSeq q;
  int tiles, bend;        // tiles, and the first of them that some rows do not see
  int64_t steps, before;  // steps of all rows; of a tile k >= bend the first `before` + 4 group k are left out
};
__device__ inline WeightsSeq weights_seq(const CacheChunkArgs& a, int s) {
  WeightsSeq w;
  w.q = chunk_seq(a, s);
  w.tiles = (w.q.len + kWTokens - 1) / kWTokens;
  w.bend = w.q.held <= 0 ? 0 : min((w.q.held + kWTokens - 1) / kWTokens, w.tiles);
  w.steps = ((int64_t)w.q.n * a.group + kWRows - 1) / kWRows;
  w.before = (-(int64_t)w.q.held * a.group) >> 6;  // (rounded down)
  return w;
}
__device__ inline int64_t weights_first_step(const CacheChunkArgs& a, const WeightsSeq& w, int k) {
  return k < w.bend ? 0 : min(w.before + 4ll * a.group * k, w.steps);
}
__device__ inline int64_t weights_upto(const CacheChunkArgs& a, const WeightsSeq& w, int64_t k) {
  int64_t x = k * (w.steps + kWTileCost);
  if (k > w.bend) x -= (k - w.bend) * w.before + 4ll * a.group * ((k * (k - 1) - (int64_t)w.bend * (w.bend - 1)) / 2);
  return x;
}

// Adds 32 registers over the 32 lanes of a half wave: lane l is left with the sum of register l.
__device__ inline float sum_of_lane(float (&x)[32], int lane) {
#pragma unroll
  for (int half = 16; half >= 1; half >>= 1) {
    const bool upper = lane & half;
#pragma unroll
    for (int i = 0; i < half; ++i) {
      const float give = upper ? x[i] : x[i + half], keep = upper ? x[i + half] : x[i];
      x[i] = keep + __shfl_xor(give, half);
    }
  }
  return x[0];
}

__device__ inline float scale_of(uint32_t bytes, int i) { return __uint_as_float(i < 3 ? bytes << (23 - 8 * i) : bytes >> 1); }  // (the exponent alone counts)

// SPLIT: parts of a query number, 1 for bf16, 3 for fp32.  CUT: tiles may be shared among workgroups.
template <int D, int SPLIT, bool CUT>
__global__ __launch_bounds__(64 * kWWaves, 2) void cache4_weights_kernel(CacheChunkArgs a) {
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  using L = WeightsLds<D, SPLIT>;
  constexpr int KS = D / 16, G = D / kCacheGroup;
  constexpr bool F32 = SPLIT > 1;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int lq = lane & 31, h = lane >> 5;

  auto cost = [&](int s) -> int64_t {
    const WeightsSeq w = weights_seq(a, s);
    return a.c.Hk * weights_upto(a, w, w.tiles);
  };
  int64_t before;
  const int64_t total = chunk_line(a.n_seq, lane, &before, cost);
  int parts = (int)min((int64_t)a.parts, max(total / a.least_run, (int64_t)1));
  if (parts > 8) parts &= ~7;
  int part = blockIdx.x;
  if (part < parts && (parts & 7) == 0) part = (part & 7) * (parts >> 3) + (part >> 3);  // a run of the line per XCD: neighbours share rows
  if (CUT && threadIdx.x == 0) a.joins[4 * part] = -1;
  if (part >= parts || total == 0) return;
  auto part_begin = [&](int p) { return total / parts * p + total % parts * p / parts; };
  const int64_t u0 = part_begin(part), u1 = part_begin(part + 1);
  int64_t tile_first;
  int s = chunk_place(a.n_seq, before, u0, &tile_first, cost);
  WeightsSeq w = weights_seq(a, s);
  w.q = uniform_seq(w.q);
  int kv, k;
  {
    const int64_t head_cost = weights_upto(a, w, w.tiles), rem = u0 - tile_first;
    kv = __builtin_amdgcn_readfirstlane((int)(rem / head_cost));
    const int64_t in_head = rem - kv * head_cost;
    int lo = 0, hi = w.tiles;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (weights_upto(a, w, mid) <= in_head) lo = mid;
      else hi = mid;
    }
    k = __builtin_amdgcn_readfirstlane(lo);
    tile_first = uniform64(tile_first + kv * head_cost + weights_upto(a, w, k));
  }

  const int64_t page_bytes = (int64_t)a.c.Hk * a.c.block_bytes();
  for (;;) {
    const int64_t step0 = uniform64(weights_first_step(a, w, k)), length = uniform64(w.steps) - step0 + kWTileCost;
    const int nsteps = (int)(length - kWTileCost);
    auto step_at = [&](int64_t x) { return (int)min(max(x, (int64_t)0), (int64_t)nsteps); };
    const bool begins = tile_first >= u0;
    // without CUT a tile is that workgroup's in whose run it begins
    const int first = CUT ? step_at(u0 - tile_first) : 0, last = CUT ? step_at(u1 - tile_first) : begins ? nsteps : 0;
    if (first < last || (begins && nsteps == 0 && a.fresh)) {
      const int32_t* blocks = a.table + (int64_t)s * a.max_blocks;
      // ---- K of the wave's 64 tokens ----
      bf16x8 kf[2][KS];
#pragma unroll
      for (int sub = 0; sub < 2; ++sub) {
        const int tok = k * kWTokens + wave * 64 + 32 * sub + lq;
        const int page = blocks[min(tok, w.q.len - 1) >> a.c.log_page], at = tok & (a.c.page - 1);
        const unsigned char* b = a.cache + (int64_t)((unsigned)page < (unsigned)a.c.n_pages ? page : 0) * page_bytes + (int64_t)kv * a.c.block_bytes();
        uint32_t words[KS], sc;  // words KS h ... of the token
#pragma unroll
        for (int i = 0; i < KS; i += 4) {
          const u32x4 x = *reinterpret_cast<const u32x4*>(b + at * (D / 2) + 4 * (KS * h + i));
#pragma unroll
          for (int e = 0; e < 4; ++e) words[i + e] = x[e];
        }
        if constexpr (D == 128) sc = *reinterpret_cast<const uint32_t*>(b + a.c.k_scale_at() + at * 4);
        else sc = *reinterpret_cast<const uint16_t*>(b + a.c.k_scale_at() + at * 2);
#pragma unroll
        for (int i = 0; i < KS; ++i) {
          const float f = scale_of(sc, i % G);
          const u32x4 x = {__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(words[i], f, 0)),
                           __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(words[i], f, 1)),
                           __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(words[i], f, 2)),
                           __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(words[i], f, 3))};
          kf[sub][i] = __builtin_bit_cast(bf16x8, x);
        }
      }
      float sum[32];
#pragma unroll
      for (int i = 0; i < 32; ++i) sum[i] = 0.f;

      // ---- rows of Q through LDS ----
      constexpr int CPR = D / 8, NC = kWRows * CPR / (64 * kWWaves);  // pieces of eight channels a row, a thread
      const int rows = w.q.n * a.group;
      u32x4 raw[NC][F32 ? 2 : 1];
      float raw_lse = 0.f;
      auto load_rows = [&](int step) {
        const int row0 = (int)(step0 + step) * kWRows;
#pragma unroll
        for (int i = 0; i < NC; ++i) {
          const int r = row0 + threadIdx.x / CPR + i * (64 * kWWaves / CPR), c = threadIdx.x % CPR * 8;
          const int use = min(r, rows - 1), tok = a.div_group.div(use), head = kv * a.group + use - tok * a.group;
          const int64_t at = (int64_t)(w.q.start + tok) * a.q.row + (int64_t)head * a.q.head + c;
          if constexpr (F32) {
            const u32x4* p = reinterpret_cast<const u32x4*>(reinterpret_cast<const float*>(a.Q) + at);
            raw[i][0] = p[0];
            raw[i][1] = p[1];
          } else {
            raw[i][0] = *reinterpret_cast<const u32x4*>(reinterpret_cast<const uint16_t*>(a.Q) + at);
          }
        }
        if (threadIdx.x < kWRows) {
          const int use = min(row0 + (int)threadIdx.x, rows - 1), tok = a.div_group.div(use), head = kv * a.group + use - tok * a.group;
          raw_lse = a.lse[(int64_t)head * a.rows + w.q.start + tok];
        }
      };
      auto store_rows = [&](int step) {
        unsigned char* buf = smem + (step & 1) * L::BUF;
#pragma unroll
        for (int i = 0; i < NC; ++i) {
          unsigned char* to = buf + (threadIdx.x / CPR + i * (64 * kWWaves / CPR)) * L::STR + threadIdx.x % CPR * 16;
          if constexpr (F32) {
            uint32_t part[3][4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              float x0 = 0.5f * __uint_as_float(raw[i][e / 2][2 * (e % 2)]), x1 = 0.5f * __uint_as_float(raw[i][e / 2][2 * (e % 2) + 1]);
#pragma unroll
              for (int z = 0; z < 3; ++z) {  // (at half: rounding the first part up leaves the largest finite)
                part[z][e] = pack_bf16x2(x0, x1);
                x0 -= __uint_as_float(part[z][e] << 16);
                x1 -= __uint_as_float(part[z][e] & 0xffff0000u);
              }
            }
#pragma unroll
            for (int z = 0; z < 3; ++z) *reinterpret_cast<u32x4*>(to + z * L::PART) = (u32x4){part[z][0], part[z][1], part[z][2], part[z][3]};
          } else {
            *reinterpret_cast<u32x4*>(to) = raw[i][0];
          }
        }
        // a row that sees nothing has lse -inf, and gives nothing
        if (threadIdx.x < kWRows)
          reinterpret_cast<float*>(buf + SPLIT * L::PART)[threadIdx.x] = raw_lse == -INFINITY ? -INFINITY : F32 ? -raw_lse : -raw_lse * kLog2e;
      };

      if (first < last) {
        load_rows(first);
        __syncthreads();  // (the tile before has left LDS)
        store_rows(first);
        __syncthreads();
      }
      const int tok_end = k * kWTokens + wave * 64 + 64;
      for (int step = first; step < last; ++step) {
        if (step + 1 < last) load_rows(step + 1);
        const unsigned char* buf = smem + (step & 1) * L::BUF;
        const int row0 = (int)(step0 + step) * kWRows;
        // whether the step's rows are all there and all see the wave's tokens
        const bool plain = row0 + kWRows <= rows && w.q.held + a.div_group.div(row0) + 1 >= tok_end;
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          const float shift = reinterpret_cast<const float*>(buf + SPLIT * L::PART)[32 * half + lq];
          f32x16 c[2];
#pragma unroll
          for (int i = 0; i < 16; ++i) c[0][i] = c[1][i] = 0.f;
#pragma unroll
          for (int i = 0; i < KS; ++i) {
            const int j = KS * h + i, ch = 32 * (j % G) + 8 * (j / G);  // the channels of word j
#pragma unroll
            for (int z = SPLIT - 1; z >= 0; --z) {
              const bf16x8 qf = *reinterpret_cast<const bf16x8*>(buf + z * L::PART + (32 * half + lq) * L::STR + ch * 2);
              c[0] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[0][i], qf, c[0], 0, 0, 0);
              c[1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[1][i], qf, c[1], 0, 0, 0);
            }
          }
          auto weight = [&](float x) { return F32 ? exp_split(__builtin_fmaf(x, 2.f, shift)) : __builtin_amdgcn_exp2f(__builtin_fmaf(x, kLog2e, shift)); };
          if (plain) {
#pragma unroll
            for (int i = 0; i < 32; ++i) sum[i] += weight(c[i / 16][i % 16]);
          } else {
            const int r = row0 + 32 * half + lq;
            const int see = r < rows ? w.q.held + a.div_group.div(r) + 1 - (k * kWTokens + wave * 64 + 4 * h) : 0;  // of the wave's tokens
#pragma unroll
            for (int i = 0; i < 32; ++i) {
              const float x = weight(c[i / 16][i % 16]);
              sum[i] += 32 * (i / 16) + 8 * (i % 16 / 4) + i % 4 < see && shift != -INFINITY ? x : 0.f;
            }
          }
        }
        if (step + 1 < last) store_rows(step + 1);
        __syncthreads();
      }

      const float mine = sum_of_lane(sum, lq);
      const int in_tile = wave * 64 + 32 * (lq / 16) + 8 * (lq % 16 / 4) + 4 * h + lq % 4, tok = k * kWTokens + in_tile;
      if (!CUT || (first == 0 && last == nsteps)) {
        if (tok < w.q.len) {
          const int page = blocks[tok >> a.c.log_page];
          if ((unsigned)page < (unsigned)a.c.n_pages) {
            float* to = a.weights + ((int64_t)page * a.c.Hk + kv) * a.c.page + (tok & (a.c.page - 1));
            *to = a.fresh || tok >= w.q.held ? mine : *to + mine;
          }
        }
      } else {
        a.part_o[(2 * (int64_t)part + begins) * kWTokens + in_tile] = mine;
        if (last == nsteps && threadIdx.x == 0) {  // others began the tile: the second launch adds up
          int p = (int)min(tile_first / (total / parts), (int64_t)part - 1);
          while (part_begin(p) > tile_first) --p;
          while (part_begin(p + 1) <= tile_first) ++p;
          a.joins[4 * part + 1] = kv;
          a.joins[4 * part + 2] = k;
          a.joins[4 * part + 3] = p;
          a.joins[4 * part] = s;
        }
      }
    }
    tile_first += length;
    if (tile_first >= u1) return;
    if (++k == w.tiles) {
      k = 0;
      if (++kv == a.c.Hk) {
        kv = 0;
        do {
          if (++s >= a.n_seq) return;
          w = weights_seq(a, s);
          w.q = uniform_seq(w.q);
        } while (w.tiles == 0);
      }
    }
  }
}

// Adds up the sums of tiles that a cut divides: workgroup p those of the tile that run p ended, a thread a token.
__global__ __launch_bounds__(kWTokens) void cache4_weights_join_kernel(CacheChunkArgs a) {
  const int p1 = blockIdx.x, s = a.joins[4 * p1];
  if (s < 0) return;
  const int kv = a.joins[4 * p1 + 1], k = a.joins[4 * p1 + 2], p0 = a.joins[4 * p1 + 3];
  const ChunkSeq q = chunk_seq(a, s);
  const int tok = k * kWTokens + threadIdx.x;
  if (tok >= q.len) return;
  const int page = a.table[(int64_t)s * a.max_blocks + (tok >> a.c.log_page)];
  float sum = 0.f;
#pragma unroll 4
  for (int p = p0; p <= p1; ++p) sum += a.part_o[(2 * (int64_t)p + (p == p0)) * kWTokens + threadIdx.x];
  if ((unsigned)page >= (unsigned)a.c.n_pages) return;
  float* to = a.weights + ((int64_t)page * a.c.Hk + kv) * a.c.page + (tok & (a.c.page - 1));
  *to = a.fresh || tok >= q.held ? sum : *to + sum;
}

// Tiles are shared among workgroups where a sequence can have many rows.
void cache4_weights_split(CacheChunkArgs* a) {
  a->div_group = make_fast_div(a->group);
  const int64_t tokens = (int64_t)a->max_blocks << a->c.log_page, steps = ((int64_t)a->rows * a->group + kWRows - 1) / kWRows;
  const int64_t tiles = ((tokens + kWTokens - 1) / kWTokens) * a->n_seq * a->c.Hk;
  a->cut = steps > 4;
  a->least_run = a->cut ? 8 : 1;
  const int64_t runs = tiles * (steps + kWTileCost) / a->least_run;
  a->parts = (int32_t)(runs < 1 ? 1 : runs > kWeightsParts ? kWeightsParts : runs);
}

template <int D, int SPLIT, bool CUT>
static int launch_weights_one(const CacheChunkArgs& a, hipStream_t st) {
  constexpr size_t lds = 2 * WeightsLds<D, SPLIT>::BUF;
  static std::atomic<uint64_t> set{0};
  const auto kernel = &cache4_weights_kernel<D, SPLIT, CUT>;
  const int rc = allow_full_lds(reinterpret_cast<const void*>(kernel), set);
  if (rc != HA_OK) return rc;
  hipLaunchKernelGGL(kernel, dim3((unsigned)a.parts), dim3(64 * kWWaves), lds, st, a);
  return check_launch();
}

template <int D, int SPLIT>
static int launch_weights_cut(const CacheChunkArgs& a, hipStream_t st) {
  if (!a.cut) return launch_weights_one<D, SPLIT, false>(a, st);
  const int rc = launch_weights_one<D, SPLIT, true>(a, st);
  if (rc != HA_OK) return rc;
  hipLaunchKernelGGL(cache4_weights_join_kernel, dim3((unsigned)a.parts), dim3(kWTokens), 0, st, a);
  return check_launch();
}

int launch_cache4_weights(const CacheChunkArgs& a, int dtype, hipStream_t st) {
  if (a.c.d == 128) return dtype == HA_BF16 ? launch_weights_cut<128, 1>(a, st) : launch_weights_cut<128, 3>(a, st);
  return dtype == HA_BF16 ? launch_weights_cut<64, 1>(a, st) : launch_weights_cut<64, 3>(a, st);
}

}  // namespace ha
