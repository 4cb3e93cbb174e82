// What attention weight the tokens of the 4-bit cache got from new queries (ha_cache4_weights): w[t] += sum over the rows that see token t, and the query heads of
// its key head, of exp(<q, k_t> - lse).
//
// A second pass over K alone, after attention has found lse: nothing is rounded below fp32 (-lse log2 e once, up front, so that a weight's exponent is one multiply-add: 1.7e-7
// from 64 bits where 6e-8 is the plain form's), and no sum depends on the order of workgroups, which sums added up beside P V by
// all workgroups of a head would.  S = Q K^T has rows of Q along the matrix instructions' M, tokens along N: a lane's registers are rows of one token, whose sum
// takes additions alone and one or two exchanges at the end.
//   many rows   a wave keeps the K of 64 tokens as operands in registers, made from codes once, and rows of Q pass by, 64 a step, in LDS for the four waves of a
//               workgroup (v_mfma_f32_32x32x16_bf16).  Per 64 tokens and 32 rows of d = 128: 16 products (512 cycles) beside 32 times a multiply-add, an exponential
//               and an addition (some 450): the exponentials of one half of a step run beside the products of the other.
//   few rows    a wave keeps 16 rows (a decoding step's queries of a key head), and tokens pass by, 64 at a time, from codes to operands in registers
//               (v_mfma_f32_16x16x32_bf16): bound by K's bytes, which every wave asks for a step ahead.
// Split: all sequences and key heads are one line.  Many rows: tiles of 256 tokens, a tile's length the steps of rows that see it; cut into equal runs like the tiles of
// attention, and sums of tiles that a cut divides are added up, in order, by a second launch.  Few rows: 64 tokens after the other, a run for every wave.
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
// What a tile's start and end cost, in steps.  (1 / 2 / 3 / 4: 2048 queries behind 16384, 32 and 8 heads, d = 128 347 / 343 / 338 / 334 us, fp32 1050 / 1050 / 1040 / 1029, 16 and 4 heads of d = 64,
// fp32, 298 / 291 / 286 / 278; 64 mixed, most of one token, 280 / 286 / 288 / 290; 24 of up to 200 behind up to 4096 48 / 52 / 51 / 52.)
constexpr int kWTileCost = 4;
// Steps that a workgroup takes, at least.  (8 / 4 / 2: 600 queries behind 3000, 8 and 2 heads, 34 / 23 / 20 us; 200 behind 700, d = 64, 20 / 16 / 13; fp32, six of 200 46 / 34 / 28.)
constexpr int kWLeastRun = 2;

template <int D, int SPLIT>
struct WeightsLds {
  static constexpr int STR = (D + 8) * 2;  // bytes per row (+16: conflict-free 16-byte row reads)
  static constexpr int PART = kWRows * STR;
  static constexpr int LEFT_OUT = SPLIT * PART + kWRows * 4;
  static constexpr int BUF = LEFT_OUT + 16;  // rows in parts, what their exponents start from, and of either half whether it has rows that give nothing
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
  w.tiles = (int64_t)w.q.n * a.group <= a.narrow ? 0 : (w.q.len + kWTokens - 1) / kWTokens;
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

// SPLIT: parts of a query number, 1 for bf16, 3 for fp32
template <int D, int SPLIT>
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
  const int64_t total = chunk_line(a, lane, &before, cost);
  int parts = (int)min((int64_t)a.parts, max(total / kWLeastRun, (int64_t)1));
  if (parts > 8) parts &= ~7;
  int part = blockIdx.x;
  if (part < parts && (parts & 7) == 0) part = (part & 7) * (parts >> 3) + (part >> 3);  // a run of the line per XCD: neighbours share rows
  if (threadIdx.x == 0) a.joins[4 * part] = -1;
  if (part >= parts || total == 0) return;
  const int64_t u0 = run_begin(total, parts, part), u1 = run_begin(total, parts, part + 1);
  int64_t tile_first;
  int s = chunk_place(a.n_seq, before, u0, &tile_first, cost);
  WeightsSeq w = weights_seq(a, s);
  w.q = uniform_seq(w.q);
  int kv, k;
  {
    const int64_t head_cost = weights_upto(a, w, w.tiles), rem = u0 - tile_first;
    kv = __builtin_amdgcn_readfirstlane(whole_part(rem, head_cost));
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
    const int first = step_at(u0 - tile_first), last = step_at(u1 - tile_first);
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
      float sum[2] = {0.f, 0.f};  // of the lane's token of each half, over the rows of its registers

      // ---- rows of Q through LDS ----
      constexpr int CPR = D / 8, NC = kWRows * CPR / (64 * kWWaves);  // pieces of eight channels a row, a thread
      const int rows = w.q.n * a.group;
      u32x4 raw[NC][F32 ? 2 : 1];
      float raw_lse = 0.f;
      // The thread's rows of a step lie 64 behind those of the step before: token and head go on by 64 / group and 64 % group.  (A division for every row and step took a
      // third of the vector instructions.)
      const int esz = F32 ? 4 : 2, on_tok = kWRows / a.group, on_head = kWRows - on_tok * a.group;
      struct Place {
        const unsigned char* at;
        int row, head;  // within the sequence and key head, within the group
      };
      Place from[NC], from_lse;
      auto begin = [&](Place& p, int row, const void* base, int64_t per_tok, int64_t per_head) {
        const int tok = a.div_group.div(row);
        p.row = row;
        p.head = row - tok * a.group;
        p.at = reinterpret_cast<const unsigned char*>(base) + (w.q.start + tok) * per_tok + (kv * a.group + p.head) * per_head;
      };
      auto go_on = [&](Place& p, int64_t per_tok, int64_t per_head) {
        p.row += kWRows;
        p.at += on_tok * per_tok + on_head * per_head;
        if (on_head != 0) {
          p.head += on_head;
          if (p.head >= a.group) {
            p.head -= a.group;
            p.at += per_tok - a.group * per_head;
          }
        }
      };
      const int64_t q_tok = a.q.row * esz, q_head = a.q.head * esz, l_tok = 4, l_head = 4 * (int64_t)a.rows;
      auto begin_rows = [&](int step) {
        const int row0 = (int)(step0 + step) * kWRows;
#pragma unroll
        for (int i = 0; i < NC; ++i) {
          begin(from[i], row0 + (int)threadIdx.x / CPR + i * (64 * kWWaves / CPR), a.Q, q_tok, q_head);
          from[i].at += threadIdx.x % CPR * 8 * esz;
          raw[i][0] = (u32x4){0, 0, 0, 0};
          raw[i][F32 ? 1 : 0] = (u32x4){0, 0, 0, 0};
        }
        begin(from_lse, row0 + (int)threadIdx.x % kWRows, a.lse, l_tok, l_head);
      };
      auto load_rows = [&]() {  // (of rows behind the last what was there before: they count for nothing)
#pragma unroll
        for (int i = 0; i < NC; ++i) {
          if (from[i].row < rows) {
            const u32x4* p = reinterpret_cast<const u32x4*>(from[i].at);
            raw[i][0] = p[0];
            if constexpr (F32) raw[i][1] = p[1];
          }
          go_on(from[i], q_tok, q_head);
        }
        if (threadIdx.x < kWRows) {
          if (from_lse.row < rows) raw_lse = *reinterpret_cast<const float*>(from_lse.at);
          go_on(from_lse, l_tok, l_head);
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
        // a row that sees nothing has lse -inf, and gives nothing, whatever it holds: a half with such a row takes its weights
        // one by one (2048 queries behind 16384: 343.6 -> 346.8 us; without, a NaN there went into every token that the row sees)
        if (threadIdx.x < kWRows) {
          const bool none = raw_lse == -INFINITY;
          const unsigned long long out = __ballot(none);
          reinterpret_cast<float*>(buf + SPLIT * L::PART)[threadIdx.x] = none ? -INFINITY : F32 ? -raw_lse : -raw_lse * kLog2e;
          if (threadIdx.x < 2) reinterpret_cast<uint32_t*>(buf + L::LEFT_OUT)[threadIdx.x] = (uint32_t)(out >> (32 * threadIdx.x));
        }
      };

      if (first < last) {
        begin_rows(first);
        load_rows();
        __syncthreads();  // (the tile before has left LDS)
        store_rows(first);
        if (first + 1 < last) load_rows();  // (rows are asked for a step before they are stored, two before they are used)
        __syncthreads();
      }
      const int tok0 = k * kWTokens + wave * 64, tok_end = tok0 + 64;
      struct Half {  // scores of 32 rows, what they are exponentiated against, and which of the rows give nothing
        f32x16 c[2];
        f32x4 shift[4];
        uint32_t out;
      };
      auto products = [&](int step, int half, Half& x) {
        const unsigned char* buf = smem + (step & 1) * L::BUF;
#pragma unroll
        for (int g = 0; g < 4; ++g) x.shift[g] = *reinterpret_cast<const f32x4*>(buf + SPLIT * L::PART + (32 * half + 8 * g + 4 * h) * 4);
        x.out = reinterpret_cast<const uint32_t*>(buf + L::LEFT_OUT)[half];
#pragma unroll
        for (int i = 0; i < 16; ++i) x.c[0][i] = x.c[1][i] = 0.f;
#pragma unroll
        for (int i = 0; i < KS; ++i) {
          const int ch = 32 * ((KS * h + i) % G) + 8 * ((KS * h + i) / G);  // the channels of word KS h + i
#pragma unroll
          for (int z = SPLIT - 1; z >= 0; --z) {
            const bf16x8 qf = *reinterpret_cast<const bf16x8*>(buf + z * L::PART + (32 * half + lq) * L::STR + ch * 2);
            x.c[0] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(qf, kf[0][i], x.c[0], 0, 0, 0);
            x.c[1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(qf, kf[1][i], x.c[1], 0, 0, 0);
          }
        }
      };
      auto weight = [&](float x, float shift) { return F32 ? exp_split(__builtin_fmaf(x, 2.f, shift)) : __builtin_amdgcn_exp2f(__builtin_fmaf(x, kLog2e, shift)); };
      auto add_weights = [&](const Half& x) {
#pragma unroll
        for (int sub = 0; sub < 2; ++sub) {
          float part[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int i = 0; i < 16; ++i) part[i % 4] += weight(x.c[sub][i], x.shift[i / 4][i % 4]);
          sum[sub] += (part[0] + part[1]) + (part[2] + part[3]);
        }
      };
      auto add_some_weights = [&](const Half& x, int row0) {  // rows behind the last, or that do not see all
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int r = row0 + 8 * (i / 4) + 4 * h + i % 4;
          const int see = r < rows ? w.q.held + a.div_group.div(r) + 1 - tok0 : 0;  // of the wave's tokens
          const float shift = x.shift[i / 4][i % 4];
#pragma unroll
          for (int sub = 0; sub < 2; ++sub) {
            const float p = weight(x.c[sub][i], shift);
            sum[sub] += 32 * sub + lq < see && shift != -INFINITY ? p : 0.f;
          }
        }
      };
      auto plain = [&](const Half& x, int row0) {  // whether 32 rows are all there, all give something and all see the wave's tokens
        return row0 + 32 <= rows && __builtin_amdgcn_readfirstlane(x.out) == 0 && w.q.held + a.div_group.div(row0) + 1 >= tok_end;
      };
      // Weights of one half beside products of the next: a slice of the vector work behind every two products, rows two products ahead.  (The order is held by hand: left to
      // itself, the compiler puts all products before all exponentials.)
      auto both = [&](const Half& x, int row0, int step, int half, Half& next) {
        if (!plain(x, row0)) {
          products(step, half, next);
          add_some_weights(x, row0);
          return;
        }
        const unsigned char* buf = smem + (step & 1) * L::BUF;
        const unsigned char* at = buf + (32 * half + lq) * L::STR;
        auto fragment = [&](int i, int z) {
          return *reinterpret_cast<const bf16x8*>(at + z * L::PART + (32 * ((KS * h + i) % G) + 8 * ((KS * h + i) / G)) * 2);
        };
        next.out = reinterpret_cast<const uint32_t*>(buf + L::LEFT_OUT)[half];
        bf16x8 qf[2][SPLIT];
        __builtin_amdgcn_s_setprio(1);  // (2048 queries behind 16384: 335.4 -> 331.6 us)
#pragma unroll
        for (int z = 0; z < SPLIT; ++z) qf[0][z] = fragment(0, z);
#pragma unroll
        for (int z = 0; z < SPLIT; ++z) qf[1][z] = fragment(1, z);
#pragma unroll
        for (int i = 0; i < 16; ++i) next.c[0][i] = next.c[1][i] = 0.f;
        float part[4] = {0.f, 0.f, 0.f, 0.f};  // even and odd rows of both tokens
#pragma unroll
        for (int i = 0; i < KS; ++i) {
          __builtin_amdgcn_sched_barrier(0);
#pragma unroll
          for (int z = SPLIT - 1; z >= 0; --z) {
            next.c[0] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(qf[i % 2][z], kf[0][i], next.c[0], 0, 0, 0);
            next.c[1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(qf[i % 2][z], kf[1][i], next.c[1], 0, 0, 0);
          }
          if (i + 2 < KS)
#pragma unroll
            for (int z = 0; z < SPLIT; ++z) qf[i % 2][z] = fragment(i + 2, z);
          if (i >= KS - 4) next.shift[i - KS + 4] = *reinterpret_cast<const f32x4*>(buf + SPLIT * L::PART + (32 * half + 8 * (i - KS + 4) + 4 * h) * 4);
#pragma unroll
          for (int e = i * 16 / KS; e < (i + 1) * 16 / KS; ++e) {
            part[e % 2] += weight(x.c[0][e], x.shift[e / 4][e % 4]);
            part[2 + e % 2] += weight(x.c[1][e], x.shift[e / 4][e % 4]);
          }
        }
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_setprio(0);
        sum[0] += part[0] + part[1];
        sum[1] += part[2] + part[3];
      };
      auto add = [&](const Half& x, int row0) {
        if (plain(x, row0)) add_weights(x);
        else add_some_weights(x, row0);
      };
      if (first < last) {
        Half xa, xb;
        products(first, 0, xa);
        int step = first;
        for (; step + 1 < last; ++step) {
          const int row0 = (int)(step0 + step) * kWRows;
          both(xa, row0, step, 1, xb);
          store_rows(step + 1);
          if (step + 2 < last) load_rows();
          __syncthreads();
          both(xb, row0 + 32, step + 1, 0, xa);
        }
        const int row0 = (int)(step0 + step) * kWRows;
        both(xa, row0, step, 1, xb);
        add(xb, row0 + 32);
      }
      __syncthreads();

      // a lane of the upper half takes the wave's tokens 32 ... 63
      const float give = h ? sum[0] : sum[1], keep = h ? sum[1] : sum[0], mine = keep + __shfl_xor(give, 32);
      const int in_tile = wave * 64 + lane, tok = k * kWTokens + in_tile;
      if (first == 0 && last == nsteps) {
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
          a.joins[4 * part + 1] = kv;
          a.joins[4 * part + 2] = k;
          a.joins[4 * part + 3] = run_of(total, parts, tile_first);
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

// ---- few rows ----
constexpr int kNUnit = 64;       // tokens of a wave's step
constexpr int kNStart = 3;       // what the start of a sequence and key head costs, in steps (0 / 3 / 8: 256 decoding behind up to 2048 16.2 / 16.3 / 18.0 us, 1000 of up to 512 21.4 / 21.8 / 23.5)
struct FewSeq {
  ChunkSeq q;
  int rows, tiles, units;  // query rows, tiles of 16 of them, steps of 64 tokens (0: not of these)
};
__device__ inline FewSeq few_seq(const CacheChunkArgs& a, int s) {
  FewSeq f;
  f.q = chunk_seq(a, s);
  f.rows = f.q.n * a.group;
  f.tiles = (f.rows + 15) / 16;
  f.units = f.rows > a.narrow || (f.rows == 0 && !a.fresh) ? 0 : (f.q.len + kNUnit - 1) / kNUnit;
  return f;
}

template <int D, int SPLIT>
__global__ __launch_bounds__(256, SPLIT == 1 ? 3 : 2) void cache4_weights_few_kernel(CacheChunkArgs a) {
  constexpr int G = D / kCacheGroup;
  constexpr bool F32 = SPLIT > 1;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r = lane & 15, kq = lane >> 4;
  auto each_of = [&](const FewSeq& f) { return f.units > 0 ? (int64_t)f.units * max(f.tiles, 1) + kNStart : 0; };  // of a key head
  auto cost = [&](int s) -> int64_t { return a.c.Hk * each_of(few_seq(a, s)); };
  int64_t before;
  const int64_t total = chunk_line(a, lane, &before, cost);
  const int waves = (int)min((int64_t)gridDim.x * 4, total), me = blockIdx.x * 4 + wave;
  if (me >= waves) return;
  const int64_t u0 = run_begin(total, waves, me), u1 = run_begin(total, waves, me + 1);
  int64_t at;
  int s = chunk_place(a.n_seq, before, u0, &at, cost);
  const int64_t page_bytes = (int64_t)a.c.Hk * a.c.block_bytes();
  const int in_page = a.c.page - 1;

  int kv = 0;
  FewSeq f = few_seq(a, s);
  {
    const int64_t each = each_of(f);
    kv = __builtin_amdgcn_readfirstlane(whole_part(u0 - at, each));
    at = uniform64(at + kv * each);
  }
  for (;;) {
    f.q = uniform_seq(f.q);
    const int units = __builtin_amdgcn_readfirstlane(f.units), tiles = __builtin_amdgcn_readfirstlane(f.tiles), rows = __builtin_amdgcn_readfirstlane(f.rows);
    const int per = max(tiles, 1);
    auto unit_at = [&](int64_t x) { return x <= 0 ? 0 : (int)min((x + per - 1) / per, (int64_t)units); };
    const int first = unit_at(u0 - at), last = unit_at(u1 - at);
    if (first < last) {
      const int32_t* blocks = a.table + (int64_t)s * a.max_blocks;
      const int last_block = (f.q.len - 1) >> a.c.log_page;
      const unsigned char* head_base = a.cache + (int64_t)kv * a.c.block_bytes();
      bf16x8 q[SPLIT][G];
      f32x4 shift;
      int see[4];  // tokens that the lane's rows see: rows 4 kq ... + 3 of the tile
      auto load_rows = [&](int tile) {
        const int row = min(tile * 16 + r, rows - 1), tok = a.div_group.div(row), head = kv * a.group + row - tok * a.group;
        const int64_t from = (int64_t)(f.q.start + tok) * a.q.row + (int64_t)head * a.q.head + 8 * kq;
#pragma unroll
        for (int g = 0; g < G; ++g) {
          if constexpr (!F32) {
            q[0][g] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4*>(reinterpret_cast<const uint16_t*>(a.Q) + from + 32 * g));
          } else {
            const f32x4* p = reinterpret_cast<const f32x4*>(reinterpret_cast<const float*>(a.Q) + from + 32 * g);
            const f32x4 x0 = p[0], x1 = p[1];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              float x = 0.5f * (i < 4 ? x0[i % 4] : x1[i % 4]);  // (at half: rounding the first part up leaves the largest finite)
#pragma unroll
              for (int z = 0; z < SPLIT; ++z) {
                q[z][g][i] = (__bf16)x;
                x -= (float)q[z][g][i];
              }
            }
          }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int row4 = tile * 16 + 4 * kq + i, use = min(row4, rows - 1), tok4 = a.div_group.div(use);
          const float l = a.lse[(int64_t)(kv * a.group + use - tok4 * a.group) * a.rows + f.q.start + tok4];
          see[i] = row4 < rows && l != -INFINITY ? f.q.held + tok4 + 1 : 0;  // (a row that sees nothing has lse -inf, and gives nothing)
          shift[i] = F32 ? -l : -l * kLog2e;
        }
      };
      int page_of[4];
      auto find_pages = [&](int unit) {
#pragma unroll
        for (int t = 0; t < 4; ++t) page_of[t] = blocks[min((unit * kNUnit + 16 * t) >> a.c.log_page, last_block)];
      };
      uint32_t words[4][G], scales[4];
      float had = 0.f;
      float* place = nullptr;  // of the lane's token, unit * 64 + lane
      auto load_codes = [&](int unit) {
        int mine = 0;
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          const int p = __builtin_amdgcn_readfirstlane(page_of[t]);
          const bool there = (unsigned)p < (unsigned)a.c.n_pages;
          const unsigned char* b = head_base + (int64_t)(there ? p : 0) * page_bytes;
          const int tok = ((unit * kNUnit + 16 * t) & in_page) + r;
          if constexpr (D == 128) {
            const u32x4 w = *reinterpret_cast<const u32x4*>(b + tok * (D / 2) + kq * (D / 8));
#pragma unroll
            for (int g = 0; g < G; ++g) words[t][g] = w[g];
            scales[t] = *reinterpret_cast<const uint32_t*>(b + a.c.k_scale_at() + tok * 4);
          } else {
            typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
            const u32x2 w = *reinterpret_cast<const u32x2*>(b + tok * (D / 2) + kq * (D / 8));
#pragma unroll
            for (int g = 0; g < G; ++g) words[t][g] = w[g];
            scales[t] = *reinterpret_cast<const uint16_t*>(b + a.c.k_scale_at() + tok * 2);
          }
          if (kq == t) mine = p;
        }
        const int tok = unit * kNUnit + lane;
        place = nullptr;
        if (tok < f.q.len && (unsigned)mine < (unsigned)a.c.n_pages) {
          place = a.weights + ((int64_t)mine * a.c.Hk + kv) * a.c.page + (tok & in_page);
          had = a.fresh || tok >= f.q.held ? 0.f : *place;
        }
      };
      find_pages(first);
      if (rows > 0) load_rows(0);
      load_codes(first);
      if (first + 1 < last) find_pages(first + 1);
      for (int unit = first; unit < last; ++unit) {
        bf16x8 kf[4][G];
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
          for (int g = 0; g < G; ++g) {
            const float sc = scale_of(scales[t], g);
            const u32x4 x = {__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(words[t][g], sc, 0)),
                             __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(words[t][g], sc, 1)),
                             __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(words[t][g], sc, 2)),
                             __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(words[t][g], sc, 3))};
            kf[t][g] = __builtin_bit_cast(bf16x8, x);
          }
        float* const to = place;
        const float old = had;
        if (unit + 1 < last) {
          load_codes(unit + 1);
          if (unit + 2 < last) find_pages(unit + 2);
        }
        float sum[4] = {0.f, 0.f, 0.f, 0.f};  // of token 16 t + r, over the lane's rows
        for (int tile = 0; tile < tiles; ++tile) {
          if (tiles > 1) load_rows(tile);
          f32x4 c[4];
#pragma unroll
          for (int t = 0; t < 4; ++t) {
            c[t] = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int g = 0; g < G; ++g)
#pragma unroll
              for (int z = SPLIT - 1; z >= 0; --z) c[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(q[z][g], kf[t][g], c[t], 0, 0, 0);
          }
#pragma unroll
          for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const float p = F32 ? exp_split(__builtin_fmaf(c[t][i], 2.f, shift[i])) : __builtin_amdgcn_exp2f(__builtin_fmaf(c[t][i], kLog2e, shift[i]));
              sum[t] += unit * kNUnit + 16 * t + r < see[i] ? p : 0.f;
            }
        }
        // over the four lanes of a token; lane (r, kq) is left with token 16 kq + r
        const bool up = lane & 32, odd = lane & 16;
        const float g0 = up ? sum[0] : sum[2], g1 = up ? sum[1] : sum[3];
        const float k0 = (up ? sum[2] : sum[0]) + __shfl_xor(g0, 32), k1 = (up ? sum[3] : sum[1]) + __shfl_xor(g1, 32);
        const float mine = (odd ? k1 : k0) + __shfl_xor(odd ? k0 : k1, 16);
        if (to) *to = old + mine;
      }
    }
    at += units > 0 ? (int64_t)units * per + kNStart : 0;
    if (at >= u1) return;
    if (++kv == a.c.Hk) {
      kv = 0;
      do {
        if (++s >= a.n_seq) return;
        f = few_seq(a, s);
      } while (__builtin_amdgcn_readfirstlane(f.units) == 0);
    }
  }
}

// Which form takes a sequence goes by its own rows of a key head: up to 48 the one for few, where there can be several sequences (64 sequences of 32, 48, 64 and 128 rows, behind up to
// 8192, 8 key heads, few / many: 65 / 95, 69 / 81, 95 / 82, 176 / 134 us; where none has so few, its launch costs 2 to 3).  The host knows the batch's rows and the table's tokens, no more
// of which one sequence can have new.  Where both leave a sequence few rows, the form for few takes everything, in one launch instead of three (32 decoding of up to 1000: 10 / 16 us, 64 of
// up to 16384 77 / 80, 176 of up to 46, most of one new token 12.7 / 25, but 300 of up to 1000, which are more rows than that, 28 / 33), as one sequence may have no more (63 decoding and one
// of n x 4 rows, behind up to 8192, 8 key heads: n = 128 51 / 58 us, 200 70 / 70, 400 114 / 82; fp32 118 / 117, 163 / 140; 511 and one of 2048 x 4: 665 / 283).
// One sequence alone crosses earlier (behind 16384, 8 key heads, 128, 256, 512, 1024 rows: 17 / 18, 27 / 25, 45 / 39, 83 / 65; fp32, d = 64, 256 rows 33 / 17).
constexpr int kFewRows = 48, kAllFew = 128, kAllFewShared = 1024;
void cache4_weights_split(CacheChunkArgs* a) {
  a->div_group = make_fast_div(a->group);
  const int64_t tokens = (int64_t)a->max_blocks << a->c.log_page, rows = (int64_t)a->rows * a->group, steps = (rows + kWRows - 1) / kWRows;
  const int64_t heads = (int64_t)a->n_seq * a->c.Hk;
  const int64_t most = rows < tokens * a->group ? rows : tokens * a->group;  // of a sequence
  a->narrow = rows <= kAllFew || (most <= kAllFewShared && rows <= 32 * (int64_t)a->n_seq) ? 0x7fffffff : a->n_seq >= 4 ? kFewRows : -1;
  const int64_t units = (tokens + kNUnit - 1) / kNUnit * heads * (steps < 1 ? 1 : steps * 4);
  a->few_wgs = a->narrow < 0 ? 0 : (int32_t)(units / 4 + 1 > 768 ? 768 : units / 4 + 1);
  const int64_t runs = (tokens + kWTokens - 1) / kWTokens * heads * (steps + kWTileCost) / kWLeastRun;
  a->parts = a->narrow == 0x7fffffff ? 0 : (int32_t)(runs < 1 ? 1 : runs > kWeightsParts ? kWeightsParts : runs);
}

template <int D, int SPLIT>
static int launch_weights_one(const CacheChunkArgs& a, hipStream_t st) {
  if (a.few_wgs > 0) {
    hipLaunchKernelGGL((cache4_weights_few_kernel<D, SPLIT>), dim3((unsigned)a.few_wgs), dim3(256), 0, st, a);
    const int rc = check_launch();
    if (rc != HA_OK || a.parts == 0) return rc;
  }
  constexpr size_t lds = 2 * WeightsLds<D, SPLIT>::BUF;
  static std::atomic<uint64_t> set{0};
  const auto kernel = &cache4_weights_kernel<D, SPLIT>;
  int rc = allow_full_lds(reinterpret_cast<const void*>(kernel), set);
  if (rc != HA_OK) return rc;
  hipLaunchKernelGGL(kernel, dim3((unsigned)a.parts), dim3(64 * kWWaves), lds, st, a);
  rc = check_launch();
  if (rc != HA_OK) return rc;
  hipLaunchKernelGGL(cache4_weights_join_kernel, dim3((unsigned)a.parts), dim3(kWTokens), 0, st, a);
  return check_launch();
}

int launch_cache4_weights(const CacheChunkArgs& a, int dtype, hipStream_t st) {
  if (a.c.d == 128) return dtype == HA_BF16 ? launch_weights_one<128, 1>(a, st) : launch_weights_one<128, 3>(a, st);
  return dtype == HA_BF16 ? launch_weights_one<64, 1>(a, st) : launch_weights_one<64, 3>(a, st);
}

}  // namespace ha
