// Attention of each sequence's last tokens over its pages of the 4-bit cache (ha_cache4_attn).
//
// One pass over the keys with a running reference and sum of the softmax.  What bounds it is the cache's bytes: a query row costs four flops per cached
// value that 4.25 bits are read for, so a wave keeps 16 query rows (the query heads of one key head, times the tokens of the call) and turns
// codes into bf16 operands in registers, never through LDS:
//   * S^T = K Q^T by v_mfma_f32_16x16x32_bf16: tokens run along M, query rows along N, and one product takes one group of 32 channels.  K's words lie
//     as that operand wants them; v_cvt_scalef32_pk_bf16_fp4 makes two bf16 values of a byte, scale included, and the values are exact.
//   * the accumulators, exponentiated, are the B operand of O^T += V^T P^T: a lane's eight contraction elements are its four tokens of
//     two runs of 16, which is how V's words lie.  A conversion yields two channels of one token, two byte permutations make two tokens of
//     one channel each of two such.
// So per 16 tokens of d = 128 and lane: 32 conversions, 16 permutations, 20 for scales, and some 20 for the softmax, against 2176 bytes.
//
// Split: the tokens of all sequences, in units of 64 (one wave's step), are one line, cut into `parts` equal runs, a workgroup of four waves each per key
// head and tile of 16 query rows: however unlike the sequences' lengths are, every workgroup has the same to read.  The waves of a workgroup take the
// units of a sequence in turn and merge through LDS; a sequence that lies in one workgroup is finished there, the others' parts go to the
// workspace and are joined by a second launch.
#include <type_traits>

#include "attn_common.h"
#include "cache4_common.h"

namespace ha {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

constexpr int kJoinThreads = 256;
constexpr unsigned kJoinsAtOnce = 2048;  // workgroups of the joining launch that the chip holds at once
constexpr int kFewParts = 16;
constexpr int kMostParts = 768;  // workgroups of four waves that the chip holds at once, three per CU
constexpr int kUnit = 64;        // tokens of a wave's step
constexpr int kTilesPerUnit = 4; // of 16 tokens
constexpr int kCRows = 16;       // query rows of a workgroup
// V's scales from here on are taken by the rows that see the token alone: 4 times 2^126 and 2 times 2^127 are infinite, 255 is NaN, and 0 times either is NaN.
constexpr uint32_t kFarScale = 253, kFarSteps = 256 - kFarScale;

// Units of all sequences before s (exclusive), found by one wave: lane l sums a run of sequences.
__device__ inline int seq_len(const CacheAttnArgs& a, int s) { return min(max(a.lens[s], 0), a.max_blocks << a.c.log_page); }
__device__ inline int seq_units(const CacheAttnArgs& a, int s) { return (seq_len(a, s) + kUnit - 1) / kUnit; }
// What a sequence takes of the line: its units and what its start and its end cost a workgroup, in units.  (0 / 2 / 4 / 8: 64 sequences of up to 16384 tokens,
// three queries each, 54 / 51 / 45 / 42 us, 12 and 16 44 and 45; 256 of up to 8192 94 / 76 / 69 / 68, since then 62 and with 12 or 16 69; lengths alike +-0.)
constexpr int kSeqCost = 8;
__device__ inline int seq_cost(const CacheAttnArgs& a, int s) {
  const int n = seq_units(a, s);
  return n > 0 ? n + kSeqCost : 0;
}

// The line's length, and *before: what precedes the lane's run of sequences.  Wave-uniform results.
__device__ inline int line_total(const CacheAttnArgs& a, int lane, int* before) {
  const int each = (a.n_seq + 63) / 64, s0 = min(a.n_seq, lane * each), s1 = min(a.n_seq, s0 + each);
  int sum = 0;
  for (int s = s0; s < s1; s += 4) {  // (four lengths asked for at a time: 1000 sequences of up to 4096 52.2 -> 51.2 us)
    int cost[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) cost[i] = seq_cost(a, min(s + i, s1 - 1));
#pragma unroll
    for (int i = 0; i < 4; ++i) sum += s + i < s1 ? cost[i] : 0;
  }
  int inc = sum;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int up = __shfl_up(inc, o);
    if (lane >= o) inc += up;
  }
  *before = inc - sum;
  return __builtin_amdgcn_readfirstlane(__shfl(inc, 63));
}
// The sequence at place u of the line (u < total), and where it begins
__device__ inline int find_place(const CacheAttnArgs& a, int lane, int before, int u, int* seq_first) {
  const int each = (a.n_seq + 63) / 64;
  // the last lane whose run starts at or before u (runs without units start where the next one does)
  const unsigned long long le = __ballot(before <= u);
  const int run = 63 - __builtin_clzll(le);
  int at = __builtin_amdgcn_readfirstlane(__shfl(before, run));
  int s = run * each;
  for (; s < a.n_seq - 1; ++s) {
    const int n = seq_cost(a, s);
    if (u < at + n) break;
    at += n;
  }
  *seq_first = at;
  return __builtin_amdgcn_readfirstlane(s);
}

// 16 tokens' raw words
template <int D>
struct RawTile {
  uint32_t k[D / 32];
  u32x4 v;              // a token's word each
  uint32_t ks;          // the token's scales, a byte per group
  uint32_t vs[D == 128 ? 4 : 2];  // of the lane's four tokens
};

template <int SPLIT>
struct Weights {
  uint32_t w[SPLIT][4];  // eight tokens in bf16: parts of each weight, the largest first
};

// SPLIT: parts of a query number and of a weight: 1 for bf16 queries, 3 for fp32 ones (24 bits); cached values have one.
// NW waves.  WHOLE: a workgroup per sequence, which it finishes (small tables: no second launch).  ONCE: codes are read past the caches.
// MULTI: several queries a sequence, which see its last tokens in part.
// bf16, four waves, d = 128, tokens shared out: held to the 168 registers of three workgroups a CU, which costs 2 spilled ones, MULTI 4 (12 and 20 bytes of scratch).
template <int D, int SPLIT, int NW, bool WHOLE, bool ONCE, bool MULTI>
__global__ __launch_bounds__(64 * NW, SPLIT == 1 && NW == 4 ? 3 : 2) void cache4_attn_kernel(CacheAttnArgs a) {
  constexpr int kCWaves = NW, kCThreads = 64 * NW;
  constexpr int G = D / 32;     // groups of channels, products per score
  constexpr int MT = D / 16;    // tiles of 16 channels of the output
  constexpr bool F32 = SPLIT > 1;
  __shared__ float merge_o[kCWaves][kCRows][D + 4];
  __shared__ float merge_m[kCWaves][kCRows], merge_l[kCWaves][kCRows];

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r = lane & 15, kq = lane >> 4;
  const int hk = blockIdx.y % a.c.Hk, tile = blockIdx.y / a.c.Hk;

  int s, part = 0, u0 = 0, u1 = 0x7fffffff, seq_first = 0;
  if constexpr (WHOLE) {
    s = blockIdx.x;
  } else {
    int before;
    const int total = line_total(a, lane, &before);
    part = blockIdx.x;
    const int parts = min(a.parts, (total + NW - 1) / NW);  // (a unit for every wave)
    if (part >= parts) return;
    u0 = (int)((int64_t)total * part / parts);
    u1 = (int)((int64_t)total * (part + 1) / parts);
    s = find_place(a, lane, before, u0, &seq_first);
  }

  const int row = tile * kCRows + r;                   // query row within the key head
  const int row_use = row < a.rows ? row : 0;
  const int q_tok = row_use / a.group, q_head = hk * a.group + row_use % a.group;

  const int64_t page_bytes = (int64_t)a.c.Hk * a.c.block_bytes();
  const unsigned char* head_base = a.cache + (int64_t)hk * a.c.block_bytes();
  const int log_page = a.c.log_page, in_page = a.c.page - 1;

  for (;;) {
    const int len = seq_len(a, s);
    const int n_units = (len + kUnit - 1) / kUnit;
    const int first = max(u0 - seq_first, 0), last = min(u1 - seq_first, n_units);  // units of the sequence that are this workgroup's
    if (WHOLE || first < last) {
    const int32_t* blocks = a.table + (int64_t)s * a.max_blocks;
    const int last_block = max(len - 1, 0) >> log_page;

    bf16x8 q[SPLIT][G];
    {
      const int64_t at = ((int64_t)s * a.q_len + q_tok) * a.q.row + (int64_t)q_head * a.q.head + 8 * kq;
#pragma unroll
      for (int g = 0; g < G; ++g) {
        if constexpr (!F32) {
          q[0][g] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4*>(reinterpret_cast<const uint16_t*>(a.Q) + at + 32 * g));
        } else {
          const f32x4* p = reinterpret_cast<const f32x4*>(reinterpret_cast<const float*>(a.Q) + at + 32 * g);
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
    }
    const int limit = len - a.q_len + 1 + q_tok;  // tokens that the lane's row sees
    const int all_see = len - a.q_len + 1;        // that every row sees

    RawTile<D> raw[kTilesPerUnit];
    f32x4 o[MT];
#pragma unroll
    for (int i = 0; i < MT; ++i) o[i] = (f32x4){0.f, 0.f, 0.f, 0.f};
    // reference of the exponentials, moved (and the sums rescaled) where a row's scores exceed it by more than 8; log2 domain for bf16
    // queries, natural for fp32 ones; l: this lane's share of the row sum
    float m = -INFINITY, l = 0.f;
    bool some_taken = false;  // (wave-uniform) a group was taken out
    constexpr float unit_of = F32 ? 2.f : kLog2e;
    auto fetch = [](const auto* p) { return ONCE ? __builtin_nontemporal_load(p) : *p; };
    int page_of[kTilesPerUnit];
    auto find_pages = [&](int unit) {
#pragma unroll
      for (int t = 0; t < kTilesPerUnit; ++t) page_of[t] = blocks[min((unit * kUnit + 16 * t) >> log_page, last_block)];
    };
    auto tile_base = [&](int unit, int t, bool* there) {  // the page's block, and whether the page exists
      const int p = __builtin_amdgcn_readfirstlane(page_of[t]);
      *there = (unsigned)p < (unsigned)a.c.n_pages;
      return head_base + (int64_t)(*there ? p : 0) * page_bytes;
    };
    auto load_k = [&](int unit) {
#pragma unroll
      for (int t = 0; t < kTilesPerUnit; ++t) {
        bool there;
        const unsigned char* b = tile_base(unit, t, &there);
        const int tok = (unit * kUnit + 16 * t) & in_page;
        const unsigned char* kp = b + (tok + r) * (D / 2) + kq * (D / 8);
        if constexpr (D == 128) {
          const u32x4 w = fetch(reinterpret_cast<const u32x4*>(kp));
#pragma unroll
          for (int g = 0; g < G; ++g) raw[t].k[g] = w[g];
          raw[t].ks = *reinterpret_cast<const uint32_t*>(b + a.c.k_scale_at() + (tok + r) * 4);
        } else {
          const u32x2 w = fetch(reinterpret_cast<const u32x2*>(kp));
#pragma unroll
          for (int g = 0; g < G; ++g) raw[t].k[g] = w[g];
          raw[t].ks = *reinterpret_cast<const uint16_t*>(b + a.c.k_scale_at() + (tok + r) * 2);
        }
      }
    };
    auto load_v = [&](int unit) {
#pragma unroll
      for (int t = 0; t < kTilesPerUnit; ++t) {
        bool there;
        const unsigned char* b = tile_base(unit, t, &there);
        const int tok = (unit * kUnit + 16 * t) & in_page;
        raw[t].v = fetch(reinterpret_cast<const u32x4*>(b + a.c.v_at() + ((tok >> 2) + kq) * (D * 2) + (D == 128 ? r : r >> 1) * 16));
        if constexpr (D == 128) {
          const u32x4 sc = *reinterpret_cast<const u32x4*>(b + a.c.v_scale_at() + (tok + 4 * kq) * 4);
#pragma unroll
          for (int i = 0; i < 4; ++i) raw[t].vs[i] = sc[i];
        } else {
          const u32x2 sc = *reinterpret_cast<const u32x2*>(b + a.c.v_scale_at() + (tok + 4 * kq) * 2);
          raw[t].vs[0] = sc[0];
          raw[t].vs[1] = sc[1];
        }
      }
    };

    int unit = first + wave;
    if (unit < last) {
      find_pages(unit);
      load_k(unit);
      load_v(unit);
    }
    for (; unit < last; unit += kCWaves) {
      const int next = unit + kCWaves;
      const bool more = next < last;
      bool there[kTilesPerUnit];
#pragma unroll
      for (int t = 0; t < kTilesPerUnit; ++t) there[t] = (unsigned)__builtin_amdgcn_readfirstlane(page_of[t]) < (unsigned)a.c.n_pages;
      if (more) find_pages(next);

      // ---- scores ----
      f32x4 c[kTilesPerUnit];
#pragma unroll
      for (int t = 0; t < kTilesPerUnit; ++t) {
        c[t] = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int g = 0; g < G; ++g) {
          const float sc = __uint_as_float(g < 3 ? raw[t].ks << (23 - 8 * g) : raw[t].ks >> 1);  // (the exponent alone counts)
          const uint32_t w = raw[t].k[g];
          u32x4 f;
          f[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, sc, 0));
          f[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, sc, 1));
          f[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, sc, 2));
          f[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, sc, 3));
#pragma unroll
          for (int z = SPLIT - 1; z >= 0; --z)
            c[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, f), q[z][g], c[t], 0, 0, 0);
        }
      }
      if (more) load_k(next);

      // ---- masks: tokens behind the row's own, behind the sequence, of pages that are not there ----
      const int base = unit * kUnit;
      bool special = base + kUnit > all_see;
#pragma unroll
      for (int t = 0; t < kTilesPerUnit; ++t) special = special || !there[t];
      if (special) {
        uint32_t taken = 0;
#pragma unroll
        for (int t = 0; t < kTilesPerUnit; ++t)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int tok = base + 16 * t + 4 * kq + i;
            if (!there[t] || tok >= limit) c[t][i] = -INFINITY;
            if (!there[t] || tok >= len) {  // whatever lies there: weight 0 times a NaN would be NaN
              raw[t].v[i] = 0;
              if (D == 128) raw[t].vs[i % (D / 32)] = 0;
              else raw[t].vs[i / 2] &= i & 1 ? 0x0000ffffu : 0xffff0000u;
            }
            if constexpr (MULTI) {  // groups that are NaN or may lie past the largest number, of tokens that some rows see alone, are taken out here
              uint32_t& w = raw[t].vs[D == 128 ? i % (D / 32) : i / 2];
              const uint32_t bytes = D == 128 ? 0x01010101u : i & 1 ? 0x01010000u : 0x00000101u;
              const uint32_t far = (((w & 0x7f7f7f7fu) + kFarSteps * 0x01010101u) & w) >> 7 & (tok >= all_see ? bytes : 0u);  // 1 in every byte from kFarScale on
              w &= ~((far << 8) - far);
              taken |= far;
            }
          }
        if (MULTI && __any(taken != 0)) some_taken = true;
      }

      // ---- weights ----
      float mx = fmaxf(fmaxf(c[0][0], c[0][1]), fmaxf(c[0][2], c[0][3]));
#pragma unroll
      for (int t = 1; t < kTilesPerUnit; ++t) mx = fmaxf(mx, fmaxf(fmaxf(c[t][0], c[t][1]), fmaxf(c[t][2], c[t][3])));
      mx *= unit_of;
      if (__any(mx > m + (F32 ? 5.5f : 8.f))) {
        mx = fmaxf(mx, __shfl_xor(mx, 16));
        mx = fmaxf(mx, __shfl_xor(mx, 32));
        const float m_new = fmaxf(m, mx), ref = m_new == -INFINITY ? 0.f : m_new;
        const float alpha = F32 ? expf(m - ref) : __builtin_amdgcn_exp2f(m - ref);
#pragma unroll
        for (int i = 0; i < MT; ++i) o[i] *= alpha;
        l *= alpha;
        m = m_new;
      }
      const float ref = m == -INFINITY ? 0.f : m;
      Weights<SPLIT> p[kTilesPerUnit / 2];
#pragma unroll
      for (int t = 0; t < kTilesPerUnit; ++t)
#pragma unroll
        for (int i = 0; i < 4; i += 2) {
          float x0, x1;
          if constexpr (F32) {
            x0 = exp_split(__builtin_fmaf(c[t][i], unit_of, -ref));
            x1 = exp_split(__builtin_fmaf(c[t][i + 1], unit_of, -ref));
          } else {
            x0 = __builtin_amdgcn_exp2f(__builtin_fmaf(c[t][i], unit_of, -ref));
            x1 = __builtin_amdgcn_exp2f(__builtin_fmaf(c[t][i + 1], unit_of, -ref));
          }
          l += x0 + x1;
#pragma unroll
          for (int z = 0; z < SPLIT; ++z) {
            const uint32_t w = pack_bf16x2(x0, x1);
            p[t / 2].w[z][2 * (t % 2) + i / 2] = w;
            if (z + 1 < SPLIT) {
              x0 -= __uint_as_float(w << 16);
              x1 -= __uint_as_float(w & 0xffff0000u);
            }
          }
        }

      // ---- O^T += V^T P^T, two runs of 16 tokens at a time ----
#pragma unroll
      for (int pr = 0; pr < kTilesPerUnit / 2; ++pr) {
#pragma unroll
        for (int g = 0; g < G; ++g) {
          u32x4 f[2];  // the group's even and odd channels of the lane, eight tokens each
#pragma unroll
          for (int half = 0; half < 2; ++half) {
            const RawTile<D>& t = raw[2 * pr + half];
            uint32_t x[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              float sc;
              uint32_t b;
              if constexpr (D == 128) {
                sc = __uint_as_float(g < 3 ? t.vs[i] << (23 - 8 * g) : t.vs[i] >> 1);
                if (g == 0) b = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(t.v[i], sc, 0));
                else if (g == 1) b = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(t.v[i], sc, 1));
                else if (g == 2) b = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(t.v[i], sc, 2));
                else b = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(t.v[i], sc, 3));
              } else {
                const int byte = 2 * (i & 1) + g;   // of the word with the scales of tokens i & ~1 and behind
                sc = __uint_as_float(byte < 3 ? t.vs[i / 2] << (23 - 8 * byte) : t.vs[i / 2] >> 1);
                const uint32_t w = t.v[i] >> (8 * (r & 1));
                if (g == 0) b = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, sc, 0));
                else b = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, sc, 2));
              }
              x[i] = b;
            }
            f[0][2 * half] = __builtin_amdgcn_perm(x[1], x[0], 0x05040100u);
            f[0][2 * half + 1] = __builtin_amdgcn_perm(x[3], x[2], 0x05040100u);
            f[1][2 * half] = __builtin_amdgcn_perm(x[1], x[0], 0x07060302u);
            f[1][2 * half + 1] = __builtin_amdgcn_perm(x[3], x[2], 0x07060302u);
          }
#pragma unroll
          for (int e = 0; e < 2; ++e)
#pragma unroll
            for (int z = SPLIT - 1; z >= 0; --z) {
              const u32x4 w = {p[pr].w[z][0], p[pr].w[z][1], p[pr].w[z][2], p[pr].w[z][3]};
              o[2 * g + e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, f[e]), __builtin_bit_cast(bf16x8, w), o[2 * g + e], 0, 0, 0);
            }
        }
      }
      if (more) load_v(next);
    }

    // ---- the waves' sums through LDS.  Lane (r, kq), register i of o[2 g + e]: query row r, channel 32 g + 8 kq + 2 i + e ----
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    if (MULTI && some_taken) {  // rare: these groups of the wave's own tokens, for the rows that see them
      // (all that this needs beside m and o is formed again, the query read again: kept, it would take registers from the loop)
      int thread = threadIdx.x;
      asm volatile("" : "+v"(thread));
      const int quad = (thread & 63) >> 4, own_row = tile * kCRows + (thread & 15), own = own_row < a.rows ? own_row : 0, own_tok = own / a.group;
      const int64_t q_at = ((int64_t)s * a.q_len + own_tok) * a.q.row + (int64_t)(hk * a.group + own % a.group) * a.q.head + 8 * quad;
      for (int u = first + wave; u < last; u += kCWaves)
        for (int tok = max(u * kUnit, max(all_see, 0)); tok < min(u * kUnit + kUnit, len); ++tok) {
          const int page = blocks[tok >> log_page], at = tok & in_page;
          if ((unsigned)page >= (unsigned)a.c.n_pages) continue;
          const unsigned char* b = head_base + (int64_t)page * page_bytes;
          const unsigned char* k_scales = b + a.c.k_scale_at() + at * G;
          const unsigned char* v_scales = b + a.c.v_scale_at() + at * G;
          bool any = false;
#pragma unroll
          for (int g = 0; g < G; ++g) any = any || v_scales[g] >= kFarScale;
          if (!any) continue;
          auto two = [](uint32_t w, uint32_t byte, auto sel) {
            return __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, __uint_as_float(byte << 23), decltype(sel)::value);
          };
          float score = 0.f;
          auto add = [&](int c, f32x2 k) {
            f32x2 x;
            if constexpr (F32) {
              x = *reinterpret_cast<const f32x2*>(reinterpret_cast<const float*>(a.Q) + q_at + c);
            } else {
              const uint32_t w = *reinterpret_cast<const uint32_t*>(reinterpret_cast<const uint16_t*>(a.Q) + q_at + c);
              x = (f32x2){__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u)};
            }
            score = __builtin_fmaf(x[1], k[1], __builtin_fmaf(x[0], k[0], score));
          };
#pragma unroll 1
          for (int g = 0; g < G; ++g) {
            const uint32_t w = *reinterpret_cast<const uint32_t*>(b + at * (D / 2) + quad * (D / 8) + 4 * g), byte = k_scales[g];
            add(32 * g, two(w, byte, std::integral_constant<int, 0>{}));
            add(32 * g + 2, two(w, byte, std::integral_constant<int, 1>{}));
            add(32 * g + 4, two(w, byte, std::integral_constant<int, 2>{}));
            add(32 * g + 6, two(w, byte, std::integral_constant<int, 3>{}));
          }
          score += __shfl_xor(score, 16);
          score += __shfl_xor(score, 32);
          const float ref = m == -INFINITY ? 0.f : m;
          const float weight = F32 ? expf(score - ref) : (float)(__bf16)__builtin_amdgcn_exp2f(__builtin_fmaf(score, kLog2e, -ref));
          const unsigned char* v_row = b + a.c.v_at() + (at >> 2) * (D * 2) + (at & 3) * 4;
#pragma unroll
          for (int g = 0; g < G; ++g) {
            if (v_scales[g] < kFarScale || tok >= all_see + own_tok) continue;
#pragma unroll
            for (int i = 0; i < 4; ++i) {  // channels 32 g + 8 quad + 2 i and the next
              const int pair = 4 * quad + i, word = D == 128 ? pair : pair / 2, byte = D == 128 ? g : 2 * g + i % 2;
              const uint32_t w = *reinterpret_cast<const uint32_t*>(v_row + word * 16) >> (8 * byte);
              const f32x2 v = two(w, v_scales[g], std::integral_constant<int, 0>{});
              o[2 * g][i] = __builtin_fmaf(weight, v[0], o[2 * g][i]);
              o[2 * g + 1][i] = __builtin_fmaf(weight, v[1], o[2 * g + 1][i]);
            }
          }
        }
    }
    if (kq == 0) {
      merge_m[wave][r] = m;
      merge_l[wave][r] = l;
    }
#pragma unroll
    for (int g = 0; g < G; ++g) {
      float* at = &merge_o[wave][r][32 * g + 8 * kq];
      *reinterpret_cast<f32x4*>(at) = (f32x4){o[2 * g][0], o[2 * g + 1][0], o[2 * g][1], o[2 * g + 1][1]};
      *reinterpret_cast<f32x4*>(at + 4) = (f32x4){o[2 * g][2], o[2 * g + 1][2], o[2 * g][3], o[2 * g + 1][3]};
    }
    __syncthreads();
    const bool whole = WHOLE || (first == 0 && last == n_units);
    constexpr int LPR = D / 4;
    for (int idx = threadIdx.x; idx < kCRows * LPR; idx += kCThreads) {
      const int rr = idx / LPR, ch = (idx % LPR) * 4;
      const int rw = tile * kCRows + rr;
      if (rw >= a.rows) break;
      float top = merge_m[0][rr];
#pragma unroll
      for (int w = 1; w < kCWaves; ++w) top = fmaxf(top, merge_m[w][rr]);
      const float ref = top == -INFINITY ? 0.f : top;
      f32x4 acc = {0.f, 0.f, 0.f, 0.f};
      float sum = 0.f;
#pragma unroll
      for (int w = 0; w < kCWaves; ++w) {
        const float wt = F32 ? expf(merge_m[w][rr] - ref) : __builtin_amdgcn_exp2f(merge_m[w][rr] - ref);
        sum += wt * merge_l[w][rr];
        acc += wt * *reinterpret_cast<const f32x4*>(&merge_o[w][rr][ch]);
      }
      if (whole) {
        const bool empty = sum == 0.f;
        const float inv = empty ? 0.f : 1.f / sum;
        acc *= inv;
        const int64_t orow = (int64_t)s * a.q_len + rw / a.group;
        const int head = hk * a.group + rw % a.group;
        const int64_t at = orow * a.o.row + (int64_t)head * a.o.head + ch;
        if constexpr (F32) *reinterpret_cast<f32x4*>(reinterpret_cast<float*>(a.out) + at) = acc;
        else *reinterpret_cast<u32x2*>(reinterpret_cast<uint16_t*>(a.out) + at) = (u32x2){pack_bf16x2(acc[0], acc[1]), pack_bf16x2(acc[2], acc[3])};
        if (ch == 0)
          a.lse[(int64_t)head * a.n_seq * a.q_len + orow] = empty ? -INFINITY : F32 ? top + logf(sum) : (top + log2f(sum)) * kLn2;
      } else {
        const int64_t slot = ((int64_t)blockIdx.y * (a.parts + a.n_seq) + part + s) * kCRows + rr;
        *reinterpret_cast<f32x4*>(a.part_o + slot * D + ch) = acc;
        if (ch == 0) {
          a.part_ml[2 * slot] = top;
          a.part_ml[2 * slot + 1] = sum;
        }
      }
    }
    if (!WHOLE && blockIdx.y == 0 && threadIdx.x == 0) {
      if (first == 0) a.span[2 * s] = part;
      if (last == n_units) a.span[2 * s + 1] = part;
    }
    if constexpr (WHOLE) return;
    __syncthreads();
    }
    seq_first += n_units > 0 ? n_units + kSeqCost : 0;
    if (seq_first >= u1) return;
    ++s;  // (the line goes on: another sequence follows)
  }
}

// Joins the parts of the query rows, or writes the result of one that sees nothing.  A group of D / 4 threads holds a row's sums and takes parts eight at a time
// while there are, so that their numbers and rows are read without waiting for one another (one sequence of 131072 tokens, one key head, whose rows have hundreds of
// parts, one at a time -> eight, the whole call: 44 -> 17 us).  A row has a workgroup to itself, whose groups take its parts in turn; in launches of more rows than
// workgroups run at once, a row of few parts has one group alone, and the workgroups too many end at once (the whole call: 64 sequences of up to 16384 tokens, three queries
// each, 6144 rows, 44.2 -> 42.0 us; 32 of up to 4096, eight each, 8192 rows, 29.5 -> 26.3; but 60 of up to 8000, 960 rows, 24.6 -> 25.5).
template <int D, int SPLIT>
__global__ __launch_bounds__(kJoinThreads) void cache4_join_kernel(CacheAttnArgs a) {
  constexpr bool F32 = SPLIT > 1;
  constexpr int LPR = D / 4, PAR = kJoinThreads / LPR, AHEAD = 8;
  __shared__ f32x4 sum_o[PAR][LPR];
  __shared__ float sum_l[PAR], sum_m[PAR];
  const int s = blockIdx.x, lane = threadIdx.x % LPR, mine = threadIdx.x / LPR, ch = lane * 4;
  const int len = seq_len(a, s);
  const int p0 = a.span[2 * s], p1 = a.span[2 * s + 1];  // (asked for with the length; of an empty sequence they are what was there)
  const int parts = len > 0 ? p1 - p0 + 1 : 0;
  if (parts == 1) return;  // finished where its tokens were read
  const bool few = parts <= kFewParts && gridDim.x * gridDim.y > kJoinsAtOnce;
  const int rows = a.Hq * a.q_len, y = few ? (int)blockIdx.y * PAR + mine : (int)blockIdx.y;
  if (y >= rows) return;   // (few: no barrier follows; many: all threads alike)
  const int hq = y % a.Hq, tok = y / a.Hq;
  const int hk = hq / a.group, row = tok * a.group + hq % a.group, tile = row / kCRows, rr = row % kCRows;
  const int64_t orow = (int64_t)s * a.q_len + tok;
  const int64_t slot0 = ((int64_t)(tile * a.c.Hk + hk) * (a.parts + a.n_seq) + s + p0) * kCRows + rr;
  auto exp_of = [](float x) { return F32 ? expf(x) : __builtin_amdgcn_exp2f(x); };
  float m = -INFINITY, l = 0.f;
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  const int step = few ? 1 : PAR;
  int p = few ? 0 : mine;
  auto take = [&](auto count) {
    constexpr int N = decltype(count)::value;
    float pm[N], pl[N];
    f32x4 v[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int64_t slot = slot0 + (int64_t)(p + i * step) * kCRows;
      pm[i] = a.part_ml[2 * slot];
      pl[i] = a.part_ml[2 * slot + 1];
      v[i] = *reinterpret_cast<const f32x4*>(a.part_o + slot * D + ch);
    }
    float top = m;
#pragma unroll
    for (int i = 0; i < N; ++i) top = fmaxf(top, pm[i]);
    const float ref = top == -INFINITY ? 0.f : top, w0 = exp_of(m - ref);
    acc *= w0;
    l *= w0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float w = exp_of(pm[i] - ref);
      acc += w * v[i];
      l += w * pl[i];
    }
    m = top;
    p += N * step;
  };
  while (p + (AHEAD - 1) * step < parts) take(std::integral_constant<int, AHEAD>{});
  while (p + step < parts) take(std::integral_constant<int, 2>{});
  if (p < parts) take(std::integral_constant<int, 1>{});
  auto finish = [&] {
    const bool empty = l == 0.f;
    acc *= empty ? 0.f : 1.f / l;
    const int64_t at = orow * a.o.row + (int64_t)hq * a.o.head + ch;
    if constexpr (F32) *reinterpret_cast<f32x4*>(reinterpret_cast<float*>(a.out) + at) = acc;
    else *reinterpret_cast<u32x2*>(reinterpret_cast<uint16_t*>(a.out) + at) = (u32x2){pack_bf16x2(acc[0], acc[1]), pack_bf16x2(acc[2], acc[3])};
    if (lane == 0) a.lse[(int64_t)hq * a.n_seq * a.q_len + orow] = empty ? -INFINITY : F32 ? m + logf(l) : (m + log2f(l)) * kLn2;
  };
  if (few) {
    finish();
    return;
  }
  sum_o[mine][lane] = acc;
  if (lane == 0) {
    sum_m[mine] = m;
    sum_l[mine] = l;
  }
  __syncthreads();
  if (mine != 0) return;
#pragma unroll
  for (int i = 1; i < PAR; ++i) m = fmaxf(m, sum_m[i]);
  const float ref = m == -INFINITY ? 0.f : m;
  acc = (f32x4){0.f, 0.f, 0.f, 0.f};
  l = 0.f;
#pragma unroll
  for (int i = 0; i < PAR; ++i) {
    const float w = exp_of(sum_m[i] - ref);
    acc += w * sum_o[i][lane];
    l += w * sum_l[i];
  }
  finish();
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
