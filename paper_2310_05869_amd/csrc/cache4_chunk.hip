// Attention of chunks of new tokens over their sequences' pages of the 4-bit cache (ha_cache4_attn_chunk).
//
// One pass over the keys with a running reference and sum of the softmax, as in attn_mfma.hip: a wave keeps 32 query rows, S^T = K Q^T by
// v_mfma_f32_32x32x16_bf16 over 64 tokens a step, the weights are the B operand of O^T += V^T P^T.  What differs is where tiles come from: the query
// heads of a key head and some tokens of theirs share a workgroup (128 rows), which turns the codes of a step into bf16 once, in registers, and lays them
// into LDS for its four waves.  Cached values are exact in bf16, so products are those of bf16 tensors.  Weights of bf16 queries enter P V rounded to bf16 once, by at most 2^-8 of each (the
// row's sum is of unrounded ones): the instruction's other operand is exact in bf16, and two parts would be twice the products.  Results lie 1.7 to 2.3e-3 from those of 64 bits, where
// rounding them to bf16 is 1.6e-3.  Weights of fp32 queries have three parts, 24 bits.
//   * A wave takes the K codes, V codes and scales of 16 tokens, which lie in one page: a uniform base.  v_cvt_scalef32_pk_bf16_fp4 makes two values of a
//     byte, scale included; a lane's words become whole pieces of 16 bytes of LDS rows, because channels may lie in any order that the other
//     operand shares: K's rows hold the page's words in their order, Q is loaded alike; V's rows hold a word's eight channels together, and
//     the output's channels are put in order when it is written.
//   * Split: the tiles of all sequences and heads are one line, a tile's length in it the tokens that its last row sees (and what its start and end
//     cost), cut into equal runs, a workgroup each: whatever the lengths are, all have the same to do.  Sums of tiles that a cut divides go to the
//     workspace and are joined by a second launch.
#include <type_traits>

#include "cache4_attn.h"
#include "cache4_chunk.h"

namespace ha {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef s16x4 __attribute__((address_space(3))) * lds_s16x4_ptr;

constexpr int kStep = 64;           // tokens of a step
// What a tile's start and end cost a workgroup, in tokens.  (128 / 256 / 400 / 600: 64 sequences, most of one token, behind up to 16384, 32 and 8 heads, d = 128 259 / 231 / 217 / 220 us;
// 24 of up to 200 behind up to 4096, 12 and 4 heads 58 / 55 / 55 / 57; 16 of up to 1024 behind up to 8192, 16 heads, d = 64 118 / 106 / 108 / 109.  Later, 256 / 320 / 400: 64 with 8 pieces of
// prompts 484 / 483 / 482; 24 of up to 200 77 / 76 / 75; fp32, 6 of up to 150 behind up to 4000, 8 and 2 heads, d = 128 53 / 52 / 61; one of 100 and one of 50 35 / 34 / 36.)
constexpr int kTileCost = 320;
static_assert(chunk_upto(0x7fffffff - 257, 1, 1, kTileCost) == 0x7fffffffll - 257 + kTileCost + 1);  // (the most tokens that a call may hold: past 32 bits)
constexpr int kLeastRun = 256;      // tokens of the line that a workgroup takes, at least (fp32, 6 sequences of up to 150 behind up to 2000, d = 64: 512 36 us, 256 29)
constexpr int kChunkParts = 512;    // workgroups that the chip holds at once, two per CU

template <int D>
struct ChunkLds {
  static constexpr int KSTR = (D + 8) * 2;   // bytes per K row (+16: conflict-free 16-byte row reads)
  static constexpr int VSTR = (D + 32) * 2;  // bytes per V row (+64: conflict-free transposing reads)
  static constexpr int K_BYTES = kStep * KSTR;
  static constexpr int BUF = K_BYTES + kStep * VSTR;
  static constexpr int ROW = D * 4 + 16;           // a row of the output on its way out
  static constexpr int WAVE = 32 * ROW + 32 * 8;
  static constexpr int FLAGS = 3 * 16;             // far_flag; per buffer, which quarters of its K lie in pages that are not there
  static constexpr int bytes(int nw) { return (2 * BUF > nw * WAVE ? 2 * BUF : nw * WAVE) + FLAGS; }
};

// What a wave holds of 16 tokens: K words and scales of a token, V words and scales of four (d = 64: two) tokens
template <int D>
struct RawK {
  std::conditional_t<D == 128, u32x4, u32x2> w;
  uint32_t sc;
};
template <int D>
struct RawV {
  std::conditional_t<D == 128, u32x4, u32x2> w;
  std::conditional_t<D == 128, u32x4, uint32_t> sc;
};

template <int SEL>
__device__ inline uint32_t two_values(uint32_t w, float sc) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, sc, SEL));
}

// SPLIT: parts of a query number and of a weight: 1 for bf16 queries, 3 for fp32 ones (24 bits); cached values have one.  WHOLE: a workgroup per tile.
// x: the workgroup's number.
template <int D, int SPLIT, int NW, bool WHOLE>
__device__ __forceinline__ void cache4_chunk_run(const CacheChunkArgs& a, unsigned char* smem, int x) {
  using L = ChunkLds<D>;
  constexpr int QT = 32 * NW, KS = D / 16, DT = D / 32, G = D / kCacheGroup;
  constexpr bool F32 = SPLIT > 1;
  int* far_flag = reinterpret_cast<int*>(smem + L::bytes(NW) - L::FLAGS);
  u32x4* gone_flags = reinterpret_cast<u32x4*>(far_flag + 4);

  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int part16 = wave & 3;  // the 16 tokens of a step that the wave lays into LDS

  // ---- place ----
  const int tt = a.tile_tokens, heads = a.c.Hk * a.subs;
  auto tiles_of = [&](const ChunkSeq& q) { return (int64_t)q.n * a.group <= a.narrow ? 0 : a.div_tokens.div(q.n + tt - 1); };
  auto upto = [&](const ChunkSeq& q, int64_t t) { return chunk_upto(q.held, tt, t, kTileCost); };  // line before tile t of a head
  auto cost = [&](int s) -> int64_t {
    const ChunkSeq q = chunk_seq(a, s);
    const int T = tiles_of(q);
    return heads * (WHOLE ? (int64_t)T : upto(q, T));
  };
  int64_t before;
  const int64_t total = chunk_line(a, threadIdx.x & 63, &before, cost);
  int parts = 1, part = 0;
  int64_t u0 = x, u1 = 0;
  if constexpr (WHOLE) {
    if (u0 >= total) return;
  } else {
    parts = (int)min((int64_t)a.parts, max(total / kLeastRun, (int64_t)1));
    if (parts > 8) parts &= ~7;
    part = x;
    if (part < parts && (parts & 7) == 0) part = (part & 7) * (parts >> 3) + (part >> 3);  // a run of the line per XCD: neighbours share keys
    if (threadIdx.x == 0) a.joins[8 * part] = -1;
    if (part >= parts || total == 0) return;
    u0 = run_begin(total, parts, part);
    u1 = run_begin(total, parts, part + 1);
  }
  int64_t tile_first;
  int s = chunk_place(a.n_seq, before, u0, &tile_first, cost);
  ChunkSeq q = uniform_seq(chunk_seq(a, s));
  int T = tiles_of(q), hh, t;
  {
    const int64_t head_cost = WHOLE ? (int64_t)T : upto(q, T), rem = u0 - tile_first;
    hh = whole_part(rem, head_cost);
    const int64_t in_head = rem - (int64_t)hh * head_cost;
    if constexpr (WHOLE) {
      t = T - 1 - (int)in_head;
    } else {
      int lo = 0, hi = T;  // upto(lo) <= in_head < upto(hi)
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (upto(q, mid) <= in_head) lo = mid;
        else hi = mid;
      }
      t = lo;
      tile_first += hh * head_cost + upto(q, t);
    }
    hh = __builtin_amdgcn_readfirstlane(hh);
    t = __builtin_amdgcn_readfirstlane(t);
    tile_first = uniform64(tile_first);
  }

  const int64_t page_bytes = (int64_t)a.c.Hk * a.c.block_bytes();
  const int log_page = a.c.log_page, in_page = a.c.page - 1;

  for (;;) {
    const int seen = min(max(q.held + min((t + 1) * tt, q.n), 0), q.len);  // tokens that the tile's last row sees
    const int all_see = q.held + t * tt + 1;                               // that all rows see
    const int nsteps = (seen + kStep - 1) / kStep;
    const int64_t length = max(q.held, 0) + (int64_t)(t + 1) * tt + kTileCost;
    auto step_at = [&](int64_t x) { return x <= 0 ? 0 : (int)min((x + kStep - 1) / kStep, (int64_t)nsteps); };
    const int first = WHOLE ? 0 : step_at(u0 - tile_first), last = WHOLE ? nsteps : step_at(min(u1 - tile_first, length));
    if (first < last || (nsteps == 0 && (WHOLE || tile_first >= u0))) {
      int lane = threadIdx.x & 63;
      asm volatile("" : "+v"(lane));  // (what follows from it is formed again for every tile: kept from one to the next, it takes registers from the loop)
      const int lq = lane & 31, h = lane >> 5;
      const int kv = hh / a.subs, head0 = kv * a.group + (hh - kv * a.subs) * a.sub_group;
      const int head_end = (kv + 1) * a.group;
      const unsigned char* head_base = a.cache + (int64_t)kv * a.c.block_bytes();
      const int32_t* blocks = a.table + (int64_t)s * a.max_blocks;
      const int last_block = max(q.len - 1, 0) >> log_page;

      // ---- the lane's query row ----
      const int r = wave * 32 + lq, r_tok = a.div_heads.div(r), r_head = head0 + (r - r_tok * a.sub_group);
      const bool valid = r_tok < tt && t * tt + r_tok < q.n && r_head < head_end;
      const int tok = t * tt + (valid ? r_tok : 0), head = valid ? r_head : head0;  // (a lane without a row repeats the tile's first)
      const int limit = q.held + tok + 1;  // tokens that it sees
      bf16x8 qreg[SPLIT][KS];
      {
        const int64_t at = (int64_t)(q.start + tok) * a.q.row + (int64_t)head * a.q.head;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
          const int j = 2 * ks + h, c = 32 * (j % G) + 8 * (j / G);  // piece j of a K row: word j of the token
          if constexpr (!F32) {
            qreg[0][ks] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4*>(reinterpret_cast<const uint16_t*>(a.Q) + at + c));
          } else {
            const f32x4* p = reinterpret_cast<const f32x4*>(reinterpret_cast<const float*>(a.Q) + at + c);
            const f32x4 x0 = p[0], x1 = p[1];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              float x = 0.5f * (i < 4 ? x0[i % 4] : x1[i % 4]);  // (at half: rounding the first part up leaves the largest finite)
#pragma unroll
              for (int z = 0; z < SPLIT; ++z) {
                qreg[z][ks][i] = (__bf16)x;
                x -= (float)qreg[z][ks][i];
              }
            }
          }
        }
      }

      // ---- codes into LDS ----
      auto find_page = [&](int step) { return blocks[min((step * kStep + 16 * part16) >> log_page, last_block)]; };
      auto there = [&](int page) { return (unsigned)page < (unsigned)a.c.n_pages; };
      auto base_of = [&](int page) { return head_base + (int64_t)(there(page) ? page : 0) * page_bytes; };
      auto load_k = [&](int step, int page, RawK<D>& k) {
        const unsigned char* b = base_of(page);
        const int at = ((step * kStep + 16 * part16) & in_page) + (lane >> 2);
        k.w = *reinterpret_cast<const decltype(k.w)*>(b + at * (D / 2) + (lane & 3) * (D / 8));
        if constexpr (D == 128) k.sc = *reinterpret_cast<const uint32_t*>(b + a.c.k_scale_at() + at * 4);
        else k.sc = *reinterpret_cast<const uint16_t*>(b + a.c.k_scale_at() + at * 2);
      };
      // V: a lane has a word (of D / 8) of four tokens (d = 64: of two)
      const int v_word = D == 128 ? lane & 15 : lane & 7;
      const int v_tok = D == 128 ? 4 * (lane >> 4) : 4 * ((lane >> 3) & 3) + 2 * (lane >> 5);  // the first of them
      constexpr int VT = D == 128 ? 4 : 2;
      auto load_v = [&](int step, int page, RawV<D>& v) {
        const unsigned char* b = base_of(page);
        const int at = (step * kStep + 16 * part16) & in_page;
        v.w = *reinterpret_cast<const decltype(v.w)*>(b + a.c.v_at() + ((at + v_tok) >> 2) * (D * 2) + v_word * 16 + (v_tok & 3) * 4);
        v.sc = *reinterpret_cast<const decltype(v.sc)*>(b + a.c.v_scale_at() + (at + v_tok) * G);
      };
      auto buf_at = [&](int kt) { return smem + (kt & 1) * L::BUF; };  // (kt: steps of this workgroup's, from 0)
      auto store_k = [&](int kt, int page, const RawK<D>& k) {
        unsigned char* to = buf_at(kt) + (16 * part16 + (lane >> 2)) * L::KSTR + (lane & 3) * (16 * G);
#pragma unroll
        for (int g = 0; g < G; ++g) {
          const float sc = scale_of(k.sc, g);
          *reinterpret_cast<u32x4*>(to + 16 * g) = (u32x4){two_values<0>(k.w[g], sc), two_values<1>(k.w[g], sc), two_values<2>(k.w[g], sc), two_values<3>(k.w[g], sc)};
        }
        reinterpret_cast<uint32_t*>(gone_flags + (kt & 1))[part16] = !there(page);  // (all lanes alike)
      };
      auto clean_v = [&](int kt, int page, RawV<D>& v) {  // what must not reach a product
        const int base = (first + kt) * kStep, tok0 = base + 16 * part16 + v_tok;
        if (!F32 && base + kStep <= all_see && there(page)) return;
        const bool here = there(page);
        uint32_t taken = 0;
#pragma unroll
        for (int i = 0; i < VT; ++i) {
          uint32_t sc;
          if constexpr (D == 128) sc = v.sc[i];
          else sc = (v.sc >> (16 * i)) & 0xffffu;
          if (!here || tok0 + i >= seen) {  // whatever lies there: weight 0 times a NaN would be NaN
            v.w[i] = 0;
            sc = 0;
          } else if (F32 || tok0 + i >= all_see) {
            // groups that are NaN or may lie past the largest number, of tokens that some rows see alone, are taken out here (fp32 queries: of all
            // tokens; an infinity times the parts of a weight, some of them 0 or negative, would be NaN)
            const uint32_t far = ((sc & 0x7f7f7f7fu) + (256 - kFarScale) * 0x01010101u) & sc & 0x80808080u;  // the top bit of every byte from kFarScale on
            sc &= ~((far << 1) - (far >> 7));
            taken |= far;
          }
          if constexpr (D == 128) v.sc[i] = sc;
          else v.sc = i == 0 ? (v.sc & 0xffff0000u) | sc : (v.sc & 0xffffu) | sc << 16;
        }
        if (taken) *far_flag = 1;
      };
      auto store_v = [&](int kt, const RawV<D>& v) {
        unsigned char* to = buf_at(kt) + L::K_BYTES + (16 * part16 + v_tok) * L::VSTR + v_word * 16;
#pragma unroll
        for (int i = 0; i < VT; ++i) {
          u32x4 x;
          if constexpr (D == 128) {
            x = (u32x4){two_values<0>(v.w[i], scale_of(v.sc[i], 0)), two_values<1>(v.w[i], scale_of(v.sc[i], 1)),
                        two_values<2>(v.w[i], scale_of(v.sc[i], 2)), two_values<3>(v.w[i], scale_of(v.sc[i], 3))};
          } else {
            const float s0 = scale_of(v.sc, 2 * i), s1 = scale_of(v.sc, 2 * i + 1);
            x = (u32x4){two_values<0>(v.w[i], s0), two_values<1>(v.w[i], s0), two_values<2>(v.w[i], s1), two_values<3>(v.w[i], s1)};
          }
          *reinterpret_cast<u32x4*>(to + i * L::VSTR) = x;
        }
      };

      // ---- state ----
      f32x16 o[DT];
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[dt][i] = 0.f;
      // reference of the exponentials, moved (and the sums rescaled) where a row's scores exceed it by more than 8; log2 domain for bf16
      // queries, natural for fp32 ones; l: this lane's share of the row sum
      float m = -INFINITY, l = 0.f;
      constexpr float unit_of = F32 ? 2.f : kLog2e;
      const int vtr_off = ((lane & 15) >> 2) * L::VSTR + ((lane & 3) * 4 + ((lane >> 4) & 1) * 16) * 2 + (4 * h) * L::VSTR;

      auto mask = [&](f32x16& c, int kt, int sub, uint32_t gone) {
        const int base = (first + kt) * kStep + 32 * sub;
        const int lim = limit - base - 4 * h;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int off = 8 * (i / 4) + i % 4;
          if (off >= lim || (gone >> (2 * sub + i / 8) & 1)) c[i] = -INFINITY;
        }
      };
      auto gone_of = [&](int kt) {  // quarters of a step that lie in pages that are not there
        const u32x4 f = gone_flags[kt & 1];
        return (uint32_t)__builtin_amdgcn_readfirstlane(f[0] | f[1] << 1 | f[2] << 2 | f[3] << 3);
      };
      auto values_at = [&](int kt, int j, int dt) {  // V^T of 16 tokens, 32 channels
        const unsigned char* vp = buf_at(kt) + L::K_BYTES + vtr_off + (16 * j) * L::VSTR + (32 * dt) * 2;
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_ptr)(vp));
        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_ptr)(vp + 8 * L::VSTR));
        return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
      };
      auto move_reference = [&](float mx) {
        const float m_new = fmaxf(m, fmaxf(mx, __shfl_xor(mx, 32))), ref = m_new == -INFINITY ? 0.f : m_new;
        const float alpha = F32 ? expf(m - ref) : __builtin_amdgcn_exp2f(m - ref);
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
          for (int i = 0; i < 16; ++i) o[dt][i] *= alpha;
        l *= alpha;
        m = m_new;
      };

      __syncthreads();  // (the tile before has left LDS)
      if (threadIdx.x == 0) *far_flag = 0;
      __syncthreads();

      // bf16 queries: step kt lays K of kt + 2 and V of kt + 1 into LDS, over K of kt and V of kt - 1, which all waves have left behind, and then asks for the codes that step
      // kt + 1 will lay out; fp32 queries have K no further than V.  Codes have a step to come, their pages' numbers two.  (Asked for earlier, they take 13 more registers,
      // and every reload of a spilled one waits for them: 2.8 us a step where few workgroups are the launch.  Past the end the last step comes again, and is not read.)
      const int ntiles = last - first;
      const bool live = __any(valid);  // (a wave without rows lays out its share of the tokens, no more)
      auto step_of = [&](int kt) { return first + min(kt, ntiles - 1); };
      RawK<D> k;
      RawV<D> v;
      int pages[4];  // of steps kt ... kt + 3
      int next_page = 0;
      auto request = [&](int kt) {
        pages[3] = __builtin_amdgcn_readfirstlane(next_page);
        next_page = find_page(step_of(kt + 4));
        if constexpr (!F32) load_k(step_of(kt + 3), pages[3], k);
        else load_k(step_of(kt + 2), pages[2], k);
        load_v(step_of(kt + 2), pages[2], v);
#pragma unroll
        for (int i = 0; i < 3; ++i) pages[i] = pages[i + 1];
      };
      auto lay_out = [&](auto parity) {  // (V is clean)
        constexpr int P = decltype(parity)::value;
        if constexpr (!F32) store_k(P, pages[2], k);
        else store_k(P ^ 1, pages[1], k);
        store_v(P ^ 1, v);
      };
      const auto even = std::integral_constant<int, 0>{};
      const auto odd = std::integral_constant<int, 1>{};
      if (ntiles > 0) {
#pragma unroll
        for (int i = 0; i < 3; ++i) pages[i] = find_page(step_of(i));
        next_page = find_page(step_of(3));
#pragma unroll
        for (int i = 0; i < 3; ++i) pages[i] = __builtin_amdgcn_readfirstlane(pages[i]);
        RawK<D> k0;
        RawV<D> v0;
        load_k(step_of(0), pages[0], k0);
        load_v(step_of(0), pages[0], v0);
        load_k(step_of(1), pages[1], k);
        load_v(step_of(1), pages[1], v);
        store_k(0, pages[0], k0);
        clean_v(0, pages[0], v0);
        store_v(0, v0);
        if constexpr (!F32) {
          store_k(1, pages[1], k);
          load_k(step_of(2), pages[2], k);
        }
      }
      __syncthreads();
      if (ntiles > 0 && !live) {
        if constexpr (!F32) __syncthreads();
        auto one = [&](int kt, auto parity) {
          if (kt + 1 < ntiles) {
            clean_v(kt + 1, pages[1], v);
            lay_out(parity);
            request(kt);
          }
          __syncthreads();
        };
        for (int kt = 0; kt < ntiles; kt += 2) {
          one(kt, even);
          if (kt + 1 < ntiles) one(kt + 1, odd);
        }
      } else if (ntiles > 0) {
        if constexpr (!F32) {
          // Scores of step kt + 1 on the matrix cores beside weights of step kt, P V of step kt beside row maxima of kt + 1 and codes on their way to LDS
          auto tile_max = [&](const f32x16 (&c)[2]) {
            float mx = fmaxf(c[0][0], c[1][0]);
#pragma unroll
            for (int i = 1; i < 16; ++i) mx = fmaxf(fmaxf(mx, c[0][i]), c[1][i]);
            return mx * kLog2e;
          };
          auto mask_step = [&](f32x16 (&c)[2], int kt) {
            const uint32_t gone = gone_of(kt);
            if ((first + kt) * kStep + kStep > all_see || gone) {
              mask(c[0], kt, 0, gone);
              mask(c[1], kt, 1, gone);
            }
          };
          f32x16 ca[2], cb[2];
          float t_max;
          {
#pragma unroll
            for (int sub = 0; sub < 2; ++sub) {
#pragma unroll
              for (int i = 0; i < 16; ++i) ca[sub][i] = 0.f;
              const unsigned char* kp = buf_at(0) + (32 * sub + lq) * L::KSTR + 16 * h;
#pragma unroll
              for (int j = 0; j < KS; ++j) ca[sub] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*reinterpret_cast<const bf16x8*>(kp + 32 * j), qreg[0][j], ca[sub], 0, 0, 0);
            }
            mask_step(ca, 0);
            t_max = tile_max(ca);
          }
          __syncthreads();  // (the loop's first step writes over K of step 0)
          auto body = [&](int kt, f32x16 (&c)[2], f32x16 (&cn)[2], auto parity, auto has_next) {
            constexpr int P = decltype(parity)::value;
            constexpr bool HN = decltype(has_next)::value;
            if (__any(t_max > m + 8.f)) move_reference(t_max);
            const float shift = m == -INFINITY ? 0.f : -m;
            bf16x8 pf[4];
            __builtin_amdgcn_s_setprio(1);
            {
              if constexpr (HN) {
#pragma unroll
                for (int sub = 0; sub < 2; ++sub)
#pragma unroll
                  for (int i = 0; i < 16; ++i) cn[sub][i] = 0.f;
                const unsigned char* kp0 = buf_at(P + 1) + lq * L::KSTR + 16 * h;
                const unsigned char* kp1 = kp0 + 32 * L::KSTR;
                bf16x8 kf[2 * KS];
#pragma unroll
                for (int j = 0; j < KS; ++j) {
                  kf[2 * j] = *reinterpret_cast<const bf16x8*>(kp0 + 32 * j);
                  kf[2 * j + 1] = *reinterpret_cast<const bf16x8*>(kp1 + 32 * j);
                }
#pragma unroll
                for (int j = 0; j < KS; ++j) {
                  cn[0] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[2 * j], qreg[0][j], cn[0], 0, 0, 0);
                  cn[1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[2 * j + 1], qreg[0][j], cn[1], 0, 0, 0);
                }
              }
              float ls[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
              for (int j = 0; j < 4; ++j) {
                u32x4 pk;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                  const float p0 = __builtin_amdgcn_exp2f(__builtin_fmaf(c[j / 2][8 * (j % 2) + 2 * e], kLog2e, shift));
                  const float p1 = __builtin_amdgcn_exp2f(__builtin_fmaf(c[j / 2][8 * (j % 2) + 2 * e + 1], kLog2e, shift));
                  ls[e] += p0 + p1;
                  pk[e] = pack_bf16x2(p0, p1);
                }
                pf[j] = __builtin_bit_cast(bf16x8, pk);
              }
              l += (ls[0] + ls[1]) + (ls[2] + ls[3]);
#pragma unroll
              for (int j = 0; j < 4; ++j) asm volatile("" : "+v"(pf[j]));  // (the weights stay in this block, beside its products)
              asm volatile("" : "+v"(l));
              if constexpr (HN) {
                constexpr int kPre = 4, kValu = KS == 8 ? 5 : 18;
                __builtin_amdgcn_sched_group_barrier(0x100, kPre, 0);
#pragma unroll
                for (int j = 0; j < 2 * KS; ++j) {
                  __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                  if (j < 2 * KS - kPre) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
                  __builtin_amdgcn_sched_group_barrier(0x002, kValu, 0);
                }
              }
            }
            __builtin_amdgcn_s_setprio(0);
            if constexpr (HN) {
              mask_step(cn, kt + 1);
              clean_v(kt + 1, pages[1], v);
            }
            {
#pragma unroll
              for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int dt = 0; dt < DT; ++dt) o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(values_at(P, j, dt), pf[j], o[dt], 0, 0, 0);
              if constexpr (HN) {
                t_max = tile_max(cn);
                lay_out(parity);
              }
              constexpr int kPreV = 8;
              __builtin_amdgcn_sched_group_barrier(0x100, kPreV, 0);
#pragma unroll
              for (int j = 0; j < 4 * DT; ++j) {
                __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                if (2 * j < 8 * DT - kPreV) __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
                if constexpr (HN) __builtin_amdgcn_sched_group_barrier(0x002, 6, 0);
              }
            }
            if constexpr (HN) request(kt);
            __syncthreads();
          };
          int kt = 0;
          for (; kt + 2 < ntiles; kt += 2) {
            body(kt, ca, cb, even, std::true_type{});
            body(kt + 1, cb, ca, odd, std::true_type{});
          }
          if (kt + 2 == ntiles) {
            body(kt, ca, cb, even, std::true_type{});
            body(kt + 1, cb, ca, odd, std::false_type{});
          } else {
            body(kt, ca, cb, even, std::false_type{});
          }
        } else {
          // fp32 queries: one step after the other, 32 tokens at a time (three parts of queries and weights leave no registers for more)
          auto body = [&](int kt, auto parity) {
            constexpr int P = decltype(parity)::value;
            const bool more = kt + 1 < ntiles;
            const uint32_t gone = gone_of(P);
#pragma unroll
            for (int sub = 0; sub < 2; ++sub) {
              f32x16 c;
#pragma unroll
              for (int i = 0; i < 16; ++i) c[i] = 0.f;
              const unsigned char* kp = buf_at(P) + (32 * sub + lq) * L::KSTR + 16 * h;
#pragma unroll
              for (int j = 0; j < KS; ++j) {
                const bf16x8 kf = *reinterpret_cast<const bf16x8*>(kp + 32 * j);
#pragma unroll
                for (int z = SPLIT - 1; z >= 0; --z) c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, qreg[z][j], c, 0, 0, 0);
              }
              if ((first + kt) * kStep + 32 * sub + 32 > all_see || gone) mask(c, kt, sub, gone);
              float mx = c[0];
#pragma unroll
              for (int i = 1; i < 16; ++i) mx = fmaxf(mx, c[i]);
              mx *= unit_of;
              if (__any(mx > m + 5.5f)) move_reference(mx);
              const float ref = m == -INFINITY ? 0.f : m;
#pragma unroll
              for (int jj = 0; jj < 2; ++jj) {
                u32x4 w[SPLIT];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                  float x0 = exp_split(__builtin_fmaf(c[8 * jj + 2 * e], unit_of, -ref)), x1 = exp_split(__builtin_fmaf(c[8 * jj + 2 * e + 1], unit_of, -ref));
                  l += x0 + x1;
#pragma unroll
                  for (int z = 0; z < SPLIT; ++z) {
                    w[z][e] = pack_bf16x2(x0, x1);
                    if (z + 1 < SPLIT) {
                      x0 -= __uint_as_float(w[z][e] << 16);
                      x1 -= __uint_as_float(w[z][e] & 0xffff0000u);
                    }
                  }
                }
#pragma unroll
                for (int dt = 0; dt < DT; ++dt) {
                  const bf16x8 vf = values_at(P, 2 * sub + jj, dt);
#pragma unroll
                  for (int z = SPLIT - 1; z >= 0; --z) o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, __builtin_bit_cast(bf16x8, w[z]), o[dt], 0, 0, 0);
                }
              }
            }
            if (more) {
              clean_v(kt + 1, pages[1], v);
              lay_out(parity);
              request(kt);
            }
            __syncthreads();
          };
          for (int kt = 0; kt < ntiles; kt += 2) {
            body(kt, even);
            if (kt + 1 < ntiles) body(kt + 1, odd);
          }
        }
      }

      // ---- groups that were taken out, for the rows that see them (rare) ----
      if (*far_flag) {
        for (int x = F32 ? first * kStep : max(first * kStep, max(all_see, 0)); x < min(last * kStep, seen); ++x) {
          const int page = blocks[x >> log_page], at = x & in_page;
          if (!there(page)) continue;
          const unsigned char* b = base_of(page);
          const unsigned char* k_scales = b + a.c.k_scale_at() + at * G;
          const unsigned char* v_scales = b + a.c.v_scale_at() + at * G;
          bool any = false;
#pragma unroll
          for (int g = 0; g < G; ++g) any = any || v_scales[g] >= kFarScale;
          if (!any) continue;
          float score = 0.f;
#pragma unroll
          for (int ks = 0; ks < KS; ++ks) {
            const int j = 2 * ks + h;
            const uint32_t w = *reinterpret_cast<const uint32_t*>(b + at * (D / 2) + 4 * j);
            const float sc = __uint_as_float((uint32_t)k_scales[j % G] << 23);
            const f32x2 k01 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, sc, 0), k23 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, sc, 1);
            const f32x2 k45 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, sc, 2), k67 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, sc, 3);
            const float kk[8] = {k01[0], k01[1], k23[0], k23[1], k45[0], k45[1], k67[0], k67[1]};
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              float x = 0.f;
#pragma unroll
              for (int z = SPLIT - 1; z >= 0; --z) x += (float)qreg[z][ks][i];
              score = __builtin_fmaf(F32 ? 2.f * x : x, kk[i], score);
            }
          }
          score += __shfl_xor(score, 32);
          const float ref = m == -INFINITY ? 0.f : m;
          const float weight = F32 ? expf(score - ref) : (float)(__bf16)__builtin_amdgcn_exp2f(__builtin_fmaf(score, kLog2e, -ref));
          if (x < limit) {
#pragma unroll
            for (int dt = 0; dt < DT; ++dt)
#pragma unroll
              for (int i = 0; i < 16; i += 2) {  // word 4 dt + i / 4, byte 2 h + i % 4 / 2
                const int byte = 2 * h + i % 4 / 2, g = D == 128 ? byte : byte / 2;
                if (v_scales[g] < kFarScale) continue;
                const uint32_t w = *reinterpret_cast<const uint32_t*>(b + a.c.v_at() + (at >> 2) * (D * 2) + (4 * dt + i / 4) * 16 + (at & 3) * 4) >> (8 * byte);
                const f32x2 v = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, __uint_as_float((uint32_t)v_scales[g] << 23), 0);
                o[dt][i] = __builtin_fmaf(weight, v[0], o[dt][i]);
                o[dt][i + 1] = __builtin_fmaf(weight, v[1], o[dt][i + 1]);
              }
          }
        }
      }

      // ---- out: rows through LDS, channels in their order ----
      __syncthreads();  // (far_flag has been read, tiles too)
      const bool whole = WHOLE || (first == 0 && last == nsteps);
      l += __shfl_xor(l, 32);
      const bool empty = l == 0.f;
      if (whole) {
        const float inv = empty ? 0.f : 1.f / l;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
          for (int i = 0; i < 16; ++i) o[dt][i] *= inv;
      }
      unsigned char* ep = smem + wave * L::WAVE;
      int64_t* ep_rows = reinterpret_cast<int64_t*>(ep + 32 * L::ROW);
      const int64_t slot = WHOLE ? 0 : 2 * (int64_t)part + (tile_first >= u0);
      if (h == 0) {
        ep_rows[lq] = !valid ? -1 : whole ? (int64_t)(q.start + tok) * a.o.row + (int64_t)head * a.o.head : (slot * QT + r) * D;
        if (valid) {
          if (whole) {
            a.lse[(int64_t)head * a.rows + q.start + tok] = empty ? -INFINITY : F32 ? m + logf(l) : (m + log2f(l)) * kLn2;
          } else {
            a.part_ml[2 * (slot * QT + r)] = m;
            a.part_ml[2 * (slot * QT + r) + 1] = l;
          }
        }
      }
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int g4 = 0; g4 < 4; ++g4) {
          const int word = 4 * dt + g4;
          unsigned char* to = ep + lq * L::ROW;
          if constexpr (D == 128) {
            *reinterpret_cast<f32x2*>(to + (64 * h + 2 * word) * 4) = (f32x2){o[dt][4 * g4], o[dt][4 * g4 + 1]};
            *reinterpret_cast<f32x2*>(to + (64 * h + 32 + 2 * word) * 4) = (f32x2){o[dt][4 * g4 + 2], o[dt][4 * g4 + 3]};
          } else {
            *reinterpret_cast<f32x4*>(to + (32 * h + 4 * word) * 4) = (f32x4){o[dt][4 * g4], o[dt][4 * g4 + 1], o[dt][4 * g4 + 2], o[dt][4 * g4 + 3]};
          }
        }
      __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
      __builtin_amdgcn_wave_barrier();
      __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
      constexpr int CH = D / 8;  // pieces of eight channels
#pragma unroll
      for (int it = 0; it < 32 * CH / 64; ++it) {
        const int idx = lane + 64 * it, row = idx / CH, ch = idx % CH * 8;
        const int64_t at = ep_rows[row];
        const f32x4 x0 = *reinterpret_cast<const f32x4*>(ep + row * L::ROW + ch * 4), x1 = *reinterpret_cast<const f32x4*>(ep + row * L::ROW + ch * 4 + 16);
        if (at < 0) continue;
        if (!whole || F32) {
          f32x4* to = reinterpret_cast<f32x4*>((whole ? reinterpret_cast<float*>(a.out) : a.part_o) + at + ch);
          to[0] = x0;
          to[1] = x1;
        } else {
          *reinterpret_cast<u32x4*>(reinterpret_cast<uint16_t*>(a.out) + at + ch) =
              (u32x4){pack_bf16x2(x0[0], x0[1]), pack_bf16x2(x0[2], x0[3]), pack_bf16x2(x1[0], x1[1]), pack_bf16x2(x1[2], x1[3])};
        }
      }
      if (!WHOLE && first > 0 && threadIdx.x == 0) {  // others began the tile: the second launch joins it
        int32_t* j = a.joins + 8 * part;
        j[1] = head0;
        j[2] = q.start + t * tt;
        j[3] = min(q.n - t * tt, tt);
        j[4] = head_end - head0;
        j[5] = run_of(total, parts, tile_first + (int64_t)(nsteps - 1) * kStep);  // that has the last step
        j[0] = run_of(total, parts, tile_first);
      }
    }
    if constexpr (WHOLE) return;
    tile_first += length;
    if (tile_first >= u1) return;
    if (++t == T) {
      t = 0;
      if (++hh == heads) {
        hh = 0;
        do {
          if (++s >= a.n_seq) return;
          q = uniform_seq(chunk_seq(a, s));
          T = tiles_of(q);
        } while (T == 0);
      }
    }
  }
}

// Tiles of many rows and sequences of few in one launch.  WHOLE: the first workgroups have a tile each, the others a sequence and key head.  Else every workgroup has a run of
// both lines, the few rows' last, from the last workgroup on, which has the least of the others.  (64 sequences, most of one token, 24 of up to 200, 16 of up to 1024: half of the
// workgroups begin with the few rows 212 / 49 / 107 us, none 205 / 47 / 101.)
template <int D, int SPLIT, int NW, bool WHOLE>
__global__ __launch_bounds__(64 * NW, 2) void cache4_chunk_kernel(CacheChunkArgs a, CacheAttnArgs n) {
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  auto few = [&](int x, int y) {
    cache4_attn_run<D, SPLIT, NW, WHOLE, false, true, true>(n, *reinterpret_cast<CacheAttnLds<D, NW>*>(smem), x, y);
  };
  if constexpr (WHOLE) {
    const int i = (int)blockIdx.x - a.tiles;
    if (i < 0) cache4_chunk_run<D, SPLIT, NW, true>(a, smem, blockIdx.x);
    else few(i / a.c.Hk, i % a.c.Hk);
    return;
  }
  if ((int)blockIdx.x < a.parts) cache4_chunk_run<D, SPLIT, NW, false>(a, smem, blockIdx.x);
  const int last = gridDim.x - 1 - blockIdx.x;
  if (last < n.parts * a.c.Hk) {
    __syncthreads();
    few(last / a.c.Hk, last % a.c.Hk);
  }
}

// Joins the sums of tiles that a cut divides, D / 4 threads a row.  Of the runs p0 ... p1 that share a tile those behind the first have kJoinWgs workgroups each for its
// rows: a tile of few runs has several rows a thread, in turn, a tile of many (few rows behind a long sequence) a row of some threads, and pieces in flight.
constexpr int kJoinWgs = 4;
template <int D, int SPLIT, int NW>
__device__ __forceinline__ void cache4_chunk_join(const CacheChunkArgs& a, int p, int block) {
  constexpr bool F32 = SPLIT > 1;
  constexpr int LPR = D / 4, ROWS = kJoinThreads / LPR, QT = 32 * NW, GROUPS = QT / ROWS;
  const int32_t* j = a.joins + 8 * p;
  const int p0 = j[0], head0 = j[1], row0 = j[2], tokens = j[3], heads = min(j[4], a.sub_group), p1 = j[5];
  if (p0 < 0) return;
  const int ch = threadIdx.x % LPR * 4;
  auto exp_of = [](float x) { return F32 ? expf(x) : __builtin_amdgcn_exp2f(x); };
  auto join = [&](auto rows_tag, auto ahead_tag, int first_group, int step) {  // rows of groups first_group, first_group + step, ...
    constexpr int U = decltype(rows_tag)::value, Z = decltype(ahead_tag)::value;
    float m[U], l[U];
    f32x4 acc[U];
    int r[U], tok[U], head[U];
    bool live[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      r[u] = (first_group + u * step) * ROWS + threadIdx.x / LPR;
      tok[u] = a.div_heads.div(r[u]);
      head[u] = r[u] - tok[u] * a.sub_group;
      live[u] = tok[u] < tokens && head[u] < heads;
      m[u] = -INFINITY;
      l[u] = 0.f;
      acc[u] = (f32x4){0.f, 0.f, 0.f, 0.f};
    }
    for (int q = p0; q <= p1; q += Z) {
      float pm[Z][U], pl[Z][U];
      f32x4 v[Z][U];
#pragma unroll
      for (int z = 0; z < Z; ++z)
#pragma unroll
        for (int u = 0; u < U; ++u) {  // (past the last the last again, which counts once)
          const int qq = min(q + z, p1);
          const int64_t row = (2 * (int64_t)qq + (qq == p0)) * QT + (live[u] ? r[u] : 0);
          pm[z][u] = a.part_ml[2 * row];
          pl[z][u] = a.part_ml[2 * row + 1];
          v[z][u] = *reinterpret_cast<const f32x4*>(a.part_o + row * D + ch);
        }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        float top = m[u];
#pragma unroll
        for (int z = 0; z < Z; ++z) top = fmaxf(top, pm[z][u]);
        const float ref = top == -INFINITY ? 0.f : top, w0 = exp_of(m[u] - ref);
        acc[u] *= w0;
        l[u] *= w0;
#pragma unroll
        for (int z = 0; z < Z; ++z) {
          if (q + z > p1) break;
          const float w = exp_of(pm[z][u] - ref);
          acc[u] += w * v[z][u];
          l[u] += w * pl[z][u];
        }
        m[u] = top;
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (!live[u]) continue;
      const bool empty = l[u] == 0.f;
      acc[u] *= empty ? 0.f : 1.f / l[u];
      const int64_t row = row0 + tok[u], hq = head0 + head[u], at = row * a.o.row + hq * a.o.head + ch;
      if constexpr (F32) *reinterpret_cast<f32x4*>(reinterpret_cast<float*>(a.out) + at) = acc[u];
      else *reinterpret_cast<u32x2*>(reinterpret_cast<uint16_t*>(a.out) + at) = (u32x2){pack_bf16x2(acc[u][0], acc[u][1]), pack_bf16x2(acc[u][2], acc[u][3])};
      if (ch == 0) a.lse[hq * a.rows + row] = empty ? -INFINITY : F32 ? m[u] + logf(l[u]) : (m[u] + log2f(l[u])) * kLn2;
    }
  };
  const int helpers = (p1 - p0) * kJoinWgs, me = (p - p0 - 1) * kJoinWgs + block;
  if (helpers < GROUPS) {
    constexpr int U = GROUPS / kJoinWgs;
    if (p == p1) join(std::integral_constant<int, U>{}, std::integral_constant<int, 2>{}, block, kJoinWgs);
  } else if (me < GROUPS) {
    join(std::integral_constant<int, 1>{}, std::integral_constant<int, 8>{}, me, 0);
  }
}

// Tables of few tokens: a workgroup per tile, and no second launch (shared out -> a workgroup per tile: 64 sequences of 20 new behind up to 900, 32 and 8 heads, 50 -> 36 us, 60 of one and 4 of
// 300 behind up to 700 51 -> 28, 17 behind 300 14.7 -> 10.2, a prompt of 1000 42 -> 30, but 60 behind 900, 8 and 2 heads, 23 -> 26; up to 2048 tokens: 60 behind 1800 23 -> 44, fp32 28 -> 74,
// 32 of 60 behind up to 1800 72 -> 61).  Sequences whose rows of a key head fit 16 are read with the waves of a workgroup on different tokens (cache4_attn.h), where there can be several (64
// that decode behind up to 16384 230 -> 127, 56 of them beside 8 pieces of prompts 605 -> 483, 60 beside 4 in short tables 40 -> 28, three, two of which decode behind 16000, 43 -> 28; of one and 300
// 49.6 -> 49.0; where none has so few: 100 and 50 34.3 -> 35.4, fp32, six of up to 150, 27.3 -> 28.3).
void cache4_chunk_split(CacheChunkArgs* a, CacheAttnArgs* narrow) {
  a->subs = (a->group + kChunkRows - 1) / kChunkRows;
  a->sub_group = (a->group + a->subs - 1) / a->subs;
  a->tile_tokens = kChunkRows / a->sub_group;
  a->div_tokens = make_fast_div(a->tile_tokens);
  a->div_heads = make_fast_div(a->sub_group);
  a->narrow = a->group <= kNarrowRows && (a->n_seq >= 2 || (int64_t)a->rows * a->group <= kNarrowRows) ? kNarrowRows : 0;
  narrow->parts = a->narrow ? (a->c.Hk < kChunkParts ? kChunkParts / a->c.Hk : 1) : 0;
  const int64_t tokens = (int64_t)a->max_blocks << a->c.log_page, heads = (int64_t)a->c.Hk * a->subs;
  const int64_t tiles = ((int64_t)a->rows / a->tile_tokens + a->n_seq) * heads;
  if (tokens <= 1024 && tiles + heads * a->n_seq <= kMaxLaunch) {
    a->tiles = (int32_t)tiles;
    a->parts = 0;
    return;
  }
  const int64_t runs = tiles * (tokens + kTileCost) / kLeastRun;
  a->parts = (int32_t)(runs < 1 ? 1 : runs > kChunkParts ? kChunkParts : runs);
}

// Both kinds' joins
template <int D, int SPLIT, int NW>
__global__ __launch_bounds__(kJoinThreads) void cache4_chunk_join_kernel(CacheChunkArgs a, CacheAttnArgs n, int wide, int each) {
  __shared__ CacheJoinLds<D, SPLIT> lds;
  constexpr int PER = kJoinWgs;
  const int i = (int)blockIdx.x - wide;
  if (i < 0) cache4_chunk_join<D, SPLIT, NW>(a, blockIdx.x / PER, blockIdx.x % PER);
  else cache4_join_run<D, SPLIT, true>(n, lds, i / each, i % each, 0);
}

template <int D, int SPLIT, int NW>
static int launch_chunk_one(const CacheChunkArgs& args, const CacheAttnArgs& few, hipStream_t st) {
  constexpr size_t chunk_lds = ChunkLds<D>::bytes(NW), few_lds = sizeof(CacheAttnLds<D, NW>), lds = chunk_lds > few_lds ? chunk_lds : few_lds;
  static std::atomic<uint64_t> set_whole{0}, set_parts{0};
  const CacheChunkArgs& a = args;
  const CacheAttnArgs& n = few;
  if (a.parts == 0) {
    const auto kernel = &cache4_chunk_kernel<D, SPLIT, NW, true>;
    const int rc = allow_full_lds(reinterpret_cast<const void*>(kernel), set_whole);
    if (rc != HA_OK) return rc;
    hipLaunchKernelGGL(kernel, dim3((unsigned)(a.tiles + (a.narrow ? a.n_seq * a.c.Hk : 0))), dim3(64 * NW), lds, st, a, n);
    return check_launch();
  }
  const auto kernel = &cache4_chunk_kernel<D, SPLIT, NW, false>;
  int rc = allow_full_lds(reinterpret_cast<const void*>(kernel), set_parts);
  if (rc != HA_OK) return rc;
  const int few_runs = n.parts * a.c.Hk, grid = few_runs > a.parts ? few_runs : a.parts;
  hipLaunchKernelGGL(kernel, dim3((unsigned)grid), dim3(64 * NW), lds, st, a, n);
  rc = check_launch();
  if (rc != HA_OK) return rc;
  constexpr int PAR = kJoinThreads / (D / 4);
  const int wide = a.parts * kJoinWgs, each = a.c.Hk * (kNarrowRows / PAR);
  hipLaunchKernelGGL((cache4_chunk_join_kernel<D, SPLIT, NW>), dim3((unsigned)(wide + (a.narrow ? a.n_seq * each : 0))), dim3(kJoinThreads), 0, st, a, n, wide, each);
  return check_launch();
}

int launch_cache4_chunk(const CacheChunkArgs& a, const CacheAttnArgs& n, int dtype, hipStream_t st) {
  if (a.c.d == 128) return dtype == HA_BF16 ? launch_chunk_one<128, 1, 4>(a, n, st) : launch_chunk_one<128, 3, 4>(a, n, st);
  return dtype == HA_BF16 ? launch_chunk_one<64, 1, 4>(a, n, st) : launch_chunk_one<64, 3, 4>(a, n, st);
}

}  // namespace ha
