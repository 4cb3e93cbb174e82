// Rows of K and V into the 4-bit cache and back (format: include/hyperattn.h).
//
// A thread holds eight channels of one row of one head: a quarter of a group of 32, whose largest magnitude comes by two lane exchanges, and one
// 32-bit word of K codes.  With |x| <= m = 1.f 2^k the smallest power of two s with m <= 6 s is 2^(k - 2) where 1.f <= 1.5 and 2^(k - 1)
// above: two integer operations on m's bits.  Dividing by s is exact, and the conversion (v_cvt_scalef32_pk_fp4_*, two numbers an instruction) rounds to
// the nearest code, ties to even, and ends at 6: checked on the card against the seven half-way points, at scales from 2^-125 to 2^100.
// V's words hold channels that lie 32 apart, so their bytes change places among the lanes of a row, by exchanges too.
//
// Bound by memory: rows in (16 or 32 bytes a thread, a row of a head at a time), 17/32 byte a value out.  16411 rows of 8 heads, d = 128, bf16 (MI355X; a copy
// moves 4.75 TB/s): into consecutive slots 18.6 us, 4.6 TB/s, from them 13.3 us, 6.4 TB/s; slots in random order, where a row's V takes a quarter of the bytes of
// two lines, 25.4 and 21.4 us.  (Four heads a thread: 17.6, 14.1; 27.4, 21.4.)  fp32 rows: two pieces of 16 bytes a thread, which only meet in a
// cache: past the caches the read took 65 us, now 32.
#include "cache4_common.h"

namespace ha {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

constexpr int kRowsThreads = 256;

// Eight numbers as two halves of 16 bytes each, bf16 in the first alone
template <bool F32>
struct Eight {
  u32x4 w[F32 ? 2 : 1];
};

template <bool F32>
__device__ inline Eight<F32> load_eight(const void* base, int64_t elem) {
  Eight<F32> x;
  const u32x4* p = reinterpret_cast<const u32x4*>(reinterpret_cast<const unsigned char*>(base) + elem * (F32 ? 4 : 2));
  if constexpr (F32) {
    x.w[0] = p[0];
    x.w[1] = p[1];
  } else {
    x.w[0] = __builtin_nontemporal_load(p);
  }
  return x;
}

template <bool F32>
__device__ inline void store_eight(void* base, int64_t elem, const Eight<F32>& x) {
  u32x4* p = reinterpret_cast<u32x4*>(reinterpret_cast<unsigned char*>(base) + elem * (F32 ? 4 : 2));
  if constexpr (F32) {
    p[0] = x.w[0];
    p[1] = x.w[1];
  } else {
    __builtin_nontemporal_store(x.w[0], p);
  }
}

// Bits of the largest magnitude as a float's
template <bool F32>
__device__ inline uint32_t largest_bits(const Eight<F32>& x) {
  uint32_t m = 0;
  if constexpr (F32) {
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, x.w[i / 4][i % 4] & 0x7fffffffu);
    return m;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) m = max(max(m, x.w[0][i] & 0x7fff0000u), (x.w[0][i] << 16) & 0x7fff0000u);
  return m;
}

// The group's scale byte, from the largest of its 32 magnitudes; 255 where that is an infinity or NaN
__device__ inline uint32_t scale_byte(uint32_t m) {
  if (m >= 0x7f800000u) return 255u;
  const int e = (int)(m >> 23) - 2 + ((m & 0x7fffffu) > 0x400000u ? 1 : 0);
  return (uint32_t)min(max(e, kLeastScale), kLargestScale);
}

__device__ inline float scale_of(uint32_t byte) { return __uint_as_float(byte << 23); }

// Codes of eight numbers, number i in nibble i
template <bool F32>
__device__ inline uint32_t codes_of(const Eight<F32>& x, float s) {
  uint32_t w = 0;
  if constexpr (F32) {
    auto f = [&](int i) { return __uint_as_float(x.w[i / 4][i % 4]); };
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, f(0), f(1), s, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, f(2), f(3), s, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, f(4), f(5), s, 2);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, f(6), f(7), s, 3);
  } else {
    auto f = [&](int i) { return __builtin_bit_cast(bf16x2, (uint32_t)x.w[0][i]); };
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, f(0), s, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, f(1), s, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, f(2), s, 2);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, f(3), s, 3);
  }
  return w;
}

// What the codes stand for.  The conversion's scale operand counts by its exponent alone, 255 in it makes NaN, 0 is 2^-127 (checked on the card
// for all bytes and codes).  (bf16: exact down to 2^-133; scales of foreign writers below 2^-126 round.)
template <bool F32>
__device__ inline Eight<F32> values_of(uint32_t w, uint32_t byte) {
  Eight<F32> x;
  const float s = scale_of(byte);
  if constexpr (F32) {
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    const f32x2 p[4] = {__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, s, 0), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, s, 1),
                        __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, s, 2), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, s, 3)};
#pragma unroll
    for (int i = 0; i < 8; ++i) x.w[i / 4][i % 4] = __float_as_uint(p[i / 2][i % 2]);
  } else {
    x.w[0][0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 0));
    x.w[0][1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 1));
    x.w[0][2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 2));
    x.w[0][3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 3));
  }
  return x;
}

// The lanes of a row: lane t of D / 8 holds channels 8 t ... + 7: group t / 4, pairs m = 4 (t % 4) ... + 3.
// V's bytes between the lanes' own order (byte j: pair 4 (t % 4) + j of group t / 4) and the words' order; its own inverse.
//   d = 128: the lane ends with word 4 (t % 4) + t / 4, whose byte g is pair 4 (t % 4) + t / 4 of group g: a 4 x 4 transpose over t / 4
//   d = 64: word 2 (t % 4) + t / 4, bytes 2 g + z: pair 4 (t % 4) + 2 (t / 4) + z of group g: 2 x 2, of halves
template <int D>
__device__ inline uint32_t swap_v_bytes(uint32_t w, int t) {
  if constexpr (D == 64) {
    const uint32_t other = __shfl_xor(w, 4);
    return t & 4 ? (w & 0xffff0000u) | (other >> 16) : (w & 0xffffu) | (other << 16);
  } else {
    uint32_t other = __shfl_xor(w, 8);   // halves over bit 1 of t / 4
    w = t & 8 ? (w & 0xffff0000u) | (other >> 16) : (w & 0xffffu) | (other << 16);
    other = __shfl_xor(w, 4);            // bytes within the halves over bit 0
    return t & 4 ? (w & 0xff00ff00u) | ((other >> 8) & 0x00ff00ffu) : (w & 0x00ff00ffu) | ((other << 8) & 0xff00ff00u);
  }
}

template <int D>
struct RowPlace {
  int row, head, t;
  int64_t block;   // byte of the page's block of the head
  int token;       // within the page
  bool live;
};

template <int D>
__device__ inline RowPlace<D> row_place(const CacheRowsArgs& a) {
  constexpr int LPR = D / 8;
  RowPlace<D> p;
  p.row = blockIdx.x * (kRowsThreads / LPR) + threadIdx.x / LPR;
  p.head = blockIdx.y;
  p.t = threadIdx.x % LPR;
  const int slot = p.row < a.rows ? a.slots[p.row] : -1;
  const int page = slot >> a.c.log_page;
  p.live = p.row < a.rows && slot >= 0 && page < a.c.n_pages;
  p.token = slot & (a.c.page - 1);
  p.block = p.live ? ((int64_t)page * a.c.Hk + p.head) * a.c.block_bytes() : 0;
  return p;
}

template <int D>
__device__ inline int k_word_at(const RowPlace<D>& p) { return p.token * (D / 2) + ((p.t & 3) * (D / 32) + (p.t >> 2)) * 4; }
template <int D>
__device__ inline int v_word_at(const RowPlace<D>& p) {  // of the word that swap_v_bytes leaves the lane
  const int word = (D == 128 ? 4 : 2) * (p.t & 3) + (p.t >> 2);
  return (p.token >> 2) * (D * 2) + word * 16 + (p.token & 3) * 4;
}

template <int D, bool F32>
__global__ __launch_bounds__(kRowsThreads) void cache4_write_kernel(CacheRowsArgs a) {
  const RowPlace<D> p = row_place<D>(a);
  const int row = p.live ? p.row : 0;  // (a row that is left out keeps its lanes for the exchanges)
  const Eight<F32> k = load_eight<F32>(a.K, row * a.k.row + p.head * a.k.head + 8 * p.t);
  const Eight<F32> v = load_eight<F32>(a.V, row * a.v.row + p.head * a.v.head + 8 * p.t);
  auto quantise = [&](const Eight<F32>& x, uint32_t* byte) {
    uint32_t m = largest_bits(x);
    m = max(m, (uint32_t)__shfl_xor(m, 1));
    m = max(m, (uint32_t)__shfl_xor(m, 2));
    *byte = scale_byte(m);
    return codes_of(x, scale_of(*byte));
  };
  auto all_bytes = [&](uint32_t byte) {  // the row's scales, group g in byte g
    uint32_t b = byte << (8 * (p.t >> 2));
    b |= __shfl_xor(b, 4);
    if (D == 128) b |= __shfl_xor(b, 8);
    return b;
  };
  uint32_t kb, vb;
  const uint32_t kw = quantise(k, &kb);
  const uint32_t vw = swap_v_bytes<D>(quantise(v, &vb), p.t);
  const uint32_t ks = all_bytes(kb), vs = all_bytes(vb);
  if (!p.live) return;
  unsigned char* block = a.cache + p.block;
  *reinterpret_cast<uint32_t*>(block + k_word_at(p)) = kw;
  *reinterpret_cast<uint32_t*>(block + a.c.v_at() + v_word_at(p)) = vw;
  if (p.t < 2) {
    unsigned char* at = block + (p.t == 0 ? a.c.k_scale_at() : a.c.v_scale_at()) + p.token * (D / 32);
    const uint32_t s = p.t == 0 ? ks : vs;
    if (D == 128) *reinterpret_cast<uint32_t*>(at) = s;
    else *reinterpret_cast<uint16_t*>(at) = (uint16_t)s;
  }
}

template <int D, bool F32>
__global__ __launch_bounds__(kRowsThreads) void cache4_read_kernel(CacheRowsArgs a) {
  const RowPlace<D> p = row_place<D>(a);
  Eight<F32> k{}, v{};
  uint32_t kw = 0, vw = 0, kb = 0, vb = 0;
  if (p.live) {
    const unsigned char* block = a.cache + p.block;
    kw = *reinterpret_cast<const uint32_t*>(block + k_word_at(p));
    vw = *reinterpret_cast<const uint32_t*>(block + a.c.v_at() + v_word_at(p));
    kb = block[a.c.k_scale_at() + p.token * (D / 32) + (p.t >> 2)];
    vb = block[a.c.v_scale_at() + p.token * (D / 32) + (p.t >> 2)];
  }
  vw = swap_v_bytes<D>(vw, p.t);
  if (p.live) {
    k = values_of<F32>(kw, kb);
    v = values_of<F32>(vw, vb);
  }
  if (p.row >= a.rows) return;
  store_eight<F32>(a.K, p.row * a.k.row + p.head * a.k.head + 8 * p.t, k);
  store_eight<F32>(a.V, p.row * a.v.row + p.head * a.v.head + 8 * p.t, v);
}

template <int D, bool F32>
static int launch_rows(const CacheRowsArgs& a, bool write, hipStream_t st) {
  constexpr int per = kRowsThreads / (D / 8);
  const dim3 grid((unsigned)((a.rows + per - 1) / per), (unsigned)a.c.Hk);
  if (write) hipLaunchKernelGGL((cache4_write_kernel<D, F32>), grid, dim3(kRowsThreads), 0, st, a);
  else hipLaunchKernelGGL((cache4_read_kernel<D, F32>), grid, dim3(kRowsThreads), 0, st, a);
  return check_launch();
}

static int launch_rows_any(const CacheRowsArgs& a, int dtype, bool write, hipStream_t st) {
  if (a.c.d == 128) return dtype == HA_BF16 ? launch_rows<128, false>(a, write, st) : launch_rows<128, true>(a, write, st);
  return dtype == HA_BF16 ? launch_rows<64, false>(a, write, st) : launch_rows<64, true>(a, write, st);
}

int launch_cache4_write(const CacheRowsArgs& a, int dtype, hipStream_t st) { return launch_rows_any(a, dtype, true, st); }
int launch_cache4_read(const CacheRowsArgs& a, int dtype, hipStream_t st) { return launch_rows_any(a, dtype, false, st); }

}  // namespace ha
