// Block tables and slots of a step's rows from the sequences' lengths (ha_page_plan).
//
// With rows_s = max(add_s, 0), need_s = pages that the rows of s take beyond those it has, and the prefix sums R_s, N_s of rows and needs and F_s of
// the pages of sequences that end, everything is an index:
//   stack(k)              = free_pages[k] below the count, page k - count of the ended sequences' above
//   new page j of s       = stack(avail - 1 - (N_s - need_s + j)),  avail = count + F
//   slot of row i         = page of token lens_s + i - R_s of the s that holds i, found by bisection of R
// Every workgroup forms the three sums by itself, in LDS (16 bytes a sequence, with the lengths), and takes its share of the outputs: a scan of a
// few thousand lengths is cheaper than a second launch.  Nothing that is written is read by another workgroup: new entries of the table are
// computed where a slot needs them, and the stack is written from its old count upwards and read below it.
// Bound by latency: three dependent reads of memory, two scans, and for a row up to two bisections of LDS (its sequence; the ended sequence whose page it gets).
// MI355X: 256 sequences of a decoding step 5.7 us, 1000 sequences and 500000 rows, a fifth of them ending, 11.4 us, 5.4 of it the sums (tables and slots one
// behind the other by the same workgroups, lengths and additions from memory: 6.4 and 15.2; eight rows a thread, half the workgroups: 18).
#include "cache4_common.h"

namespace ha {

constexpr int kPlanThreads = 256;

// Exclusive prefix over the workgroup's threads and the total.
template <class T>
__device__ inline T plan_scan(T v, T* total, T* lds) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  T inc = v;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const T up = __shfl_up(inc, o);
    if (lane >= o) inc += up;
  }
  if (lane == 63) lds[wave] = inc;
  __syncthreads();
  T before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < kPlanThreads / 64; ++w) {
    if (w < wave) before += lds[w];
    all += lds[w];
  }
  __syncthreads();
  *total = all;
  return before + inc - v;
}

constexpr int kServed = 1 << 31;  // of a need's sum (at most 2^30): the sequence gets its rows

// The s with upto[s - 1] <= i < upto[s] (upto: inclusive prefix sums, i below the last)
__device__ inline int plan_find(const int32_t* upto, int n, int i) {
  int lo = 0, hi = n - 1;
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if ((upto[mid] & ~kServed) > i) hi = mid;
    else lo = mid + 1;
  }
  return lo;
}

constexpr int kPlanRows = 2;      // rows of a thread, a workgroup's width apart, whose page numbers are asked for together

__global__ __launch_bounds__(kPlanThreads) void page_plan_kernel(PagePlanArgs a) {
  extern __shared__ __attribute__((aligned(16))) int32_t plan_lds[];
  long long* wide = reinterpret_cast<long long*>(plan_lds);  // one word a wave, of either width
  int* narrow = plan_lds;
  const int n = a.n_seq, tid = threadIdx.x;
  int32_t* row_upto = plan_lds + kPlanThreads / 32;  // rows up to and with s, at most 2^31 - 1
  int32_t* need_upto = row_upto + n;  // pages asked for
  int32_t* free_upto = need_upto + n; // pages of ended sequences
  int32_t* length = free_upto + n;
  const int cap = a.max_blocks << a.log_page;
  const int count = min(max(*a.free_count, 0), a.n_pages);
  auto pages_of = [&](int tokens) { return (int)(((int64_t)tokens + a.page - 1) >> a.log_page); };
  const int each = (n + kPlanThreads - 1) / kPlanThreads, s0 = min(n, tid * each), s1 = min(n, s0 + each);

#pragma unroll 4
  for (int s = tid; s < n; s += kPlanThreads) {
    row_upto[s] = a.add[s];
    length[s] = min(max(a.lens[s], 0), cap);
  }
  __syncthreads();
  long long rows = 0, all_rows;
  for (int s = s0; s < s1; ++s) rows += max(row_upto[s], 0);
  long long at = plan_scan(rows, &all_rows, wide);
  int need = 0, freed = 0;
  for (int s = s0; s < s1; ++s) {
    const int more = row_upto[s], have = length[s];
    at += max(more, 0);
    row_upto[s] = (int32_t)min(at, 0x7fffffffll);
    const bool fits = more >= 0 && (int64_t)have + more <= cap && at <= a.rows;
    int asks = 0;
    if (fits) asks = pages_of(have + more) - pages_of(have);
    if (more < 0) freed += pages_of(have);
    need += asks;
    need_upto[s] = need | (fits ? kServed : 0);
    free_upto[s] = freed;
  }
  // (sums of at most n_seq * max_blocks pages)
  int all_need, all_freed;
  const int need0 = plan_scan(need, &all_need, narrow), freed0 = plan_scan(freed, &all_freed, narrow);
  const int avail = (int)min((int64_t)count + all_freed, (int64_t)a.n_pages);
  // Sequences that need pages are served up to the first whose pages are not there.
  int before = need0, last_fit = 0;  // of the thread's sequences: the sum of the last one that fits
  for (int s = s0; s < s1; ++s) {
    const int w = need_upto[s], upto = (w & ~kServed) + need0;
    const bool served = (w & kServed) && (upto == before || upto <= avail);
    if (upto <= avail) last_fit = upto;
    need_upto[s] = upto | (served ? kServed : 0);
    free_upto[s] += freed0;
    before = upto;
  }
  // pages that are taken: the largest sum within avail
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) last_fit = max(last_fit, __shfl_xor(last_fit, o));
  if ((tid & 63) == 0) narrow[tid >> 6] = last_fit;
  __syncthreads();
  int taken = 0;
#pragma unroll
  for (int w = 0; w < kPlanThreads / 64; ++w) taken = max(taken, narrow[w]);
  auto need_before = [&](int s) { return s > 0 ? need_upto[s - 1] & ~kServed : 0; };
  auto stack = [&](int k) -> const int32_t* {
    if (k < count) return a.free_pages + k;
    const int s = plan_find(free_upto, n, k - count);
    return a.table + (int64_t)s * a.max_blocks + (k - count - (s > 0 ? free_upto[s - 1] : 0));
  };

  // the first slot_wgs workgroups make the slots, the others what the sequences have
  if ((int)blockIdx.x >= a.slot_wgs) {
  const int64_t first = (int64_t)(blockIdx.x - a.slot_wgs) * kPlanThreads + tid, step = (int64_t)(gridDim.x - a.slot_wgs) * kPlanThreads;
  for (int64_t s = first; s < n; s += step) {
    const int more = row_upto[s] - (s > 0 ? row_upto[s - 1] : 0);
    const bool ended = free_upto[s] != (s > 0 ? free_upto[s - 1] : 0);
    // (an end without pages had no tokens)
    a.lens_out[s] = ended ? 0 : need_upto[s] & kServed ? length[s] + more : length[s];
    a.cu[s + 1] = row_upto[s];
  }
  if (first == 0) {
    a.cu[0] = 0;
    *a.free_count_out = avail - taken;
  }
  for (int64_t k = first; k < taken; k += step) {
    const int s = plan_find(need_upto, n, (int)k);
    const int j = pages_of(length[s]) + (int)k - need_before(s);
    a.table[(int64_t)s * a.max_blocks + j] = *stack(avail - 1 - (int)k);
  }
  for (int64_t k = count + first; k < avail - taken; k += step) a.free_pages[k] = *stack((int)k);
  return;
  }
  const int live_rows = n > 0 ? row_upto[n - 1] : 0;
  for (int64_t base = (int64_t)blockIdx.x * (kPlanThreads * kPlanRows); base < a.rows;
       base += (int64_t)a.slot_wgs * (kPlanThreads * kPlanRows)) {
    const int32_t* from[kPlanRows];  // where the row's page number lies; all of them are asked for together
    int token[kPlanRows];            // within the page; < 0: no slot
    int s = -1;
#pragma unroll
    for (int z = 0; z < kPlanRows; ++z) {
      const int64_t i = base + z * kPlanThreads + tid;
      from[z] = a.free_count;
      token[z] = -1;
      if (i >= live_rows || i >= a.rows) continue;
      if (s < 0 || row_upto[s] <= i) {  // often the sequence of the row before, or the next one
        if (s < 0 || row_upto[s + 1] <= i) s = plan_find(row_upto, n, (int)i);
        else ++s;
      }
      if (!(need_upto[s] & kServed)) continue;
      const int pos = length[s] + (int)i - (s > 0 ? row_upto[s - 1] : 0), blk = pos >> a.log_page, new0 = pages_of(length[s]);
      from[z] = blk >= new0 ? stack(avail - 1 - (need_before(s) + blk - new0)) : a.table + (int64_t)s * a.max_blocks + blk;
      token[z] = pos & (a.page - 1);
    }
    int page[kPlanRows];
#pragma unroll
    for (int z = 0; z < kPlanRows; ++z) page[z] = *from[z];
#pragma unroll
    for (int z = 0; z < kPlanRows; ++z) {
      const int64_t i = base + z * kPlanThreads + tid;
      if (i < a.rows) a.slots[i] = token[z] >= 0 && (unsigned)page[z] < (unsigned)a.n_pages ? (page[z] << a.log_page) + token[z] : -1;
    }
  }
}

// A workgroup's sums take it one to three microseconds, so it gets 512 rows; up to four workgroups per CU, and one for the tables.
int launch_page_plan(const PagePlanArgs& args, hipStream_t st) {
  PagePlanArgs a = args;
  const int64_t slots = ((int64_t)a.rows + kPlanThreads * kPlanRows - 1) / (kPlanThreads * kPlanRows);
  const int64_t tables = ((int64_t)a.n_seq + a.rows / a.page + kPlanThreads - 1) / kPlanThreads;
  a.slot_wgs = (int32_t)(slots > 1024 ? 1024 : slots);
  const int64_t grid = a.slot_wgs + (tables < 1 ? 1 : tables > 256 ? 256 : tables);
  const size_t lds = (kPlanThreads / 32 + 4 * (size_t)a.n_seq) * 4;
  static std::atomic<uint64_t> lds_set{0};
  if (allow_full_lds(reinterpret_cast<const void*>(&page_plan_kernel), lds_set) != HA_OK) return HA_ERR_LAUNCH;
  hipLaunchKernelGGL(page_plan_kernel, dim3((unsigned)grid), dim3(kPlanThreads), lds, st, a);
  return check_launch();
}

}  // namespace ha
