// Block tables and slots of a step's rows from the sequences' lengths (ha_page_plan).
//
// With rows_s = max(add_s, 0), need_s = pages that the rows of s take beyond those it has, and the prefix sums R_s, N_s of rows and needs and F_s of
// the pages of sequences that end, everything is an index:
//   stack(k)              = free_pages[k] below the count, page k - count of the ended sequences' above
//   new page j of s       = stack(avail - 1 - (N_s - need_s + j)),  avail = count + F
//   slot of row i         = page of token lens_s + i - R_s of the s that holds i, found by bisection of R
// Every workgroup forms the three sums by itself, in LDS (12 bytes a sequence), and takes its share of the outputs: a scan of a
// few thousand lengths is cheaper than a second launch.  Nothing that is written is read by another workgroup: new entries of the table are
// computed where a slot needs them, and the stack is written from its old count upwards and read below it.
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

// The s with upto[s - 1] <= i < upto[s] (upto: inclusive prefix sums, i below the last)
__device__ inline int plan_find(const int32_t* upto, int n, int i) {
  int lo = 0, hi = n - 1;
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (upto[mid] > i) hi = mid;
    else lo = mid + 1;
  }
  return lo;
}

__global__ __launch_bounds__(kPlanThreads) void page_plan_kernel(PagePlanArgs a) {
  extern __shared__ __attribute__((aligned(16))) int32_t plan_lds[];
  long long* wide = reinterpret_cast<long long*>(plan_lds);  // one word a wave, of either width
  int* narrow = plan_lds;
  const int n = a.n_seq, tid = threadIdx.x;
  int32_t* row_upto = plan_lds + kPlanThreads / 32;  // rows up to and with s, at most 2^31 - 1
  int32_t* need_upto = row_upto + n;  // pages asked for
  int32_t* free_upto = need_upto + n; // pages of ended sequences
  const int cap = a.max_blocks << a.log_page;
  auto held = [&](int s) { return min(max(a.lens[s], 0), cap); };
  auto pages_of = [&](int tokens) { return (int)(((int64_t)tokens + a.page - 1) >> a.log_page); };
  const int each = (n + kPlanThreads - 1) / kPlanThreads, s0 = min(n, tid * each), s1 = min(n, s0 + each);

  long long rows = 0, all_rows;
  for (int s = s0; s < s1; ++s) rows += max(a.add[s], 0);
  long long at = plan_scan(rows, &all_rows, wide);
  int need = 0, freed = 0;
  for (int s = s0; s < s1; ++s) {
    const int more = a.add[s], have = held(s);
    at += max(more, 0);
    row_upto[s] = (int32_t)min(at, 0x7fffffffll);
    const bool fits = more >= 0 && (int64_t)have + more <= cap && at <= a.rows;
    if (fits) need += pages_of(have + more) - pages_of(have);
    if (more < 0) freed += pages_of(have);
    need_upto[s] = need;
    free_upto[s] = freed;
  }
  // (sums of at most n_seq * max_blocks pages)
  int all_need, all_freed;
  const int need0 = plan_scan(need, &all_need, narrow), freed0 = plan_scan(freed, &all_freed, narrow);
  for (int s = s0; s < s1; ++s) {
    need_upto[s] += need0;
    free_upto[s] += freed0;
  }
  __syncthreads();
  const int count = min(max(*a.free_count, 0), a.n_pages);
  const int avail = (int)min((int64_t)count + all_freed, (int64_t)a.n_pages);
  // sequences that need pages are served up to the first whose pages are not there
  int taken = all_need;
  if (all_need > avail) {  // the last prefix that fits
    int lo = 0, hi = n;    // sequences [0, lo) fit
    while (lo < hi) {
      const int mid = (lo + hi) >> 1;
      if (need_upto[mid] <= avail) lo = mid + 1;
      else hi = mid;
    }
    taken = lo > 0 ? need_upto[lo - 1] : 0;
  }
  auto need_of = [&](int s) { return need_upto[s] - (s > 0 ? need_upto[s - 1] : 0); };
  auto served = [&](int s, int more, int have) {
    if (more < 0 || (int64_t)have + more > cap || row_upto[s] > a.rows) return false;
    return need_of(s) == 0 || need_upto[s] <= avail;
  };
  auto stack = [&](int k) -> int {
    if (k < count) return a.free_pages[k];
    const int s = plan_find(free_upto, n, k - count);
    return a.table[(int64_t)s * a.max_blocks + (k - count - (s > 0 ? free_upto[s - 1] : 0))];
  };

  const int64_t first = (int64_t)blockIdx.x * kPlanThreads + tid, step = (int64_t)gridDim.x * kPlanThreads;
  for (int64_t s = first; s < n; s += step) {
    const int more = a.add[s], have = held((int)s);
    a.lens_out[s] = more < 0 ? 0 : served((int)s, more, have) ? have + more : have;
    a.cu[s + 1] = row_upto[s];
  }
  if (first == 0) {
    a.cu[0] = 0;
    *a.free_count_out = avail - taken;
  }
  for (int64_t k = first; k < taken; k += step) {
    const int s = plan_find(need_upto, n, (int)k);
    const int j = pages_of(held(s)) + (int)k - (s > 0 ? need_upto[s - 1] : 0);
    a.table[(int64_t)s * a.max_blocks + j] = stack(avail - 1 - (int)k);
  }
  for (int64_t k = count + first; k < avail - taken; k += step) a.free_pages[k] = stack((int)k);
  const int live_rows = n > 0 ? row_upto[n - 1] : 0;
  for (int64_t i = first; i < a.rows; i += step) {
    int slot = -1;
    if (i < live_rows) {
      const int s = plan_find(row_upto, n, (int)i);
      const int more = a.add[s], have = held(s);
      if (served(s, more, have)) {
        const int pos = have + (int)i - (s > 0 ? row_upto[s - 1] : 0), blk = pos >> a.log_page, new0 = pages_of(have);
        const int page = blk >= new0 ? stack(avail - 1 - ((s > 0 ? need_upto[s - 1] : 0) + blk - new0)) : a.table[(int64_t)s * a.max_blocks + blk];
        if ((unsigned)page < (unsigned)a.n_pages) slot = (page << a.log_page) + (pos & (a.page - 1));
      }
    }
    a.slots[i] = slot;
  }
}

// A workgroup's sums take it one to three microseconds, so it gets 1024 rows, up to two workgroups per CU.
int launch_page_plan(const PagePlanArgs& a, hipStream_t st) {
  int64_t grid = ((int64_t)a.rows + 1023) / 1024;
  if (grid < 1) grid = 1;
  if (grid > 512) grid = 512;
  const size_t lds = (kPlanThreads / 32 + 3 * (size_t)a.n_seq) * 4;
  static std::atomic<uint64_t> lds_set{0};
  if (allow_full_lds(reinterpret_cast<const void*>(&page_plan_kernel), lds_set) != HA_OK) return HA_ERR_LAUNCH;
  hipLaunchKernelGGL(page_plan_kernel, dim3((unsigned)grid), dim3(kPlanThreads), lds, st, a);
  return check_launch();
}

}  // namespace ha
