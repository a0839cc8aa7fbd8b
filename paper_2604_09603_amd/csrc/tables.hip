// Block tables and slot maps of a paged cache, from the requests' lengths.
//
//   build_tables  one workgroup: how many pages each request gives back or takes (one
//                 scan over the requests), then the pages themselves, one thread each,
//                 whose request is found in the scan by bisection: a prompt's
//                 thousand pages are no more work for one thread than a token's.
//                 Few rows get their slots in the same launch.
//   slot_map      more rows: one thread each, in a launch of its own.
//
// Both are bound by latency: the 16 bytes a request and the 4 bytes a page of the first
// fit in the caches, and the second writes 8 bytes a row.  128 requests that take a token
// each: 5.7 us, most of it the launch and three dependent round trips to memory (lengths,
// stack, tables) with their barriers; 256 requests with prompts of up to 2048 rows: 7.4 and
// 4.2 us (medians).
#include "echo_device.h"
#include "echo_internal.h"

namespace echo {
namespace {

constexpr int kTableThreads = 1024;
constexpr int kMapThreads = 256;
// Slot maps up to this long need no second launch.  With 128 requests, here | in a launch of
// its own (calls back to back): 512 rows 6.3 | 9.0 us, 2048 rows 7.5 | 9.0, 4096 rows
// 9.6 | 9.0, 32768 rows 39 | 9.3.
constexpr int kFusedRows = 2 * kTableThreads;

// Offset r of the rows; bad if it is not one of non-decreasing numbers in [0, max_rows].
__device__ __forceinline__ int32_t row_offset(const TablesArgs& a, int r, bool& bad) {
  const int32_t o = a.row_offsets[r];
  const int32_t next = a.row_offsets[min(r + 1, a.R)];
  bad |= o < 0 || next < o || next > a.max_rows;
  return o;
}

// The slot of row i, or -1: rows past the last request's, and those whose page their
// request does not hold (missing).  held(r): the pages of request r.
template <typename Held>
__device__ __forceinline__ long long slot_of(const TablesArgs& a, int page_shift, int i,
                                             const int32_t* row_offsets, const Held& held,
                                             bool& missing) {
  missing = false;
  if (i < row_offsets[0] || i >= row_offsets[a.R]) return -1;
  const int r = upper_bound_idx(row_offsets, a.R, int32_t(i));
  const long long pos = (long long)a.row_start[r] + i - row_offsets[r];
  const long long e = pos >> page_shift;
  missing = pos < 0 || e >= held(r);
  if (missing) return -1;
  const long long page = a.block_table[size_t(r) * size_t(a.max_pages) + size_t(e)];
  missing = page < 0;
  return missing ? -1 : (page << page_shift) + (pos & (a.page_size - 1));
}

__global__ __launch_bounds__(kTableThreads) void build_tables_kernel(TablesArgs a, int page_shift,
                                                                     bool map) {
  extern __shared__ int32_t s_mem[];
  __shared__ int2 s_scan[kTableThreads / kWave + 1];
  __shared__ int s_last, s_bad_rows;
  const int tid = threadIdx.x;
  const int R = a.R;
  int32_t* s_held = s_mem;            // R: pages held before
  int32_t* s_give = s_mem + R;        // R + 1: pages given back by the requests before, and by all
  int32_t* s_take = s_give + (R + 1); // R + 1: pages wanted by the requests before, and by all
  int32_t* s_off = s_take + (R + 1);  // R + 1: row offsets (map)
  const int before = *a.num_free;     // (in the round trip of the lengths, as the offsets)
  bool bad_rows = false;
  if (map)
    for (int r = tid; r <= R; r += kTableThreads) s_off[r] = row_offset(a, r, bad_rows);
  if (tid == 0) s_last = s_bad_rows = 0;
  int bits = 0;
  int give_run = 0, take_run = 0;
  for (int base = 0; base < R; base += kTableThreads) {
    const int r = base + tid;
    int give = 0, take = 0;
    if (r < R) {
      const long long want = a.want_len[r];
      const int held = a.num_held[r];
      const long long need = (want + a.page_size - 1) >> page_shift;
      const bool held_ok = held >= 0 && held <= a.max_pages;
      if (!held_ok || want < 0 || need > a.max_pages) {
        bits |= ECHO_DATA_BAD_OFFSETS;  // left as it is
      } else {
        give = max(0, held - int(need));
        take = max(0, int(need) - held);
      }
      s_held[r] = held;
    }
    int g_tot, t_tot;
    const int2 ex = block_exclusive_sum2<kTableThreads>(make_int2(give, take), s_scan, &g_tot, &t_tot);
    if (r < R) {
      s_give[r] = give_run + ex.x;
      s_take[r] = take_run + ex.y;
    }
    give_run += g_tot;
    take_run += t_tot;
  }
  if (bad_rows) s_bad_rows = 1;
  if (tid == 0) {
    s_give[R] = give_run;
    s_take[R] = take_run;
  }
  const bool stack_ok = before >= 0 && before <= a.max_free && give_run <= a.max_free - before;
  if (!stack_ok) bits |= ECHO_DATA_BAD_OFFSETS;
  const int gives = stack_ok ? give_run : 0;
  const int top = stack_ok ? before + give_run : 0;
  __syncthreads();
  // requests are served in order until the pages run out
  const auto served = [&](int r) { return stack_ok && s_take[r + 1] <= top; };
  for (int r = tid; r < R; r += kTableThreads) {
    const int take = s_take[r + 1] - s_take[r];
    int now = s_held[r];
    if (take > 0) {
      if (served(r)) {
        now += take;
        atomicMax(&s_last, s_take[r + 1]);
      } else {
        bits |= ECHO_DATA_NO_PAGES;
      }
    } else if (stack_ok) {
      now -= s_give[r + 1] - s_give[r];
    }
    a.num_held_out[r] = now;
  }
  // pages given back, in request order
  for (int t = tid; t < gives; t += kTableThreads) {
    const int r = upper_bound_idx(s_give, R, t);
    const int first = s_held[r] - (s_give[r + 1] - s_give[r]);
    a.free_pages[before + t] =
        a.block_table[size_t(r) * size_t(a.max_pages) + size_t(first + t - s_give[r])];
  }
  __syncthreads();
  const int takes = s_last;
  if (tid == 0) *a.num_free_out = stack_ok ? top - takes : before;
  // pages taken, from the top of the stack
  for (int t = tid; t < takes; t += kTableThreads) {
    const int r = upper_bound_idx(s_take, R, t);
    a.block_table[size_t(r) * size_t(a.max_pages) + size_t(s_held[r] + t - s_take[r])] =
        a.free_pages[top - 1 - t];
  }
  if (map) {
    __syncthreads();
    bad_rows = s_bad_rows != 0;  // then no row has a slot
    if (bad_rows) bits |= ECHO_DATA_BAD_OFFSETS;
    const auto held = [&](int r) {
      const int take = s_take[r + 1] - s_take[r];
      const int h = s_held[r];
      const int now = take > 0 ? (served(r) ? h + take : h)
                               : (stack_ok ? h - (s_give[r + 1] - s_give[r]) : h);
      return now <= a.max_pages ? now : 0;
    };
    for (int i = tid; i < a.max_rows; i += kTableThreads) {
      bool missing = false;
      a.slot_map[i] = bad_rows ? -1 : slot_of(a, page_shift, i, s_off, held, missing);
      if (missing) bits |= ECHO_DATA_NO_PAGES;
    }
  }
  wave_status_or(a.status, bits);
}

__global__ __launch_bounds__(kMapThreads) void slot_map_kernel(TablesArgs a, int page_shift) {
  extern __shared__ int32_t s_off[];  // R + 1
  __shared__ bool s_bad[kMapThreads / kWave];
  bool bad_rows = false;
  for (int r = threadIdx.x; r <= a.R; r += kMapThreads) s_off[r] = row_offset(a, r, bad_rows);
  const uint64_t bad_lanes = __ballot(bad_rows);
  if ((threadIdx.x & (kWave - 1)) == 0) s_bad[threadIdx.x / kWave] = bad_lanes != 0ull;
  __syncthreads();
  bad_rows = false;  // of any wave's: then no row has a slot
#pragma unroll
  for (int w = 0; w < kMapThreads / kWave; ++w) bad_rows |= s_bad[w];
  const int i = blockIdx.x * kMapThreads + threadIdx.x;
  int bits = bad_rows ? ECHO_DATA_BAD_OFFSETS : 0;
  if (i < a.max_rows) {
    const auto held = [&](int r) {
      const int h = a.num_held_out[r];
      return h <= a.max_pages ? h : 0;
    };
    bool missing = false;
    a.slot_map[i] = bad_rows ? -1 : slot_of(a, page_shift, i, s_off, held, missing);
    if (missing) bits = ECHO_DATA_NO_PAGES;
  }
  wave_status_or(a.status, bits);
}

}  // namespace

int32_t launch_build_block_tables(const TablesArgs& a, hipStream_t stream) {
  (void)hipGetLastError();
  int page_shift = 0;
  while ((1 << page_shift) < a.page_size) ++page_shift;
  const bool map = a.slot_map != nullptr;
  const bool fused = map && a.max_rows <= kFusedRows;
  const size_t lds = (3 * size_t(a.R) + 2 + (fused ? size_t(a.R) + 1 : 0)) * sizeof(int32_t);
  if (lds > 60 * 1024 && hipFuncSetAttribute(reinterpret_cast<const void*>(build_tables_kernel),
                                             hipFuncAttributeMaxDynamicSharedMemorySize,
                                             int(lds)) != hipSuccess)
    return ECHO_ERR_HIP;
  hipLaunchKernelGGL(build_tables_kernel, dim3(1), dim3(kTableThreads), lds, stream, a, page_shift,
                     fused);
  if (map && !fused)
    hipLaunchKernelGGL(slot_map_kernel, dim3(unsigned((a.max_rows + kMapThreads - 1) / kMapThreads)),
                       dim3(kMapThreads), (size_t(a.R) + 1) * sizeof(int32_t), stream, a,
                       page_shift);
  return hipGetLastError() == hipSuccess ? ECHO_OK : ECHO_ERR_HIP;
}

}  // namespace echo
