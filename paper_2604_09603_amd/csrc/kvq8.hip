// The writers of the 8-bit paged KV cache (kvq8_device.h has its layout and scales):
//
//   store_kv_q8    rows at the slots of a slot map (prompts, single tokens): one wave
//                  for each head and tensor of a run, that is rows whose slots are
//                  consecutive within one block.
//   commit_kv_q8   the verified root and the accepted path of each request: one
//                  workgroup per request, one wave for each head, tensor and block of
//                  the (at most two) that the path touches.
//
// A block's scale is the maximum over its new values, so a wave holds a whole block's new
// rows in registers: they are read once, and written once as bytes.  Prompts are bound
// by HBM: 40960 rows of eight heads, 252 MB, in 53.4 us a call back to back, 4.7 TB/s (a large copy
// on the same card moves 4.4-5.3, by its size).  Single tokens (128 rows of four heads: 4.3 us
// a kernel, median) and commits (128 requests: 5.0 us) are bound by latency: the slot, the row and the block's scale and bytes
// are two or three dependent round trips.
#include "kvq8_device.h"

namespace echo {
namespace {

constexpr int kStoreThreads = 256;
// Rows per wave: as few as this many waves allow, up to a block's.  A wave with many rows
// appends the runs that start in them one after another, 1.5 us each; a wave that starts
// no run is a launch for nothing.  With eight heads, 1 | 8 | 32 rows per wave, the same rows over
// and over (so from the caches): 1024 single tokens take 16.2 | 17.4 | 55 us (by the rule, 4:
// 13.3), 2048 prompt rows 22 | 10.6 | 8.8 us (8), 40960 prompt rows 356 | 143 | 51 us (32).
constexpr int kStoreWaves = 4096;
constexpr int kCommitQ8Threads = 1024;

// Wave -> (chunk of rows_per_wave rows, tensor, head), head fastest: a workgroup's waves read
// neighbouring heads of the same rows.  The
// wave appends the runs that start in its chunk; a run ends within 32 rows.
template <int kFmt>
__global__ __launch_bounds__(kStoreThreads) void store_kv_q8_kernel(
    const uint16_t* __restrict__ k, const uint16_t* __restrict__ v, long long k_stride,
    long long v_stride, const int64_t* __restrict__ slot_map, int T, int rows_per_wave, CacheQ8 c,
    int32_t* status) {
  const int lane = threadIdx.x & (kWave - 1);
  const long long wave = (long long)blockIdx.x * (kStoreThreads / kWave) + threadIdx.x / kWave;
  const int per = 2 * c.hkv;
  const long long chunk = wave / per;
  const int tensor = int(wave % per) >= c.hkv ? 1 : 0, head = int(wave % per) - tensor * c.hkv;
  const long long i0 = chunk * rows_per_wave;
  if (i0 >= T) return;  // uniform
  // the slots of the chunk's rows and of those that its last run may take in
  const long long total = c.num_pages * c.page_size;
  const long long i = i0 + lane;
  const long long slot = i < T ? slot_map[i] : -1;
  const long long before = i > 0 && i <= T ? slot_map[i - 1] : -1;
  const bool live = slot >= 0 && slot < total;
  if (lane < rows_per_wave && slot >= total) status_or(status, ECHO_DATA_BAD_OFFSETS);
  const bool joined = live && before >= 0 && before + 1 == slot && (slot & (kBlockTokens - 1)) != 0;
  const uint64_t starts = __ballot(live && !joined);
  const uint64_t ends = __ballot(!joined);  // a run reaches up to the next of these
  uint64_t todo = starts & (rows_per_wave >= 64 ? ~0ull : (1ull << rows_per_wave) - 1);
  const uint16_t* base = tensor == 0 ? k : v;
  const long long stride = tensor == 0 ? k_stride : v_stride;
  while (todo != 0ull) {  // uniform
    const int a = __ffsll((unsigned long long)todo) - 1;
    todo &= todo - 1;
    const uint64_t later = ends & ~((2ull << a) - 1);
    const int n = min(kBlockTokens, (later == 0ull ? kWave : __ffsll((unsigned long long)later) - 1) - a);
    const long long s = __shfl(slot, a);
    const int off = int(s & (c.page_size - 1));
    const size_t blk = block_index(c, s >> c.page_shift, head, off);
    const uint16_t* first = base + (i0 + a) * stride + size_t(head) * ECHO_HEAD_DIM;
    append_block<kFmt>([&](int j) { return first + j * stride; }, n, off & (kBlockTokens - 1),
                       (tensor == 0 ? c.k_pages : c.v_pages) + blk * kBlockBytes,
                       (tensor == 0 ? c.k_scale : c.v_scale) + blk);
  }
}

template <int kFmt>
__global__ __launch_bounds__(kCommitQ8Threads) void commit_kv_q8_kernel(
    const int32_t* __restrict__ q_offsets, const int32_t* __restrict__ accept_len,
    const int32_t* __restrict__ accept_slots, int max_depth, const uint16_t* __restrict__ k_new,
    const uint16_t* __restrict__ v_new, int max_rows, CacheQ8 c,
    const int32_t* __restrict__ block_table, int max_pages, const int32_t* prefix_len,
    int32_t* new_len, int32_t* status) {
  __shared__ int s_slot[ECHO_MAX_DEPTH + 1];
  __shared__ int s_page[ECHO_MAX_DEPTH + 1];
  __shared__ int s_bad;
  const int r = blockIdx.x;
  const int tid = threadIdx.x;
  const int q0 = q_offsets[r], q1 = q_offsets[r + 1];
  const int L = accept_len[r];
  const int P = prefix_len[r];
  bool ok = true;
  int n = 0;
  if (q1 > q0) {  // a request without slots verified nothing and commits nothing
    ok = q0 >= 0 && q1 <= max_rows && L >= 0 && L <= max_depth && P >= 0;
    n = ok ? 1 + L : 0;
  }
  if (tid == 0) s_bad = ok ? 0 : 1;
  __syncthreads();
  // thread j resolves committed row j: its slot and its page
  if (tid < n) {
    const int s = tid == 0 ? q0 : accept_slots[size_t(r) * max_depth + (tid - 1)];
    const long long e = ((long long)P + tid) >> c.page_shift;
    const int page = e < max_pages ? block_table[size_t(r) * max_pages + size_t(e)] : -1;
    // (the new length stays below 2^31: pages may be shared, so that a table's tokens can exceed the pool's)
    if (s < 0 || s >= max_rows || page < 0 || page >= c.num_pages || P > 0x7FFFFFFE - tid)
      atomicOr(&s_bad, 1);
    s_slot[tid] = s;
    s_page[tid] = page;
  }
  __syncthreads();
  if (s_bad) n = 0;  // nothing of the request is written
  if (tid == 0) {
    if (s_bad) status_or(status, ECHO_DATA_BAD_OFFSETS);
    new_len[r] = P + n;
  }
  if (n == 0) return;
  // rows [0, n0) fill up the block of position P, the rest start the next one
  const int o = P & (kBlockTokens - 1);
  const int n0 = min(n, kBlockTokens - o);
  const int items = 2 * c.hkv * (n > n0 ? 2 : 1);
  const size_t row = size_t(c.hkv) * ECHO_HEAD_DIM;
  for (int it = tid / kWave; it < items; it += kCommitQ8Threads / kWave) {
    const int second = it >= 2 * c.hkv ? 1 : 0;
    const int head = (it - second * 2 * c.hkv) >> 1, tensor = it & 1;
    const int j0 = second ? n0 : 0;
    const size_t blk = block_index(c, s_page[j0], head, (P + j0) & (c.page_size - 1));
    const uint16_t* base = (tensor == 0 ? k_new : v_new) + size_t(head) * ECHO_HEAD_DIM;
    append_block<kFmt>([&](int j) { return base + size_t(s_slot[j0 + j]) * row; },
                       second ? n - n0 : n0, second ? 0 : o,
                       (tensor == 0 ? c.k_pages : c.v_pages) + blk * kBlockBytes,
                       (tensor == 0 ? c.k_scale : c.v_scale) + blk);
  }
}

CacheQ8 cache_of(const CacheQ8Args& a) {
  CacheQ8 c;
  c.k_pages = a.k_pages;
  c.v_pages = a.v_pages;
  c.k_scale = a.k_scale;
  c.v_scale = a.v_scale;
  c.num_pages = static_cast<long long>(a.num_pages);
  c.page_size = a.page_size;
  c.page_shift = 0;
  while ((1 << c.page_shift) < a.page_size) ++c.page_shift;
  c.hkv = a.hkv;
  return c;
}

}  // namespace

int32_t launch_store_kv_q8(const uint16_t* k, const uint16_t* v, int64_t k_stride, int64_t v_stride,
                           const int64_t* slot_map, int32_t num_rows, const CacheQ8Args& a,
                           int32_t* status, hipStream_t stream) {
  (void)hipGetLastError();
  const CacheQ8 c = cache_of(a);
  int rows_per_wave = 1;
  while (rows_per_wave < kBlockTokens &&
         (long long)num_rows * (2 * a.hkv) > (long long)rows_per_wave * kStoreWaves)
    rows_per_wave *= 2;
  const long long waves =
      ((long long)num_rows + rows_per_wave - 1) / rows_per_wave * (2ll * a.hkv);
  const long long wgs = (waves + kStoreThreads / kWave - 1) / (kStoreThreads / kWave);
  if (wgs > 0x7FFFFFFFll) return ECHO_ERR_UNSUPPORTED;
  hipLaunchKernelGGL(a.format == ECHO_KV_E4M3 ? store_kv_q8_kernel<ECHO_KV_E4M3>
                                              : store_kv_q8_kernel<ECHO_KV_E5M2>,
                     dim3(unsigned(wgs)), dim3(kStoreThreads), 0, stream, k, v,
                     static_cast<long long>(k_stride), static_cast<long long>(v_stride), slot_map,
                     num_rows, rows_per_wave, c, status);
  return hipGetLastError() == hipSuccess ? ECHO_OK : ECHO_ERR_HIP;
}

int32_t launch_commit_kv_q8(const int32_t* q_offsets, const int32_t* accept_len,
                            const int32_t* accept_slots, int32_t max_depth, const uint16_t* k_new,
                            const uint16_t* v_new, int32_t R, int32_t max_rows,
                            const CacheQ8Args& a, const int32_t* block_table, int32_t max_pages,
                            const int32_t* prefix_len, int32_t* new_len, int32_t* status,
                            hipStream_t stream) {
  (void)hipGetLastError();
  hipLaunchKernelGGL(a.format == ECHO_KV_E4M3 ? commit_kv_q8_kernel<ECHO_KV_E4M3>
                                              : commit_kv_q8_kernel<ECHO_KV_E5M2>,
                     dim3(unsigned(R)), dim3(kCommitQ8Threads), 0, stream, q_offsets, accept_len,
                     accept_slots, max_depth, k_new, v_new, max_rows, cache_of(a), block_table,
                     max_pages, prefix_len, new_len, status);
  return hipGetLastError() == hipSuccess ? ECHO_OK : ECHO_ERR_HIP;
}

}  // namespace echo
