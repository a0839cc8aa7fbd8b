// The writers of the latent cache, rows of 576 bfloat16: 512 normalised dims, which are keys and
// values of every head, then 64 rotated ones, which only the scores see.
//
//   store_latent    rows of the projection's output, normalised and rotated: to the slots of a
//                   slot map, to rows beside a draft tree, or both.  One wave per row:
//                   c = x * rsqrt(mean x^2 + eps) * weight over dims 0-511 (eight a lane),
//                   the turns of dims 512-575 (a pair in each of 32 lanes).
//   commit_latent   the verified root and the accepted path of each request: one workgroup
//                   per request copies their rows and moves the length on.
//
// A row is exactly a wave's loads (16 bytes a lane and a pair), so that its sum needs no LDS and
// no barrier.  Both are bound by memory: 40000 rows, 93 MB, take 16.6 us (5.5 TB/s; a copy of
// 256 MB reaches 5.4), the weight and the table of frequencies coming from L2; 384 rows
// 2.3 us and 128 commits 2.4 us in a captured graph, which is near an empty launch
// (a commit is two dependent round trips, the offsets and the rows); as eager calls
// 6.9 and 6.4 us, the host's part.
#include "echo_device.h"
#include "echo_internal.h"
#include "rope_device.h"

namespace echo {
namespace {

constexpr int kC = ECHO_LATENT_DIM, kRope = ECHO_LATENT_ROPE_DIM, kRow = kC + kRope;
static_assert(kC == 8 * kWave && kRope == kWave, "a row is a wave's");
constexpr int kLatentThreads = 256;

__device__ __forceinline__ float wave_add(float v) {
#pragma unroll
  for (int d = 1; d < kWave; d *= 2) v += __shfl_xor(v, d);
  return v;
}

struct StoreLatentKernelArgs {
  const uint16_t* kv;
  long long kv_stride;
  const uint16_t* weight;
  float eps;
  const int32_t* positions;
  const double* inv_freq;
  float scale;
  int num_rows;
  const int32_t* row_count;
  uint16_t* latent_new;
  const int64_t* slot_map;
  uint16_t* pages;
  long long slots;
  int32_t* status;
};

template <bool kInterleaved>
__global__ __launch_bounds__(kLatentThreads) void store_latent_kernel(StoreLatentKernelArgs a) {
  const int lane = threadIdx.x & (kWave - 1);
  const int n = rope_rows(a.row_count, a.num_rows);
  if (n < 0) {
    if (blockIdx.x == 0 && threadIdx.x == 0) status_or(a.status, ECHO_DATA_BAD_OFFSETS);
    return;
  }
  const int row = int(blockIdx.x) * (kLatentThreads / kWave) + int(threadIdx.x) / kWave;
  if (row >= n) return;  // uniform in a wave
  const uint16_t* x = a.kv + row * a.kv_stride;
  const uint4 v = *reinterpret_cast<const uint4*>(x + 8 * lane);
  uint32_t w[4] = {v.x, v.y, v.z, v.w};
  const int i = lane & 31;  // (the upper lanes' pairs are dropped)
  const int ia = kC + (kInterleaved ? 2 * i : i), ib = kC + (kInterleaved ? 2 * i + 1 : i + 32);
  uint16_t ra = x[ia], rb = x[ib];
  long long slot = -1;
  if (a.slot_map != nullptr) {
    slot = a.slot_map[row];
    if (slot >= a.slots) {
      if (lane == 0) status_or(a.status, ECHO_DATA_BAD_OFFSETS);
      slot = -1;
    }
  }
  if (a.weight != nullptr) {
    const uint4 g = *reinterpret_cast<const uint4*>(a.weight + 8 * lane);
    const uint32_t gw[4] = {g.x, g.y, g.z, g.w};
    float sum = 0.0f;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      sum = __builtin_fmaf(bf16_lo(w[j]), bf16_lo(w[j]), sum);
      sum = __builtin_fmaf(bf16_hi(w[j]), bf16_hi(w[j]), sum);
    }
    const float r = rsqrtf(wave_add(sum) * (1.0f / kC) + a.eps);
#pragma unroll
    for (int j = 0; j < 4; ++j)
      w[j] = rope_pack(bf16_lo(w[j]) * r * bf16_lo(gw[j]), bf16_hi(w[j]) * r * bf16_hi(gw[j]));
  }
  if (a.inv_freq != nullptr) {
    const float2 o = rope_pair(bf16_lo(ra), bf16_lo(rb),
                               rope_turn(a.positions[row], a.inv_freq[i], a.scale));
    const uint32_t p = rope_pack(o.x, o.y);
    ra = uint16_t(p);
    rb = uint16_t(p >> 16);
  }
  const auto put = [&](uint16_t* y) {
    *reinterpret_cast<uint4*>(y + 8 * lane) = make_uint4(w[0], w[1], w[2], w[3]);
    if (lane < 32) {
      y[ia] = ra;
      y[ib] = rb;
    }
  };
  if (a.latent_new != nullptr) put(a.latent_new + size_t(row) * kRow);
  if (slot >= 0) put(a.pages + size_t(slot) * kRow);
}

__global__ __launch_bounds__(kLatentThreads) void commit_latent_kernel(
    const int32_t* __restrict__ q_offsets, const int32_t* __restrict__ accept_len,
    const int32_t* __restrict__ accept_slots, int max_depth, const uint16_t* __restrict__ latent_new,
    int max_rows, uint16_t* __restrict__ pages, long long num_pages, int page_shift,
    const int32_t* __restrict__ block_table, int max_pages, const int32_t* prefix_len,
    int32_t* new_len, int32_t* status) {
  __shared__ int s_src[ECHO_MAX_DEPTH + 1];
  __shared__ long long s_dst[ECHO_MAX_DEPTH + 1];
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
  if (tid < n) {  // thread j resolves committed row j: its slot and its place in the pages
    const int s = tid == 0 ? q0 : accept_slots[size_t(r) * max_depth + (tid - 1)];
    const long long e = ((long long)P + tid) >> page_shift;
    const int page = e < max_pages ? block_table[size_t(r) * max_pages + size_t(e)] : -1;
    // (the new length stays below 2^31)
    if (s < 0 || s >= max_rows || page < 0 || page >= num_pages || P > 0x7FFFFFFE - tid)
      atomicOr(&s_bad, 1);
    s_src[tid] = s;
    s_dst[tid] = ((long long)page << page_shift) + (((long long)P + tid) & ((1 << page_shift) - 1));
  }
  __syncthreads();
  if (s_bad) n = 0;  // nothing of the request is written
  constexpr int kChunks = kRow / 8;  // of 16 bytes
  for (int it = tid; it < n * kChunks; it += kLatentThreads) {
    const int j = it / kChunks, c = it - j * kChunks;
    reinterpret_cast<uint4*>(pages)[size_t(s_dst[j]) * kChunks + c] =
        reinterpret_cast<const uint4*>(latent_new)[size_t(s_src[j]) * kChunks + c];
  }
  if (tid == 0) {
    if (s_bad) status_or(status, ECHO_DATA_BAD_OFFSETS);
    new_len[r] = P + n;
  }
}

}  // namespace

int32_t launch_store_latent(const StoreLatentArgs& x, hipStream_t stream) {
  (void)hipGetLastError();
  StoreLatentKernelArgs a;
  a.kv = x.kv;
  a.kv_stride = static_cast<long long>(x.kv_stride);
  a.weight = x.norm_weight;
  a.eps = x.eps;
  a.positions = x.positions;
  a.inv_freq = x.inv_freq;
  a.scale = x.scale;
  a.num_rows = x.num_rows;
  a.row_count = x.row_count;
  a.latent_new = x.latent_new;
  a.slot_map = x.slot_map;
  a.pages = x.cache.pages;
  a.slots = static_cast<long long>(x.cache.num_pages) * x.cache.page_size;
  a.status = x.status;
  constexpr int kPer = kLatentThreads / kWave;
  const unsigned wgs = unsigned((static_cast<long long>(x.num_rows) + kPer - 1) / kPer);
  hipLaunchKernelGGL(x.layout == ECHO_ROPE_INTERLEAVED ? store_latent_kernel<true>
                                                       : store_latent_kernel<false>,
                     dim3(wgs), dim3(kLatentThreads), 0, stream, a);
  return hipGetLastError() == hipSuccess ? ECHO_OK : ECHO_ERR_HIP;
}

int32_t launch_commit_latent(const int32_t* q_offsets, const int32_t* accept_len,
                             const int32_t* accept_slots, int32_t max_depth,
                             const uint16_t* latent_new, int32_t R, int32_t max_rows,
                             const LatentCacheArgs& c, const int32_t* block_table,
                             int32_t max_pages, const int32_t* prefix_len, int32_t* new_len,
                             int32_t* status, hipStream_t stream) {
  (void)hipGetLastError();
  int shift = 0;
  while ((1 << shift) < c.page_size) ++shift;
  hipLaunchKernelGGL(commit_latent_kernel, dim3(unsigned(R)), dim3(kLatentThreads), 0, stream,
                     q_offsets, accept_len, accept_slots, max_depth, latent_new, max_rows, c.pages,
                     static_cast<long long>(c.num_pages), shift, block_table, max_pages, prefix_len,
                     new_len, status);
  return hipGetLastError() == hipSuccess ? ECHO_OK : ECHO_ERR_HIP;
}

}  // namespace echo
