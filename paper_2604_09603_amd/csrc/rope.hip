// Rotary positions of queries and keys (rope_device.h has the rotation), one launch for both.
//
// A workgroup has a row, or with few rows a share of one's heads: the turns of the row's
// pairs, once for all heads, into LDS; then its threads go through the heads, 16 dims at a time
// (two 16-byte loads and stores: eight pairs of either layout), the first of which is on
// its way while the turns are formed.  What is not 16-byte aligned, or whose rotated
// part is no multiple of 16, goes pair by pair.
//
// Bound by memory: four bytes are moved for three operations.  40000 rows of 40 heads of 128 dims,
// 819 MB, take 138-142 us (5.8-5.9 TB/s; a copy of 1 GB reaches 5.2); 384 rows of 68 heads
// 3.6 us in a captured graph, of which an empty launch is about two, and 11 us as
// an eager call, the host's part.
#include "echo_device.h"
#include "echo_internal.h"
#include "rope_device.h"

namespace echo {
namespace {

constexpr int kRopeThreads = 256;
// Workgroups at a time: eight of 256 threads on each of 256 CUs.  384 rows of 68 heads take 4.4 us
// with a workgroup per row, 3.6 with two rounds of threads' items shared by two and the
// loads beside the turns.
constexpr int kRopeFill = 2048;

struct RopeSide {
  const uint16_t* x;
  uint16_t* y;
  long long x_row, x_head, y_row, y_head;
};
struct RopeKernelArgs {
  RopeSide q, k;
  int hq, heads, half;
  const int32_t* positions;
  const int32_t* row_count;
  const double* inv_freq;
  float scale;
  int num_rows, share;  // items that a workgroup has of a row
  int32_t* status;
};

// An item: 16 dims of a head (kWide), or a pair.
template <bool kWide, bool kInterleaved>
__global__ __launch_bounds__(kRopeThreads) void rope_kernel(RopeKernelArgs a) {
  extern __shared__ __attribute__((aligned(16))) float2 s_turn[];  // [half]
  const int tid = threadIdx.x;
  const int n = rope_rows(a.row_count, a.num_rows);
  if (n < 0) {
    if (blockIdx.x == 0 && blockIdx.y == 0 && tid == 0) status_or(a.status, ECHO_DATA_BAD_OFFSETS);
    return;
  }
  const int row = int(blockIdx.x);
  if (row >= n) return;
  const int per = kWide ? a.half / 8 : a.half;  // items of a head
  const int first = int(blockIdx.y) * a.share;
  const int last = min(first + a.share, a.heads * per);
  struct Item {
    uint16_t* y;
    int c;
    uint4 a, b;
  };
  const auto load = [&](int it) {
    const int head = it / per;
    const bool is_q = head < a.hq;
    const RopeSide& side = is_q ? a.q : a.k;
    const long long hd = is_q ? head : head - a.hq;
    const uint16_t* x = side.x + row * side.x_row + hd * side.x_head;
    Item i;
    i.y = side.y + row * side.y_row + hd * side.y_head;
    i.c = it - head * per;
    if (kWide) {
      x += kInterleaved ? 16 * i.c : 8 * i.c;
      i.a = *reinterpret_cast<const uint4*>(x);
      i.b = *reinterpret_cast<const uint4*>(x + (kInterleaved ? 8 : a.half));
    } else {
      i.a.x = x[kInterleaved ? 2 * i.c : i.c];
      i.b.x = x[kInterleaved ? 2 * i.c + 1 : i.c + a.half];
    }
    return i;
  };
  int it = first + tid;
  Item i = {};
  if (it < last) i = load(it);
  for (int t = tid; t < a.half; t += kRopeThreads) s_turn[t] = rope_turn(a.positions[row], a.inv_freq[t], a.scale);
  __syncthreads();
  while (it < last) {
    if (!kWide) {
      const float2 o = rope_pair(bf16_lo(i.a.x), bf16_lo(i.b.x), s_turn[i.c]);
      const uint32_t w = rope_pack(o.x, o.y);
      i.y[kInterleaved ? 2 * i.c : i.c] = uint16_t(w);
      i.y[kInterleaved ? 2 * i.c + 1 : i.c + a.half] = uint16_t(w >> 16);
    } else {
      const float2* cs = s_turn + 8 * i.c;
      const uint32_t wa[4] = {i.a.x, i.a.y, i.a.z, i.a.w}, wb[4] = {i.b.x, i.b.y, i.b.z, i.b.w};
      uint32_t oa[4], ob[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if (kInterleaved) {
          const float2 u = rope_pair(bf16_lo(wa[j]), bf16_hi(wa[j]), cs[j]);
          const float2 v = rope_pair(bf16_lo(wb[j]), bf16_hi(wb[j]), cs[4 + j]);
          oa[j] = rope_pack(u.x, u.y);
          ob[j] = rope_pack(v.x, v.y);
        } else {
          const float2 u = rope_pair(bf16_lo(wa[j]), bf16_lo(wb[j]), cs[2 * j]);
          const float2 v = rope_pair(bf16_hi(wa[j]), bf16_hi(wb[j]), cs[2 * j + 1]);
          oa[j] = rope_pack(u.x, v.x);
          ob[j] = rope_pack(u.y, v.y);
        }
      }
      uint16_t* y = i.y + (kInterleaved ? 16 * i.c : 8 * i.c);
      *reinterpret_cast<uint4*>(y) = make_uint4(oa[0], oa[1], oa[2], oa[3]);
      *reinterpret_cast<uint4*>(y + (kInterleaved ? 8 : a.half)) = make_uint4(ob[0], ob[1], ob[2], ob[3]);
    }
    it += kRopeThreads;
    if (it < last) i = load(it);
  }
}

}  // namespace

int32_t launch_rope(const RopeArgs& x, hipStream_t stream) {
  (void)hipGetLastError();
  RopeKernelArgs a;
  a.q = RopeSide{x.q, x.q_out, x.q_row, x.q_head, x.q_out_row, x.q_out_head};
  a.k = RopeSide{x.k, x.k_out, x.k_row, x.k_head, x.k_out_row, x.k_out_head};
  a.hq = x.hq;
  a.heads = x.hq + x.hk;
  a.half = x.rot_dim / 2;
  a.positions = x.positions;
  a.row_count = x.row_count;
  a.inv_freq = x.inv_freq;
  a.scale = x.scale;
  a.num_rows = x.num_rows;
  a.status = x.status;
  const auto whole = [](const RopeSide& s) {
    return ((reinterpret_cast<uintptr_t>(s.x) | reinterpret_cast<uintptr_t>(s.y)) & 15u) == 0 &&
           ((s.x_row | s.x_head | s.y_row | s.y_head) & 7) == 0;
  };
  const bool wide = x.rot_dim % 16 == 0 && (x.hq == 0 || whole(a.q)) && (x.hk == 0 || whole(a.k));
  const bool inter = x.layout == ECHO_ROPE_INTERLEAVED;
  // With few rows, a row's items over up to as many workgroups as it has rounds of threads.
  const long long items = (long long)a.heads * (wide ? a.half / 8 : a.half);
  const long long rounds = (items + kRopeThreads - 1) / kRopeThreads;
  long long parts = kRopeFill / x.num_rows;
  parts = parts < 1 ? 1 : parts > rounds ? rounds : parts;
  a.share = int((rounds + parts - 1) / parts) * kRopeThreads;
  parts = (items + a.share - 1) / a.share;
  hipLaunchKernelGGL(wide ? (inter ? rope_kernel<true, true> : rope_kernel<true, false>)
                          : (inter ? rope_kernel<false, true> : rope_kernel<false, false>),
                     dim3(unsigned(x.num_rows), unsigned(parts)), dim3(kRopeThreads), size_t(a.half) * sizeof(float2), stream, a);
  return hipGetLastError() == hipSuccess ? ECHO_OK : ECHO_ERR_HIP;
}

}  // namespace echo
