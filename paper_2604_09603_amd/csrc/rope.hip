// Rotary positions of queries and keys (rope_device.h has the rotation), one launch for both.
//
// A workgroup has a row, a few where there are many short ones, or with few rows a share of one's
// heads: first the turns of its rows' pairs, once for all heads, into LDS; then its
// threads go through the heads, 16 dims at a time (two 16-byte loads and stores: eight
// pairs of either layout), the first of which is on its way while the turns are
// formed.  What is only 8-byte aligned, or a rotated part that is a multiple of 8 but not of
// 16, goes eight dims at a time, the rest pair by pair.
//
// Bound by memory: four bytes are moved for three operations.  40000 rows of 40 heads of 128 dims,
// 819 MB, take 138-142 us (5.8-5.9 TB/s; a copy of 1 GB reaches 5.2); 384 rows of 68 heads
// 3.7 us in a captured graph, of which an empty launch is about two, and 11.5 us as
// an eager call, the host's part.
#include "echo_device.h"
#include "echo_internal.h"
#include "rope_device.h"

namespace echo {
namespace {

constexpr int kRopeThreads = 256;
// Workgroups at a time: eight of 256 threads on each of 256 CUs.  384 rows of 68 heads take 4.4 us
// with a workgroup per row, 3.6 with two rounds of threads' items shared by two and the
// loads beside the turns; 17449 rows of 17 heads of 24 dims 9.4 us with five rows a workgroup
// and eight dims at a time, 18.1 with one and pair by pair.
constexpr int kRopeFill = 2048;

template <int kPairs>
struct RopeVec;
template <>
struct RopeVec<8> {
  typedef uint4 type;
};
template <>
struct RopeVec<4> {
  typedef uint2 type;
};
template <>
struct RopeVec<1> {
  typedef uint16_t type;
};

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
  int num_rows, rows_wg, share;  // a workgroup's rows, or the items it has of one
  int32_t* status;
};

// An item: kPairs pairs of a head.
template <int kPairs, bool kInterleaved>
__global__ __launch_bounds__(kRopeThreads) void rope_kernel(RopeKernelArgs a) {
  typedef typename RopeVec<kPairs>::type Vec;  // kPairs values
  extern __shared__ __attribute__((aligned(16))) float2 s_turn[];  // [rows_wg][half]
  const int tid = threadIdx.x;
  const int n = rope_rows(a.row_count, a.num_rows);
  if (n < 0) {
    if (blockIdx.x == 0 && blockIdx.y == 0 && tid == 0) status_or(a.status, ECHO_DATA_BAD_OFFSETS);
    return;
  }
  const int row0 = int(blockIdx.x) * a.rows_wg;
  if (row0 >= n) return;
  const int rows = min(a.rows_wg, n - row0);
  const int per = a.half / kPairs, items = a.heads * per;  // of a head, of a row
  const int first = int(blockIdx.y) * a.share;
  const int last = a.rows_wg > 1 ? rows * items : min(first + a.share, items);
  struct Item {
    uint16_t* y;
    const float2* cs;
    Vec a, b;
  };
  // the values of an item: in either layout two vectors, step apart
  const int step = kInterleaved ? kPairs : a.half;
  const auto load = [&](int it) {
    const int r = a.rows_wg > 1 ? it / items : 0;
    it -= r * items;
    const int head = it / per, c = (it - head * per) * kPairs;
    const bool is_q = head < a.hq;
    const RopeSide& side = is_q ? a.q : a.k;
    const long long hd = is_q ? head : head - a.hq, row = row0 + r;
    const int at = kInterleaved ? 2 * c : c;
    const uint16_t* x = side.x + row * side.x_row + hd * side.x_head + at;
    Item i;
    i.y = side.y + row * side.y_row + hd * side.y_head + at;
    i.cs = s_turn + r * a.half + c;
    i.a = *reinterpret_cast<const Vec*>(x);
    i.b = *reinterpret_cast<const Vec*>(x + step);
    return i;
  };
  int it = first + tid;
  Item i = {};
  if (it < last) i = load(it);
  for (int t = tid; t < rows * a.half; t += kRopeThreads) {
    const int r = a.rows_wg > 1 ? t / a.half : 0;
    s_turn[t] = rope_turn(a.positions[row0 + r], a.inv_freq[t - r * a.half], a.scale);
  }
  __syncthreads();
  while (it < last) {
    if constexpr (kPairs == 1) {
      const float2 o = rope_pair(bf16_lo(i.a), bf16_lo(i.b), *i.cs);
      const uint32_t w = rope_pack(o.x, o.y);
      i.y[0] = uint16_t(w);
      i.y[step] = uint16_t(w >> 16);
    } else {
      constexpr int kWords = kPairs / 2;
      typedef uint32_t Words __attribute__((ext_vector_type(kWords)));
      const Words wa = __builtin_bit_cast(Words, i.a), wb = __builtin_bit_cast(Words, i.b);
      Words oa, ob;
#pragma unroll
      for (int j = 0; j < kWords; ++j) {
        if (kInterleaved) {
          const float2 u = rope_pair(bf16_lo(wa[j]), bf16_hi(wa[j]), i.cs[j]);
          const float2 v = rope_pair(bf16_lo(wb[j]), bf16_hi(wb[j]), i.cs[kWords + j]);
          oa[j] = rope_pack(u.x, u.y);
          ob[j] = rope_pack(v.x, v.y);
        } else {
          const float2 u = rope_pair(bf16_lo(wa[j]), bf16_lo(wb[j]), i.cs[2 * j]);
          const float2 v = rope_pair(bf16_hi(wa[j]), bf16_hi(wb[j]), i.cs[2 * j + 1]);
          oa[j] = rope_pack(u.x, v.x);
          ob[j] = rope_pack(u.y, v.y);
        }
      }
      *reinterpret_cast<Vec*>(i.y) = __builtin_bit_cast(Vec, oa);
      *reinterpret_cast<Vec*>(i.y + step) = __builtin_bit_cast(Vec, ob);
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
  const auto whole = [&](int values) {  // whether vectors of so many are aligned everywhere
    uintptr_t p = 0;
    long long strides = 0;
    for (const RopeSide* s : {x.hq > 0 ? &a.q : nullptr, x.hk > 0 ? &a.k : nullptr}) {
      if (s == nullptr) continue;
      p |= reinterpret_cast<uintptr_t>(s->x) | reinterpret_cast<uintptr_t>(s->y);
      strides |= s->x_row | s->x_head | s->y_row | s->y_head;
    }
    return x.rot_dim % (2 * values) == 0 && p % (2u * unsigned(values)) == 0 && strides % values == 0;
  };
  const int pairs = whole(8) ? 8 : whole(4) ? 4 : 1;
  const bool inter = x.layout == ECHO_ROPE_INTERLEAVED;
  const long long items = (long long)a.heads * (a.half / pairs);
  const long long rounds = (items + kRopeThreads - 1) / kRopeThreads;
  a.rows_wg = 1;
  a.share = int(items);
  long long parts = 1;
  if (x.num_rows < kRopeFill) {  // a row's items over up to as many workgroups as it has rounds of threads
    parts = kRopeFill / x.num_rows;
    parts = parts > rounds ? rounds : parts;
    a.share = int((rounds + parts - 1) / parts) * kRopeThreads;
    parts = (items + a.share - 1) / a.share;
  } else if (items <= kRopeThreads / 2) {  // as many rows as a round of threads has items for, or fewer
    const long long most = x.num_rows / kRopeFill, fit = kRopeThreads / items;
    a.rows_wg = int(fit < most ? fit : most);
  }
  const dim3 grid(unsigned((x.num_rows + a.rows_wg - 1) / a.rows_wg), unsigned(parts));
  const size_t lds = size_t(a.rows_wg) * size_t(a.half) * sizeof(float2);
  void (*const kernels[3][2])(RopeKernelArgs) = {{rope_kernel<8, false>, rope_kernel<8, true>},
                                                 {rope_kernel<4, false>, rope_kernel<4, true>},
                                                 {rope_kernel<1, false>, rope_kernel<1, true>}};
  hipLaunchKernelGGL(kernels[pairs == 8 ? 0 : pairs == 4 ? 1 : 2][inter], grid, dim3(kRopeThreads), lds, stream, a);
  return hipGetLastError() == hipSuccess ? ECHO_OK : ECHO_ERR_HIP;
}

}  // namespace echo
