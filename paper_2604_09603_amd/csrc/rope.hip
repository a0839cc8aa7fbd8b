// Rotary positions of queries and keys (rope_device.h has the rotation), one launch for both.
//
// A workgroup has a few rows: first the turns of its rows' pairs, once for all heads, into
// LDS; then its threads go through the heads of its rows, 16 dims at a time (two 16-byte loads
// and stores: eight pairs of either layout).  What is not 16-byte aligned, or whose rotated
// part is no multiple of 16, goes pair by pair.
#include "echo_device.h"
#include "echo_internal.h"
#include "rope_device.h"

namespace echo {
namespace {

constexpr int kRopeThreads = 256;

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
  int num_rows, rows_wg;
  int32_t* status;
};

// kWide: items of 16 dims, else of one pair.
template <bool kWide, bool kInterleaved>
__global__ __launch_bounds__(kRopeThreads) void rope_kernel(RopeKernelArgs a) {
  extern __shared__ __attribute__((aligned(16))) float2 s_turn[];  // [rows_wg][half]
  const int tid = threadIdx.x;
  const int n = rope_rows(a.row_count, a.num_rows);
  if (n < 0) {
    if (blockIdx.x == 0 && tid == 0) status_or(a.status, ECHO_DATA_BAD_OFFSETS);
    return;
  }
  const int row0 = int(blockIdx.x) * a.rows_wg;
  if (row0 >= n) return;
  const int rows = min(a.rows_wg, n - row0);
  for (int t = tid; t < rows * a.half; t += kRopeThreads) {
    const int row = t / a.half;
    s_turn[t] = rope_turn(a.positions[row0 + row], a.inv_freq[t - row * a.half], a.scale);
  }
  __syncthreads();
  const int per = kWide ? a.half / 8 : a.half;  // items of a head
  const int items = rows * a.heads * per;
  for (int it = tid; it < items; it += kRopeThreads) {
    const int h = it / per, c = it - h * per;
    const int row = h / a.heads, head = h - row * a.heads;
    const bool is_q = head < a.hq;
    const RopeSide& side = is_q ? a.q : a.k;
    const long long hd = is_q ? head : head - a.hq;
    const uint16_t* x = side.x + (row0 + row) * side.x_row + hd * side.x_head;
    uint16_t* y = side.y + (row0 + row) * side.y_row + hd * side.y_head;
    const float2* cs = s_turn + row * a.half + (kWide ? 8 * c : c);
    if (!kWide) {
      const int ia = kInterleaved ? 2 * c : c, ib = kInterleaved ? 2 * c + 1 : c + a.half;
      const float2 o = rope_pair(bf16_lo(x[ia]), bf16_lo(x[ib]), *cs);
      const uint32_t w = rope_pack(o.x, o.y);
      y[ia] = uint16_t(w);
      y[ib] = uint16_t(w >> 16);
      continue;
    }
    const int ia = kInterleaved ? 16 * c : 8 * c, ib = kInterleaved ? 16 * c + 8 : 8 * c + a.half;
    const uint4 va = *reinterpret_cast<const uint4*>(x + ia), vb = *reinterpret_cast<const uint4*>(x + ib);
    const uint32_t wa[4] = {va.x, va.y, va.z, va.w}, wb[4] = {vb.x, vb.y, vb.z, vb.w};
    uint32_t oa[4], ob[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (kInterleaved) {
        const float2 u = rope_pair(bf16_lo(wa[i]), bf16_hi(wa[i]), cs[i]);
        const float2 v = rope_pair(bf16_lo(wb[i]), bf16_hi(wb[i]), cs[4 + i]);
        oa[i] = rope_pack(u.x, u.y);
        ob[i] = rope_pack(v.x, v.y);
      } else {
        const float2 u = rope_pair(bf16_lo(wa[i]), bf16_lo(wb[i]), cs[2 * i]);
        const float2 v = rope_pair(bf16_hi(wa[i]), bf16_hi(wb[i]), cs[2 * i + 1]);
        oa[i] = rope_pack(u.x, v.x);
        ob[i] = rope_pack(u.y, v.y);
      }
    }
    *reinterpret_cast<uint4*>(y + ia) = make_uint4(oa[0], oa[1], oa[2], oa[3]);
    *reinterpret_cast<uint4*>(y + ib) = make_uint4(ob[0], ob[1], ob[2], ob[3]);
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
  a.rows_wg = 1;
  a.status = x.status;
  const auto whole = [](const RopeSide& s) {
    return ((reinterpret_cast<uintptr_t>(s.x) | reinterpret_cast<uintptr_t>(s.y)) & 15u) == 0 &&
           ((s.x_row | s.x_head | s.y_row | s.y_head) & 7) == 0;
  };
  const bool wide = x.rot_dim % 16 == 0 && (x.hq == 0 || whole(a.q)) && (x.hk == 0 || whole(a.k));
  const bool inter = x.layout == ECHO_ROPE_INTERLEAVED;
  const unsigned wgs = unsigned((x.num_rows + a.rows_wg - 1) / a.rows_wg);
  const size_t lds = size_t(a.rows_wg) * size_t(a.half) * sizeof(float2);
  hipLaunchKernelGGL(wide ? (inter ? rope_kernel<true, true> : rope_kernel<true, false>)
                          : (inter ? rope_kernel<false, true> : rope_kernel<false, false>),
                     dim3(wgs), dim3(kRopeThreads), lds, stream, a);
  return hipGetLastError() == hipSuccess ? ECHO_OK : ECHO_ERR_HIP;
}

}  // namespace echo
