// Tree-masked grouped-query verification attention over an 8-bit paged cache
// (kvq8_device.h has the cache's layout).  Three launches, and one more before them
// for large block tables:
//
//   q8_pages    checks the page ids (small tables: the plan does).
//   q8_plan     one workgroup.  A unit is one KV head of one request with up to 64 of
//               its rows (verify slots x query heads of the GQA group); its tiles
//               are first the tree's (32 new keys each), then the prefix's, one
//               32-token block each.  The tiles of all units are cut into equal
//               contiguous ranges, one per wave of the main kernel: a head's blocks
//               lie in one piece, so nothing is gained by waves that read the heads
//               of the same tokens side by side, and one head's keys are spread over
//               as many waves as they can feed.
//   q8_main     persistent, one workgroup of four independent waves per CU.  A wave
//               copies its tiles HBM -> LDS into a ring of its own with direct-to-LDS
//               loads, converts a tile to bfloat16 (exact) and multiplies it with
//               all rows of the unit: S^T = K Q^T and O^T = V^T P^T on
//               v_mfma_f32_16x16x32_bf16 with an online softmax in base 2.  The K
//               scale goes into the softmax's factor, the V scale into its exponent.
//   q8_combine  merges the partial sums of units that several waves share.
//
// Softmax statistics and sums are fp32.  The weights p are rounded to bfloat16 for
// the product with V (at most 2^-8 each) and the output is divided by the sum of the
// weights used, so that it stays a convex combination of V rows; the output's own
// rounding to bfloat16 is as large, so the residuals of the weights are not
// multiplied.  Partial sums are stored as fp16 with a power-of-two scale per row
// (at most 2^-11 of the row's largest).
#include <type_traits>

#include "attn_core.h"
#include "kvq8_device.h"

namespace echo {
namespace {

constexpr int kQ8Rows = 64;        // rows per unit
constexpr int kQ8Waves = 4;        // waves per workgroup and CU
constexpr int kQ8Stages = 4;       // tiles in a wave's ring
constexpr int kQ8ScaleOff = 2 * kBlockBytes;      // a stage: K, V, then the two scales
constexpr int kQ8StageBytes = 2 * kBlockBytes + 256;
constexpr int kQ8Scratch = 16 * kD * 2;           // 16 rows of bfloat16 V (tree tiles)
constexpr int kQ8WaveLds = kQ8Stages * kQ8StageBytes + kQ8Scratch;
static_assert(kQ8Waves * kQ8WaveLds <= 160 * 1024, "gfx950 LDS per workgroup");
constexpr int kQ8Copies = 9;       // copy instructions per tile: 4 of K, 4 of V, the scales
constexpr int kPlanThreads = 1024;
constexpr int kPlanPages = 8 * kPlanThreads;      // block-table entries the plan checks itself

typedef int intx2 __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) intx2 lds_intx2_t;

// One request as the plan shapes it: `units` = Hkv * passes units of tpu tiles from tile0
// on (unit = head * passes + pass), ntail of each unit's tiles are the tree's.
struct Q8Req {
  int32_t tile0, tpu;
  int32_t q0, nslots;
  int32_t P, passes, rpp, ntail;
};

// A wave's range of tiles and where it starts.  cut_last: if the range's first tile lies
// inside a unit, and is the first range start that does, the last wave of that unit
// (else 0): the unit's sums are merged from waves b - 1 .. cut_last.
struct Q8Start {
  int32_t lo, hi, r, unit;
  int32_t cut_last, pad[3];
  Q8Req q;
};
static_assert(sizeof(Q8Start) == 64, "one 64-byte record");

struct Q8Ws {
  Q8Start* starts;   // [waves]
  Q8Req* reqs;       // [R]
  int32_t* bad;      // [R][chunks] flags of q8_pages
  float* part_ml;    // [waves][2][64][4]: max, sum, sum of the weights used, scale exponent
  _Float16* part_o;  // [waves][2][64][128]
};

struct Q8Args {
  const uint16_t* q;
  const uint16_t* k_new;
  const uint16_t* v_new;
  const uint8_t* k_pages;
  const uint8_t* v_pages;
  const float* k_scale;
  const float* v_scale;
  const int32_t* block_table;
  const int32_t* prefix_len;
  const int32_t* q_offsets;
  const uint32_t* tree_mask;
  long long num_pages;
  int page_shift, max_pages, W, R, max_rows, hq, hkv, G;
  float scale2;
  uint16_t* out;
  float* lse;
  int32_t* status;
};

__host__ __device__ inline int q8_page_chunks(int max_pages) {
  return (max_pages + kPageChunk - 1) / kPageChunk;
}

__host__ inline bool q8_plan_checks(int R, int max_pages) {
  return (long long)R * max_pages <= kPlanPages;
}

__host__ inline Q8Ws q8_layout(void* base, int R, int max_pages, int nw, size_t* bytes) {
  char* p = static_cast<char*>(base);
  Q8Ws w;
  w.starts = reinterpret_cast<Q8Start*>(p);
  p += al(size_t(nw) * sizeof(Q8Start));
  w.reqs = reinterpret_cast<Q8Req*>(p);
  p += al(size_t(R) * sizeof(Q8Req));
  w.bad = reinterpret_cast<int32_t*>(p);
  if (!q8_plan_checks(R, max_pages)) p += al(size_t(R) * size_t(q8_page_chunks(max_pages)) * 4);
  w.part_ml = reinterpret_cast<float*>(p);
  p += al(size_t(nw) * 2 * kQ8Rows * 4 * sizeof(float));
  w.part_o = reinterpret_cast<_Float16*>(p);
  p += al(size_t(nw) * 2 * kQ8Rows * kD * sizeof(_Float16));
  if (bytes != nullptr) *bytes = size_t(p - static_cast<char*>(base));
  return w;
}

int q8_waves() { return device_cu_count() * kQ8Waves; }

// Pages of a request's prefix, or -1 if its length does not fit its table row.
__device__ __forceinline__ int prefix_pages(long long P, const Q8Args& a) {
  if (P < 0 || P > ((long long)a.max_pages << a.page_shift)) return -1;
  return int((P + (1 << a.page_shift) - 1) >> a.page_shift);
}

__global__ __launch_bounds__(kPageChunk) void q8_pages_kernel(Q8Args a, int32_t* bad_flags) {
  const int r = blockIdx.x, c = blockIdx.y;
  const int np = prefix_pages(a.prefix_len[r], a);
  const int e = c * kPageChunk + int(threadIdx.x);
  int bad = 0;
  if (e < np) {
    const int pg = a.block_table[size_t(r) * size_t(a.max_pages) + size_t(e)];
    bad = pg < 0 || pg >= a.num_pages;
  }
  bad = __syncthreads_or(bad);
  if (threadIdx.x == 0) bad_flags[size_t(r) * gridDim.y + c] = bad;
}

// ---------------------------------------------------------------- plan ----
__device__ __forceinline__ Q8Req shape_of(const Q8Args& a, int r, bool ok) {
  Q8Req s = {};
  if (!ok) return s;
  s.q0 = a.q_offsets[r];
  s.nslots = a.q_offsets[r + 1] - s.q0;
  s.P = a.prefix_len[r];
  const int rows = s.nslots * a.G;
  s.passes = (rows + kQ8Rows - 1) / kQ8Rows;
  if (s.passes == 0) return s;
  s.rpp = (rows + s.passes - 1) / s.passes;
  s.ntail = (s.nslots + kTileKeys - 1) / kTileKeys;
  s.tpu = s.ntail + int(((long long)s.P + kTileKeys - 1) / kTileKeys);
  return s;
}

__global__ __launch_bounds__(kPlanThreads) void q8_plan_kernel(Q8Args a, Q8Ws ws, int nw_max,
                                                               int chunks) {
  extern __shared__ int32_t s_tile0[];  // R + 1: first tile of each request
  __shared__ uint8_t s_bad[ECHO_MAX_REQUESTS + 1];
  __shared__ long long s_total[kPlanThreads / kWave + 1];
  __shared__ int s_scan[kPlanThreads / kWave + 1];
  const int tid = threadIdx.x;
  const int R = a.R;
  int bits = 0;
  // requests whose offsets, length or pages cannot be used
  const bool own = chunks == 0;
  int pg[8];
  if (own) {  // every load in flight at once
    const long long total = (long long)R * a.max_pages;
#pragma unroll
    for (int k = 0; k < 8; ++k)
      pg[k] = a.block_table[min((long long)tid + k * kPlanThreads, total - 1)];
  }
  for (int r = tid; r < R; r += kPlanThreads) {
    const int q0 = a.q_offsets[r], q1 = a.q_offsets[r + 1];
    bool bad = !(q0 >= 0 && q1 >= q0 && q1 <= a.max_rows) || prefix_pages(a.prefix_len[r], a) < 0;
    for (int c = 0; c < chunks; ++c) bad = bad || ws.bad[size_t(r) * chunks + c] != 0;
    s_bad[r] = bad ? 1 : 0;
  }
  __syncthreads();
  if (own) {
    const long long total = (long long)R * a.max_pages;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const long long e = (long long)tid + k * kPlanThreads;
      if (e < total && (pg[k] < 0 || pg[k] >= a.num_pages)) {
        const int r = int(e / a.max_pages), c = int(e % a.max_pages);
        if (c < prefix_pages(a.prefix_len[r], a)) s_bad[r] = 1;
      }
    }
    __syncthreads();
  }
  // tiles of every request; 64-bit first, as offsets that overlap may ask for any number
  long long mine = 0;
  for (int r = tid; r < R; r += kPlanThreads) {
    if (s_bad[r]) bits |= ECHO_DATA_BAD_OFFSETS;
    const Q8Req s = shape_of(a, r, !s_bad[r]);
    mine += (long long)a.hkv * s.passes * s.tpu;
  }
  for (int d = kWave / 2; d > 0; d >>= 1) mine += __shfl_xor(mine, d);
  if ((tid & (kWave - 1)) == 0) s_total[tid / kWave] = mine;
  __syncthreads();
  long long T = 0;
  for (int k = 0; k < kPlanThreads / kWave; ++k) T += s_total[k];
  if (T > 0x7FFFFFFFll) {
    bits |= ECHO_DATA_BAD_OFFSETS;
    T = 0;
  }
  wave_status_or(a.status, bits);
  const int nw = T < nw_max ? int(T) : nw_max;
  for (int b = nw + tid; b < nw_max; b += kPlanThreads) ws.starts[b] = Q8Start{};
  if (T == 0) return;
  int run = 0;
  for (int base = 0; base < R; base += kPlanThreads) {
    const int r = base + tid;
    Q8Req s = {};
    if (r < R) s = shape_of(a, r, !s_bad[r]);
    int tot;
    const int ex = block_exclusive_sum<kPlanThreads>(a.hkv * s.passes * s.tpu, s_scan, &tot);
    s.tile0 = run + ex;
    if (r < R) {
      s_tile0[r] = s.tile0;
      ws.reqs[r] = s;
    }
    run += tot;
  }
  if (tid == 0) s_tile0[R] = run;
  __syncthreads();
  const DivBy by_t(T), by_nw(nw);
  for (int b = tid; b < nw; b += kPlanThreads) {
    Q8Start st = {};
    st.lo = int(range_lo(T, b, by_nw));
    st.hi = int(range_lo(T, b + 1, by_nw));
    st.r = upper_bound_idx(s_tile0, R + 1, st.lo);
    st.q = shape_of(a, st.r, true);
    st.q.tile0 = s_tile0[st.r];
    st.unit = (st.lo - st.q.tile0) / st.q.tpu;
    const int u0 = st.q.tile0 + st.unit * st.q.tpu;
    if (u0 < st.lo && int(range_lo(T, b - 1, by_nw)) <= u0)
      st.cut_last = range_of((long long)u0 + st.q.tpu - 1, T, nw, by_t);
    ws.starts[b] = st;
  }
}

// ---------------------------------------------------------------- main ----
// A tile in LDS: 32 rows x 128 bytes per tensor.  The 16-byte chunk c of row r is at chunk
// position c ^ f(r), f(r) = ((r >> 1) ^ 4 (r >> 4)) & 7: the 16 rows of a K read (one
// chunk each), and the 16 rows that half a wave's transposed V read takes one chunk
// of (rows 8 g .. 8 g + 7 and 16 more), fall into 16 different sixteenths of the banks.
__device__ __forceinline__ int q8_swz(int row) { return ((row >> 1) ^ ((row >> 4) << 2)) & 7; }

template <int N>
__device__ __forceinline__ void q8_wait(int later) {  // later < N tiles may still be in flight
  if (N > 1 && later >= N - 1) wait_vm<(N - 1) * kQ8Copies>();
  else if constexpr (N > 1) q8_wait<N - 1>(later);
  else wait_vm<0>();
  asm volatile("" ::: "memory");  // the tile's reads stay behind the wait
}

// Every LDS read so far has its data (and stays ahead of what follows).
__device__ __forceinline__ void q8_wait_lds() {
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
}

// Copies one tile into the stage at LDS address lds: K, V and the scales.  Lane offsets
// offa (rows 0-7 and 24-31 of a tile) and offb (rows 8-23) of a full tile; the
// instructions' offset moves both addresses.  In inline assembly because the compiler
// would wait for every copy in flight before each LDS read; M0 (the LDS address) is the
// compiler's and is restored, and needs a wait state before a load reads it.
__device__ __forceinline__ void q8_copy(uint32_t lds, uint64_t kb, uint64_t vb, uint32_t offa,
                                        uint32_t offb, uint64_t scale) {
  uint32_t saved;
  asm volatile(
      "s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\t"
      "global_load_lds_dwordx4 %2, %4 nt\n\t"
      "global_load_lds_dwordx4 %3, %4 offset:1024 nt\n\t"
      "global_load_lds_dwordx4 %3, %4 offset:2048 nt\n\t"
      "global_load_lds_dwordx4 %2, %4 offset:3072 nt\n\t"
      "s_add_u32 m0, m0, 0x1000\n\ts_nop 0\n\t"
      "global_load_lds_dwordx4 %2, %5 nt\n\t"
      "global_load_lds_dwordx4 %3, %5 offset:1024 nt\n\t"
      "global_load_lds_dwordx4 %3, %5 offset:2048 nt\n\t"
      "global_load_lds_dwordx4 %2, %5 offset:3072 nt\n\t"
      "s_add_u32 m0, m0, 0x1000\n\ts_nop 0\n\t"
      "global_load_lds_dword %6, off\n\t"
      "s_mov_b32 m0, %0"
      : "=&s"(saved)
      : "s"(lds), "v"(offa), "v"(offb), "s"(kb), "s"(vb), "v"(scale)
      : "memory", "scc");
}

// The same with an offset for each group of eight rows (a tile whose last rows hold no
// tokens: they read its last token's row again, so that nothing unwritten is
// multiplied, and are masked).
__device__ __forceinline__ void q8_copy_part(uint32_t lds, uint64_t kb, uint64_t vb, uint32_t o0,
                                             uint32_t o1, uint32_t o2, uint32_t o3,
                                             uint64_t scale) {
  uint32_t saved;
  asm volatile(
      "s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %2, %6\n\t"
      "s_add_u32 m0, m0, 0x400\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %3, %6\n\t"
      "s_add_u32 m0, m0, 0x400\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %4, %6\n\t"
      "s_add_u32 m0, m0, 0x400\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %5, %6\n\t"
      "s_add_u32 m0, m0, 0x400\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %2, %7\n\t"
      "s_add_u32 m0, m0, 0x400\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %3, %7\n\t"
      "s_add_u32 m0, m0, 0x400\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %4, %7\n\t"
      "s_add_u32 m0, m0, 0x400\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %5, %7\n\t"
      "s_add_u32 m0, m0, 0x400\n\ts_nop 0\n\tglobal_load_lds_dword %8, off\n\t"
      "s_mov_b32 m0, %0"
      : "=&s"(saved)
      : "s"(lds), "v"(o0), "v"(o1), "v"(o2), "v"(o3), "s"(kb), "s"(vb), "v"(scale)
      : "memory", "scc");
}

__device__ __forceinline__ Q8Req load_req(const Q8Req* reqs, int r) {
  const_i32_t* p = (const_i32_t*)(reqs + r);
  int32_t w[8];
#pragma unroll
  for (int k = 0; k < 8; ++k) w[k] = p[k];
  return __builtin_bit_cast(Q8Req, w);
}

__device__ __forceinline__ Q8Start load_start(const Q8Start* starts, int b) {
  const_i32_t* p = (const_i32_t*)(starts + b);
  int32_t w[16];
#pragma unroll
  for (int k = 0; k < 16; ++k) w[k] = p[k];
  return __builtin_bit_cast(Q8Start, w);
}

// A place in the tile stream (wave-uniform): the unit and its first tile.
struct Q8Walk {
  Q8Req q;
  int r, unit, u0;
};

__device__ __forceinline__ void q8_next_unit(Q8Walk& w, const Q8Args& a, const Q8Ws& ws) {
  if (w.unit + 1 < a.hkv * w.q.passes) {
    w.unit += 1;
    w.u0 += w.q.tpu;
    return;
  }
  while (w.r + 1 < a.R) {
    w.r = __builtin_amdgcn_readfirstlane(w.r + 1);
    w.q = load_req(ws.reqs, w.r);
    if (w.q.passes > 0) break;
  }
  w.unit = 0;
  w.u0 = w.q.tile0;
}

// The copy side: `t` is the next tile to look at, `sent` the prefix tiles copied so far.
struct Q8Issue {
  Q8Walk w;
  int t, sent;
};

__device__ __forceinline__ void q8_send(Q8Issue& is, const Q8Args& a, const Q8Ws& ws, int hi,
                                        uint32_t ring, uint32_t offa, uint32_t offb,
                                        uint64_t scale_base) {
  while (is.t < hi) {
    if (is.t >= is.w.u0 + is.w.q.tpu) q8_next_unit(is.w, a, ws);
    else if (is.t - is.w.u0 < is.w.q.ntail) is.t = min(hi, is.w.u0 + is.w.q.ntail);
    else break;
  }
  if (is.t >= hi) return;
  const int key = (is.t - is.w.u0 - is.w.q.ntail) * kTileKeys;
  const int head = is.w.unit / is.w.q.passes;
  const int page = ((const const_i32_t*)(a.block_table + size_t(is.w.r) * size_t(a.max_pages)))
      [key >> a.page_shift];
  const uint64_t blk =
      ((uint64_t(page) * uint32_t(a.hkv) + uint32_t(head)) << (a.page_shift - 5)) +
      uint32_t((key & ((1 << a.page_shift) - 1)) >> 5);
  const uint64_t kb = uniform64(reinterpret_cast<uint64_t>(a.k_pages) + blk * kBlockBytes);
  const uint64_t vb = uniform64(reinterpret_cast<uint64_t>(a.v_pages) + blk * kBlockBytes);
  const uint32_t lds = __builtin_amdgcn_readfirstlane(
      ring + uint32_t((is.sent & (kQ8Stages - 1)) * kQ8StageBytes));
  const uint64_t scale = scale_base + blk * 4;
  const int tn = is.w.q.P - key;
  if (tn >= kTileKeys) {
    q8_copy(lds, kb, vb, offa, offb, scale);
  } else {
    const int lane = threadIdx.x & (kWave - 1);
    uint32_t o[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int row = 8 * j + (lane >> 3);
      o[j] = uint32_t(min(row, tn - 1) * kD + (((lane & 7) ^ q8_swz(row)) << 4));
    }
    q8_copy_part(lds, kb, vb, o[0], o[1], o[2], o[3], scale);
  }
  is.t += 1;
  is.sent += 1;
}

template <int kFmt>
__device__ __forceinline__ bf16x8 widen8(uint32_t lo, uint32_t hi) {
  bf16x2 a, b, c, d;
  if (kFmt == ECHO_KV_E4M3) {
    a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, false);
    b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, true);
    c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, false);
    d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, true);
  } else {
    a = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(lo, 1.0f, false);
    b = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(lo, 1.0f, true);
    c = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(hi, 1.0f, false);
    d = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(hi, 1.0f, true);
  }
  return as_bf16x8(make_uint4(__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b),
                              __builtin_bit_cast(uint32_t, c), __builtin_bit_cast(uint32_t, d)));
}

// Maximum and sum over the four lanes of a row (l, l ^ 16, l ^ 32, l ^ 48).
__device__ __forceinline__ float quad_max(float v) {
  const uint32_t u = __float_as_uint(v);
  const auto a = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  v = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  const uint32_t w = __float_as_uint(v);
  const auto b = __builtin_amdgcn_permlane32_swap(w, w, false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float quad_sum(float v) {
  const uint32_t u = __float_as_uint(v);
  const auto a = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  v = __uint_as_float(a[0]) + __uint_as_float(a[1]);
  const uint32_t w = __float_as_uint(v);
  const auto b = __builtin_amdgcn_permlane32_swap(w, w, false, false);
  return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

// 16 rows: O^T (lane: dims 16 dt + 4 (lane / 16) + i of row lane % 16) and the softmax's
// state, of which each of the row's four lanes has its share of the sums.
struct Q8Rows {
  floatx4 o[8];
  float m;      // reference maximum (log2 units)
  float l, lq;  // sums of the weights, and of the weights as multiplied with V
  float mgrow;  // a logit above it raises the reference
};

// What a tile's products take: K and V^T fragments.  K fragment kk (0..3) of 16 keys: lane
// holds dims 64 (kk >> 1) + 16 (lane / 16) + 8 (kk & 1) .. + 7 of key lane % 16 (the
// order of dims that two 16-byte reads give; Q is loaded in the same).  V^T
// fragment dt: dim 16 dt + lane % 16 of keys 4 (lane / 16) + 0..3 and the same + 16: the
// order in which S^T leaves the keys in the lanes.

// Scores to weights: S^T of 16 rows (two subtiles of 16 keys), c = softmax factor x K
// scale, lvs = log2 of V's scale, which the weights take along (ivs takes it out of
// the sums again).  word: bit k set iff the row sees key k.
__device__ __forceinline__ bf16x8 q8_softmax(floatx4 s0, floatx4 s1, Q8Rows& rt, bool masked,
                                             uint32_t word, float c, float lvs, float ivs) {
  float sv[8] = {s0[0], s0[1], s0[2], s0[3], s1[0], s1[1], s1[2], s1[3]};
  if (masked) {
    const uint32_t w = word >> (4 * ((threadIdx.x & (kWave - 1)) >> 4));
#pragma unroll
    for (int e = 0; e < 8; ++e)
      sv[e] = ((w >> (16 * (e >> 2) + (e & 3))) & 1u) ? sv[e] : -__builtin_inff();
  }
  const float lmt = fmaxf(fmaxf(fmaxf(sv[0], sv[1]), fmaxf(sv[2], sv[3])),
                          fmaxf(fmaxf(sv[4], sv[5]), fmaxf(sv[6], sv[7]))) * c;
  // the reference is raised only when a logit exceeds it by more than 2^8, so that
  // weights stay <= 256
  if (__ballot(lmt > rt.mgrow) != 0ull) {
    const float mt = quad_max(lmt);
    const bool grow = mt > rt.mgrow;
    const float alpha = grow ? __builtin_amdgcn_exp2f(rt.m - mt) : 1.0f;  // 0 from -inf
    rt.l *= alpha;
    rt.lq *= alpha;
#pragma unroll
    for (int dt = 0; dt < 8; ++dt) rt.o[dt] *= alpha;
    rt.m = grow ? mt : rt.m;
    rt.mgrow = rt.m + kRescaleSlack;
  }
  const float off = lvs - (rt.m == -__builtin_inff() ? 0.0f : rt.m);
  float sum = 0.0f;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    sv[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(sv[e], c, off));
    sum += sv[e];
  }
  uint4 pk;
  pk.x = pack_bf16x2(sv[0], sv[1]);
  pk.y = pack_bf16x2(sv[2], sv[3]);
  pk.z = pack_bf16x2(sv[4], sv[5]);
  pk.w = pack_bf16x2(sv[6], sv[7]);
  const float used = add_bf16x2(pk.w, add_bf16x2(pk.z, add_bf16x2(pk.y, add_bf16x2(pk.x, 0.0f))));
  rt.l = __builtin_fmaf(sum, ivs, rt.l);
  rt.lq = __builtin_fmaf(used, ivs, rt.lq);
  return as_bf16x8(pk);
}

// One tile against MT row tiles.  kf(s2, kk), vf(dt): its fragments.
template <int MT, typename KF, typename VF>
__device__ __forceinline__ void q8_tile(const KF& kf, const VF& vf, const bf16x8 (*qf)[4],
                                        Q8Rows* rt, bool masked, const uint32_t* word, float c,
                                        float lvs, float ivs) {
  floatx4 st[MT][2];
#pragma unroll
  for (int s2 = 0; s2 < 2; ++s2)
#pragma unroll
    for (int kk = 0; kk < 4; ++kk) {
      const bf16x8 f = kf(s2, kk);
#pragma unroll
      for (int i = 0; i < MT; ++i)
        st[i][s2] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
            f, qf[i][kk], kk == 0 ? floatx4{0.f, 0.f, 0.f, 0.f} : st[i][s2], 0, 0, 0);
    }
  bf16x8 pf[MT];
#pragma unroll
  for (int i = 0; i < MT; ++i)
    pf[i] = q8_softmax(st[i][0], st[i][1], rt[i], masked, word[i], c, lvs, ivs);
#pragma unroll
  for (int dt = 0; dt < 8; ++dt) {
    const bf16x8 f = vf(dt);
#pragma unroll
    for (int i = 0; i < MT; ++i)
      rt[i].o[dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f, pf[i], rt[i].o[dt], 0, 0, 0);
  }
}

// A tile of the tree's new keys (bfloat16, tn <= 32 of them from slot s0 on), read from
// global memory; V goes through 4 KB of LDS to be transposed, 16 keys at a time.
template <int MT>
__device__ __forceinline__ void q8_tree_tile(const Q8Args& a, int head, int s0, int tn,
                                             char* scratch, const bf16x8 (*qf)[4], Q8Rows* rt,
                                             const uint32_t* word) {
  const int lane = threadIdx.x & (kWave - 1);
  const int lr = lane & 15, lg = lane >> 4;
  const size_t row = size_t(a.hkv) * kD;
  const uint16_t* kh = a.k_new + size_t(s0) * row + size_t(head) * kD;
  const uint16_t* vh = a.v_new + size_t(s0) * row + size_t(head) * kD;
  bf16x8 kfr[2][4];
  uint4 vr[2][4];
#pragma unroll
  for (int s2 = 0; s2 < 2; ++s2) {
    const uint16_t* p = kh + size_t(min(16 * s2 + lr, tn - 1)) * row + 16 * lg;
#pragma unroll
    for (int kk = 0; kk < 4; ++kk)
      kfr[s2][kk] = as_bf16x8(
          *reinterpret_cast<const uint4*>(p + 64 * (kk >> 1) + 8 * (kk & 1)));
#pragma unroll
    for (int j = 0; j < 4; ++j)
      vr[s2][j] = *reinterpret_cast<const uint4*>(
          vh + size_t(min(16 * s2 + 4 * j + lg, tn - 1)) * row + 8 * lr);
  }
  shortx4 vt[2][8];
#pragma unroll
  for (int s2 = 0; s2 < 2; ++s2) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int r16 = 4 * j + lg;
      *reinterpret_cast<uint4*>(scratch + r16 * 256 + ((lr ^ swz_pattern(r16)) << 4)) = vr[s2][j];
    }
    q8_wait_lds();
    const int key = 4 * lg + (lr >> 2);
#pragma unroll
    for (int dt = 0; dt < 8; ++dt) {
      const int d = 16 * dt + 4 * (lr & 3);
      vt[s2][dt] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
          (lds_shortx4_t*)(scratch + key * 256 + (((d >> 3) ^ swz_pattern(key)) << 4) +
                           ((d & 4) << 1)));
    }
    q8_wait_lds();
  }
  q8_tile<MT>([&](int s2, int kk) { return kfr[s2][kk]; },
              [&](int dt) {
                return __builtin_bit_cast(bf16x8, __builtin_shufflevector(vt[0][dt], vt[1][dt], 0,
                                                                          1, 2, 3, 4, 5, 6, 7));
              },
              qf, rt, true, word, a.scale2, 0.0f, 1.0f);
}

// The wave's tiles [lo, hi) of one unit, then its output or partial sums.
template <int kFmt, int MT>
__device__ __forceinline__ void q8_segment(const Q8Args& a, const Q8Ws& ws, const Q8Walk& w, int lo,
                                           int hi, int range_hi, int b, char* lds_wave,
                                           uint32_t ring, Q8Issue& is, int& done, uint32_t offa,
                                           uint32_t offb, uint64_t scale_base, bool whole,
                                           int part_slot) {
  const int lane = threadIdx.x & (kWave - 1);
  const int lr = lane & 15, lg = lane >> 4;
  const int head = w.unit / w.q.passes;
  const int row0 = (w.unit % w.q.passes) * w.q.rpp;
  const int rows = min(w.q.rpp, w.q.nslots * a.G - row0);
  bf16x8 qf[MT][4];
  Q8Rows rt[MT];
#pragma unroll
  for (int i = 0; i < MT; ++i) {
    const int ra = row0 + 16 * i + lr;
    const int slot = w.q.q0 + ra / a.G;
    const uint16_t* p = a.q + (size_t(slot) * a.hq + size_t(head) * a.G + ra % a.G) * kD + 16 * lg;
#pragma unroll
    for (int kk = 0; kk < 4; ++kk) {
      uint4 v = make_uint4(0, 0, 0, 0);
      if (16 * i + lr < rows) v = *reinterpret_cast<const uint4*>(p + 64 * (kk >> 1) + 8 * (kk & 1));
      qf[i][kk] = as_bf16x8(v);
    }
#pragma unroll
    for (int dt = 0; dt < 8; ++dt) rt[i].o[dt] = floatx4{0.f, 0.f, 0.f, 0.f};
    rt[i].m = -__builtin_inff();
    rt[i].l = 0.0f;
    rt[i].lq = 0.0f;
    rt[i].mgrow = -__builtin_inff();
  }
  wait_vm<0>();  // no load that the compiler knows of is in flight in the loops below

  int t = lo;
  for (; t < hi && t - w.u0 < w.q.ntail; ++t) {
    const int lt = t - w.u0;
    const int tn = min(kTileKeys, w.q.nslots - lt * kTileKeys);
    uint32_t word[MT];
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      const int rho = 16 * i + lr;
      const int slot = w.q.q0 + (row0 + rho) / a.G;
      word[i] = rho < rows && lt < a.W ? a.tree_mask[size_t(slot) * a.W + lt] : 0u;
      if (tn < kTileKeys) word[i] &= (1u << tn) - 1u;
    }
    q8_tree_tile<MT>(a, head, w.q.q0 + lt * kTileKeys, tn, lds_wave + kQ8Stages * kQ8StageBytes, qf,
                     rt, word);
  }
  wait_vm<0>();

  const int kswz = q8_swz(lr);  // rows 16 apart: the same but for bit 2
  const int vkey = 4 * lg + ((lr >> 1) & 3) + ((lr >> 3) << 4);
  const int vswz = q8_swz(vkey);
  for (; t < hi; ++t) {
    q8_wait<kQ8Stages>(is.sent - done - 1);
    const char* stg = lds_wave + (done & (kQ8Stages - 1)) * kQ8StageBytes;
    uint4 kr[2][2];
    intx2 vr[8];
#pragma unroll
    for (int s2 = 0; s2 < 2; ++s2)
#pragma unroll
      for (int j = 0; j < 2; ++j)
        kr[s2][j] = *reinterpret_cast<const uint4*>(
            stg + (16 * s2 + lr) * kD + (((4 * j + lg) ^ kswz ^ (s2 << 2)) << 4));
#pragma unroll
    for (int dt = 0; dt < 8; ++dt)
      vr[dt] = __builtin_amdgcn_ds_read_tr8_b64_v2i32(
          (lds_intx2_t*)(const_cast<char*>(stg) + kBlockBytes + vkey * kD + ((dt ^ vswz) << 4) +
                         ((lr & 1) << 3)));
    const float2 scales = *reinterpret_cast<const float2*>(stg + kQ8ScaleOff);
    q8_wait_lds();
    ++done;
    // the stage is in registers: refill it while the tile is multiplied
    q8_send(is, a, ws, range_hi, ring, offa, offb, scale_base);
    const int tn = w.q.P - (t - w.u0 - w.q.ntail) * kTileKeys;
    const bool masked = tn < kTileKeys;
    uint32_t word[MT];
#pragma unroll
    for (int i = 0; i < MT; ++i) word[i] = masked ? (1u << tn) - 1u : 0xFFFFFFFFu;
    q8_tile<MT>(
        [&](int s2, int kk) {
          const uint4& v = kr[s2][kk >> 1];
          return kk & 1 ? widen8<kFmt>(v.z, v.w) : widen8<kFmt>(v.x, v.y);
        },
        [&](int dt) { return widen8<kFmt>(uint32_t(vr[dt][0]), uint32_t(vr[dt][1])); }, qf, rt,
        masked, word, a.scale2 * scales.x, __builtin_amdgcn_logf(scales.y),
        __builtin_amdgcn_rcpf(scales.y));
  }

#pragma unroll
  for (int i = 0; i < MT; ++i) {
    const float L = quad_sum(rt[i].l);
    const float Lq = quad_sum(rt[i].lq);
    const int rho = 16 * i + lr;
    if (whole) {
      if (rho < rows) {
        const int ra = row0 + rho;
        const size_t orow = size_t(w.q.q0 + ra / a.G) * a.hq + size_t(head) * a.G + ra % a.G;
        const float inv = Lq > 0.0f ? 1.0f / Lq : 0.0f;
#pragma unroll
        for (int dt = 0; dt < 8; ++dt) {
          const floatx4 v = rt[i].o[dt] * inv;
          *reinterpret_cast<uint2*>(a.out + orow * kD + 16 * dt + 4 * lg) =
              make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
        }
        if (a.lse != nullptr && lg == 0)
          a.lse[orow] = L > 0.0f ? (rt[i].m + log2f(L)) * kLn2 : -__builtin_inff();
      }
    } else {
      float mx = 0.0f;
#pragma unroll
      for (int dt = 0; dt < 8; ++dt)
#pragma unroll
        for (int c = 0; c < 4; ++c) mx = fmaxf(mx, fabsf(rt[i].o[dt][c]));
      mx = quad_max(mx);
      const int e = mx > 0.0f ? __builtin_amdgcn_frexp_expf(mx) - 15 : 0;
      if (rho < rows) {
        const float sc = __builtin_amdgcn_ldexpf(1.0f, -e);
        const size_t prow = (size_t(b) * 2 + part_slot) * kQ8Rows + rho;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const halfx4 a0 = __builtin_convertvector(rt[i].o[2 * j] * sc, halfx4);
          const halfx4 a1 = __builtin_convertvector(rt[i].o[2 * j + 1] * sc, halfx4);
          *reinterpret_cast<halfx8*>(ws.part_o + prow * kD + part_dim(32 * j + 4 * lg)) =
              halfx8{a0[0], a0[1], a0[2], a0[3], a1[0], a1[1], a1[2], a1[3]};
        }
        if (lg == 0)
          *reinterpret_cast<floatx4*>(ws.part_ml + prow * 4) = floatx4{rt[i].m, L, Lq, float(e)};
      }
    }
  }
}

template <int kFmt>
__global__ __launch_bounds__(kQ8Waves * kWave, 1) void q8_main_kernel(Q8Args a, Q8Ws ws) {
  __shared__ __attribute__((aligned(1024))) char smem[kQ8Waves * kQ8WaveLds];
  const int wid = wave_id();
  const int b = __builtin_amdgcn_readfirstlane(int(blockIdx.x) * kQ8Waves + wid);
  const Q8Start st = load_start(ws.starts, b);
  if (st.lo >= st.hi) return;  // (no barrier in this kernel: the waves are independent)
  const int lane = threadIdx.x & (kWave - 1);
  char* lds_wave = smem + wid * kQ8WaveLds;
  const uint32_t ring = __builtin_amdgcn_readfirstlane(
      uint32_t(reinterpret_cast<uintptr_t>((lds_void_t*)lds_wave)));
  // rows 0-7 of a tile (and 24-31), rows 8-15 (and 16-23): see q8_swz
  const uint32_t offa = uint32_t((lane >> 3) * kD + (((lane & 7) ^ (lane >> 4)) << 4));
  const uint32_t offb = offa ^ 64u;
  const uint64_t scale_base =
      lane == 0 ? reinterpret_cast<uint64_t>(a.k_scale) : reinterpret_cast<uint64_t>(a.v_scale);
  Q8Walk w;
  w.q = st.q;
  w.r = st.r;
  w.unit = st.unit;
  w.u0 = st.q.tile0 + st.unit * st.q.tpu;
  Q8Issue is;
  is.w = w;
  is.t = st.lo;
  is.sent = 0;
#pragma unroll 1
  for (int k = 0; k < kQ8Stages; ++k) q8_send(is, a, ws, st.hi, ring, offa, offb, scale_base);
  int done = 0;
  while (true) {
    const int lo = max(st.lo, w.u0), hi = min(st.hi, w.u0 + w.q.tpu);
    const bool whole = w.u0 >= st.lo && w.u0 + w.q.tpu <= st.hi;
    const int slot = w.u0 >= st.lo ? 1 : 0;
    const int rows = min(w.q.rpp, w.q.nslots * a.G - (w.unit % w.q.passes) * w.q.rpp);
    const auto seg = [&](auto mt) {
      q8_segment<kFmt, decltype(mt)::value>(a, ws, w, lo, hi, st.hi, b, lds_wave, ring, is, done,
                                            offa, offb, scale_base, whole, slot);
    };
    if (rows <= 16) seg(std::integral_constant<int, 1>{});
    else if (rows <= 32) seg(std::integral_constant<int, 2>{});
    else if (rows <= 48) seg(std::integral_constant<int, 3>{});
    else seg(std::integral_constant<int, 4>{});
    if (hi >= st.hi) break;
    q8_next_unit(w, a, ws);
  }
}

// ------------------------------------------------------------- combine ----
// Workgroup (b, y): rows 16 y .. 16 y + 15 of the unit that is cut first at wave b's
// range (if any); a thread has 8 dims of a row.  Parts in the order of the waves.
__global__ __launch_bounds__(256) void q8_combine_kernel(Q8Args a, Q8Ws ws) {
  const int b = blockIdx.x;
  const Q8Start st = load_start(ws.starts, b);
  if (st.cut_last == 0) return;
  const int head = st.unit / st.q.passes;
  const int row0 = (st.unit % st.q.passes) * st.q.rpp;
  const int rows = min(st.q.rpp, st.q.nslots * a.G - row0);
  const int rho = blockIdx.y * 16 + threadIdx.x / 16;
  if (rho >= rows) return;
  const int piece = threadIdx.x & 15;  // 8 halves of the partial: dims as in part_dim
  const int np = st.cut_last - b + 2;
  const auto prow = [&](int i) {
    return (size_t(b - 1 + i) * 2 + (i == 0 ? 1 : 0)) * kQ8Rows + size_t(rho);
  };
  float M = -__builtin_inff();
  for (int i = 0; i < np; ++i) M = fmaxf(M, ws.part_ml[prow(i) * 4]);
  float L = 0.0f, Lq = 0.0f;
  float acc[8] = {};
  if (M != -__builtin_inff())
    for (int i = 0; i < np; ++i) {
      const floatx4 ml = *reinterpret_cast<const floatx4*>(ws.part_ml + prow(i) * 4);
      const halfx8 h = *reinterpret_cast<const halfx8*>(ws.part_o + prow(i) * kD + piece * 8);
      if (ml[0] == -__builtin_inff()) continue;
      const float wgt = __builtin_amdgcn_exp2f(ml[0] - M);
      L = __builtin_fmaf(wgt, ml[1], L);
      Lq = __builtin_fmaf(wgt, ml[2], Lq);
      const float ws8 = wgt * __builtin_amdgcn_ldexpf(1.0f, int(ml[3]));
#pragma unroll
      for (int k = 0; k < 8; ++k) acc[k] = __builtin_fmaf(ws8, float(h[k]), acc[k]);
    }
  const int ra = row0 + rho;
  const size_t orow = size_t(st.q.q0 + ra / a.G) * a.hq + size_t(head) * a.G + ra % a.G;
  const float inv = Lq > 0.0f ? 1.0f / Lq : 0.0f;
  // halves 0-3: dims 32 (piece / 4) + 4 (piece % 4) + i, halves 4-7: the same + 16
  uint16_t* po = a.out + orow * kD + 32 * (piece >> 2) + 4 * (piece & 3);
  *reinterpret_cast<uint2*>(po) =
      make_uint2(pack_bf16x2(acc[0] * inv, acc[1] * inv), pack_bf16x2(acc[2] * inv, acc[3] * inv));
  *reinterpret_cast<uint2*>(po + 16) =
      make_uint2(pack_bf16x2(acc[4] * inv, acc[5] * inv), pack_bf16x2(acc[6] * inv, acc[7] * inv));
  if (a.lse != nullptr && piece == 0)
    a.lse[orow] = L > 0.0f ? (M + log2f(L)) * kLn2 : -__builtin_inff();
}

}  // namespace

size_t attn_q8_workspace_bytes(int32_t R, int32_t max_rows, int32_t hq, int32_t hkv,
                               int32_t max_pages) {
  (void)max_rows;
  (void)hq;
  (void)hkv;
  size_t n = 0;
  q8_layout(nullptr, R, max_pages, q8_waves(), &n);
  return n;
}

int32_t launch_tree_verify_attn_q8(const AttnQ8Args& x, hipStream_t stream) {
  (void)hipGetLastError();
  const int nw = q8_waves();
  const Q8Ws ws = q8_layout(x.workspace, x.R, x.max_pages, nw, nullptr);
  Q8Args a;
  a.q = x.q;
  a.k_new = x.k_new;
  a.v_new = x.v_new;
  a.k_pages = x.cache.k_pages;
  a.v_pages = x.cache.v_pages;
  a.k_scale = x.cache.k_scale;
  a.v_scale = x.cache.v_scale;
  a.block_table = x.block_table;
  a.prefix_len = x.prefix_len;
  a.q_offsets = x.q_offsets;
  a.tree_mask = x.tree_mask;
  a.num_pages = static_cast<long long>(x.cache.num_pages);
  a.page_shift = 0;
  while ((1 << a.page_shift) < x.cache.page_size) ++a.page_shift;
  a.max_pages = x.max_pages;
  a.W = x.mask_words;
  a.R = x.R;
  a.max_rows = x.max_rows;
  a.hq = x.hq;
  a.hkv = x.cache.hkv;
  a.G = a.hq / a.hkv;
  a.scale2 = x.sm_scale * kLog2e;
  a.out = x.out;
  a.lse = x.lse;
  a.status = x.status;
  int chunks = 0;
  if (!q8_plan_checks(a.R, a.max_pages)) {
    chunks = q8_page_chunks(a.max_pages);
    hipLaunchKernelGGL(q8_pages_kernel, dim3(unsigned(a.R), unsigned(chunks)), dim3(kPageChunk), 0,
                       stream, a, ws.bad);
  }
  hipLaunchKernelGGL(q8_plan_kernel, dim3(1), dim3(kPlanThreads),
                     (size_t(a.R) + 1) * sizeof(int32_t), stream, a, ws, nw, chunks);
  hipLaunchKernelGGL(x.cache.format == ECHO_KV_E4M3 ? q8_main_kernel<ECHO_KV_E4M3>
                                                    : q8_main_kernel<ECHO_KV_E5M2>,
                     dim3(unsigned(nw / kQ8Waves)), dim3(kQ8Waves * kWave), 0, stream, a, ws);
  const long long rows = (long long)a.max_rows * a.G;
  hipLaunchKernelGGL(q8_combine_kernel, dim3(unsigned(nw), unsigned((rows < kQ8Rows ? rows : kQ8Rows) + 15) / 16),
                     dim3(256), 0, stream, a, ws);
  return hipGetLastError() == hipSuccess ? ECHO_OK : ECHO_ERR_HIP;
}

}  // namespace echo
