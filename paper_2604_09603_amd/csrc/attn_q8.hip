// Tree-masked grouped-query verification attention over an 8-bit paged cache
// (kvq8_device.h has the cache's layout).  Two launches, and one more before them for
// large block tables:
//
//   q8_pages    checks the page ids (small tables: the main kernel's waves do).
//   q8_main     persistent, two workgroups of four waves per CU.  A unit is one KV head of
//               one request with up to 32, 64 or 128 of its rows (verify slots x query
//               heads of the GQA group); its steps are first the tree's (32 new keys
//               each), then the prefix's, two 32-token blocks each.  The steps of all
//               units are cut into equal contiguous ranges: a head's blocks lie in one
//               piece, so nothing is gained by waves that read the heads of the same
//               tokens side by side, and one head's keys are spread over as many waves
//               as they can feed.  Every workgroup finds its ranges by itself, from the
//               requests' lengths.
//               A wave has 32 rows.  It copies its tiles HBM -> LDS into slots of its own
//               with direct-to-LDS loads: S^T = K Q^T and O^T += V^T P^T with K and V
//               widened to bfloat16 (exact), an online softmax in base 2 between them.
//               The K scale goes into the softmax's factor, the V scale into its
//               exponent.
//   q8_combine  merges the partial sums of units that several waves share.
//
// What bounds it (medians of 60 launches; whole calls back to back are up to 5% shorter than their
// kernels under the profiler).  Few rows per head: HBM.  64 requests decoding over 1024-8192
// tokens (32 query and 8 KV heads, 604 MB) take 97 us in the main kernel, 6.2 TB/s, and 6 us in
// the merge; the 10 us until the first tiles are there (lengths, page ids, scales and tiles are
// dependent round trips) are most of the rest.  Many rows: the vector instructions.  A step
// of 64 keys and 32 rows takes 32 matrix products (1044 cycles) and about 400 other vector
// instructions (1700 cycles: 128 conversions, 32 exponentials of two each, 96 products,
// sums and roundings of the weights), which share a SIMD's issue; with trees of 13 slots on
// average (16 rows each) over 16384-32768 tokens, 79 us of products, the main kernel takes
// 234 us, 64% of it issuing vector instructions.  128 trees of 3 slots on average (617 MB) are
// between the two: 145 us and 11 in the merge.  Units of 32 rows because a 32x32x16 product
// leaves room for five vector instructions, where 16x16x32 leaves two for the same work;
// two waves per SIMD, so that one's softmax runs beside the other's products.
//
// Softmax statistics and sums are fp32.  The weights p are rounded to bfloat16 for
// the product with V (at most 2^-8 each) and the output is divided by the sum of the
// weights used, so that it stays a convex combination of V rows; the output's own
// rounding to bfloat16 is as large, so the residuals of the weights are not
// multiplied.  Partial sums are stored in fp32.
#include "attn_core.h"
#include "kvq8_device.h"
#include "q8_ranges.h"

namespace echo {
namespace {

static_assert(kQ8TreeKeys == kTileKeys, "a step of the tree is a tile");
constexpr int kQ8Wgs = 2;          // workgroups per CU: two waves per SIMD
constexpr int kQ8Slot = 2 * kBlockBytes;          // one tensor's tiles of a step
constexpr int kQ8Scratch = 16 * kD * 2;           // 16 rows of bfloat16 V (tree tiles)
constexpr int kQ8WaveLds = 2 * kQ8Slot + kQ8Scratch;  // K, V, scratch
static_assert(kQ8Wgs * kQ8Waves * kQ8WaveLds <= 160 * 1024, "gfx950 LDS per CU");
constexpr int kGangSlots = 4;      // slots of a gang of four waves, which share their tiles
constexpr int kOwnPages = 512;     // block tables up to this wide are checked by the waves

typedef int intx2 __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) intx2 lds_intx2_t;
typedef uint32_t uint4v __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) const uint4v lds_uint4_t;
typedef __attribute__((address_space(3))) char lds_char_t;
typedef float floatx16 __attribute__((ext_vector_type(16)));

// The LDS byte address x as a pointer (constant offsets go into the instructions).
__device__ __forceinline__ lds_char_t* lds_at(uint32_t x) { return (lds_char_t*)(uintptr_t(x)); }

// A gang is the k waves (1, 2 or 4, of one workgroup) that take the same steps of a unit,
// each with 32 of its rows.  Four share their tiles in LDS (each copies a quarter of them,
// with a barrier per step); of two one copies them from HBM, the other at about the same
// time from the caches.  A head's rows are dealt to gangs of four, and what is left to one of
// one, two or (three) four waves: without the remainder's own gang, waves that have no
// rows would be idle through its steps.  The requests with a part for gangs of k
// waves form a class, whose steps are cut into equal ranges, one per gang.

// A request's part in a class: Hkv * passes units (unit = head * passes + pass) of tpu steps
// each, from step tile0 of the class on; gang member m has rows row0 + 32 (k pass + m) .. of
// a head, as far as there are so many.
struct Q8Part {
  int tile0, tpu;
  int q0, nslots;
  int P, r, passes, row0;
};

// Where a wave's range begins inside a unit, and is the first that does: the unit's partial
// sums are those of `parts` gangs from the one before on (0: there is nothing to merge).
// Gangs go round the class's places wg0 .. wg0 + nwg - 1, so that few of them spread over
// the CUs: the one before has place wg0 + at and is that workgroup's gang number `slot`.
struct Q8Cut {
  int32_t parts, at, slot, k;
  int32_t wg0, nwg, member, q0;
  int32_t nslots, head, row0, pad;
};
static_assert(sizeof(Q8Cut) == 48, "12 words");

struct Q8Ws {
  Q8Cut* cuts;       // [waves]
  int32_t* bad;      // [R][chunks] flags of q8_pages
  float* part_ml;    // [waves][2][32][4]: max, sum, sum of the weights used
  float* part_o;     // [waves][2][16][32][8]: 8 dims of each of the 32 rows, 16 times
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
  int chunks;        // flags of q8_pages per request, 0: the waves check
  int wgs;           // workgroups of the main kernel (even)
  float scale2;
  uint16_t* out;
  float* lse;
  int32_t* status;
};

// Narrow tables need a few loads a wave and request; a launch of its own costs 2 us, which wide
// ones are worth (64 requests of so many pages of 32 tokens, 8 heads, waves | launch: 64 pages
// 32.0 | 34.0 us, 512 pages 133 | 134, 2048 pages 487 | 486).
__host__ inline int q8_page_chunks(int max_pages) {
  return max_pages <= kOwnPages ? 0 : (max_pages + kPageChunk - 1) / kPageChunk;
}

__host__ inline Q8Ws q8_layout(void* base, int R, int max_pages, int nw, size_t* bytes) {
  char* p = static_cast<char*>(base);
  Q8Ws w;
  w.cuts = reinterpret_cast<Q8Cut*>(p);
  p += al(size_t(nw) * sizeof(Q8Cut));
  w.bad = reinterpret_cast<int32_t*>(p);
  p += al(size_t(R) * size_t(q8_page_chunks(max_pages)) * 4);
  w.part_ml = reinterpret_cast<float*>(p);
  p += al(size_t(nw) * 2 * kQ8Rows * 4 * sizeof(float));
  w.part_o = reinterpret_cast<float*>(p);
  p += al(size_t(nw) * 2 * kQ8Rows * kD * sizeof(float));
  if (bytes != nullptr) *bytes = size_t(p - static_cast<char*>(base));
  return w;
}

int q8_waves() { return device_cu_count() * kQ8Wgs * kQ8Waves; }

// Pages of a request's prefix, or -1 if its length does not fit its table row.
__device__ __forceinline__ int prefix_pages(long long P, const Q8Args& a) {
  if (P < 0 || P > ((long long)a.max_pages << a.page_shift)) return -1;
  return int((P + (1 << a.page_shift) - 1) >> a.page_shift);
}

__global__ __launch_bounds__(kPageChunk) void q8_pages_kernel(Q8Args a, int32_t* bad_flags) {
  const int c = blockIdx.x, r = blockIdx.y;
  const int np = prefix_pages(a.prefix_len[r], a);
  const int e = c * kPageChunk + int(threadIdx.x);
  int bad = 0;
  if (e < np) {
    const int pg = a.block_table[size_t(r) * size_t(a.max_pages) + size_t(e)];
    bad = pg < 0 || pg >= a.num_pages;
  }
  bad = __syncthreads_or(bad);
  if (threadIdx.x == 0) bad_flags[size_t(r) * gridDim.x + c] = bad;
}

// ---------------------------------------------------------------- main ----
// A tile in LDS: 32 rows x 128 bytes per tensor.  The 16-byte chunk c of row r is at chunk
// position c ^ f(r), with bits 2, 1, 3 of r as bits 0, 1, 2 of f: the 16 rows of which
// a phase of a K read takes one chunk each, and the eight rows (four of each parity)
// of which half a wave's transposed V read takes two chunks, fall into 16 different
// sixteenths of the banks.
__device__ __forceinline__ int q8_swz(int row) {
  return ((row >> 2) & 1) | (row & 2) | ((row >> 1) & 4);
}

// Every LDS read so far has its data (and stays ahead of what follows).
__device__ __forceinline__ void q8_wait_lds() {
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
}

// Copies a step's two tiles of one tensor to LDS address lds.  Lane offsets offa (rows 0-7
// and 16-23 of a tile) and offb (the other rows); the instructions' offset moves both
// addresses.  In inline assembly because the compiler would wait for every copy in
// flight before each LDS read; M0 (the LDS address) is the compiler's and is restored,
// and needs a wait state before a load reads it.  Non-temporal where no other wave of a
// gang reads the tiles (alone).
#define ECHO_Q8_COPY(POL)                                                              \
  "s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\t"                                 \
  "global_load_lds_dwordx4 %2, %4" POL "\n\t"                                          \
  "global_load_lds_dwordx4 %3, %4 offset:0x400" POL "\n\t"                              \
  "global_load_lds_dwordx4 %2, %4 offset:0x800" POL "\n\t"                              \
  "global_load_lds_dwordx4 %3, %4 offset:0xc00" POL "\n\t"                              \
  "s_add_u32 m0, m0, 0x1000\n\ts_nop 0\n\t"                                            \
  "global_load_lds_dwordx4 %2, %5" POL "\n\t"                                          \
  "global_load_lds_dwordx4 %3, %5 offset:0x400" POL "\n\t"                              \
  "global_load_lds_dwordx4 %2, %5 offset:0x800" POL "\n\t"                              \
  "global_load_lds_dwordx4 %3, %5 offset:0xc00" POL "\n\t"                              \
  "s_mov_b32 m0, %0"
__device__ __forceinline__ void q8_copy(uint32_t lds, uint64_t tile0, uint64_t tile1, uint32_t offa,
                                        uint32_t offb, bool alone) {
  uint32_t saved;
  if (alone)  // uniform
    asm volatile(ECHO_Q8_COPY(" nt")
                 : "=&s"(saved)
                 : "s"(lds), "v"(offa), "v"(offb), "s"(tile0), "s"(tile1)
                 : "memory", "scc");
  else
    asm volatile(ECHO_Q8_COPY("")
                 : "=&s"(saved)
                 : "s"(lds), "v"(offa), "v"(offb), "s"(tile0), "s"(tile1)
                 : "memory", "scc");
}
#undef ECHO_Q8_COPY

// 4 KB to LDS address lds: 1 KB from base + each of the lane's four offsets.
__device__ __forceinline__ void q8_copy4(uint32_t lds, uint64_t base, const uint32_t (&o)[4]) {
  uint32_t saved;
  asm volatile(
      "s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %2, %6\n\t"
      "s_add_u32 m0, m0, 0x400\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %3, %6\n\t"
      "s_add_u32 m0, m0, 0x400\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %4, %6\n\t"
      "s_add_u32 m0, m0, 0x400\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %5, %6\n\t"
      "s_mov_b32 m0, %0"
      : "=&s"(saved)
      : "s"(lds), "v"(o[0]), "v"(o[1]), "v"(o[2]), "v"(o[3]), "s"(base)
      : "memory", "scc");
}

// What a lane knows of a request.  tiles: row tiles per head, -1: it cannot be used.
struct Q8Look {
  int q0, nslots, P, tiles, tpu;
};
__device__ __forceinline__ Q8Look q8_look(const Q8Args& a, int q0, int q1, int P) {
  Q8Look x;
  const bool ok = q0 >= 0 && q1 >= q0 && q1 <= a.max_rows && prefix_pages(P, a) >= 0;
  x.q0 = q0;
  x.nslots = ok ? q1 - q0 : 0;
  x.P = ok ? P : 0;
  x.tiles = ok ? q8_row_tiles(x.nslots, a.G) : -1;
  x.tpu = q8_unit_steps(x.nslots, x.P);
  return x;
}
__device__ __forceinline__ Q8Look q8_look(const Q8Args& a, int r) {
  return q8_look(a, a.q_offsets[r], a.q_offsets[r + 1], a.prefix_len[r]);
}

// Where a wave is in its class's steps: a unit (of part q), whose first step is u0.
struct Q8Walk {
  Q8Part q;
  int unit, u0, cls;
  bool bad;  // the request has pages that are not in the pool: no step of it is taken
  bool met;  // this or an earlier one had
  // steps before the prefix's
  __device__ __forceinline__ int head() const {
    return kQ8Enter + (q.nslots + kTileKeys - 1) / kTileKeys;
  }
};

__device__ __forceinline__ int lane_of(int v, int i) { return __builtin_amdgcn_readlane(v, i); }
__device__ __forceinline__ float lane_of(float v, int i) {
  return __uint_as_float(uint32_t(__builtin_amdgcn_readlane(int(__float_as_uint(v)), i)));
}

// What tells whether a request's pages are in the pool: its page ids, or q8_pages' flags.
struct Q8Pages {
  const int32_t* e;
  int n;
  bool own;
  __device__ Q8Pages(const Q8Args& a, const Q8Ws& ws, int r, int P) : own(a.chunks == 0) {
    const int np = prefix_pages(P, a);
    n = own ? np : (np + kPageChunk - 1) / kPageChunk;
    e = own ? a.block_table + size_t(r) * size_t(a.max_pages) : ws.bad + size_t(r) * size_t(a.chunks);
  }
  __device__ __forceinline__ bool bad(const Q8Args& a, int i) const {  // (past n: the last again)
    return bad_value(a, at(i));
  }
  __device__ __forceinline__ int at(int i) const { return e[min(i, n - 1)]; }
  __device__ __forceinline__ bool bad_value(const Q8Args& a, int v) const {
    return own ? v < 0 || v >= a.num_pages : v != 0;
  }
};

// Puts w at the class's part of request r, which lane i has looked at.
__device__ __forceinline__ void q8_enter(Q8Walk& w, const Q8Look& x, int i, int r, int tile0) {
  w.q.tile0 = tile0;
  w.q.tpu = lane_of(x.tpu, i);
  w.q.q0 = lane_of(x.q0, i);
  w.q.nslots = lane_of(x.nslots, i);
  w.q.P = lane_of(x.P, i);
  w.q.r = r;
  const int tiles = lane_of(x.tiles, i);
  w.q.passes = q8_passes(tiles, w.cls);
  w.q.row0 = w.cls == 2 ? 0 : (tiles & ~3) * kQ8Rows;
  w.unit = 0;
  w.u0 = tile0;
}

// Checks the pages of w's request, from place j of what tells it on.
__device__ __forceinline__ void q8_check(Q8Walk& w, const Q8Args& a, const Q8Pages& pages, bool bad,
                                         int j) {
  const int lane = threadIdx.x & (kWave - 1);
  for (; j < pages.n; j += 2 * kWave)  // (two loads at a time)
    bad |= pages.bad(a, j + lane) | pages.bad(a, j + kWave + lane);
  w.bad = __ballot(bad) != 0ull;
  w.met |= w.bad;
}

// (Only called where steps are left: there is a next unit.)
__device__ __forceinline__ void q8_next_unit(Q8Walk& w, const Q8Args& a, const Q8Ws& ws) {
  const int units = a.hkv * w.q.passes;
  if (w.unit + 1 < units) {
    w.unit += 1;
    w.u0 += w.q.tpu;
    return;
  }
  const int lane = threadIdx.x & (kWave - 1);
  const int tile0 = w.q.tile0 + units * w.q.tpu;
  for (int r = w.q.r + 1; r < a.R; r += kWave) {
    Q8Look x = {};
    if (r + lane < a.R) x = q8_look(a, r + lane);
    const uint64_t in = __ballot(x.tiles > 0 && q8_passes(x.tiles, w.cls) > 0);
    if (in != 0ull) {
      const int i = __ffsll((unsigned long long)in) - 1;
      q8_enter(w, x, i, r + i, tile0);
      q8_check(w, a, Q8Pages(a, ws, r + i, w.q.P), false, 0);
      return;
    }
  }
}

// -------------------------------------------------------------- ranges ----
// The wave's range and where it starts (its request's pages are not checked).  Every workgroup
// counts the steps of all requests (thread t those of requests K t .. K t + K - 1): that is
// a round trip, a scan and a search, where a launch for it took 10-15 us.  s: 3.1 KB and 8
// bytes a request, of LDS.
__device__ __forceinline__ Q8Range q8_begin(const Q8Args& a, const Q8Ws& ws, uint32_t* s, Q8Walk& w) {
  constexpr int kThreads = kQ8Waves * kWave, kBatch = 2;
  const int tid = threadIdx.x, lane = tid & (kWave - 1), wid = wave_id();
  uint32_t* s_tot = s + kQ8Classes * kThreads;  // [waves][classes + 1]
  int* s_q = reinterpret_cast<int*>(s_tot + kQ8Waves * (kQ8Classes + 1));  // [R + 1] offsets
  int* s_P = s_q + a.R + 1;                                                // [R] lengths
  const int K = (a.R + kThreads - 1) / kThreads;
  Q8Steps T;
  int bits = 0;
#pragma unroll 1
  for (int i = 0; i < K; i += kBatch) {
    int q0[kBatch], q1[kBatch], P[kBatch];
#pragma unroll
    for (int j = 0; j < kBatch; ++j) {
      const int r = min(tid * K + i + j, a.R - 1);
      q0[j] = a.q_offsets[r];
      q1[j] = a.q_offsets[r + 1];
      P[j] = a.prefix_len[r];
    }
    uint64_t idle[kBatch];  // lanes whose request has nothing to do, but whose pages count for the status
#pragma unroll
    for (int j = 0; j < kBatch; ++j) {
      const int r = tid * K + i + j;
      const bool there = i + j < K && r < a.R;
      Q8Look x = {};
      x.tiles = -1;
      if (there) {
        s_q[r] = q0[j];
        s_P[r] = P[j];
        if (r + 1 == a.R) s_q[r + 1] = q1[j];
        x = q8_look(a, q0[j], q1[j], P[j]);
        if (x.tiles < 0 && blockIdx.x == 0) bits = ECHO_DATA_BAD_OFFSETS;
        if (x.tiles > 0) T.add(a.hkv, x.tiles, x.tpu);
      }
      idle[j] = __ballot(x.tiles == 0 && r % int(gridDim.x) == int(blockIdx.x));
    }
#pragma unroll
    for (int j = 0; j < kBatch; ++j)
      while (idle[j] != 0ull) {  // uniform
        const int l = __ffsll((unsigned long long)idle[j]) - 1;
        idle[j] &= idle[j] - 1;
        const Q8Pages pages(a, ws, (wid * kWave + l) * K + i + j, lane_of(P[j], l));
        for (int e = 0; e < pages.n; e += 2 * kWave) {  // (two loads at a time)
          const int v0 = pages.at(e + lane), v1 = pages.at(e + kWave + lane);
          if (pages.bad_value(a, v0) || pages.bad_value(a, v1)) bits = ECHO_DATA_BAD_OFFSETS;
        }
      }
  }
  // (a sum that could matter is rare)
  float all = T.all;
  if (__ballot(all > kQ8MaxSteps / kThreads) != 0ull) {
#pragma unroll
    for (int d = 1; d < kWave; d *= 2) all += __shfl_xor(all, d);
  } else {
    all = 0.0f;
  }
#pragma unroll
  for (int c = 0; c < kQ8Classes; ++c) {
    const uint32_t inc = uint32_t(wave_inclusive_sum(int(T.of[c])));
    s[c * kThreads + tid] = inc - T.of[c];
    if (lane == kWave - 1) s_tot[wid * (kQ8Classes + 1) + c] = inc;
  }
  if (lane == 0) s_tot[wid * (kQ8Classes + 1) + kQ8Classes] = __float_as_uint(all);
  __syncthreads();
  int tot[kQ8Classes] = {0, 0, 0};
  all = 0.0f;
#pragma unroll
  for (int v = 0; v < kQ8Waves; ++v) {
#pragma unroll
    for (int c = 0; c < kQ8Classes; ++c)
      tot[c] += __builtin_amdgcn_readfirstlane(int(s_tot[v * (kQ8Classes + 1) + c]));
    all += __uint_as_float(s_tot[v * (kQ8Classes + 1) + kQ8Classes]);
  }
  // (what passes fits 31 bits: four waves that are not summed have less than 2^30 between them, and
  // the sum's own rounding is far smaller)
  if (q8_refuses(__uint_as_float(uint32_t(__builtin_amdgcn_readfirstlane(int(__float_as_uint(all))))), tot))
    bits = ECHO_DATA_BAD_OFFSETS;
  wave_status_or(a.status, bits);
  const int g = q8_place(blockIdx.x, a.wgs);
  const float per =
      float(a.wgs) * __builtin_amdgcn_rcpf(q8_cost(tot, 0) + q8_cost(tot, 1) + q8_cost(tot, 2));
  Q8Share share = q8_share(tot, a.wgs, per, g);
  share.cls = __builtin_amdgcn_readfirstlane(share.cls);
  share.wg0 = __builtin_amdgcn_readfirstlane(share.wg0);
  share.nwg = __builtin_amdgcn_readfirstlane(share.nwg);
  const int cls = share.cls;
  // the steps that each wave's threads counted, of the class
  int part[kQ8Waves];
#pragma unroll
  for (int v = 0; v < kQ8Waves; ++v)
    part[v] = __builtin_amdgcn_readfirstlane(int(s_tot[v * (kQ8Classes + 1) + cls]));
  const Q8Range x = q8_range_at(share, cls == 0 ? tot[0] : cls == 1 ? tot[1] : tot[2], g, wid);
  if (x.lo < x.hi) {
    w.cls = cls;
    // the last thread whose requests' steps start at lo or before: of four in each lane
    const uint4 v = reinterpret_cast<const uint4*>(s + cls * kThreads)[lane];
    const auto offset = [&](int u) {
      int o = 0;
#pragma unroll
      for (int v = 0; v + 1 < kQ8Waves; ++v) o += u > v ? part[v] : 0;
      return o;
    };
    const int o = offset(lane / (kWave / kQ8Waves));
    const int th = __popcll(__ballot(int(v.x) + o <= x.lo)) + __popcll(__ballot(int(v.y) + o <= x.lo)) +
                   __popcll(__ballot(int(v.z) + o <= x.lo)) + __popcll(__ballot(int(v.w) + o <= x.lo)) - 1;
    const int start = __builtin_amdgcn_readfirstlane(int(s[cls * kThreads + th])) + offset(th / kWave);
    // and which of them it is
    Q8Look q = {};
    const int rl = th * K + lane;
    if (lane < K && rl < a.R) q = q8_look(a, s_q[rl], s_q[rl + 1], s_P[rl]);
    const int steps = q.tiles > 0 ? a.hkv * q.tpu * q8_passes(q.tiles, cls) : 0;
    const int end = start + wave_inclusive_sum(steps);
    const int i = __ffsll((unsigned long long)__ballot(end > x.lo)) - 1;
    q8_enter(w, q, i, th * K + i, lane_of(end - steps, i));
    w.unit = int(unsigned(x.lo - w.q.tile0) / unsigned(w.q.tpu));
    w.u0 = w.q.tile0 + w.unit * w.q.tpu;
  }
  __syncthreads();  // the tiles take this memory
  return x;
}

// The first of the member's rows of the unit.
__device__ __forceinline__ int q8_row0(const Q8Walk& w, int k, int member) {
  return w.q.row0 + (w.unit % w.q.passes * k + member) * kQ8Rows;
}

// Whether the member has rows of the unit, of a request that can be used.
__device__ __forceinline__ bool q8_has_rows(const Q8Walk& w, const Q8Args& a, int k, int member) {
  return !w.bad && q8_row0(w, k, member) < w.q.nslots * a.G;
}

// What the merge has to know of the wave's range, w being where it starts.
__device__ __forceinline__ Q8Cut q8_cut(const Q8Walk& w, const Q8Range& x) {
  Q8Cut c = {};
  if (!w.bad && w.u0 < x.lo && x.ranges.first(x.gang - 1) <= w.u0)
    c.parts = x.ranges.range_of(w.u0 + w.q.tpu - 1) - x.gang + 2;
  const int before = max(x.gang - 1, 0);
  c.slot = int(unsigned(before) / unsigned(x.nwg));
  c.at = before - c.slot * x.nwg;
  c.k = x.k;
  c.member = x.member;
  c.wg0 = x.wg0;
  c.nwg = x.nwg;
  c.q0 = w.q.q0;
  c.nslots = w.q.nslots;
  c.head = w.unit / w.q.passes;
  c.row0 = q8_row0(w, x.k, x.member);
  return c;
}

// What a wave knows of the next 32 steps of its range, tile i (two per step) in lane
// i & 63: the block, the tokens it holds (32 or more: all), and what the softmax takes
// of its scales.  A request's last step may have one tile: its second entry is that
// block again, without tokens.  One vector of loads instead of scalar ones for every
// tile; once in 32 steps the ring runs empty for it (a gang of four's does not).  Steps [.., known) are in the
// table; K of those below k_sent and V of those below v_sent have been copied, and
// those below `done` multiplied.
struct Q8Table {
  uint32_t blk;
  int tokens;
  float c, lvs;       // softmax factor x K scale; log2 of the V scale
  int known, k_sent, v_sent, done;  // (a gang of four: k_sent for both)
  bool more;          // the range has steps past the table's
  int k, member;      // of the wave's gang
  bool raw;           // c and lvs are still the scales (which may be on their way)
};

// The lane's LDS and copy offsets in one register (three would be reloaded from memory in
// the main loop, behind every copy in flight).
//   K reads   row lane % 32, chunks 4 j + 2 (lane / 32) + e: an exclusive-or of bits 6 and 4
//   V reads   (transposed) of a 16-key group, keys 4 h + 0..3 and the same + 8 (h: lane / 32;
//             the order in which S^T leaves them in the lanes), dims 32 dt + lane % 32: the
//             lane supplies half of one key's 16-byte chunk 2 dt + (lane / 16) % 2, an
//             exclusive-or of bits 5 and 6
//   copies    eight rows of a tile from row_of_copy on (rows 0-7, and 16-23; the other
//             rows have bit 6 flipped)
__device__ __forceinline__ uint32_t q8_lane_offsets(int row_of_copy) {
  const int lane = threadIdx.x & (kWave - 1);
  const int row = lane & 31, h = lane >> 5, i = lane & 15;
  const int vkey = 4 * h + ((i >> 1) & 3) + ((i >> 3) << 3);
  const uint32_t k = uint32_t(row * kD + (((2 * h) ^ q8_swz(row)) << 4));
  const uint32_t v = uint32_t(vkey * kD + ((((lane >> 4) & 1) ^ q8_swz(vkey)) << 4) + ((i & 1) << 3));
  const int crow = row_of_copy + (lane >> 3);
  const uint32_t c = uint32_t(crow * kD + (((lane & 7) ^ q8_swz(crow)) << 4));
  return (k >> 4) | (v << 8) | (c << 16);  // k a multiple of 16 and v of 8 below 2^12 (2^11)
}
__device__ __forceinline__ uint32_t q8_opaque(uint32_t x) {  // (not kept unpacked)
  asm volatile("" : "+v"(x));
  return x;
}
__device__ __forceinline__ uint32_t k_offset(uint32_t p) { return (q8_opaque(p) & 0xFFu) << 4; }
__device__ __forceinline__ uint32_t v_offset(uint32_t p) { return (q8_opaque(p) >> 8) & 0x7FFu; }
__device__ __forceinline__ uint32_t copy_offset(uint32_t p) { return (q8_opaque(p) >> 20) << 4; }

// Copies a tensor's tiles of the next step, if the table has one.  Where a tile's last rows
// hold no tokens they read its last token's row again, so that nothing unwritten is
// multiplied (they are masked).
__device__ __forceinline__ void q8_send(const Q8Table& tb, int& sent, const uint8_t* pages,
                                        uint32_t lds, uint32_t offs) {
  sent = __builtin_amdgcn_readfirstlane(sent);
  if (sent >= tb.known) return;  // uniform
  const int i = (2 * sent) & (kWave - 1);
  const uint64_t base = reinterpret_cast<uint64_t>(pages);
  const uint64_t t0 = base + uint64_t(uint32_t(lane_of(int(tb.blk), i))) * kBlockBytes;
  const uint64_t t1 = base + uint64_t(uint32_t(lane_of(int(tb.blk), i + 1))) * kBlockBytes;
  const int tn1 = lane_of(tb.tokens, i + 1);
  if (tn1 >= kTileKeys) {
    const uint32_t offa = copy_offset(offs);
    q8_copy(lds, t0, t1, offa, offa ^ 64u, tb.k == 1);
  } else {
    const int lane = threadIdx.x & (kWave - 1);
    const int tn0 = lane_of(tb.tokens, i);
#pragma unroll 1
    for (int k = 0; k < 2; ++k) {
      const int last = min(max(k == 0 ? tn0 : tn1, 1), kTileKeys) - 1;
      uint32_t o[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int row = 8 * j + (lane >> 3);
        o[j] = uint32_t(min(row, last) * kD + (((lane & 7) ^ q8_swz(row)) << 4));
      }
      q8_copy4(lds + uint32_t(k * kBlockBytes), k == 0 ? t0 : t1, o);
    }
  }
  sent += 1;
}

// The wave's quarter (eight rows of each tile) of the next step's tiles, for its gang of four.
__device__ __forceinline__ void q8_send_gang(Q8Table& tb, const Q8Args& a, uint32_t ring, uint32_t offs) {
  const int sent = __builtin_amdgcn_readfirstlane(tb.k_sent);
  if (sent >= tb.known) return;  // uniform
  const int i = (2 * sent) & (kWave - 1);
  const uint64_t b0 = uint64_t(uint32_t(lane_of(int(tb.blk), i))) * kBlockBytes;
  const uint64_t b1 = uint64_t(uint32_t(lane_of(int(tb.blk), i + 1))) * kBlockBytes;
  const uint64_t k = reinterpret_cast<uint64_t>(a.k_pages), v = reinterpret_cast<uint64_t>(a.v_pages);
  const uint32_t c = copy_offset(offs);
  const int row = int(c) / kD;
  const uint32_t in_row = c & (kD - 1);
  const auto offset = [&](int tokens) {  // (rows past the tile's tokens: the last one again)
    return uint32_t(min(row, min(max(tokens, 1), kTileKeys) - 1) * kD) + in_row;
  };
  const uint32_t o0 = offset(lane_of(tb.tokens, i)), o1 = offset(lane_of(tb.tokens, i + 1));
  const uint32_t lds = ring + uint32_t((sent & (kGangSlots - 1)) * 2 * kQ8Slot + tb.member * 1024);
  uint32_t saved;
  asm volatile(
      "s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %2, %4 nt\n\t"
      "s_add_u32 m0, m0, 0x1000\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %3, %5 nt\n\t"
      "s_add_u32 m0, m0, 0x1000\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %2, %6 nt\n\t"
      "s_add_u32 m0, m0, 0x1000\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %3, %7 nt\n\t"
      "s_mov_b32 m0, %0"
      : "=&s"(saved)
      : "s"(lds), "v"(o0), "v"(o1), "s"(k + b0), "s"(k + b1), "s"(v + b0), "s"(v + b1)
      : "memory", "scc");
  tb.k_sent = sent + 1;
}

// What the table's lanes take next.
struct Q8Next {
  int n, pos;  // lanes to be filled; the lane's place among them
  uint32_t entry, head;
  int key, tokens;
};

// What follows the table's steps, given that step t of the unit at w is the next to be taken.
template <bool kGang>
__device__ __forceinline__ Q8Next q8_next_steps(Q8Table& tb, const Q8Args& a, const Q8Ws& ws, Q8Walk w,
                                                int t, int hi) {
  const int lane = threadIdx.x & (kWave - 1);
  int skip = tb.known - tb.done;  // steps that it holds
  const int room = kWave - 2 * skip;
  Q8Next x = {};
  x.pos = (lane - 2 * tb.known) & (kWave - 1);
  while (x.n < room && t < hi) {  // uniform
    const int end = min(hi, w.u0 + w.q.tpu);
    const int p0 = w.u0 + w.head();
    t = max(t, min(end, p0));
    // (a wave without rows of this unit takes none of its steps, unless its gang counts on it)
    if (kGang ? w.bad : !q8_has_rows(w, a, tb.k, tb.member)) t = end;
    if (kGang) {
      const int held = min(skip, end - t);
      skip -= held;
      t += held;
    }
    const int m = min((room - x.n) / 2, end - t);
    if (x.pos >= x.n && x.pos < x.n + 2 * m) {
      x.key = (t - p0) * kQ8StepKeys + (x.pos - x.n) * kTileKeys;
      x.tokens = max(w.q.P - x.key, 0);
      if (x.tokens == 0) x.key -= kTileKeys;
      x.entry = uint32_t(w.q.r) * uint32_t(a.max_pages) + uint32_t(x.key >> a.page_shift);
      x.head = uint32_t(w.unit / w.q.passes);
    }
    x.n += 2 * m;
    t += m;
    if (t >= end && t < hi) q8_next_unit(w, a, ws);
  }
  tb.more = t < hi;
  return x;
}

// The softmax factor of a block.  Not 0, by which the scores of masked keys, -inf, are not to be
// multiplied (the smallest normal number instead: a score is 0 with either).
__device__ __forceinline__ float q8_factor(const Q8Args& a, float k_scale) {
  return fmaxf(a.scale2 * k_scale, 1.17549435e-38f);
}

// Fills the table with them (page: the lane's) and sends for the first steps' tiles; the scales
// come in the same round trip, the first time beside Q and the tree's keys if a unit begins.
template <bool kGang>
__device__ __forceinline__ void q8_fill(Q8Table& tb, const Q8Args& a, const Q8Next& x, uint32_t page,
                                        uint32_t ring, uint32_t offs) {
  const bool first = tb.known == 0;
  tb.known += x.n / 2;
  float ks = 1.0f, vs = 1.0f;
  if (x.pos < x.n) {
    tb.blk = ((page * uint32_t(a.hkv) + x.head) << (a.page_shift - 5)) +
             (uint32_t(x.key & ((1 << a.page_shift) - 1)) >> 5);
    tb.tokens = x.tokens;
    ks = a.k_scale[tb.blk];
    vs = a.v_scale[tb.blk];
  }
  if (kGang) {
    for (int j = tb.k_sent - tb.done; j < kGangSlots - 1; ++j) q8_send_gang(tb, a, ring, offs);
  } else {
    q8_send(tb, tb.k_sent, a.k_pages, ring, offs);
    q8_send(tb, tb.v_sent, a.v_pages, ring + kQ8Slot, offs);
  }
  if (first) {
    tb.c = ks;
    tb.lvs = vs;
    tb.raw = true;
  } else if (x.pos < x.n) {
    tb.c = q8_factor(a, ks);
    tb.lvs = __builtin_amdgcn_logf(vs);
  }
}
template <bool kGang>
__device__ __forceinline__ void q8_refill(Q8Table& tb, const Q8Args& a, const Q8Ws& ws, const Q8Walk& w,
                                          int t, int hi, uint32_t ring, uint32_t offs) {
  const Q8Next x = q8_next_steps<kGang>(tb, a, ws, w, t, hi);
  q8_fill<kGang>(tb, a, x, x.pos < x.n ? uint32_t(a.block_table[x.entry]) : 0u, ring, offs);
}

// The scales' values, once they are there, become what the softmax takes.
__device__ __forceinline__ void q8_scales(Q8Table& tb, const Q8Args& a) {
  tb.c = q8_factor(a, tb.c);
  tb.lvs = __builtin_amdgcn_logf(tb.lvs);
  tb.raw = false;
}

// Two bytes (the upper two of w if hi) as bfloat16 (exact).
template <int kFmt>
__device__ __forceinline__ uint32_t widen2(uint32_t w, bool hi) {  // hi: a constant
  if (kFmt == ECHO_KV_E4M3)
    return __builtin_bit_cast(uint32_t, hi ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, true)
                                           : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, false));
  return __builtin_bit_cast(uint32_t, hi ? __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(w, 1.0f, true)
                                         : __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(w, 1.0f, false));
}

// Maximum and sum over the two lanes of a row.
__device__ __forceinline__ float pair_max(float v) {
  const uint32_t u = __float_as_uint(v);
  const auto a = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
}
__device__ __forceinline__ float pair_sum(float v) {
  const uint32_t u = __float_as_uint(v);
  const auto a = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return __uint_as_float(a[0]) + __uint_as_float(a[1]);
}

// A wave's 32 rows: the lane's row is lane % 32, which it shares with lane ^ 32.
struct Q8Rows {
  floatx16 o[4];  // O^T: dims 32 dt + 8 (r >> 2) + 4 (lane / 32) + (r & 3)
  float m;        // reference maximum (log2 units)
  float l, lq;    // the lane's share of the weights' sum, and of those multiplied with V
  float mgrow;    // a logit above it raises the reference
};

// The reference is raised only when a logit (lmt: the largest of the lane's) exceeds it by
// more than 2^8, so that weights stay <= 256.
__device__ __forceinline__ void q8_raise(Q8Rows& rt, float lmt) {
  if (__ballot(lmt > rt.mgrow) == 0ull) return;
  const float mt = pair_max(lmt);
  const bool grow = mt > rt.mgrow;
  const float alpha = grow ? __builtin_amdgcn_exp2f(rt.m - mt) : 1.0f;  // 0 from -inf
  rt.l *= alpha;
  rt.lq *= alpha;
#pragma unroll
  for (int dt = 0; dt < 4; ++dt) rt.o[dt] *= alpha;
  rt.m = grow ? mt : rt.m;
  rt.mgrow = rt.m + kRescaleSlack;
}

// Scores that a row does not see (bit k of word: key k of the tile) become -inf.
__device__ __forceinline__ void q8_mask(floatx16& s, uint32_t word) {
  const uint32_t w = word >> (4 * ((threadIdx.x & (kWave - 1)) >> 5));
#pragma unroll
  for (int r = 0; r < 16; ++r)
    s[r] = ((w >> (8 * (r >> 2) + (r & 3))) & 1u) ? s[r] : -__builtin_inff();
}

__device__ __forceinline__ float max3(float a, float b, float c) { return fmaxf(fmaxf(a, b), c); }
__device__ __forceinline__ float max16(const floatx16& s) {  // (eight instructions)
  const float a = max3(s[0], s[1], s[2]), b = max3(s[3], s[4], s[5]), c = max3(s[6], s[7], s[8]);
  const float d = max3(s[9], s[10], s[11]), e = max3(s[12], s[13], s[14]);
  return fmaxf(max3(a, b, s[15]), max3(c, d, e));
}

#define ECHO_FENCE() __builtin_amdgcn_sched_barrier(0)
// The softmax of NT tiles' scores and O^T += V^T P^T.  frag(g, dt): V^T of 16-key group g
// (2 per tile), dims 32 dt .., as four words of bfloat16.  c: softmax factor x K scale of
// a tile; lvs: log2 of its V scale, which the weights take along (the sums are taken
// without it).  The weights of a group are computed between the products of the group
// before (a 32x32x16 product leaves room for five vector instructions).
template <int NT, typename Frag>
__device__ __forceinline__ void q8_values(const Frag& frag, floatx16 (&s)[NT], Q8Rows& rt,
                                          const float (&c)[NT], const float (&lvs)[NT]) {
  float lmt = max16(s[0]) * c[0];
  if (NT == 2) lmt = fmaxf(lmt, max16(s[NT - 1]) * c[NT - 1]);
  q8_raise(rt, lmt);
  const float neg_m = rt.m == -__builtin_inff() ? 0.0f : -rt.m;
  float off[NT], sum[NT][2], used[NT][2];
#pragma unroll
  for (int j = 0; j < NT; ++j) {
    off[j] = lvs[j] + neg_m;
    sum[j][0] = sum[j][1] = used[j][0] = used[j][1] = 0.0f;
  }
  uint32_t pk[2][4];
  const auto two = [&](int g, int i) {  // weights 2 i and 2 i + 1 of the lane's 8 of group g
    const int j = g >> 1, e = 8 * (g & 1) + 2 * i;
    const float p0 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[j][e], c[j], off[j]));
    const float p1 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[j][e + 1], c[j], off[j]));
    sum[j][0] += p0;
    sum[j][1] += p1;
    pk[g & 1][i] = pack_bf16x2(p0, p1);
    used[j][i & 1] = add_bf16x2(pk[g & 1][i], used[j][i & 1]);
    // (added here, not at the end)
    asm volatile("" : "+v"(sum[j][0]), "+v"(sum[j][1]), "+v"(used[j][i & 1]));
  };
#pragma unroll
  for (int i = 0; i < 4; ++i) two(0, i);
#pragma unroll
  for (int g = 0; g < 2 * NT; ++g) {
    const bf16x8 pf = as_bf16x8(make_uint4(pk[g & 1][0], pk[g & 1][1], pk[g & 1][2], pk[g & 1][3]));
#pragma unroll
    for (int dt = 0; dt < 4; ++dt) {
      const bf16x8 f = as_bf16x8(frag(g, dt));
      ECHO_FENCE();
      rt.o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f, pf, rt.o[dt], 0, 0, 0);
      ECHO_FENCE();
      if (g + 1 < 2 * NT) two(g + 1, dt);
    }
  }
  ECHO_FENCE();
#pragma unroll
  for (int j = 0; j < NT; ++j) {
    const float ivs = __builtin_amdgcn_exp2f(-lvs[j]);
    rt.l = __builtin_fmaf(sum[j][0] + sum[j][1], ivs, rt.l);
    rt.lq = __builtin_fmaf(used[j][0] + used[j][1], ivs, rt.lq);
  }
}
// A row's 8 dims that the lane has in part n (of 8) of the product of Q and K: dims
// 64 (n / 4) + 32 (lane / 32) + 8 (n % 4) on, so that the lane's cached bytes of a key
// are two runs of 32.
__device__ __forceinline__ bf16x8 q8_dims(const uint16_t* row, int n) {
  const int h = (threadIdx.x & (kWave - 1)) >> 5;
  return as_bf16x8(*reinterpret_cast<const uint4*>(row + 64 * (n >> 2) + 32 * h + 8 * (n & 3)));
}

// A tile of the tree's new keys (tn <= 32 of them from slot s0 on).  V goes through 4 KB
// of LDS at `scratch` to be transposed, 16 keys at a time (the second 16 only if there
// are so many).
__device__ __forceinline__ void q8_tree_tile(const Q8Args& a, int head, int s0, int tn,
                                             uint32_t scratch, const bf16x8 (&q)[8], Q8Rows& rt,
                                             uint32_t word) {
  const int lane = threadIdx.x & (kWave - 1);
  const int h = lane >> 5, lr = lane & 15;
  const uint32_t row_bytes = uint32_t(a.hkv) * kD * 2;
  const uint64_t vh = uniform64(reinterpret_cast<uint64_t>(a.v_new) + uint64_t(uint32_t(s0)) * row_bytes +
                                uint32_t(head) * (kD * 2));
  const auto copy_v = [&](int g) {
    uint32_t o[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      // (LDS: 256-byte rows, 16-byte chunk c of row r at place c ^ swz_pattern(r))
      const int row = 4 * j + (lane >> 4);
      o[j] = uint32_t(min(16 * g + row, tn - 1)) * row_bytes + uint32_t((lr ^ swz_pattern(row)) << 4);
    }
    q8_copy4(scratch, vh, o);
  };
  copy_v(0);
  const uint16_t* kp = a.k_new + (size_t(s0 + min(lane & 31, tn - 1)) * a.hkv + head) * kD;
  floatx16 s[1] = {};
#pragma unroll
  for (int n = 0; n < 8; ++n)
    s[0] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(q8_dims(kp, n), q[n], s[0], 0, 0, 0);
  wait_vm<0>();
  asm volatile("" ::: "memory");
  // V^T of a 16-key group: keys 4 h + 0..3 and the same + 8 of dims 32 dt + lane % 32
  const int vrow = 4 * h + (lr >> 2);
  const uint32_t vt = scratch + uint32_t(vrow * 256 + ((lr & 1) << 3));
  const uint32_t chunk = uint32_t((2 * ((lane >> 4) & 1) + ((lr & 3) >> 1)) ^ swz_pattern(vrow));
  shortx4 v[2][4][2];
  const auto read_v = [&](int g) {
#pragma unroll
    for (int dt = 0; dt < 4; ++dt)
#pragma unroll
      for (int k = 0; k < 2; ++k)  // (8 rows on: bit 1 of the pattern)
        v[g][dt][k] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            (lds_shortx4_t*)(lds_at(vt + ((chunk ^ uint32_t(4 * dt) ^ uint32_t(2 * k)) << 4)) + 2048 * k));
    q8_wait_lds();
  };
  read_v(0);
  if (tn > 16) {  // uniform
    copy_v(1);
    wait_vm<0>();
    asm volatile("" ::: "memory");
    read_v(1);
  } else {
#pragma unroll
    for (int dt = 0; dt < 4; ++dt) v[1][dt][0] = v[1][dt][1] = shortx4{0, 0, 0, 0};
  }
  q8_mask(s[0], word);
  const float c[1] = {a.scale2}, lvs[1] = {0.0f};
  q8_values<1>(
      [&](int g, int dt) {
        return __builtin_bit_cast(uint4, __builtin_shufflevector(v[g][dt][0], v[g][dt][1], 0, 1, 2, 3,
                                                                 4, 5, 6, 7));
      },
      s, rt, c, lvs);
}

// A wave's steps [lo, hi) of one unit, then its output or partial sums.
//
// K is widened to bfloat16 between the products.  (v_mfma_f32_32x32x64_f8f6f4 would take its
// bytes as they are and Q as the sum of two e4m3 numbers, in as many cycles, but it drops
// what is below 2^-13 of the largest of its products.)
template <int kFmt, bool kGang>
__device__ __forceinline__ void q8_segment(const Q8Args& a, const Q8Ws& ws, const Q8Walk& w, int lo,
                                           int hi, int range_hi, int b, uint32_t ring, uint32_t scratch,
                                           Q8Table& tb, uint32_t offs, bool whole, int part_slot) {
  const int lane = threadIdx.x & (kWave - 1);
  const int h = lane >> 5;
  const int head = w.unit / w.q.passes;
  const int row0 = q8_row0(w, tb.k, tb.member);
  const int rows = min(kQ8Rows, w.q.nslots * a.G - row0);
  bf16x8 q[8];
  Q8Rows rt;
  int t = max(lo, min(hi, w.u0 + kQ8Enter));
  if (!kGang || rows > 0) {  // uniform
    // (a row past the last one computes the last one again, to be dropped)
    const int ra = row0 + min(lane & 31, rows - 1);
    const int slot = w.q.q0 + ra / a.G;
    const size_t row = size_t(slot) * a.hq + size_t(head) * a.G + ra % a.G;
#pragma unroll
    for (int n = 0; n < 8; ++n) q[n] = q8_dims(a.q + row * kD, n);
#pragma unroll
    for (int dt = 0; dt < 4; ++dt) rt.o[dt] = floatx16{};
    rt.m = -__builtin_inff();
    rt.l = 0.0f;
    rt.lq = 0.0f;
    rt.mgrow = -__builtin_inff();
    for (; t < hi && t - w.u0 < w.head(); ++t) {
      const int lt = t - w.u0 - kQ8Enter;
      const int tn = min(kTileKeys, w.q.nslots - lt * kTileKeys);
      uint32_t word = lt < a.W ? a.tree_mask[size_t(slot) * a.W + lt] : 0u;
      if (tn < kTileKeys) word &= (1u << tn) - 1u;
      q8_tree_tile(a, head, w.q.q0 + lt * kTileKeys, tn, scratch, q, rt, word);
    }
  }
  if (kGang) t = max(t, min(hi, w.u0 + w.head()));
  if (tb.raw) q8_scales(tb, a);  // uniform
  wait_vm<0>();  // no load that the compiler knows of is in flight in the loop

  for (; t < hi; ++t) {
    tb.done = __builtin_amdgcn_readfirstlane(tb.done);  // (uniform, which the compiler loses)
    tb.known = __builtin_amdgcn_readfirstlane(tb.known);
    const int i = (2 * tb.done) & (kWave - 1);
    uint32_t tiles = ring;
    if (kGang) {
      if (tb.more && tb.k_sent == tb.known) q8_refill<true>(tb, a, ws, w, t, range_hi, ring, offs);
      // the wave's quarter of the step has landed (up to two steps are behind it), and the others'
      const int behind = tb.k_sent - tb.done - 1;
      if (behind >= 2) wait_vm<8>();
      else if (behind == 1) wait_vm<4>();
      else wait_vm<0>();
      asm volatile("" ::: "memory");
      __builtin_amdgcn_s_barrier();
      asm volatile("" ::: "memory");
      tiles += uint32_t((tb.done & (kGangSlots - 1)) * 2 * kQ8Slot);
      if (rows <= 0) {
        q8_send_gang(tb, a, ring, offs);
        tb.done += 1;
        continue;
      }
    } else {
      // (the table is used up, and the ring empty)
      if (tb.done == tb.known) q8_refill<false>(tb, a, ws, w, t, range_hi, ring, offs);
      wait_vm<0>();
      asm volatile("" ::: "memory");  // the tiles' reads stay behind the wait
    }
    // K and V of the step to registers; then their places are refilled while they are multiplied
    uint4v kr[2][2][2];  // [tile][half of the dims][chunk]
    const uint32_t ka = tiles + k_offset(offs);
#pragma unroll
    for (int n = 0; n < 2; ++n)
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int e = 0; e < 2; ++e)
          kr[n][j][e] = *(lds_uint4_t*)(lds_at(ka ^ uint32_t(64 * j + 16 * e)) + kBlockBytes * n);
    intx2 vr[4][4];  // [16-key group][32 dims]
    const uint32_t va = tiles + kQ8Slot + v_offset(offs);
#pragma unroll
    for (int g = 0; g < 4; ++g)
#pragma unroll
      for (int dt = 0; dt < 4; ++dt)
        vr[g][dt] = __builtin_amdgcn_ds_read_tr8_b64_v2i32(
            (lds_intx2_t*)(lds_at(va ^ uint32_t(dt << 5)) + 16 * kD * g));
    q8_wait_lds();
    if (kGang) {
      // (into the last step's slot: the others have read it, or they had not come to the barrier)
      q8_send_gang(tb, a, ring, offs);
    } else {
      q8_send(tb, tb.k_sent, a.k_pages, ring, offs);
      q8_send(tb, tb.v_sent, a.v_pages, ring + kQ8Slot, offs);
    }
    tb.done += 1;
    floatx16 s[2] = {};
    const auto widen_k = [&](int x) {  // part x / 2 of tile x % 2
      const uint4v c = kr[x & 1][x >> 3][(x >> 2) & 1];
      const uint32_t lo = c[x & 2 ? 2 : 0], hi = c[x & 2 ? 3 : 1];
      return as_bf16x8(make_uint4(widen2<kFmt>(lo, false), widen2<kFmt>(lo, true),
                                  widen2<kFmt>(hi, false), widen2<kFmt>(hi, true)));
    };
    bf16x8 kf = widen_k(0);
#pragma unroll
    for (int x = 0; x < 16; ++x) {
      ECHO_FENCE();
      s[x & 1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, q[x >> 1], s[x & 1], 0, 0, 0);
      ECHO_FENCE();
      if (x < 15) kf = widen_k(x + 1);
    }
    ECHO_FENCE();
    const int tn1 = lane_of(tb.tokens, i + 1);
    if (tn1 < kTileKeys) {
      const int tn0 = lane_of(tb.tokens, i);
      q8_mask(s[0], tn0 < kTileKeys ? (1u << tn0) - 1u : 0xFFFFFFFFu);
      q8_mask(s[1], (1u << tn1) - 1u);
    }
    const float c[2] = {lane_of(tb.c, i), lane_of(tb.c, i + 1)};
    const float lvs[2] = {lane_of(tb.lvs, i), lane_of(tb.lvs, i + 1)};
    // Without priorities the older of a SIMD's two waves goes first in every phase, and the other
    // ends its range long after it (a long context: 239 us without, 229 with).
    __builtin_amdgcn_s_setprio(1);
    q8_values<2>(
        [&](int g, int dt) {
          const uint32_t x = uint32_t(vr[g][dt][0]), y = uint32_t(vr[g][dt][1]);
          return make_uint4(widen2<kFmt>(x, false), widen2<kFmt>(x, true), widen2<kFmt>(y, false),
                            widen2<kFmt>(y, true));
        },
        s, rt, c, lvs);
    __builtin_amdgcn_s_setprio(0);
  }

  if (kGang && rows <= 0) return;
  int rho = lane & 31;  // (opaque: the output's addresses are formed here, not kept in registers)
  asm volatile("" : "+v"(rho));
  const float L = pair_sum(rt.l);
  const float Lq = pair_sum(rt.lq);
  if (whole) {
    if (rho < rows) {
      const int ra = row0 + rho;
      const size_t orow = size_t(w.q.q0 + ra / a.G) * a.hq + size_t(head) * a.G + ra % a.G;
      const float inv = Lq > 0.0f ? 1.0f / Lq : 0.0f;
      uint16_t* po = a.out + orow * kD + 4 * h;
#pragma unroll
      for (int dt = 0; dt < 4; ++dt)
#pragma unroll
        for (int r = 0; r < 16; r += 4)
          *reinterpret_cast<uint2*>(po + 32 * dt + 2 * r) =
              make_uint2(pack_bf16x2(rt.o[dt][r] * inv, rt.o[dt][r + 1] * inv),
                         pack_bf16x2(rt.o[dt][r + 2] * inv, rt.o[dt][r + 3] * inv));
      if (a.lse != nullptr && h == 0)
        a.lse[orow] = L > 0.0f ? (rt.m + log2f(L)) * kLn2 : -__builtin_inff();
    }
  } else {
    if (rho < rows) {
      const size_t part = size_t(b) * 2 + part_slot;
      float* po = ws.part_o + (part * 16 * kQ8Rows + rho) * 8 + 4 * h;  // (a store: 1 KB in one piece)
#pragma unroll
      for (int dt = 0; dt < 4; ++dt)
#pragma unroll
        for (int r = 0; r < 16; r += 4)
          *reinterpret_cast<floatx4*>(po + (4 * dt + (r >> 2)) * kQ8Rows * 8) =
              floatx4{rt.o[dt][r], rt.o[dt][r + 1], rt.o[dt][r + 2], rt.o[dt][r + 3]};
      if (h == 0)
        *reinterpret_cast<floatx4*>(ws.part_ml + (part * kQ8Rows + rho) * 4) =
            floatx4{rt.m, L, Lq, 0.0f};
    }
  }
  asm volatile("");  // (the lanes meet here: what follows stays known to be uniform)
}

// A wave's range.
template <int kFmt, bool kGang>
__device__ __forceinline__ void q8_range(const Q8Args& a, const Q8Ws& ws, const Q8Range& st, Q8Walk& w,
                                         int b, uint32_t ring, uint32_t scratch) {
  const uint32_t offs = q8_lane_offsets(kGang ? 8 * st.member : 0);
  Q8Table tb = {};
  tb.k = st.k;
  tb.member = st.member;
  // the first steps' page ids in one round trip with those that the check takes
  const int lane = threadIdx.x & (kWave - 1);
  const Q8Pages pages(a, ws, w.q.r, w.q.P);
  int e[2] = {0, 0};
  if (pages.n > 0) {
    e[0] = pages.at(lane);
    e[1] = pages.at(kWave + lane);
  }
  Q8Next x;
  uint32_t page;
#pragma unroll 1
  for (bool checked = false;; checked = true) {
    x = q8_next_steps<kGang>(tb, a, ws, w, st.lo, st.hi);
    page = x.pos < x.n ? uint32_t(a.block_table[x.entry]) : 0u;
    if (checked) break;
    q8_check(w, a, pages, pages.n > 0 && (pages.bad_value(a, e[0]) || pages.bad_value(a, e[1])),
             2 * kWave);
    if (!w.bad) break;
  }
  q8_fill<kGang>(tb, a, x, page, ring, offs);
  const Q8Cut cut = q8_cut(w, st);
  if (lane == 0) ws.cuts[b] = cut;
  while (true) {
    const int lo = max(st.lo, w.u0), hi = min(st.hi, w.u0 + w.q.tpu);
    const bool whole = w.u0 >= st.lo && w.u0 + w.q.tpu <= st.hi;
    const int slot = w.u0 >= st.lo ? 1 : 0;
    if (kGang ? !w.bad : q8_has_rows(w, a, tb.k, tb.member))
      q8_segment<kFmt, kGang>(a, ws, w, lo, hi, st.hi, b, ring, scratch, tb, offs, whole, slot);
    if (hi >= st.hi) break;
    q8_next_unit(w, a, ws);
  }
}

template <int kFmt>
__global__ __launch_bounds__(kQ8Waves * kWave) __attribute__((amdgpu_waves_per_eu(2, 2))) void
q8_main_kernel(Q8Args a, Q8Ws ws) {
  __shared__ __attribute__((aligned(1024))) char smem[kQ8Waves * kQ8WaveLds];
  static_assert(4096 + 8 * (ECHO_MAX_REQUESTS + 1) <= sizeof(smem), "the requests fit");
  static_assert(kGangSlots * 2 * kQ8Slot + kQ8Waves * kQ8Scratch == sizeof(smem), "a gang's LDS");
  const int wid = wave_id();
  const int b = __builtin_amdgcn_readfirstlane(int(blockIdx.x) * kQ8Waves + wid);
  Q8Walk w = {};
  const Q8Range st = q8_begin(a, ws, reinterpret_cast<uint32_t*>(smem), w);
  if (st.lo >= st.hi) {
    if ((threadIdx.x & (kWave - 1)) == 0) ws.cuts[b] = Q8Cut{};
    return;
  }
  const uint32_t base = __builtin_amdgcn_readfirstlane(
      uint32_t(reinterpret_cast<uintptr_t>((lds_void_t*)smem)));
  if (st.k == kQ8Waves) {
    q8_range<kFmt, true>(a, ws, st, w, b, base,
                         base + uint32_t(kGangSlots * 2 * kQ8Slot + wid * kQ8Scratch));
  } else {
    const uint32_t ring = base + uint32_t(wid * kQ8WaveLds);  // (no barrier: independent waves)
    q8_range<kFmt, false>(a, ws, st, w, b, ring, ring + 2 * kQ8Slot);
  }
  if (w.met && (threadIdx.x & (kWave - 1)) == 0) status_or(a.status, ECHO_DATA_BAD_OFFSETS);
}

#undef ECHO_FENCE

// ------------------------------------------------------------- combine ----
constexpr int kQ8Parts = 8;  // partial sums per round trip

__device__ __forceinline__ Q8Cut load_cut(const Q8Cut* cuts, int b) {
  const_i32_t* p = (const_i32_t*)(cuts + b);
  int32_t w[12];
#pragma unroll
  for (int i = 0; i < 12; ++i) w[i] = p[i];
  return __builtin_bit_cast(Q8Cut, w);
}

// Workgroup (b, y): rows 16 y .. 16 y + 15 that wave b has of the unit that is cut first at its
// range (if any); a thread has 8 dims of a row.  Parts in the order of the gangs.  4 us for a
// few partial sums, 11 us for 2900 of them, 50 MB: latency and the launch, then their bytes (in
// fp16 they were half of these and the call 2-8% shorter; a sum below 2^-113 had no scale there).
__global__ __launch_bounds__(256) void q8_combine_kernel(Q8Args a, Q8Ws ws) {
  const int b = blockIdx.x;
  const Q8Cut st = load_cut(ws.cuts, b);
  if (st.parts == 0) return;
  const int rows = min(kQ8Rows, st.nslots * a.G - st.row0);
  const int rho = blockIdx.y * 16 + (threadIdx.x & 15);
  if (rho >= rows) return;
  const int piece = threadIdx.x / 16;  // dims 8 piece .. 8 piece + 7
  float M = -__builtin_inff(), L = 0.0f, Lq = 0.0f;
  float acc[8] = {};
  int at = st.at, slot = st.slot, half = 1;  // (the first part is the end of its wave's range)
  for (int i0 = 0; i0 < st.parts; i0 += kQ8Parts) {  // (a batch's loads in one round trip)
    floatx4 ml[kQ8Parts];
    floatx4 o[kQ8Parts][2];
#pragma unroll
    for (int j = 0; j < kQ8Parts; ++j) {
      ml[j] = floatx4{-__builtin_inff(), 0.0f, 0.0f, 0.0f};
      o[j][0] = o[j][1] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
      if (i0 + j < st.parts) {  // uniform
        const int wave = q8_first_wave(st.wg0 + at, a.wgs) + slot * st.k + st.member;
        const size_t part = size_t(wave) * 2 + half;
        ml[j] = *reinterpret_cast<const floatx4*>(ws.part_ml + (part * kQ8Rows + rho) * 4);
        const float* po = ws.part_o + ((part * 16 + piece) * kQ8Rows + rho) * 8;
        o[j][0] = *reinterpret_cast<const floatx4*>(po);
        o[j][1] = *reinterpret_cast<const floatx4*>(po + 4);
      }
      half = 0;
      at += 1;
      slot += at == st.nwg ? 1 : 0;
      at = at == st.nwg ? 0 : at;
    }
    float m = M;
#pragma unroll
    for (int j = 0; j < kQ8Parts; ++j)
      m = fmaxf(m, ml[j][0]);
    if (m == -__builtin_inff()) continue;
    const float alpha = __builtin_amdgcn_exp2f(M - m);  // 0 from -inf
    M = m;
    L *= alpha;
    Lq *= alpha;
#pragma unroll
    for (int k = 0; k < 8; ++k) acc[k] *= alpha;
#pragma unroll
    for (int j = 0; j < kQ8Parts; ++j) {
      const float wgt = __builtin_amdgcn_exp2f(ml[j][0] - m);  // 0 from -inf
      L = __builtin_fmaf(wgt, ml[j][1], L);
      Lq = __builtin_fmaf(wgt, ml[j][2], Lq);
#pragma unroll
      for (int k = 0; k < 8; ++k) acc[k] = __builtin_fmaf(wgt, o[j][k >> 2][k & 3], acc[k]);
    }
  }
  const int ra = st.row0 + rho;
  const size_t orow = size_t(st.q0 + ra / a.G) * a.hq + size_t(st.head) * a.G + ra % a.G;
  const float inv = Lq > 0.0f ? 1.0f / Lq : 0.0f;
  *reinterpret_cast<uint4*>(a.out + orow * kD + 8 * piece) =
      make_uint4(pack_bf16x2(acc[0] * inv, acc[1] * inv), pack_bf16x2(acc[2] * inv, acc[3] * inv),
                 pack_bf16x2(acc[4] * inv, acc[5] * inv), pack_bf16x2(acc[6] * inv, acc[7] * inv));
  if (a.lse != nullptr && piece == 0)
    a.lse[orow] = L > 0.0f ? (M + log2f(L)) * kLn2 : -__builtin_inff();
}

}  // namespace

// Records and partial sums for every wave of the device, whatever the batch: 70 MB.
size_t attn_q8_workspace_bytes(int32_t R, int32_t max_pages) {
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
  a.wgs = nw / kQ8Waves;
  a.chunks = q8_page_chunks(a.max_pages);
  if (a.chunks > 0)
    hipLaunchKernelGGL(q8_pages_kernel, dim3(unsigned(a.chunks), unsigned(a.R)), dim3(kPageChunk), 0,
                       stream, a, ws.bad);
  hipLaunchKernelGGL(x.cache.format == ECHO_KV_E4M3 ? q8_main_kernel<ECHO_KV_E4M3>
                                                    : q8_main_kernel<ECHO_KV_E5M2>,
                     dim3(unsigned(nw / kQ8Waves)), dim3(kQ8Waves * kWave), 0, stream, a, ws);
  const long long rows = (long long)a.max_rows * a.G;
  hipLaunchKernelGGL(q8_combine_kernel, dim3(unsigned(nw), unsigned((rows < kQ8Rows ? rows : kQ8Rows) + 15) / 16),
                     dim3(256), 0, stream, a, ws);
  return hipGetLastError() == hipSuccess ? ECHO_OK : ECHO_ERR_HIP;
}

}  // namespace echo
